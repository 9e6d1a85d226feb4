// A key/value cache of grouped heads held in 8 bits: rows in, one query over it, eviction by accumulated weight, rows out.
//
// A block is 64 rows of one (sequence, head); its values are code * 2^e with the smallest e, -60 <= e <= 60, for which the
// block's largest magnitude is at most 127 * 2^e.  A power of two costs half a bit of the codes on average against a
// free scale.  It buys: no division (x * 2^-e is exact, the only rounding is that to a code); values that are exact in
// bf16; and a block whose scale grows, because a row was appended or moved in, is moved to the new scale by one
// rounding, or by none where the scale stays, so that rows which move often do not wear out.
//
// Every kernel here may be set up while the launch ahead of it runs (programmatic dependent launch) and waits for it
// before the first access to memory, in every block (the attention's joining launch reads the row counts ahead of that).
#include "st3_common.cuh"

#include <cooperative_groups.h>
#include <cuda.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "st3_launch.cuh"

namespace {

constexpr int kBlockRows = 64;
constexpr int kMaxExp = 60;

__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ float exp2i(int e) { return __int_as_float((e + 127) << 23); }   // -126 <= e <= 127
// log2 of a scale; whatever a caller's array holds, the result stays in the range of scales
__device__ __forceinline__ int scale_exp(float s) {
  const int e = (int)((__float_as_uint(s) >> 23) & 0xffu) - 127;
  return min(max(e, -kMaxExp), kMaxExp);
}
// The smallest e in [-60, 60] with amax <= 127 * 2^e: 1.m * 2^x <= 127/64 * 2^(e + 6).
__device__ __forceinline__ int block_exp(float amax) {
  const unsigned b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 133 + ((b & 0x7fffffu) > 0x7e0000u);
  return min(max(e, -kMaxExp), kMaxExp);
}
// Conversions between codes and floats without the conversion instructions, of which an SM has 16 a clock (two of them an element
// bound the storing kernel at 22 of its 44 us for 24 000 rows of 8 heads).
// x / scale rounded half to even, in the low byte: adding 1.5 * 2^23 leaves no bits below one.
__device__ __forceinline__ unsigned code_bits(float x, float inv_scale) {
  return __float_as_uint(fminf(fmaxf(x * inv_scale, -127.f), 127.f) + 12582912.f);
}
__device__ __forceinline__ unsigned pack4(unsigned a, unsigned b, unsigned c, unsigned d) {   // the low bytes
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// Code i of a word whose codes' sign bits have been inverted: 2^23 + 128 + code, less 2^23 + 128.
__device__ __forceinline__ unsigned flip(unsigned w) { return w ^ 0x80808080u; }
__device__ __forceinline__ float code_value(unsigned flipped, int i) {
  return __uint_as_float(__byte_perm(flipped, 0x4b000000u, 0x7650 + i)) - 8388736.f;
}
// four codes times f, a power of two, rounded again
__device__ __forceinline__ unsigned rescale4(unsigned w, float f) {
  w = flip(w);
  return pack4(code_bits(code_value(w, 0), f), code_bits(code_value(w, 1), f), code_bits(code_value(w, 2), f), code_bits(code_value(w, 3), f));
}
__device__ __forceinline__ int clamp_rows(int n, int cap) { return min(max(n, 0), cap); }

struct CacheView {
  int8_t* code[2];       // k, v
  float* scale[2];
  int* ids;
  float* weights;
  int batch, heads, cap;
};

// ------------------------------------------------------------------------------------------------------------------
// Rows in.  One thread block per (64-row block that receives rows, head), for K and V together: a block's life is a chain of
// round trips (offsets, rows, codes), and what hides it is the bytes that the blocks of an SM have under way.
// ------------------------------------------------------------------------------------------------------------------
struct StoreParams {
  CacheView c;
  const void* src[2];
  long long token_stride[2], head_stride[2];
  const int* cu;
  const int* start;
  const int* pos;
  int* status;
  int total;
  int wide;            // rows of both tensors start on 32 bytes
};

constexpr int kStoreThreads = 256;

// 16 elements of a row as they come; `wide`: they start on 32 bytes
template <typename T>
struct Raw16 { uint4 w[sizeof(T)]; };
template <typename T>
__device__ __forceinline__ Raw16<T> load16(const T* p, bool wide) {
  Raw16<T> r;
  const uint4* q = reinterpret_cast<const uint4*>(p);
#pragma unroll
  for (int i = 0; i < (int)sizeof(T); i += 2) {
    if (wide) {
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(r.w[i].x), "=r"(r.w[i].y), "=r"(r.w[i].z), "=r"(r.w[i].w), "=r"(r.w[i + 1].x), "=r"(r.w[i + 1].y),
                     "=r"(r.w[i + 1].z), "=r"(r.w[i + 1].w)
                   : "l"(q + i));
    } else {
      r.w[i] = q[i];
      r.w[i + 1] = q[i + 1];
    }
  }
  return r;
}
// eight of them as floats
template <typename T>
__device__ __forceinline__ void values8(const Raw16<T>& r, int half, float (&f)[8]) {
  if constexpr (sizeof(T) == 2) {
    unpack16(r.w[half], f);
  } else {
    const uint4 a = r.w[2 * half], b = r.w[2 * half + 1];
    const unsigned u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(u[i]);
  }
}
// the largest magnitude; NaN if one of them is
template <typename T>
__device__ __forceinline__ float top16(const Raw16<T>& r) {
  if constexpr (sizeof(T) == 2) {
    unsigned m = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const unsigned u[4] = {r.w[h].x, r.w[h].y, r.w[h].z, r.w[h].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(u[i] & 0x7fff7fffu));
    }
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  } else {
    float m = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float f[8];
      values8(r, h, f);
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max_nan(m, fabsf(f[i]));
    }
    return m;
  }
}
__device__ __forceinline__ float finite_or_0(float x) { return fabsf(x) <= 3.4028235e38f ? x : 0.f; }

// Whether rows c0 .. c1-1 of the tensors can become rows start and on of a sequence.
__device__ __forceinline__ bool store_ok(const StoreParams& p, int c0, int c1, int start) {
  return c0 >= 0 && c1 >= c0 && c1 <= p.total && start >= 0 && start <= p.c.cap - (c1 - c0);
}

// The sequences' pieces are numbered so that no table is needed: sequence s has the numbers cu[s]/64 + 2 s and on, which are
// at least as many as the blocks that its rows touch wherever they start (n/64 + 2).
template <typename T, int D>
__global__ void __launch_bounds__(kStoreThreads) st3_cache_store_kernel(const StoreParams p) {
  constexpr int kLanes = D / 16, kPass = kStoreThreads / kLanes, kIter = kBlockRows / kPass;
  __shared__ float s_max[2][kStoreThreads / 32];
  __shared__ int s_seq, s_of[4];
  pdl_wait();
  pdl_next();
  const int tid = threadIdx.x, slot = blockIdx.x, head = blockIdx.y;
  // The sequence whose numbers hold `slot`, with its offsets: one round trip for all sequences.
  if (tid == 0) s_seq = -1;
  __syncthreads();
  int found = -1, c0 = 0, c1 = 0, start = 0, pos = 0;
  for (int b = tid; b < p.c.batch; b += kStoreThreads) {
    const int from = p.cu[b], to = p.cu[b + 1], st = p.start ? p.start[b] : 0, ps = p.pos ? p.pos[b] : st;
    // the first block reports for all sequences: one that ends ahead of its start may have no number
    if (slot == 0 && head == 0 && from != to && !store_ok(p, from, to, st) && p.status) atomicOr(p.status, ST3_DEV_RANGE);
    if (from / kBlockRows + 2 * b <= slot && (b + 1 == p.c.batch || to / kBlockRows + 2 * (b + 1) > slot)) {
      found = b; c0 = from; c1 = to; start = st; pos = ps;
    }
  }
  if (found >= 0) atomicMax(&s_seq, found);   // one, unless the offsets are not ascending
  __syncthreads();
  const int b = s_seq;
  if (b < 0) return;
  if (b == found) { s_of[0] = c0; s_of[1] = c1; s_of[2] = start; s_of[3] = pos; }
  __syncthreads();
  c0 = s_of[0]; c1 = s_of[1]; start = s_of[2]; pos = s_of[3];
  const int n = c1 - c0;
  if (n == 0 || !store_ok(p, c0, c1, start)) return;
  const int place = slot - (c0 / kBlockRows + 2 * b);
  if (place < 0) return;
  const int blk = start / kBlockRows + place;
  const int row0 = blk * kBlockRows;
  if (row0 >= start + n) return;
  const int lo = max(start - row0, 0), hi = min(start + n - row0, kBlockRows);   // new rows of this block
  const size_t bh = (size_t)b * p.c.heads + head;
  const int col = (tid % kLanes) * 16, r0 = tid / kLanes;
  Raw16<T> raw[2][kIter];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const T* src = static_cast<const T*>(p.src[side]) + (long long)(c0 + row0 - start) * p.token_stride[side] +
                   (long long)head * p.head_stride[side] + col;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      const int r = r0 + i * kPass;
      if (r >= lo && r < hi) raw[side][i] = load16(src + (long long)r * p.token_stride[side], p.wide);
    }
  }
  float was[2];   // read ahead of the barrier, written after it
#pragma unroll
  for (int side = 0; side < 2; ++side) was[side] = lo > 0 ? p.c.scale[side][bh * (p.c.cap / kBlockRows) + blk] : 0.f;
  float amax[2] = {0.f, 0.f};
#pragma unroll
  for (int side = 0; side < 2; ++side)
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      const int r = r0 + i * kPass;
      if (r >= lo && r < hi) amax[side] = max_nan(amax[side], top16(raw[side][i]));
    }
  // What is not finite counts as 0: rare, so that only blocks that hold some look at every element for it.
  const bool bad = __syncthreads_or(!(amax[0] <= 3.4028235e38f && amax[1] <= 3.4028235e38f));
  if (bad) {
    if (tid == 0 && p.status) atomicOr(p.status, ST3_DEV_NONFINITE);
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      amax[side] = 0.f;
#pragma unroll
      for (int i = 0; i < kIter; ++i) {
        const int r = r0 + i * kPass;
        if (r < lo || r >= hi) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float f[8];
          values8(raw[side][i], h, f);
#pragma unroll
          for (int e = 0; e < 8; ++e) amax[side] = fmaxf(amax[side], fabsf(finite_or_0(f[e])));
        }
      }
    }
  }
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    amax[side] = warp_max(amax[side]);
    if ((tid & 31) == 0) s_max[side][tid >> 5] = amax[side];
  }
  __syncthreads();
#pragma unroll
  for (int side = 0; side < 2; ++side) {
#pragma unroll
    for (int i = 0; i < kStoreThreads / 32; ++i) amax[side] = fmaxf(amax[side], s_max[side][i]);
    int e = block_exp(amax[side]);
    const int e_was = scale_exp(was[side]);
    if (lo > 0) e = max(e, e_was);
    const float inv = exp2i(-e);
    int8_t* codes = p.c.code[side] + (bh * p.c.cap + row0) * D;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      const int r = r0 + i * kPass;
      uint4* at = reinterpret_cast<uint4*>(codes + r * D + col);
      if (r >= lo && r < hi) {
        unsigned w[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float f[8];
          values8(raw[side][i], h, f);
          if (bad) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = finite_or_0(f[j]);
          }
          unsigned c[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) c[j] = code_bits(f[j], inv);
          w[2 * h] = pack4(c[0], c[1], c[2], c[3]);
          w[2 * h + 1] = pack4(c[4], c[5], c[6], c[7]);
        }
        *at = make_uint4(w[0], w[1], w[2], w[3]);
      } else if (r < lo && e > e_was) {
        const uint4 w = *at;
        const float f = exp2i(max(e_was - e, -126));
        *at = make_uint4(rescale4(w.x, f), rescale4(w.y, f), rescale4(w.z, f), rescale4(w.w, f));
      }
    }
    if (tid == 0) p.c.scale[side][bh * (p.c.cap / kBlockRows) + blk] = exp2i(e);
  }
  if (tid >= lo && tid < hi) {
    const size_t at = bh * p.c.cap + row0 + tid;
    p.c.ids[at] = pos + row0 + tid - start;
    p.c.weights[at] = 0.f;
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Rows out
// ------------------------------------------------------------------------------------------------------------------
struct RowsParams {
  CacheView c;
  void* dst[2];
  int* ids;
  float* weights;
  const int* first;
  const int* held;
  int num_rows;
  int wide;            // the values' rows start on 32 bytes
};

constexpr int kRowsThreads = 256;

// A thread reads 16 codes of a row and writes 16 values; K and V are two halves of the grid's last dimension.  (Two or four rows a
// thread, or 8 codes, were slower by 10-15 %.)
template <typename T, int D>
__global__ void __launch_bounds__(kRowsThreads) st3_cache_rows_kernel(const RowsParams p) {
  constexpr int kLanes = D / 16, kPer = kRowsThreads / kLanes;
  pdl_wait();
  pdl_next();
  const int side = blockIdx.z & 1, h = blockIdx.y, b = blockIdx.z >> 1, tid = threadIdx.x;
  const int i0 = blockIdx.x * kPer, i = i0 + tid / kLanes;
  const int held = clamp_rows(p.held[b], p.c.cap);
  const long long first = p.first ? p.first[b] : 0, r = first + i;
  const size_t bh = (size_t)b * p.c.heads + h;
  // selected, not indexed: an index would put the parameters into local memory
  T* dst = static_cast<T*>(side ? p.dst[1] : p.dst[0]);
  const int8_t* codes = side ? p.c.code[1] : p.c.code[0];
  const float* scales = side ? p.c.scale[1] : p.c.scale[0];
  if (i < p.num_rows && dst) {
    const int col = (tid % kLanes) * 16;
    uint4 w = make_uint4(0, 0, 0, 0);
    float s = 0.f;
    if (r >= 0 && r < held) {
      w = *reinterpret_cast<const uint4*>(codes + (bh * p.c.cap + r) * D + col);
      s = scales[bh * (p.c.cap / kBlockRows) + r / kBlockRows];
    }
    const unsigned in[4] = {flip(w.x), flip(w.y), flip(w.z), flip(w.w)};
    float f[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) f[e] = code_value(in[e >> 2], e & 3) * s;
    T* out = dst + (bh * p.num_rows + i) * D + col;
    if constexpr (sizeof(T) == 2) {
      unsigned o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const __nv_bfloat162 v2 = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
        o[e] = *reinterpret_cast<const unsigned*>(&v2);
      }
      if (p.wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]),
                     "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7])
                     : "memory");
      } else {
        reinterpret_cast<uint4*>(out)[0] = make_uint4(o[0], o[1], o[2], o[3]);
        reinterpret_cast<uint4*>(out)[1] = make_uint4(o[4], o[5], o[6], o[7]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) reinterpret_cast<float4*>(out)[e] = make_float4(f[4 * e], f[4 * e + 1], f[4 * e + 2], f[4 * e + 3]);
    }
  }
  if (side == 0 && tid < kPer && i0 + tid < p.num_rows) {   // ids and weights: the K half
    const long long r2 = first + i0 + tid;
    const bool live = r2 >= 0 && r2 < held;
    const size_t at = bh * p.num_rows + i0 + tid;
    if (p.ids) p.ids[at] = live ? p.c.ids[bh * p.c.cap + r2] : 0;
    if (p.weights) p.weights[at] = live ? p.c.weights[bh * p.c.cap + r2] : 0.f;
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Eviction: a thread block per (sequence, head) decides, then one per block of rows moves.
// ------------------------------------------------------------------------------------------------------------------
struct EvictParams {
  CacheView from, to;
  const int* held;
  const int* seen;
  int* held_out;
  int* status;
  int* src;            // [bh][cap_src] row that each row below the new length comes from
  int* movers;         // [bh][cap]     kept rows from behind the new length, in order; for clusters and heads that are not staged
  unsigned* words;     // [bh][cap/32]  bits of the rows that stay, for heads that are not staged
  int2* before;        // [bh][cap/32]  holes and movers ahead of a word's rows, likewise
  int* changed;        // [bh][cap/64]  blocks that receive rows
  int* length;         // [bh]          rows that stay
  float* edge;         // [bh][2]       scales of the block that the new length cuts
  int keep, recent, in_place;
};

constexpr int kEvictThreads = 512;
constexpr int kBins = 2048;

// Weights as unsigned keys of the same order; -0 is 0, NaN the lowest, a recent row the highest.
__device__ __forceinline__ unsigned weight_key(float w, bool recent) {
  if (recent) return 0xffffffffu;
  if (w != w) return 0u;
  const unsigned b = __float_as_uint(w + 0.f);
  return min((b & 0x80000000u) ? ~b : b | 0x80000000u, 0xfffffffeu);
}

__device__ __forceinline__ int warp_sum_upto(int v) {   // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += y;
  }
  return v;
}
__device__ __forceinline__ int block_sum_below(int x, int* s_warp, int& total) {   // exclusive sum over the block
  static_assert(kEvictThreads <= 1024, "a lane for each warp's sum");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int v = warp_sum_upto(x);
  __syncthreads();
  if (lane == 31) s_warp[warp] = v;
  __syncthreads();
  const int sums = warp_sum_upto(lane < kEvictThreads / 32 ? s_warp[lane] : 0);
  total = __shfl_sync(0xffffffffu, sums, 31);
  const int before = warp ? __shfl_sync(0xffffffffu, sums, warp - 1) : 0;
  return before + v - x;
}

// In a histogram: the bin that holds the want-th element from the top (1-based), its place in the bin and how many it shares
// that with.  All threads return the same.
struct Pick { unsigned bin; int want; int in_bin; };

__device__ __forceinline__ Pick pick_bin(const int* s_hist, int want, int* s_warp, int* s_out) {
  constexpr int per = kBins / kEvictThreads;   // thread t sums the bins from t * per on, counted from the top
  int mine = 0;
  for (int j = 0; j < per; ++j) mine += s_hist[kBins - 1 - (threadIdx.x * per + j)];
  int total;
  int above = block_sum_below(mine, s_warp, total);
  if (above < want && want <= above + mine) {
    for (int j = 0; j < per; ++j) {
      const int bin = kBins - 1 - (threadIdx.x * per + j), c = s_hist[bin];
      if (want <= above + c) { s_out[0] = bin; s_out[1] = want - above; s_out[2] = c; break; }
      above += c;
    }
  }
  __syncthreads();
  Pick r;
  r.bin = (unsigned)s_out[0]; r.want = s_out[1]; r.in_bin = s_out[2];
  __syncthreads();
  return r;
}

constexpr int kEvictStage = 8192;    // rows whose weight and position a block keeps in shared memory
constexpr int kEvictDirect = 512;    // rows at the cut that are ranked one against the other
constexpr int kEvictSmem = kEvictStage * 8;
constexpr int kEvictBatch = 8;       // rows of a thread under way at once
constexpr int kEvictAhead = 4;
constexpr int kEvictRanged = 1536;   // rows from which on the first histogram covers their weights' range
constexpr int kEvictRanks = 8;       // blocks of a cluster

// Finds the last row that stays by histograms of the rows' composites (the weight's key, then the earlier position): the first one
// over their leading 11 bits or, where there are many rows, over the range of the weights, as weights of a few octaves crowd into a
// few bins of their leading bits (the whole eviction of 64 heads with 3 043 uniform weights: 28.6 -> 18.5 us; under some 1 500
// rows the pass that finds the range costs more); each further one over the range of what the cut's bin holds, until these are few
// enough to be ranked one against the other.
// The rows that stay become bits, a word for 32 rows: those above the cut's bin when its rows are collected, the others once they
// have been ranked.  One sum over the words numbers the holes and the rows that fill them.
// What bounds it: the round trips and barriers of one block, some 11 us at 1 040 rows of 256 heads, ahead of the moves.
//   kCluster: the blocks of a cluster share a head that is longer than one of them stages, a run of rows each, and add up their
// histograms through each other's shared memory.  Beyond what eight stage the rows come from L2 in every pass.
template <bool kCluster>
__global__ void __launch_bounds__(kEvictThreads, 2) st3_cache_select_kernel(const EvictParams p) {
  extern __shared__ __align__(16) unsigned char dyn[];
  unsigned* s_key = reinterpret_cast<unsigned*>(dyn);
  int* s_id = reinterpret_cast<int*>(dyn) + kEvictStage;
  __shared__ int s_hist[kBins];
  __shared__ int s_sums[kCluster ? kBins : 1];          // of all blocks' histograms
  __shared__ u64 s_at_cut[kEvictDirect];
  __shared__ u64 s_all_at_cut[kCluster ? kEvictDirect : 1];
  __shared__ int s_row[kEvictDirect];
  __shared__ unsigned s_word[kEvictStage / 32];
  __shared__ int2 s_before[kEvictStage / 32];
  __shared__ int s_warp[kEvictThreads / 32];
  __shared__ int s_out[3];
  __shared__ unsigned s_range[4];
  __shared__ int s_count[3];        // rows at the cut; holes; movers
  const cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
  const int ranks = kCluster ? (int)cluster.num_blocks() : 1, rank = kCluster ? (int)cluster.block_rank() : 0;
  auto sync = [&] { if (kCluster) cluster.sync(); else __syncthreads(); };
  auto of = [&](auto* mine, int r) { return kCluster ? cluster.map_shared_rank(mine, r) : mine; };
  pdl_wait();
  pdl_next();
  const int tid = threadIdx.x, lane = tid & 31, bh = blockIdx.x / ranks, b = bh / p.from.heads;
  const float* w = p.from.weights + (size_t)bh * p.from.cap;
  const int* ids = p.from.ids + (size_t)bh * p.from.cap;
  // without a cluster the first rows travel with the count of them; what lies behind the count is not used
  float w_ahead[kEvictAhead];
  int id_ahead[kEvictAhead];
  if (!kCluster)
#pragma unroll
    for (int j = 0; j < kEvictAhead; ++j) {
      const int i = tid + j * kEvictThreads;
      w_ahead[j] = i < p.from.cap ? w[i] : 0.f;
      id_ahead[j] = i < p.from.cap ? ids[i] : 0;
    }
  const int raw = p.held[b];
  const int border = p.seen[b] - p.recent;   // the first position that counts as recent
  const int n = clamp_rows(raw, p.from.cap), k = min(n, p.keep);
  const int blocks = p.from.cap / kBlockRows;
  if (tid == 0 && rank == 0) {
    p.length[bh] = k;
    if (raw != n && p.status) atomicOr(p.status, ST3_DEV_RANGE);
  }
  // this block's rows: [first, end)
  const int run = ((n + kBlockRows - 1) / kBlockRows + ranks - 1) / ranks * kBlockRows, first = min(n, rank * run), end = min(n, first + run);
  for (int i = tid + rank * kEvictThreads; i < blocks; i += ranks * kEvictThreads) p.changed[(size_t)bh * blocks + i] = 0;
  int* src = p.src + (size_t)bh * p.from.cap;
  if (n <= p.keep) {   // no row comes from behind the new length: no scale is kept
    for (int i = tid + rank * kEvictThreads; i < k; i += ranks * kEvictThreads) src[i] = i;
    return;
  }
  const bool staged = run <= kEvictStage;
  if (tid < 4) s_range[tid] = 0xffffffffu;
  if (tid == 0) s_count[0] = 0;
  for (int i = tid; i < kBins; i += kEvictThreads) s_hist[i] = 0;
  __syncthreads();
  // f(row, whether there is one, weight, position) for this block's rows from `from` on, a warp's 32 rows together
  auto each_loaded = [&](int from, auto&& f) {
    for (int i0 = from + tid; i0 - lane < end; i0 += kEvictBatch * kEvictThreads) {
      float wi[kEvictBatch];
      int id[kEvictBatch];
#pragma unroll
      for (int j = 0; j < kEvictBatch; ++j) {
        const int i = i0 + j * kEvictThreads;
        wi[j] = i < end ? w[i] : 0.f;
        id[j] = i < end ? ids[i] : 0;
      }
#pragma unroll
      for (int j = 0; j < kEvictBatch; ++j) {
        const int i = i0 + j * kEvictThreads;
        if (i - lane < end) f(i, i < end, wi[j], id[j]);
      }
    }
  };
  bool nan = false;
  // the same with keys, from shared memory where they are staged
  auto each_row = [&](auto&& f) {
    if (staged)
      for (int i = first + tid; i - lane < end; i += kEvictThreads) {
        const bool live = i < end;
        f(i, live, live ? s_key[i - first] : 0u, live ? s_id[i - first] : 0);
      }
    else
      each_loaded(first, [&](int i, bool live, float wi, int id) {
        nan |= live && wi != wi;
        f(i, live, weight_key(wi, id >= border), id);
      });
  };
  // composite order of a row: its key, then the earlier position
  auto place = [](int id) { return ~((unsigned)id ^ 0x80000000u); };
  auto composite = [&](unsigned key, int id) { return ((u64)key << 32) | place(id); };
  // The range of keys and of places, each as lowest and inverted highest, over all blocks.
  auto range = [&](unsigned (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = __reduce_min_sync(0xffffffffu, x[e]);
      if (lane == 0) atomicMin(&s_range[e], x[e]);
    }
    sync();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = s_range[e];
      if (kCluster)
        for (int r = 0; r < ranks; ++r) x[e] = min(x[e], of(s_range, r)[e]);
    }
  };
  // the cut lies in [lo, lo + width]: all rows, then those of a bin
  u64 lo = 0, width = ~0ull;
  int shift = 53, want = k, in_bin;
  const bool ranged = staged && n > kEvictRanged;
  if (staged) {
    unsigned x[4] = {0xffffffffu, 0xffffffffu, 0u, 0u};
    auto take = [&](int i, bool live, float wi, int id) {
      if (!live) return;
      nan |= wi != wi;
      const unsigned key = weight_key(wi, id >= border);
      s_key[i - first] = key;
      s_id[i - first] = id;
      if (!ranged) atomicAdd(&s_hist[key >> 21], 1);
      else if (key != 0xffffffffu) { x[0] = min(x[0], key); x[1] = min(x[1], ~key); }
    };
    if (!kCluster)
#pragma unroll
      for (int j = 0; j < kEvictAhead; ++j) take(tid + j * kEvictThreads, tid + j * kEvictThreads < n, w_ahead[j], id_ahead[j]);
    each_loaded(kCluster ? first : kEvictAhead * kEvictThreads, take);
    if (ranged) {
      range(x);
      if (x[0] <= ~x[1]) {   // else every row is a recent one
        // no weight is in the bin of the recent rows, be it the last one or one ahead of it
        shift = 32;
        while ((~x[1] - x[0]) >> (shift - 32) > kBins - 2) ++shift;
        lo = (u64)x[0] << 32;
      }
    }
  }
  for (int pass = 0;; ++pass) {
    if (pass > 0 || !staged || ranged)
      each_row([&](int, bool live, unsigned key, int id) {
        const u64 at = composite(key, id) - lo;
        if (live && at <= width) atomicAdd(&s_hist[min((unsigned)(at >> shift), (unsigned)kBins - 1)], 1);
      });
    if (__syncthreads_or(nan) && tid == 0 && p.status) atomicOr(p.status, ST3_DEV_NONFINITE);
    int* hist = s_hist;
    if (kCluster) {
      sync();
      for (int i = tid; i < kBins; i += kEvictThreads) {
        int all = 0;
        for (int r = 0; r < ranks; ++r) all += of(s_hist, r)[i];
        s_sums[i] = all;
      }
      hist = s_sums;
      __syncthreads();
    }
    const Pick cut = pick_bin(hist, want, s_warp, s_out);
    want = cut.want;
    in_bin = cut.in_bin;
    if (pass == 0 && ranged && cut.bin == kBins - 1) {   // among the recent rows
      lo = 0xffffffffull << 32;
      shift = 32;
      width = 0xffffffffull;
    } else {   // the last bin ends where the range does: rows behind it have been counted
      const u64 skipped = (u64)cut.bin << shift, rest = width - skipped, all = (1ull << shift) - 1;
      lo += skipped;
      width = rest < all ? rest : all;
    }
    if (in_bin <= kEvictDirect || shift == 0) break;
    // The next histogram covers what the bin holds: weights, or where they are equal places.
    if (tid < 4) s_range[tid] = 0xffffffffu;
    sync();   // the histograms have been read
    for (int i = tid; i < kBins; i += kEvictThreads) s_hist[i] = 0;
    unsigned x[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
    each_row([&](int, bool live, unsigned key, int id) {
      if (live && composite(key, id) - lo <= width) {
        x[0] = min(x[0], key); x[1] = min(x[1], ~key);
        x[2] = min(x[2], place(id)); x[3] = min(x[3], ~place(id));
      }
    });
    range(x);
    if (x[0] == ~x[1]) { lo = ((u64)x[0] << 32) | x[2]; width = ~x[3] - x[2]; }
    else { lo = (u64)x[0] << 32; width = ((u64)(~x[1] - x[0]) << 32) | 0xffffffffull; }
    shift = 0;
    while (width >> shift > kBins - 1) ++shift;
  }
  const bool rank_them = in_bin <= kEvictDirect;   // else they have one weight and one position, and stay
  unsigned* word = staged ? s_word : p.words + ((size_t)bh * p.from.cap + first) / 32;
  each_row([&](int i, bool live, unsigned key, int id) {
    const u64 c = composite(key, id);
    const bool inside = live && c - lo <= width;
    const unsigned stay = __ballot_sync(0xffffffffu, live && c >= lo && (!inside || !rank_them)), who = __ballot_sync(0xffffffffu, inside);
    if (lane == 0) word[(i - first) / 32] = stay;
    if (who && rank_them) {
      int at = 0;
      if (lane == 0) at = atomicAdd(&s_count[0], __popc(who));
      at = __shfl_sync(0xffffffffu, at, 0) + __popc(who & ((1u << lane) - 1));
      if (inside && at < kEvictDirect) { s_at_cut[at] = c; s_row[at] = i - first; }   // at < in_bin, if nobody writes the weights meanwhile
    }
  });
  sync();
  if (rank_them) {
    const int mine = min(s_count[0], kEvictDirect);
    const u64* all = s_at_cut;
    if (kCluster) {
      int at = 0;
      for (int r = 0; r < ranks; ++r) {
        const int theirs = min(of(s_count, r)[0], kEvictDirect - at);
        if (tid < theirs) s_all_at_cut[at + tid] = of(s_at_cut, r)[tid];
        at += theirs;
      }
      all = s_all_at_cut;
      __syncthreads();
    }
    // four lanes to a row, each against every fourth row
    for (int c0 = 0; c0 < mine; c0 += kEvictThreads / 4) {
      const int c = c0 + (tid >> 2);
      int above = 0;
      if (c < mine) {
        const u64 me = s_at_cut[c];
#pragma unroll 4
        for (int i = tid & 3; i < in_bin; i += 4) above += all[i] > me;
      }
      above += __shfl_xor_sync(0xffffffffu, above, 1);
      above += __shfl_xor_sync(0xffffffffu, above, 2);
      // rows of the same weight and position are equal, and stay or go together
      if (c < mine && above < want && (tid & 3) == 0) atomicOr(&word[s_row[c] / 32], 1u << (s_row[c] & 31));
    }
  }
  __syncthreads();   // the keys have been read for the last time, too: the rows that move take their place
  // thread t numbers the holes and the rows that fill them in its words from t * per on
  unsigned holes = 0, movers = 0;
  auto split = [&](int at, unsigned& hole, unsigned& mover) {   // rows below k that go, rows from k on that stay
    const int below = k - first - at * 32;
    const unsigned mask = below >= 32 ? 0xffffffffu : below <= 0 ? 0u : (1u << below) - 1;
    hole = ~word[at] & mask;
    mover = word[at] & ~mask;
  };
  int2* before = staged ? s_before : p.before + ((size_t)bh * p.from.cap + first) / 32;
  const int words = (end - first + 31) / 32, per = (words + kEvictThreads - 1) / kEvictThreads;
  int below = 0, behind = 0, moved;
  for (int at = tid * per; at < min(words, (tid + 1) * per); ++at) {
    split(at, holes, movers);
    below += __popc(holes);
    behind += __popc(movers);
    if (holes) p.changed[(size_t)bh * blocks + (first + at * 32) / kBlockRows] = 1;
  }
  if (staged) {   // both in one sum
    const int sums = block_sum_below(below | (behind << 16), s_warp, moved);
    if (kCluster && tid == 0) { s_count[1] = moved & 0xffff; s_count[2] = moved >> 16; }
    below = sums & 0xffff; behind = sums >> 16; moved >>= 16;
  } else {
    below = block_sum_below(below, s_warp, moved);
    if (kCluster && tid == 0) s_count[1] = moved;
    behind = block_sum_below(behind, s_warp, moved);
    if (kCluster && tid == 0) s_count[2] = moved;
  }
  if (kCluster) {   // those of the blocks ahead
    sync();
    moved = 0;
    for (int r = 0; r < ranks; ++r) {
      const int2 theirs = make_int2(of(s_count, r)[1], of(s_count, r)[2]);
      if (r < rank) { below += theirs.x; behind += theirs.y; }
      moved += theirs.y;
    }
  }
  for (int at = tid * per; at < min(words, (tid + 1) * per); ++at) {
    split(at, holes, movers);
    before[at] = make_int2(below, behind);
    below += __popc(holes);
    behind += __popc(movers);
  }
  __syncthreads();
  int* mover = staged && !kCluster ? reinterpret_cast<int*>(s_key) : p.movers + (size_t)bh * p.from.cap;
  for (int i = max(first, k / 32 * 32) + tid; i < end; i += kEvictThreads) {
    split((i - first) / 32, holes, movers);
    if (movers >> (i & 31) & 1) mover[before[(i - first) / 32].y + __popc(movers & ((1u << (i & 31)) - 1))] = i;
  }
  sync();   // and the others' shared memory has been read
  for (int i = first + tid; i < min(k, end); i += kEvictThreads) {
    split((i - first) / 32, holes, movers);
    const int at = before[(i - first) / 32].x + __popc(holes & ((1u << (i & 31)) - 1));
    // positions that are not distinct could leave a hole without a row for it; it then keeps its own
    src[i] = (holes >> (i & 31) & 1) && at < moved ? (kCluster ? __ldcg(mover + at) : mover[at]) : i;
  }
  // k < n <= capacity
  if (tid < 2 && rank == 0) p.edge[2 * bh + tid] = p.from.scale[tid][(size_t)bh * blocks + k / kBlockRows];
}

constexpr int kMoveThreads = 128;

template <int D>
__global__ void __launch_bounds__(kMoveThreads) st3_cache_move_kernel(const EvictParams p) {
  constexpr int kLanes = D / 16, kIter = kBlockRows * kLanes / kMoveThreads;   // 16-byte pieces of a row; pieces a thread
  static_assert(kBlockRows * (64 / 16) % kMoveThreads == 0, "pieces");
  __shared__ int s_src[kBlockRows];
  __shared__ float s_scale[2][kBlockRows];
  __shared__ float s_max[2][kMoveThreads / 32];
  pdl_wait();
  pdl_next();
  const int tid = threadIdx.x, bh = blockIdx.y, blk = blockIdx.x;
  const int from_blocks = p.from.cap / kBlockRows, row0 = blk * kBlockRows;
  // one round trip for all three; what `mine` holds behind the new length is not used
  const int k = p.length[bh];
  const bool changed = p.changed[(size_t)bh * from_blocks + blk];
  const int mine = tid < kBlockRows ? p.src[(size_t)bh * p.from.cap + row0 + tid] : 0;
  if (blk == 0 && bh % p.from.heads == 0 && tid == 0) p.held_out[bh / p.from.heads] = k;
  if (row0 >= k) return;
  if (p.in_place && !changed) return;
  const int rows = min(k - row0, kBlockRows);
  if (tid < kBlockRows) s_src[tid] = tid < rows ? mine : 0;
  __syncthreads();
  uint4 piece[2][kIter];
  float amax[2] = {0.f, 0.f};
#pragma unroll
  for (int side = 0; side < 2; ++side)
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      const int at = tid + i * kMoveThreads, r = at / kLanes, col = (at % kLanes) * 16;
      if (r < rows) piece[side][i] = *reinterpret_cast<const uint4*>(p.from.code[side] + ((size_t)bh * p.from.cap + s_src[r]) * D + col);
    }
  int id = 0;
  float weight = 0.f;
  if (tid < kBlockRows) {
    const int s = s_src[tid];
    // in place the scale of the block that the new length cuts may already be that of the rows moved into it
    const bool edge = s >= k && s / kBlockRows == k / kBlockRows;
#pragma unroll
    for (int side = 0; side < 2; ++side)
      s_scale[side][tid] = edge ? p.edge[2 * bh + side] : p.from.scale[side][(size_t)bh * from_blocks + s / kBlockRows];
    id = p.from.ids[(size_t)bh * p.from.cap + s];
    weight = p.from.weights[(size_t)bh * p.from.cap + s];
  }
  __syncthreads();
#pragma unroll
  for (int side = 0; side < 2; ++side)
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      const int r = (tid + i * kMoveThreads) / kLanes;
      if (r < rows) {
        const unsigned w[4] = {piece[side][i].x, piece[side][i].y, piece[side][i].z, piece[side][i].w};
        unsigned m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) m = __vmaxu4(m, __vabs4(w[j]));   // of -128, which no code is, 128
        m = __vmaxu4(m, m >> 16);
        m = max(m & 0xffu, (m >> 8) & 0xffu);
        amax[side] = fmaxf(amax[side], __uint_as_float(0x4b000000u | m) * s_scale[side][r] - 8388608.f * s_scale[side][r]);
      }
    }
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const float m = warp_max(amax[side]);
    if ((tid & 31) == 0) s_max[side][tid >> 5] = m;
  }
  __syncthreads();   // every row of this block has been read, too
  const int to_blocks = p.to.cap / kBlockRows;
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < kMoveThreads / 32; ++i) m = fmaxf(m, s_max[side][i]);
    // a block without a hole keeps its scale
    const int e = changed ? block_exp(m) : scale_exp(s_scale[side][0]);
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      const int at = tid + i * kMoveThreads, r = at / kLanes, col = (at % kLanes) * 16;
      if (r < rows) {
        const int d = scale_exp(s_scale[side][r]) - e;
        uint4 o = piece[side][i];
        if (d) {
          const float f = exp2i(max(d, -126));
          o = make_uint4(rescale4(o.x, f), rescale4(o.y, f), rescale4(o.z, f), rescale4(o.w, f));
        }
        *reinterpret_cast<uint4*>(p.to.code[side] + ((size_t)bh * p.to.cap + row0 + r) * D + col) = o;
      }
    }
    if (tid == 0) p.to.scale[side][(size_t)bh * to_blocks + blk] = exp2i(e);
  }
  if (tid < rows) {
    const size_t to = (size_t)bh * p.to.cap + row0 + tid;
    p.to.ids[to] = id;
    p.to.weights[to] = weight;
  }
}

}  // namespace

#include "st3_cache_attend.cuh"

// ------------------------------------------------------------------------------------------------------------------
// C ABI
// ------------------------------------------------------------------------------------------------------------------
namespace {

bool aligned16(const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

st3_status check_shape(const st3_cache* c) {
  if (!c) return ST3_ERR_INVALID_ARG;
  if (c->batch < 1 || c->num_kv_heads < 1 || c->capacity < 1 || c->capacity % kBlockRows) return ST3_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return ST3_ERR_UNSUPPORTED;
  // rows are numbered with 31 bits (codes of up to 2^38 bytes); the grids' second and third dimensions
  if ((long long)c->batch * c->num_kv_heads * c->capacity > 0x7fffffffLL) return ST3_ERR_UNSUPPORTED;
  if (c->batch > 32767 || c->num_kv_heads > 65535 || (long long)c->batch * c->num_kv_heads > 65535) return ST3_ERR_UNSUPPORTED;
  return ST3_OK;
}
st3_status check_cache(const st3_cache* c) {
  const st3_status st = check_shape(c);
  if (st != ST3_OK) return st;
  if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_scale) || !aligned16(c->v_scale) || !aligned16(c->ids) || !aligned16(c->weights))
    return ST3_ERR_INVALID_ARG;
  return ST3_OK;
}
CacheView view_of(const st3_cache* c) {
  CacheView v;
  v.code[0] = c->k; v.code[1] = c->v;
  v.scale[0] = c->k_scale; v.scale[1] = c->v_scale;
  v.ids = c->ids; v.weights = c->weights;
  v.batch = c->batch; v.heads = c->num_kv_heads; v.cap = c->capacity;
  return v;
}
size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

extern "C" st3_status st3_cache_store(const st3_cache* cache, const void* k, const void* v, int32_t dtype,
                                      int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                                      int64_t v_head_stride, const int32_t* cu, int32_t total, const int32_t* start,
                                      const int32_t* pos, int* dev_status, void* cuda_stream) {
  const st3_status st = check_cache(cache);
  if (st != ST3_OK) return st;
  if (total < 0 || !aligned4(cu) || (start && !aligned4(start)) || (pos && !aligned4(pos))) return ST3_ERR_INVALID_ARG;
  if (dtype != ST3_BF16 && dtype != ST3_F32) return ST3_ERR_UNSUPPORTED;
  if (total == 0) return ST3_OK;
  if (!aligned16(k) || !aligned16(v)) return ST3_ERR_INVALID_ARG;
  const int unit = dtype == ST3_BF16 ? 8 : 4;   // elements of 16 bytes
  if (total == 1) k_token_stride = v_token_stride = 0;   // never used, and whatever the caller's tensors call them
  if (cache->num_kv_heads == 1) k_head_stride = v_head_stride = 0;
  for (int64_t s : {k_token_stride, k_head_stride, v_token_stride, v_head_stride})
    if (s < 0 || s % unit) return ST3_ERR_INVALID_ARG;
  StoreParams p;
  p.c = view_of(cache);
  p.src[0] = k; p.src[1] = v;
  p.token_stride[0] = k_token_stride; p.token_stride[1] = v_token_stride;
  p.head_stride[0] = k_head_stride; p.head_stride[1] = v_head_stride;
  p.cu = cu; p.start = start; p.pos = pos; p.status = dev_status; p.total = total;
  p.wide = ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 31u) == 0 &&
           ((k_token_stride | k_head_stride | v_token_stride | v_head_stride) & (2 * unit - 1)) == 0;
  const dim3 grid((unsigned)(total / kBlockRows + 2 * cache->batch), (unsigned)cache->num_kv_heads);
  const dim3 block(kStoreThreads);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (dtype == ST3_BF16)
    return cache->head_dim == 128 ? launch(st3_cache_store_kernel<__nv_bfloat16, 128>, grid, block, 0, s, p)
                                  : launch(st3_cache_store_kernel<__nv_bfloat16, 64>, grid, block, 0, s, p);
  return cache->head_dim == 128 ? launch(st3_cache_store_kernel<float, 128>, grid, block, 0, s, p)
                                : launch(st3_cache_store_kernel<float, 64>, grid, block, 0, s, p);
}

extern "C" st3_status st3_cache_rows(const st3_cache* cache, const int32_t* first, const int32_t* held,
                                     int32_t num_rows, void* k, void* v, int32_t dtype, int32_t* ids, float* weights,
                                     void* cuda_stream) {
  const st3_status st = check_cache(cache);
  if (st != ST3_OK) return st;
  if (num_rows < 0 || !aligned4(held) || (first && !aligned4(first)) || (k && !aligned16(k)) || (v && !aligned16(v)) ||
      (ids && !aligned4(ids)) || (weights && !aligned4(weights)))
    return ST3_ERR_INVALID_ARG;
  if (dtype != ST3_BF16 && dtype != ST3_F32) return ST3_ERR_UNSUPPORTED;
  if (num_rows == 0) return ST3_OK;
  RowsParams p;
  p.c = view_of(cache);
  p.dst[0] = k; p.dst[1] = v; p.ids = ids; p.weights = weights; p.first = first; p.held = held; p.num_rows = num_rows;
  p.wide = ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 31u) == 0;
  const int per = kRowsThreads / (cache->head_dim / 16);
  const dim3 grid((unsigned)((num_rows + per - 1) / per), (unsigned)cache->num_kv_heads, 2 * (unsigned)cache->batch);
  const dim3 block(kRowsThreads);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (dtype == ST3_BF16)
    return cache->head_dim == 128 ? launch(st3_cache_rows_kernel<__nv_bfloat16, 128>, grid, block, 0, s, p)
                                  : launch(st3_cache_rows_kernel<__nv_bfloat16, 64>, grid, block, 0, s, p);
  return cache->head_dim == 128 ? launch(st3_cache_rows_kernel<float, 128>, grid, block, 0, s, p)
                                : launch(st3_cache_rows_kernel<float, 64>, grid, block, 0, s, p);
}

namespace {
// Blocks that share a head in the eviction: as many as hold its rows staged.  (us for one sequence of 8 heads, shared by 1 / 2 / 4 / 8
// blocks: 16 000 rows 36 / 26 / 23 / 23, 65 536: 138 / 96 / 67 / 46; for 16 sequences: 16 000 rows 88 / 76 / 90 / 132.)
int select_ranks(const st3_cache* c) {
  int ranks = 1;
  while (ranks < kEvictRanks && c->capacity > kEvictStage * ranks) ranks *= 2;
  return ranks;
}

struct EvictLayout { size_t src, movers, words, before, changed, length, edge, total; };
EvictLayout evict_layout(const st3_cache* c) {
  const size_t bh = (size_t)c->batch * c->num_kv_heads;
  EvictLayout l;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t x = at; at += up256(bytes); return x; };
  l.src = take(bh * c->capacity * 4);
  const int ranks = select_ranks(c);
  const size_t rows = c->capacity > kEvictStage * ranks ? bh * c->capacity : 0;   // not staged
  l.movers = take(ranks > 1 || rows ? bh * c->capacity * 4 : 0);
  l.words = take(rows / 32 * 4);
  l.before = take(rows / 32 * sizeof(int2));
  l.changed = take(bh * (c->capacity / kBlockRows) * 4);
  l.length = take(bh * 4);
  l.edge = take(bh * 8);
  l.total = at;
  return l;
}
}  // namespace

extern "C" st3_status st3_cache_evict_workspace(const st3_cache* from, size_t* bytes) {
  const st3_status st = check_shape(from);
  if (st != ST3_OK) return st;
  if (!bytes) return ST3_ERR_INVALID_ARG;
  *bytes = evict_layout(from).total;
  return ST3_OK;
}

extern "C" st3_status st3_cache_evict(const st3_cache* from, const st3_cache* to, const int32_t* held,
                                      const int32_t* seen, int32_t keep, int32_t recent, int32_t* held_out,
                                      void* workspace, size_t bytes, int* dev_status, void* cuda_stream) {
  st3_status st = check_cache(from);
  if (st == ST3_OK) st = check_cache(to);
  if (st != ST3_OK) return st;
  if (from->batch != to->batch || from->num_kv_heads != to->num_kv_heads || from->head_dim != to->head_dim) return ST3_ERR_INVALID_ARG;
  if (keep < 1 || recent < 0 || recent > keep || !aligned4(held) || !aligned4(seen) || !aligned4(held_out)) return ST3_ERR_INVALID_ARG;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return ST3_ERR_INVALID_ARG;
  // in place is all arrays in place
  const int same = (from->k == to->k) + (from->v == to->v) + (from->k_scale == to->k_scale) + (from->v_scale == to->v_scale) +
                   (from->ids == to->ids) + (from->weights == to->weights);
  if (same != 0 && (same != 6 || from->capacity != to->capacity)) return ST3_ERR_INVALID_ARG;
  if (to->capacity < keep && to->capacity < from->capacity) return ST3_ERR_CAPACITY;
  const EvictLayout l = evict_layout(from);
  if (bytes < l.total) return ST3_ERR_WORKSPACE_TOO_SMALL;
  char* ws = static_cast<char*>(workspace);
  EvictParams p;
  p.from = view_of(from); p.to = view_of(to);
  p.held = held; p.seen = seen; p.held_out = held_out; p.status = dev_status;
  p.src = reinterpret_cast<int*>(ws + l.src);
  p.movers = reinterpret_cast<int*>(ws + l.movers);
  p.words = reinterpret_cast<unsigned*>(ws + l.words);
  p.before = reinterpret_cast<int2*>(ws + l.before);
  p.changed = reinterpret_cast<int*>(ws + l.changed);
  p.length = reinterpret_cast<int*>(ws + l.length);
  p.edge = reinterpret_cast<float*>(ws + l.edge);
  p.keep = keep; p.recent = recent; p.in_place = same == 6;
  const unsigned bh = (unsigned)(from->batch * from->num_kv_heads);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const int ranks = select_ranks(from);
  if (ranks > 1 ? !allow_smem<st3_cache_select_kernel<true>>(kEvictSmem) : !allow_smem<st3_cache_select_kernel<false>>(kEvictSmem)) return ST3_ERR_CUDA;
  st = launch_clusters(ranks, ranks > 1 ? st3_cache_select_kernel<true> : st3_cache_select_kernel<false>, dim3(bh * (unsigned)ranks),
                       dim3(kEvictThreads), kEvictSmem, s, p);
  if (st != ST3_OK) return st;
  const int most = keep < from->capacity ? keep : from->capacity;
  const dim3 grid((unsigned)((most + kBlockRows - 1) / kBlockRows), bh);
  return from->head_dim == 128 ? launch(st3_cache_move_kernel<128>, grid, dim3(kMoveThreads), 0, s, p)
                               : launch(st3_cache_move_kernel<64>, grid, dim3(kMoveThreads), 0, s, p);
}

namespace {

struct AttendLayout { size_t ml, acc, logits, total; int group, passes, pitch, grid; };
AttendLayout attend_layout(const st3_cache* c, int heads, bool weights) {
  AttendLayout l;
  l.group = heads / c->num_kv_heads;
  l.passes = (l.group + kCaHeads - 1) / kCaHeads;
  l.pitch = l.group <= 8 ? 8 : kCaHeads;
  const long long blocks = (long long)c->batch * c->num_kv_heads * l.passes * (c->capacity / kBlockRows + kCaStart);
  l.grid = blocks < kCaGrid ? (int)blocks : kCaGrid;
  const size_t slots = (size_t)l.grid + (size_t)c->batch * c->num_kv_heads * l.passes;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t x = at; at += up256(bytes); return x; };
  l.ml = take(slots * l.pitch * 3 * 4);
  l.acc = take(slots * l.pitch * c->head_dim * 4);
  l.logits = take(weights ? (size_t)c->batch * heads * c->capacity * 4 : 0);
  l.total = at;
  return l;
}

bool make_code_map(EncodeTiledFn fn, CUtensorMap* map, const st3_cache* c, const int8_t* base) {
  const cuuint64_t rows = (cuuint64_t)c->batch * c->num_kv_heads * c->capacity;
  const cuuint64_t dims[2] = {(cuuint64_t)c->head_dim, rows};
  const cuuint64_t strides[1] = {(cuuint64_t)c->head_dim};
  const cuuint32_t box[2] = {(cuuint32_t)c->head_dim, kBlockRows};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            c->head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D, int kTiles>
st3_status attend_launch(const CUtensorMap& mk, const CUtensorMap& mv, const CacheAttendParams& p, cudaStream_t s) {
  if (!allow_smem<st3_cache_attend_kernel<T, D, kTiles>>(CaLayout<D>::kTotal)) return ST3_ERR_CUDA;
  st3_status st = launch(st3_cache_attend_kernel<T, D, kTiles>, dim3((unsigned)p.grid), dim3(kCaThreads), CaLayout<D>::kTotal, s, mk, mv, p);
  if (st != ST3_OK) return st;
  const unsigned pairs = (unsigned)(p.c.batch * p.c.heads), group = (unsigned)p.group;
  auto chunks = [&](int split) { return p.weights_out ? (unsigned)((p.c.cap + ca_chunk(split) - 1) / ca_chunk(split)) : 0u; };
  const dim3 block(kCaMergeThreads);
  // five segments a pair or more on average (the wave's thread blocks over the pairs): four warps to a head
  if (pairs * (unsigned)p.passes * 4 <= kCaGrid)
    return launch(st3_cache_merge_kernel<T, D, 4>, dim3(pairs, group + chunks(4)), block, 0, s, p);
  return launch(st3_cache_merge_kernel<T, D, 1>, dim3(pairs, (group + 3) / 4 + chunks(1)), block, 0, s, p);
}

st3_status check_heads(const st3_cache* c, int heads) {
  if (heads < 1 || heads % c->num_kv_heads) return ST3_ERR_INVALID_ARG;
  if (heads / c->num_kv_heads > 1024 || (long long)c->batch * heads * c->capacity > 0x7fffffffffLL) return ST3_ERR_UNSUPPORTED;
  const long long passes = (heads / c->num_kv_heads + kCaHeads - 1) / kCaHeads;
  if ((long long)c->batch * c->num_kv_heads * passes * (c->capacity / kBlockRows + kCaStart) > 0x3fffffffLL) return ST3_ERR_UNSUPPORTED;
  if (heads / c->num_kv_heads + c->capacity / ca_chunk(4) + 1 > 65535) return ST3_ERR_UNSUPPORTED;
  return ST3_OK;
}

}  // namespace

extern "C" st3_status st3_cache_attend_workspace(const st3_cache* cache, int32_t num_heads, int32_t with_weights, size_t* bytes) {
  st3_status st = check_shape(cache);
  if (st == ST3_OK) st = check_heads(cache, num_heads);
  if (st != ST3_OK) return st;
  if (!bytes) return ST3_ERR_INVALID_ARG;
  *bytes = attend_layout(cache, num_heads, with_weights != 0).total;
  return ST3_OK;
}

extern "C" st3_status st3_cache_attend(const st3_cache* cache, const void* q, void* out, int32_t dtype, int32_t num_heads,
                                       const int32_t* held, const float* weights_in, float* weights_out,
                                       void* workspace, size_t bytes, int* dev_status, void* cuda_stream) {
  st3_status st = check_cache(cache);
  if (st == ST3_OK) st = check_heads(cache, num_heads);
  if (st != ST3_OK) return st;
  if (!aligned16(q) || !aligned16(out) || !aligned4(held) || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return ST3_ERR_INVALID_ARG;
  if (weights_out && (!aligned4(weights_in) || !aligned4(weights_out))) return ST3_ERR_INVALID_ARG;
  if (dtype != ST3_BF16 && dtype != ST3_F32) return ST3_ERR_UNSUPPORTED;
  const AttendLayout l = attend_layout(cache, num_heads, weights_out != nullptr);
  if (bytes < l.total) return ST3_ERR_WORKSPACE_TOO_SMALL;
  const EncodeTiledFn encode = tensor_map_encoder();
  CUtensorMap mk, mv;
  if (!encode || !make_code_map(encode, &mk, cache, cache->k) || !make_code_map(encode, &mv, cache, cache->v)) return ST3_ERR_CUDA;
  char* ws = static_cast<char*>(workspace);
  CacheAttendParams p;
  p.c = view_of(cache);
  p.q = q; p.out = out; p.held = held; p.weights_in = weights_in; p.weights_out = weights_out; p.status = dev_status;
  p.part_ml = reinterpret_cast<float*>(ws + l.ml);
  p.part_acc = reinterpret_cast<float*>(ws + l.acc);
  p.logits = weights_out ? reinterpret_cast<float*>(ws + l.logits) : nullptr;
  p.group = l.group; p.passes = l.passes; p.pitch = l.pitch; p.grid = l.grid;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const bool wide = l.group > 8, d128 = cache->head_dim == 128;
  if (dtype == ST3_BF16) {
    if (d128) return wide ? attend_launch<__nv_bfloat16, 128, 2>(mk, mv, p, s) : attend_launch<__nv_bfloat16, 128, 1>(mk, mv, p, s);
    return wide ? attend_launch<__nv_bfloat16, 64, 2>(mk, mv, p, s) : attend_launch<__nv_bfloat16, 64, 1>(mk, mv, p, s);
  }
  if (d128) return wide ? attend_launch<float, 128, 2>(mk, mv, p, s) : attend_launch<float, 128, 1>(mk, mv, p, s);
  return wide ? attend_launch<float, 64, 2>(mk, mv, p, s) : attend_launch<float, 64, 1>(mk, mv, p, s);
}
