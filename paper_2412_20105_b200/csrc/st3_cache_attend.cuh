// One query per head over the 8-bit cache; included by st3_cache.cu only.
//
// What bounds it: the codes, 2 D bytes a row and key/value head, read once for all query heads of the group.  At one byte an
// element a group of four does 8 flops a byte, beyond what the fp32 pipes keep up with, so the products run on mma.sync
// (m16n8k16, f16 x f16 -> fp32): codes are exact in f16, the query is scaled by a power of two into f16's range (bf16 fits
// exactly, fp32 is split in two halves of 11 bits), and the accumulators are fp32.  tcgen05 has nothing to win here: its
// 128 rows of M would hold 1 to 16 queries.
//
// Work: the blocks of 64 rows of all (sequence, head) pairs, end to end, cut into equal runs, one for each thread block of
// one wave (two to an SM), so that ragged lengths and single long sequences fill the GPU alike.  What a run holds of one pair
// is a segment; a segment leaves one partial (max, sum, un-normalised output), and a second launch joins the partials and
// adds the probabilities to the accumulated weights from the logits left by the first.  Thread block c and pair i share at
// most one segment, and along the runs either c or i grows from one segment to the next: c + i numbers them without a table.
//
// A producer warp brings whole blocks by TMA (K and V, 8 KB each at D = 128) into a ring; four consumer warps take 16 rows
// of a block each.  The codes lie in shared memory as TMA's swizzle puts them, so that ldmatrix reads without bank conflicts:
// for S = K q^T a register holds four neighbouring dims of a row, which become two f16 pairs; for O^T = V^T P^T ldmatrix
// transposes 16-bit units, and a register holds two neighbouring dims of two rows, which become two pairs of rows.
#ifndef ST3_CACHE_ATTEND_CUH_
#define ST3_CACHE_ATTEND_CUH_

namespace {

constexpr int kCaGrid = 2 * 148;       // one wave
constexpr int kCaConsumers = 4;
constexpr int kCaThreads = (kCaConsumers + 1) * 32;
constexpr int kCaHeads = 16;           // query heads of one pass over a group's rows; larger groups take several
constexpr int kCaStart = 2;            // units of a pair beside its blocks (none: 42.7 us, 1: 40.9, 2: 40.1, 3: 40.2 for 32 users)
// log2 of the largest probability * scale that goes into f16, whose numbers reach 2^16 and have all their bits down to 2^-14: rows
// that weigh 2^-29 of the heaviest one do, and lighter ones an absolute step of 2^-39 of it.  (From 1 down there would be 2^15
// less: a row without a value of its own, e^14 above the others, cost the output 1e-3, and e^17.4 all of it.)
constexpr float kCaTop = 15.f;
constexpr int kCaMergeThreads = 128;
// Rows of the second launch's blocks that add weights: one round of loads, or two where blocks are many.
__host__ __device__ constexpr int ca_chunk(int split) { return split == 4 ? 512 : 1024; }

struct CacheAttendParams {
  CacheView c;
  const void* q;
  void* out;
  const int* held;
  const float* weights_in;
  float* weights_out;
  int* status;
  float* part_ml;    // [segment][heads of a pass][3]: max of the logits, max of logit + log2(V scale), sum
  float* part_acc;   // [segment][heads of a pass][D]
  float* logits;     // [(sequence, kv head)][row][group] in the log2 domain, or null
  int group;         // query heads per key/value head
  int passes;        // ceil(group / kCaHeads)
  int pitch;         // heads of a pass, rounded up to 8
  int grid;
};

template <int D>
struct CaLayout {
  static constexpr int kSide = kBlockRows * D;               // bytes of a block's K or V
  static constexpr int kStage = 2 * kSide;
  static constexpr int kStages = 80 * 1024 / kStage;
  static constexpr int kPitch = D + 4;                       // floats from one head's sums to the next: no bank conflicts
  static constexpr int kRed = kStages * kStage;              // sums of the four warps, 8 heads at a time
  static constexpr int kBars = kRed + kCaConsumers * 8 * kPitch * 4;
  static constexpr int kMl = kBars + 2 * kStages * 8;
  static constexpr int kTotal = kMl + kCaConsumers * 8 * 3 * 4 + 64;
};

// The run of thread block c: blocks [total * c / grid, total * (c + 1) / grid), with grid <= total, so that none is empty.
__device__ __forceinline__ int run_start(int total, int c, int grid) { return (int)((long long)total * c / grid); }
// The thread block whose run holds block x.
__device__ __forceinline__ int run_of(int total, int x, int grid) { return (int)((((long long)x + 1) * grid - 1) / total); }
// Rows held, from L2: the joining launch reads them ahead of its wait, when nothing says that this SM's L1 is not older than them.
__device__ __forceinline__ int held_of(const CacheAttendParams& p, int b) { return clamp_rows(__ldcg(p.held + b), p.c.cap); }
__device__ __forceinline__ int blocks_of(const CacheAttendParams& p, int b) { return (held_of(p, b) + kBlockRows - 1) / kBlockRows; }
// Runs are counted in units: a pair's blocks, and kCaStart in front of them for what a segment costs beside its blocks (queries and
// scales to fetch, sums to join), so that runs of many short pairs are not the last ones to end.
__device__ __forceinline__ int units_of(int blocks) { return blocks ? blocks + kCaStart : 0; }

__device__ __forceinline__ void tma_rows(void* dst, const CUtensorMap* map, int row, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(dst)),
      "l"(map), "r"(0), "r"(row), "r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ bool ca_wait(uint64_t* bar, uint32_t parity) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity))
    if (clock64() - t0 > kWaitCycles) return false;
  return true;
}
__device__ __forceinline__ void ca_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// A barrier of the consumer warps that tells each of them whether any has failed.
__device__ __forceinline__ bool ca_any_failed(bool failed) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, 1, %2, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"((uint32_t)failed), "n"(kCaConsumers * 32)
      : "memory");
  return any != 0;
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Two codes of a word as f16: biased by 128 they are the low bits of 1024 + u, from which 1152 is taken.  `flipped` is the
// word with every code's sign bit inverted.
template <int kSel>
__device__ __forceinline__ uint32_t codes_f16(uint32_t flipped) {
  const uint32_t w = __byte_perm(flipped, 0x64646464u, kSel);
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&w), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t half_pair(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// what rounding the pair to f16 has lost, as another pair
__device__ __forceinline__ uint32_t half_rest(float a, float b, uint32_t hi) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  return half_pair(a - f.x, b - f.y);
}

// kTiles: groups of 8 query heads of a pass.  fp32 queries and probabilities go in as two f16 terms each.
template <typename T, int D, int kTiles>
__global__ void __launch_bounds__(kCaThreads, 2)
st3_cache_attend_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const CacheAttendParams p) {
  using L = CaLayout<D>;
  constexpr int kTerms = sizeof(T) == 4 ? 2 : 1;
  constexpr int kSteps = D / 16;
  extern __shared__ __align__(1024) unsigned char smem[];
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBars);
  uint64_t* empty = full + L::kStages;
  float* s_ml = reinterpret_cast<float*>(smem + L::kMl);
  int* s_int = reinterpret_cast<int*>(s_ml + kCaConsumers * 8 * 3);   // 16 ints
  float* s_red = reinterpret_cast<float*>(smem + L::kRed);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    prefetch_map(&map_k);
    prefetch_map(&map_v);
    for (int i = 0; i < L::kStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], kCaConsumers); }
    mbar_fence_init();
    s_int[8] = 0;
  }
  if (smem_u32(smem) & 1023u) {   // the swizzle assumes aligned tiles: reported, nothing computed
    if (tid == 0 && p.status) atomicOr(p.status, ST3_DEV_RANGE);
    pdl_wait();
    return;
  }
  pdl_wait();
  pdl_next();
  // ---- this block's run, and the sequence that its first block lies in ----
  const int per = (p.c.batch + kCaThreads - 1) / kCaThreads, pairs = p.c.heads * p.passes;
  int mine = 0;
  for (int i = 0; i < per; ++i) {
    const int b = tid * per + i;
    if (b < p.c.batch) {
      mine += units_of(blocks_of(p, b));
      if (blockIdx.x == 0 && p.status && p.held[b] != clamp_rows(p.held[b], p.c.cap)) atomicOr(p.status, ST3_DEV_RANGE);
    }
  }
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) s_int[warp] = incl;
  __syncthreads();
  int before = incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w <= kCaConsumers; ++w) {
    if (w < warp) before += s_int[w];
    total += s_int[w];
  }
  total *= pairs;
  before *= pairs;   // units of all pairs in front of this thread's first sequence
  const int grid = min(p.grid, total);
  const bool works = (int)blockIdx.x < grid;
  const int x0 = works ? run_start(total, blockIdx.x, grid) : 0, x1 = works ? run_start(total, blockIdx.x + 1, grid) : 0;
  if (x0 < x1 && x0 >= before && x0 < before + mine * pairs) {
    int b = tid * per;
    for (;; ++b) {
      const int n = units_of(blocks_of(p, b)) * pairs;
      if (x0 < before + n) break;
      before += n;
    }
    s_int[6] = b;
    s_int[7] = before;
  }
  __syncthreads();
  if (x0 >= x1) return;
  int b = s_int[6], x = x0, seq0 = s_int[7];
  volatile int* fail = s_int + 8;

  if (warp == kCaConsumers) {
    // ===================== producer =====================
    if (lane == 0) {
      bool ok = true;
      int stage = 0, parity = 1, issued = 0;
      while (x < x1 && ok) {
        int units = units_of(blocks_of(p, b));
        while (x >= seq0 + units * pairs) { seq0 += units * pairs; units = units_of(blocks_of(p, ++b)); }
        const int pair = (x - seq0) / units, head = pair / p.passes;
        const int u = x - seq0 - pair * units, take = min(units - u, x1 - x);
        const int i0 = max(u - kCaStart, 0), i1 = u + take - kCaStart;   // none, where the run holds a pair's start only
        const int row = (b * p.c.heads + head) * p.c.cap;
        for (int i = i0; i < i1; ++i) {
          if (!ca_wait(&empty[stage], parity) || *fail) { ok = false; break; }
          unsigned char* dst = smem + stage * L::kStage;
          mbar_expect_tx(&full[stage], L::kStage);
          tma_rows(dst, &map_k, row + i * kBlockRows, &full[stage]);
          tma_rows(dst + L::kSide, &map_v, row + i * kBlockRows, &full[stage]);
          ++issued;
          if (++stage == L::kStages) { stage = 0; parity ^= 1; }
        }
        x += take;
      }
      if (!ok) {
        *fail = 1;
        if (p.status) atomicOr(p.status, ST3_DEV_COPY_TIMEOUT);
      }
      // shared memory is not given back before the copies into it have landed, also where a consumer gave up
      for (int u = max(0, issued - L::kStages); u < issued; ++u) ca_wait(&full[u % L::kStages], (u / L::kStages) & 1);
    }
    return;
  }

  // ===================== consumers =====================
  const int g = lane >> 2, t = lane & 3;
  const float sc = 1.4426950408889634f * rsqrtf((float)D);
  const uint32_t ring = smem_u32(smem);
  // ldmatrix addresses inside a block: row 16 warp + (lane & 15) for K and V; the lane's 16-byte chunk is 2 i + (lane >> 4)
  const int lrow = warp * 16 + (lane & 15);
  const int lxor = D == 128 ? (lrow & 7) : ((lrow >> 1) & 3);
  const uint32_t lbase = (uint32_t)(lrow * D);
  int stage = 0;
  uint32_t parity = 0;
  bool ok = true;
  // A segment, and what it needs from memory, which is requested ahead of the end of the one before it.
  struct Segment { int b, pair, h0, heads, i0, i1, held; size_t bh; } seg;
  using Four = typename std::conditional<sizeof(T) == 2, uint2, float4>::type;
  Four raw[kTiles][kSteps];   // queries: head g, dims 16 i + 4 t .. + 3
  float ks32, vs32;           // the scales of 32 blocks, one a lane
  auto request = [&] {   // the run's next segment; false at its end
    int units = 0, pair = 0, i0 = 0, i1 = 0;
    do {
      if (x >= x1) return false;
      units = units_of(blocks_of(p, b));
      while (x >= seq0 + units * pairs) { seq0 += units * pairs; units = units_of(blocks_of(p, ++b)); }
      pair = (x - seq0) / units;
      const int u = x - seq0 - pair * units, take = min(units - u, x1 - x);
      i0 = max(u - kCaStart, 0);
      i1 = u + take - kCaStart;
      x += take;
    } while (i1 <= i0);
    const int head = pair / p.passes;
    seg.b = b;
    seg.pair = pair;
    seg.h0 = (pair - head * p.passes) * kCaHeads;
    seg.heads = min(p.group - seg.h0, kCaHeads);   // of this pass
    seg.i0 = i0;
    seg.i1 = i1;
    seg.held = held_of(p, b);
    seg.bh = (size_t)b * p.c.heads + head;
    const size_t at = seg.bh * (p.c.cap / kBlockRows) + min(seg.i0 + lane, seg.i1 - 1);
    ks32 = p.c.scale[0][at];
    vs32 = p.c.scale[1][at];
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      const bool live = n * 8 + g < seg.heads;
      const T* src = static_cast<const T*>(p.q) + (seg.bh * p.group + seg.h0 + n * 8 + g) * D + 4 * t;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        raw[n][i] = Four{};
        if (live) raw[n][i] = *reinterpret_cast<const Four*>(src + 16 * i);
      }
    }
    return true;
  };
  if (!request()) return;
  while (true) {
    const Segment now = seg;
    const int i0 = now.i0, i1 = now.i1, heads = now.heads, h0 = now.h0, held = now.held;
    const size_t bh = now.bh;
    const float* ks = p.c.scale[0] + bh * (p.c.cap / kBlockRows);
    const float* vs = p.c.scale[1] + bh * (p.c.cap / kBlockRows);
    // ---- the queries of this pass as B fragments ----
    uint32_t qf[kTerms][kTiles][kSteps][2];
    float qs[kTiles][2];   // factor of the logits of heads 2 t and 2 t + 1
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      float f[kSteps][4];
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        if constexpr (sizeof(T) == 2) {
          f[i][0] = __uint_as_float(raw[n][i].x << 16); f[i][1] = __uint_as_float(raw[n][i].x & 0xffff0000u);
          f[i][2] = __uint_as_float(raw[n][i].y << 16); f[i][3] = __uint_as_float(raw[n][i].y & 0xffff0000u);
        } else {
          f[i][0] = raw[n][i].x; f[i][1] = raw[n][i].y; f[i][2] = raw[n][i].z; f[i][3] = raw[n][i].w;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(f[i][e]));
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // |q| * 2^-e lies in [2^13, 2^14): f16 keeps its 11 bits down to 2^-27 of the largest element
      const int e = min(max((int)(__float_as_uint(top) >> 23) - 127 - 13, -100), 114);
      const float down = exp2i(-e), up = exp2i(e);
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const float a = f[i][2 * w] * down, c = f[i][2 * w + 1] * down;
          qf[0][n][i][w] = half_pair(a, c);
          if constexpr (kTerms == 2) qf[kTerms - 1][n][i][w] = half_rest(a, c, qf[0][n][i][w]);
        }
      }
      qs[n][0] = sc * __shfl_sync(0xffffffffu, up, 8 * t);
      qs[n][1] = sc * __shfl_sync(0xffffffffu, up, 8 * t + 4);
    }
    // m: running maximum of a head's logits, l: sum of exp2(s - m) over this lane's rows; mv: running maximum of
    // s + log2(V scale), which the probabilities that meet V are relative to, so that blocks of any scale share one
    // accumulator and the largest term is 2^kCaTop.
    float m[kTiles][2], mv[kTiles][2], l[kTiles][2];
    float acc[kTiles][kSteps][4];
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      m[n][0] = m[n][1] = mv[n][0] = mv[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) acc[n][i][0] = acc[n][i][1] = acc[n][i][2] = acc[n][i][3] = 0.f;
    }
    for (int i = i0; i < i1; ++i) {
      const int at = (i - i0) & 31;
      if (at == 0 && i > i0) {
        const int j = min(i + lane, i1 - 1);
        ks32 = ks[j];
        vs32 = vs[j];
      }
      const float kscale = exp2i(scale_exp(__shfl_sync(0xffffffffu, ks32, at)));
      const float vexp = (float)scale_exp(__shfl_sync(0xffffffffu, vs32, at));
      if (ok) ok = __all_sync(0xffffffffu, ca_wait(&full[stage], parity)) && !*fail;
      if (!ok) break;
      const uint32_t kb = ring + stage * L::kStage + lbase, vb = kb + L::kSide;
      // ---- S = K q^T: 16 rows x 8 heads a tile ----
      float s[kTiles][4];
#pragma unroll
      for (int n = 0; n < kTiles; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
      float s2[kTiles][4];   // every other step, a second chain
#pragma unroll
      for (int n = 0; n < kTiles; ++n) s2[n][0] = s2[n][1] = s2[n][2] = s2[n][3] = 0.f;
#pragma unroll
      for (int c = 0; c < kSteps; c += 2) {
        uint32_t r[4];
        ldsm4(r, kb + (((c + (lane >> 4)) ^ lxor) << 4));
        // matrices: rows 0-7 and 8-15 of chunk c, then of chunk c + 1
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] ^= 0x80808080u;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t a0 = codes_f16<0x4140>(r[2 * j]), a1 = codes_f16<0x4140>(r[2 * j + 1]);
          const uint32_t a2 = codes_f16<0x4342>(r[2 * j]), a3 = codes_f16<0x4342>(r[2 * j + 1]);
#pragma unroll
          for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int term = 0; term < kTerms; ++term)
              mma_f16(j ? s2[n] : s[n], a0, a1, a2, a3, qf[term][n][c + j][0], qf[term][n][c + j][1]);
        }
      }
      // ---- softmax over this warp's 16 rows; lane: rows g and g + 8, heads 2 t and 2 t + 1 ----
      const int row = i * kBlockRows + warp * 16 + g;
      const bool in0 = row < held, in1 = row + 8 < held;
      uint32_t pf[kTerms][kTiles][2];
#pragma unroll
      for (int n = 0; n < kTiles; ++n) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = ((e < 2) ? in0 : in1) ? (s[n][e] + s2[n][e]) * (kscale * qs[n][e & 1]) : -INFINITY;
        if (p.logits) {
          float* dst = p.logits + ((size_t)bh * p.c.cap + row) * p.group + h0 + n * 8 + 2 * t;
          if (p.group & 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (((e < 2) ? in0 : in1) && n * 8 + 2 * t + (e & 1) < heads) dst[(e >> 1) * 8 * p.group + (e & 1)] = v[e];
          } else if (n * 8 + 2 * t < heads) {   // pairs of heads side by side, on 8 bytes
            if (in0) *reinterpret_cast<float2*>(dst) = make_float2(v[0], v[1]);
            if (in1) *reinterpret_cast<float2*>(dst + 8 * p.group) = make_float2(v[2], v[3]);
          }
        }
        float top[2] = {fmaxf(v[0], v[2]), fmaxf(v[1], v[3])};
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          top[0] = fmaxf(top[0], __shfl_xor_sync(0xffffffffu, top[0], o));
          top[1] = fmaxf(top[1], __shfl_xor_sync(0xffffffffu, top[1], o));
        }
        float ref[2], refv[2];
        bool grown = false;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float m1 = fmaxf(m[n][j], top[j]), mv1 = fmaxf(mv[n][j], top[j] + vexp);
          ref[j] = m1 > -INFINITY ? m1 : 0.f;
          refv[j] = mv1 > -INFINITY ? mv1 : 0.f;
          if (m1 > m[n][j]) { l[n][j] *= fast_exp2(m[n][j] - ref[j]); m[n][j] = m1; }
          grown |= mv1 > mv[n][j];
        }
        if (__any_sync(0xffffffffu, grown)) {
          float f[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            f[j] = fast_exp2(mv[n][j] - refv[j]);   // 0 where nothing has been added yet
            mv[n][j] = fmaxf(mv[n][j], top[j] + vexp);
            if (!(mv[n][j] > -INFINITY)) f[j] = 1.f;
          }
#pragma unroll
          for (int c = 0; c < kSteps; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[n][c][e] *= f[e & 1];
        }
        float w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          l[n][e & 1] += fast_exp2(v[e] - ref[e & 1]);
          w[e] = fast_exp2(v[e] + vexp - refv[e & 1] + kCaTop);   // the difference is 0 at most, also where logits have no bits below 1
        }
        const uint32_t lo = half_pair(w[0], w[1]), hi = half_pair(w[2], w[3]);
        pf[0][n][0] = transpose8x8(lo);   // head g, rows 2 t and 2 t + 1
        pf[0][n][1] = transpose8x8(hi);   // rows 2 t + 8 and 2 t + 9
        if constexpr (kTerms == 2) {
          pf[kTerms - 1][n][0] = transpose8x8(half_rest(w[0], w[1], lo));
          pf[kTerms - 1][n][1] = transpose8x8(half_rest(w[2], w[3], hi));
        }
      }
      // ---- O^T += V^T P^T: 16 dims x 8 heads a tile; row g is dim 16 c + 2 g, row g + 8 the one after it ----
#pragma unroll
      for (int c = 0; c < kSteps; c += 2) {
        uint32_t r[4];
        ldsm4_t(r, vb + (((c + (lane >> 4)) ^ lxor) << 4));
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] ^= 0x80808080u;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t a0 = codes_f16<0x4240>(r[2 * j]), a1 = codes_f16<0x4341>(r[2 * j]);
          const uint32_t a2 = codes_f16<0x4240>(r[2 * j + 1]), a3 = codes_f16<0x4341>(r[2 * j + 1]);
#pragma unroll
          for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int term = 0; term < kTerms; ++term) mma_f16(acc[n][c + j], a0, a1, a2, a3, pf[term][n][0], pf[term][n][1]);
        }
      }
      __syncwarp();
      if (lane == 0) ca_arrive(&empty[stage]);
      if (++stage == L::kStages) { stage = 0; parity ^= 1; }
    }
    // ---- the four warps' shares become the segment's partial ----
    if (!ok) {
      *fail = 1;
      if (lane == 0 && p.status) atomicOr(p.status, ST3_DEV_COPY_TIMEOUT);
    }
    // ahead of the sums where the registers allow it: a round trip under them
    constexpr bool kEarly = sizeof(T) == 2 && kTiles == 1;
    bool more = kEarly && ok && request();
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l[n][j] += __shfl_xor_sync(0xffffffffu, l[n][j], o);
    const size_t slot = (size_t)blockIdx.x + (size_t)now.b * pairs + now.pair;
    float* out_acc = p.part_acc + slot * p.pitch * D;
    float* out_ml = p.part_ml + slot * p.pitch * 3;
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      // One verdict for the four warps, as these barriers count on all of them; and nobody still reads what is overwritten here.
      if (ca_any_failed(!ok)) return;
      float* dst = s_red + (size_t)warp * 8 * L::kPitch;
#pragma unroll
      for (int c = 0; c < kSteps; ++c)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          *reinterpret_cast<float2*>(dst + (2 * t + j) * L::kPitch + 16 * c + 2 * g) = make_float2(acc[n][c][j], acc[n][c][2 + j]);
      if (g < 3) {   // lanes of three rows write one of the three numbers each
#pragma unroll
        for (int j = 0; j < 2; ++j) s_ml[(warp * 8 + 2 * t + j) * 3 + g] = g == 0 ? m[n][j] : g == 1 ? mv[n][j] : l[n][j];
      }
      asm volatile("bar.sync 1, %0;" ::"n"(kCaConsumers * 32) : "memory");
      // 16 threads to a head
      const int h = tid >> 4, d0 = (tid & 15) * 4;
      float a[kCaConsumers], av[kCaConsumers], top = -INFINITY, topv = -INFINITY;
#pragma unroll
      for (int w = 0; w < kCaConsumers; ++w) {
        a[w] = s_ml[(w * 8 + h) * 3];
        av[w] = s_ml[(w * 8 + h) * 3 + 1];
        top = fmaxf(top, a[w]);
        topv = fmaxf(topv, av[w]);
      }
      const float ref = top > -INFINITY ? top : 0.f, refv = topv > -INFINITY ? topv : 0.f;
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < kCaConsumers; ++w) {
        sum += s_ml[(w * 8 + h) * 3 + 2] * fast_exp2(a[w] - ref);
        av[w] = fast_exp2(av[w] - refv);
      }
      if (n * 8 + h < heads) {
#pragma unroll
        for (int d = 0; d < D; d += 64) {
          float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int w = 0; w < kCaConsumers; ++w) {
            const float4 v = *reinterpret_cast<const float4*>(s_red + (w * 8 + h) * L::kPitch + d0 + d);
            o.x = fmaf(v.x, av[w], o.x); o.y = fmaf(v.y, av[w], o.y); o.z = fmaf(v.z, av[w], o.z); o.w = fmaf(v.w, av[w], o.w);
          }
          *reinterpret_cast<float4*>(out_acc + (n * 8 + h) * D + d0 + d) = o;
        }
        if (d0 == 0) {
          float* dst3 = out_ml + (n * 8 + h) * 3;
          dst3[0] = top; dst3[1] = topv; dst3[2] = sum;
        }
      }
    }
    if (!kEarly) more = request();
    if (!more) break;
  }
}

// Joins the partials.  Grid y < out_blocks: the outputs of 4 / kSplit heads, a head's segments shared out over kSplit warps; the
// other y: kChunk rows of a (sequence, key/value head), whose weights get the probabilities of the group's heads.
// Bound by round trips: the row counts are read before the wait (the attention launch ahead has started only after everything
// before it was complete, and leaves them alone); a head's maxima and sums are requested together with the sums of its
// outputs, or with the logits.  Four warps a head where a pair has many segments (4 x 65 000 rows of 8 heads: 11 -> 5 us
// against one block for all heads), one where the pairs are many and the blocks would take several rounds of the GPU.
template <typename T, int D, int kSplit>
__global__ void __launch_bounds__(kCaMergeThreads) st3_cache_merge_kernel(const CacheAttendParams p) {
  constexpr int kWarps4 = kCaMergeThreads / 32, kHeads = kWarps4 / kSplit, kAhead = kSplit == 4 ? 8 : 4, kVec = D / 32;
  constexpr int kChunk = ca_chunk(kSplit);
  __shared__ int s_sum[2][kWarps4];
  __shared__ float s_ml[kHeads][3][kCaGrid + 1];
  __shared__ float s_ref[128], s_inv[128];
  __shared__ float s_acc[kWarps4][D];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, bh = blockIdx.x;
  const int b = bh / p.c.heads, head = bh - b * p.c.heads, pairs = p.c.heads * p.passes;
  int all = 0, below = 0;
  for (int i = tid; i < p.c.batch; i += kCaMergeThreads) {
    const int n = units_of(blocks_of(p, i));
    all += n;
    if (i < b) below += n;
  }
  const int held = held_of(p, b), nb = (held + kBlockRows - 1) / kBlockRows;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    all += __shfl_xor_sync(0xffffffffu, all, o);
    below += __shfl_xor_sync(0xffffffffu, below, o);
  }
  if (lane == 0) { s_sum[0][warp] = all; s_sum[1][warp] = below; }
  __syncthreads();
  all = below = 0;
#pragma unroll
  for (int w = 0; w < kWarps4; ++w) { all += s_sum[0][w]; below += s_sum[1][w]; }
  const int total = all * pairs, grid = min(p.grid, total);
  pdl_wait();
  pdl_next();
  const int out_blocks = (p.group + kHeads - 1) / kHeads;
  if ((int)blockIdx.y < out_blocks) {
    // ---- outputs ----
    const int sub = warp % kSplit, h = blockIdx.y * kHeads + warp / kSplit, pass = h / kCaHeads, pair = head * p.passes + pass;
    const bool live = h < p.group;
    float (&mls)[3][kCaGrid + 1] = s_ml[warp / kSplit];
    T* dst = static_cast<T*>(p.out) + ((size_t)bh * p.group + h) * D;
    if (nb == 0) {
      if (live && sub == 0)
        for (int e = lane; e < D; e += 32) store_out(dst + e, 0.f);
      return;
    }
    const int x = below * pairs + pair * units_of(nb) + kCaStart;   // the pair's first block
    const int c0 = run_of(total, x, grid), n = live ? run_of(total, x + nb - 1, grid) - c0 + 1 : 0;   // n <= grid segments
    const size_t slot0 = ((size_t)b * pairs + pair + c0) * p.pitch + h - pass * kCaHeads;
    const float* ml = p.part_ml + slot0 * 3;
    const float* acc = p.part_acc + slot0 * D + lane * kVec;
    float ahead[kAhead][kVec];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int c = sub + j * kSplit;
#pragma unroll
      for (int e = 0; e < kVec; ++e) ahead[j][e] = 0.f;
      if (c < n) {
        if constexpr (kVec == 4) {
          const float4 v = *reinterpret_cast<const float4*>(acc + (size_t)c * p.pitch * D);
          ahead[j][0] = v.x; ahead[j][1] = v.y; ahead[j][kVec - 2] = v.z; ahead[j][kVec - 1] = v.w;
        } else {
          const float2 v = *reinterpret_cast<const float2*>(acc + (size_t)c * p.pitch * D);
          ahead[j][0] = v.x; ahead[j][1] = v.y;
        }
      }
    }
    for (int c = sub * 32 + lane; c < n; c += kSplit * 32)
#pragma unroll
      for (int e = 0; e < 3; ++e) mls[e][c] = ml[(size_t)c * p.pitch * 3 + e];
    __syncthreads();
    float a = -INFINITY, av = -INFINITY, sum = 0.f;
    for (int c = lane; c < n; c += 32) { a = fmaxf(a, mls[0][c]); av = fmaxf(av, mls[1][c]); }
    a = warp_max(a);
    av = warp_max(av);
    const float ref = a > -INFINITY ? a : 0.f, refv = av > -INFINITY ? av : 0.f;
    for (int c = lane; c < n; c += 32) sum += mls[2][c] * fast_exp2(mls[0][c] - ref);
    sum = warp_sum(sum);
    float o[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) o[e] = 0.f;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int c = sub + j * kSplit;
      if (c < n) {
        const float f = fast_exp2(mls[1][c] - refv);
#pragma unroll
        for (int e = 0; e < kVec; ++e) o[e] = fmaf(ahead[j][e], f, o[e]);
      }
    }
#pragma unroll 4
    for (int c = sub + kAhead * kSplit; c < n; c += kSplit) {
      const float f = fast_exp2(mls[1][c] - refv);
#pragma unroll
      for (int e = 0; e < kVec; ++e) o[e] = fmaf(acc[(size_t)c * p.pitch * D + e], f, o[e]);
    }
    const float inv = fast_exp2(refv - ref - kCaTop) / sum;   // sums relative to 2^(refv - kCaTop) over a denominator relative to 2^ref
    if constexpr (kSplit > 1) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) s_acc[warp][lane * kVec + e] = o[e];
      __syncthreads();
      if (sub > 0) return;
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        for (int w = 1; w < kSplit; ++w) o[e] += s_acc[warp + w][lane * kVec + e];
    }
    if (live)
#pragma unroll
      for (int e = 0; e < kVec; ++e) store_out(dst + lane * kVec + e, o[e] * inv);
    return;
  }
  // ---- weights ----
  constexpr int kRowsEach = 4, kRound = kRowsEach * kCaMergeThreads;
  const int row0 = ((int)blockIdx.y - out_blocks) * kChunk, rows = min(held - row0, kChunk);
  if (rows <= 0) return;
  const float* logits = p.logits + ((size_t)bh * p.c.cap + row0) * p.group;
  const size_t at = (size_t)bh * p.c.cap + row0;
  // A row's logits start on 16 bytes: its first eight are read so (32 users, groups of 8 / 16: 50.2 -> 48.1 us, 95.0 -> 88.8).  The rest
  // stay with single words: in fours, 16 take 82.4, but all other groups 1 % more.
  const bool fours = p.group % 4 == 0;
  float add[kRowsEach], first[kRowsEach][8];   // a round's weights, and its logits of the first eight heads
  auto request = [&](int from) {
#pragma unroll
    for (int i = 0; i < kRowsEach; ++i) {
      const int r = from + tid + i * kCaMergeThreads;
      add[i] = r < rows ? p.weights_in[at + r] : 0.f;
      if (fours) {
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
          const float4 v = j < p.group && r < rows ? *reinterpret_cast<const float4*>(logits + (size_t)r * p.group + j) : make_float4(0.f, 0.f, 0.f, 0.f);
          first[i][j] = v.x; first[i][j + 1] = v.y; first[i][j + 2] = v.z; first[i][j + 3] = v.w;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) first[i][j] = j < p.group && r < rows ? logits[(size_t)r * p.group + j] : 0.f;
      }
    }
  };
  request(0);
  for (int h0 = 0; h0 < p.group; h0 += 128) {   // 128 heads at a time; with more, the weights take several passes
    __syncthreads();
    for (int h = h0 + warp; h < min(p.group, h0 + 128); h += kWarps4) {
      const int pass = h / kCaHeads, pair = head * p.passes + pass;
      const int x = below * pairs + pair * units_of(nb) + kCaStart;
      const int c0 = run_of(total, x, grid), n = run_of(total, x + nb - 1, grid) - c0 + 1;
      const float* ml = p.part_ml + (((size_t)b * pairs + pair + c0) * p.pitch + h - pass * kCaHeads) * 3;
      float a = -INFINITY, sum = 0.f;
      for (int c = lane; c < n; c += 32) {   // relative to the lane's own maximum so far
        const float m = ml[(size_t)c * p.pitch * 3], l = ml[(size_t)c * p.pitch * 3 + 2];
        const float top = fmaxf(a, m), ref = top > -INFINITY ? top : 0.f;
        sum = sum * fast_exp2(a - ref) + l * fast_exp2(m - ref);
        a = top;
      }
      const float top = warp_max(a), ref = top > -INFINITY ? top : 0.f;
      sum = warp_sum(sum * fast_exp2(a - ref));
      if (lane == 0) { s_ref[h - h0] = ref; s_inv[h - h0] = 1.f / sum; }
    }
    __syncthreads();
    const int n = min(p.group - h0, 128);
    for (int from = 0; from < rows; from += kRound) {
      if (from > 0 || h0 > 0) request(from);
#pragma unroll
      for (int i = 0; i < kRowsEach; ++i) {
        const int r = from + tid + i * kCaMergeThreads;
        if (r >= rows) continue;
        float sum = 0.f;
        int j = 0;
        if (h0 == 0) {
#pragma unroll
          for (; j < 8; ++j)
            if (j < n) sum += fast_exp2(first[i][j] - s_ref[j]) * s_inv[j];
        }
        for (; j < n; ++j) sum += fast_exp2(logits[(size_t)r * p.group + h0 + j] - s_ref[j]) * s_inv[j];
        p.weights_out[at + r] = (h0 ? p.weights_out[at + r] : add[i]) + sum;
      }
    }
  }
}

}  // namespace

#endif  // ST3_CACHE_ATTEND_CUH_
