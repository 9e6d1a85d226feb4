// Prompts of different lengths packed one behind the other, with grouped heads: causal attention, and the attention weight
// that every token has received.  Both run on the tcgen05 tensor cores with accumulators in tensor memory.
//
// Work items are two tiles of 128 rows that read the same other operand, so that every tile that comes through the ring
// feeds two tiles of MMAs: for the attention 128 queries of two heads of one group (or, where a group has an odd number
// of heads, 256 queries of one head) against key/value tiles of 128 rows; for the weights 256 keys of a key/value
// head against tiles of 128 queries.  A block per SM is persistent: the first item is its block index, the others are block
// indices that it takes from the hardware's queue (cluster launch control), so that items of very different lengths
// spread without a counter in memory and the next item's loads run under the end of this one.  Where the weights have few items,
// a cluster of blocks shares each of them instead.
//
// Items need no table either: sequence s has the numbers cu[s]/R + s and on (R rows an item), which are at least as many as
// the ceil(n/R) that it needs; numbers without an item are passed over.  The weights' items go in two rounds, the longer half of
// each sequence's and then the shorter, so that the queue ends with short ones (16 x 690 tokens, three items of 24, 16 and 8
// steps a head: 85 -> 77 us); the attention's, of which a block does many more, lost 2 % that way.
//
// Roles: four warps (attention) or eight (weights) own a tile each, a row (= tensor memory lane) per thread, in the weights
// with half of the columns; two warps issue the MMAs of one tile each; one takes items, decodes them and issues the TMA loads; in the
// weights one more brings the sums of exponentials.
// Every wait is bounded, and a wait that runs out ends the block's others.
#include "st3_common.cuh"
#include "st3_launch.cuh"
#include "st3_tensor.cuh"

namespace {

// A block of kWarps warps that own rows and a warpgroup of control warps (in the attention one of them idle).  The registers of the launch are
// shared out anew: what the owners of rows get and the control warps keep adds up to them.
template <int kWarps>
struct PkRoles {
  static constexpr int kMma = kWarps, kLoader = kWarps + 2, kThreads = (kWarps + 4) * 32;
  static constexpr int kReaders = kWarps == 16 ? kWarps + 3 : kWarps + 2;   // warps that read items
  static constexpr int kScores = kWarps == 16 ? 2 : 1;                      // arrivals that complete an S
  // In the attention the control warps are the block's first ones, which the schedulers prefer: its MMAs are issued beside warps that
  // always have something to issue (2 % at 12 000 tokens).  The weights lose 5 % that way.
  static __device__ __forceinline__ int warp() {
    const int w = threadIdx.x >> 5;
    return kWarps == 16 ? w : w < 4 ? kWarps + w : w - 4;
  }
  static constexpr int kRegsRows = kWarps == 8 ? 208 : 104, kRegsControl = kWarps == 8 ? 88 : 64;
  static_assert(kWarps == 8 || kWarps == 16, "2 * 208 + 88 = 3 * 168; 4 * 104 + 64 = 5 * 96");
};
using AttendRoles = PkRoles<8>;
using WeightRoles = PkRoles<16>;
constexpr int kPkRows = 128;                 // rows of a tile
constexpr int kBox = kPkRows * 128;          // one TMA box: 128 rows x 64 bf16
constexpr uint32_t kPkTmem = 512;
constexpr int kPkKeys = 64;                  // keys of a step of the attention
constexpr uint32_t kIdescKeys = kIdescBase | ((kPkKeys >> 3) << 17);   // N = 64, both operands K-major
constexpr uint32_t kIdescScores = kIdescBase | ((128u >> 3) << 17);    // N = 128
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// log2(e) / sqrt(D).  The tensor core cuts its running sum toward zero after every 16 dims, which takes 1.9e-7 off a score whose 128
// terms grow it evenly and nothing off one whose sums have few bits: it depends on the inputs, so nothing is given back.
template <int D>
constexpr float kScoreScale = (float)(1.4426950408889634 / (D == 128 ? 11.313708498984761 : 8.0));

struct PackedParams {
  const int* cu;
  void* out;
  float* lse;
  const float* lse_in;
  float* weights;
  int* status;
  long long out_token_stride, out_head_stride;
  int num_seqs, total, heads, kv_heads, group;
  int pairs;       // items of one number: head pairs, or heads where an item is 256 queries of one
  int items;
  int by_heads;    // an item's tiles are two heads (else two runs of 128 queries)
  int wide_out;    // rows of the output start on 32 bytes
  int capacity, window;
};

struct PkItem {
  int stop;
  int row;        // first token of the sequence in the packed tensor
  int len;
  int seq;
  int head[2];    // of the two tiles
  int first[2];   // first row of the two tiles inside the sequence
  int steps[2];   // tiles of the other operand
  int begin;      // weights: first query that counts
};

struct PkShared {
  uint64_t full[8], empty[8];           // ring of the other operand
  uint64_t own[2], own_free[2];         // the item's own two tiles (weights: two buffers of them)
  uint64_t scores[4];                   // S is complete (two buffers a tile)
  uint64_t taken[4];                    // attention: P is in tensor memory; weights: S has been read
  uint64_t added[2], done[2];           // attention: a P V, and the last one of an item, is complete
  uint64_t ready[2], read[2];           // items
  uint64_t lse_free[2];                 // weights: a step's lse has been read
  uint64_t next;                        // answer of the queue
  uint4 answer;
  PkItem item[2];
  uint32_t tmem;
  int fail;
};

// kBuffers: of an item's own tiles.  Two in the weights, whose items can be as short as one step a head: the next one's keys come
// while this one's are used.  The attention's own tiles come while its outputs are written.
template <int D, int kBuffers>
struct PkLayout {
  static constexpr int kBoxes = D / 64;
  static constexpr int kTile = kBoxes * kBox;
  static constexpr int kStages = D == 128 ? 7 - 2 * kBuffers : 8;
  static constexpr int kRing = 2 * kBuffers * kTile;
  static constexpr int kShared = kRing + kStages * kTile;
  static constexpr int kSums = kShared + 512;  // weights: of a tile's second half of columns, and the lse of two steps
  static constexpr int kLse = kSums + 2 * kPkRows * 4;
  static constexpr int kTotal = kBuffers == 2 ? kLse + 2 * kPkRows * 4 : kSums;
};
static_assert(sizeof(PkShared) <= 512, "PkShared must fit its slot");
static_assert(PkLayout<128, 2>::kTotal <= 227 * 1024 && PkLayout<128, 1>::kTotal <= 227 * 1024, "shared memory");

// Bounded wait that also ends when another role of the block has given up.
__device__ __forceinline__ bool pk_wait(uint64_t* bar, uint32_t parity, volatile int* fail) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity))
    if (*fail || clock64() - t0 > kWaitCycles) return false;
  return true;
}
__device__ __forceinline__ bool pk_wait_warp(uint64_t* bar, uint32_t parity, volatile int* fail) {
  return __all_sync(0xffffffffu, pk_wait(bar, parity, fail));
}

__device__ __forceinline__ void mbar_arrive_count(uint64_t* bar, uint32_t count) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}

__device__ __forceinline__ void take_next(void* answer, uint64_t* bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(answer)),
               "r"(smem_u32(bar))
               : "memory");
}
// The block index that was taken, or -1 when the queue is empty.
__device__ __forceinline__ int taken_index(const void* answer) {
  uint32_t got, x;
  asm volatile(
      "{\n\t.reg .b128 r;\n\t.reg .pred p;\n\t.reg .b32 y, z, w;\n\t"
      "ld.shared.b128 r, [%2];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "mov.u32 %1, 0;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, y, z, w}, r;\n\t}"
      : "=r"(got), "=r"(x)
      : "r"(smem_u32(answer))
      : "memory");
  return got ? (int)x : -1;
}

template <int kBoxes>
__device__ __forceinline__ void load_tile(unsigned char* dst, const CUtensorMap* map, int head, int row, uint64_t* bar) {
#pragma unroll
  for (int x = 0; x < kBoxes; ++x) tma_load_3d(dst + x * kBox, map, x * 64, head, row, bar);
}

// The sequence of number `slot` (`rows` tokens a number): how many sequences start at or below it, less one.  A whole warp.
__device__ __forceinline__ int seq_of(const int* cu, int num_seqs, int rows, int slot) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = num_seqs;
  while (n > 0) {   // sequences lo .. lo + n - 1 are left to look at
    const int step = (n + 31) / 32, b = lo + lane * step;
    const bool below = b < lo + n && cu[b] / rows + b <= slot;
    const int c = __popc(__ballot_sync(0xffffffffu, below));
    if (c == 0) break;
    const int base = lo + (c - 1) * step;
    if (step == 1) { lo = base; break; }
    n = min(step, lo + n - base);
    lo = base;
  }
  return lo;
}

// Where sequence b lies; false (and reported) if cu is not ascending inside [0, total].
__device__ __forceinline__ bool seq_rows(const PackedParams& p, int b, int& row, int& len) {
  row = p.cu[b];
  len = p.cu[b + 1] - row;
  const bool ok = row >= 0 && len >= 0 && row <= p.total - len;
  if (!ok && p.status && (threadIdx.x & 31) == 0) atomicOr(p.status, ST3_DEV_RANGE);
  return ok;
}

// Reports offsets that are not what they should be, as items alone do not see all of them: a sequence that ends ahead of its start
// may have no number.  The `threads` owners of rows do it in every block, ahead of their first item.  (Inside the branch of a role
// the attention's loops came out 1.5 % slower.)
__device__ __forceinline__ void check_offsets(const PackedParams& p, int thread, int threads) {
#pragma unroll 1
  for (int b = thread; b < p.num_seqs; b += threads) {
    const int from = p.cu[b], to = p.cu[b + 1];
    if ((from < 0 || to < from || to > p.total) && p.status) atomicOr(p.status, ST3_DEV_RANGE);
  }
  __syncwarp();
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// The barriers, the tensor memory and the start of a block; false if its shared memory is not where it must be.
template <int kStages, typename Roles>
__device__ __forceinline__ bool pk_begin(unsigned char* smem, PkShared& sh, int* status) {
  if (smem_u32(smem) & 1023u) {   // the swizzle assumes aligned tiles: reported, not used
    if (threadIdx.x == 0 && status) atomicOr(status, ST3_DEV_RANGE);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    return false;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 2); }
    for (int i = 0; i < 2; ++i) { mbar_init(&sh.own[i], 1); mbar_init(&sh.own_free[i], 2); }
    for (int i = 0; i < 4; ++i) { mbar_init(&sh.scores[i], Roles::kScores); mbar_init(&sh.taken[i], Roles::kMma / 2); }
    for (int i = 0; i < 2; ++i) mbar_init(&sh.lse_free[i], Roles::kMma);
    for (int i = 0; i < 2; ++i) { mbar_init(&sh.added[i], 1); mbar_init(&sh.done[i], 1); mbar_init(&sh.ready[i], 1); mbar_init(&sh.read[i], Roles::kReaders); }
    mbar_init(&sh.next, 1);
    sh.fail = 0;
    mbar_fence_init();
  }
  __syncthreads();
  if (Roles::warp() == Roles::kMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(kPkTmem) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  return true;
}
template <typename Roles>
__device__ __forceinline__ void pk_end(PkShared& sh, uint32_t tmem) {
  tc_fence_before();
  __syncthreads();
  if (Roles::warp() == Roles::kMma)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kPkTmem) : "memory");
}

// Inside the branch of each role: behind a join of the two the compiler would hold everything to the smaller number.
template <typename Roles>
__device__ __forceinline__ void pk_more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Roles::kRegsRows)); }
template <typename Roles>
__device__ __forceinline__ void pk_fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Roles::kRegsControl)); }

// Waits for the next item, sh.item[slot]; false when there is none left, or a wait ran out (then `fail` is set).
__device__ __forceinline__ bool pk_next(PkShared& sh, int slot, uint32_t phase) {
  if (!pk_wait_warp(&sh.ready[slot], phase, &sh.fail)) { *(volatile int*)&sh.fail = 1; return false; }
  return !*(volatile int*)&sh.item[slot].stop;
}
__device__ __forceinline__ void pk_release(PkShared& sh, int& slot, uint32_t& phase) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive_cta(&sh.read[slot]);
  if (++slot == 2) { slot = 0; phase ^= 1; }
}
// The same with a copy of the item.
__device__ __forceinline__ bool pk_item(PkShared& sh, int& slot, uint32_t& phase, PkItem& it) {
  const bool more = pk_next(sh, slot, phase);
  if (more) {
    it = sh.item[slot];
    pk_release(sh, slot, phase);
  }
  return more;
}

// The MMA warp's end where a wait has run out: what it has issued (a microsecond's work) ends before tensor memory is given
// back.
__device__ __forceinline__ void pk_give_up(PkShared& sh, int* status) {
  *(volatile int*)&sh.fail = 1;
  if ((threadIdx.x & 31) == 0 && status) atomicOr(status, ST3_DEV_COPY_TIMEOUT);
  const long long t0 = clock64();
  while (clock64() - t0 < 2000000) {}
  __syncwarp();
}

// A barrier of the eight warps of a tile of the weights that tells each of them whether any has failed.
__device__ __forceinline__ bool pk_any_failed(int tile, bool failed) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, 256, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"((uint32_t)failed), "r"(1 + tile)
      : "memory");
  return any != 0;
}

// The loader's loop over items, the same for both kernels: `decode(index, item)` fills an item (false: nothing to do) and
// `load(item)` brings its tiles.
// With kOne the block has item `index` and no other.
template <bool kOne, typename Decode, typename Load>
__device__ __forceinline__ void pk_loader(PkShared& sh, int* status, int index, Decode&& decode, Load&& load) {
  const int lane = threadIdx.x & 31;
  int slot = 0;
  uint32_t phase = 1, answer = 0;
  bool ok = true;
  while (true) {
    PkItem it;
    if (decode(index, it)) {
      ok = pk_wait_warp(&sh.read[slot], phase, &sh.fail);
      if (ok) {
        if (lane == 0) { it.stop = 0; sh.item[slot] = it; mbar_arrive_cta(&sh.ready[slot]); }
        __syncwarp();
        if (++slot == 2) { slot = 0; phase ^= 1; }
        ok = load(it);
      }
      if (!ok) break;
    }
    if (kOne) break;
    // The next item is taken when this one's last tiles have been requested, which is a few steps ahead of their use: taken any
    // earlier, it would stay with this block while others run out of work (weights of 16 x 690 tokens: 98 -> 85 us).
    if (lane == 0) {
      mbar_expect_tx(&sh.next, 16);
      take_next(&sh.answer, &sh.next);
    }
    // the answer is waited for also where the block gives up: it is written into this block's shared memory
    if (!pk_wait_warp(&sh.next, answer, &sh.fail) && !pf_wait_warp(&sh.next, answer)) { ok = false; break; }
    answer ^= 1;
    index = taken_index(&sh.answer);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // read before the next answer may be written
    __syncwarp();
    if (index < 0) break;
  }
  if (ok) ok = pk_wait_warp(&sh.read[slot], phase, &sh.fail);
  if (lane == 0) {
    if (!ok) {
      *(volatile int*)&sh.fail = 1;
      if (status) atomicOr(status, ST3_DEV_COPY_TIMEOUT);
    }
    sh.item[slot].stop = 1;
    mbar_arrive_cta(&sh.ready[slot]);
  }
  __syncwarp();
}

// The same value in every lane, for the compiler to know.
template <typename T>
__device__ __forceinline__ T uniform(T x) { return __shfl_sync(0xffffffffu, x, 0); }

// A ring's place: stage and parity of its next use.
template <int kStages>
struct Ring {
  int stage = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void step() { if (++stage == kStages) { stage = 0; phase ^= 1; } }
};

// Copies still in flight when the loader leaves: the last use of every stage, and of the buffers of an item's own tiles.
template <int kStages, int kBuffers>
__device__ __forceinline__ void pk_settle(PkShared& sh, int issued, int owned) {
  for (int u = max(0, issued - kStages); u < issued; ++u) pf_wait(&sh.full[u % kStages], (u / kStages) & 1);
  for (int u = max(0, owned - kBuffers); u < owned; ++u) pf_wait(&sh.own[u % kBuffers], (u / kBuffers) & 1);
}

// ------------------------------------------------------------------------------------------------------------------
// Causal attention, in steps of 64 keys, two to a tile that comes through the ring.
//   S = Q K^T (128 x 64, D/16 MMAs of K = 16), P = exp2(S - ref) as bf16 over the first half of its S, O += P V.
// The tensor pipe runs S(0) S(1) | PV(0) S(2) | PV(1) S(3) | ... for each tile, so that the softmax of a step runs under the products
// of the one before it and of the other tile.  `ref` follows a row's maximum only when that has grown by 2^8: bf16 and
// fp32 lose no bits by it, O is hardly ever rescaled (as rarely as at 2^64, which values beyond 2^63 would make infinite), and
// values that add up to less than 2^119 over a sequence stay finite.
// What bounds it at long prompts: the MMAs, of which a 128x128x16 takes 64 cycles but a 128x64x16 49, as long as its operands take to
// read from shared memory: 2 600 cycles for both tiles and 128 keys at D = 128, of 3 200 measured (12 000 and 3 043 tokens, 32 heads
// of 128: 1.00 ms, 1 250 TFLOP/s, in the first 20 ms; 1.17 ms, 1 070 TFLOP/s, in a loop, where the power cap takes the clock to
// 1 507 MHz).  Scores of 128 keys would cost 64 cycles an MMA but leave tensor memory no second buffer: a tile's softmax and
// products then form one chain (3 850 cycles).  At short ones (16 prompts of 690 tokens: 101 us, 117 in a loop at 1 597 MHz) it is
// the start and the end of an item, some 6 000 cycles of its 17 000.
// ------------------------------------------------------------------------------------------------------------------
// exp2(s * sc - ref) of a step's columns, as bf16 pairs in w and added up in `add`.  Whole steps take every fourth pair on the
// FMA pipe; where columns are masked (-Inf, which have to give 0) the special-function unit does them all.  A score of NaN, or of
// +Inf, makes the row's sum NaN.
template <bool kWhole>
__device__ __forceinline__ void probs(const uint32_t (&v)[64], float sc, float ref, u64 (&add)[2], uint32_t (&w)[32]) {
  const float nrf = ref > -INFINITY ? -ref : 0.f;
  const u64 sc2 = pack2(sc, sc), nrf2 = pack2(nrf, nrf);
#pragma unroll
  for (int c = 0; c < 32; ++c) {
    const u64 t = mul_add2(pack2(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1])), sc2, nrf2);
    float pa, pb;
    if (kWhole && c % 4 == 2) {
      poly_exp2<4>(t, pa, pb);
    } else {
      split2(t, pa, pb);
      pa = fast_exp2(pa);
      pb = fast_exp2(pb);
    }
    add[c & 1] = add2(add[c & 1], pack2(pa, pb));
    w[c] = bf16_pair(pa, pb);
  }
}

template <int D>
__global__ void __launch_bounds__(AttendRoles::kThreads, 1)
st3_packed_attend_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                         const __grid_constant__ CUtensorMap map_v, const PackedParams p) {
  using L = PkLayout<D, 1>;
  extern __shared__ __align__(1024) unsigned char smem[];
  PkShared& sh = *reinterpret_cast<PkShared*>(smem + L::kShared);
  if (threadIdx.x == 0) { prefetch_map(&map_q); prefetch_map(&map_k); prefetch_map(&map_v); }
  if (!pk_begin<L::kStages, AttendRoles>(smem, sh, p.status)) return;
  const uint32_t tmem = sh.tmem;
  const int lane = threadIdx.x & 31, warp = AttendRoles::warp();
  volatile int* fail = &sh.fail;
  const int rows = p.by_heads ? kPkRows : 2 * kPkRows;
  if (warp < AttendRoles::kMma) check_offsets(p, warp * 32 + lane, AttendRoles::kMma * 32);
  if (warp >= AttendRoles::kMma) pk_fewer_registers<AttendRoles>();
  if (warp > AttendRoles::kLoader) {
    // idle
  } else if (warp == AttendRoles::kLoader) {
    // ===================== loader =====================
    Ring<L::kStages> ring;
    int issued = 0, owned = 0;
    pk_loader<false>(
        sh, p.status, blockIdx.x,
        [&](int index, PkItem& it) {
          const int number = index / p.pairs, pair = index - number * p.pairs;
          const int slot = p.items / p.pairs - 1 - number;    // a sequence's last rows, the longest items, first
          const int b = seq_of(p.cu, p.num_seqs, rows, slot);
          if (!seq_rows(p, b, it.row, it.len)) return false;
          const int rank = slot - (p.cu[b] / rows + b);
          if (rank < 0 || rank >= (it.len + rows - 1) / rows) return false;
          it.seq = b;
          it.head[0] = p.by_heads ? 2 * pair : pair;
          it.head[1] = p.by_heads ? 2 * pair + 1 : pair;
          it.first[0] = rank * rows;
          it.first[1] = it.first[0] + rows - kPkRows;
#pragma unroll
          for (int x = 0; x < 2; ++x) it.steps[x] = it.first[x] < it.len ? it.first[x] / kPkRows + 1 : 0;
          it.begin = 0;
          return true;
        },
        [&](const PkItem& it) {
          bool ok = pk_wait_warp(&sh.own_free[0], (owned & 1) ^ 1, fail);
          if (!ok) return false;
          if (lane == 0) {
            mbar_expect_tx(&sh.own[0], 2 * L::kTile);
#pragma unroll
            for (int x = 0; x < 2; ++x) load_tile<L::kBoxes>(smem + x * L::kTile, &map_q, it.head[x], it.row + it.first[x], &sh.own[0]);
          }
          ++owned;
          const int n = max(it.steps[0], it.steps[1]), kv = it.head[0] / p.group;
          for (int j = 0; j < 2 * n && ok; ++j) {   // K(0) V(0) K(1) V(1) ...
            ok = pk_wait_warp(&sh.empty[ring.stage], ring.phase ^ 1, fail);
            if (!ok) break;
            if (lane == 0) {
              mbar_expect_tx(&sh.full[ring.stage], L::kTile);
              load_tile<L::kBoxes>(smem + L::kRing + ring.stage * L::kTile, j & 1 ? &map_v : &map_k, kv, it.row + (j >> 1) * kPkRows, &sh.full[ring.stage]);
            }
            __syncwarp();
            ++issued;
            ring.step();
          }
          return ok;
        });
    if (lane == 0) pk_settle<L::kStages, 1>(sh, issued, owned);
    __syncwarp();
  } else if (warp >= AttendRoles::kMma) {
    // ===================== MMA: a warp for each tile =====================
    constexpr uint32_t kIdescOut = kIdescBase | (((uint32_t)D >> 3) << 17) | (1u << 16);   // N = D, V MN-major
    const int x = warp - AttendRoles::kMma;
    const uint32_t own_lo = uniform(desc_lo(smem_u32(smem + x * L::kTile), 16)), ring_lo = uniform(desc_lo(smem_u32(smem + L::kRing), 16));
    const uint32_t v_lo = uniform(desc_lo(smem_u32(smem + L::kRing), kBox));
    const uint32_t tS = uniform(tmem + x * 128), tO = uniform(tmem + 256 + x * 128);
    Ring<L::kStages> ring;
    int slot = 0;
    uint32_t phase = 0, own = 0, use = 0;   // use: steps so far, two to a tile of keys
    PkItem it;
    bool ok = true;
    while (ok && pk_item(sh, slot, phase, it)) {
      const int mine = uniform(2 * (x ? it.steps[1] : it.steps[0])), n = uniform(max(it.steps[0], it.steps[1])), len = uniform(it.len);
      ok = pk_wait_warp(&sh.own[0], own, fail);
      own ^= 1;
      // S = Q K^T of the two steps of a tile of keys at the ring's place, which is then left
      Ring<L::kStages> k;
      auto scores = [&](int t) {
        if (t < mine) {
          if (elected()) {
            const uint32_t k_lo = ring_lo + ((uint32_t)k.stage * L::kTile + (t & 1) * (kPkKeys * 128) >> 4);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
              const uint32_t off = ((ks >> 2) * kBox + (ks & 3) * 32) >> 4;
              umma_bf16(tS + (t & 1) * kPkKeys, own_lo + off, k_lo + off, kIdescKeys, ks > 0);
            }
            umma_commit(&sh.scores[2 * x + (t & 1)]);
          }
          __syncwarp();
        }
        if (t & 1) {
          if (elected()) {
            umma_commit(&sh.empty[k.stage]);
            if (t == 2 * n - 1) umma_commit(&sh.own_free[0]);
          }
          __syncwarp();
        }
      };
      k = ring;
      ring.step();
      if (ok) ok = pk_wait_warp(&sh.full[k.stage], k.phase, fail);
      if (!ok) break;
      tc_fence_after();
      scores(0);
      scores(1);
      for (int j = 0; j < n && ok; ++j) {
        const Ring<L::kStages> v = ring;
        ring.step();
        k = ring;                          // K(j + 1)
        if (j + 1 < n) ring.step();
        ok = pk_wait_warp(&sh.full[v.stage], v.phase, fail);
        if (!ok) break;
        // Rows of V behind the sequence belong to others: their probability is 0, but 0 times Inf or NaN is not.  Both warps
        // clear them, each before its own product.
        const int valid = len - j * kPkRows;
        if (valid < kPkRows) {
          unsigned char* tile = smem + L::kRing + v.stage * L::kTile;
          for (int i = valid * 8 + lane; i < kPkRows * 8; i += 32)
#pragma unroll
            for (int y = 0; y < L::kBoxes; ++y) *reinterpret_cast<uint4*>(tile + y * kBox + i * 16) = make_uint4(0, 0, 0, 0);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int t = 2 * j + h;
          if (t < mine) {
            ok = pk_wait_warp(&sh.taken[2 * x + h], (use >> 1) & 1, fail);
            ++use;
            if (!ok) break;
            tc_fence_after();
            if (elected()) {
              const uint32_t vb = v_lo + ((uint32_t)v.stage * L::kTile + h * (kPkKeys * 128) >> 4);
#pragma unroll
              for (int ks = 0; ks < kPkKeys / 16; ++ks)
                umma_bf16_ta(tO, tS + h * kPkKeys + ks * 8, vb + ks * (2048 >> 4), kIdescOut, (t > 0 || ks > 0));
              umma_commit(&sh.added[x]);
              if (t == mine - 1) umma_commit(&sh.done[x]);
            }
            __syncwarp();
          }
          if (h == 1) {
            if (elected()) umma_commit(&sh.empty[v.stage]);
            __syncwarp();
          }
          if (j + 1 < n) {
            if (h == 0) {
              ok = pk_wait_warp(&sh.full[k.stage], k.phase, fail);
              if (!ok) break;
              tc_fence_after();
            }
            scores(t + 2);
          }
        }
      }
    }
    if (!ok || *fail) pk_give_up(sh, p.status);
  } else {
    // ===================== softmax: thread <-> query row =====================
    pk_more_registers<AttendRoles>();
    const int x = warp >> 2, w32 = (warp & 3) * 32, r = w32 + lane;
    const uint32_t lane_addr = (uint32_t)w32 << 16;
    const uint32_t tS = tmem + x * 128 + lane_addr, tO = tmem + 256 + x * 128 + lane_addr;
    constexpr float sc = kScoreScale<D>;
    int slot = 0;
    uint32_t phase = 0, use = 0, d_phase = 0;   // use: steps so far
    bool ok = true;
    while (ok && pk_next(sh, slot, phase)) {
      const PkItem& it = sh.item[slot];
      const int n = 2 * it.steps[x];
      if (n == 0) { pk_release(sh, slot, phase); continue; }
      float ref = -INFINITY, l = 0.f;
      for (int t = 0; t < n; ++t, ++use) {
        const int h = t & 1;
        ok = pk_wait_warp(&sh.scores[2 * x + h], (use >> 1) & 1, fail);
        if (!ok) break;
        tc_fence_after();
        const uint32_t tH = tS + h * kPkKeys;
        const int seen = t >= n - 2 ? r - h * kPkKeys : kPkKeys;   // columns up to this one are seen by this row
        uint32_t w[32];
        if (t >= n - 2 && w32 + 31 < h * kPkKeys) {   // none of this warp's rows sees any of them
#pragma unroll
          for (int c = 0; c < 32; ++c) w[c] = 0u;
        } else {
          uint32_t v[64];
          tmem_ld64(tH, v);
          if (t >= n - 2) {
#pragma unroll
            for (int c = 0; c < 64; ++c)
              if (c > seen) v[c] = 0xff800000u;
          }
          float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int c = 0; c < 64; c += 8)
#pragma unroll
            for (int e = 0; e < 4; ++e) m4[e] = fmax3(m4[e], __uint_as_float(v[c + e]), __uint_as_float(v[c + 4 + e]));
          const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * sc;
          const bool away = mx > ref + 8.f || (ref == -INFINITY && mx > ref);
          if (__any_sync(0xffffffffu, away)) {
            const float factor = away ? fast_exp2(ref - mx) : 1.f;   // 0 for the first step
            if (away) ref = mx;
            l = sum_or_nan(l) * factor;   // here and at the end: a sum only grows otherwise
            if (t > 0) {
              // The P V of the step before must be complete.  Waiting for its parity is enough although this thread has not
              // watched every phase: S is complete, hence the P V issued before it, of two steps ago; and this step's cannot
              // be issued before the arrival below.
              ok = pk_wait_warp(&sh.added[x], (use - 1) & 1, fail);
              if (!ok) break;
              tc_fence_after();
#pragma unroll 1
              for (int cb = 0; cb < D / 32; ++cb) {
                uint32_t o[32];
                tmem_ld32(tO + cb * 32, o);
#pragma unroll
                for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * factor);
                tmem_st32(tO + cb * 32, o);
              }
            }
          }
          u64 add[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
          if (t < n - 2) probs<true>(v, sc, ref, add, w);
          else probs<false>(v, sc, ref, add, w);
          l += sum2(add2(add[0], add[1]));
        }
        tmem_st32(tH, w);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cta(&sh.taken[2 * x + h]);
      }
      if (!ok) break;
      ok = pk_wait_warp(&sh.done[x], d_phase, fail);
      d_phase ^= 1;
      if (!ok) break;
      tc_fence_after();
      const int qi = it.first[x] + r, head = it.head[x], row = it.row + qi;
      const bool live = qi < it.len;
      pk_release(sh, slot, phase);
      l = sum_or_nan(l);
      const float inv = ref > -INFINITY ? 1.f / l : NAN;   // NaN where every score is -Inf, and where the sum is NaN
      if (live && p.lse) p.lse[(size_t)head * p.total + row] = ref * kLn2 + logf(l);
      __nv_bfloat16* orow = static_cast<__nv_bfloat16*>(p.out) + (long long)row * p.out_token_stride + (long long)head * p.out_head_stride;
#pragma unroll 1
      for (int cb = 0; cb < D / 32; ++cb) {
        uint32_t o[32];
        tmem_ld32(tO + cb * 32, o);
        if (live) {
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) w[e] = bf16_pair(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv);
          if (p.wide_out) {
#pragma unroll
            for (int e = 0; e < 16; e += 8)
              asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(orow + cb * 32 + 2 * e), "r"(w[e]),
                           "r"(w[e + 1]), "r"(w[e + 2]), "r"(w[e + 3]), "r"(w[e + 4]), "r"(w[e + 5]), "r"(w[e + 6]), "r"(w[e + 7])
                           : "memory");
          } else {
#pragma unroll
            for (int e = 0; e < 16; e += 4) *reinterpret_cast<uint4*>(orow + cb * 32 + 2 * e) = make_uint4(w[e], w[e + 1], w[e + 2], w[e + 3]);
          }
        }
      }
      tc_fence_before();
      __syncwarp();
    }
    if (!ok) *fail = 1;
  }
  pk_end<AttendRoles>(sh, tmem);
}

// ------------------------------------------------------------------------------------------------------------------
// What each token has received: w_j = sum over heads of the group and queries i >= j of exp2(S_ij - lse_i).
//   S^T = K Q^T with the keys as rows: a thread owns a key and adds up its row, so nothing is exchanged and no sum's order
// changes.  Tensor memory holds two S^T for each of the two key tiles; a product runs while the one before it is read.
// Queries that do not count (before the window, behind the sequence) are left out of the sums.
// What bounds it: the exponentials, of which the special-function unit does 16 a clock and the FMA pipe takes a quarter (1 540 cycles
// for both tiles and 128 queries), beside the products, sums and lse that go with them (1 300 without the exponentials), of 2 350
// measured at 12 000 tokens (0.70 ms, in a loop at 1 785 MHz 0.77; 67 and 70 us for 16 prompts of 690); the MMAs take 1 030.  The lse
// comes by a warp of its own: with barriers between the warps that read it these stayed in step with each other (0.79 ms, 77 us).
// ------------------------------------------------------------------------------------------------------------------
// Adds exp2(s * sc - lse) of 32 queries; kSome: of those in [lo, hi) only, whatever the others are.
template <bool kSome>
__device__ __forceinline__ void add_weights(const uint32_t (&v)[64], int part, const float* s_lse, float sc, int lo, int hi, u64 (&acc)[4]) {
  const u64 sc2 = pack2(sc, sc);
#pragma unroll
  for (int c = 0; c < 32; c += 4) {
    const float4 z = *reinterpret_cast<const float4*>(s_lse + c);
    const int at = part * 32 + c;
    const u64 a = mul_add2(pack2(__uint_as_float(v[at]), __uint_as_float(v[at + 1])), sc2, pack2(z.x, z.y));
    const u64 b = mul_add2(pack2(__uint_as_float(v[at + 2]), __uint_as_float(v[at + 3])), sc2, pack2(z.z, z.w));
    float e[4];
    split2(a, e[0], e[1]);
    e[0] = fast_exp2(e[0]);
    e[1] = fast_exp2(e[1]);
    if (c >= 16) {   // a quarter of the exponentials on the FMA pipe, together (spread out: 2 % slower at 12 000 tokens)
      poly_exp2<5>(b, e[2], e[3]);
    } else {
      split2(b, e[2], e[3]);
      e[2] = fast_exp2(e[2]);
      e[3] = fast_exp2(e[3]);
    }
    if (kSome) {
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i] = c + i >= lo && c + i < hi ? e[i] : 0.f;
    }
    acc[(c >> 1) & 3] = add2(acc[(c >> 1) & 3], pack2(e[0], e[1]));
    acc[((c >> 1) & 3) + 1] = add2(acc[((c >> 1) & 3) + 1], pack2(e[2], e[3]));
  }
}

// The (query tile, head) pairs that a block of a cluster takes part in, from query tile t0 on: every `ranks`-th one, ranks a power
// of two.
struct WeightSteps {
  int t, g;
  const int group, ranks;
  __device__ __forceinline__ WeightSteps(int t0, int group_, int rank, int ranks_) : t(t0), g((rank - t0 * group_) & (ranks_ - 1)), group(group_), ranks(ranks_) { carry(); }
  __device__ __forceinline__ void carry() { while (g >= group) { g -= group; ++t; } }
  __device__ __forceinline__ void next() { g += ranks; carry(); }
};

__device__ __forceinline__ int cluster_rank() { int r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ int cluster_ranks() { int r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <typename T>
__device__ __forceinline__ T peer_value(const T* mine, int rank) {
  static_assert(sizeof(T) == 4, "one word");
  uint32_t at, x;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(mine)), "r"(rank));
  asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  T value;
  memcpy(&value, &x, 4);
  return value;
}

// kSplit: an item belongs to the blocks of a cluster, which share out its steps and have no other item.  The sums are
// joined, in the order of the blocks, through the first one's reads of the others' shared memory.
template <int D, bool kSplit>
__global__ void __launch_bounds__(WeightRoles::kThreads, 1)
st3_packed_weights_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const PackedParams p) {
  using L = PkLayout<D, 2>;
  extern __shared__ __align__(1024) unsigned char smem[];
  PkShared& sh = *reinterpret_cast<PkShared*>(smem + L::kShared);
  if (threadIdx.x == 0) { prefetch_map(&map_q); prefetch_map(&map_k); }
  if (!pk_begin<L::kStages, WeightRoles>(smem, sh, p.status)) return;
  const uint32_t tmem = sh.tmem;
  const int lane = threadIdx.x & 31, warp = WeightRoles::warp();
  volatile int* fail = &sh.fail;
  const int rows = 2 * kPkRows;
  const int ranks = kSplit ? cluster_ranks() : 1, rank = kSplit ? cluster_rank() : 0;
  float* s_sums = reinterpret_cast<float*>(smem + L::kSums);
  float* s_lse = reinterpret_cast<float*>(smem + L::kLse);

  // Query tiles start at the first query that counts.  steps[x] is the first of them that key tile x takes part in, and
  // `begin` the number of them in all.
  if (warp < WeightRoles::kMma) check_offsets(p, warp * 32 + lane, WeightRoles::kMma * 32);
  if (warp >= WeightRoles::kMma) pk_fewer_registers<WeightRoles>();
  if (warp > WeightRoles::kLoader) {
    // Brings the lse of each step's queries, the same for both tiles: an S^T is complete for its readers once they are there, too.
    // Two steps ahead of them at most, like the products: an arrival at an S^T's barrier must not meet the use before.
    int slot = 0, at = 0;
    uint32_t phase = 0, free = 1, use[2] = {0, 0};
    PkItem it;
    bool ok = true;
    while (ok && pk_item(sh, slot, phase, it)) {
      const int tiles = (it.len - it.begin + kPkRows - 1) / kPkRows;
      const float* lse = p.lse_in + (size_t)it.head[0] * p.group * p.total + it.row;
      WeightSteps s(it.steps[0], p.group, rank, ranks);
      float next[4];
      auto request = [&] {   // a step ahead; what it brings for queries past the end is not used
#pragma unroll
        for (int j = 0; j < 4; ++j) next[j] = lse[(size_t)s.g * p.total + min(it.begin + s.t * kPkRows + 32 * j + lane, it.len - 1)];
      };
      request();
      while (s.t < tiles) {
        ok = pk_wait_warp(&sh.lse_free[at], free, fail);
        if (!ok) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) s_lse[at * kPkRows + 32 * j + lane] = -kLog2e * next[j];
        __syncwarp();
        const bool both = s.t >= it.steps[1];
        if (lane == 0) {
          mbar_arrive_cta(&sh.scores[use[0] & 1]);
          if (both) mbar_arrive_cta(&sh.scores[2 + (use[1] & 1)]);
          else mbar_arrive_count(&sh.lse_free[at], 8);   // for the warps of the tile that does not take part
        }
        __syncwarp();
        ++use[0];
        use[1] += both;
        at ^= 1;
        free ^= at == 0;
        s.next();
        request();
      }
    }
    if (!ok) *fail = 1;
  } else if (warp == WeightRoles::kLoader) {
    Ring<L::kStages> ring;
    int issued = 0, owned = 0;
    pk_loader<kSplit>(
        sh, p.status, blockIdx.x / ranks,
        [&](int index, PkItem& it) {
          const int number = index / p.kv_heads, head = index - number * p.kv_heads, half = p.items / p.kv_heads / 2;
          const bool second = number >= half;
          const int slot = second ? number - half : number;   // a sequence's first keys, the longest items, first
          const int b = seq_of(p.cu, p.num_seqs, 2 * rows, slot);
          if (!seq_rows(p, b, it.row, it.len)) return false;
          if (it.len > p.capacity) {
            if (p.status && lane == 0) atomicOr(p.status, ST3_DEV_RANGE);
            return false;
          }
          const int n = (it.len + rows - 1) / rows, longer = (n + 1) / 2, place = slot - (p.cu[b] / (2 * rows) + b);
          if (place < 0 || place >= (second ? n - longer : longer)) return false;
          const int tile = second ? longer + place : place;
          it.seq = b;
          it.begin = p.window > 0 ? max(0, it.len - p.window) : 0;
          const int tiles = (it.len - it.begin + kPkRows - 1) / kPkRows;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            it.head[x] = head;
            it.first[x] = tile * rows + x * kPkRows;
            it.steps[x] = it.first[x] < it.len ? max(0, it.first[x] - it.begin) / kPkRows : tiles;
          }
          return true;
        },
        [&](const PkItem& it) {
          const int buf = owned & 1;
          bool ok = pk_wait_warp(&sh.own_free[buf], ((owned >> 1) & 1) ^ 1, fail);
          if (!ok) return false;
          if (lane == 0) {
            mbar_expect_tx(&sh.own[buf], 2 * L::kTile);
#pragma unroll
            for (int x = 0; x < 2; ++x) load_tile<L::kBoxes>(smem + (2 * buf + x) * L::kTile, &map_k, it.head[x], it.row + it.first[x], &sh.own[buf]);
          }
          ++owned;
          const int tiles = (it.len - it.begin + kPkRows - 1) / kPkRows;
          for (WeightSteps s(it.steps[0], p.group, rank, ranks); s.t < tiles; s.next()) {
            ok = pk_wait_warp(&sh.empty[ring.stage], ring.phase ^ 1, fail);
            if (!ok) break;
            if (lane == 0) {
              mbar_expect_tx(&sh.full[ring.stage], L::kTile);
              load_tile<L::kBoxes>(smem + L::kRing + ring.stage * L::kTile, &map_q, it.head[0] * p.group + s.g, it.row + it.begin + s.t * kPkRows, &sh.full[ring.stage]);
            }
            __syncwarp();
            ++issued;
            ring.step();
          }
          return ok;
        });
    if (lane == 0) pk_settle<L::kStages, 2>(sh, issued, owned);
    __syncwarp();
  } else if (warp >= WeightRoles::kMma) {
    const int x = warp - WeightRoles::kMma;   // a warp for each tile
    const uint32_t own_lo = uniform(desc_lo(smem_u32(smem + x * L::kTile), 16)), ring_lo = uniform(desc_lo(smem_u32(smem + L::kRing), 16));
    Ring<L::kStages> ring;
    int slot = 0;
    uint32_t phase = 0, owned = 0, use = 0;   // owned: items so far; use: S^T buffers used so far
    PkItem it;
    bool ok = true;
    while (ok && pk_item(sh, slot, phase, it)) {
      const int tiles = uniform((it.len - it.begin + kPkRows - 1) / kPkRows), mine = uniform(x ? it.steps[1] : it.steps[0]);
      const uint32_t own_buf = owned & 1, mine_lo = uniform(own_lo + own_buf * (2 * L::kTile >> 4));
      ok = pk_wait_warp(&sh.own[own_buf], (owned >> 1) & 1, fail);
      ++owned;
      for (WeightSteps s(uniform(it.steps[0]), p.group, rank, ranks); s.t < tiles && ok; s.next()) {
        ok = pk_wait_warp(&sh.full[ring.stage], ring.phase, fail);
        if (!ok) break;
        const bool works = s.t >= mine;
        const uint32_t bar = 2 * x + (use & 1);
        if (works) {
          ok = pk_wait_warp(&sh.taken[bar], ((use >> 1) & 1) ^ 1, fail);
          if (!ok) break;
          ++use;
        }
        tc_fence_after();
        const uint32_t q_lo = uniform(ring_lo + (uint32_t)ring.stage * (L::kTile >> 4)), tS = uniform(tmem + bar * 128);
        if (elected()) {
          if (works) {
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
              const uint32_t off = ((ks >> 2) * kBox + (ks & 3) * 32) >> 4;
              umma_bf16(tS, mine_lo + off, q_lo + off, kIdescScores, ks > 0);
            }
            umma_commit(&sh.scores[bar]);
          }
          umma_commit(&sh.empty[ring.stage]);
          if (!kSplit && s.t == tiles - 1 && s.g == p.group - 1) umma_commit(&sh.own_free[own_buf]);
        }
        __syncwarp();
        ring.step();
      }
    }
    if (!ok || *fail) pk_give_up(sh, p.status);
  } else {
    pk_more_registers<WeightRoles>();
    const int group = warp >> 2, x = group >> 1, half = group & 1, w32 = (warp & 3) * 32, r = w32 + lane;
    const uint32_t lane_addr = (uint32_t)w32 << 16;
    constexpr float sc = kScoreScale<D>;
    int at = 0;   // the step's lse
    int slot = 0;
    uint32_t phase = 0, use = 0;
    bool ok = true;
    // the warps of a tile meet in barriers, so they leave together
    while (!pk_any_failed(x, !pk_next(sh, slot, phase))) {
      const PkItem& it = sh.item[slot];
      const int begin = it.begin, len = it.len, first = it.first[x], t0 = it.steps[x];
      const int tiles = (len - begin + kPkRows - 1) / kPkRows;
      const int key = first + r;
      float sum = 0.f;
      for (WeightSteps s(it.steps[0], p.group, rank, ranks); s.t < tiles; s.next()) {
        const float* lse = s_lse + at * kPkRows + half * 64;
        uint64_t* lse_free = &sh.lse_free[at];
        at ^= 1;
        if (s.t < t0) continue;
        const int q0 = begin + s.t * kPkRows + half * 64, valid = len - q0;
        const uint32_t buf = use & 1;
        ok = pk_wait_warp(&sh.scores[2 * x + buf], (use >> 1) & 1, fail);
        if (!ok) { *fail = 1; break; }
        ++use;
        tc_fence_after();
        uint32_t v[64];
        tmem_ld64(tmem + (2 * x + buf) * 128 + half * 64 + lane_addr, v);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cta(&sh.taken[2 * x + buf]);   // the next product may overwrite it
        u64 acc[4];   // 32-bit sums of 16 terms each
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = pack2(0.f, 0.f);
#pragma unroll
        for (int part = 0; part < 2; ++part) {   // 32 queries, of which none, all or some count for this warp's keys
          const int c0 = part * 32, lo = key - q0 - c0, hi = valid - c0;
          const int warp_lo = first + w32 - q0 - c0;   // the warp's first key; its last is 31 further
          if (warp_lo > 31 || hi <= 0) continue;
          if (warp_lo + 31 <= 0 && hi >= 32) add_weights<false>(v, part, lse + c0, sc, 0, 32, acc);
          else add_weights<true>(v, part, lse + c0, sc, lo, hi, acc);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive_cta(lse_free);
        sum += (sum2(acc[0]) + sum2(acc[1])) + (sum2(acc[2]) + sum2(acc[3]));
      }
      const int seq = it.seq, head = it.head[0];
      pk_release(sh, slot, phase);
      // the second half's sums go to the first half's threads
      const int pair_bar = 3 + x * 4 + (warp & 3);
      float* s_sum = s_sums + x * kPkRows + r;
      if (pk_any_failed(x, !ok)) { ok = false; break; }
      sum = sum_or_nan(sum);
      if (half == 1) *s_sum = sum;
      asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory");
      if (kSplit && half == 0) *s_sum += sum;
      if (!kSplit && half == 0 && key < len) p.weights[((size_t)seq * p.kv_heads + head) * p.capacity + key] = sum + *s_sum;
      asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory");
    }
    if (!ok) *fail = 1;
  }
  if (kSplit) {
    __syncwarp();
    cluster_sync();
    const PkItem& it = sh.item[0];
    const int x = threadIdx.x >> 7, r = threadIdx.x & 127;
    if (rank == 0 && x < 2 && !it.stop && it.first[x] + r < it.len) {
      float sum = 0.f;
      int failed = 0;   // in any of the blocks: its share of the sums is not there
      for (int c = 0; c < ranks; ++c) {
        sum += peer_value(s_sums + x * kPkRows + r, c);
        failed |= peer_value(&sh.fail, c);
      }
      if (!failed) p.weights[((size_t)it.seq * p.kv_heads + it.head[0]) * p.capacity + it.first[x] + r] = sum;
    }
    __syncwarp();
    cluster_sync();   // the others' shared memory stays until it has been read
  }
  pk_end<WeightRoles>(sh, tmem);
}

// ------------------------------------------------------------------------------------------------------------------
// C ABI
// ------------------------------------------------------------------------------------------------------------------
// [total][heads][D] bf16 with any strides, boxes of 128 tokens x 64 elements of one head; tokens outside read as zeros.
bool packed_map(EncodeTiledFn fn, CUtensorMap* map, const void* base, int dim, int heads, int total, int64_t token_stride, int64_t head_stride) {
  const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)total};
  // the stride of a dimension of one is never used, but has to be a valid one
  const cuuint64_t strides[2] = {(cuuint64_t)(heads > 1 ? head_stride : dim) * 2, (cuuint64_t)(total > 1 ? token_stride : dim) * 2};
  const cuuint32_t box[3] = {64, 1, kPkRows};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool aligned(const void* p, unsigned a) { return p && (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool stride_ok(int64_t s) { return s > 0 && s % 8 == 0 && s < (1ll << 39); }   // what a tensor map takes: positive multiples of 16 bytes below 2^40
bool strides_ok(const st3_packed* p, int heads, int64_t token, int64_t head) {   // of one token or one head none is used
  return (p->total <= 1 || stride_ok(token)) && (heads == 1 || stride_ok(head));
}

st3_status check_packed(const st3_packed* p) {
  if (!p) return ST3_ERR_INVALID_ARG;
  if (p->num_seqs < 0 || p->total < 0 || p->num_heads < 1 || p->num_kv_heads < 1 || p->num_heads % p->num_kv_heads) return ST3_ERR_INVALID_ARG;
  if (p->dtype != ST3_BF16 || (p->head_dim != 64 && p->head_dim != 128)) return ST3_ERR_UNSUPPORTED;
  if (!strides_ok(p, p->num_heads, p->q_token_stride, p->q_head_stride) || !strides_ok(p, p->num_kv_heads, p->k_token_stride, p->k_head_stride))
    return ST3_ERR_INVALID_ARG;
  // items and tokens are numbered with 31 bits
  if (((long long)p->total / kPkRows + 2ll * p->num_seqs) * p->num_heads > 0x7fffffffLL || p->total > 0x7fffff00) return ST3_ERR_UNSUPPORTED;
  return ST3_OK;
}

PackedParams packed_params(const st3_packed* p, const int32_t* cu, int* status) {
  PackedParams d = {};
  d.cu = cu; d.status = status;
  d.num_seqs = p->num_seqs; d.total = p->total; d.heads = p->num_heads; d.kv_heads = p->num_kv_heads;
  d.group = p->num_heads / p->num_kv_heads;
  return d;
}

template <int D>
st3_status attend_launch(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const PackedParams& d, cudaStream_t s) {
  if (!allow_smem<st3_packed_attend_kernel<D>>(PkLayout<D, 1>::kTotal)) return ST3_ERR_CUDA;
  return launch(st3_packed_attend_kernel<D>, dim3((unsigned)d.items), dim3(AttendRoles::kThreads), PkLayout<D, 1>::kTotal, s, mq, mk, mv, d);
}
template <int D>
st3_status weights_launch(const CUtensorMap& mq, const CUtensorMap& mk, const PackedParams& d, int split, cudaStream_t s) {
  const dim3 grid((unsigned)(d.items * split)), block(WeightRoles::kThreads);
  constexpr int smem = PkLayout<D, 2>::kTotal;
  if (split > 1) {
    if (!allow_smem<st3_packed_weights_kernel<D, true>>(smem)) return ST3_ERR_CUDA;
    return launch_clusters(split, st3_packed_weights_kernel<D, true>, grid, block, smem, s, mq, mk, d);
  }
  if (!allow_smem<st3_packed_weights_kernel<D, false>>(smem)) return ST3_ERR_CUDA;
  return launch(st3_packed_weights_kernel<D, false>, grid, block, smem, s, mq, mk, d);
}

// Blocks that share an item of the weights.  A prompt alone has fewer items than the GPU has SMs, and the longest, the first
// keys' with all queries, takes as long as a block needs for them.  Shared by the blocks of a cluster, items become more and
// shorter; against that stand a block's start (2 us, which the queue hides) and that it is done once for each of the blocks.
// So: as many as the SMs hold, or up to about three rounds of blocks where an item has steps enough (us, shared by 1 / 2 / 4 / 8
// blocks; 32 heads on 8, D = 128: 700 tokens 32 / 19 / 13 / 16, 2 500: 106 / 58 / 51 / 71, 4 000: 173 / 89 / 104 / 137; 8 heads on
// 2, D = 64: 700: 31 / 18 / 11 / 9; one head to a group, 32 heads: 700: 12 / 14 / 24 / 50).  Clusters of eight fit less well: 16
// of them take two rounds.
int weights_split(const PackedParams& d) {
  const long long items = ((long long)d.total / (2 * kPkRows) + d.num_seqs) * d.kv_heads;   // at most
  const int longest = d.total / d.num_seqs + 1, queries = d.window > 0 ? min(d.window, longest) : longest;   // for even lengths
  const long long steps = (long long)((queries + kPkRows - 1) / kPkRows) * d.group;
  int split = 1;
  for (int blocks = 2; blocks <= 8 && blocks <= steps; blocks *= 2) {
    const int most = blocks < 8 ? (steps < 16 ? 148 : 400) : (steps < 40 ? 112 : 200);
    if (items * blocks <= most) split = blocks;
  }
  return split;
}

}  // namespace

extern "C" st3_status st3_packed_attend(const st3_packed* p, const void* q, const void* k, const void* v, const int32_t* cu,
                                        void* out, float* lse, int* dev_status, void* cuda_stream) {
  const st3_status st = check_packed(p);
  if (st != ST3_OK) return st;
  if (!strides_ok(p, p->num_kv_heads, p->v_token_stride, p->v_head_stride) || !strides_ok(p, p->num_heads, p->out_token_stride, p->out_head_stride))
    return ST3_ERR_INVALID_ARG;
  if (!aligned(cu, 4) || (lse && !aligned(lse, 4))) return ST3_ERR_INVALID_ARG;
  if (p->total == 0 || p->num_seqs == 0) return ST3_OK;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16)) return ST3_ERR_INVALID_ARG;
  const EncodeTiledFn encode = tensor_map_encoder();
  CUtensorMap mq, mk, mv;
  if (!encode || !packed_map(encode, &mq, q, p->head_dim, p->num_heads, p->total, p->q_token_stride, p->q_head_stride) ||
      !packed_map(encode, &mk, k, p->head_dim, p->num_kv_heads, p->total, p->k_token_stride, p->k_head_stride) ||
      !packed_map(encode, &mv, v, p->head_dim, p->num_kv_heads, p->total, p->v_token_stride, p->v_head_stride))
    return ST3_ERR_CUDA;
  PackedParams d = packed_params(p, cu, dev_status);
  d.out = out; d.lse = lse;
  d.out_token_stride = p->out_token_stride; d.out_head_stride = p->out_head_stride;
  d.wide_out = aligned(out, 32) && (p->total == 1 || p->out_token_stride % 16 == 0) && (p->num_heads == 1 || p->out_head_stride % 16 == 0);
  d.by_heads = d.group % 2 == 0;
  d.pairs = d.by_heads ? d.heads / 2 : d.heads;
  d.items = (d.total / (d.by_heads ? kPkRows : 2 * kPkRows) + d.num_seqs) * d.pairs;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return p->head_dim == 128 ? attend_launch<128>(mq, mk, mv, d, s) : attend_launch<64>(mq, mk, mv, d, s);
}

extern "C" st3_status st3_packed_weights(const st3_packed* p, const void* q, const void* k, const float* lse, const int32_t* cu,
                                         float* weights, int32_t capacity, int32_t window, int* dev_status, void* cuda_stream) {
  const st3_status st = check_packed(p);
  if (st != ST3_OK) return st;
  if (capacity < 1 || window < 0 || !aligned(cu, 4)) return ST3_ERR_INVALID_ARG;
  if (p->total == 0 || p->num_seqs == 0) return ST3_OK;   // empty tensors have no address
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(weights, 4) || !aligned(lse, 4)) return ST3_ERR_INVALID_ARG;
  const EncodeTiledFn encode = tensor_map_encoder();
  CUtensorMap mq, mk;
  if (!encode || !packed_map(encode, &mq, q, p->head_dim, p->num_heads, p->total, p->q_token_stride, p->q_head_stride) ||
      !packed_map(encode, &mk, k, p->head_dim, p->num_kv_heads, p->total, p->k_token_stride, p->k_head_stride))
    return ST3_ERR_CUDA;
  PackedParams d = packed_params(p, cu, dev_status);
  d.lse_in = lse; d.weights = weights; d.capacity = capacity; d.window = window;
  d.pairs = d.kv_heads;
  d.items = 2 * (d.total / (4 * kPkRows) + d.num_seqs) * d.pairs;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const int split = weights_split(d);
  return p->head_dim == 128 ? weights_launch<128>(mq, mk, d, split, s) : weights_launch<64>(mq, mk, d, split, s);
}
