// Attention of several new tokens per request over a paged cache of bf16 rows (pact_chunk_attention): Eq. 11 of the paper for prompts and further turns.
//
//   s_ip = scale q_i.k_p + logw_p  (p up to the token's own row, or all),   out_i = sum_p exp(s_ip - m) v_p / sum_p exp(s_ip - m)
//
// Work.  The query heads of a key head read the same rows, so an item is 256 rows (token, head) of one key head: two blocks of 128, a tensor-memory lane
// per row, against tiles of 128 cached rows that arrive once for both.  Per tile and SM 6 x 512 clocks of tcgen05 (128 x 128 x 128, logits and two terms of values, two
// blocks), 2048 clocks of exponentials (16 a clock) and 64 KB from the L2.  None of them bounds a tile: a block's steps follow one another, and the two blocks take turns.  Items of up to 128 rows (a few tokens: HBM bounds them) have one block; its even and odd tiles then take the place of the two blocks, each with a running
// maximum and sums of its own.
// Above 128 columns there is one block (tensor memory has room for one result), with tiles of 64.
//
// Warps: two groups of four have a row per lane (softmax, results), one copies pages through the tensor-copy unit, one issues the products, one looks
// after the values: where a tile has rows that some token must not see, zero times an infinity or a NaN would not be zero, so rows that do not count are
// cleared and other values that are not finite are replaced by zero; their columns and first rows are noted, and the tokens that see them get NaN at the end.
// Logits lie in tensor memory, probabilities take their place there, and results stay in it until the end.  The maximum that logits are taken from lags behind
// the true one by at most 2^8 of a probability, so that results are rescaled a few times per item only.
//
// Measured (four calls in a graph): 1,024 tokens of 32 heads of 128 on 8 key heads over 65,536 rows 1.51 ms, 720 TFLOP/s, and 1.65 ms once the power limit has brought the clock down (1.70 launched one by
// one; a tile 5,700 clocks: 1,000 to 1,250 for the maximum, 2,000 to 2,350 for probabilities, 550 at its beginning, 1,800 until the next logits are there); 12 prompts of up to 2,948 rows 0.73 ms, 480
// TFLOP/s of what the mask leaves (nine tiles an item, then 7,000 clocks for results and the next queries), with 16 heads of 192 and 256 on 4: 0.91 and 1.05 ms; 32 requests of five tokens over up to 8,192
// rows 160 us, 4.2 TB/s; with fp32 results eight times 256 tokens over up to 2,916 rows 242 us (64 columns of the sums of earlier tiles in shared memory instead of all in the L2: 277 -> 270 us then), 30
// times 879 tokens 937 us, heads of 64, all of whose columns fit, 360 us.  What is done once per item is mostly fetching of its code: results 32 columns at a time took 3 % longer, the queries' loop unrolled 1 %.
//
// Rounding: probabilities go into the products with bf16 values as two bf16 terms where results are bf16 (off by 2^-17 of a weight at most: 2 to 4 of
// 1,000 results differ from those of fp32 probabilities; with one term 240 to 370 did), as three, which hold all of fp32's 24 bits, where they are fp32.  The tensor cores cut their running sums
// off towards 0 (some 2^-25 at each of 16 rows and terms), so the products of 32 tiles (fp32 results: of two) at a time are added with rounding: 512 cuts of sums that grow from nothing, 2^-16 in the mean.
// Sums of probabilities are taken before the rounding.
// The second term took the long case from 1.14 to 1.51 ms, the prompts from 0.70 to 0.73, those with heads of 192 and 256 from 0.75 and 0.80 to 0.91 and 1.05; the drafts, 165 us then, and fp32 results, 265, are faster.  For that the loops over
// a tile are rolled: each is 32 columns of code, and logits go back to tensor memory with their biases.  All of a tile's columns in registers and straight code for them, as one term had it, took 1.99, 1.02
// and, for the drafts, 0.26 ms: the warps waited for instructions (1.4 warps per one that was issued, instead of 0.3).  Columns 16 at a time: 1.66 ms; two loads of 32 under way at once: 1.57.
#include "chunk_row.cuh"

namespace pact {
namespace {

constexpr int kSoftmaxWarps = 8;
constexpr int kCopyWarp = 8, kMmaWarp = 9, kValueWarp = 10, kCutWarp = 11;
constexpr int kChunkThreads = 12 * 32;
constexpr float kLag = 8.f;                // of the reference behind the maximum, in powers of two
constexpr size_t kChunkSmem = 227 * 1024;

template <int NB, bool WIDE> struct ChunkShape {
  static constexpr int kBlocks = NB <= 2 ? 2 : 1;                    // of 128 rows in an item
  static constexpr int kRows = kBlocks * 128;
  static constexpr int kTileRows = NB <= 2 && !WIDE ? 128 : 64;
  static constexpr int kGroups = kTileRows / 16;
  static constexpr int kQBytes = NB * 128 * 128;                     // of a block
  static constexpr int kStage = NB * kTileRows * 128;                // K or V of a tile
  // Columns of the sums of earlier tiles that stay in shared memory where there are many (fp32 results); the others go to the L2.
  static constexpr int kKept = WIDE && NB <= 2 ? 64 : 0;
  static constexpr int kKeptBytes = kBlocks * kKept * 128 * 4;
  static constexpr int kFit = (int)((kChunkSmem - kBlocks * kQBytes - kKeptBytes - 4096) / kStage);
  static constexpr int kStages = NB == 2 && !WIDE ? 5 : kFit > 10 ? 10 : kFit;   // (five of 32 KB leave 3 KB for everything else)
  static constexpr int kRing = kStages <= 5 ? 4 : 8;                 // biases of tiles: the copies run ahead by fewer
  static constexpr int kTerms = WIDE ? 3 : 2;                        // of a probability
  static constexpr int kSummed = WIDE ? 2 : 32;                      // tiles whose products are summed by the tensor cores before they are added to the earlier ones with rounding
  static constexpr int kRegion = WIDE ? 96 : kTileRows;              // columns of tensor memory for logits, then the terms of probabilities
  // First column of a term of the probabilities of rows 32 c ..: 16 columns, where logits have been read already (a third term begins behind the logits).
  __host__ __device__ static constexpr int term_at(int c, int term) { return ((WIDE ? kTileRows : 0) + (c * kTerms + term) * 16) % kRegion; }
  static constexpr int kO = kBlocks * kRegion;                       // first column of the results
  static constexpr int kWidth = NB * 64;
  static_assert(kO + kBlocks * kWidth <= 512 && kTerms * kTileRows / 2 <= kRegion && 2 * kRing - 3 >= kStages, "");
  // Where every segment has one tile, half of the stages hold values of as many segments, all after the one whose results are being written.
  static_assert(kStages / 2 + 1 <= kChunkPoison, "");
};

template <int NB, bool WIDE> struct ChunkShared {
  using C = ChunkShape<NB, WIDE>;
  char q[C::kBlocks][C::kQBytes];
  char stage[C::kStages][C::kStage];
  float4 kept[C::kKept ? C::kBlocks : 1][C::kKept ? C::kKept / 4 : 1][C::kKept ? 128 : 1];
  float bias[C::kRing][C::kTileRows];
  uint64_t full[C::kStages], empty[C::kStages];
  uint64_t b_full[C::kRing], b_ready[C::kRing], clean[C::kRing];
  uint64_t q_full[2], s_full[2], p_half[2], p_ready[2], o_full[2], drained;
  int flags[C::kRing];                     // 1: biases count, 2: some are minus infinity
  int poison[2 * C::kRing];                // a tile had values that are not finite beside rows that some token must not see
  int abort, issued;
  uint32_t tmem;
  ChunkLineKept line;
};

__device__ __forceinline__ void chunk_load_4d(void *dst, const CUtensorMap *map, uint64_t *bar, int x, int y, int z, int w) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void chunk_copy16(void *dst, const void *src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void chunk_arrive_after_copies(uint64_t *bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Products whose operands are given by the lower words of their descriptors; the upper ones are the same for all (rows of 128 bytes swizzled, groups of 8 rows 1024 bytes apart).
constexpr uint32_t kDescUpper = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ void umma_ss(uint32_t d_tmem, uint32_t a_desc, uint32_t b_desc, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 x, {%1, %5};\n\t"
      "mov.b64 y, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_desc), "r"(b_desc), "r"(idesc), "r"(accum), "n"(kDescUpper) : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_desc, uint32_t idesc, uint32_t accum) {   // A from tensor memory
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 y, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "r"(b_desc), "r"(idesc), "r"(accum), "n"(kDescUpper) : "memory");
}
// After the wait for loads from tensor memory: what was loaded is used from here on.  The loads are asynchronous and the wait names no registers, so nothing else keeps the
// compiler from using them, and then others in their place, before they have been written.
__device__ __forceinline__ void tmem_arrived(uint32_t (&r)[32]) {
  asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                    "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                    "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                    "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :: "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                 "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_arrived(uint32_t (&r)[16]) {
  asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                    "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :: "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// An operand whose rows are the summed index (values: columns contiguous): 128-byte blocks of columns `block` bytes apart, 8 rows 1024 bytes.
__device__ __forceinline__ uint64_t smem_desc_rows(uint32_t addr, uint32_t block) {
  return smem_desc(addr) & ~((uint64_t)0x3FFF << 16) | ((uint64_t)(block >> 4) << 16);
}

__device__ __forceinline__ unsigned long long pair_of(float x, float y) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void unpair(unsigned long long v, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ unsigned long long of_pair(uint32_t x, uint32_t y) {   // the same of bits
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(x), "r"(y));
  return r;
}
__device__ __forceinline__ void to_pair(uint32_t &x, uint32_t &y, unsigned long long v) { asm("mov.b64 {%0, %1}, %2;" : "=r"(x), "=r"(y) : "l"(v)); }
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float4 lds_here(uint32_t at) {            // (in this place of the program: asked for well before it is used)
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at));
  return v;
}
// The order in which the tiles of a segment of n are asked for: with one tile ahead K0 V0 K1 V1 .., with two K0 K1 V0 K2 V1 ..; load x of 2 n.
struct LoadAt {
  bool v;
  int j;
};
__device__ __forceinline__ LoadAt chunk_load_at(int x, int n, int ahead) {
  if (ahead == 1) return {(x & 1) != 0, x >> 1};
  if (x == 2 * n - 1) return {true, n - 1};
  if (x == 0 || (x & 1)) return {false, (x + 1) >> 1};
  return {true, (x - 2) >> 1};
}
__device__ __forceinline__ int chunk_v_load(int j, int n, int ahead) { return ahead == 1 ? 2 * j + 1 : min(2 * j + 2, 2 * n - 1); }

// A warp's bounded wait: false once kWaitNs or `polls` have run out, or another warp has given up.
struct ChunkWait {
  int *abort;
  int32_t *status;
  int polls;
  __device__ __forceinline__ bool first(uint64_t *bar, uint32_t parity) const { return polls == INT32_MAX ? mbar_try_wait(bar, parity & 1) : mbar_test(bar, parity & 1); }
  __device__ __forceinline__ bool more(uint64_t *bar, uint32_t parity) const {
    const unsigned long long t0 = global_ns();
    bool ok = false;
    for (int i = 1; i < polls && !*const_cast<volatile int *>(abort); ++i)
      if ((ok = mbar_try_wait(bar, parity & 1)) || ((i & 63) == 63 && global_ns() - t0 > kWaitNs)) break;
    if (!ok) {
      atomicExch(abort, 1);
      if (status) atomicMin(status, (int)PACT_ERR_TIMEOUT);
    }
    return ok;
  }
  __device__ __forceinline__ bool alone(uint64_t *bar, uint32_t parity) const { return first(bar, parity) || more(bar, parity); }   // one thread
  __device__ __forceinline__ bool operator()(uint64_t *bar, uint32_t parity) const {
    int ok = first(bar, parity) ? 1 : 0;
    if (!__all_sync(0xffffffffu, ok)) {
      if ((threadIdx.x & 31) == 0) ok = more(bar, parity) ? 1 : 0;
      ok = __shfl_sync(0xffffffffu, ok, 0);
    }
    __syncwarp();
    return ok != 0;
  }
};

template <int NB, bool WIDE>
__global__ void __launch_bounds__(kChunkThreads, 1)
    k_chunk(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ ChunkArgs a) {
  using C = ChunkShape<NB, WIDE>;
  constexpr int N = C::kTileRows, S = C::kStages, R = C::kRing;
  extern __shared__ __align__(1024) char smem_raw[];
  ChunkShared<NB, WIDE> &sh = *reinterpret_cast<ChunkShared<NB, WIDE> *>(smem_raw);
  static_assert(sizeof(sh) <= kChunkSmem && sizeof(ChunkLineSetup) <= C::kStage, "");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid < S) {
    mbar_init(sh.full + tid, 1);
    mbar_init(sh.empty + tid, 1);
  }
  if (tid < R) {
    mbar_init(sh.clean + tid, 1);
    mbar_init(sh.b_full + tid, 33);
    mbar_init(sh.b_ready + tid, 1);
  }
  if (tid < 2) {
    mbar_init(sh.q_full + tid, 4);
    mbar_init(sh.s_full + tid, 1);
    mbar_init(sh.p_half + tid, 4);
    mbar_init(sh.p_ready + tid, 4);
    mbar_init(sh.o_full + tid, 1);
  }
  if (tid == 0) {
    mbar_init(&sh.drained, 1);
    sh.abort = sh.issued = 0;
  }
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  if (warp == kMmaWarp) tmem_alloc(&sh.tmem, 512);
  tc_fence_before();
  pdl_wait();
  pdl_trigger();
  ChunkCuts cuts;
  ChunkLine line = chunk_line<kChunkThreads, C::kRows, N>(a, sh.line, *reinterpret_cast<ChunkLineSetup *>(sh.stage[0]), cuts);
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // (the set-up's words lie where copies will land)
  __syncthreads();
  __syncwarp();                                                      // (one thread has had more to do; what follows asks for whole warps)
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  const ChunkWait wait = {&sh.abort, a.status, a.polls};
  ChunkSegment s;
  bool ok = true;

  if (warp < kSoftmaxWarps) {
    // ---- rows: softmax and results ----
    const int t = warp >> 2, row = tid & 127;                        // of the block
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;
    const uint32_t my_s = tmem + t * C::kRegion + lanes, my_o = tmem + C::kO + t * C::kWidth + lanes;
    const int d16 = (a.d_h + 15) / 16 * 16;
    // Sums of earlier tiles: columns c0 .. c0 + 3 of this row, the next four kept_step(c0) vectors on (32 columns lie in one memory).  Those in the L2 take the place of the segment's part, which
    // the same thread puts there in the end.
    const auto kept_step = [](int c0) { return C::kKept && c0 < C::kKept ? 128 : C::kRows; };
    const auto kept_at = [&](int block, int c0) {
      if (C::kKept && c0 < C::kKept) return &sh.kept[block][c0 / 4][row];
      return reinterpret_cast<float4 *>(a.part_o) + ((long long)s.place * (C::kWidth / 4) + c0 / 4) * C::kRows + block * 128 + row;
    };
    const float scale = a.scale;                                     // (logits stay in natural units, a multiplication more than powers of two: a bias may be any float)
    const unsigned long long scale2 = pair_of(scale, scale), log2e2 = pair_of(kChunkLog2e, kChunkLog2e);
    uint32_t s_phase = 0, o_phase = 0;
    int tiles = 0, segment = 0;
    const auto is_split = [](const ChunkSegment &x) { return C::kBlocks == 2 && x.rows <= 128; };
    const auto fills_q = [&](const ChunkSegment &x) { return t < C::kBlocks && (t == 0 || !is_split(x)); };
    // This warp's 32 rows of Q, swizzled as the copies of K are; zeros past d_h and the last row.
    const auto ask_for_q = [&](const ChunkSegment &x) {
      constexpr int kLanes = NB == 1 ? 8 : NB == 2 ? 16 : 32, kAtOnce = 32 / kLanes;
      const int c = lane % kLanes, rr = (warp & 3) * 32 + lane / kLanes, at_row = x.first + t * 128 + rr, token = at_row / a.group;
      const int tokens = kAtOnce / a.group, heads = kAtOnce - tokens * a.group;   // from one row of this lane to the next
      const long long step = tokens * a.ldQ + heads * a.ldQh, over = a.ldQ - a.group * a.ldQh;   // over: where the heads of a token end in between
      int head = at_row - token * a.group, left = c * 8 < a.d_h ? x.rows - t * 128 - rr : 0;
      const __nv_bfloat16 *from = static_cast<const __nv_bfloat16 *>(a.Q) + (x.row0 + token) * a.ldQ + (x.kv * a.group + head) * a.ldQh + c * 8;
      uint32_t to = smem_u32(sh.q[t]) + c / 8 * (128 * 128) + rr * 128;
      if (c < NB * 8)
#pragma unroll 4                                                     // (executed once per item: code that is fetched for it costs more than the loop)
        for (int i = 0; i < 32; i += kAtOnce) {
          const bool there = left > i;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + i * 128 + (((c & 7) ^ ((rr + i) & 7)) << 4)), "l"(there ? from : a.Q), "r"(there ? 16 : 0) : "memory");
          from += step;
          head += heads;
          if (head >= a.group) {
            head -= a.group;
            from += over;
          }
        }
    };
    const auto give_q = [&] {
      asm volatile("cp.async.wait_all;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(sh.q_full + t);
    };
    bool have = line.next<C::kRows, N>(a, s), being_read = false;
    if (have && fills_q(s)) {
      ask_for_q(s);
      give_q();
    }
    while (have) {
      const int n = s.j1 - s.j0;
      const bool split = is_split(s);
      const int my_first = split ? t : 0, step = split ? 2 : 1;
      const bool active = t < C::kBlocks && my_first < n;
      const int r = (split ? 0 : t * 128) + row;                     // of the item
      const int at_row = s.first + r, token = at_row / a.group, head = s.kv * a.group + at_row - token * a.group;
      const bool there = r < s.rows;
      // (rows that are not there take part as if they were of the last token, so that no tile is treated as an edge for their sake; a warp of such rows alone only keeps step)
      const int limit = s.limit(there ? token : (s.first + s.rows - 1) / a.group, a.causal);
      const bool idle = !__any_sync(0xffffffffu, there);
      if (being_read) asm volatile("bar.sync 2, %0;" ::"n"(kSoftmaxWarps * 32) : "memory");   // (the first group has read this one's results)
      being_read = false;
      float m = -INFINITY, l = 0.f, f_flush = 1.f;
      bool poisoned = false, flushed = false;
      // The results of kSummed tiles to those of the earlier ones, with rounding.
      const auto keep = [&] {
#pragma unroll 1
        for (int c0 = 0; c0 < d16; c0 += 32) {
          float4 *p = kept_at(t, c0), z[8];
          const int at = kept_step(c0);
#pragma unroll
          for (int i = 0; i < 8; ++i) {                                // (all of them before the first store: one trip to the L2 instead of eight)
            z[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (flushed && c0 + 4 * i < d16) z[i] = p[i * at];
          }
          uint32_t v[32];
          tmem_ld32(my_o + c0, v);
          tmem_ld_wait();
          tmem_arrived(v);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (c0 + 4 * i < d16)
              p[i * at] = make_float4(fmaf(z[i].x, f_flush, __uint_as_float(v[4 * i])), fmaf(z[i].y, f_flush, __uint_as_float(v[4 * i + 1])),
                                      fmaf(z[i].z, f_flush, __uint_as_float(v[4 * i + 2])), fmaf(z[i].w, f_flush, __uint_as_float(v[4 * i + 3])));
        }
        flushed = true;
        f_flush = 1.f;
      };
      if (active)
        for (int j = my_first; j < n && ok; j += step) {
          const int tile = tiles + j, at = tile % R, row0 = (s.j0 + j) * N, nth = split ? j >> 1 : j;
          ok = wait(sh.s_full + t, s_phase++) && wait(sh.b_ready + at, tile / R);
          if (!ok) break;
          tc_fence_after();
          if (idle) {
            if (lane == 0) {
              if (!WIDE) mbar_arrive(sh.p_half + t);
              mbar_arrive(sh.p_ready + t);
            }
            continue;
          }
          const int flags = sh.flags[at];
          if (nth > 0) poisoned = poisoned || sh.poison[(tile - step) % (2 * R)];   // (the products before this tile's are done)
          if (nth > 0 && nth % C::kSummed == 0) keep();
          const int valid = min(max(limit - row0, 0), N);
          const uint32_t bias = smem_u32(sh.bias[at]);
          const bool edge = __any_sync(0xffffffffu, valid < N);
          constexpr uint32_t kNone = 0xFF800000u;                    // minus infinity
          // 32 logits, as they are loaded, with biases
          const auto biased = [&](int c, uint32_t (&x)[32]) {
            float4 w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = lds_here(bias + c * 128 + k * 16);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              uint32_t *y = x + k * 4;
              to_pair(y[0], y[1], fma2(of_pair(y[0], y[1]), scale2, pair_of(w[k].x, w[k].y)));
              to_pair(y[2], y[3], fma2(of_pair(y[2], y[3]), scale2, pair_of(w[k].z, w[k].w)));
            }
          };
          bool plain = (flags & 1) != 0;                             // biases are still to come
          if (edge || (flags & 2)) {                                 // (a pass of its own: code that is seldom executed slows down the loop that it lies in)
#pragma unroll 1
            for (int c = 0; c < N / 32; ++c) {
              uint32_t x[32];
              tmem_ld32(my_s + c * 32, x);
              tmem_ld_wait();
              tmem_arrived(x);
              if (flags & 1) biased(c, x);
              const int left = valid - c * 32;                       // rows that the token sees
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                float4 w = make_float4(0.f, 0.f, 0.f, 0.f);          // hidden rows, whose keys may be anything
                if (flags & 2) w = lds_here(bias + c * 128 + i * 4);
                if (i >= left || w.x == -INFINITY) x[i] = kNone;
                if (i + 1 >= left || w.y == -INFINITY) x[i + 1] = kNone;
                if (i + 2 >= left || w.z == -INFINITY) x[i + 2] = kNone;
                if (i + 3 >= left || w.w == -INFINITY) x[i + 3] = kNone;
              }
              tmem_st32(my_s + c * 32, x);
            }
            tmem_st_wait();
            plain = false;
          }
          float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
          for (int c = 0; c < N / 32; ++c) {                         // (32 at a time: the code of a larger step takes longer to fetch than it saves)
            uint32_t x[32];
            tmem_ld32(my_s + c * 32, x);
            tmem_ld_wait();
            tmem_arrived(x);
            if (plain) {
              biased(c, x);
              tmem_st32(my_s + c * 32, x);
            }
#pragma unroll
            for (int i = 0; i < 32; i += 8)
#pragma unroll
              for (int k = 0; k < 4; ++k) tops[k] = max3(tops[k], __uint_as_float(x[i + 2 * k]), __uint_as_float(x[i + 2 * k + 1]));
          }
          tmem_st_wait();
          // (without biases x are still products of queries and keys, and the scale, which is positive then, comes with the exponent)
          const float unit = flags & 1 ? 1.f : scale, top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * unit;
          if (nth == 0) {
            m = top;
          } else if (__any_sync(0xffffffffu, top > m && (m == -INFINITY || (top - m) * kChunkLog2e > kLag))) {
            const float to = fmaxf(m, top), f = part_weight(m, to);
            m = to;
            l *= f;
            f_flush *= f;
            if (nth % C::kSummed != 0) {                             // (otherwise they are among the earlier ones, and begin anew)
#pragma unroll 1
              for (int c0 = 0; c0 < d16; c0 += 32) {
                uint32_t v[32];
                tmem_ld32(my_o + c0, v);
                tmem_ld_wait();
                tmem_arrived(v);
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
                tmem_st32(my_o + c0, v);
              }
            }
          }
          const float ref = m == -INFINITY ? 0.f : m;
          const unsigned long long ref2 = pair_of(-ref, -ref), unit2 = pair_of(unit, unit), minus2 = pair_of(-1.f, -1.f);
          unsigned long long sums[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll 1
          for (int c = 0; c < N / 32; ++c) {
            uint32_t x[32], p[C::kTerms][16];
            tmem_ld32(my_s + c * 32, x);
            tmem_ld_wait();
            tmem_arrived(x);
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              float u, w;
              unpair(mul2(fma2(of_pair(x[i], x[i + 1]), unit2, ref2), log2e2), u, w);
              unsigned long long y = pair_of(ex2_approx(u), ex2_approx(w));
              sums[i / 2 % 4] = add2(sums[i / 2 % 4], y);
#pragma unroll
              for (int k = 0; k < C::kTerms; ++k) {
                unpair(y, u, w);
                const uint32_t h = bf16_pair(u, w);
                p[k][i / 2] = h;
                y = fma2(of_pair(h << 16, h & 0xFFFF0000u), minus2, y);   // (exact)
              }
            }
#pragma unroll
            for (int k = 0; k < C::kTerms; ++k) tmem_st16(my_s + C::term_at(c, k), p[k]);
            if (!WIDE && c == N / 64 - 1) {                          // products with the first half of the rows may begin
              tmem_st_wait();
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(sh.p_half + t);
            }
          }
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(sh.p_ready + t);
          float u[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) unpair(sums[k], u[2 * k], u[2 * k + 1]);
          l += ((u[0] + u[1]) + (u[2] + u[3])) + ((u[4] + u[5]) + (u[6] + u[7]));
        }
      // ---- results ----
      // The next segment's queries come meanwhile: once this block's logits are done with these (where both groups have the same ones, once all products are).
      ChunkSegment next;
      const bool more = line.next<C::kRows, N>(a, next), fills = more && fills_q(next);
      if (fills && ok && !split) ask_for_q(next);
      if (active && ok) {
        ok = wait(sh.o_full + t, o_phase++);
        tc_fence_after();
        const int last = my_first + (n - 1 - my_first) / step * step;
        poisoned = poisoned || sh.poison[(tiles + last) % (2 * R)];
      }
      if (fills && ok && split) ask_for_q(next);
      if (fills && ok && !split) give_q();
      const int *poison = a.poison + ((long long)blockIdx.x * kChunkPoison + segment % kChunkPoison) * kChunkMaxWidth;
      float f_flush1 = 1.f;
      bool flushed1 = false;
      float m1 = -INFINITY, l1 = 0.f, f0 = 1.f, f1 = 0.f;
      if (split) {
        // The odd tiles' results lie in the same lanes of tensor memory: the first group reads them there, with the reference and sum that the second leaves.
        if (t == 1 && ok) {
          const uint32_t v[16] = {__float_as_uint(m), __float_as_uint(l), __float_as_uint(f_flush), (flushed ? 1u : 0u) | (poisoned ? 2u : 0u)};
          tmem_st16(my_s, v);
          tmem_st_wait();
          tc_fence_before();
        }
        asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxWarps * 32) : "memory");
        if (t == 0 && ok) {
          tc_fence_after();
          uint32_t v[32];
          tmem_ld32(my_s + C::kRegion, v);
          tmem_ld_wait();
          tmem_arrived(v);
          m1 = __uint_as_float(v[0]);
          l1 = __uint_as_float(v[1]);
          const float to = fmaxf(m, m1);
          f0 = part_weight(m, to);
          f1 = part_weight(m1, to);
          f_flush1 = __uint_as_float(v[2]);
          flushed1 = v[3] & 1u;
          poisoned = poisoned || (v[3] & 2u);
          m = to;
          l = l * f0 + l1 * f1;
        }
        if (fills && ok) give_q();                                   // (the next logits take the place of what has just been read)
      }
      if (active && ok && (!split || t == 0) && !idle) {
        const bool both = split && __any_sync(0xffffffffu, l1 != 0.f);
        const float inv = s.slot >= 0 ? 1.f : l == 0.f ? 0.f : 1.f / l;
        const long long out_at = (s.row0 + token) * a.ldO + head * a.ldOh;
        f0 *= inv;
        f1 *= inv;
        // sixteen columns at a time: the code of a larger step takes longer to fetch than it saves
        const auto columns = [&](uint32_t from, const float4 *kept, int at, bool has_kept, float f_kept, float (&o)[16]) {
          uint32_t v[16];
          tmem_ld16(from, v);
          tmem_ld_wait();
          tmem_arrived(v);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = __uint_as_float(v[i]);
          if (has_kept) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const float4 z = kept[i / 4 * at];
              o[i] = fmaf(z.x, f_kept, o[i]);
              o[i + 1] = fmaf(z.y, f_kept, o[i + 1]);
              o[i + 2] = fmaf(z.z, f_kept, o[i + 2]);
              o[i + 3] = fmaf(z.w, f_kept, o[i + 3]);
            }
          }
        };
#pragma unroll 1
        for (int c0 = 0; c0 < d16; c0 += 16) {
          float o[16];
          columns(my_o + c0, kept_at(t, c0), kept_step(c0), flushed, f_flush, o);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] *= f0;
          if (both) {
            float o1[16];
            columns(my_o + C::kWidth + c0, kept_at(C::kBlocks - 1, c0), kept_step(c0), flushed1, f_flush1, o1);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = l1 != 0.f ? fmaf(o1[i], f1, o[i]) : o[i];
          }
          if (poisoned) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (c0 + i < a.d_h && __ldcg(poison + c0 + i) < limit) o[i] = __int_as_float(0x7fffffff);
          }
          if (there && s.slot >= 0) {
            float4 *p = reinterpret_cast<float4 *>(a.part_o) + ((long long)s.slot * (C::kWidth / 4) + c0 / 4) * C::kRows + r;
#pragma unroll
            for (int i = 0; i < 16; i += 4) p[i / 4 * C::kRows] = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
          } else if (there) {
            if (c0 + 16 <= a.d_h) store16(a, out_at + c0, o);
            else store8(a, out_at + c0, o);
          }
          __syncwarp();
        }
        if (there) {
          if (s.slot >= 0) a.part_ml[(long long)s.slot * C::kRows + r] = make_float2(m, l);
          else if (a.lse) a.lse[(s.row0 + token) * (a.n_kvh * a.group) + head] = l == 0.f ? -INFINITY : m + logf(l);
        }
      }
      tc_fence_before();
      if (split) {
        if (t == 0) asm volatile("bar.arrive 2, %0;" ::"n"(kSoftmaxWarps * 32) : "memory");
        else being_read = true;
      }
      tiles += n;
      ++segment;
      have = more;
      s = next;
    }
    if (being_read) asm volatile("bar.sync 2, %0;" ::"n"(kSoftmaxWarps * 32) : "memory");
  } else {
    if (warp == kCopyWarp) {
      // ---- pages ----
      constexpr int kAtOnce = 32 / C::kGroups;                         // tiles whose pages the lanes hold: 16 rows each
      const int per_box = a.box_rows / 16, boxes = N / a.box_rows, my_box = lane / NB, my_nb = lane % NB;
      struct {
        int at, id, off;
        uint32_t bad;
      } win[2] = {{-1, -1, 0, 0u}, {-1, -1, 0, 0u}};                   // of K and of V
      int loads = 0, tiles = 0;
      while (ok && line.next<C::kRows, N>(a, s)) {
        const int n = s.j1 - s.j0, ahead = C::kBlocks == 2 && s.rows <= 128 ? 2 : 1;
        win[0].at = win[1].at = -1;
        for (int x = 0; x < 2 * n; ++x, ++loads) {
          const LoadAt l = chunk_load_at(x, n, ahead);
          const int j = s.j0 + l.j, w = j / kAtOnce, in = j % kAtOnce;
          auto &pages = win[l.v];
          if (pages.at != w) {                                         // page and place of 16 rows per lane
            const long long pos = ((long long)w * 32 + lane) * 16;
            pages.at = w;
            pages.id = -1;
            bool bad = false;
            if (pos < s.len) {
              const int place = (int)pos / a.page;
              pages.off = (int)pos - place * a.page;
              pages.id = a.table[(long long)s.b * a.width + place];
              bad = pages.id < 0 || pages.id >= a.n_pages;
              if (bad) {
                pages.id = -1;
                if (a.status) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
              }
            }
            pages.bad = __ballot_sync(0xffffffffu, bad);
          }
          const int from = in * C::kGroups + my_box * per_box;
          const int id = __shfl_sync(0xffffffffu, pages.id, from & 31), off = __shfl_sync(0xffffffffu, pages.off, from & 31);
          const bool mine = my_box < boxes && id >= 0;
          const uint32_t n_boxes = __popc(__ballot_sync(0xffffffffu, mine));
          const int st = loads % S;
          ok = wait(sh.empty + st, loads / S + 1);
          if (!ok) break;
          if (lane == 0) mbar_arrive_expect_tx(sh.full + st, n_boxes * a.box_rows * 128);
          __syncwarp();
          if (mine)
            chunk_load_4d(sh.stage[st] + (my_nb * N + my_box * a.box_rows) * 128, l.v ? &map_v : &map_k, sh.full + st, my_nb * 64, off, s.kv, id);
          if (!l.v) {                                                  // the biases come with the keys
            const int at = (tiles + l.j) % R;
            const bool counts = a.logw || !(a.scale > 0.f) || (pages.bad >> (in * C::kGroups) & ((1u << C::kGroups) - 1u));
            const int g = in * C::kGroups + lane / 4, bid = __shfl_sync(0xffffffffu, pages.id, g & 31), boff = __shfl_sync(0xffffffffu, pages.off, g & 31);
            if (counts && lane < N / 4) {
              float *to = sh.bias[at] + lane * 4;
              if (bid < 0) *reinterpret_cast<float4 *>(to) = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
              else if (a.logw) chunk_copy16(to, a.logw + (long long)bid * a.page + boff + (lane & 3) * 4);
              else *reinterpret_cast<float4 *>(to) = make_float4(0.f, 0.f, 0.f, 0.f);
            }
            chunk_arrive_after_copies(sh.b_full + at);
            if (lane == 0) sh.flags[at] = counts;
            __syncwarp();
            if (lane == 0) mbar_arrive(sh.b_full + at);
          }
        }
        tiles += n;
      }
      if (lane == 0) sh.issued = loads;
    } else if (warp == kCutWarp) {
      cuts.write<C::kRows, N>(a, line);
    } else if (warp == kMmaWarp) {
      // ---- products, all by one thread: what it does between two of them is time in which none is under way ----
      if (lane == 0) {
        const int d16 = (a.d_h + 15) / 16 * 16, steps = d16 / 16;
        constexpr uint32_t kTypes = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24);
        constexpr uint32_t kLogits = kTypes | ((uint32_t)(N >> 3) << 17);
        const uint32_t values = kTypes | (1u << 16) | ((uint32_t)(d16 >> 3) << 17);
        // (lower words of the descriptors of the first blocks, from which the others are an addition away)
        const uint32_t q0 = (uint32_t)smem_desc(smem_u32(sh.q[0])), k0 = (uint32_t)smem_desc(smem_u32(sh.stage[0])), v0 = (uint32_t)smem_desc_rows(smem_u32(sh.stage[0]), N * 128);
        int tiles = 0, stage = 0;
        uint32_t phase = 0, q_phase = 0, p_phase = 0;                // (of the ring; a bit for each block)
        const auto logits = [&](int t, int q, int st) {
          const uint32_t da = q0 + q * (C::kQBytes / 16), db = k0 + st * (C::kStage / 16), to = tmem + t * C::kRegion;
          if (steps == NB * 4) {
#pragma unroll
            for (int k = 0; k < NB * 4; ++k) umma_ss(to, da + (k / 4 * (128 * 128) + k % 4 * 32) / 16, db + (k / 4 * (N * 128) + k % 4 * 32) / 16, kLogits, k != 0);
          } else {
#pragma unroll 1
            for (int k = 0; k < steps; ++k) umma_ss(to, da + (k / 4 * (128 * 128) + k % 4 * 32) / 16, db + (k / 4 * (N * 128) + k % 4 * 32) / 16, kLogits, k != 0);
          }
          umma_commit(sh.s_full + t);
        };
        // rows [half N / 2, (half + 1) N / 2) of a tile, or all of them
        const auto add_values = [&](int t, int st, int half, bool accumulate) {
          const uint32_t db = v0 + st * (C::kStage / 16) + half * (N / 32) * (2048 / 16), to = tmem + C::kO + t * C::kWidth, from = tmem + t * C::kRegion;
#pragma unroll
          for (int term = C::kTerms - 1; term >= 0; --term)          // the small terms first
#pragma unroll
            for (int k = 0; k < (WIDE ? N / 16 : N / 32); ++k)
              umma_ts(to, from + C::term_at((half * (N / 32) + k) / 2, term) + k % 2 * 8, db + k * (2048 / 16), values, k != 0 || term != C::kTerms - 1 ? 1 : accumulate);
        };
        // the stage of the next load in the order in which they were asked for, and its phase
        const auto take = [&](uint32_t &ph) {
          const int st = stage;
          ph = phase;
          if (++stage == S) {
            stage = 0;
            phase ^= 1;
          }
          return st;
        };
        while (ok && line.next<C::kRows, N>(a, s)) {
          const int n = s.j1 - s.j0;
          const bool split = C::kBlocks == 2 && s.rows <= 128;       // even and odd tiles
          const int blocks = split ? 1 : C::kBlocks, ahead = split ? 2 : 1;
          uint32_t ph;
          for (int t = 0; t < blocks && ok; ++t) {
            ok = wait.alone(sh.q_full + t, q_phase >> t);
            q_phase ^= 1u << t;
          }
          for (int j = 0; j < min(ahead, n) && ok; ++j) {
            const int st = take(ph);
            ok = wait.alone(sh.full + st, ph);
            if (!ok) break;
            tc_fence_after();
            if (split) logits(j, 0, st);
            else
              for (int t = 0; t < blocks; ++t) logits(t, t, st);
            umma_commit(sh.empty + st);
          }
          for (int j = 0; j < n && ok; ++j) {
            const bool more = j + ahead < n;
            uint32_t ph_k = 0;
            const int sv = take(ph), sk = more ? take(ph_k) : 0;
            ok = wait.alone(sh.clean + (tiles + j) % R, (tiles + j) / R) && (!more || wait.alone(sh.full + sk, ph_k));   // (values that are clean have arrived)
            for (int i = 0; i < blocks && ok; ++i) {
              const int t = split ? j & 1 : i, nth = split ? j >> 1 : j;
              if (!WIDE) {
                ok = wait.alone(sh.p_half + t, p_phase >> t);
                if (!ok) break;
                tc_fence_after();
                add_values(t, sv, 0, nth % C::kSummed != 0);
              }
              ok = wait.alone(sh.p_ready + t, p_phase >> t);
              p_phase ^= 1u << t;
              if (!ok) break;
              tc_fence_after();
              if (WIDE) add_values(t, sv, 0, nth % C::kSummed != 0);
              else add_values(t, sv, 1, true);
              if (more) logits(t, split ? 0 : t, sk);
              else umma_commit(sh.o_full + t);
            }
            if (!ok) break;
            umma_commit(sh.empty + sv);
            if (more) umma_commit(sh.empty + sk);
          }
          tiles += n;
        }
        umma_commit(&sh.drained);
      }
      __syncwarp();
    } else if (warp == kValueWarp) {
      // ---- values beside rows that must not be seen ----
      int loads = 0, tiles = 0, segment = 0;
      while (ok && line.next<C::kRows, N>(a, s)) {
        const int n = s.j1 - s.j0, ahead = C::kBlocks == 2 && s.rows <= 128 ? 2 : 1;
        const int seen = s.limit(s.first / a.group, a.causal);         // by all tokens of the item
        int *poison = a.poison + ((long long)blockIdx.x * kChunkPoison + segment % kChunkPoison) * kChunkMaxWidth;
        bool poisoned = false;
        for (int j = 0; j < n; ++j) {
          const int tile = tiles + j, at = tile % R, row0 = (s.j0 + j) * N;
          ok = wait(sh.b_full + at, tile / R);
          if (!ok) break;
          const bool counts = sh.flags[at] & 1;
          float4 b = make_float4(0.f, 0.f, 0.f, 0.f);
          if (counts && lane < N / 4) b = *reinterpret_cast<const float4 *>(sh.bias[at] + lane * 4);
          const float bs[4] = {b.x, b.y, b.z, b.w};
          const int left = s.len - row0 - lane * 4;
          uint32_t live[4];                                            // bit l of live[i]: row 4 l + i
          bool hidden = false;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            hidden = hidden || bs[i] == -INFINITY;
            live[i] = __ballot_sync(0xffffffffu, i < left && bs[i] != -INFINITY);
          }
          hidden = __any_sync(0xffffffffu, hidden);
          __syncwarp();
          if (lane == 0) {
            sh.flags[at] = (counts ? 1 : 0) | (hidden ? 2 : 0);
            mbar_arrive(sh.b_ready + at);
          }
          const int x = loads + chunk_v_load(j, n, ahead), st = x % S;
          ok = wait(sh.full + st, x / S);
          if (!ok) break;
          bool found = false;
          if (hidden || chunk_edge(row0, N, seen)) {
            // (rows that every token of the item sees may hold what they like)
            const int c = lane & 7, from = hidden ? 0 : max(0, seen - row0) & ~3;
            constexpr uint32_t kAll = N == 128 ? 0xffffffffu : (1u << (N / 4 % 32)) - 1u;
            const bool all_live = (live[0] & live[1] & live[2] & live[3] & kAll) == kAll;
            const auto is_live = [&](int r) { return (((r & 2) ? ((r & 1) ? live[3] : live[2]) : ((r & 1) ? live[1] : live[0])) >> (r >> 2) & 1u) != 0; };
            for (int nb = 0; nb < NB; ++nb) {
              char *base = sh.stage[st] + nb * N * 128 + c * 16;
              uint32_t top = 0;
              for (int r0 = from; r0 < N; r0 += 32) {                // eight rows of a lane at a time
                uint4 v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  const int r = r0 + 4 * k + (lane >> 3);
                  v[k] = r < N ? *reinterpret_cast<const uint4 *>(base + r * 128) : make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  const uint32_t m = 0x7FFF7FFFu, most = __vmaxu2(__vmaxu2(v[k].x & m, v[k].y & m), __vmaxu2(v[k].z & m, v[k].w & m));
                  if (all_live || is_live(r0 + 4 * k + (lane >> 3))) top = __vmaxu2(top, most);
                }
              }
              found = found || (top & 0xFFFFu) >= 0x7F80u || (top >> 16) >= 0x7F80u;
              if (!all_live)
                for (int r = from + (lane >> 3); r < N; r += 4)
                  if (!is_live(r)) *reinterpret_cast<uint4 *>(base + r * 128) = make_uint4(0, 0, 0, 0);
            }
            __syncwarp();
            found = __any_sync(0xffffffffu, found);
            if (found) {                                               // (rare)
              if (!poisoned)
                for (int i = lane; i < kChunkMaxWidth; i += 32) poison[i] = INT32_MAX;
              poisoned = true;
              __syncwarp();
              for (int nb = 0; nb < NB; ++nb)
                for (int r0 = from; r0 < N; r0 += 4) {
                  const int r = r0 + (lane >> 3);
                  __nv_bfloat16 *p = reinterpret_cast<__nv_bfloat16 *>(sh.stage[st] + (nb * N + r) * 128 + c * 16);
                  for (int e = 0; e < 8; ++e) {
                    const uint16_t bits = *reinterpret_cast<const uint16_t *>(p + e);
                    if ((bits & 0x7FFFu) >= 0x7F80u) {
                      *reinterpret_cast<uint16_t *>(p + e) = 0;
                      atomicMin(poison + nb * 64 + (c ^ (r & 7)) * 8 + e, row0 + r);
                    }
                  }
                }
              __threadfence();
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
          if (lane == 0) sh.poison[tile % (2 * R)] = found;
          __syncwarp();
          if (lane == 0) mbar_arrive(sh.clean + at);
        }
        loads += 2 * n;
        tiles += n;
        ++segment;
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");                   // (queries and biases asked for before a wait ran out)
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) mbar_wait_slow(&sh.drained, 0);
  if (sh.abort && tid < min(S, sh.issued)) mbar_wait_slow(sh.full + tid, (sh.issued - 1 - tid) / S & 1);   // copies under way still write to this CTA's shared memory
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
}

// ---- host side -----------------------------------------------------------------------------------

typedef CUresult (*ChunkEncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                  const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Pages as [page][head][row][column], boxes of box_rows rows and 128 bytes (zeros past d_h).
bool encode_chunk_pages(const ChunkCfg &cfg, CUtensorMap *map, void *base, const ChunkArgs &a, long long ld_page, long long ld_head, long long ld_row) {
  const cuuint64_t dims[4] = {(cuuint64_t)a.d_h, (cuuint64_t)a.page, (cuuint64_t)a.n_kvh, (cuuint64_t)a.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)ld_row * 2, (cuuint64_t)ld_head * 2, (cuuint64_t)ld_page * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)a.box_rows, 1, 1}, estr[4] = {1, 1, 1, 1};
  return reinterpret_cast<ChunkEncodeFn>(cfg.encode_tiled)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

using ChunkKernel = void (*)(CUtensorMap, CUtensorMap, ChunkArgs);
struct ChunkForm {
  ChunkKernel kernel;
  int rows, tile, smem;
};
template <int NB, bool WIDE> ChunkForm form() {
  return {k_chunk<NB, WIDE>, ChunkShape<NB, WIDE>::kRows, ChunkShape<NB, WIDE>::kTileRows, (int)sizeof(ChunkShared<NB, WIDE>)};
}
ChunkForm form_of(const ChunkCfg &cfg) {
  switch (cfg.blocks) {
    case 1: return cfg.wide ? form<1, true>() : form<1, false>();
    case 2: return cfg.wide ? form<2, true>() : form<2, false>();
    case 3: return cfg.wide ? form<3, true>() : form<3, false>();
    case 4: return cfg.wide ? form<4, true>() : form<4, false>();
  }
  return {nullptr, 0, 0, 0};
}

size_t round256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

cudaError_t chunk_configure(ChunkCfg *cfg, const DeviceCfg &dev, int d_h, bool bf16, bool out_bf16) {
  const int blocks = (d_h * (bf16 ? 2 : 4) + 127) / 128;
  if (blocks > 4 || dev.sm_count > kChunkMaxSms) return cudaSuccess;
  cfg->bf16 = bf16;
  cfg->blocks = blocks;
  cfg->ctas = dev.sm_count;
  if (!bf16) {
    const ChunkFormF32 f = chunk_form_f32();
    cfg->rows = f.rows;
    cfg->tile = f.tile;
    cfg->width = f.width;
    return chunk_configure_f32(*cfg, d_h);
  }
  void *fn = nullptr;
  cudaDriverEntryPointQueryResult qres;
  cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
  if (e != cudaSuccess) return e;
  if (qres != cudaDriverEntryPointSuccess || !fn) return cudaErrorNotSupported;
  cfg->encode_tiled = fn;
  cfg->wide = !out_bf16;
  const ChunkForm f = form_of(*cfg);
  cfg->rows = f.rows;
  cfg->tile = f.tile;
  cfg->width = blocks * 64;
  return cudaFuncSetAttribute(f.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, f.smem);
}

size_t chunk_scratch(const ChunkCfg &cfg, int requests, ChunkArgs *a, char *base) {
  if (!cfg.blocks) return 0;
  const size_t G = cfg.ctas, parts = 4 * G * cfg.rows;
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    char *p = base + at;
    at += round256(bytes);
    return p;
  };
  char *o = take(parts * cfg.width * sizeof(float)), *ml = take(parts * sizeof(float2)),
       *cut = take(2 * G * sizeof(ChunkCut)), *tail = take(G * sizeof(int)), *head = take(G * G * sizeof(int)),
       *pre = take(requests < kChunkPreInSmem ? 0 : G * ((size_t)requests + 1) * sizeof(int)), *poison = take(G * kChunkPoison * kChunkMaxWidth * sizeof(int));
  if (a) {
    a->part_o = reinterpret_cast<float *>(o);
    a->part_ml = reinterpret_cast<float2 *>(ml);
    a->cut = reinterpret_cast<ChunkCut *>(cut);
    a->tail = reinterpret_cast<int *>(tail);
    a->head = reinterpret_cast<int *>(head);
    a->pre = reinterpret_cast<int *>(pre);
    a->poison = reinterpret_cast<int *>(poison);
  }
  return at;
}

cudaError_t launch_chunk(ChunkArgs a, const pact_paged_cache &cache, const ChunkCfg &cfg, cudaStream_t st, int *launches) {
  *launches = 2;
  if (!cfg.bf16) {
    const cudaError_t e = launch_chunk_f32(a, cache, cfg, st);
    return e != cudaSuccess ? e : launch_chunk_join(a, cfg, st);
  }
  a.box_rows = 16;
  while (a.box_rows < cfg.tile && a.page % (2 * a.box_rows) == 0) a.box_rows *= 2;
  CUtensorMap mk, mv;
  if (!encode_chunk_pages(cfg, &mk, cache.K, a, cache.k_page, cache.k_head, cache.k_row) ||
      !encode_chunk_pages(cfg, &mv, cache.V, a, cache.v_page, cache.v_head, cache.v_row))
    return cudaErrorInvalidValue;
  const ChunkForm f = form_of(cfg);
  const cudaError_t e = launch_k(f.kernel, dim3((unsigned)cfg.ctas), dim3(kChunkThreads), (size_t)f.smem, st, true, mk, mv, a);
  if (e != cudaSuccess) return e;
  return launch_chunk_join(a, cfg, st);
}

}  // namespace pact
