// Block attention over the 4-bit paged cache: tcgen05 with the cache as the A operand.
//
// Both products are taken transposed, so that the dequantised cache is the
// 128-row A operand in tensor memory and never passes through shared memory:
//   S^T[128 tokens x N rows] = K[128 x D] Q^T      A: TMEM lane = token
//   O^T[D channels x N rows] += V^T[D x 128] P^T   A: TMEM lane = channel
// A K row is a token's codes and a V row a channel's codes, each read by the
// one thread that owns the lane. Shared memory then carries the packed
// records (20 D bytes per 16 tokens, 0.31 of bf16), Q, and P (bf16).
//
// A step is 128 tokens x up to 160 rows, or 256 tokens x up to 64 rows: a
// hand-over between two roles costs some 300 cycles however little work lies
// between, so a step carries twice the work of the smallest tile. (With no
// work in the roles at all, 155 rows in two chunks still took 154 of 267 us.)
//
// Roles: one warp lists the CTA's units, one streams their records with bulk
// copies into a ring; four or eight warps dequantise K, and V; eight or 16
// softmax warps take a token per lane, in groups of four with equal shares of
// the rows; one warp issues the score products, one the value products, so that
// neither waits for the other's operands. The softmax paces steps of 128
// tokens, the dequantisation steps of 256, so each gets the warps of the other.
//
// Bound: the latency of the hand-overs. No pipe is full: 155 rows of 16 sequences
// of 8192 to 16384 tokens (8 KV heads of 128) take 186 us, 655 TFLOP/s, with issue
// slots used to 66% and the tensor pipe to 33%; 128 rows of one of 32768 tokens 38
// us, 455 TFLOP/s, 52% and 21%.
//
// Softmax over tokens runs along TMEM lanes, where a row maximum would cost a
// cross-lane reduction per row and tile, and even a reference per row a
// broadcast load per element. Neither is needed: P and O are scale free in
// bf16 and fp32, so one reference for all rows of a group will do as long as
// their terms 2^(score - reference) stay well inside the exponent range. The
// reference is the largest score of the unit's first token plus 45, so there
// is room for scores 2^46 times that token's and for rows 2^40 below it. A
// term of 2 or more sets a bit of its packed bf16 that no smaller one has (one
// logic operation per three words); a row whose terms are too small shows in
// its sum. (Padding rows score 0 and take part in the first check: a group with
// some is run again where its first token scores below some -46.) A unit that trips either check writes nothing and is run again at
// the end of the batch, once for its rows' maxima and once with the scores
// taken relative to them. Row sums stay per lane in fp32 until the end.
//
// The loops of the roles are kept short, because together they have to stay in
// the SM's instruction cache.
#include <type_traits>

#include "kv4.cuh"

namespace nld {
namespace {

constexpr int kTok = 128;                   // tokens per tile (lanes of A)
constexpr int kTileRecs = kTok / kRecTok;   // 8
constexpr float kHead = 45.f;               // log2 room above the score a reference is taken from
// Smallest row sum taken at its word. Terms below 2^-126 are lost, and so is a
// partial 2^126 below another in the merge: of n tokens, n 2^-41 of such a sum
// (2^-11 at the 2^30 tokens that a page table may hold).
constexpr float kTiny = 0x1p-85f;
constexpr int kSoftBar = 1;                 // named barriers: all softmax warps; 2, 3: a group
constexpr int kBatch = 32;                  // segments handed to the roles at a time
enum Mode { kFirstToken = 0, kMaxima = 1, kKnownMaxima = 2 };  // where a unit's references come from

// Warps by role, for NR rows and TPS tiles per step. 160 rows leave tensor
// memory for one K tile, so the next is dequantised between two score products
// and gets the warps of V, which has two (155 rows, 16 sequences of 8192 to
// 16384 tokens in pieces: 217 us, with four warps for K and eight for V 278).
template <int NR, int TPS>
struct Roles {
  static constexpr bool kOneK = NR > 128;
  static constexpr int kK = TPS == 2 || kOneK ? 8 : 4, kV = kOneK ? 4 : 8, kSoft = TPS == 2 ? 8 : 16;
  static constexpr int kFirstV = kK, kFirstSoft = kFirstV + kV, kLoad = kFirstSoft + kSoft, kScores = kLoad + 1,
                       kPlan = kLoad + 2, kValues = kLoad + 3;
  static constexpr int kThreads = (kLoad + 4) * 32;  // whole warpgroups (register shares)
  static constexpr int kSoftThreads = kSoft * 32;
  // Registers a thread: what the launch gives, and what is left of it to each
  // role; the softmax warps keep their row sums in registers.
  static constexpr int kRegLaunch = TPS == 2 ? 72 : 64;
  static constexpr int kRegDeq = TPS == 2 ? 56 : 48, kRegSoft = TPS == 2 ? 104 : 80, kRegTail = TPS == 2 ? 72 : 48;
  static_assert((kK + kV) * kRegDeq + kSoft * kRegSoft + 4 * kRegTail <= (kLoad + 4) * kRegLaunch,
                "more registers than the launch holds");
};

// NR rows of Q (padded), TPS tiles per step. P comes in pieces of 64 rows: of
// each of two tiles (TPS = 2), or of one tile.
template <int D, int NR, int TPS>
struct Lay {
  static constexpr int kStageBytes = TPS * kTileRecs * Rec<D>::kBytes;
  static constexpr int kQBytes = NR * D * 2;
  static constexpr int kPieceBytes = kTok * 128;       // 128 tokens x 64 rows of P
  static constexpr int kPBytes = (TPS == 2 ? 2 : (NR + 63) / 64) * kPieceBytes;
  static constexpr int kPOff = kQBytes;                // Q first; every operand 1024-byte aligned
  static constexpr int kRingOff = kPOff + 2 * kPBytes;
  static constexpr int kStages = (NR == 160 ? 4 : 6 / TPS) * (128 / D);
  static constexpr int kSmallOff = kRingOff + kStages * kStageBytes;
  static constexpr int CPT = NR * 4 / Roles<NR, TPS>::kSoft;  // rows per softmax group
  // TMEM columns: K tiles (128 bf16 per lane: 64 columns; one beside 160 rows,
  // else two), S, O, and as many V tiles as the rest holds
  static constexpr int kKTiles = Roles<NR, TPS>::kOneK ? 1 : 2;
  static constexpr int kORows = TPS == 2 ? 64 : NR;    // columns of O (TPS = 2: whole 128-byte rows of P)
  static constexpr int kCols = 512;
  static constexpr int kKCol = 0, kSCol = kKTiles * 64, kOCol = kSCol + TPS * NR, kVCol = kOCol + kORows;
  static constexpr int kVTiles = (kCols - kVCol) / 64;
  static_assert(kVTiles >= 2 && kVTiles <= 4, "TMEM");
};

template <int NR>
struct Small {
  uint64_t full[12], empty[12];
  uint64_t k_full[2], k_free[2];  // per K buffer
  uint64_t s_done[2], s_free[2];  // per tile of a step, a phase per step
  uint64_t v_full[4], pv_done[4]; // per V buffer
  uint64_t p_full[2];             // per step
  uint64_t q_full, o_free, drain;
  uint32_t tmem;
  int count;                      // segments of the batch
  int last[2];                    // by parity of the batch: no more after them, unless some have failed
  int num_failed[2];              // by parity of the batch: units with terms out of range
  float ref[4];                   // reference per softmax group
  float max_row[NR];              // maxima per row (a unit's second run)
  uint32_t bits[NR];              // visible block slots per row
  float inv[NR];                  // factor of each row's output
  float red[4][NR];               // per lane quadrant: sums or maxima
  int out_row[NR];                // row of out, or of the partials
  Kv4Segment seg[2 * kBatch];
  int mode[2 * kBatch];
  int failed[kBatch];
};

// Registers a thread of this warpgroup may use from here on.
template <int N>
__device__ __forceinline__ void set_regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void set_regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// One lane of a converged warp. The compiler keeps what it guards in uniform
// registers, where the MMA descriptors have to be: an MMA is issued every 12
// to 31 cycles (N = 16 to 64), against about 100 behind a test of the lane
// number, which moves each descriptor there from a vector register first.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\tselp.u32 %0, 1, 0, e;\n\t}" : "=r"(r));
  return r != 0;
}

__device__ __forceinline__ bool barrier_or(int id, int threads, bool p) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred a, b;\n\tsetp.ne.u32 a, %3, 0;\n\t"
      "barrier.cta.red.or.pred b, %1, %2, a;\n\t"
      "selp.u32 %0, 1, 0, b;\n\t}"
      : "=r"(r)
      : "r"(id), "r"(threads), "r"(p ? 1u : 0u)
      : "memory");
  return r != 0;
}

// Maximum of a float over the warp (order-preserving integer keys).
__device__ __forceinline__ float warp_max(float x) {
  const int i = __float_as_int(x);
  const int k = __reduce_max_sync(0xffffffffu, i ^ ((i >> 31) & 0x7fffffff));
  return __int_as_float(k ^ ((k >> 31) & 0x7fffffff));
}

template <int N>
__device__ __forceinline__ void tmem_store(uint32_t addr, const float* in) {
  uint32_t w[N];
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = __float_as_uint(in[i]);
  tmem_st_u32<N>(addr, w);
}

// 16 TMEM lanes x 16 columns: thread l holds columns 2 (l % 4), + 1 of each 8
// in lanes l / 4 (first two words of a block) and l / 4 + 8 (next two).
__device__ __forceinline__ void tmem_st_16x256b_x2(uint32_t addr, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                   uint32_t b0, uint32_t b1, uint32_t b2, uint32_t b3) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(addr), "r"(a0),
               "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "r"(b2), "r"(b3)
               : "memory");
}

__device__ __forceinline__ void tmem_ld8(uint32_t addr, float* out) {
  uint32_t r[8];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
               "tcgen05.wait::ld.sync.aligned;"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(addr)
               : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) out[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_ld24(uint32_t addr, float* out) {
  uint32_t r[24];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%24];\n\t"
               "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%16, %17, %18, %19, %20, %21, %22, %23}, [%25];\n\t"
               "tcgen05.wait::ld.sync.aligned;"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23])
               : "r"(addr), "r"(addr + 16)
               : "memory");
#pragma unroll
  for (int i = 0; i < 24; ++i) out[i] = __uint_as_float(r[i]);
}
template <int N>
__device__ __forceinline__ void tmem_load(uint32_t addr, float* out) {
  if constexpr (N == 32) tmem_ld32(addr, out);
  else if constexpr (N == 24) tmem_ld24(addr, out);
  else if constexpr (N == 16) tmem_ld16(addr, out);
  else tmem_ld8(addr, out);
}

// Sums of N (8, 16 or 32) values per lane over the warp: lane i gets that of value i mod N.
template <int N>
__device__ __forceinline__ float warp_sums(float* v, int lane) {
#pragma unroll
  for (int w = 16; w >= N; w >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], w);
#pragma unroll
  for (int w = N / 2; w >= 1; w >>= 1) {
    const bool up = (lane & w) != 0;
#pragma unroll
    for (int i = 0; i < w; ++i) {
      const float keep = up ? v[i + w] : v[i], send = up ? v[i] : v[i + w];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, w);
    }
  }
  return v[0];
}

template <int D, int NR, int TPS>
__global__ void __launch_bounds__(Roles<NR, TPS>::kThreads, 1) block_attn_kv4_tc_kernel(Kv4AttnArgs a, int rows) {
  using Ly = Lay<D, NR, TPS>;
  using Ro = Roles<NR, TPS>;
  constexpr int kSt = Ly::kStages;
  constexpr int CPT = Ly::CPT;
  constexpr int kStepTok = TPS * kTok, kStepRecs = TPS * kTileRecs;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sq = smem;
  uint8_t* sp = smem + Ly::kPOff;
  uint8_t* ring = smem + Ly::kRingOff;
  Small<NR>& sh = *reinterpret_cast<Small<NR>*>(smem + Ly::kSmallOff);

  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int quad = warp & 3;
  grid_launch_dependents();
  if (warp == Ro::kScores) {
    if (lane == 0) {
      for (int i = 0; i < kSt; ++i) {
        mbar_init(&sh.full[i], 1);
        mbar_init(&sh.empty[i], Ro::kK + Ro::kV);
      }
      for (int i = 0; i < 2; ++i) {
        mbar_init(&sh.k_full[i], Ro::kK);
        mbar_init(&sh.k_free[i], 1);
        mbar_init(&sh.s_done[i], 1);
        mbar_init(&sh.s_free[i], Ro::kSoft);
        mbar_init(&sh.p_full[i], Ro::kSoft);
      }
      for (int i = 0; i < Ly::kVTiles; ++i) {
        mbar_init(&sh.v_full[i], Ro::kV);
        mbar_init(&sh.pv_done[i], 1);
      }
      mbar_init(&sh.q_full, Ro::kSoft);
      mbar_init(&sh.o_free, Ro::kSoft);
      mbar_init(&sh.drain, 2);
      fence_mbar_init();
      sh.num_failed[1] = 0;
    }
    __syncwarp();
    tmem_alloc(&sh.tmem, Ly::kCols);
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  grid_dependency_wait();

  const int max_len = static_cast<int>((static_cast<long>(a.max_pages) << a.log2_page) - a.bl);
  const Kv4Sched sc{a.lens, a.B, a.Hkv * a.chunks, a.bl, kStepTok, max_len, a.ctas, a.workers,
                     a.ranges_above, a.min_piece};
  bool ok = true;  // false after a wait passed its limit
  // Runs a role over the CTA's segments, which the planning warp lists in
  // batches; g = steps and s0 = segments of the batches before.
  const auto batches = [&](auto plan, auto role) {
    int g = 0, s0 = 0;
    for (int batch = 0;; batch ^= 1) {
      plan(s0, batch);
      __syncthreads();
      const int count = sh.count;
      role(count, g, s0, batch);
      for (int k = 0; k < count; ++k) g += sh.seg[k].end - sh.seg[k].begin;
      s0 += count;
      __syncthreads();  // the batch has been read
      if (sh.last[batch] && sh.num_failed[batch] == 0) break;
    }
  };
  // Scores are issued, and read, tile by tile of a step: while one is read, the
  // other's product is on its way. (Splitting a tile's rows in the same way made
  // steps of one tile slower: 236 -> 275 us for 155 rows.)
  const auto scores_done = [&](int p, int step) { return warp_wait(&sh.s_done[p], step & 1, a.err); };
  // The value products of a tile have completed.
  const auto values_done = [&](int tile, auto patient) {
    return warp_wait<decltype(patient)::value>(&sh.pv_done[tile % Ly::kVTiles], (tile / Ly::kVTiles) & 1, a.err);
  };
  constexpr std::true_type patient;
  constexpr std::false_type at_once;
  const auto no_plan = [](int, int) {};
  // Register shares are set inside the branches, so that each role's code is
  // compiled to its own.
  if (warp < Ro::kFirstV) {
    set_regs_down<Ro::kRegDeq>();
    batches(no_plan, [&](int count, int g, int, int) {
      // ---- K: codes -> TMEM, lane = token --------------------------------------
      const int rec = 2 * quad + (lane >> 4), t = lane & 15;
      // the warps of a lane quadrant deal a tile's groups between them
      constexpr int kGroups = Rec<D>::kGroups, kMine = kGroups * 4 / Ro::kK;
      const int first = (warp >> 2) * kMine;
#pragma unroll 1
      for (int k = 0; ok && k < count; ++k) {
        const int g_end = g + sh.seg[k].end - sh.seg[k].begin;
#pragma unroll 1
        for (; g < g_end; ++g) {
          const int st = g % kSt;
          ok = warp_wait<true>(&sh.full[st], (g / kSt) & 1, a.err);
          const uint8_t* src = ring + st * Ly::kStageBytes + rec * Rec<D>::kBytes;
#pragma unroll 1
          for (int tile = g * TPS; ok && tile < (g + 1) * TPS; ++tile, src += kTileRecs * Rec<D>::kBytes) {
            if (tile >= Ly::kKTiles)  // the scores have read this buffer
              ok = warp_wait<true>(&sh.k_free[tile % Ly::kKTiles], (tile / Ly::kKTiles - 1) & 1, a.err);
            if (!ok) break;
            tc_fence_after();
            const uint32_t dst = tmem + (static_cast<uint32_t>(quad * 32) << 16) + Ly::kKCol + (tile % Ly::kKTiles) * 64;
            uint32_t scales[4];  // the token's groups' (a, c), next one first
            {
              const uint8_t* from = src + Rec<D>::kKScale + (t * kGroups + first) * 4;
              if constexpr (kMine == 4) {
                const uint4 v = *reinterpret_cast<const uint4*>(from);
                scales[0] = v.x, scales[1] = v.y, scales[2] = v.z, scales[3] = v.w;
              } else if constexpr (kMine == 2) {
                const uint2 v = *reinterpret_cast<const uint2*>(from);
                scales[0] = v.x, scales[1] = v.y;
              } else {
                scales[0] = *reinterpret_cast<const uint32_t*>(from);
              }
            }
#pragma unroll 1
            for (int gr = first; gr < first + kMine; ++gr) {
              const uint4 v = *reinterpret_cast<const uint4*>(src + t * (D / 2) + Rec<D>::k_chunk(t, gr) * 16);
              const uint32_t ac = scales[0];
#pragma unroll
              for (int i = 0; i + 1 < kMine; ++i) scales[i] = scales[i + 1];
              const uint32_t w[4] = {v.x, v.y, v.z, v.w};
              const uint32_t sa = dup_lo(ac), sb = dup_hi(ac);
              uint32_t x[16];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                uint32_t y[4];
                kv4_pairs(w[i], y);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * i + e] = fma_bf16x2(y[e], sa, sb);
              }
              tmem_st_u32<16>(dst + gr * 16, x);
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.k_full[tile % Ly::kKTiles]);
          }
          if (!ok) break;
          if (lane == 0) mbar_arrive(&sh.empty[st]);
        }
      }
    });
  } else if (warp < Ro::kFirstSoft) {
    set_regs_down<Ro::kRegDeq>();
    batches(no_plan, [&](int count, int g, int, int) {
      // ---- V: codes -> TMEM, TMEM lane = channel ----------------------------------
      const int code_at = Rec<D>::kVCode + (quad * 32 + (lane >> 2)) * 8 + ((lane & 3) >> 1) * 4;
      const int code_shift = (lane & 1) * 8;
      // two warps to a lane quadrant, half of a tile's records each
      constexpr int kMine = kTileRecs * 4 / Ro::kV;
      const int r0 = ((warp - Ro::kFirstV) >> 2) * kMine;
#pragma unroll 1
      for (int k = 0; ok && k < count; ++k) {
        int have = sh.seg[k].len + a.bl - sh.seg[k].begin * kStepTok;  // tokens from the tile on
        const int g_end = g + sh.seg[k].end - sh.seg[k].begin;
#pragma unroll 1
        for (; g < g_end; ++g) {
          const int st = g % kSt;
          ok = warp_wait<true>(&sh.full[st], (g / kSt) & 1, a.err);
          const uint8_t* base = ring + st * Ly::kStageBytes;
#pragma unroll 1
          for (int tile = g * TPS; ok && tile < (g + 1) * TPS; ++tile, have -= kTok, base += kTileRecs * Rec<D>::kBytes) {
            if (tile >= Ly::kVTiles) ok = values_done(tile - Ly::kVTiles, patient);  // they have read this buffer
            if (!ok) break;
            tc_fence_after();
            if (quad * 32 < D) {  // D = 64: the upper lanes of A are never read out
              const uint32_t dst =
                  tmem + (static_cast<uint32_t>(quad * 32) << 16) + Ly::kVCol + (tile % Ly::kVTiles) * 64;
              // Two records: 32 channels x 32 tokens -> 16 columns, in the
              // 16x256b shape: lane l holds 4 tokens, from 4 (l % 4) on, of
              // channels l / 4 + 8 j. A scale is then read by 8 lanes at a time
              // instead of being broadcast to 32: with a whole channel per lane
              // the scales alone took 512 shared-memory cycles a tile, here 128.
              // Cells past the end hold anything and become 0 (not 0 * NaN).
              const auto records = [&](int r, bool whole) {
                uint32_t x[4][4];  // [channel j][record, pair]
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                  const uint8_t* from = base + (r + i) * Rec<D>::kBytes;
                  const uint8_t* sc8 = from + Rec<D>::kVScale + quad * 64 + (lane & 3) * 8;
                  uint2 va = *reinterpret_cast<const uint2*>(sc8), vc = *reinterpret_cast<const uint2*>(sc8 + 32);
                  if (!whole) {
                    const int left = have - (r + i) * kRecTok - 4 * (lane & 3);
                    const uint32_t l0 = left >= 2 ? 0xffffffffu : left == 1 ? 0x0000ffffu : 0u;
                    const uint32_t l1 = left >= 4 ? 0xffffffffu : left == 3 ? 0x0000ffffu : 0u;
                    va.x &= l0, vc.x &= l0, va.y &= l1, vc.y &= l1;
                  }
#pragma unroll
                  for (int j = 0; j < 4; ++j) {
                    const uint32_t w = *reinterpret_cast<const uint32_t*>(from + code_at + j * 64) >> code_shift;
                    uint32_t y0, y1;
                    kv4_two_pairs(w, y0, y1);
                    x[j][2 * i] = fma_bf16x2(y0, va.x, vc.x);
                    x[j][2 * i + 1] = fma_bf16x2(y1, va.y, vc.y);
                  }
                }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                  const uint32_t* lo = x[2 * half];
                  const uint32_t* hi = x[2 * half + 1];
                  tmem_st_16x256b_x2(dst + (static_cast<uint32_t>(16 * half) << 16) + r * 8, lo[0], lo[1], hi[0], hi[1],
                                     lo[2], lo[3], hi[2], hi[3]);
                }
              };
              if (have >= kTok) {
#pragma unroll 1
                for (int r = r0; r < r0 + kMine; r += 2) records(r, true);
              } else {
#pragma unroll 1
                for (int r = r0; r < r0 + kMine; r += 2) records(r, false);
              }
              tmem_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.v_full[tile % Ly::kVTiles]);
          }
          if (!ok) break;
          if (lane == 0) mbar_arrive(&sh.empty[st]);
        }
      }
    });
  } else if (warp < Ro::kLoad) {
    set_regs_up<Ro::kRegSoft>();
    batches(no_plan, [&](int count, int g, int, int batch) {
      // ---- softmax: lane = token, a group's rows -----------------------------
      const int st_id = threadIdx.x - Ro::kFirstSoft * 32;
      const int grp = (warp - Ro::kFirstSoft) >> 2, gt_id = st_id & 127;
      constexpr int kW = CPT % 16 == 0 ? 16 : 8;  // columns at a time where speed does not count
      const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
      const float2 scale2 = make_float2(a.scale_log2, a.scale_log2);
      const int tok = quad * 32 + lane;
      const int row0 = grp * CPT;  // the group's rows of Q: row0 .. row0 + CPT - 1
      const int my_row = gt_id < CPT ? row0 + gt_id : -1;
      // a warp whose wait ran out stays in step (the barriers count every warp) but waits no more
#pragma unroll 1
      for (int k = 0; k < count; ++k) {
        const int b = sh.seg[k].b, L = sh.seg[k].len;
        {
          const int h = sh.seg[k].unit / a.chunks, r0 = (sh.seg[k].unit - h * a.chunks) * rows;
          const int live = min(rows, a.R - r0);
          // Q rows, K-major with the 128-byte swizzle; rows past the chunk are zero
#pragma unroll 1
          for (int idx = st_id; idx < NR * (D / 8); idx += Ro::kSoftThreads) {
            const int row = idx / (D / 8), c = idx - row * (D / 8);
            uint4 v = make_uint4(0, 0, 0, 0);
            if (row < live) {
              const int i = (r0 + row) / a.G;
              v = __ldg(reinterpret_cast<const uint4*>(
                            a.q + ((static_cast<long>(b) * a.bl + i) * a.Hq + h * a.G + (r0 + row - i * a.G)) * D) + c);
            }
            *reinterpret_cast<uint4*>(sq + (c >> 3) * (NR * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = v;
          }
          if (st_id < NR) {
            const int i = (r0 + st_id) / a.G;
            const bool real = st_id < live;
            sh.bits[st_id] = real ? kv4_block_bits(a, i) : 0u;
            sh.out_row[st_id] = !real ? -1
                                : sh.seg[k].slot >= 0 ? sh.seg[k].slot * rows + st_id
                                                      : (b * a.bl + i) * a.Hq + h * a.G + (r0 + st_id - i * a.G);
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_full);
        named_bar_sync(kSoftBar, Ro::kSoftThreads);  // the masks are in place

        const int mode = sh.mode[k];
        uint32_t any = 0;  // bit 14 of a bf16: the value is 2 or more
        float ref = 0.f;
        constexpr int kSums = CPT == 24 ? 32 : CPT;
        float l[kSums];
#pragma unroll
        for (int c = 0; c < kSums; ++c) l[c] = 0.f;
        if (mode == kMaxima) {
          for (int c = gt_id; c < 4 * NR; c += 128) sh.red[0][c] = -INFINITY;
          named_bar_sync(kSoftBar, Ro::kSoftThreads);
        }
        int t0 = sh.seg[k].begin * kStepTok;
        const int g_first = g, g_end = g + sh.seg[k].end - sh.seg[k].begin;
#pragma unroll 1
        for (; g < g_end; ++g, t0 += kStepTok) {
          uint8_t* const p_addr = sp + (g & 1) * Ly::kPBytes + tok * 128;
          // the value products of step g - 2 have read this P buffer
          if (ok && g >= 2) ok = values_done((g - 1) * TPS - 1, at_once);
          const auto terms_of = [&](int p) {
            const uint32_t s_addr = tmem + lanes + Ly::kSCol + p * NR + row0;
            if (ok) ok = scores_done(p, g);
            tc_fence_after();
            if (g == g_first && p == 0) {
              if (quad == 0) {
                float top = mode == kFirstToken ? kNoMax : 0.f;
#pragma unroll 1
                for (int c = 0; mode == kFirstToken && c < CPT; c += kW) {
                  float s[kW];
                  tmem_load<kW>(s_addr + c, s);
#pragma unroll
                  for (int e = 0; e < kW; ++e)
                    if (sh.out_row[row0 + c + e] >= 0) top = fmaxf(top, s[e] * scale2.x);
                }
                if (lane == 0) sh.ref[grp] = top > kNoMax ? top + kHead : 0.f;
              }
              named_bar_sync(kSoftBar + 1 + grp, 128);
              ref = sh.ref[grp];
            }
            if (t0 + (p + 1) * kTok > L) {  // hidden cells at -inf
              const int slot = t0 + p * kTok + tok - L;  // < 0: prefix
#pragma unroll 1
              for (int c = 0; c < CPT; c += kW) {
                float s[kW];
                tmem_load<kW>(s_addr + c, s);
#pragma unroll
                for (int e = 0; e < kW; ++e)
                  if (slot >= 0 && (slot >= 32 || !((sh.bits[row0 + c + e] >> slot) & 1u))) s[e] = -INFINITY;
                tmem_store<kW>(s_addr + c, s);
              }
              tmem_wait_st();
            }
            if (mode == kKnownMaxima) {  // scores relative to their row's maximum
#pragma unroll 1
              for (int c = 0; c < CPT; c += kW) {
                float s[kW];
                tmem_load<kW>(s_addr + c, s);
#pragma unroll
                for (int e = 0; e < kW; ++e) s[e] = fmaf(sh.max_row[row0 + c + e], -a.inv_scale_log2, s[e]);
                tmem_store<kW>(s_addr + c, s);
              }
              tmem_wait_st();
            }
            const float2 ref2 = make_float2(-ref, -ref);
            const auto read = [&] {  // the next step's scores may overwrite these
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&sh.s_free[p]);
            };
            if (mode == kMaxima) {
#pragma unroll 1
              for (int c = 0; c < CPT; c += kW) {
                float s[kW];
                tmem_load<kW>(s_addr + c, s);
#pragma unroll
                for (int e = 0; e < kW; ++e) {
                  const float m = warp_max(s[e] * scale2.x);
                  float* const at = &sh.red[quad][row0 + c + e];
                  if (lane == e) *at = fmaxf(*at, m);
                }
                __syncwarp();
              }
              read();
            } else {
              // as many scores at a time as the registers hold
              const auto terms = [&](auto count, int c) {
                constexpr int kLoad = decltype(count)::value;
                float s[kLoad];
                tmem_load<kLoad>(s_addr + c, s);
                if (c == CPT - kLoad) read();
#pragma unroll
                for (int v = 0; v < kLoad; v += 8) {
                  uint32_t w[4];
#pragma unroll
                  for (int i = 0; i < 2; ++i) {
                    const int e = v + 4 * i, le = c + e;
                    float2 x = fma2(make_float2(s[e], s[e + 1]), scale2, ref2);
                    float2 y = fma2(make_float2(s[e + 2], s[e + 3]), scale2, ref2);
                    x = make_float2(ex2(x.x), ex2(x.y));
                    y = make_float2(ex2(y.x), ex2(y.y));
                    const float2 lx = add2(make_float2(l[le], l[le + 1]), x);
                    const float2 ly = add2(make_float2(l[le + 2], l[le + 3]), y);
                    l[le] = lx.x, l[le + 1] = lx.y, l[le + 2] = ly.x, l[le + 3] = ly.y;
                    w[2 * i] = pack_bf16(x.x, x.y);  // P in bf16 for the tensor product; its sum stays in fp32
                    w[2 * i + 1] = pack_bf16(y.x, y.y);
                    any |= w[2 * i] | w[2 * i + 1];
                  }
                  const int at = (row0 + c + v) >> 3;  // 16-byte part of the token's rows
                  uint8_t* const to = p_addr + (TPS == 2 ? p : at >> 3) * Ly::kPieceBytes;
                  *reinterpret_cast<uint4*>(to + (((at & 7) ^ (tok & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                }
              };
              using Sixteen = std::integral_constant<int, 16>;
              if constexpr (TPS == 2 || CPT == 24) {
                terms(std::integral_constant<int, CPT>(), 0);
              } else {
                terms(Sixteen(), 0);
                terms(Sixteen(), 16);
                if constexpr (CPT == 40) terms(std::integral_constant<int, 8>(), 32);
              }
            }
          };
          if constexpr (TPS == 1) {
            terms_of(0);
          } else {
#pragma unroll 1
            for (int p = 0; p < TPS; ++p) terms_of(p);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.p_full[g & 1]);
        }

        // ---- end of the unit: sums over the lanes, then O ----
        if (mode != kMaxima) {
          const float sum = warp_sums<(kSums < 32 ? kSums : 32)>(l, lane);
          if (lane < CPT) sh.red[quad][row0 + lane] = sum;
          if constexpr (CPT == 40) {
            const float rest = warp_sums<8>(l + 32, lane);
            if (lane < 8) sh.red[quad][row0 + 32 + lane] = rest;
          }
        }
        const bool far = barrier_or(kSoftBar, Ro::kSoftThreads, mode == kFirstToken && (any & 0x40004000u) != 0u);
        float sum = 0.f, row_ref = ref;
        bool faint = false;
        if (my_row >= 0) {
          const float r0 = sh.red[0][my_row], r1 = sh.red[1][my_row], r2 = sh.red[2][my_row], r3 = sh.red[3][my_row];
          if (mode == kMaxima) {
            const float m = fmaxf(fmaxf(r0, r1), fmaxf(r2, r3));
            sh.max_row[my_row] = m > kNoMax ? m : 0.f;
          } else {
            sum = (r0 + r1) + (r2 + r3);
            if (mode == kKnownMaxima) {
              row_ref += sh.max_row[my_row];
            } else if (sh.out_row[my_row] >= 0 && !(sum >= kTiny)) {
              // too small, unless the row sees nothing of this unit
              const int slot = sh.seg[k].begin * kStepTok - L;  // < 0: prefix
              faint = slot < 0 || (slot < 32 && (sh.bits[my_row] >> slot) != 0u);
            }
          }
        }
        const bool failed = barrier_or(kSoftBar, Ro::kSoftThreads, faint) || far;
        const bool write = mode != kMaxima && !failed;
        if (failed && st_id == 0) sh.failed[sh.num_failed[batch]++] = k;
        if (my_row >= 0 && write) {
          const int row = sh.out_row[my_row];
          const bool part = sh.seg[k].slot >= 0;
          sh.inv[my_row] = part ? 1.f : sum != 0.f ? 1.f / sum : 0.f;
          if (row >= 0) {
            if (part) {
              a.part_ml[row] = make_float2(sum != 0.f ? row_ref : kNoMax, sum);
            } else if (a.lse != nullptr) {
              const int bi = row / a.Hq, hq = row - bi * a.Hq, i = bi - b * a.bl;
              a.lse[(static_cast<long>(b) * a.Hq + hq) * a.bl + i] = sum != 0.f ? (lg2(sum) + row_ref) * kLn2 : -INFINITY;
            }
          }
        }
        if (ok) ok = values_done(g * TPS - 1, at_once);
        tc_fence_after();
        named_bar_sync(kSoftBar + 1 + grp, 128);
        if (write) {  // here lane = channel
          const bool part = sh.seg[k].slot >= 0;
          float* const to = a.part_o + (static_cast<long>(sh.seg[k].slot) * rows + row0) * D + tok;
#pragma unroll 1
          for (int c = 0; c < CPT; c += kW) {
            float o[kW];
            tmem_load<kW>(tmem + lanes + Ly::kOCol + row0 + c, o);
            if (tok >= D) continue;
            if (part) {
#pragma unroll
              for (int e = 0; e < kW; ++e)
                if (row0 + c + e < rows) to[(c + e) * D] = o[e];
            } else {
#pragma unroll
              for (int e = 0; e < kW; ++e) {
                const int row = sh.out_row[row0 + c + e];
                if (row >= 0) a.out[static_cast<long>(row) * D + tok] = __float2bfloat16_rn(o[e] * sh.inv[row0 + c + e]);
              }
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.o_free);
        named_bar_sync(kSoftBar, Ro::kSoftThreads);  // the shared rows are free again
      }
    });
  } else {
    set_regs_down<Ro::kRegTail>();
    if (warp == Ro::kLoad) {
      int issued = 0;  // steps whose copies have been started
      batches(no_plan, [&](int count, int g, int, int) {
        // ---- records -> ring ---------------------------------------------------
        constexpr int kPageSteps = 32 / kStepRecs;  // steps whose page ids one load of the warp brings
        const int per = (1 << a.log2_page) / kRecTok;
#pragma unroll 1
        for (int k = 0; ok && k < count; ++k) {
          const Kv4Segment seg = sh.seg[k];
          const int n_tok = seg.len + a.bl;
          const int h = seg.unit / a.chunks;
          const int32_t* table = a.page_table + static_cast<long>(seg.b) * a.max_pages;
          const auto load_page = [&](int t) { return __ldg(table + (min(t, n_tok - 1) >> a.log2_page)); };
          // one load ahead: lane = record of the load
          int page_next = load_page(seg.begin * kStepTok + lane * kRecTok), page = 0;
#pragma unroll 1
          for (int i = seg.begin; i < seg.end; ++i, ++g) {
            const int in_load = (i - seg.begin) % kPageSteps;
            if (in_load == 0) {
              page = page_next;
              if (page < 0 || page >= a.num_pages) {
                atomicOr(a.err, NLD_DEVERR_PAGE_RANGE);
                page = min(max(page, 0), a.num_pages - 1);
              }
              page_next = load_page((i + kPageSteps) * kStepTok + lane * kRecTok);
            }
            const int st = g % kSt;
            if (g >= kSt) ok = warp_wait<true>(&sh.empty[st], (g / kSt - 1) & 1, a.err);
            if (!ok) break;
            const int t0 = i * kStepTok;
            const int recs = min(kStepRecs, (n_tok - t0 + kRecTok - 1) / kRecTok);
            if (lane == 0) mbar_arrive_expect_tx(&sh.full[st], recs * Rec<D>::kBytes);
            __syncwarp();
            const int mine = __shfl_sync(0xffffffffu, page, in_load * kStepRecs + (lane & (kStepRecs - 1)));
            if (lane < recs) {
              const size_t at = (static_cast<size_t>(mine) * a.Hkv + h) * per + (((t0 >> 4) + lane) & (per - 1));
              bulk_load(ring + st * Ly::kStageBytes + lane * Rec<D>::kBytes, a.pool + at * Rec<D>::kBytes,
                        Rec<D>::kBytes, &sh.full[st]);
            }
            issued = g + 1;
          }
        }
      });
      // every copy lands before the CTA ends, whatever became of its readers
      for (int i = max(0, issued - kSt); i < issued; ++i) warp_wait(&sh.full[i % kSt], (i / kSt) & 1, a.err);
    } else if (warp == Ro::kScores) {
      batches(no_plan, [&](int count, int g, int s0, int) {
        // ---- scores ------------------------------------------------------------
        constexpr uint32_t idesc = umma_idesc_bf16(128, NR, false);
#pragma unroll 1
        for (int k = 0; ok && k < count; ++k) {
          const int g_first = g, g_end = g + sh.seg[k].end - sh.seg[k].begin;
          ok = warp_wait(&sh.q_full, (s0 + k) & 1, a.err);
#pragma unroll 1
          for (; ok && g < g_end; ++g) {
#pragma unroll 1
            for (int p = 0; p < TPS; ++p) {
              const int tile = g * TPS + p, buf = tile % Ly::kKTiles;
              ok = warp_wait(&sh.k_full[buf], (tile / Ly::kKTiles) & 1, a.err);
              // the softmax has read this tile of the step before
              if (ok && g > g_first) ok = warp_wait(&sh.s_free[p], (g - 1) & 1, a.err);
              if (!ok) break;
              tc_fence_after();
              if (elect_one()) {
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
                  umma_bf16_ts(tmem + Ly::kSCol + p * NR, tmem + Ly::kKCol + buf * 64 + i * 8,
                               sw128_desc(smem_u32(sq) + (i >> 2) * (NR * 128) + (i & 3) * 32, 0, 1024), idesc, i > 0);
                umma_commit(&sh.s_done[p]);
                umma_commit(&sh.k_free[buf]);
              }
              __syncwarp();
            }
          }
        }
      });
      // no product is in flight when the columns are freed
      if (elect_one()) umma_commit(&sh.drain);
      __syncwarp();
      warp_wait(&sh.drain, 0, a.err);
    } else if (warp == Ro::kValues) {
      batches(no_plan, [&](int count, int g, int s0, int) {
        // ---- values ------------------------------------------------------------
        constexpr uint32_t idesc = umma_idesc_bf16(128, Ly::kORows, true);
#pragma unroll 1
        for (int k = 0; ok && k < count; ++k) {
          const int g_first = g, g_end = g + sh.seg[k].end - sh.seg[k].begin, s = s0 + k;
#pragma unroll 1
          for (; ok && g < g_end; ++g) {
            ok = warp_wait(&sh.p_full[g & 1], (g >> 1) & 1, a.err);
            if (ok && g == g_first && s > 0) ok = warp_wait(&sh.o_free, (s - 1) & 1, a.err);
#pragma unroll 1
            for (int p = 0; p < TPS; ++p) {
              const int tile = g * TPS + p, buf = tile % Ly::kVTiles;
              ok = ok && warp_wait(&sh.v_full[buf], (tile / Ly::kVTiles) & 1, a.err);
              if (!ok) break;
              tc_fence_after();
              if (elect_one()) {
                const uint32_t p_addr = smem_u32(sp) + (g & 1) * Ly::kPBytes + p * Ly::kPieceBytes;
#pragma unroll
                for (int i = 0; i < kTok / 16; ++i)
                  umma_bf16_ts(tmem + Ly::kOCol, tmem + Ly::kVCol + buf * 64 + i * 8,
                               sw128_desc(p_addr + i * 2048, Ly::kPieceBytes, 1024), idesc,
                               g > g_first || p > 0 || i > 0);
                umma_commit(&sh.pv_done[buf]);
              }
              __syncwarp();
            }
          }
        }
      });
      if (elect_one()) umma_commit(&sh.drain);
      __syncwarp();
      warp_wait(&sh.drain, 0, a.err);
    } else if (warp == Ro::kPlan) {
      Kv4Walk walk;
      batches(
          [&](int s0, int batch) {
            if (s0 == 0) {
              walk.start(sc, blockIdx.x, blockIdx.x, lane, a.err);
            }
            int k = 0;
            if (const int failed = sh.num_failed[batch ^ 1]; failed > 0) {
              Kv4Segment again{};
              if (lane < failed) again = sh.seg[sh.failed[lane]];
              __syncwarp();
              if (lane < failed) {
                sh.seg[2 * lane] = sh.seg[2 * lane + 1] = again;
                sh.mode[2 * lane] = kMaxima;
                sh.mode[2 * lane + 1] = kKnownMaxima;
              }
              k = 2 * failed;
            } else {
              Kv4Segment seg;
              for (int n = 0; n < kBatch && walk.next(&seg); ++n) {
                // the first token is visible to every row that sees anything after it, unless a table says otherwise
                const bool blind = a.mode == kModeBlockMask && seg.begin * kStepTok >= seg.len;
                if (lane == 0) {
                  sh.seg[k] = seg;
                  sh.mode[k] = blind ? kMaxima : kFirstToken;
                  if (blind) {
                    sh.seg[k + 1] = seg;
                    sh.mode[k + 1] = kKnownMaxima;
                  }
                }
                k += blind ? 2 : 1;
              }
            }
            __syncwarp();
            if (lane == 0) {
              sh.count = k;
              sh.last[batch] = walk.x >= walk.x_end;
              sh.num_failed[batch] = 0;
            }
          },
          [&](int, int, int s0, int) {
            if (s0 == 0 && blockIdx.x == 0 && a.plan != nullptr) walk.publish(a.plan, lane);
          });
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == Ro::kScores) tmem_dealloc(tmem, Ly::kCols);
}

template <int D, int NR, int TPS>
cudaError_t launch_t(const Kv4AttnArgs& a, int rows, cudaStream_t stream) {
  constexpr size_t kSmem = 1024 + Lay<D, NR, TPS>::kSmallOff + sizeof(Small<NR>);
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static int configured[64] = {0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!__atomic_load_n(&configured[dev], __ATOMIC_ACQUIRE)) {
    e = cudaFuncSetAttribute(block_attn_kv4_tc_kernel<D, NR, TPS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    __atomic_store_n(&configured[dev], 1, __ATOMIC_RELEASE);
  }
  return launch_kernel(block_attn_kv4_tc_kernel<D, NR, TPS>, dim3(a.ctas), dim3(Roles<NR, TPS>::kThreads), kSmem, stream, a, rows);
}

}  // namespace

// The least padding that the softmax groups' multiples of 8 rows and the value
// product's 16 allow: 78 rows padded to 96 take 267 us where 128 take 297, and
// 155 in one chunk of 160 take 236 where two of 96 take 267 (all in pieces).
cudaError_t launch_block_attn_kv4_tc(const Kv4AttnArgs& a, int D, int rows, cudaStream_t stream) {
  if (D == 128)
    return rows <= 32 ? launch_t<128, 32, 2>(a, rows, stream)
                      : rows <= 64 ? launch_t<128, 64, 2>(a, rows, stream)
           : rows <= 96 ? launch_t<128, 96, 1>(a, rows, stream)
           : rows <= 128 ? launch_t<128, 128, 1>(a, rows, stream) : launch_t<128, 160, 1>(a, rows, stream);
  return rows <= 32 ? launch_t<64, 32, 2>(a, rows, stream)
                    : rows <= 64 ? launch_t<64, 64, 2>(a, rows, stream)
         : rows <= 96 ? launch_t<64, 96, 1>(a, rows, stream)
         : rows <= 128 ? launch_t<64, 128, 1>(a, rows, stream) : launch_t<64, 160, 1>(a, rows, stream);
}

}  // namespace nld
