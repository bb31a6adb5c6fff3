// Block attention over the 4-bit paged cache: the kernel for up to 16 query
// rows per KV head (single tokens, short blocks), the merge of cut units and
// the choice between the kernels.
//
// K and V are dequantised in registers, straight into the operand fragments
// of mma.sync.m16n8k16 (bf16 inputs, fp32 sums), with the cache as the 16-row
// A operand and the query rows as columns, in one or two blocks of 8. The order
// of a product's k, and of the tokens in a score tile, is free as long as both
// operands use the same one, so each lane takes the packed words it can load
// whole. Over a tile of 64 tokens (4 records), lane (g, t) = (lane / 4, lane % 4):
//   scores S^T[16 tokens x 8 rows], step s of 4: rows g and g + 8 of A are
//     tokens 4 s + g % 2 and 4 s + 2 + g % 2 of record g / 2; the lane holds
//     channels D/4 t .. D/4 (t + 1), one contiguous piece of a K row and of
//     one scale group;
//   P: an 8 x 8 transpose across the warp turns the score fragment into the B
//     fragment in which lane (g, t) has tokens 4 s .. 4 s + 3 of record t;
//   values O^T[16 channels x 8 rows], step s: the lane holds those tokens of
//     channels g and g + 8, from the 8 bytes a record keeps for a channel.
// Softmax is online, per warp (running max and sum in fp32). All warps run the
// same code on tiles of their own. A warp has room for one tile in shared
// memory: the K half of its next tile is copied in (bulk copies) while it works
// on V, the V half while it works on K. With few units a CTA's warps share a
// piece and join their sums; with many each warp has a range of its own, and
// waits for no other.
// Bound: HBM by bytes; here the instructions (13 to dequantise 8 values, 1570 in
// all for a tile of 64 tokens) of three warps a scheduler. Measured, single tokens
// of 64 sequences of 512 to 8192 tokens (8 KV heads of 128, 347 MB of cache): 88
// us, 4.0 TB/s, an instruction issued in 61% of the cycles. Records loaded straight into registers: 222 us; units
// shared by a CTA's warps: 132 us; 16 warps, two spilled: 88 us.
#include "kv4.cuh"

namespace nld {
namespace {

constexpr int kFewRows = 16;                    // rows this kernel takes, in blocks of 8
// Warps of a CTA: what the registers hold with one block of rows, or two.
constexpr int warps_for(int blocks) { return blocks == 1 ? 12 : 8; }
constexpr int kTile = 64;                       // tokens per warp step, and per schedule unit
constexpr int kTileRecs = kTile / kRecTok;

// A warp's tile: four records, each padded by 32 bytes so that the same fields
// of the four lie in different banks.
template <int D>
struct Tile {
  static constexpr int kRecBytes = Rec<D>::kBytes + 32;
  static constexpr int kBytes = kTileRecs * kRecBytes;
};

template <int D, int NB>
struct Share {
  static constexpr int kWarps = warps_for(NB), kRows = 8 * NB;
  struct Warp {
    union {
      uint8_t tile[Tile<D>::kBytes];
      float o[kRows][D];  // a finished segment's sums
    };
    float m[kRows], l[kRows];
    uint64_t full[2];  // K half, V half
  } warp[kWarps];
};

__device__ __forceinline__ Kv4Sched schedule(const Kv4AttnArgs& a, int span) {
  const int max_len = static_cast<int>((static_cast<long>(a.max_pages) << a.log2_page) - a.bl);
  return {a.lens, a.B, a.Hkv * a.chunks, a.bl, span, max_len, a.ctas, a.workers, a.ranges_above, a.min_piece};
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Transpose of an 8 x 8 matrix of 16-bit values held two to a lane.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

template <int D, int NB>
__global__ void __launch_bounds__(warps_for(NB) * 32, 1) block_attn_kv4_kernel(Kv4AttnArgs a) {
  constexpr int kWarps = warps_for(NB), kRows = 8 * NB;
  extern __shared__ __align__(128) unsigned char smem_raw[];
  Share<D, NB>& sh = *reinterpret_cast<Share<D, NB>*>(smem_raw);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  grid_launch_dependents();
  typename Share<D, NB>::Warp& mine = sh.warp[warp];
  if (lane < 2) mbar_init(&mine.full[lane], 1);  // (used by this warp alone)
  fence_mbar_init();
  __syncwarp();
  grid_dependency_wait();
  constexpr int kWords = D / 32;  // words of a lane's piece of a K row
  constexpr int kMt = D / 16;     // channel tiles of a value product
  const int per = (1 << a.log2_page) / kRecTok;

  Kv4Walk walk;
  walk.start(schedule(a, kTile), blockIdx.x, blockIdx.x * kWarps + warp, lane, a.err);
  if (blockIdx.x == 0 && warp == 0 && a.plan != nullptr) walk.publish(a.plan, lane);
  const bool alone = walk.q == 0;  // this warp has its own segments
  const int first = alone ? 0 : warp, stride = alone ? 1 : kWarps;
  bool ok = true;  // false after a wait passed its limit: the rest is computed from what is there
  uint32_t phase = 0;
  uint8_t* const stage = mine.tile;
  Kv4Segment seg;
  while (walk.next(&seg)) {
    const int b = seg.b, h = seg.unit / a.chunks, chunk = seg.unit - h * a.chunks;
    const int L = seg.len, n_tok = L + a.bl, n = seg.end - seg.begin;
    const int32_t* table = a.page_table + static_cast<long>(b) * a.max_pages;

    // lanes r and r + 4: page of record r of tile i; then the copies of a half
    const auto page_of = [&](int i) {
      return lane < 2 * kTileRecs ? __ldg(table + (min(i * kTile + (lane & 3) * kRecTok, n_tok - 1) >> a.log2_page)) : 0;
    };
    const auto fill = [&](int i, int page, int half) {
      const int recs = min(kTileRecs, (n_tok - i * kTile + kRecTok - 1) / kRecTok);
      if (page < 0 || page >= a.num_pages) {
        atomicOr(a.err, NLD_DEVERR_PAGE_RANGE);
        page = min(max(page, 0), a.num_pages - 1);
      }
      if (lane == 0) mbar_arrive_expect_tx(&mine.full[half], recs * (Rec<D>::kBytes / 2));
      __syncwarp();
      if (lane < 2 * kTileRecs && (lane & 3) < recs) {  // lanes 0..3: codes; 4..7: scales
        const size_t at = (static_cast<size_t>(page) * a.Hkv + h) * per + ((i * kTileRecs + (lane & 3)) & (per - 1));
        const int off = lane < 4 ? half * Rec<D>::kVCode : half ? Rec<D>::kVScale : Rec<D>::kKScale;
        bulk_load(stage + (lane & 3) * Tile<D>::kRecBytes + off, a.pool + at * Rec<D>::kBytes + off,
                  lane < 4 ? Rec<D>::kVCode : Rec<D>::kVScale - Rec<D>::kKScale, &mine.full[half]);
      }
    };
    const auto wait = [&](int half, bool other_in_flight) {
      if (!ok) return;
      ok = __all_sync(0xffffffffu, mbar_wait(&mine.full[half], phase, a.err));
      if (!ok && other_in_flight) mbar_wait(&mine.full[half ^ 1], phase ^ half, a.err);
    };
    if (first < n && ok) {
      const int page = page_of(seg.begin + first);
      fill(seg.begin + first, page, 0);
      fill(seg.begin + first, page, 1);
    }

    // Q fragments (B): row g of a block, channels D/4 t + 4 s ..; masks of rows 2 t and 2 t + 1
    uint32_t qf[NB][2 * kWords][2], bits[NB][2];
    float o[NB][kMt][4], m[NB][2], l[NB][2];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int r = chunk * kRows + 8 * n + g, i = r / a.G;
      const __nv_bfloat16* src =
          a.q + ((static_cast<long>(b) * a.bl + i) * a.Hq + h * a.G + (r - i * a.G)) * D + (D / 4) * t;
#pragma unroll
      for (int v = 0; v < kWords; ++v) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (r < a.R) w = __ldg(reinterpret_cast<const uint4*>(src) + v);
        qf[n][2 * v][0] = w.x, qf[n][2 * v][1] = w.y, qf[n][2 * v + 1][0] = w.z, qf[n][2 * v + 1][1] = w.w;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r2 = chunk * kRows + 8 * n + 2 * t + e;
        bits[n][e] = r2 < a.R ? kv4_block_bits(a, r2 / a.G) : 0u;
        m[n][e] = kNoMax;
        l[n][e] = 0.f;
      }
#pragma unroll
      for (int i2 = 0; i2 < kMt; ++i2)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][i2][e] = 0.f;
    }

#pragma unroll 1
    for (int i = seg.begin + first; i < seg.end; i += stride) {
      const bool more = i + stride < seg.end;
      const int page = more ? page_of(i + stride) : 0;

      // scores
      float s[NB][4][4];
      wait(0, true);
      const uint8_t* krec = stage + (g >> 1) * Tile<D>::kRecBytes;
      const int grp = t * (D / 4) / kGroupCh;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t w[2][kWords], sa[2], sb[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int tok = 4 * j + 2 * e + (g & 1);
          const uint8_t* src = krec + tok * (D / 2) + Rec<D>::k_chunk(tok, grp) * 16 + (D == 64 ? (t & 1) * 8 : 0);
          if constexpr (D == 128) {
            const uint4 v = *reinterpret_cast<const uint4*>(src);
            w[e][0] = v.x, w[e][1] = v.y, w[e][2] = v.z, w[e][3] = v.w;
          } else {
            const uint2 v = *reinterpret_cast<const uint2*>(src);
            w[e][0] = v.x, w[e][1] = v.y;
          }
          const uint32_t ac =
              *reinterpret_cast<const uint32_t*>(krec + Rec<D>::kKScale + (tok * Rec<D>::kGroups + grp) * 4);
          sa[e] = dup_lo(ac), sb[e] = dup_hi(ac);
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) s[n][j][0] = s[n][j][1] = s[n][j][2] = s[n][j][3] = 0.f;
#pragma unroll
        for (int k = 0; k < kWords; ++k) {
          uint32_t x[4], y[4];
          kv4_pairs(w[0][k], x);
          kv4_pairs(w[1][k], y);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[e] = fma_bf16x2(x[e], sa[0], sb[0]);
            y[e] = fma_bf16x2(y[e], sa[1], sb[1]);
          }
#pragma unroll
          for (int n = 0; n < NB; ++n) {
            mma_bf16(s[n][j], x[0], y[0], x[1], y[1], qf[n][2 * k][0], qf[n][2 * k][1]);
            mma_bf16(s[n][j], x[2], y[2], x[3], y[3], qf[n][2 * k + 1][0], qf[n][2 * k + 1][1]);
          }
        }
      }

      __syncwarp();  // the K half has been read
      if (more && ok) {
        fence_proxy_async_smem();
        fill(i + stride, page, 0);
      }

      // softmax: rows 2 t and 2 t + 1 of a block; tokens of record g / 2
      const bool whole = (i + 1) * kTile <= L;  // every token is prefix
      const int slot0 = i * kTile + (g >> 1) * kRecTok + (g & 1) - L;  // slot of j = 0, e = 0; < 0: prefix
      uint32_t pb[NB][4][2];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        if (!whole) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int slot = slot0 + 4 * j + (e & 2);
              if (slot >= 0 && (slot >= 32 || !((bits[n][e & 1] >> slot) & 1u))) s[n][j][e] = -INFINITY;
            }
        }
        float f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = fmax3(fmax3(s[n][0][e], s[n][0][e + 2], s[n][1][e]),
                            fmax3(s[n][1][e + 2], s[n][2][e], s[n][2][e + 2]), fmaxf(s[n][3][e], s[n][3][e + 2]));
#pragma unroll
          for (int x = 4; x <= 16; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
          top = fmaxf(top * a.scale_log2, m[n][e]);
          f[e] = ex2(m[n][e] - top);
          m[n][e] = top;
          l[n][e] *= f[e];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[e] = ex2(fmaf(s[n][j][e], a.scale_log2, -m[n][e & 1]));
            l[n][e & 1] += p[e];
          }
          pb[n][j][0] = transpose8x8(pack_bf16(p[0], p[1]));  // P in bf16 for the tensor product; its sum stays in fp32
          pb[n][j][1] = transpose8x8(pack_bf16(p[2], p[3]));
        }
        if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
          for (int k = 0; k < kMt; ++k) {
            o[n][k][0] *= f[0], o[n][k][1] *= f[1];
            o[n][k][2] *= f[0], o[n][k][3] *= f[1];
          }
        }
      }

      // values: this lane's tokens are those of record t
      wait(1, more);
      const uint8_t* vrec = stage + t * Tile<D>::kRecBytes;
      const int have = n_tok - (i * kTile + t * kRecTok);  // tokens of record t that exist (may be <= 0)
#pragma unroll
      for (int gr = 0; gr < Rec<D>::kGroups; ++gr) {
        uint32_t va[8], vc[8];
        {
          const uint4* src = reinterpret_cast<const uint4*>(vrec + Rec<D>::kVScale + gr * 64);
          const uint4 a0 = src[0], a1 = src[1], c0 = src[2], c1 = src[3];
          va[0] = a0.x, va[1] = a0.y, va[2] = a0.z, va[3] = a0.w, va[4] = a1.x, va[5] = a1.y, va[6] = a1.z, va[7] = a1.w;
          vc[0] = c0.x, vc[1] = c0.y, vc[2] = c0.z, vc[3] = c0.w, vc[4] = c1.x, vc[5] = c1.y, vc[6] = c1.z, vc[7] = c1.w;
        }
        if (!whole) {  // cells past the end hold anything: their values become 0, not 0 * NaN
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const uint32_t live = have >= 2 * k + 2 ? 0xffffffffu : have == 2 * k + 1 ? 0x0000ffffu : 0u;
            va[k] &= live;
            vc[k] &= live;
          }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int mt = gr * 2 + u;
          const uint8_t* src = vrec + Rec<D>::kVCode + (mt * 16 + g) * 8;
          const uint2 lo = *reinterpret_cast<const uint2*>(src), hi = *reinterpret_cast<const uint2*>(src + 64);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            uint32_t x[4], y[4];
            kv4_pairs(half ? lo.y : lo.x, x);
            kv4_pairs(half ? hi.y : hi.x, y);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              x[e] = fma_bf16x2(x[e], va[4 * half + e], vc[4 * half + e]);
              y[e] = fma_bf16x2(y[e], va[4 * half + e], vc[4 * half + e]);
            }
#pragma unroll
            for (int n = 0; n < NB; ++n) {
              mma_bf16(o[n][mt], x[0], y[0], x[1], y[1], pb[n][2 * half][0], pb[n][2 * half][1]);
              mma_bf16(o[n][mt], x[2], y[2], x[3], y[3], pb[n][2 * half + 1][0], pb[n][2 * half + 1][1]);
            }
          }
        }
      }
      __syncwarp();  // the V half has been read
      if (more && ok) {
        fence_proxy_async_smem();
        fill(i + stride, page, 1);
      }
      phase ^= 1;
    }

    // the segment's sums go over this warp's tile, which has been used; its
    // warps' sums are joined and stored
#pragma unroll
    for (int n = 0; n < NB; ++n) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int row = 8 * n + 2 * t + e;
#pragma unroll
        for (int x = 4; x <= 16; x <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], x);
        if (g == 0) {
          mine.m[row] = m[n][e];
          mine.l[row] = l[n][e];
        }
#pragma unroll
        for (int k = 0; k < kMt; ++k) {
          mine.o[row][k * 16 + g] = o[n][k][e];
          mine.o[row][k * 16 + g + 8] = o[n][k][e + 2];
        }
      }
    }
    if (alone) __syncwarp(); else __syncthreads();
    const int w0 = alone ? warp : 0, w1 = alone ? warp + 1 : min(n, kWarps);  // warps that had a tile
    for (int idx = alone ? lane : threadIdx.x; idx < kRows * (D / 4); idx += alone ? 32 : kWarps * 32) {
      const int row = idx / (D / 4), d = (idx - row * (D / 4)) * 4;
      const int r = chunk * kRows + row;
      if (r >= a.R) continue;
      float mm = kNoMax;
      for (int w = w0; w < w1; ++w) mm = fmaxf(mm, sh.warp[w].m[row]);
      float ll = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int w = w0; w < w1; ++w) {
        const float c = ex2(sh.warp[w].m[row] - mm);
        ll = fmaf(c, sh.warp[w].l[row], ll);
        const float4 v = *reinterpret_cast<const float4*>(&sh.warp[w].o[row][d]);
        acc.x = fmaf(c, v.x, acc.x);
        acc.y = fmaf(c, v.y, acc.y);
        acc.z = fmaf(c, v.z, acc.z);
        acc.w = fmaf(c, v.w, acc.w);
      }
      if (seg.slot < 0) {
        const float inv = ll > 0.f ? 1.f / ll : 0.f;
        const int i = r / a.G, hq = h * a.G + (r - i * a.G);
        const long at = ((static_cast<long>(b) * a.bl + i) * a.Hq + hq) * D + d;
        *reinterpret_cast<uint2*>(a.out + at) =
            make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
        if (d == 0 && a.lse != nullptr)
          a.lse[(static_cast<long>(b) * a.Hq + hq) * a.bl + i] = ll > 0.f ? (mm + lg2(ll)) * kLn2 : -INFINITY;
      } else {
        const long pr = static_cast<long>(seg.slot) * kRows + row;
        *reinterpret_cast<float4*>(a.part_o + pr * D + d) = acc;
        if (d == 0) a.part_ml[pr] = make_float2(mm, ll);
      }
    }
    if (!alone) break;  // a CTA has one piece
    __syncwarp();
    fence_proxy_async_smem();  // the tile is written by copies again
  }
}

// Merge of the partials of units cut over several CTAs, one warp per output
// row: out = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.
constexpr int kMergeWarps = 4;

template <int D>
__global__ void __launch_bounds__(kMergeWarps * 32) kv4_merge_kernel(Kv4AttnArgs a, int rows, int span) {
  grid_launch_dependents();
  grid_dependency_wait();
  constexpr int V = D / 32;
  const int lane = threadIdx.x & 31;
  const long row = static_cast<long>(blockIdx.x) * kMergeWarps + (threadIdx.x >> 5);
  const long per_seq = static_cast<long>(a.Hkv) * a.R;
  if (row >= a.B * per_seq) return;
  const int b = static_cast<int>(row / per_seq);
  const int in_seq = static_cast<int>(row - b * per_seq);
  const int h = in_seq / a.R, r = in_seq - h * a.R;
  const int chunk = r / rows;
  const Kv4Sched sc = schedule(a, span);
  const int q = a.plan[0], tot = a.plan[1], before = a.plan[2 + b];
  const int cnt = sc.count(sc.spans(b), q);
  const int first = before + (h * a.chunks + chunk) * cnt;  // first piece or span
  int c0, c1;  // workers first to last
  if (q > 0) {
    c0 = first;
    c1 = c0 + cnt - 1;
  } else {
    c0 = sc.range_owner(tot, first);
    c1 = sc.range_owner(tot, first + cnt - 1);
  }
  if (c0 == c1) return;  // written by its one worker
  const int n = c1 - c0 + 1;
  const auto slot_row = [&](int k) {
    const int slot = 2 * (c0 + k) + (q == 0 && k == 0 ? 1 : 0);
    return static_cast<long>(slot) * rows + (r - chunk * rows);
  };
  // rounds of 16 partials, all of a round's loads in flight at once; the sums
  // are rescaled when a round raises the maximum
  constexpr int kRound = 16;
  float mm = kNoMax, acc[V], ll = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) acc[v] = 0.f;
#pragma unroll 1
  for (int k0 = 0; k0 < n; k0 += kRound) {
    float x[kRound][V];
#pragma unroll
    for (int k = 0; k < kRound; ++k) {
      const float* src = a.part_o + slot_row(min(k0 + k, n - 1)) * D + lane * V;
      if constexpr (V == 4) {
        const float4 v = *reinterpret_cast<const float4*>(src);
        x[k][0] = v.x, x[k][1] = v.y, x[k][2] = v.z, x[k][3] = v.w;
      } else {
        const float2 v = *reinterpret_cast<const float2*>(src);
        x[k][0] = v.x, x[k][1] = v.y;
      }
    }
    float2 ml = make_float2(kNoMax, 0.f);
    if (lane < kRound && k0 + lane < n) ml = a.part_ml[slot_row(k0 + lane)];
    float top = fmaxf(mm, ml.x);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    top = __shfl_sync(0xffffffffu, top, 0);
    const float f = ex2(mm - top), w = lane < kRound && k0 + lane < n ? ex2(ml.x - top) : 0.f;
    mm = top;
    ll = fmaf(ll, f, w * ml.y);
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] *= f;
#pragma unroll
    for (int k = 0; k < kRound; ++k) {
      const float wk = __shfl_sync(0xffffffffu, w, k);
#pragma unroll
      for (int v = 0; v < V; ++v) acc[v] = fmaf(wk, x[k][v], acc[v]);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, o);
  const float inv = ll > 0.f ? 1.f / ll : 0.f;
  const int i = r / a.G, hq = h * a.G + (r - i * a.G);
  __nv_bfloat16* dst = a.out + ((static_cast<long>(b) * a.bl + i) * a.Hq + hq) * D + lane * V;
#pragma unroll
  for (int v = 0; v < V; v += 2) *reinterpret_cast<uint32_t*>(dst + v) = pack_bf16(acc[v] * inv, acc[v + 1] * inv);
  if (a.lse != nullptr && lane == 0)
    a.lse[(static_cast<long>(b) * a.Hq + hq) * a.bl + i] = ll > 0.f ? (mm + lg2(ll)) * kLn2 : -INFINITY;
}

template <int D, int NB>
cudaError_t launch_few(const Kv4AttnArgs& a, cudaStream_t stream) {
  static_assert(sizeof(Share<D, NB>) <= 227 * 1024, "shared memory");
  static int configured[64] = {0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!__atomic_load_n(&configured[dev], __ATOMIC_ACQUIRE)) {
    e = cudaFuncSetAttribute(block_attn_kv4_kernel<D, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             sizeof(Share<D, NB>));
    if (e != cudaSuccess) return e;
    __atomic_store_n(&configured[dev], 1, __ATOMIC_RELEASE);
  }
  return launch_kernel(block_attn_kv4_kernel<D, NB>, dim3(a.ctas), dim3(warps_for(NB) * 32), sizeof(Share<D, NB>),
                       stream, a);
}

template <int D>
cudaError_t launch_d(const Kv4AttnArgs& a, bool merge, cudaStream_t stream) {
  const cudaError_t e = !a.few ? launch_block_attn_kv4_tc(a, D, a.rows, stream)
                        : a.rows == 8 ? launch_few<D, 1>(a, stream) : launch_few<D, 2>(a, stream);
  if (e != cudaSuccess || !merge) return e;
  const long rows = static_cast<long>(a.B) * a.Hkv * a.R;
  return launch_kernel(kv4_merge_kernel<D>, dim3(static_cast<unsigned>((rows + kMergeWarps - 1) / kMergeWarps)),
                       dim3(kMergeWarps * 32), 0, stream, a, a.rows, a.span);
}

}  // namespace

// Up to 16 rows: the register kernel dequantises each tile once and its warps
// need no hand-overs (64 sequences of 512 to 8192 tokens, 8 KV heads of 128: 4
// rows 88 us, 12 rows 136, 16 rows 146; the tcgen05 kernel 162 to 166 us). With
// more rows its registers do not hold the sums, so they go to the tcgen05
// kernel: up to 160 rows in one chunk, the rest in two equal ones, with steps
// of 256 tokens for up to 64 rows and 128 tokens beyond. But where the page
// table holds so few tokens that a unit is over in one step, that kernel's chain
// from unit to unit costs more than dequantising again for every 16 rows, as
// long as these are few: 48 rows of 83 sequences of up to 52 tokens (3 tiles of
// 16 rows) take 31 us, with the tcgen05 kernel 59; 160 rows of 49 sequences of up
// to 37 tokens (10 tiles) 59 us and 44.
//
// The register kernel's schedule: ranges of single warps once they cut a unit
// into about 16 or fewer (what the merge reads in one go); with fewer units,
// pieces of CTAs, of at least 8 tiles: two warps to a scheduler hardly slow each
// other down, and a short unit needs no merge (1000 tokens of 4 sequences: 10.4
// us; pieces of 1 tile 11.1, of 12 tiles 11.3). In the other kernel a CTA is one
// worker.
Kv4Shape kv4_attn_shape(int R, long tokens, int sms) {
  const long tiles = (tokens + kTile - 1) / kTile, blocks = (R + kFewRows - 1) / kFewRows;
  if (blocks == 1 || blocks * tiles <= 4) {
    const int warps = warps_for(R <= 8 ? 1 : 2);
    return {true, R <= 8 ? 8 : kFewRows, kTile, warps, sms * warps / 16, 8};
  }
  const int chunks = R <= 160 ? 1 : 2, rows = (R + chunks - 1) / chunks;
  return {false, rows, rows <= 64 ? 256 : 128, 1, sms, 1};
}

cudaError_t launch_block_attn_kv4(const Kv4AttnArgs& a, int D, bool merge, cudaStream_t stream) {
  return D == 128 ? launch_d<128>(a, merge, stream) : launch_d<64>(a, merge, stream);
}

}  // namespace nld
