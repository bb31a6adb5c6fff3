// Appends to the paged caches with the rotary position rotation applied on
// the way, and the read-back of the 4-bit cache.
//
// Rotation of a pair (x1, x2) at position p with angle p f_i, from a table of
// cosines and sines: (x1 c - x2 s, x2 c + x1 s), in fp32 (products and the
// difference each rounded, so that the result does not depend on contraction),
// then rounded to bf16 as the cache and the attention take it.
//
// Everything here streams its rows once; the kernels are bound by HBM on long
// prompts and by launch and dependent-load latency on single blocks. The bf16
// append of prompts of up to 8192 rows (28,000 rows, 32 and 8 heads of 128)
// takes 110 us, 6.4 TB/s; with a thread's items in any order of heads, each
// loading its cosines and sines, it took 122 us.
#include "kv4.cuh"

namespace nld {
namespace {

constexpr int kRowThreads = 128;
constexpr int kGroupWarps = kRowThreads / 32;
constexpr long kUnitCtas = 8 * 152;
constexpr int kReadRowBytes = 512;  // of a row that a CTA of the read-back puts together

__device__ __forceinline__ float4 ldg_f4(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }

struct Vec8 {
  float x[8];
};

__device__ __forceinline__ Vec8 unpack8(uint4 w) {
  Vec8 r;
  unpack_bf16(w.x, r.x[0], r.x[1]);
  unpack_bf16(w.y, r.x[2], r.x[3]);
  unpack_bf16(w.z, r.x[4], r.x[5]);
  unpack_bf16(w.w, r.x[6], r.x[7]);
  return r;
}

__device__ __forceinline__ uint4 pack8(const Vec8& v) {
  return make_uint4(pack_bf16(v.x[0], v.x[1]), pack_bf16(v.x[2], v.x[3]), pack_bf16(v.x[4], v.x[5]),
                    pack_bf16(v.x[6], v.x[7]));
}

__device__ __forceinline__ Vec8 load_f8(const float* p) {
  const float4 a = ldg_f4(p), b = ldg_f4(p + 4);
  return Vec8{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}

// x c - y s and x c + y s, every operation rounded on its own.
__device__ __forceinline__ float turn_lo(float x, float y, float c, float s) {
  return __fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s));
}
__device__ __forceinline__ float turn_hi(float x, float y, float c, float s) {
  return __fadd_rn(__fmul_rn(x, c), __fmul_rn(y, s));
}

// Pairs inside one vector (interleaved order): cos/sin of the vector's 4 pairs.
__device__ __forceinline__ void turn_within(Vec8& v, const float* c, const float* s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = v.x[2 * i], b = v.x[2 * i + 1];
    v.x[2 * i] = turn_lo(a, b, c[i], s[i]);
    v.x[2 * i + 1] = turn_hi(b, a, c[i], s[i]);
  }
}

// Position of packed row r, clamped into the table.
__device__ __forceinline__ long row_position(const AppendArgs& a, long r, long t) {
  long p = a.positions != nullptr ? static_cast<long>(__ldg(a.positions + r)) : t;
  if (a.rot > 0 && (p < 0 || p >= a.max_positions)) {
    atomicOr(a.err, NLD_DEVERR_POSITION_RANGE);
    p = p < 0 ? 0 : a.max_positions - 1;
  }
  return p;
}

// First packed row of sequence b.
__device__ __forceinline__ long row_begin(const AppendArgs& a, int b) {
  if (a.cu == nullptr) return static_cast<long>(b) * (a.T / a.B);
  return min(max(static_cast<long>(__ldg(a.cu + b)), 0l), a.T);
}

// lens + new rows, by one warp or more of the grid.
__device__ __forceinline__ void write_lens(const AppendArgs& a, int first, int step) {
  for (int b = first; b < a.B; b += step)
    a.new_lens[b] = a.lens[b] + static_cast<int>(max(row_begin(a, b + 1) - row_begin(a, b), 0l));
}

// The rows belong to sequences only as cu_tokens says: it has to ascend from 0
// to T. Its entries are dealt to the grid's threads, after their rows' work, so
// that nothing waits for these loads.
__device__ __forceinline__ void check_cover(const AppendArgs& a) {
  if (a.cu == nullptr) return;
  const long threads = static_cast<long>(gridDim.x) * kRowThreads;
  for (long i = static_cast<long>(blockIdx.x) * kRowThreads + threadIdx.x; i <= a.B; i += threads) {
    const int at = __ldg(a.cu + i), before = i > 0 ? __ldg(a.cu + i - 1) : 0;
    if (at < before || (i == 0 && at != 0) || (i == a.B && at != a.T)) atomicOr(a.err, NLD_DEVERR_PREFIX_RANGE);
  }
}

// `threads` threads (a warp or a CTA; tid is the one's number) rotate or copy
// the heads of packed row r: the queries (when present), then K, then V.
template <bool kWithKv>
__device__ __forceinline__ void append_row(const AppendArgs& a, long r, int tid, int threads) {
  const int lane = threadIdx.x & 31;
  const int b = a.cu == nullptr
                    ? static_cast<int>(r / (a.T / a.B))
                    : warp_last_le(a.B, r, lane, [&](int i) { return static_cast<long>(__ldg(a.cu + i)); });
  const long r0 = row_begin(a, b);
  if (r < r0 || r >= row_begin(a, b + 1)) {  // cu_tokens does not cover the row
    if (tid == 0) atomicOr(a.err, NLD_DEVERR_PREFIX_RANGE);
    return;
  }
  const long t = static_cast<long>(__ldg(a.lens + b)) + (r - r0);
  const long pos = row_position(a, r, t);
  long cell = -1;  // (page * Hkv * P + slot) * D, head 0
  if (kWithKv) {
    if (t < 0 || t >= static_cast<long>(a.max_pages) * a.P) {
      if (tid == 0) atomicOr(a.err, NLD_DEVERR_PREFIX_RANGE);
    } else {
      const int page = __ldg(a.page_table + static_cast<long>(b) * a.max_pages + (t >> a.log2_page));
      if (page < 0 || page >= a.num_pages) {
        if (tid == 0) atomicOr(a.err, NLD_DEVERR_PAGE_RANGE);
      } else {
        cell = (static_cast<long>(page) * a.Hkv * a.P + (t & (a.P - 1))) * a.D;
      }
    }
  }
  // this thread's 16 channels of every step-th head: two vectors at d0 and d1,
  // whose cosines and sines stay in registers
  const int hq = a.q != nullptr ? a.Hq : 0, heads = kWithKv ? hq + 2 * a.Hkv : hq;
  const int per_head = a.D / 16, step = threads / per_head;
  const int h0 = tid / per_head, i = tid - h0 * per_head;
  const bool halves = !a.interleaved && i < a.rot / 16, within = a.interleaved && i < a.rot / 16;
  const int d0 = halves ? 8 * i : 16 * i, d1 = halves ? d0 + a.rot / 2 : d0 + 8;
  Vec8 c, s;
  if (halves || within) {
    const float* cs = a.rope + pos * a.rot + (halves ? d0 : d0 / 2);
    c = load_f8(cs);
    s = load_f8(cs + a.rot / 2);
  }
  for (int h = h0; h < heads; h += step) {
    const __nv_bfloat16* src;
    __nv_bfloat16* dst;
    const bool turns = h < hq + a.Hkv;
    if (h < hq) {
      src = a.q + r * a.q_stride + h * a.D;
      dst = a.q_out + (r * a.Hq + h) * a.D;
    } else {
      if (cell < 0) break;
      const int kh = h - hq - (turns ? 0 : a.Hkv);
      src = turns ? a.k + r * a.k_stride + kh * a.D : a.v + r * a.v_stride + kh * a.D;
      dst = (turns ? a.k_pages : a.v_pages) + cell + static_cast<long>(kh) * a.P * a.D;
    }
    // (may be rotated in place: not the read-only path)
    uint4 w0 = *reinterpret_cast<const uint4*>(src + d0), w1 = *reinterpret_cast<const uint4*>(src + d1);
    if (turns && (halves || within)) {  // else the bits as they are, a NaN's too
      Vec8 x = unpack8(w0), y = unpack8(w1);
      if (halves) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float lo = x.x[e], hi = y.x[e];
          x.x[e] = turn_lo(lo, hi, c.x[e], s.x[e]);
          y.x[e] = turn_hi(hi, lo, c.x[e], s.x[e]);
        }
      } else {
        turn_within(x, c.x, s.x);
        turn_within(y, c.x + 4, s.x + 4);
      }
      w0 = pack8(x);
      w1 = pack8(y);
    }
    *reinterpret_cast<uint4*>(dst + d0) = w0;
    *reinterpret_cast<uint4*>(dst + d1) = w1;
  }
}

// The rows of block `block`: one, or one per warp.
template <bool kWithKv>
__device__ __forceinline__ void append_rows(const AppendArgs& a, unsigned block, int by_warp) {
  if (!by_warp) {
    append_row<kWithKv>(a, block, threadIdx.x, kRowThreads);
  } else {
    const long r = static_cast<long>(block) * kGroupWarps + (threadIdx.x >> 5);
    if (r < a.T) append_row<kWithKv>(a, r, threadIdx.x & 31, 32);
  }
}

// Rows in great number go to warps: a CTA's turn costs more than a narrow row's
// work (23185 rows of 4 and 1 heads of 64: 15 us, with a CTA each 38), and the
// lookups are made by fewer threads (28,000 rows of 32 and 8 heads of 128: 109 us
// and 113). Few rows keep a CTA each, for the shorter chain.
bool rows_by_warp(const AppendArgs& a) { return a.T >= 16 * 152; }
long row_blocks(long T, bool by_warp) { return by_warp ? (T + kGroupWarps - 1) / kGroupWarps : T; }

__global__ void __launch_bounds__(kRowThreads) rope_append_kernel(AppendArgs a, int by_warp) {
  grid_launch_dependents();
  grid_dependency_wait();  // the rows, lengths and tables come from earlier kernels
  if (a.fuse_lens && blockIdx.x == 0) write_lens(a, threadIdx.x, kRowThreads);
  append_rows<true>(a, blockIdx.x, by_warp);
  check_cover(a);
}

__global__ void __launch_bounds__(kRowThreads) advance_lens_kernel(AppendArgs a) {
  grid_launch_dependents();
  grid_dependency_wait();  // every append has read the old lengths
  write_lens(a, blockIdx.x * kRowThreads + threadIdx.x, gridDim.x * kRowThreads);
}

// ---------------------------------------------------------------------------
// 4-bit records
// ---------------------------------------------------------------------------

// A CTA's work on the 4-bit cache: one record's 16 slots of a sequence, for all
// KV heads or a share of them (what is looked up, and the rotation's cosines
// and sines, serve every head). A warp takes one group of 32 channels; a lane
// takes 8 channels (chunk lane / 8) of two tokens, unit_token(lane) and 8 more.
struct UnitTask {
  long row, t;     // packed row and slot of the record's first token
  int lo, hi;      // tokens [lo, hi) of the record are rows of the call
  bool page_ok;    // their slots lie in the page table, on a page of the pool
  size_t rec;      // byte offset of the record of head 0
  size_t head;     // bytes between heads
};

// Token t of 8 has nibble (t & 1) * 4 + t / 2 of a V word, and so has channel
// t of 8 in a K word: lane i of 8 takes the token (channel) of nibble i.
__device__ __forceinline__ int unit_token(int lane) { return ((lane >> 2) & 1) | ((lane & 3) << 1); }

// Records a sequence of n rows touches: at most n / 16 + 2. Sequence b's
// units start at (cu_b >> 4) + 2 b (ragged) or b (n / 16 + 2) (equal counts),
// both ascending with at least that many units between neighbours.
__host__ __device__ __forceinline__ long record_units(long T, int B, bool ragged) {
  return ragged ? (T >> 4) + 2l * B : static_cast<long>(B) * ((T / B) / 16 + 2);
}

// False if unit u holds no row of the call.
template <int D>
__device__ __forceinline__ bool unit_task(const AppendArgs& a, long u, int lane, UnitTask* o) {
  long first;  // first unit of the sequence
  int b;
  if (a.cu == nullptr) {
    const long per = (a.T / a.B) / 16 + 2;
    b = static_cast<int>(u / per);
    first = b * per;
  } else {
    b = warp_last_le(a.B, u, lane, [&](int i) { return (row_begin(a, i) >> 4) + 2l * i; });
    first = (row_begin(a, b) >> 4) + 2l * b;
  }
  const long r0 = row_begin(a, b), r1 = row_begin(a, b + 1);
  const long L = a.lens != nullptr ? static_cast<long>(__ldg(a.lens + b)) : 0;
  const long rec = (L >> 4) + (u - first), t0 = rec * kRecTok;
  o->t = t0;
  o->row = r0 + (t0 - L);
  o->lo = static_cast<int>(min(max(L - t0, 0l), 16l));
  o->hi = static_cast<int>(min(max(r1 - o->row, 0l), 16l));
  const bool any = o->lo < o->hi;
  o->page_ok = L >= 0 && t0 < static_cast<long>(a.max_pages) * a.P;  // a record lies in one page
  if (!o->page_ok && (any || L < 0) && lane == 0) atomicOr(a.err, NLD_DEVERR_PREFIX_RANGE);
  if (!any) return false;
  int page = 0;
  if (o->page_ok) {
    page = __ldg(a.page_table + static_cast<long>(b) * a.max_pages + (t0 >> a.log2_page));
    if (page < 0 || page >= a.num_pages) {
      if (lane == 0) atomicOr(a.err, NLD_DEVERR_PAGE_RANGE);
      o->page_ok = false;
      page = 0;
    }
  }
  o->head = static_cast<size_t>(a.P / kRecTok) * Rec<D>::kBytes;
  o->rec = static_cast<size_t>(page) * a.Hkv * o->head + static_cast<size_t>((t0 & (a.P - 1)) >> 4) * Rec<D>::kBytes;
  return true;
}

// Transpose 8 x 8 nibbles over 8 lanes: nibble j of lane i becomes nibble i of lane j.
__device__ __forceinline__ uint32_t transpose_nibbles(uint32_t w, int lane) {
#pragma unroll
  for (int s = 1; s <= 4; s <<= 1) {
    const uint32_t m = s == 1 ? 0xF0F0F0F0u : s == 2 ? 0xFF00FF00u : 0xFFFF0000u;  // columns with bit s
    const uint32_t p = __shfl_xor_sync(0xffffffffu, w, s);
    w = (lane & s) ? ((w & m) | ((p >> (4 * s)) & ~m)) : ((w & ~m) | ((p << (4 * s)) & m));
  }
  return w;
}

__device__ __forceinline__ float rcp_estimate(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {  // NaN if either is
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// NaN to 0, and the magnitude cut at kKv4Limit.
__device__ __forceinline__ uint32_t tame_bf16x2(uint32_t w) {
  float lo, hi;
  unpack_bf16(w, lo, hi);
  lo = lo != lo ? 0.f : fminf(fmaxf(lo, -kKv4Limit), kKv4Limit);
  hi = hi != hi ? 0.f : fminf(fmaxf(hi, -kKv4Limit), kKv4Limit);
  return pack_bf16(lo, hi);  // exact: the limit is a power of two
}

// Least and largest of this lane's group (the 4 lanes of the same token), in bf16, exact.
__device__ __forceinline__ void group_range(uint4 w, float& mn, float& mx) {
  uint32_t lo = min_bf16x2(min_bf16x2(w.x, w.y), min_bf16x2(w.z, w.w));
  uint32_t hi = max_bf16x2(max_bf16x2(w.x, w.y), max_bf16x2(w.z, w.w));
#pragma unroll
  for (int o = 8; o <= 16; o <<= 1) {
    lo = min_bf16x2(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max_bf16x2(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  lo = min_bf16x2(lo, __byte_perm(lo, lo, 0x1032));
  hi = max_bf16x2(hi, __byte_perm(hi, hi, 0x1032));
  mn = __uint_as_float(lo & 0xffff0000u);
  mx = __uint_as_float(hi & 0xffff0000u);
}

// Quantise this lane's 8 values with its group: a word in storage order,
// (a, c) as a packed pair. Warp-collective.
//
// A code is d / step rounded to the nearest, ties to even, exactly; step has 8
// significant bits, so the midpoints (k + 1/2) step are exact. An estimate
// with a reciprocal that is too large by 2^-20 rounds to that code or, from at
// or just below a midpoint, to the next one; the remainder d - k step, exact
// near -step / 2, tells which. All of it runs on the pipes of multiplications
// and additions, where a division and two conversions per value did not.
__device__ __forceinline__ uint32_t quantise_group(uint4 v, bool valid, unsigned int* err, uint32_t* scale) {
  float mn, mx;
  group_range(v, mn, mx);
  if (__any_sync(0xffffffffu, !(mn >= -kKv4Limit && mx <= kKv4Limit))) {  // (also for NaN)
    if (valid && !(mn >= -kKv4Limit && mx <= kKv4Limit)) atomicOr(err, NLD_DEVERR_NONFINITE);
    v = make_uint4(tame_bf16x2(v.x), tame_bf16x2(v.y), tame_bf16x2(v.z), tame_bf16x2(v.w));
    group_range(v, mn, mx);
  }
  const float range = __fsub_rn(mx, mn);
  const bool flat = range < kKv4Flat;
  const __nv_bfloat16 a16 = __float2bfloat16_rn(flat ? 0.f : __fmul_rn(range, 16.0f / 15.0f));
  const float a = __bfloat162float(a16);
  const __nv_bfloat16 c16 = __float2bfloat16_rn(__fsub_rn(mn, a));
  const float low = __fadd_rn(a, __bfloat162float(c16));
  const float step = a * 0.0625f, half = a * 0.03125f;  // exact
  constexpr float kTop = 15.46875f;                      // estimates saturate here: code 15
  constexpr float kRound = 12582912.f;                   // 1.5 2^23: an integer is in the low bits of the sum
  const float inv = flat ? 0.f : rcp_estimate(step) * ((1.f + 0x1p-20f) / kTop);
  const Vec8 x = unpack8(v);
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float d = fmaxf(__fsub_rn(x.x[e], low), 0.f);
    const float t = __fmaf_rn(__saturatef(d * inv), kTop, kRound);
    const uint32_t k = __float_as_uint(t);
    const float rem = __fmaf_rn(__fsub_rn(kRound, t), step, d);
    // at the midpoint itself an odd code goes down, an even one stays
    const float mid = __uint_as_float(__float_as_uint(half) - (k & 1u));
    const uint32_t code = rem < -mid ? k - 1 : k;
    w += code << (4 * ((e & 1) * 4 + (e >> 1)));
  }
  *scale = static_cast<uint32_t>(__bfloat16_as_ushort(a16)) | (static_cast<uint32_t>(__bfloat16_as_ushort(c16)) << 16);
  constexpr uint32_t kBits = 0x4B400000u * 0x11111111u;  // of kRound, in every nibble's place
  return flat ? 0u : w - kBits;
}

// Cosines and sines of a lane's 8 channels of one row, the sines with the sign
// with which the partner enters: x' = x c + p s, each operation rounded on its own.
__device__ __forceinline__ void load_turn(const AppendArgs& a, long pos, int ch, float (&c)[8], float (&s)[8]) {
  const float* cs = a.rope + pos * a.rot;
  const int half = a.rot / 2;
  if (a.interleaved) {
    const float4 c4 = ldg_f4(cs + ch / 2), s4 = ldg_f4(cs + half + ch / 2);
    c[0] = c[1] = c4.x, c[2] = c[3] = c4.y, c[4] = c[5] = c4.z, c[6] = c[7] = c4.w;
    s[0] = -s4.x, s[1] = s4.x, s[2] = -s4.y, s[3] = s4.y, s[4] = -s4.z, s[5] = s4.z, s[6] = -s4.w, s[7] = s4.w;
    return;
  }
  const bool low = ch < half;
  const int f = low ? ch : ch - half;
  const Vec8 cv = load_f8(cs + f), sv = load_f8(cs + half + f);
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e] = cv.x[e], s[e] = low ? -sv.x[e] : sv.x[e];
}

// 8 of a unit's tokens, a part of its heads.
template <int D>
__device__ __forceinline__ void append_unit(const AppendArgs& a, long u, int second, int part, int parts) {
  constexpr int kWays = kGroupWarps / Rec<D>::kGroups;  // warps that take the same group of different heads
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = warp % Rec<D>::kGroups;
  UnitTask k;
  if (!unit_task<D>(a, u, lane, &k) || !k.page_ok) return;
  if (k.lo >= 8 * second + 8 || k.hi <= 8 * second) return;
  uint32_t keep = 0;  // nibbles of a V word that belong to rows of this call
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const int tok = unit_token(t) + 8 * second;
    if (tok >= k.lo && tok < k.hi) keep |= 15u << (4 * t);
  }
  const int token = unit_token(lane), tok = token + 8 * second;
  const bool valid = tok >= k.lo && tok < k.hi;
  const int chunk = lane >> 3, ch = g * kGroupCh + chunk * 8;
  const bool turns = valid && ch < a.rot;
  const int partner = ch < a.rot / 2 ? a.rot / 2 : -(a.rot / 2);
  const long row = k.row + tok;
  float c[8], s[8];
  if (turns) load_turn(a, row_position(a, row, k.t + tok), ch, c, s);
  const __nv_bfloat16* ksrc = a.k + row * a.k_stride + ch;
  const __nv_bfloat16* vsrc = a.v + row * a.v_stride + ch;
#pragma unroll 1
  for (int h = part * kWays + warp / Rec<D>::kGroups; h < a.Hkv; h += parts * kWays) {
    uint4 xk = make_uint4(0, 0, 0, 0), xp = xk, xv = xk;
    if (valid) {
      xk = __ldg(reinterpret_cast<const uint4*>(ksrc + h * D));
      if (turns && !a.interleaved) xp = __ldg(reinterpret_cast<const uint4*>(ksrc + h * D + partner));
      xv = __ldg(reinterpret_cast<const uint4*>(vsrc + h * D));
    }
    if (turns) {
      Vec8 x = unpack8(xk), p = unpack8(xp);
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p.x[e] = x.x[e ^ 1];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) p.x[e] = turn_hi(x.x[e], p.x[e], c[e], s[e]);
      xk = pack8(p);
    }
    uint32_t ks, vs;
    const uint32_t kw = quantise_group(xk, valid, a.err, &ks);
    uint32_t vw = transpose_nibbles(quantise_group(xv, valid, a.err, &vs), lane);
    uint8_t* rec = a.pool + k.rec + h * k.head;
    if (valid) {
      *reinterpret_cast<uint32_t*>(rec + tok * (D / 2) + Rec<D>::k_chunk(tok, g) * 16 + chunk * 4) = kw;
      if (chunk == 0) {
        *reinterpret_cast<uint32_t*>(rec + Rec<D>::kKScale + (tok * Rec<D>::kGroups + g) * 4) = ks;
        uint16_t* sc = reinterpret_cast<uint16_t*>(rec + Rec<D>::kVScale + g * 64) + tok;
        sc[0] = static_cast<uint16_t>(vs);
        sc[16] = static_cast<uint16_t>(vs >> 16);
      }
    }
    // transposed: this lane has the chunk's channel `token`
    uint32_t* dst = reinterpret_cast<uint32_t*>(rec + Rec<D>::kVCode + (ch + token) * 8) + second;
    if (keep != 0xffffffffu) vw = (*dst & ~keep) | (vw & keep);
    *dst = vw;
  }
}

// CTAs that rotate the queries of one packed row each and CTAs that quantise,
// one of these after every `gap` of those: the first wait for memory, the
// second for issue slots, so an SM should hold both. Prompts of up to 4096 rows
// (8 sequences, 18,000 rows, 32 and 8 heads of 128), with their read-back:
// 104 us, at 48 registers 2% more, at 64 5%. Bound: issue slots next to HBM (63%
// and 55% used).
template <int D>
__global__ void __launch_bounds__(kRowThreads, 9) rope_append_kv4_kernel(AppendArgs a, unsigned gap, unsigned units,
                                                                          unsigned parts, int by_warp) {
  grid_launch_dependents();
  grid_dependency_wait();
  if (a.fuse_lens && blockIdx.x == 0) write_lens(a, threadIdx.x, kRowThreads);
  const unsigned before = (blockIdx.x + gap) / (gap + 1);  // quantising CTAs before this one, were there no end to them
  if (blockIdx.x % (gap + 1) == 0 && before < units * 2 * parts) {
    const unsigned u2 = before / parts;
    append_unit<D>(a, u2 >> 1, u2 & 1, before - u2 * parts, parts);
  } else {
    append_rows<false>(a, blockIdx.x - min(before, units * 2 * parts), by_warp);
  }
  check_cover(a);
}

// Values of a word in storage order with one (a, c) pair for all.
__device__ __forceinline__ uint4 word_values(uint32_t w, uint32_t scale) {
  const uint32_t a = dup_lo(scale), c = dup_hi(scale);
  uint32_t y[4];
  kv4_pairs(w, y);
  return make_uint4(fma_bf16x2(y[0], a, c), fma_bf16x2(y[1], a, c), fma_bf16x2(y[2], a, c), fma_bf16x2(y[3], a, c));
}

// A row of a head is stored 64 bytes a group, which kept the L1 at 85% of its
// cycles and the kernel at 40 us for 32768 rows of 8 heads of 128. So a CTA's
// rows are put together in shared memory and leave as one bulk copy per row of
// K and of V, of 512 bytes at most: 36 us (1024 bytes: 40, 256: 43). Rows there
// are 16 bytes apart beyond their length, so that the 8 tokens of a store lie
// in different banks. With 12 CTAs to an SM: 34 us, 5.2 TB/s.
template <int D>
__device__ __forceinline__ void read_unit(const AppendArgs& a, int parts, int per, unsigned char* rows) {
  constexpr int kWays = kGroupWarps / Rec<D>::kGroups;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = warp % Rec<D>::kGroups;
  const unsigned u = blockIdx.x / parts;
  const int h0 = static_cast<int>(blockIdx.x - u * parts) * per, h1 = min(h0 + per, a.Hkv);
  UnitTask k;
  if (!unit_task<D>(a, u, lane, &k)) return;
  const int token = unit_token(lane), chunk = lane >> 3, ch = g * kGroupCh + chunk * 8;
  const int pitch = per * D * 2 + 16;
#pragma unroll 1
  for (int h = h0 + warp / Rec<D>::kGroups; h < h1; h += kWays) {
    uint4 kv[2], vv[2];
    kv[0] = kv[1] = vv[0] = vv[1] = make_uint4(0, 0, 0, 0);
    if (k.page_ok) {
      const uint8_t* rec = a.pool + k.rec + h * k.head;
      const uint2 v2 = __ldg(reinterpret_cast<const uint2*>(rec + Rec<D>::kVCode + (ch + token) * 8));
      uint32_t kw[2], ks[2], vs[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int tok = token + 8 * i;
        kw[i] = __ldg(reinterpret_cast<const uint32_t*>(rec + tok * (D / 2) + Rec<D>::k_chunk(tok, g) * 16 + chunk * 4));
        ks[i] = __ldg(reinterpret_cast<const uint32_t*>(rec + Rec<D>::kKScale + (tok * Rec<D>::kGroups + g) * 4));
        const uint16_t* sc = reinterpret_cast<const uint16_t*>(rec + Rec<D>::kVScale + g * 64) + tok;
        vs[i] = static_cast<uint32_t>(__ldg(sc)) | (static_cast<uint32_t>(__ldg(sc + 16)) << 16);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        kv[i] = word_values(kw[i], ks[i]);
        vv[i] = word_values(transpose_nibbles(i ? v2.y : v2.x, lane), vs[i]);
      }
    }
    unsigned char* dst = rows + token * pitch + ((h - h0) * D + ch) * 2;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      *reinterpret_cast<uint4*>(dst + i * 8 * pitch) = kv[i];
      *reinterpret_cast<uint4*>(dst + (16 + i * 8) * pitch) = vv[i];
    }
  }
  fence_proxy_async_smem();
  __syncthreads();
  if (warp == 0) {  // lanes 0..15: K rows, 16..31: V rows, by token
    const int token16 = lane & 15;
    if (token16 >= k.lo && token16 < k.hi) {
      __nv_bfloat16* out = (lane < 16 ? a.k_out : a.v_out) + ((k.row + token16) * a.Hkv + h0) * D;
      bulk_store(out, rows + lane * pitch, (h1 - h0) * D * 2);
    }
    bulk_store_wait_read();
  }
}

template <int D>
__global__ void __launch_bounds__(kRowThreads, 12) kv4_read_kernel(AppendArgs a, int parts, int per) {
  extern __shared__ __align__(128) unsigned char rows[];  // [2][16] of per heads
  grid_launch_dependents();
  grid_dependency_wait();
  read_unit<D>(a, parts, per, rows);
  check_cover(a);
}

// CTAs per unit: the heads are shared out until there are about 8 CTAs to an SM
// (the prompts above: with up to 16 the lookups are made twice, 114 us).
int unit_parts(const AppendArgs& a, long units) {
  const int ways = kGroupWarps / (a.D / kGroupCh), most = (a.Hkv + ways - 1) / ways;
  const long want = (kUnitCtas + units - 1) / units;
  return static_cast<int>(want < most ? want : most);
}

cudaError_t launch_lens(const AppendArgs& a, cudaStream_t stream) {
  const unsigned blocks = static_cast<unsigned>((a.B + kRowThreads - 1) / kRowThreads);
  return launch_kernel(advance_lens_kernel, dim3(blocks), dim3(kRowThreads), 0, stream, a);
}

}  // namespace

cudaError_t launch_rope_append(const AppendArgs& a, cudaStream_t stream) {
  if (a.T > 0) {
    const bool by_warp = rows_by_warp(a);
    const dim3 grid(static_cast<unsigned>(row_blocks(a.T, by_warp)));
    const cudaError_t e = launch_kernel(rope_append_kernel, grid, dim3(kRowThreads), 0, stream, a, static_cast<int>(by_warp));
    if (e != cudaSuccess) return e;
  }
  return a.new_lens != nullptr && (!a.fuse_lens || a.T == 0) ? launch_lens(a, stream) : cudaSuccess;
}

cudaError_t launch_rope_append_kv4(const AppendArgs& a, cudaStream_t stream) {
  if (a.T > 0) {
    const bool by_warp = rows_by_warp(a);
    const long units = record_units(a.T, a.B, a.cu != nullptr), q_blocks = a.q != nullptr ? row_blocks(a.T, by_warp) : 0;
    const int parts = unit_parts(a, 2 * units);
    const dim3 grid(static_cast<unsigned>(q_blocks + 2 * units * parts));
    const unsigned gap = static_cast<unsigned>(q_blocks / (2 * units * parts)), n = static_cast<unsigned>(units);
    const cudaError_t e = a.D == 128
        ? launch_kernel(rope_append_kv4_kernel<128>, grid, dim3(kRowThreads), 0, stream, a, gap, n, static_cast<unsigned>(parts),
                        static_cast<int>(by_warp))
        : launch_kernel(rope_append_kv4_kernel<64>, grid, dim3(kRowThreads), 0, stream, a, gap, n, static_cast<unsigned>(parts),
                        static_cast<int>(by_warp));
    if (e != cudaSuccess) return e;
  }
  return a.new_lens != nullptr && (!a.fuse_lens || a.T == 0) ? launch_lens(a, stream) : cudaSuccess;
}

cudaError_t launch_kv4_read(const AppendArgs& a, cudaStream_t stream) {
  if (a.T == 0) return cudaSuccess;
  const long units = record_units(a.T, a.B, a.cu != nullptr);
  const int most = kReadRowBytes / (a.D * 2), share = (a.Hkv + unit_parts(a, units) - 1) / unit_parts(a, units);
  const int per = share < most ? share : most, parts = (a.Hkv + per - 1) / per;
  const size_t smem = 32 * (static_cast<size_t>(per) * a.D * 2 + 16);
  const dim3 grid(static_cast<unsigned>(units * parts));
  return a.D == 128 ? launch_kernel(kv4_read_kernel<128>, grid, dim3(kRowThreads), smem, stream, a, parts, per)
                    : launch_kernel(kv4_read_kernel<64>, grid, dim3(kRowThreads), smem, stream, a, parts, per);
}

}  // namespace nld
