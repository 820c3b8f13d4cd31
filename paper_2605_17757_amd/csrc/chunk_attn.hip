// Attention of the newest tokens of every sequence (a prompt's chunk, drafted tokens, one
// token) over a paged cache that holds them already: bf16, 4-bit or 2-bit pages.
//
// A sequence's rows are its (token, query head) pairs of one KV head, token by token: a
// tile of them shares every key and value read.  Per page of 64 tokens:
//   S^T = K Q^T      two 32-token tiles, 8 steps of 16 channels
//   p = 2^(S^T c - m), m a running reference per row, moved when a score exceeds it by kSlack
//   O^T += V^T P^T   four 32-channel tiles, 4 steps of 16 tokens
// both on 32x32x16 matrix products with the queries as columns (lane l: column l % 32,
// half h = l / 32).  A lane then has 32 tokens' scores of one row in registers: maxima and
// sums are per lane but for one exchange between the halves, and, since the order of tokens
// inside a step is free, its p are P^T's operand as they are: with the rows of token tile T
// taken as row r -> slot 4 (r % 16) + 2 T + r / 16, register i of tile T in half h is slot
//   32 j0 + 16 h + 4 i4 + 2 T + b,   b = i / 8, j0 = i / 4 % 2, i4 = i % 4,
// so half h has 8 consecutive slots 32 j0 + 16 h + 8 i2 .. + 7 for each step (j0, i2).
//
// What a lane gives the matrix cores of a page, 16 bytes a step, 8 values:
//   K step ks of tile T: slot 4 lo + 2 T + b (l = lo + 16 b + 32 h), 8 channels
//   V step (j0, i2) of tile C: one channel, 8 slots as above
// bf16 pages hold these operands as they are.  Codes become fp16 numbers n by the conversions of
// small floating point types, two codes an instruction: as E4M3 the bytes 0 to 15 are n 2^-9 (subnormals
// up to 7, and on without a gap), as E2M1 the nibbles 0 to 3 are n / 2.  One packed multiply-add gives
//   x = s (n - z) = n s - s z
// with the scale and -s z rounded to fp16 after division by a power of two, so that the largest
// values that the page's scales and zero points allow, s times the largest code and |s z|, stay
// below 2^14: off by 2^-11 of |x| and of |s z| at most, or by 2^-31 of that largest (17 half steps of
// fp16's subnormals: one of the scale times 15, two of s z and x).  The range matters: a row without
// a range is stored with scale 1 whatever its value.  (Codes as the subnormals n 2^-24 need no
// conversion, but the scale times 2^24 then has to stay below 2^15: beside a scale of 1, 1e-3 was 2.4 %
// off and 2e-5 became 0.)  Scores take the power of two back as part of c, values through the
// accumulators' exponent, which follows the pages'.
//
// What becomes 16 bits, beside the output (whose own rounding is 1.6e-3 to 1.7e-3 of its 2-norm):
//   weights over bf16, in tiles of 128 and 256 rows past 32 rows a sequence: one bf16 value, errors
//     2.0e-3 to 2.3e-3.  Two pieces are half of the matrix products again: a prompt of 8192 tokens 734 us
//     for 548, chunks of seven sequences 259 for 202 (same card).  32 rows take two, their loads bound them.
//   over codes: weights, K^, V^ and q~ one fp16 value each (o~ too in the larger tiles), of 11 bits: 1.8e-3.
//     They are the matrix cores' operands; fp32 ones run at a sixteenth of the rate.
//
// Three kernels, by the rows of a tile (chunk_tile_rows, with both sides of each choice measured):
//   chunk_few_kernel   32 rows, waves share a tile's pages among them: bound by the bytes over bf16,
//                      by each page's chain of instructions over codes
//   chunk_kernel       128 or 256 rows, waves share every page through LDS: bound by the matrix
//                      products and the power limit
//   expand_kernel      (with 256 rows over codes) pages to fp16 operands, once: bound by the bytes
// and a merge of the partial states where the pages of a tile are shared among blocks.
#include "reduce_body.h"

#include <algorithm>
#include <type_traits>

namespace oscar {
namespace {

typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));

constexpr int kRows = 32;         // query rows of a wave
constexpr int kWaves = 4;
constexpr float kSlack = 8.0f;    // how far (log2) a score may exceed the reference before it moves
// Weights that become fp16 are 2^7 times larger, in the sums of values and of weights alike: up to
// 2^(7 + kSlack) of fp16's 2^16, and its least step is 2^-31 of the reference's weight.  (Without, 131072
// tokens of 2^-25 of the largest weight, together 0.4 %, were 0 in the sums of values.)
template <int FMT>
constexpr float kWeightUp = FMT == kBf16 ? 0.0f : 7.0f;
constexpr int kNoWindow = 1 << 30;  // positions are below it
// Least factor of scores: positive, so that a masked score stays -inf; below it scores are 0
// to fp32's precision of exp.
constexpr float kLeast = 0x1p-100f;
constexpr int kHalfLds = kP * kD * 2;    // operands of a page's K or V
constexpr int kPageLds = 2 * kHalfLds;
constexpr int kBfBlock = 2 * kP * kD * 2;  // bytes of a bf16 page-head block

template <int FMT>
__device__ inline f16v mfma(const u4v& a, const u4v& b, const f16v& c) {
  if (FMT == kBf16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0,
                                                   0);
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
template <int FMT>
__device__ inline uint32_t pack2(float a, float b) {  // to the operands' type, nearest even
  if (FMT == kBf16) return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), b2));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), h2));
}
__device__ inline float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// x itself, by a move that the compiler does not see through.
__device__ inline int stay(int x) { return __builtin_amdgcn_update_dpp(x, x, 0xE4, 0xF, 0xF, false); }
__device__ inline float stay(float x) { return __uint_as_float((uint32_t)stay((int)__float_as_uint(x))); }
// The larger one, NaN if one is: a single instruction, where fmaxf quiets each operand first.
__device__ inline float maximum(float x, float y) { return __builtin_elementwise_maximum(x, y); }
// Over the two halves of a wave: lanes l and l ^ 32.
__device__ inline float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ inline int wave_max_i(int v) {
  auto dpp = [](int x, auto ctrl) {
    return max(x, __builtin_amdgcn_update_dpp(x, x, decltype(ctrl)::value, 0xF, 0xF, false));
  };
  v = dpp(v, std::integral_constant<int, 0x128>{});  // rows of 16 lanes, rotated by 8, 4, 2, 1
  v = dpp(v, std::integral_constant<int, 0x124>{});
  v = dpp(v, std::integral_constant<int, 0x122>{});
  v = dpp(v, std::integral_constant<int, 0x121>{});
  return max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
             max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}
// The same of what is ordered as its bits are: magnitudes.
__device__ inline float half_max_bits(uint32_t x) {
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return __uint_as_float(max((uint32_t)r[0], (uint32_t)r[1]));
}
// The largest magnitude of x's fp32 bits and eight bf16 values.
constexpr uint32_t kInfBits = 0x7f800000u;  // (NaN above it)
__device__ inline uint32_t top_bf16(uint32_t x, const u4v& w) {
  typedef uint16_t us2 __attribute__((ext_vector_type(2)));
  us2 t = us2{0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) t = __builtin_elementwise_max(t, __builtin_bit_cast(us2, w[i] & 0x7fff7fffu));
  return max(x, (uint32_t)max(t.x, t.y) << 16);
}
// Exponent e of |x| < 2^(e + 1) (0 and subnormals: -127).
__device__ inline int exp_of(float x) { return (int)((__float_as_uint(x) >> 23) & 255u) - 127; }
__device__ inline bool is_nan(float x) { return (__float_as_uint(x) & 0x7fffffffu) > 0x7f800000u; }
__device__ inline float pow2(int e) {  // clamped to fp32's normal range
  return __uint_as_float((uint32_t)(min(max(e, -126), 127) + 127) << 23);
}

// A value that no one writes while the kernel runs, at an address that is the wave's: by a scalar
// load, which the waits for vector loads do not meet.
template <class T>
__device__ inline T scalar_load(const T* p) {
  return *(const __attribute__((address_space(4))) T*)p;
}
__device__ inline int64_t uniform(int64_t x) {  // the same in all lanes: into scalar registers
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
                   (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// ---------------------------------------------------------------------------
// Tiles.  Sequence b's tiles have the numbers from floor(q_start[b] g / M) + b on: for any
// chunk lengths at least as many as it has tiles, so that a block finds its sequence among
// the numbers without a sum over the sequences before.
// ---------------------------------------------------------------------------
struct Tile {
  int b;       // -1: none
  int q0, n;   // the sequence's first row of q and its new tokens
  int row0, rows;  // first (token, head) row of the tile, rows of the sequence
  int len;
};
// Tile i of sequence b.
__device__ inline Tile tile_at(const ChunkArgs& a, int b, int i, int g, int M) {  // (uniform)
  Tile t;
  t.b = b;
  t.q0 = min(max(scalar_load(a.q_start + b), 0), a.n_q);
  t.n = max(min(max(scalar_load(a.q_start + b + 1), 0), a.n_q) - t.q0, 0);
  t.len = min(max(scalar_load(a.seq_lens + b), 0), a.max_pages * kP);
  t.rows = t.n * g;
  t.row0 = i * M;
  return t;
}
__device__ inline Tile find_tile(const ChunkArgs& a, int64_t id, int g, int M) {
  const int l = threadIdx.x & 63;
  auto start = [&](int b) { return min(max(a.q_start[b], 0), a.n_q); };
  int lo = 0, n = a.B;  // the sequence is in [lo, lo + n)
  while (n > 1) {       // 64 candidates at a time
    const int step = (n + 63) / 64;
    const int b = lo + l * step;
    const bool le = l * step < n && (int64_t)start(b) * g / M + b <= id;
    const int k = 63 - __clzll((unsigned long long)(__ballot(le) | 1ull));
    lo += k * step;
    n = min(step, n - k * step);
  }
  const int b = __builtin_amdgcn_readfirstlane(lo);
  Tile t = tile_at(a, b, 0, g, M);
  const int64_t i = id - ((int64_t)t.q0 * g / M + b);
  t.row0 = (int)(i * M);
  if (i < 0 || i * M >= t.rows) t.b = -1;
  return t;
}

// Pages that rows [row0, row0 + M) of a tile see: `head` first ones, then from `from` on.
struct Pages {
  int head, from, count;
  int p_min, p_max;  // positions of the first and the last row
};
__device__ inline Pages tile_pages(const Tile& t, int g, int M, int window, int sinks) {
  Pages s;
  const int base = t.len - t.n;
  s.p_min = base + t.row0 / g;
  s.p_max = base + (min(t.row0 + M, t.rows) - 1) / g;
  const int start = max(s.p_min - window + 1, 0);
  s.from = start / kP;
  s.head = min((min(sinks, start) + kP - 1) / kP, s.from);
  s.count = s.p_max < 0 ? 0 : s.head + s.p_max / kP + 1 - s.from;
  return s;
}

// Cached tokens that some row of a sequence sees: t < end, and t >= start or t < sinks.  The others of a page that is
// read may hold anything: their weights are 0, and so are their values and scales made (0 times a NaN
// or an infinity is not, and a scale counts in the page's exponent).
struct Seen {
  int end, start, sinks;
  __device__ bool operator()(int t) const { return t < end && (t >= start || t < sinks); }
  __device__ bool whole_page(int t0) const { return t0 + kP <= end && (t0 >= start || t0 + kP <= sinks); }
  // The halves of a dword that belong to tokens t and t + 1.
  __device__ uint32_t pair(int t) const { return ((*this)(t) ? 0xffffu : 0u) | ((*this)(t + 1) ? 0xffff0000u : 0u); }
};
// Of a sequence's rows, where clearing takes instructions of its own (bf16: for the tile's rows alone
// chunks of seven sequences in a window took 2 % longer); of the tile's, where scales are made anyway.
template <int FMT>
__device__ inline Seen seen_by_rows(const Tile& t, const Pages& s, int window, int sinks) {
  return FMT == kBf16 ? Seen{t.len, max(t.len - t.n - window + 1, 0), sinks}
                      : Seen{s.p_max + 1, max(s.p_min - window + 1, 0), sinks};
}

// ---------------------------------------------------------------------------
// One page's operands from the three formats.  Bytes of channels and slots: internal.h and
// the headers of the formats' kernels.
// ---------------------------------------------------------------------------
// First channel of K step ks in half h, and channel of its element e.
template <int FMT>
__device__ inline int k_channel(int ks, int h, int e) {
  if (FMT == kBf16) return 64 * (ks / 4) + 32 * h + 8 * (ks % 4) + e;  // ks = 4 X + kc
  if (FMT == kInt4) return 32 * (ks % 4) + 16 * (ks / 4) + 8 * h + e / 2 + 4 * (e % 2);
  return 64 * h + 16 * (ks / 2) + ks % 2 + 2 * e;
}
// Slot (of 8) of element e of a V step.
template <int FMT>
__host__ __device__ constexpr int v_slot(int e) {
  return FMT == kInt4 ? (e & 4) + (e % 4) / 2 + 2 * (e % 2) : e;
}
// Rows 8 k + 4 h .. + 3 of the four tiles, row r of tile C channel 32 C + r: f(first channel, four values).
template <class F>
__device__ inline void each_four(const f16v (&o)[4], int h, F&& f) {
#pragma unroll
  for (int C = 0; C < 4; ++C)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      f(32 * C + 8 * k + 4 * h, o[C][4 * k], o[C][4 * k + 1], o[C][4 * k + 2], o[C][4 * k + 3]);
}

template <int FMT>
constexpr int kBits = FMT == kInt4 ? 4 : 2;  // of a code
template <int FMT>
constexpr int raw_loads() { return FMT == kInt4 ? 4 : 2; }  // 16-byte loads of a wave for K's codes, and for V's
constexpr int block_bytes_of(int fmt, int ng) {
  return fmt == kBf16 ? kBfBlock : fmt == kInt4 ? kv4_block_bytes(ng) : block_bytes(ng);
}
template <int FMT, int NG>
__device__ inline u4v load_k(const uint8_t* blk, int i) {  // kInt4: (T, X) = (i / 2, i % 2); kInt2: T = i
  const int l = threadIdx.x & 63, lo = l & 15, b = (l >> 4) & 1, h = l >> 5;
  const int off = FMT == kInt4 ? (64 * (2 * (i / 2) + b) + 16 * (h + 2 * (i % 2)) + lo) * 16
                               : (4 * lo + 2 * i + b) * 32 + 16 * h;
  return *reinterpret_cast<const u4v*>(blk + off);
}
template <int FMT, int NG>
__device__ inline u4v load_v(const uint8_t* blk, int i) {  // kInt4: (jp, i2) = (i / 2, i % 2); kInt2: j0 = i
  const int l = threadIdx.x & 63, lo = l & 15, jj = (l >> 4) & 1, h = l >> 5;
  const int off = FMT == kInt4 ? kKv4CodeBytes + (64 * (2 * (i / 2) + jj) + 16 * (2 * h + i % 2) + lo) * 16
                               : kOffVCodes + (l & 31) * 64 + 32 * i + 16 * h;
  return *reinterpret_cast<const u4v*>(blk + off);
}
// Lane l's slot l: scale and zero of every group, of K or of V.
template <int FMT, int NG>
__device__ inline void load_entries(const uint8_t* blk, int is_v, uint32_t (&x)[NG]) {
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const int at = FMT == kInt4 ? l * NG + g : g * kP + l;
    const int off = FMT == kInt4 ? kv4_sz_off(NG, is_v) : is_v ? off_vsz(NG) : kOffKSz;
    x[g] = reinterpret_cast<const uint32_t*>(blk + off)[at];
  }
}
// Scales of a page in LDS, a wave's own: per group the slots' (s, -s z), divided by a power of two.
// K: both halves of a dword, by slot.  V: arrays of fp16, eight slots of a step in 16 bytes, in the
// order of the step's elements.
template <int NG>
struct Scales {
  uint32_t k[NG][kP];
  __align__(16) uint16_t va[NG][kP], vb[NG][kP];
};
constexpr int kNoExp = -400;
// Exponents of operands that sums run over: with them the accumulators change their unit.
constexpr int kRoom = 2;   // a page that needs up to so much less takes the accumulators'
constexpr int kDeep = 60;  // no exponent lies further below the largest: 2^30 tokens' sums stay below 2^120
struct Exponent {
  int e = kNoExp, most = kNoExp;
  __device__ void follow(int need) {
    most = max(most, need);
    if (need > e || need < e - kRoom) e = max(need, most - kDeep);
  }
};
// What sums in units of 2^from are multiplied by to be in units of 2^to.
__device__ inline float unit_change(int from, int to) { return ldexpf(1.0f, from - to); }
// A page's entries to scales, of slots that no row sees 0; e: the exponent that the page brings its
// operands to.
template <int FMT, int NG>
__device__ inline void make_scales(const uint32_t (&ent)[NG], int is_v, int bf16, bool seen, Scales<NG>& sc,
                                   Exponent& ex) {
  const int l = threadIdx.x & 63;
  const uint32_t written = seen ? 0xffffffffu : 0u;
  float s[NG], z[NG];
  if (bf16) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      s[g] = bf_lo(ent[g] & written);
      z[g] = bf_hi(ent[g] & written);
    }
  } else {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const uint32_t both = ent[g] & written;
      const h2 x = __builtin_bit_cast(h2, both);
      s[g] = (float)x.x;
      z[g] = (float)x.y;
    }
  }
  float top = 0.0f;  // of the values' two parts, below 2^14 after division by 2^e
#pragma unroll
  for (int g = 0; g < NG; ++g)
    top = fmaxf(fmaxf(top, fabsf(s[g]) * (float)((1 << kBits<FMT>) - 1)), fabsf(s[g] * z[g]));
  ex.follow(max(wave_max_i(exp_of(top)) + 1 - 14, -120));
  const int at = FMT == kInt4 ? (l & ~3) + 2 * (l & 1) + ((l >> 1) & 1) : l;  // v_slot's inverse
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const float x = ldexpf(s[g], -ex.e);
    const uint32_t ab = pack2<kInt4>(x, -x * z[g]);
    if (is_v) {
      sc.va[g][at] = (uint16_t)ab;
      sc.vb[g][at] = (uint16_t)(ab >> 16);
    } else {
      sc.k[g][l] = ab;
    }
  }
}
__device__ inline uint32_t fma_h2(uint32_t n, uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(h2, n), __builtin_bit_cast(h2, a),
                                                                __builtin_bit_cast(h2, b)));
}
// Codes as fp16: of bytes 0 and 1 or (hi) 2 and 3, each the code times `unit`, at most 15; of the two
// nibbles of byte `byte`, at most 3 each.
__device__ inline uint32_t bytes_h2(uint32_t codes, int unit, bool hi) {
  const float scale = 512.0f / unit;
  return hi ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)codes, scale, true))
            : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)codes, scale, false));
}
template <int BYTE>
__device__ inline uint32_t nibbles_h2(uint32_t codes) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 2.0f, BYTE));
}
// K operand of step ks, tile T from its raw load.
template <int FMT, int NG>
__device__ inline u4v k_operand(const u4v& raw, int T, int ks, const Scales<NG>& sc) {
  const int l = threadIdx.x & 63, lo = l & 15, b = (l >> 4) & 1, h = l >> 5;
  constexpr int G = kD / NG;
  const int g = FMT == kInt4 ? 32 * (ks % 4) / G : (64 * h + 16 * (ks / 2)) / G;
  const uint32_t ab = sc.k[g][4 * lo + 2 * T + b];
  const uint32_t A = __builtin_amdgcn_perm(ab, ab, 0x01000100u), B = __builtin_amdgcn_perm(ab, ab, 0x03020302u);
  u4v n;
  if (FMT == kInt4) {  // low nibbles: channels 0, 4, 1, 5; high ones: 2, 6, 3, 7
    const uint32_t d = raw[ks % 4];
#pragma unroll
    for (int i = 0; i < 4; ++i) n[i] = bytes_h2((d >> (4 * (i / 2))) & 0x0f0f0f0fu, 1, i % 2);
  } else {  // even codes, odd codes
    const uint32_t d = (raw[ks / 2] >> (2 * (ks % 2))) & 0x33333333u;
    n = u4v{nibbles_h2<0>(d), nibbles_h2<1>(d), nibbles_h2<2>(d), nibbles_h2<3>(d)};
  }
  u4v r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = fma_h2(n[i], A, B);
  return r;
}
// V operand of tile C, step (j0, i2) from its raw load.
template <int FMT, int NG>
__device__ inline u4v v_operand(const u4v& raw, int C, int j0, int i2, const Scales<NG>& sc) {
  const int l = threadIdx.x & 63, jj = (l >> 4) & 1, h = l >> 5;
  constexpr int G = kD / NG;
  const int c = FMT == kInt4 ? 64 * (C / 2) + 32 * jj : 4 * (l & 31);  // a channel of the row's group
  const int t0 = 32 * j0 + 16 * h + 8 * i2;
  const u4v A = *reinterpret_cast<const u4v*>(&sc.va[c / G][t0]);
  const u4v B = *reinterpret_cast<const u4v*>(&sc.vb[c / G][t0]);
  u4v r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // a byte: two channels of a slot, slots 0, 2, 1, 3; four channels of a slot, slots in order
    const uint32_t d = FMT == kInt4 ? (raw[2 * j0 + i / 2] >> (4 * (C % 2))) & 0x0f0f0f0fu
                                    : (raw[2 * i2 + i / 2] >> (4 * (C / 2))) & (C % 2 ? 0x0c0c0c0cu : 0x03030303u);
    r[i] = fma_h2(bytes_h2(d, FMT == kInt2 && C % 2 ? 4 : 1, i % 2), A[i], B[i]);
  }
  return r;
}

// ---------------------------------------------------------------------------
// A wave's 32 rows.
// ---------------------------------------------------------------------------
struct RowState {
  int pos;         // of the row's token; -1: no row
  float m, l;      // reference maximum; this lane's part of the sum
  float c;         // factor of the scores (log2 units)
};

// The query operands of the wave's rows (row: this lane's, live or not).  Quantized caches:
// fp16 rows divided by a power of two, which c takes back.  Returns whether a NaN or an infinity is
// among this lane's channels: the row's sum then begins as NaN, and so does the row end, also where
// its scores are all -infinity.
template <int FMT>
__device__ inline bool load_queries(const ChunkArgs& a, size_t row, bool live, u4v (&q)[8], float& c) {
  const int h = (threadIdx.x & 63) >> 5;
  if (FMT == kBf16) {
    const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;  // scores are multiplied by |scale|
    uint32_t top = 0;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      q[ks] = live ? *reinterpret_cast<const u4v*>(a.q + row * kD + k_channel<FMT>(ks, h, 0)) : u4v{0, 0, 0, 0};
      top = top_bf16(top, q[ks]);
      q[ks] ^= flip;
    }
    c = fmaxf(fabsf(a.scale), kLeast);
    return top >= kInfBits;
  } else {
    const float* src = a.qt + row * kD;
    float x[8][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // 16 channels: two steps
      float y[16];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int from = FMT == kInt4 ? k_channel<FMT>(i + 4 * (j / 2), h, 0) + 4 * (j % 2) : k_channel<FMT>(2 * i, h, 2 * j);
        const float4 v = *reinterpret_cast<const float4*>(src + from);
        y[4 * j] = v.x, y[4 * j + 1] = v.y, y[4 * j + 2] = v.z, y[4 * j + 3] = v.w;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float& to = x[FMT == kInt4 ? i + 4 * j : 2 * i + j][e];
          to = live ? y[FMT == kInt4 ? 8 * j + e / 2 + 4 * (e % 2) : 2 * e + j] : 0.0f;
          top = max(top, __float_as_uint(to) & 0x7fffffffu);
        }
    }
    const int e = max(exp_of(half_max_bits(top)), -60) - 13;  // |q| < 2^14
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        q[ks][i] = pack2<FMT>(ldexpf(x[ks][2 * i], -e), ldexpf(x[ks][2 * i + 1], -e));
    c = pow2(e);
    return top >= kInfBits;
  }
}

// Scores of tokens that the row does not see: -inf.  t0: the page's first token.
__device__ inline void mask_page(f16v (&s)[2], int pos, int t0, int window, int sinks) {
  const int h = (threadIdx.x & 63) >> 5;
  const int last = pos - (t0 + 16 * h);              // last visible slot, from the half's first
  const int before = (pos - window) - (t0 + 16 * h);  // slots up to it lie before the window
  const int sink = sinks - (t0 + 16 * h);
#pragma unroll
  for (int T = 0; T < 2; ++T)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int t = 32 * (i / 4 % 2) + 4 * (i % 4) + 2 * T + i / 8;
      const bool ok = t <= last && (t > before || t < sink);
      s[T][i] = ok ? s[T][i] : -INFINITY;
    }
}

// The reference maximum for a page's scores, and the sums' scale with it.
__device__ inline void move_reference(const f16v (&s)[2], f16v (&o)[4], RowState& r, float cp) {
  float mx = s[0][0];
#pragma unroll
  for (int i = 0; i < 16; ++i) mx = maximum(maximum(mx, s[0][i]), s[1][i]);
  mx = half_max(mx) * cp;
  const bool need = mx > r.m + kSlack;
  if (__ballot(need) != 0ull) {
    const float mn = mx > r.m ? mx : r.m;  // (mx may be NaN)
    const float alpha = r.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(r.m - mn);
    r.m = mn;
    r.l *= alpha;
#pragma unroll
    for (int C = 0; C < 4; ++C) o[C] *= alpha;
  }
}

// Scores of a page in s -> the operands of P^T (HL: a second, smaller piece of each p), m and l
// and the accumulators' scale moved.  cp: c of this page.
template <int FMT, bool HL>
__device__ inline void softmax_page(f16v (&s)[2], f16v (&o)[4], RowState& r, float cp, u4v (&p)[4], u4v (&pl)[4]) {
  move_reference(s, o, r, cp);
  const float ms = (r.m == -INFINITY ? 0.0f : -r.m) + kWeightUp<FMT>;
  float sum = 0.0f;
#pragma unroll
  for (int T = 0; T < 2; ++T)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[T][i] = __builtin_amdgcn_exp2f(fmaf(s[T][i], cp, ms));
      sum += s[T][i];
    }
  r.l += sum;
  auto at = [&](int j0, int i2, int e) {  // p of slot 32 j0 + 16 h + 8 i2 + v_slot(e)
    const int x = v_slot<FMT>(e), u = x % 4;
    return s[u / 2][8 * (u % 2) + 4 * j0 + 2 * i2 + x / 4];
  };
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = at(k / 2, k % 2, 2 * i), y = at(k / 2, k % 2, 2 * i + 1);
      p[k][i] = pack2<FMT>(x, y);
      if (HL) pl[k][i] = pack2<FMT>(x - bf_lo(p[k][i]), y - bf_hi(p[k][i]));
    }
}

// ---------------------------------------------------------------------------
// What a block does.  num_splits == 1: one tile, all of its pages.  Otherwise the pages of all
// tiles of a KV head (as many for each of a sequence's tiles as one sees at most), laid end to end,
// are cut into equal ranges, one for each block that the GPU holds at once; a tile's part of
// a range leaves a partial state in the tile's slot for that range, counted from its first.
// ---------------------------------------------------------------------------
constexpr int kLeastPages = 4;  // of a range
// Sequences whose tiles every block counts; of more it looks for the tile's number in q_start, which
// leaves numbers without a tile: blocks that end at once, but where they are as far apart as a
// shader engine's blocks, that engine's share of the work is missing.  64 sequences of 4k tokens of
// bf16, 8 new ones each: counted 174 us, looked for 222; 512 of 300: 253, 349, one new: 198, 181;
// 2048 of 300, one new: 1041, 724.
constexpr int kCounted = 256;

struct Segment {
  Tile t;
  Pages pg;
  int x0, x1;   // pages of the tile
  int slot;
  bool last;    // no later range has pages of the tile
  bool whole;   // no other range has
};
struct Walk {
  int64_t x, xe, range;  // pages left, pages per range
  int r, empty;          // the range; next sequence of those that see nothing
  int empty_tile;
};
__device__ inline int64_t wave_sum_l(int64_t v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
  return v;
}
// Tiles of sequence b, and the pages that one of them sees at most: none without cached tokens.
__device__ inline int tiles_of(const ChunkArgs& a, int b, int g, int M, int window, int& pages) {
  pages = 0;
  if (b >= a.B) return 0;
  Tile t;
  t.q0 = min(max(a.q_start[b], 0), a.n_q);
  t.n = max(min(max(a.q_start[b + 1], 0), a.n_q) - t.q0, 0);
  t.len = min(max(a.seq_lens[b], 0), a.max_pages * kP);
  t.rows = t.n * g;
  t.row0 = 0;
  const int tiles = (t.rows + M - 1) / M;
  if (tiles == 1) {
    pages = tile_pages(t, g, M, window, a.sinks).count;
  } else if (tiles > 1) {
    // a window's and a tile's tokens lie in so many pages at most, the first tokens in the others
    const int64_t span = (int64_t)window + (M - 1) / g + 1;
    pages = (int)min((span + kP - 2) / kP + 1 + ((int64_t)a.sinks + kP - 1) / kP, (int64_t)(t.len + kP - 1) / kP);
  }
  return tiles;
}
__device__ inline Walk start_walk(const ChunkArgs& a, int g, int M, int window) {
  Walk k = {};
  k.r = (int)(blockIdx.x / a.Hkv);
  if (a.num_splits == 1) return k;
  const int l = threadIdx.x & 63, ranges = (int)(gridDim.x / a.Hkv);
  int64_t all = 0;
  int most = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    int pages;
    const int tiles = tiles_of(a, b0 + l, g, M, window, pages);
    all += wave_sum_l((int64_t)tiles * pages);
    most = max(most, wave_max_i(pages));
  }
  // (a tile meets ceil(pages / range) + 1 ranges at most)
  k.range = uniform(max(max((all + ranges - 1) / ranges, (int64_t)((most + a.num_splits - 2) / (a.num_splits - 1))),
                        (int64_t)kLeastPages));
  k.x = k.r * k.range;
  k.xe = min(uniform(all), k.x + k.range);
  k.empty = k.r;
  return k;
}
// Tile r of all sequences', counted from the last one's last.
__device__ inline Tile count_tile(const ChunkArgs& a, int r, int g, int M) {
  auto start = [&](int b) { return min(max(a.q_start[min(b, a.B)], 0), a.n_q); };
  int before = 0;
  for (int b0 = (a.B - 1) & ~63; b0 >= 0; b0 -= 64) {
    const int b = b0 + 63 - (threadIdx.x & 63);
    const int tiles = (max(start(b + 1) - start(b), 0) * g + M - 1) / M;
    const int incl = before + wave_prefix(tiles);
    const uint64_t hit = __ballot(incl - tiles <= r && r < incl);
    if (hit) {
      const int lane = __ffsll((unsigned long long)hit) - 1;
      return tile_at(a, b0 + 63 - lane, __builtin_amdgcn_readlane(incl, lane) - 1 - r, g, M);
    }
    before = __builtin_amdgcn_readlane(incl, 63);
  }
  Tile t = {};
  t.b = -1;
  return t;
}
// The next segment.
__device__ inline bool find_segment(const ChunkArgs& a, Walk& k, int g, int M, int window, Segment& s) {
  if (a.num_splits == 1) {
    if (k.empty) return false;
    k.empty = 1;
    s.t = a.B > 1 && a.B <= kCounted ? count_tile(a, k.r, g, M)
                                     : find_tile(a, (int64_t)a.n_q * g / M + a.B - 1 - k.r, g, M);
    if (s.t.b < 0) return false;
    s.pg = tile_pages(s.t, g, M, window, a.sinks);
    s.x0 = s.slot = 0;
    s.x1 = s.pg.count;
    s.last = s.whole = true;
    return true;
  }
  const int l = threadIdx.x & 63, ranges = (int)(gridDim.x / a.Hkv);
  for (; k.empty < a.B; k.empty += ranges, k.empty_tile = 0) {  // rows that see nothing
    Tile e = tile_at(a, k.empty, 0, g, M);
    if (e.len > 0 || k.empty_tile >= (e.rows + M - 1) / M) continue;
    e.row0 = k.empty_tile++ * M;
    s.t = e;
    s.pg = tile_pages(s.t, g, M, window, a.sinks);
    s.x0 = s.x1 = s.slot = 0;
    s.last = s.whole = true;
    return true;
  }
  if (k.x >= k.xe) return false;
  int64_t before = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    int pages;
    const int tiles = tiles_of(a, b0 + l, g, M, window, pages);
    const int64_t np = (int64_t)tiles * pages;
    const int hi = wave_prefix((int)(np >> 16)), lo = wave_prefix((int)(np & 0xffff));  // lo < 2^22
    const int64_t incl = before + ((int64_t)hi << 16) + lo;
    const uint64_t hit = __ballot(np > 0 && incl - np <= k.x && k.x < incl);
    if (hit) {
      const int lane = __ffsll((unsigned long long)hit) - 1;
      const int b = b0 + lane, count = __builtin_amdgcn_readlane(pages, lane);
      const int64_t at = uniform(__shfl(incl - np, lane, 64));
      const int tile = __builtin_amdgcn_readfirstlane((int)((k.x - at) / count));
      const int64_t first = at + (int64_t)tile * count;
      const int p0 = __builtin_amdgcn_readfirstlane((int)(k.x - first));
      const int p1 = __builtin_amdgcn_readfirstlane((int)min((int64_t)count, p0 + (k.xe - k.x)));
      s.t = tile_at(a, b, tile, g, M);
      s.pg = tile_pages(s.t, g, M, window, a.sinks);
      s.x0 = min(p0, s.pg.count);
      s.x1 = min(p1, s.pg.count);
      s.slot = __builtin_amdgcn_readfirstlane((int)(k.r - first / k.range));
      s.last = p1 == count;
      s.whole = p0 == 0 && s.last;
      k.x += p1 - p0;
      return true;
    }
    before = uniform(__shfl(incl, 63, 64));
  }
  return false;  // not reached: page x lies in some tile
}

// The next segment, in scalar registers.
__device__ inline bool next_segment(const ChunkArgs& a, Walk& k, int g, int M, int window, Segment& s) {
  Segment x = {};
  if (!__builtin_amdgcn_readfirstlane((int)find_segment(a, k, g, M, window, x))) return false;
  auto u = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  s.t = Tile{u(x.t.b), u(x.t.q0), u(x.t.n), u(x.t.row0), u(x.t.rows), u(x.t.len)};
  s.pg = Pages{u(x.pg.head), u(x.pg.from), u(x.pg.count), u(x.pg.p_min), u(x.pg.p_max)};
  s.x0 = u(x.x0);
  s.x1 = u(x.x1);
  s.slot = u(x.slot);
  s.last = u(x.last);
  s.whole = u(x.whole);
  return true;
}

// Marks in slot 0 a row that has its output already.
constexpr float kDone = INFINITY;

// The row's output (direct), or its partial state in the segment's slot.  scale: of the
// accumulators.
__device__ inline void store_row(const ChunkArgs& a, size_t row, const Segment& s, bool direct, const f16v (&o)[4],
                                 float m, float l, float scale, int h) {
  const size_t at = row * a.num_splits + s.slot;
  float2* ml = reinterpret_cast<float2*>(a.part_ml);
  if (direct) {
    const float il = (l > 0.0f ? 1.0f / l : is_nan(l) ? l : 0.0f) * scale;
    uint16_t* dst = a.out + row * kD;
    each_four(o, h, [&](int c, float x, float y, float z, float w) {
      uint2 v;
      v.x = pack2<kBf16>(x * il, y * il);
      v.y = pack2<kBf16>(z * il, w * il);
      *reinterpret_cast<uint2*>(dst + c) = v;
    });
    if (a.num_splits > 1 && h == 0) ml[at] = make_float2(kDone, 0.0f);
    return;
  }
  float* dst = a.part_o + at * kD;
  if (is_nan(l)) m = 0.0f;  // NaN in a row: its scores have no maximum, but the state is not empty
  if (m != -INFINITY)    // of an empty state only that is read
    each_four(o, h, [&](int c, float x, float y, float z, float w) {
      *reinterpret_cast<float4*>(dst + c) = make_float4(x * scale, y * scale, z * scale, w * scale);
    });
  if (h == 0) {
    ml[at] = make_float2(m, l);
    if (s.last)
      for (int i = s.slot + 1; i < a.num_splits; ++i) ml[row * a.num_splits + i] = make_float2(-INFINITY, 0.0f);
  }
}
// A segment without pages.
__device__ inline void store_empty(const ChunkArgs& a, size_t row, const Segment& s, bool direct, int h) {
  float2* ml = reinterpret_cast<float2*>(a.part_ml) + row * a.num_splits;
  if (direct) {
    u4v* dst = reinterpret_cast<u4v*>(a.out + row * kD) + 8 * h;
#pragma unroll
    for (int i = 0; i < 8; ++i) dst[i] = u4v{0, 0, 0, 0};
    if (a.num_splits > 1 && h == 0) ml[0] = make_float2(kDone, 0.0f);
  } else if (h == 0) {
    for (int i = s.slot; i < (s.last ? a.num_splits : s.slot + 1); ++i) ml[i] = make_float2(-INFINITY, 0.0f);
  }
}

// 16 bytes a lane from global memory to LDS, lane l's to dst + 16 l (dst: the wave's).  The compiler
// waits for such a load before it reads LDS that may be the load's: a kernel that reads one page
// while others come in has an array of its own for each.
__device__ inline void load_to_lds(const void* src, uint8_t* dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}
// Waits until at most N of the wave's loads are under way.
template <int N>
__device__ inline void wait_loads() {
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0xf70);  // vmcnt alone
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
}
// A barrier that waits for the waves' LDS accesses, and leaves loads under way alone.
__device__ inline void lds_barrier() {
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt alone
  __builtin_amdgcn_s_barrier();
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// ---------------------------------------------------------------------------
// Chunks over a quantized cache: R_k and R_v as operands (two fp16 pieces of each entry, so that the
// rotations cost no precision against q's and o's own rounding), for the blocks to rotate their
// rows; and where a page is read by many blocks, its codes expanded once to what a wave gives the
// matrix cores.
// ---------------------------------------------------------------------------
// Part `part` (of four) of a page's K or V: four operands of 1 KB at dst; NATURAL: V's slots in
// order within a step, whatever the codes' order.
template <int FMT, int NG, bool NATURAL>
__device__ inline void expand_part(const u4v& raw, int is_v, int part, const Scales<NG>& sc, uint8_t* dst) {
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (is_v) {
      const int C = FMT == kInt4 ? 2 * (part / 2) + i % 2 : i;
      const int j0 = FMT == kInt4 ? i / 2 : part / 2, i2 = part % 2;
      u4v v = v_operand<FMT, NG>(raw, C, j0, i2, sc);
      if (NATURAL && FMT == kInt4)  // slots (0, 2), (1, 3) -> (0, 1), (2, 3)
        v = u4v{__builtin_amdgcn_perm(v.y, v.x, 0x05040100u), __builtin_amdgcn_perm(v.y, v.x, 0x07060302u),
                __builtin_amdgcn_perm(v.w, v.z, 0x05040100u), __builtin_amdgcn_perm(v.w, v.z, 0x07060302u)};
      *reinterpret_cast<u4v*>(dst + (C * 4 + 2 * j0 + i2) * 1024 + l * 16) = v;
    } else {
      const int T = part / 2, ks = 4 * (part % 2) + i;
      *reinterpret_cast<u4v*>(dst + (T * 8 + ks) * 1024 + l * 16) = k_operand<FMT, NG>(raw, T, ks, sc);
    }
  }
}
// Channel that row r of output tile C (32 rows) of o~ V's products is.
template <int FMT>
__device__ inline int v_channel(int C, int r) {
  return FMT == kInt2 ? 4 * r + C : FMT == kInt4 ? 64 * (C / 2) + 32 * (r / 16) + 16 * (C % 2) + r % 16 : 32 * C + r;
}

// Blocks: a page of a sequence's table and a KV head each (`pages` of them, or none); behind them
// kRotParts for each rotation.  Bound by the bytes written: 8192 pages of a head, 54 MB of 2-bit
// codes read and 269 MB written, 54 us (5.9 TB/s).  Expanded by the blocks that read them instead, 2 x
// 513 tokens over 32k took 870 us, with this launch 700.
constexpr int kRotParts = 8;
template <int FMT, int NG>
__global__ __launch_bounds__(256) void expand_kernel(ChunkArgs a, int64_t pages) {
  __shared__ Scales<NG> scales[4];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  if (blockIdx.x >= pages) {
    // operand (tile, step, piece): R_k: rows the channels of q~ that the score steps take, 8 input
    // channels of q each; R_v: rows 32 output channels, steps the channels of o~ in a lane
    const int which = (int)(blockIdx.x - pages) / kRotParts, is_v = which & 1;
    const float* R = is_v ? a.Rv : a.Rk;
    if (R) R += (size_t)(which >> 1) * kD * kD;
    const int r = l & 31, h = l >> 5;
    for (int i = 4 * (int)((blockIdx.x - pages) % kRotParts) + w; i < 32; i += 4 * kRotParts) {
      const int C = i / 8, k = i % 8;
      u4v hi, lo;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float x[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int e = 2 * j + u;
          int from, to;  // R[from][to]
          if (is_v) {    // o_c = sum_j o~_j R_v[c][j]; step k: row 16 (k % 2) + 8 (e / 4) + 4 h + e % 4 of tile k / 2
            from = 32 * C + r;
            to = v_channel<FMT>(k / 2, 16 * (k % 2) + 8 * (e / 4) + 4 * h + e % 4);
          } else {       // q~_j = sum_c q_c R_k[c][j]; row r: element 4 (r / 8 % 2) + r % 4 of step
                         // 2 C + r / 16, half r / 4 % 2
            from = 16 * k + 8 * h + e;
            to = k_channel<FMT>(2 * C + r / 16, r / 4 % 2, 4 * (r / 8 % 2) + r % 4);
          }
          x[u] = R ? R[from * kD + to] : from == to ? 1.0f : 0.0f;
        }
        const uint32_t both = pack2<kInt4>(x[0], x[1]);
        const h2 t = __builtin_bit_cast(h2, both);
        hi[j] = both;
        lo[j] = pack2<kInt4>(x[0] - (float)t.x, x[1] - (float)t.y);
      }
      uint8_t* dst = a.rot + (size_t)which * kRotBytes + (C * 8 + k) * 2048 + l * 16;
      *reinterpret_cast<u4v*>(dst) = hi;
      *reinterpret_cast<u4v*>(dst + 1024) = lo;
    }
    return;
  }
  const int kvh = blockIdx.x % a.Hkv;
  const int64_t at = blockIdx.x / a.Hkv;
  const int b = (int)(at / a.max_pages), i = (int)(at % a.max_pages);
  const int q0 = min(max(a.q_start[b], 0), a.n_q), n = min(max(a.q_start[b + 1], 0), a.n_q) - q0;
  const int len = min(max(a.seq_lens[b], 0), a.max_pages * kP);
  if (n <= 0 || i * kP >= len) return;
  const int window = a.window > 0 ? min(a.window, kNoWindow) : kNoWindow;
  const int start = max(len - n - window + 1, 0), from = start / kP;
  if (i >= min((min(a.sinks, start) + kP - 1) / kP, from) && i < from) return;  // no new token sees it
  const uint8_t* blk = a.pages + ((size_t)a.block_table[at] * a.Hkv + kvh) * block_bytes_of(FMT, NG);
  const u4v rk = load_k<FMT, NG>(blk, FMT == kInt4 ? w : w / 2), rv = load_v<FMT, NG>(blk, FMT == kInt4 ? w : w / 2);
  uint32_t ek[NG], ev[NG];
  load_entries<FMT, NG>(blk, 0, ek);
  load_entries<FMT, NG>(blk, 1, ev);
  Exponent e[2];
  const bool seen = Seen{len, start, a.sinks}(i * kP + l);
  make_scales<FMT, NG>(ek, 0, a.meta_bf16, seen, scales[w], e[0]);
  make_scales<FMT, NG>(ev, 1, a.meta_bf16, seen, scales[w], e[1]);
  lane_exchange();
  uint8_t* dst = a.expanded + (size_t)blockIdx.x * kExpandedBytes;
  expand_part<FMT, NG, true>(rk, 0, w, scales[w], dst);
  expand_part<FMT, NG, true>(rv, 1, w, scales[w], dst + kExpandedBytes / 2);
  if (threadIdx.x == 0) a.exps[blockIdx.x] = make_int2(e[0].e, e[1].e);
}

// The product of a rotation's operands in LDS, half at rot, half at rot2, with x.  (Operands read
// ahead of their products changed nothing: other waves' products fill the gaps.)
__device__ inline void rotate(const u4v (&x)[8], f16v (&y)[4], const uint8_t* rot, const uint8_t* rot2) {
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int C = 0; C < 4; ++C) {
#pragma unroll
    for (int i = 0; i < 16; ++i) y[C][i] = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const u4v* op = reinterpret_cast<const u4v*>((C < 2 ? rot : rot2) + (C % 2 * 8 + k) * 2048 + l * 16);
      y[C] = mfma<kHalf>(op[64], x[k], y[C]);
      y[C] = mfma<kHalf>(op[0], x[k], y[C]);
    }
  }
}

// q~ = q R_k as the score products' operands, fp16 divided by a power of two that c takes; R_k's
// operands in LDS (rotate).  Returns as load_queries.
__device__ inline bool rotate_queries(const ChunkArgs& a, size_t row, bool live, const uint8_t* rot,
                                      const uint8_t* rot2, u4v (&q)[8], float& c) {
  const int l = threadIdx.x & 63, h = l >> 5;
  const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;
  u4v x[8];
  uint32_t top_q = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    x[k] = live ? *reinterpret_cast<const u4v*>(a.q + row * kD + 16 * k + 8 * h) : u4v{0, 0, 0, 0};
    top_q = top_bf16(top_q, x[k]);
    x[k] ^= flip;
  }
  const int e1 = max(exp_of(half_max_bits(top_q)), -100) - 13;
#pragma unroll
  for (int k = 0; k < 8; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) x[k][j] = pack2<kInt4>(ldexpf(bf_lo(x[k][j]), -e1), ldexpf(bf_hi(x[k][j]), -e1));
  f16v y[4];
  rotate(x, y, rot, rot2);
  float top = 0.0f;
#pragma unroll
  for (int C = 0; C < 4; ++C)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(y[C][i]));
  const int e2 = max(exp_of(half_max(top)), -60) - 13;
#pragma unroll
  for (int k = 0; k < 8; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      q[k][j] = pack2<kHalf>(ldexpf(y[k / 2][8 * (k % 2) + 2 * j], -e2),
                             ldexpf(y[k / 2][8 * (k % 2) + 2 * j + 1], -e2));
  c = fabsf(a.scale) * pow2(e1 + e2);
  return top_q >= kInfBits;
}
// o = o~ R_v^T, o~ = the sums / l 2^e as fp16 (divided by a power of two): rows of the output's
// channels in order; returns what they are still to be multiplied by to be the sums again.
__device__ inline float rotate_output(f16v (&o)[4], float l, int e, const uint8_t* rot, const uint8_t* rot2) {
  const float il = l > 0.0f ? 1.0f / l : is_nan(l) ? l : 0.0f;
  float top = 0.0f;
#pragma unroll
  for (int C = 0; C < 4; ++C)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      o[C][i] *= il;
      top = fmaxf(top, fabsf(o[C][i]));
    }
  const int e3 = max(exp_of(half_max(top)), -100) - 13;
  u4v x[8];
#pragma unroll
  for (int k = 0; k < 8; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      x[k][j] = pack2<kHalf>(ldexpf(o[k / 2][8 * (k % 2) + 2 * j], -e3),
                             ldexpf(o[k / 2][8 * (k % 2) + 2 * j + 1], -e3));
  rotate(x, o, rot, rot2);
  return ldexpf(l, e3 + e);
}

// ---------------------------------------------------------------------------
// Many rows: W waves of 32 rows share every page through LDS.  4 D flops per (row, token), on the
// matrix cores; per page and wave 32 products (1024 cycles of a SIMD's matrix core) beside 32
// exponentials a lane and their fp32 steps, which are issued between the value products.
//   A page's 32 KiB come by loads straight to LDS, issued W = 8: two pages, 4: one page before their
// use, so that no registers hold them; the next operands are read from LDS three steps ahead of the
// score products, one ahead of the value products.  One barrier a page: the slot that it frees is
// the one filled next.  Codes (W = 4) come to registers a page ahead, and each wave makes a quarter of
// the page's operands.
//   8 waves read a page once where 4 do twice, and hide the loads two pages deep: a prompt of 8192
// tokens, 32 query heads on 8: 500 to 550 us from card to card (1.00 to 1.10 PFLOP/s, of 1.36 that a
// large library product reaches), by 4 waves 530 to 600; 2048 tokens over 16k in 4 bits 555 (expanded beforehand), by 4 waves 770.
// Without reads from LDS the prompt takes 90 % of its time, without loads 86, without the softmax 85,
// the products alone 60.  Matrix cores are busy 48 to 54 % of it at 1.9 to 2.1 GHz, the clock that
// the power limit leaves (in the library product: 73 % at 1.4 to 1.8).
// ---------------------------------------------------------------------------
template <int FMT, int NG, int W, bool HL = false>  // HL: p in two pieces
__global__ __launch_bounds__(64 * W, 2) void chunk_kernel(ChunkArgs a) {
  constexpr int M = kRows * W;
  constexpr bool CODES = FMT == kInt4 || FMT == kInt2;
  constexpr int kSlots = W == 8 ? 3 : 2;
  static_assert(W == 4 || (W == 8 && !CODES), "a block expands codes a part per wave");
  static_assert(2 * kPageLds == kRotBytes, "a rotation's operands fit in two pages' slots");
  // (codes: no loads to LDS, one array; a loop without copies of itself for the slots needs fewer registers)
  __shared__ __align__(16) uint8_t slot0[CODES ? 2 * kPageLds : kPageLds], slot1[CODES ? 16 : kPageLds],
      slot2[kSlots == 3 ? kPageLds : 16];
  auto lds_of = [&](auto s) -> uint8_t* {
    if constexpr (CODES) return slot0 + s * kPageLds;
    else return s.value == 0 ? slot0 : s.value == 1 ? slot1 : slot2;
  };
  auto ahead_of = [](auto s) {  // the slot that is free
    if constexpr (CODES) return 1 - s;
    else return std::integral_constant<int, s.value == 0 ? kSlots - 1 : s.value - 1>{};
  };
  uint8_t* const second = CODES ? slot0 + kPageLds : slot1;
  __shared__ Scales<CODES ? NG : 1> scales[CODES ? W : 1];
  __shared__ int exps[2][kSlots];  // CODES: of the slots: K's exponent, the accumulators'
  const int g = a.Hq / a.Hkv;
  const int kvh = blockIdx.x % a.Hkv;
  const int window = a.window > 0 ? min(a.window, kNoWindow) : kNoWindow;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, n = l & 31, h = l >> 5;
  Walk walk = start_walk(a, g, M, window);
  for (Segment sg; next_segment(a, walk, g, M, window, sg);) {
    const Tile& t = sg.t;
    const Pages& pg = sg.pg;
    const int r = t.row0 + w * kRows + n;
    const bool live = r < t.rows;
    const size_t row = (size_t)(t.q0 + (live ? r / g : 0)) * a.Hq + kvh * g + (live ? r % g : 0);
    const bool direct = sg.whole;
    const Seen seen_by = seen_by_rows<FMT>(t, pg, window, a.sinks);
    const int x0 = sg.x0, x1 = sg.x1;
    if (x0 >= x1) {
      if (live) store_empty(a, row, sg, direct, h);
      continue;
    }
    RowState rs;
    rs.pos = live ? t.len - t.n + r / g : -1;
    rs.m = -INFINITY;
    rs.l = 0.0f;
    // a rotation's operands from global memory to slots 0 and 1, by all waves; until all is there
    auto fill = [&](const uint8_t* src) {
#pragma unroll 1
      for (int i = 0; i < kPageLds / 1024 / W; ++i) {
        const int at = (w + i * W) * 1024;
        load_to_lds(src + at + l * 16, slot0 + at);
        load_to_lds(src + kPageLds + at + l * 16, second + at);
      }
      wait_loads<0>();
      lds_barrier();
    };
    const uint8_t* rot = FMT != kBf16 ? a.rot + (size_t)(a.rph ? kvh : 0) * 2 * kRotBytes : nullptr;
    u4v q[8];
    bool lost;
    if constexpr (FMT != kBf16) {
      fill(rot);
      lost = rotate_queries(a, row, live, slot0, second, q, rs.c);
      lds_barrier();
    } else {
      lost = load_queries<FMT>(a, row, live, q, rs.c);
    }
    if (lost && rs.pos >= 0) rs.l = __uint_as_float(0x7fc00000u);
    const int32_t* bt = a.block_table + (size_t)t.b * a.max_pages;
    auto page_of = [&](int x) { return x < pg.head ? x : pg.from + x - pg.head; };
    // index of a page's block: its number is loaded a page before it is needed
    auto block_of = [&](int x) -> int64_t {
      const int i = page_of(min(x, x1 - 1));
      return (FMT == kHalf ? (int64_t)t.b * a.max_pages + i : (int64_t)scalar_load(bt + i)) * a.Hkv + kvh;
    };
    auto page_exps = [&](int x) {
      const int* e = reinterpret_cast<const int*>(a.exps + block_of(x));
      return make_int2(scalar_load(e), scalar_load(e + 1));
    };
    // bf16, kHalf: this wave's part of a page, straight to LDS
    constexpr int kLoads = 32 / W;
    auto fetch = [&](int64_t block, uint8_t* dst) {
      const uint8_t* src = (FMT == kHalf ? a.expanded : a.pages) + block * kPageLds + w * kLoads * 1024 + l * 16;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load_to_lds(src + i * 1024, dst + (w * kLoads + i) * 1024);
    };
    // codes: a wave takes a quarter of K's and of V's codes to registers, and a page later makes 4
    // operands of 1 KB of each
    u4v raw[2];
    uint32_t ent[2][NG];
    Exponent e_v;
    auto load_codes = [&](int64_t block) {
      const uint8_t* blk = a.pages + block * block_bytes_of(FMT, NG);
      const int i = FMT == kInt4 ? w : w / 2;
      raw[0] = load_k<FMT, NG>(blk, i);
      raw[1] = load_v<FMT, NG>(blk, i);
      load_entries<FMT, NG>(blk, 0, ent[0]);
      load_entries<FMT, NG>(blk, 1, ent[1]);
    };
    auto expand = [&](int x, int slot) {
      const bool seen = seen_by(page_of(x) * kP + l);
      Scales<NG>& sc = reinterpret_cast<Scales<NG>*>(scales)[w];
      uint8_t* dst = slot0 + slot * kPageLds;
      lane_exchange();
      Exponent e_k;
      make_scales<FMT, NG>(ent[0], 0, a.meta_bf16, seen, sc, e_k);
      make_scales<FMT, NG>(ent[1], 1, a.meta_bf16, seen, sc, e_v);
      if (threadIdx.x == 0) {
        exps[0][slot] = e_k.e;
        exps[1][slot] = e_v.e;
      }
      lane_exchange();
      expand_part<FMT, NG, false>(raw[0], 0, w, sc, dst);
      expand_part<FMT, NG, false>(raw[1], 1, w, sc, dst + kHalfLds);
    };
    f16v o[4];
#pragma unroll
    for (int C = 0; C < 4; ++C)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[C][i] = 0.0f;
    Exponent e_o;  // the accumulators'
    float unit = 1.0f;
    int64_t ahead_block = block_of(x0 + kSlots - 1);
    if (!CODES) {
      fetch(block_of(x0), slot0);
      wait_loads<0>();
      if (kSlots == 3 && x0 + 1 < x1) fetch(block_of(x0 + 1), slot1);
    } else {
      load_codes(block_of(x0));
      expand(x0, 0);
    }
    int2 ex_next = make_int2(0, 0);
    if (FMT == kHalf) ex_next = page_exps(x0);
    lds_barrier();
    // positions of the wave's first and last row (none: nothing is seen)
    const int wr0 = t.row0 + w * kRows, wr1 = min(wr0 + kRows, t.rows) - 1;
    const int w_min = t.len - t.n + wr0 / g, w_max = wr0 <= wr1 ? t.len - t.n + wr1 / g : -1;
    // A lane's offset among a step's operands; the compiler does not see that its low bits are 0, and so
    // adds a slot's address to it once (it put the address' bits in before each read otherwise).
    const int k_lane = stay(FMT == kBf16 ? (l & 15) * 16 + ((l >> 4) & 1) * 4096 + h * 256 : l * 16);
    const int v_lane = FMT == kBf16 ? stay((l & 15) * 16 + ((l >> 4) & 1) * 2048 + h * 256) : k_lane;
    int x = x0;
    auto page = [&](auto slot) {
      const auto ahead = ahead_of(slot);
      const int t0 = page_of(x) * kP;
      const bool next = x + 1 < x1;
      if (!CODES) {
        if (x + kSlots - 1 < x1) fetch(ahead_block, lds_of(ahead));
      } else if (next) {
        load_codes(ahead_block);
      }
      ahead_block = block_of(x + kSlots);
      float cp = rs.c, weight = 0.0f;  // weight (log2) of the page's values against the accumulators'
      if (FMT != kBf16) {
        int e_k;
        const int e_old = e_o.e;
        if (FMT == kHalf) {
          e_k = ex_next.x;
          e_o.follow(ex_next.y);
          weight = (float)max(ex_next.y - e_o.e, -60);
          if (next) ex_next = page_exps(x + 1);
        } else {
          e_k = __builtin_amdgcn_readfirstlane(exps[0][slot]);
          e_o.e = __builtin_amdgcn_readfirstlane(exps[1][slot]);
        }
        cp = fmaxf(rs.c * pow2(e_k), kLeast);
        if (e_o.e != e_old && e_old != kNoExp) {
          const float f = unit_change(e_old, e_o.e);
#pragma unroll
          for (int C = 0; C < 4; ++C) o[C] *= f;
        }
      }
      uint8_t* base = lds_of(slot);
      if (FMT == kBf16 && !seen_by.whole_page(t0)) {
        for (int i = threadIdx.x; i < kP * kD / 8; i += 64 * W) {  // 16 bytes: slots 16 hi + 8 kt + e
          const int first = 16 * ((i >> 4) & 3) + 8 * ((i >> 6) & 1);
          u4v& v = reinterpret_cast<u4v*>(base + kHalfLds)[i];
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] &= seen_by.pair(t0 + first + 2 * j);
        }
        lds_barrier();
      }
      // the wave's rows see something of the page
      const bool seen = t0 <= w_max && (t0 + kP - 1 > w_min - window || t0 < a.sinks);
      if (seen) {
        // scores, the operands read three steps ahead
        f16v s[2];
        {
          auto k_at = [&](int T, int k) {
            const int off = FMT == kBf16 ? T * 8192 + (k % 4) * 1024 + (k / 4) * 512 : (T * 8 + k) * 1024;
            return *reinterpret_cast<const u4v*>(base + k_lane + off);
          };
          u4v ka[4][2];
#pragma unroll
          for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int T = 0; T < 2; ++T) ka[k][T] = k_at(T, k);
#pragma unroll
          for (int T = 0; T < 2; ++T)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[T][i] = 0.0f;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            if (k + 3 < 8)
#pragma unroll
              for (int T = 0; T < 2; ++T) ka[(k + 3) % 4][T] = k_at(T, k + 3);
#pragma unroll
            for (int T = 0; T < 2; ++T) s[T] = mfma<FMT>(ka[k % 4][T], q[k], s[T]);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        auto v_at = [&](int C, int k) {
          const int off = FMT == kBf16 ? C * 4096 + (k % 2) * 1024 + (k / 2) * 512 : (C * 4 + k) * 1024;
          return *reinterpret_cast<const u4v*>(base + kHalfLds + v_lane + off);
        };
        u4v va[2][4];
#pragma unroll
        for (int C = 0; C < 4; ++C) va[0][C] = v_at(C, 0);
        if (t0 + kP - 1 > w_min || (t0 <= w_max - window && t0 + kP > a.sinks))
          mask_page(s, rs.pos, t0, window, a.sinks);
        move_reference(s, o, rs, cp);
        // weights of a step's operand, two at a time between the products of the step before
        const float ms = (rs.m == -INFINITY ? 0.0f : -rs.m) + kWeightUp<FMT> + weight;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        u4v p[2], pl[2];
        auto weights = [&](int k, int i) {
          auto one = [&](int e) {
            const int y = v_slot<FMT>(e), u = y % 4;
            return __builtin_amdgcn_exp2f(fmaf(s[u / 2][8 * (u % 2) + 4 * (k / 2) + 2 * (k % 2) + y / 4], cp, ms));
          };
          const float x = one(2 * i), y = one(2 * i + 1);
          sum[i] += x;
          sum[i] += y;
          p[k % 2][i] = pack2<FMT>(x, y);
          if (HL) pl[k % 2][i] = pack2<FMT>(x - bf_lo(p[k % 2][i]), y - bf_hi(p[k % 2][i]));
        };
#pragma unroll
        for (int i = 0; i < 4; ++i) weights(0, i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (k + 1 < 4)
#pragma unroll
            for (int C = 0; C < 4; ++C) va[(k + 1) % 2][C] = v_at(C, k + 1);
#pragma unroll
          for (int C = 0; C < 4; ++C) {
            if (HL) o[C] = mfma<FMT>(va[k % 2][C], pl[k % 2], o[C]);
            o[C] = mfma<FMT>(va[k % 2][C], p[k % 2], o[C]);
            if (k + 1 < 4) weights(k + 1, C);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        float total = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        total = stay(total);  // the additions stay among the products
        rs.l = FMT == kHalf ? fmaf(total, __builtin_amdgcn_exp2f(-weight), rs.l) : rs.l + total;
      }
      if (!CODES) {  // page x + 1 has landed
        if (kSlots == 3 && x + 2 < x1) wait_loads<kLoads>();
        else wait_loads<0>();
      }
      if constexpr (CODES) {
        if (next) expand(x + 1, ahead);
      }
      lds_barrier();
      ++x;
    };
    if constexpr (CODES) {
      int slot = 0;
      do {
        page(slot);
        slot = 1 - slot;
      } while (x < x1);
    } else {
      do {
        page(std::integral_constant<int, 0>{});
        if (x >= x1) break;
        page(std::integral_constant<int, 1>{});
        if constexpr (kSlots == 3) {
          if (x >= x1) break;
          page(std::integral_constant<int, 2>{});
        }
      } while (x < x1);
    }
    rs.l = half_sum(rs.l);
    if constexpr (FMT != kBf16) {
      fill(rot + kRotBytes);
      unit = rotate_output(o, rs.l, e_o.e, slot0, second);
    }
    if (live) store_row(a, row, sg, direct, o, rs.m, rs.l, unit, h);
    lds_barrier();  // the slots are free again
  }
}

// ---------------------------------------------------------------------------
// Few rows: a block takes one tile of 32 rows, its waves every fourth page each, from global
// memory straight to the operands; the waves' states are merged in LDS.
//   bf16: bound by the bytes.  A page's 16 KiB of K are loaded while the page before is multiplied,
// its V while its scores are: one wave a SIMD with 400 registers.  64 sequences of 16k to 32k tokens,
// one new each in a window of 4096, 32 query heads on 8: 174 us, 6.2 TB/s.
//   Codes: bound by a page's chain (scales, scores, maximum, exponentials, values) of two waves a
// SIMD: 640 (2 bits, one group) to 750 (4 bits, four groups) vector instructions, 320 to 350 of them to
// expand the codes (a conversion and a multiply-add for two, and masks), 150 the softmax of 32 rows; vector ALUs are busy
// 50 to 75 % of the time, matrix cores 20.  K and V are loaded a page ahead, V's codes into registers of
// their own.  32 sequences of 4k to 16k tokens, 5 new each, 32 heads on 8, 4 bits: 107 us and, with
// rotations and merge, 123; 16 of up to 32k, 4 new, 64 heads, 2 bits: 84 and 97.
// ---------------------------------------------------------------------------
template <int FMT, int NG>
__global__ __launch_bounds__(256, FMT == kBf16 ? 1 : 2) void chunk_few_kernel(ChunkArgs a) {
  constexpr int M = kRows;
  constexpr bool HL = FMT == kBf16;  // p in two bf16 pieces: costs nothing where the loads bound
  __shared__ Scales<FMT == kBf16 ? 1 : NG> scales[FMT == kBf16 ? 1 : kWaves];
  __shared__ float4 os[kWaves][4][4][64];
  __shared__ float2 ml[kWaves][kRows];
  const int g = a.Hq / a.Hkv;
  const int kvh = blockIdx.x % a.Hkv;
  const int window = a.window > 0 ? min(a.window, kNoWindow) : kNoWindow;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, n = l & 31, h = l >> 5;
  const int lo = l & 15, b16 = (l >> 4) & 1;
  Walk walk = start_walk(a, g, M, window);
  for (Segment sg; next_segment(a, walk, g, M, window, sg);) {
    const Tile& t = sg.t;
    const Pages& pg = sg.pg;
    const int r = t.row0 + n;
    const bool live = r < t.rows;
    const size_t row = (size_t)(t.q0 + (live ? r / g : 0)) * a.Hq + kvh * g + (live ? r % g : 0);
    const bool direct = FMT == kBf16 && sg.whole;
    const Seen seen_by = seen_by_rows<FMT>(t, pg, window, a.sinks);
    const int x0 = sg.x0, x1 = sg.x1;
    RowState rs;
    rs.pos = live ? t.len - t.n + r / g : -1;
    rs.m = -INFINITY;
    rs.l = 0.0f;
    f16v o[4];
#pragma unroll
    for (int C = 0; C < 4; ++C)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[C][i] = 0.0f;
    Exponent e_v;
    if (x0 + w < x1) {
      const int32_t* bt = a.block_table + (size_t)t.b * a.max_pages;
      auto page_of = [&](int x) { return x < pg.head ? x : pg.from + x - pg.head; };
      auto block_of = [&](int x) {
        return a.pages + ((size_t)scalar_load(bt + page_of(x)) * a.Hkv + kvh) * block_bytes_of(FMT, NG);
      };
      constexpr int kL = FMT == kBf16 ? 16 : raw_loads<FMT>();
      u4v rk[kL], rv0[kL], rv1[FMT == kBf16 ? 1 : kL];  // codes: V's of the next page beside the page's
      uint32_t ks[NG], vs[NG];
      auto fetch_k = [&](const uint8_t* blk) {
#pragma unroll
        for (int i = 0; i < kL; ++i) {
          if (FMT == kBf16) {  // (T, ks) = (i / 8, i % 8)
            const int off = (i / 8) * 8192 + (i % 4) * 1024 + (i / 4 % 2) * 512 + b16 * 4096 + h * 256 + lo * 16;
            rk[i] = __builtin_nontemporal_load(reinterpret_cast<const u4v*>(blk + off));
          } else {
            rk[i] = load_k<FMT, NG>(blk, i);
          }
        }
      };
      auto fetch_v = [&](const uint8_t* blk, auto& rv) {
#pragma unroll
        for (int i = 0; i < kL; ++i) {
          if (FMT == kBf16) {  // (C, step) = (i / 4, i % 4)
            const int off = kHalfLds + (i / 4) * 4096 + (i % 2) * 1024 + (i / 2 % 2) * 512 + b16 * 2048 + h * 256 +
                            lo * 16;
            rv[i] = __builtin_nontemporal_load(reinterpret_cast<const u4v*>(blk + off));
          } else {
            rv[i] = load_v<FMT, NG>(blk, i);
          }
        }
      };
      const uint8_t* blk = block_of(x0 + w);
      fetch_k(blk);
      if (FMT != kBf16) {
        fetch_v(blk, rv0);
        load_entries<FMT, NG>(blk, 0, ks);
        load_entries<FMT, NG>(blk, 1, vs);
      }
      u4v q[8];
      if (load_queries<FMT>(a, row, live, q, rs.c) && rs.pos >= 0) rs.l = __uint_as_float(0x7fc00000u);
      Scales<NG>& sc = reinterpret_cast<Scales<NG>*>(scales)[FMT == kBf16 ? 0 : w];
      int x = x0 + w;
      auto page = [&](auto& rv, auto& rv_next) {
        const int t0 = page_of(x) * kP;
        const bool more = x + kWaves < x1;
        const uint8_t* next = more ? block_of(x + kWaves) : blk;
        int e_k = 0;
        if (FMT == kBf16) {
          fetch_v(blk, rv);
        } else {
          const int e_old = e_v.e;
          const bool seen = seen_by(t0 + l);
          Exponent page_k;
          lane_exchange();  // the last page's scales have been read
          make_scales<FMT, NG>(ks, 0, a.meta_bf16, seen, sc, page_k);
          make_scales<FMT, NG>(vs, 1, a.meta_bf16, seen, sc, e_v);
          lane_exchange();
          e_k = page_k.e;
          if (e_v.e != e_old && e_old != kNoExp) {
            const float f = unit_change(e_old, e_v.e);
#pragma unroll
            for (int C = 0; C < 4; ++C) o[C] *= f;
          }
        }
        f16v s[2];
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[T][i] = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
          for (int T = 0; T < 2; ++T) {
            u4v ka;
            if constexpr (FMT == kBf16) ka = rk[8 * T + k];
            else ka = k_operand<FMT, NG>(rk[FMT == kInt4 ? 2 * T + k / 4 : T], T, k, sc);
            s[T] = mfma<FMT>(ka, q[k], s[T]);
          }
        if (more) {  // the next page's loads, as soon as there is room for them
          fetch_k(next);
          if (FMT != kBf16) {
            fetch_v(next, rv_next);
            load_entries<FMT, NG>(next, 0, ks);
            load_entries<FMT, NG>(next, 1, vs);
          }
        }
        const bool masked = t0 + kP - 1 > pg.p_min || (t0 <= pg.p_max - window && t0 + kP > a.sinks);
        u4v p[4], pl[4];
        if (masked) mask_page(s, rs.pos, t0, window, a.sinks);
        softmax_page<FMT, HL>(s, o, rs, FMT == kBf16 ? rs.c : fmaxf(rs.c * pow2(e_k), kLeast), p, pl);
        if (FMT == kBf16 && !seen_by.whole_page(t0)) {
#pragma unroll
          for (int i = 0; i < kL; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              rv[i][j] &= seen_by.pair(t0 + 32 * (i / 2 % 2) + 16 * h + 8 * (i % 2) + 2 * j);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int C = 0; C < 4; ++C) {
            u4v va;
            if constexpr (FMT == kBf16) va = rv[4 * C + k];
            else va = v_operand<FMT, NG>(rv[FMT == kInt4 ? 2 * (C / 2) + k % 2 : k / 2], C, k / 2, k % 2, sc);
            if (HL) o[C] = mfma<FMT>(va, pl[k], o[C]);
            o[C] = mfma<FMT>(va, p[k], o[C]);
          }
        blk = next;
        x += kWaves;
      };
      if constexpr (FMT == kBf16) {
        do page(rv0, rv0);
        while (x < x1);
      } else {
        do {
          page(rv0, rv1);
          if (x >= x1) break;
          page(rv1, rv0);
        } while (x < x1);
      }
    }
    // merge: wave w sums tile C = w of the four states
    const float unit = FMT == kBf16 || e_v.e == kNoExp ? 1.0f : ldexpf(1.0f, e_v.e);
    const float lt = half_sum(rs.l);
    // (NaN in a row: its scores have no maximum, but the state is not empty)
    if (h == 0) ml[w][n] = make_float2(is_nan(lt) ? 0.0f : rs.m, lt);
#pragma unroll
    for (int C = 0; C < 4; ++C)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        os[w][C][i][l] = make_float4(o[C][4 * i] * unit, o[C][4 * i + 1] * unit, o[C][4 * i + 2] * unit,
                                     o[C][4 * i + 3] * unit);
    __syncthreads();
    float m = -INFINITY, L = 0.0f, f[kWaves];
#pragma unroll
    for (int k = 0; k < kWaves; ++k) m = fmaxf(m, ml[k][n].x);
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      f[k] = ml[k][n].x == -INFINITY ? 0.0f : exp2f(ml[k][n].x - m);
      L += f[k] * ml[k][n].y;
    }
    // each wave stores a quarter of the channels: registers 4 w .. 4 w + 3 of every tile
    float sum[4][4] = {};
#pragma unroll
    for (int C = 0; C < 4; ++C)
#pragma unroll
      for (int k = 0; k < kWaves; ++k) {
        const float4 v = os[k][C][w][l];
        const bool counts = f[k] != 0.0f;
        sum[C][0] = fmaf(f[k], counts ? v.x : 0.0f, sum[C][0]);
        sum[C][1] = fmaf(f[k], counts ? v.y : 0.0f, sum[C][1]);
        sum[C][2] = fmaf(f[k], counts ? v.z : 0.0f, sum[C][2]);
        sum[C][3] = fmaf(f[k], counts ? v.w : 0.0f, sum[C][3]);
      }
    if (is_nan(L))  // the values as well: a merge may look at them alone
#pragma unroll
      for (int C = 0; C < 4; ++C)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[C][i] = L;
    if (live) {
      const float il = L > 0.0f ? 1.0f / L : is_nan(L) ? L : 0.0f;
      const size_t at = row * a.num_splits + sg.slot;
      auto put = [&](int c, float x, float y, float z, float v) {
        if (direct) {
          uint2 d;
          d.x = pack2<kBf16>(x * il, y * il);
          d.y = pack2<kBf16>(z * il, v * il);
          *reinterpret_cast<uint2*>(a.out + row * kD + c) = d;
        } else if (m != -INFINITY) {  // of an empty state only that is read
          *reinterpret_cast<float4*>(a.part_o + at * kD + c) = make_float4(x, y, z, v);
        }
      };
      const int rr = 8 * w + 4 * h;
      if (FMT == kInt2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) put(4 * (rr + i), sum[0][i], sum[1][i], sum[2][i], sum[3][i]);
      } else {
#pragma unroll
        for (int C = 0; C < 4; ++C)
          put(FMT == kBf16 ? 32 * C + rr : 64 * (C / 2) + 32 * (rr / 16) + 16 * (C % 2) + rr % 16, sum[C][0], sum[C][1],
              sum[C][2], sum[C][3]);
      }
      if (w == 0 && h == 0 && (!direct || a.num_splits > 1)) {
        float2* dst = reinterpret_cast<float2*>(a.part_ml) + row * a.num_splits;
        dst[sg.slot] = direct ? make_float2(kDone, 0.0f) : make_float2(m, L);
        if (sg.last && !direct)
          for (int i = sg.slot + 1; i < a.num_splits; ++i) dst[i] = make_float2(-INFINITY, 0.0f);
      }
    }
    __syncthreads();  // os, ml and the scales are free again
  }
}

// Merge of the partial states in the output's basis, of the rows that belong to a sequence and have
// no output yet: 32 lanes a row, four channels each.  A lane reads the maximum and sum of one slot in
// 32; the states' loads are issued eight slots at a time (empty ones, at the end but for pages that
// the row does not see, weigh 0).  Bound by the states' latency: a call with one token of 32
// heads over 16k of bf16 took 40 us slot by slot, 23 now.
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkArgs a, int64_t row0) {
  const int64_t row = row0 + (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int c = threadIdx.x & 31, S = a.num_splits;
  if (row >= (int64_t)min(max(scalar_load(a.q_start + a.B), 0), a.n_q) * a.Hq) return;
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + row * S;
  const float2 first = ml[min(c, S - 1)];
  if (__shfl(first.x, 0, 32) == kDone) return;
  float M = -INFINITY;
  int live = 0;  // one past the last state that is not empty
  for (int s0 = 0; s0 < S; s0 += 32) {
    const float2 x = s0 == 0 ? first : ml[min(s0 + c, S - 1)];
    const bool is = s0 + c < S && x.x != -INFINITY;
    M = fmaxf(M, is ? x.x : -INFINITY);
    live = max(live, is ? s0 + c + 1 : 0);
  }
#pragma unroll
  for (int m = 16; m >= 1; m >>= 1) {
    M = fmaxf(M, __shfl_xor(M, m, 32));
    live = max(live, __shfl_xor(live, m, 32));
  }
  const float4* po = reinterpret_cast<const float4*>(a.part_o + row * S * kD) + c;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float L = 0.0f;
  for (int s0 = 0; s0 < live; s0 += 8) {
    float2 x[8];
    float4 v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int s = min(s0 + k, live - 1);
      x[k] = ml[s];
      v[k] = po[(size_t)s * (kD / 4)];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (s0 + k >= live || x[k].x == -INFINITY) continue;  // (nothing but -inf is written of an empty state)
      const float e = __builtin_amdgcn_exp2f(x[k].x - M);
      L = fmaf(e, x[k].y, L);
      o.x = fmaf(e, v[k].x, o.x);
      o.y = fmaf(e, v[k].y, o.y);
      o.z = fmaf(e, v[k].z, o.z);
      o.w = fmaf(e, v[k].w, o.w);
    }
  }
  const float il = L > 0.0f ? 1.0f / L : is_nan(L) ? L : 0.0f;
  uint2 d;
  d.x = pack2<kBf16>(o.x * il, o.y * il);
  d.y = pack2<kBf16>(o.z * il, o.w * il);
  reinterpret_cast<uint2*>(a.out + row * kD)[c] = d;
}

// Merge of the splits and back-rotation, of the rows that belong to a sequence.
template <int RB>
__global__ __launch_bounds__(kRedThreads) void chunk_reduce_kernel(ChunkArgs a, int row0, int n_rows) {
  const int64_t used = (int64_t)min(max(a.q_start[a.B], 0), a.n_q) * a.Hq - row0;
  const int rows = (int)(used < n_rows ? used : n_rows);
  if (rows <= 0) return;
  reduce_body<false, RB>(blockIdx.x, rows, a.num_splits, a.part_o + (size_t)row0 * a.num_splits * kD,
                         a.part_ml + (size_t)row0 * a.num_splits * 2, a.Rv, a.out + (size_t)row0 * kD, 0, a.rph, a.Hq,
                         a.Hkv);
}

template <int FMT, int NG>
hipError_t launch_fmt(const ChunkArgs& args, hipStream_t st) {
  const int g = args.Hq / args.Hkv;
  const bool quantized = FMT != kBf16;
  const int64_t page_heads = (int64_t)args.B * args.max_pages * args.Hkv;
  const int M = chunk_tile_rows(quantized, args.n_q, args.B, g, args.Hkv, args.max_pages);
  const ChunkArgs& a = args;
  const int64_t tiles = (int64_t)a.n_q * g / M + a.B;
  const int ranges = std::max(1, chunk_blocks(quantized, M) / a.Hkv);
  const unsigned blocks = (unsigned)((a.num_splits == 1 ? tiles : ranges) * a.Hkv);
  if constexpr (FMT != kBf16)
    if (M != kRows) {  // the rotations' operands, and (256 rows) the pages'
      const int64_t pages = M == kManyRows ? page_heads : 0;
      hipLaunchKernelGGL((expand_kernel<FMT, NG>), dim3((unsigned)(pages + kRotParts * 2 * (a.rph ? a.Hkv : 1))),
                         dim3(256), 0, st, a, pages);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  if (M == kRows)
    hipLaunchKernelGGL((chunk_few_kernel<FMT, NG>), dim3(blocks), dim3(256), 0, st, a);
  else if (FMT == kBf16 && (int64_t)a.n_q * g <= (int64_t)kRows * a.B)  // two pieces, as in tiles of 32
    hipLaunchKernelGGL((chunk_kernel<kBf16, 1, 4, true>), dim3(blocks), dim3(256), 0, st, a);
  else if (M == 4 * kRows)
    hipLaunchKernelGGL((chunk_kernel<FMT, NG, 4>), dim3(blocks), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((chunk_kernel<FMT == kBf16 ? kBf16 : kHalf, 1, 8>), dim3(blocks), dim3(512), 0, st, a);
  hipError_t e = hipGetLastError();
  const bool rotated = quantized && M == kRows;  // partial states in the rotated basis
  if (e != hipSuccess || (a.num_splits == 1 && !rotated)) return e;
  if (!rotated)
    return by_seqs(a.n_q, launch_seqs(a.Hq), [&](int t0, int n) {
      hipLaunchKernelGGL(chunk_merge_kernel, dim3((unsigned)(((int64_t)n * a.Hq + 7) / 8)), dim3(256), 0, st, a,
                         (int64_t)t0 * a.Hq);
      return hipGetLastError();
    });
  // rows in parts of whole tokens that a launch holds
  const int per = launch_seqs(a.Hq);
  return by_seqs(a.n_q, per, [&](int t0, int n) {
    const int row0 = t0 * a.Hq, rows = n * a.Hq;
    auto go = [&](auto rb) {
      constexpr int RB = decltype(rb)::value;
      hipLaunchKernelGGL((chunk_reduce_kernel<RB>), dim3((unsigned)query_blocks(n, a.Hq, a.Hkv, a.rph, RB)),
                         dim3(kRedThreads), 0, st, a, row0, rows);
    };
    switch (reduce_rows(rows)) {
      case 16: go(std::integral_constant<int, 16>{}); break;
      case 8: go(std::integral_constant<int, 8>{}); break;
      case 4: go(std::integral_constant<int, 4>{}); break;
      default: go(std::integral_constant<int, 2>{});
    }
    return hipGetLastError();
  });
}

}  // namespace

// Rows of a tile, by the rows that a sequence and KV head have on average (32 query and 8 KV heads
// below; us with the smaller tile, with the larger).
//  32, blocks whose waves take pages of their own: codes are then expanded by every wave for itself,
//      and no wave idles.  8 sequences of 8k tokens in 4 bits, 36 rows each: 58, 69 with 128; 64 rows:
//      56, 71; 128 rows: 90, 85; 32 sequences of 2k, 64 rows: 68, 77; 128 rows: 119, 84.  Of bf16
//      pages every wave has a whole page's loads in flight, but a CU holds one block and the next
//      one's start is seen: 64 sequences of 4k tokens, 4 rows each: 167, 184; of 1k: 48, 43; 128 of
//      300: 50, 37; 32 of 2k: 46, 49; one of 1k: 14, 26.
// 128 or 256 (one block of 8 waves to a CU instead of two of 4; codes expanded beforehand, to 2 GiB
//      at most): 8 sequences of 8k, 4 bits, 512 rows: 219, 241; 768: 357, 318; 1024: 381, 350; 2048:
//      730, 609.  32 of 2k: 220, 237; 306, 316; 398, 402; 757, 679.  bf16, 32 of 2k: 151, 192; 231, 254;
//      285, 282; 540, 526.
int chunk_tile_rows(bool quantized, int64_t n_q, int B, int heads_per_kv, int Hkv, int64_t max_pages) {
  const int64_t rows = n_q * heads_per_kv, heads = (int64_t)B * Hkv;
  if (quantized ? rows <= (int64_t)2 * kRows * B
                : rows <= (int64_t)kRows * B && (max_pages > 24 || heads < 2 * device_cus()))
    return kRows;
  return rows <= (int64_t)512 * B || (quantized && heads * max_pages > 65536) ? 4 * kRows : kManyRows;
}

// Blocks that the GPU holds at once.
int chunk_blocks(bool quantized, int tile_rows) {
  return device_cus() * (tile_rows == kManyRows || (tile_rows == kRows && !quantized) ? 1 : 2);
}

hipError_t launch_chunk_attn(const ChunkArgs& a, hipStream_t st) {
  if (a.format == kBf16) return launch_fmt<kBf16, 1>(a, st);
  if (a.format == kInt4)
    return a.ng == 4   ? launch_fmt<kInt4, 4>(a, st)
           : a.ng == 2 ? launch_fmt<kInt4, 2>(a, st)
                       : launch_fmt<kInt4, 1>(a, st);
  return a.ng == 4   ? launch_fmt<kInt2, 4>(a, st)
         : a.ng == 2 ? launch_fmt<kInt2, 2>(a, st)
                     : launch_fmt<kInt2, 1>(a, st);
}

}  // namespace oscar
