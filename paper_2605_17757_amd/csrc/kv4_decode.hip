// Decode attention over the 4-bit paged cache: the split kernel, and the merge with the
// sums of attention weights (the query rotation, and the merge without them, are the
// 2-bit path's prepare and reduce kernels).
//
// For a KV head with g query heads, q~ = q R_k sm_scale log2 e, a page's K as
// Q(k~)_c = s (n - z) with codes n in 0 .. 15 and one (s, z) per token t and group G of
// channels:
//   score_t  = sum_G s (sum_{c in G} q~_c n_c - z sum_{c in G} q~_c)
//   o~_c     = sum_t w_t n_c - sum_t w_t z_t,    w_t = 2^(score_t - m) s_t (of c's group)
// Both inner sums run on the matrix cores, as exact products summed in fp32.
//   Scores, bf16: a code enters as the 16-bit pattern n, the bf16 subnormal n 2^-133
//     (for the odd nibbles of a byte 16 n, in place), which masks and one shift make of
//     the packed nibbles: 5 instructions per 8 codes.  q~ 2^64 enters as three bf16
//     pieces, 8 bits of the significand each, together the whole fp32 value.
//   Values, fp16: a code enters as (n - 8) 2^-9, a packed multiply-add of the 16-bit
//     pattern (the fp16 subnormal n 2^-24).  (Subnormal operands lose bits in the matrix
//     cores, which align products by the operands' exponents: with (n - 8) 2^-24 the
//     output's error was 1e-5, where it is 5e-7 now.)
//     With the codes centred the two sums over tokens are as small as o~ itself; the
//     matrix cores drop product bits below the accumulator's last ones, and against
//     sums of uncentred codes that left errors of 1e-5 of the output.  w is scaled by a
//     power of two per page and group (s: 2^10 .. 2^11 at the page's largest) and enters as
//     two fp16 pieces, both rounded to nearest (truncated, the errors of many small weights
//     had one sign and added up): off by 2^-22 of itself at most, or by 2^-35 of the row's
//     largest weight at the page's largest scale where that is more.
// Where the pieces go (NCH chunks of 4 heads per KV head).  As rows of one 16-row operand:
// 4 heads fill it, one product per chunk does, and a lane adds the pieces of a sum.  As
// operands of their own, a row per head: 3 products (values: 2) serve 16 heads, the matrix
// cores add the pieces, smallest first.  Scores as rows up to 8 heads, values up to 4, where
// they take fewer products; past that as operands (12 heads, 16 x 128k tokens: 682 us as
// rows, 620; 16 heads, 16 x 65k: 403 and 332; 8 heads either way within 2 %).
// |q~| must stay below 2^56 (scores: 2^-69 n q~ 2^133 2^-64).
#include <hip/hip_fp16.h>

#include <algorithm>
#include <type_traits>

#include "reduce_body.h"
#include "split_ranges.h"

namespace oscar {
namespace {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef uint16_t us2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;         // waves of a block: a team on one range of pages
constexpr int kPw = 40;           // dwords per row of the weights operand in LDS, NCH 1
constexpr int kPwWide = 36;       // wider: 16 rows read at once, 4 dwords each, take all banks
constexpr float kSlack = 4.0f;    // how far (log2) a score may exceed the reference maximum before it moves
constexpr float kIn = 0x1p64f;    // scale of q~ in the scores' products with codes
constexpr float kOut = 0x1p69f;   // back: 2^133 / kIn
constexpr int kTop = 11;          // scales of a page enter below 2^kTop: w < 2^(kTop + kSlack)

__device__ inline f4v mfma(const u4v& a, const u4v& b, const f4v& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c,
                                                 0, 0, 0);
}
__device__ inline f4v mfma_h(const u4v& a, const u4v& b, const f4v& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0,
                                                0, 0);
}
__device__ inline float top16(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ inline uint32_t pack_hi(float lo, float hi) {  // the upper halves of two floats
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
// Nibbles of d as 16-bit lanes: (0, 4), (1, 5) x 16, (2, 6), (3, 7) x 16.
__device__ inline u4v unpack(uint32_t d) {
  constexpr uint32_t m = 0x000f000fu;
  return u4v{d & m, d & (m << 4), (d >> 8) & m, (d >> 8) & (m << 4)};
}
// Over the 16 lanes of a row, the same in each of them (rotations by 8, 4, 2, 1).
template <class Op>
__device__ inline float row_reduce(float x, Op op) {
  auto ror = [](float v, auto ctrl) {
    return __int_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xF, 0xF, false));
  };
  x = op(x, ror(x, std::integral_constant<int, 0x128>{}));
  x = op(x, ror(x, std::integral_constant<int, 0x124>{}));
  x = op(x, ror(x, std::integral_constant<int, 0x122>{}));
  return op(x, ror(x, std::integral_constant<int, 0x121>{}));
}
__device__ inline float row_sum(float x) {
  return row_reduce(x, [](float a, float b) { return a + b; });
}
__device__ inline float row_max(float x) {
  return row_reduce(x, [](float a, float b) { return fmaxf(a, b); });
}
// Bytes of 8 slots as fp16 (n - 8) 2^-9, of their low (lo) and of their high nibbles (hi).
__device__ inline uint32_t centred(uint32_t v, float mul) {
  const _Float16 m = (_Float16)mul, c = (_Float16)-0x1p-6f;
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(h2, v), h2{m, m}, h2{c, c}));
}
__device__ inline void unpack_v(uint32_t d0, uint32_t d1, u4v& lo, u4v& hi) {
  constexpr uint32_t m = 0x000f000fu;
  lo = u4v{centred(d0 & m, 0x1p15f), centred((d0 >> 8) & m, 0x1p15f), centred(d1 & m, 0x1p15f),
           centred((d1 >> 8) & m, 0x1p15f)};
  hi = u4v{centred(d0 & (m << 4), 0x1p11f), centred((d0 >> 8) & (m << 4), 0x1p11f),
           centred(d1 & (m << 4), 0x1p11f), centred((d1 >> 8) & (m << 4), 0x1p11f)};
}
__device__ inline h2 half2_of(float a, float b) { return __builtin_convertvector((f2{a, b}), h2); }  // nearest even
__device__ inline uint32_t pk_max(uint32_t a, uint32_t b) {  // of unsigned 16-bit lanes
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b)));
}
// Largest of a non-negative float's bits over the 16 lanes of a row.
__device__ inline uint32_t row_max_u(uint32_t x) {
  auto ror = [](uint32_t v, auto ctrl) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, true);
  };
  x = max(x, ror(x, std::integral_constant<int, 0x128>{}));
  x = max(x, ror(x, std::integral_constant<int, 0x124>{}));
  x = max(x, ror(x, std::integral_constant<int, 0x122>{}));
  return max(x, ror(x, std::integral_constant<int, 0x121>{}));
}

// Scale and zero of an entry.  (A binary16 that feeds one fused multiply-add is converted
// by it: no instruction of its own.)
template <bool BF>
__device__ inline float meta_s(uint32_t e) {
  return BF ? __uint_as_float(e << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)e);
}
template <bool BF>
__device__ inline float meta_z(uint32_t e) {
  return BF ? __uint_as_float(e & 0xffff0000u) : (float)__builtin_bit_cast(_Float16, (uint16_t)(e >> 16));
}

// Weights operands in LDS, rows of kPw dwords (64 slots), per wave.  NCH 1: of two groups, 8
// rows (head, piece) each.  Wider: of one, 16 rows for each of the two pieces.
template <int NCH>
constexpr int weight_dwords() {
  return NCH == 1 ? 16 * kPw : std::max(32 * kPwWide, NCH * 4 * kD);
}

template <int NCH>
struct SplitSmem {
  u4v qa[NCH <= 2 ? NCH : 3][4][64];          // query operands: chunk or piece, 32-channel block, lane
  uint32_t pw[kWaves][weight_dwords<NCH>()];  // weights operands; o~ at the end
  float ml[kWaves][NCH * 4][2];               // the waves' (m, l)
};

// ---------------------------------------------------------------------------
// split: the pages of all sequences end to end, cut into equal ranges (split_ranges.h),
// as many as blocks are resident; one block per (range, KV head), so that a page-head
// block is read once.  A block's 4 waves take every fourth page of the range's part of a
// sequence and merge their states in LDS: one partial state per part, and a short
// sequence's pages at once.  Per page a wave has
//   K in 4 loads of 1 KB (lane: slot 4 lo + u, channels 8 hi .. of four blocks of 32):
//     16 products per chunk (48 in all past 8 heads), lane (hi, slot) gets the sums of
//     heads NCH hi ..;
//   V in 4 loads (lane: 16 slots of channels 32 j + lo, + 16): the weights of a group go
//     through LDS into the operand's rows, 16 products (32 past 4 heads), added to o~
//     (lane: heads NCH hi .., 8 channels) after the page.
// The next page's K is loaded once this page's is used up, so that 5 KB per wave are
// always on their way at 8 waves per CU.
//
// Bound: up to 4 heads per KV head HBM (64 sequences of 16k to 32k tokens, 32/8 heads:
// 2.0 GB; 343 us in a trace, 310 at least, 5.9 and 6.5 TB/s; 554 vector instructions per
// page, VALU busy 63 %).  Beyond, the VALU: per page about 310 instructions that all chunks
// share (unpacking 224, metadata 84) and about 170 per chunk (scores 36, weights and their
// pieces 70, softmax 20, sums 8).  12 heads (16 x 128k tokens): 828 a page, busy 74 %, matrix
// cores 28 %, 625 us, 576 at least, 4.3 and 4.7 TB/s.
// Two waves per SIMD: at three, which the 4-head instances allow, 342 us for 340.  With
// the products' sums kept in the accumulators across pages (32 registers per chunk
// instead of 8) more than 8 heads went to scratch: 16 heads 555 us, 310 now.  Rotating
// the query in these blocks instead of a launch before: 21.6 us for 18.4 at batch 1.
// ---------------------------------------------------------------------------
constexpr int kPerSimd = 2;  // waves per SIMD

template <bool BF, int NG, int NCH>
__global__ __launch_bounds__(kWaves * 64) __attribute__((
    amdgpu_waves_per_eu(kPerSimd, kPerSimd))) void kv4_split_kernel(
    const uint8_t* __restrict__ pages, int Hkv, int Hq, const int32_t* __restrict__ block_table,
    int max_pages, const int32_t* __restrict__ seq_lens, int num_splits, int n_ranges, int B,
    const float* __restrict__ qt, float* __restrict__ part_o, float* __restrict__ part_ml,
    float* __restrict__ scores) {
  __shared__ SplitSmem<NCH> sm;
  constexpr int KPG = 4 / NG;                  // 32-channel blocks per group
  constexpr int kPieces = 3;                   // of q~
  const int r = (int)(blockIdx.x / (uint32_t)Hkv), kvh = (int)(blockIdx.x % (uint32_t)Hkv);
  const int g = Hq / Hkv;
  const int t = threadIdx.x, w = t >> 6, l = t & 63, lo = l & 15, hi = l >> 4;
  auto len_of = [&](int b) { return min(max(seq_lens[b], 0), max_pages * kP); };
  auto pages_of = [&](int b) { return (len_of(b) + kP - 1) / kP; };

  // The block's waves take pages p0 + w, p0 + w + 4, .. of pages [p0, p1) of sequence b.
  auto run_piece = [&](int b, int p0, int p1, int piece, bool last) {
    const int len = len_of(b);
    // ---- loads in the order of their use: page ids, the query, the first page's K ----
    const int32_t* __restrict__ bt = block_table + (size_t)b * max_pages;
    const int n_mine = (p1 - p0 - w + kWaves - 1) / kWaves;  // <= 0: none
    auto page_ids = [&](int i0) {  // lane i: page i0 + i of the wave's
      const int p = p0 + w + kWaves * (i0 + l);
      return i0 + l < n_mine ? bt[p] : 0;
    };
    int ids = page_ids(0);
    // The lane's heads are NCH hi + ch.  Wave w makes the operands of 32-channel block w: of
    // chunk ch, row 4 h + piece of head NCH h + ch; or of a piece, row 4 h + ch of that head.
    constexpr int kXr = NCH <= 2 ? NCH : 1;
    float4 xr[kXr][2], xs[NCH][2];
    {
      const float4 none = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      const float* row = qt + ((size_t)b * Hq + kvh * g) * kD;
#pragma unroll
      for (int k = 0; k < kXr; ++k) {
        const int head = NCH <= 2 ? NCH * (lo >> 2) + k : (lo & 3) < NCH ? NCH * (lo >> 2) + (lo & 3) : g;
        xr[k][0] = xr[k][1] = none;
        if (head < g) {
          const float4* src = reinterpret_cast<const float4*>(row + head * kD + 32 * w + 8 * hi);
          xr[k][0] = src[0];
          xr[k][1] = src[1];
        }
      }
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch) {
        const int hs = NCH * hi + ch;
        xs[ch][0] = xs[ch][1] = none;
        if (hs < g) {
          const float4* src = reinterpret_cast<const float4*>(row + hs * kD + 8 * lo);
          xs[ch][0] = src[0];
          xs[ch][1] = src[1];
        }
      }
    }
    auto block_of = [&](int i) {
      return pages + ((size_t)__builtin_amdgcn_readlane(ids, i & 63) * Hkv + kvh) * kv4_block_bytes(NG);
    };
    u4v kr[4], ks[NG];
    auto load_k = [&](const uint8_t* blk) {
      const u4v* p = reinterpret_cast<const u4v*>(blk) + l;
      const u4v* z = reinterpret_cast<const u4v*>(blk + kv4_sz_off(NG, 0)) + lo * NG;
#pragma unroll
      for (int u = 0; u < 4; ++u) kr[u] = __builtin_nontemporal_load(p + 64 * u);
#pragma unroll
      for (int u = 0; u < NG; ++u) ks[u] = z[u];  // entries (slot 4 lo + u, group)
    };
    const uint8_t* blk = pages;
    if (n_mine > 0) {
      blk = block_of(0);
      load_k(blk);
    }
    // ---- query operands and group sums ----
#pragma unroll
    for (int k = 0; k < kXr; ++k) {
      float x[8] = {xr[k][0].x, xr[k][0].y, xr[k][0].z, xr[k][0].w, xr[k][1].x, xr[k][1].y, xr[k][1].z, xr[k][1].w};
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= e & 2 ? kIn / 16.0f : kIn;
      auto operand = [&]() {
        return u4v{pack_hi(x[0], x[1]), pack_hi(x[2], x[3]), pack_hi(x[4], x[5]), pack_hi(x[6], x[7])};
      };
      if (NCH <= 2) {
        const int pc = lo & 3;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (pc > 0) x[e] -= top16(x[e]);
          if (pc > 1) x[e] -= top16(x[e]);
          if (pc > 2) x[e] = 0.0f;
        }
        sm.qa[k][w][l] = operand();
      } else {
#pragma unroll
        for (int pc = 0; pc < 3; ++pc) {
          sm.qa[pc][w][l] = operand();
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] -= top16(x[e]);
        }
      }
    }
    float qs[NCH][NG];  // sums of q~ over the groups, head NCH hi + ch, in the products' scale
#pragma unroll
    for (int ch = 0; ch < NCH; ++ch) {
      float s = ((xs[ch][0].x + xs[ch][0].y) + (xs[ch][0].z + xs[ch][0].w)) +
                ((xs[ch][1].x + xs[ch][1].y) + (xs[ch][1].z + xs[ch][1].w));
#pragma unroll
      for (int k = 1; k < 16 / NG; k <<= 1) s += __shfl_xor(s, k, 64);
#pragma unroll
      for (int q = 0; q < NG; ++q) qs[ch][q] = __shfl(s, (l & 48) + q * (16 / NG), 64) * (1.0f / kOut);
    }
    __syncthreads();

    // State: o (before the zero points' part: channel 16 ct + lo of head NCH hi + ch), and
    // per lane, over its own slots, the sums of weights and of weights times (z - 8).
    float m[NCH], lsum[NCH], wz[NCH][NG], o[NCH][8];
#pragma unroll
    for (int ch = 0; ch < NCH; ++ch) {
      m[ch] = -INFINITY;
      lsum[ch] = 0.0f;
#pragma unroll
      for (int q = 0; q < NG; ++q) wz[ch][q] = 0.0f;
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) o[ch][ct] = 0.0f;
    }
    for (int i = 0; i < n_mine; ++i) {
      const int pg = p0 + w + kWaves * i, ntok = min(kP, len - pg * kP);
      if (((i + 1) & 63) == 0 && i + 1 < n_mine) ids = page_ids(i + 1);
      u4v vr[4], vs[NG];
      {
        const u4v* p = reinterpret_cast<const u4v*>(blk + kKv4CodeBytes) + l;
        const u4v* z = reinterpret_cast<const u4v*>(blk + kv4_sz_off(NG, 1)) + lo * NG;
#pragma unroll
        for (int j = 0; j < 4; ++j) vr[j] = __builtin_nontemporal_load(p + 64 * j);
#pragma unroll
        for (int u = 0; u < NG; ++u) vs[u] = z[u];
      }
      __builtin_amdgcn_sched_barrier(0);
      // ---- scores of heads NCH hi + ch, slots 4 lo + u ----
      float sc[NCH][4];
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch)
#pragma unroll
        for (int u = 0; u < 4; ++u) sc[ch][u] = 0.0f;
      auto add = [&](int q, int u, int ch, float x) {  // x: products of group q
        const uint32_t e = ks[(u * NG + q) >> 2][(u * NG + q) & 3];
        sc[ch][u] = fmaf(meta_s<BF>(e), fmaf(meta_z<BF>(e), -qs[ch][q], x), sc[ch][u]);
      };
      if (NCH <= 2) {  // a slot's sums are used while the next slot's products run
        u4v qa[2][NCH];  // query operands one 32-channel block ahead
        f4v d[4][NCH];
#pragma unroll
        for (int ch = 0; ch < NCH; ++ch) qa[0][ch] = sm.qa[ch][0][l];
#pragma unroll
        for (int i = 0; i <= 16; ++i) {
          const int kc = i / 4, u = i % 4;
          if (i < 16) {
            const u4v bop = unpack(kr[u][kc]);
#pragma unroll
            for (int ch = 0; ch < NCH; ++ch)
              d[u][ch] = mfma(qa[kc & 1][ch], bop, kc % KPG == 0 ? f4v{0.0f, 0.0f, 0.0f, 0.0f} : d[u][ch]);
            if (u == 0 && kc < 3)
#pragma unroll
              for (int ch = 0; ch < NCH; ++ch) qa[(kc + 1) & 1][ch] = sm.qa[ch][kc + 1][l];
          }
          if (i > 0 && (i - 1) / 4 % KPG == KPG - 1)
#pragma unroll
            for (int ch = 0; ch < NCH; ++ch) {
              const f4v& x = d[(i - 1) % 4][ch];
              add((i - 1) / 4 / KPG, (i - 1) % 4, ch, (x[0] + x[1]) + x[2]);
            }
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {  // a block's sums while the next block's products run, small pieces first
        f4v d[2][4];
#pragma unroll
        for (int kc = 0; kc <= 4; ++kc) {
          if (kc < 4) {
            u4v qa[kPieces], bop[4];
#pragma unroll
            for (int pc = kPieces - 1; pc >= 0; --pc) qa[pc] = sm.qa[pc][kc][l];
#pragma unroll
            for (int u = 0; u < 4; ++u) bop[u] = unpack(kr[u][kc]);
#pragma unroll
            for (int pc = kPieces - 1; pc >= 0; --pc)
#pragma unroll
              for (int u = 0; u < 4; ++u)
                d[kc & 1][u] = mfma(qa[pc], bop[u],
                                    pc < kPieces - 1 ? d[kc & 1][u]
                                    : kc % KPG == 0  ? f4v{0.0f, 0.0f, 0.0f, 0.0f}
                                                     : d[(kc - 1) & 1][u]);
          }
          if (kc > 0 && (kc - 1) % KPG == KPG - 1)
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
              for (int ch = 0; ch < NCH; ++ch) add((kc - 1) / KPG, u, ch, d[(kc - 1) & 1][u][ch]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch)
#pragma unroll
        for (int u = 0; u < 4; ++u) sc[ch][u] *= kOut;
      __builtin_amdgcn_sched_barrier(0);
      // The next page's K, while this page's V is used (after the last page its own again:
      // with a branch around the loads the compiler moves the sums above behind it, and
      // keeps the products of all slots in registers).
      blk = block_of(min(i + 1, n_mine - 1));
      load_k(blk);
      if (ntok < kP) {  // the partial last page: other slots hold anything
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (4 * lo + u >= ntok) {
#pragma unroll
            for (int ch = 0; ch < NCH; ++ch) sc[ch][u] = -INFINITY;
#pragma unroll
            for (int q = 0; q < NG; ++q) vs[(u * NG + q) >> 2][(u * NG + q) & 3] = 0u;
          }
      }
      if (scores) {
#pragma unroll
        for (int ch = 0; ch < NCH; ++ch)
          if (NCH * hi + ch < g)
            *reinterpret_cast<float4*>(
                scores + (((size_t)b * Hq + kvh * g + NCH * hi + ch) * max_pages + pg) * kP + 4 * lo) =
                make_float4(sc[ch][0], sc[ch][1], sc[ch][2], sc[ch][3]);
      }
      // ---- softmax weights; the reference maximum moves only when a score exceeds it
      // by more than kSlack ----
      bool need = false;
      float mx[NCH];
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch) {
        mx[ch] = fmaxf(fmaxf(sc[ch][0], sc[ch][1]), fmaxf(sc[ch][2], sc[ch][3]));
        need = need || mx[ch] > m[ch] + kSlack;
      }
      if (__any(need)) {
#pragma unroll
        for (int ch = 0; ch < NCH; ++ch) {
          const float mn = fmaxf(m[ch], row_max(mx[ch]));
          const float alpha = __builtin_amdgcn_exp2f(m[ch] - mn);  // m = -inf on the first page -> 0
          m[ch] = mn;
          lsum[ch] *= alpha;
#pragma unroll
          for (int q = 0; q < NG; ++q) wz[ch][q] *= alpha;
#pragma unroll
          for (int ct = 0; ct < 8; ++ct) o[ch][ct] *= alpha;
        }
      }
      float p[NCH][4];
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch) {
#pragma unroll
        for (int u = 0; u < 4; ++u) p[ch][u] = __builtin_amdgcn_exp2f(sc[ch][u] - m[ch]);
        // (one rounding of the running sum per page: beside a heavy token's 1 the roundings
        // of many equal small weights add up)
        lsum[ch] += (p[ch][0] + p[ch][1]) + (p[ch][2] + p[ch][3]);
      }
      // ---- o~ += w V, group by group: the weights' pieces to LDS as the operand's rows ----
      float back[NG];
      auto stage = [&](int q) {
        // scales 2^-ex s, below 2^kTop, and 2 (z - 8)  (single fused operations on the
        // stored halves; the scales are not negative, so that their bits order them)
        float s[4], z[4];
        uint32_t e[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) e[u] = vs[(u * NG + q) >> 2][(u * NG + q) & 3];
        const uint32_t big = row_max_u(pk_max(pk_max(e[0], e[1]), pk_max(e[2], e[3])) & 0xffffu);
        int ex = __builtin_amdgcn_frexp_expf(meta_s<BF>(big)) - kTop;
        if (BF) ex = max(ex, -120);  // 2^-ex is finite for every scale
        const float scale = __builtin_ldexpf(1.0f, -ex);
        back[q] = __builtin_ldexpf(1.0f, ex);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          s[u] = fmaf(meta_s<BF>(e[u]), scale, 0.0f);
          z[u] = fmaf(meta_z<BF>(e[u]), 2.0f, -16.0f);
        }
#pragma unroll
        for (int ch = 0; ch < NCH; ++ch) {
          float x[4], wsum = 0.0f;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            x[u] = p[ch][u] * s[u];
            wsum = fmaf(x[u], z[u], wsum);
          }
          wz[ch][q] = fmaf(wsum, 0.5f * back[q], wz[ch][q]);
          const h2 h0 = half2_of(x[0], x[1]), h1 = half2_of(x[2], x[3]);
          const h2 r0 = half2_of(fmaf((float)h0[0], -1.0f, x[0]), fmaf((float)h0[1], -1.0f, x[1]));
          const h2 r1 = half2_of(fmaf((float)h1[0], -1.0f, x[2]), fmaf((float)h1[1], -1.0f, x[3]));
          uint32_t* row = sm.pw[w] + 2 * lo + (NCH == 1 ? ((q & 1) * 8 + 2 * hi) * kPw : (4 * hi + ch) * kPwWide);
          *reinterpret_cast<uint2*>(row) =
              make_uint2(__builtin_bit_cast(uint32_t, h0), __builtin_bit_cast(uint32_t, h1));
          *reinterpret_cast<uint2*>(row + (NCH == 1 ? kPw : 16 * kPwWide)) =
              make_uint2(__builtin_bit_cast(uint32_t, r0), __builtin_bit_cast(uint32_t, r1));
        }
      };
      if (NCH == 1) stage(0);
#pragma unroll
      for (int q = 0; q < NG; ++q) {
        if (NCH > 1) {  // (a group ahead the wide instances would spill)
          __builtin_amdgcn_sched_barrier(0);
          lane_exchange();  // the last group's reads come before this one's weights
          stage(q);
        }
        lane_exchange();
        u4v a[2][2];  // (wider: piece,) half of the slots; NCH 1: rows 4 h + 2, 4 h + 3 repeat 4 h, 4 h + 1
#pragma unroll
        for (int pc = 0; pc < (NCH == 1 ? 1 : 2); ++pc)
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
            a[pc][kt] = *reinterpret_cast<const u4v*>(
                sm.pw[w] + 16 * kt + 4 * hi +
                (NCH == 1 ? ((q & 1) * 8 + (lo >> 2) * 2 + (lo & 1)) * kPw : (16 * pc + lo) * kPwWide));
        __builtin_amdgcn_sched_barrier(0);
        if (NCH == 1 && q + 1 < NG) stage(q + 1);  // into the other half of the buffer, while the reads are under way
#pragma unroll
        for (int k = 0; k < KPG; ++k) {
          const int j = q * KPG + k;
          __builtin_amdgcn_sched_barrier(0);
          f4v d[2] = {f4v{0.0f, 0.0f, 0.0f, 0.0f}, f4v{0.0f, 0.0f, 0.0f, 0.0f}};
          u4v b[2][2];  // channels 32 j + lo and 32 j + 16 + lo
#pragma unroll
          for (int kt = 0; kt < 2; ++kt) unpack_v(vr[j][2 * kt], vr[j][2 * kt + 1], b[kt][0], b[kt][1]);
#pragma unroll
          for (int pc = (NCH == 1 ? 0 : 1); pc >= 0; --pc)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
              for (int n = 0; n < 2; ++n) d[n] = mfma_h(a[pc][kt], b[kt][n], d[n]);
#pragma unroll
          for (int ch = 0; ch < NCH; ++ch)
#pragma unroll
            for (int n = 0; n < 2; ++n)
              o[ch][2 * j + n] = fmaf(NCH == 1 ? d[n][0] + d[n][1] : d[n][ch], 0x1p9f * back[q], o[ch][2 * j + n]);
        }
      }
      lane_exchange();  // the reads come before the next page's weights
    }

    // ---- the waves' states, merged into the piece's ----
    lane_exchange();
#pragma unroll
    for (int ch = 0; ch < NCH; ++ch) {
      const float lt = row_sum(lsum[ch]);
      float z[NG];
#pragma unroll
      for (int q = 0; q < NG; ++q) z[q] = row_sum(wz[ch][q]);
      float* om = reinterpret_cast<float*>(sm.pw[w]) + (NCH * hi + ch) * kD;
#pragma unroll
      for (int ct = 0; ct < 8; ++ct)
        om[16 * ct + lo] = o[ch][ct] - z[ct / 2 / KPG];
      if (lo == 0) {
        sm.ml[w][NCH * hi + ch][0] = m[ch];
        sm.ml[w][NCH * hi + ch][1] = lt;
      }
    }
    __syncthreads();
    for (int i = t; i < g * kD; i += kWaves * 64) {
      const int head = i / kD, c = i % kD;
      float M = -INFINITY;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) M = fmaxf(M, sm.ml[k][head][0]);
      float v = 0.0f, L = 0.0f;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) {
        const float e = __builtin_amdgcn_exp2f(sm.ml[k][head][0] - M);  // a wave without pages: 0
        v = fmaf(e, reinterpret_cast<const float*>(sm.pw[k])[head * kD + c], v);
        L = fmaf(e, sm.ml[k][head][1], L);
      }
      const size_t slot = ((size_t)b * Hq + kvh * g + head) * num_splits + piece;
      part_o[slot * kD + c] = v;
      if (c == 0) {
        // A query that is not finite has NaN for every score, which leaves no maximum: its
        // piece must not pass for an empty one (M = -inf), so that the NaN reaches the output.
        part_ml[2 * slot] = L == L ? M : 0.0f;
        part_ml[2 * slot + 1] = L;
      }
    }
    if (last)  // the row's other slots are empty
      for (int i = t; i < g * (num_splits - 1 - piece); i += kWaves * 64) {
        const int n = num_splits - 1 - piece;
        const size_t slot = ((size_t)b * Hq + kvh * g + i / n) * num_splits + piece + 1 + i % n;
        part_ml[2 * slot] = -INFINITY;
        part_ml[2 * slot + 1] = 0.0f;
      }
    __syncthreads();
  };

  // One piece at a time: of the block's range of pages, or (num_splits 1) whole sequences.
  const bool whole = num_splits == 1;
  RangeStart s;
  if (whole) {
    s.b = r;
    s.npg = r < B ? pages_of(r) : 0;
    s.x = s.before = 0;
    s.xe = s.pw = (int64_t)1 << 40;
  } else {
    s = range_start<true>(r, n_ranges, B, max_pages, num_splits, pages_of);
  }
  if (kvh == 0 && w == 0) mark_empty(r, n_ranges, B, Hq, num_splits, num_splits, part_ml, pages_of);
  if (!whole && s.npg == 0) return;
  int b = s.b, npg_b = s.npg;
  int64_t x = s.x, before = s.before;
  while (b < B) {
    const int64_t end = min(s.xe, before + npg_b);
    if (end > x)
      run_piece(b, (int)(x - before), (int)(end - before), whole ? 0 : (int)(r - div64<true>(before, s.pw)),
                end == before + npg_b);
    x = end;
    if (x >= s.xe) break;
    before += npg_b;
    b += whole ? n_ranges : 1;  // the next sequence; those without pages are passed over
    npg_b = b < B ? pages_of(b) : 0;
  }
}

// Merge and weights in one launch: the reduce kernel's blocks, then those of the weights,
// which need no more than the pieces' (m, l) either.  In a launch of their own the weights
// took 4 us of a small call (2 sequences of 31001 tokens, 32/8 heads: 35.0 us, 31 now).
//
//   weights_out[b][kvh][t] = weights[b][kvh][t] + sum over the g query heads of
//                            2^(score - M) / L,  M and L from the partial states of the pieces
// Four tokens per thread, kWeightTokens per block.  Bound: HBM reads, 4 (g + 1) bytes per
// token and KV head, and the writes.
constexpr int kWeightTokens = 4 * kRedThreads;

struct WeightArgs {
  int Hkv, Hq, max_pages, chunks;  // blocks per (sequence, KV head)
  const int32_t* seq_lens;
  int num_splits;
  const float* part_ml;
  const float* scores;
  const float* weights;
  float* weights_out;  // may be weights itself
};

__device__ inline void weights_body(int bx, const WeightArgs& a) {
  __shared__ float ms[kMaxGroupHeads], il[kMaxGroupHeads];
  const int chunk = bx % a.chunks, kvh = bx / a.chunks % a.Hkv, b = bx / a.chunks / a.Hkv, g = a.Hq / a.Hkv;
  const int t = threadIdx.x, w = t >> 6, l = t & 63;
  const int len = min(max(a.seq_lens[b], 0), a.max_pages * kP);
  if ((int64_t)chunk * kWeightTokens >= len) return;
  const size_t row0 = (size_t)b * a.Hq + kvh * g;
  for (int h = w; h < g; h += kRedThreads / 64) {
    const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + (row0 + h) * a.num_splits;
    float M = -INFINITY;
    for (int s = l; s < a.num_splits; s += 64) M = fmaxf(M, ml[s].x);
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) M = fmaxf(M, __shfl_xor(M, k, 64));
    float L = 0.0f;
    for (int s = l; s < a.num_splits; s += 64)
      if (ml[s].x != -INFINITY) L = fmaf(exp2f(ml[s].x - M), ml[s].y, L);
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) L += __shfl_xor(L, k, 64);
    if (l == 0) {
      ms[h] = M;
      il[h] = 1.0f / L;
    }
  }
  __syncthreads();
  const int t0 = chunk * kWeightTokens + 4 * t;
  if (t0 >= len) return;
  const size_t S = (size_t)a.max_pages * kP, at = ((size_t)b * a.Hkv + kvh) * S + t0;
  const float4 w_in = *reinterpret_cast<const float4*>(a.weights + at);
  float4 p = make_float4(0.0f, 0.0f, 0.0f, 0.0f);  // the step's part, added to the sum with one rounding
  for (int h = 0; h < g; ++h) {
    const float4 x = *reinterpret_cast<const float4*>(a.scores + (row0 + h) * S + t0);
    p.x = fmaf(__builtin_amdgcn_exp2f(x.x - ms[h]), il[h], p.x);
    p.y = fmaf(__builtin_amdgcn_exp2f(x.y - ms[h]), il[h], p.y);
    p.z = fmaf(__builtin_amdgcn_exp2f(x.z - ms[h]), il[h], p.z);
    p.w = fmaf(__builtin_amdgcn_exp2f(x.w - ms[h]), il[h], p.w);
  }
  p = make_float4(w_in.x + p.x, w_in.y + p.y, w_in.z + p.z, w_in.w + p.w);
  float* out = a.weights_out + at;
  if (t0 + 4 <= len) {
    *reinterpret_cast<float4*>(out) = p;
  } else {  // slots past the length stay as they were
    const float v[4] = {p.x, p.y, p.z, p.w};
    for (int i = 0; t0 + i < len; ++i) out[i] = v[i];
  }
}

template <int RB>
__global__ __launch_bounds__(kRedThreads) void kv4_finish_kernel(int reduce_blocks, int rows,
                                                                 const float* __restrict__ part_o,
                                                                 const float* __restrict__ Rv,
                                                                 void* __restrict__ out, int out_f32, int rph,
                                                                 WeightArgs a) {
  const int bx = blockIdx.x;
  if (bx >= reduce_blocks) {
    weights_body(bx - reduce_blocks, a);
    return;
  }
  reduce_body<false, RB>(bx, rows, a.num_splits, part_o, a.part_ml, Rv, out, out_f32, rph, a.Hq, a.Hkv);
}

template <bool BF, int NG>
void launch_nch(int nch, const dim3& grid, hipStream_t st, const uint8_t* pages, int Hkv, int Hq,
                const int32_t* block_table, int max_pages, const int32_t* seq_lens, int num_splits,
                int ranges, int B, const float* qt, float* part_o, float* part_ml, float* scores) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kWaves * 64), 0, st, pages, Hkv, Hq, block_table, max_pages,
                       seq_lens, num_splits, ranges, B, qt, part_o, part_ml, scores);
  };
  if (nch == 1) go(kv4_split_kernel<BF, NG, 1>);
  else if (nch == 2) go(kv4_split_kernel<BF, NG, 2>);
  else if (nch == 3) go(kv4_split_kernel<BF, NG, 3>);
  else go(kv4_split_kernel<BF, NG, 4>);
}

}  // namespace

hipError_t launch_kv4_split(const uint8_t* pages, int Hkv, int B, int Hq, const int32_t* block_table,
                            int max_pages, const int32_t* seq_lens, int num_splits, const float* qt,
                            float* part_o, float* part_ml, float* scores, hipStream_t st,
                            int meta_bf16, int ng) {
  const int nch = split_chunks(Hq / Hkv);
  // As many ranges as blocks are resident at once (of the Hkv heads' each), and no more
  // than the block table can fill at the least pages of a range.
  const int64_t resident = (int64_t)kPerSimd * device_cus();
  int64_t ranges = std::max<int64_t>(1, resident / Hkv);
  if (num_splits > 1) {
    const int64_t least = std::max<int64_t>(kMinRange, (max_pages + (int64_t)num_splits - 2) / (num_splits - 1));
    ranges = std::min(ranges, ((int64_t)B * max_pages + least - 1) / least);
  } else {
    ranges = std::min<int64_t>(ranges, B);
  }
  const dim3 grid((unsigned)(ranges * Hkv));
  auto by_ng = [&](auto bf) {
    constexpr bool BF = decltype(bf)::value;
    auto go = [&](auto n) {
      launch_nch<BF, decltype(n)::value>(nch, grid, st, pages, Hkv, Hq, block_table, max_pages, seq_lens,
                                         num_splits, (int)ranges, B, qt, part_o, part_ml, scores);
    };
    if (ng == 4) go(std::integral_constant<int, 4>{});
    else if (ng == 2) go(std::integral_constant<int, 2>{});
    else go(std::integral_constant<int, 1>{});
  };
  if (meta_bf16) by_ng(std::true_type{});
  else by_ng(std::false_type{});
  return hipGetLastError();
}

hipError_t launch_kv4_finish(int Hkv, int B, int Hq, int max_pages, const int32_t* seq_lens,
                             int num_splits, const float* part_o, const float* part_ml, const float* Rv,
                             void* out, int out_f32, int rph, const float* scores, const float* weights,
                             float* weights_out, hipStream_t st) {
  const size_t S = (size_t)max_pages * kP;
  const int chunks = (int)((S + kWeightTokens - 1) / kWeightTokens);
  // a launch holds fewer than 2^32 threads: at most 2^20 blocks of the merge and 2^22 of the weights
  const int most = (int)std::min<int64_t>(launch_seqs(Hq),
                                          std::max<int64_t>(1, (1 << 22) / ((int64_t)chunks * Hkv)));
  return by_seqs(B, most, [&](int b0, int nb) {
    const size_t row = (size_t)b0 * Hq, part = row * num_splits, kv = (size_t)b0 * Hkv;
    const WeightArgs a{Hkv, Hq, max_pages, chunks, seq_lens + b0, num_splits, part_ml + part * 2,
                       scores + row * S, weights + kv * S, weights_out + kv * S};
    const int rows = nb * Hq, rb = reduce_rows(rows), rblocks = query_blocks(nb, Hq, Hkv, rph, rb);
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)(rblocks + (int64_t)nb * Hkv * chunks)), dim3(kRedThreads), 0, st,
                         rblocks, rows, part_o + part * kD, Rv,
                         static_cast<void*>(static_cast<char*>(out) + row * kD * (out_f32 ? 4 : 2)), out_f32,
                         rph, a);
    };
    if (rb == 16) go(kv4_finish_kernel<16>);
    else if (rb == 8) go(kv4_finish_kernel<8>);
    else if (rb == 4) go(kv4_finish_kernel<4>);
    else go(kv4_finish_kernel<2>);
    return hipGetLastError();
  });
}

}  // namespace oscar
