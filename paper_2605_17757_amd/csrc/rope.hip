// Queries and keys of new tokens on their way from the projection: RMS norm per head and
// rotation by position, into rows of their own or (keys, with the values) into the bf16
// cache's pages.
//   x^_c = x_c / sqrt(mean_c x_c^2 + eps) w_c             (without weights: x^ = x)
//   pair (a, b) of x^ -> f (a cos t - b sin t, b cos t + a sin t),  t = pos * freq_i
// for the rotary / 2 pairs of the head's first channels, the others as they are.
// All steps in fp32 and one rounding to bf16 at the end, but for the angle: its turns,
// (pos / 2 pi) * freq, and their fraction are fp64 (each rounded to 2^-53 of itself), since an
// fp32 angle of position 10^5 is off by 0.004 already.  The hardware's sine and cosine take turns.
// Rows whose mean square is outside [2^-100, 2^100] are divided by a power of two first (bf16 values
// reach 3e38, the sum of their squares would leave fp32's range).
// Eight lanes hold a (token, head) row, two chunks of 8 channels each, so chosen that a
// lane has both channels of its pairs; the norm's sum is three DPP steps.
// Bound: memory.  8191 tokens of 32 + 8 heads, 168 MB read and written: 35 us, 4.7 TB/s, inputs new to
// the caches (the same again and again, which the last-level cache holds: 30); with pages, 16503 tokens
// of 64 + 8 heads, 676 MB: 146 us, 4.6 TB/s (a copy of 2 GiB: 4.9).
#include "internal.h"

#include <type_traits>

namespace oscar {
namespace {

constexpr int kBlockElems = 2 * kP * kD;  // bf16 elements of a page-head block
constexpr int kUnitHeads = 8;             // rows per wave

typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));

__device__ inline uint32_t bf16x2(float lo, float hi) {  // nearest even
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{lo, hi}), b2));
}
__device__ inline void unpack8(const u4v& w, float* x) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = __uint_as_float(w[j] << 16);
    x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
  }
}
__device__ inline u4v pack8(const float* x) {
  return u4v{bf16x2(x[0], x[1]), bf16x2(x[2], x[3]), bf16x2(x[4], x[5]), bf16x2(x[6], x[7])};
}
// Sum over the 8 lanes of a row (the same bits in each: both sides of every addition swap).
__device__ inline float sum8(float v) {
  auto dpp = [](float x, auto ctrl) {
    return __int_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xF, 0xF, false));
  };
  v += dpp(v, std::integral_constant<int, 0xB1>{});  // lanes ^ 1
  v += dpp(v, std::integral_constant<int, 0x4E>{});  // lanes ^ 2
  v += dpp(v, std::integral_constant<int, 0x141>{}); // lanes 7 - l: the other four
  return v;
}

// Chunks of 8 channels that lane j of a row holds.
__device__ inline void lane_chunks(int j, int rotary, int interleaved, int& c0, int& c1) {
  if (interleaved) {
    c0 = 2 * j;
    c1 = c0 + 1;
  } else {
    const int n = rotary / 16;  // lanes that rotate: chunk j with chunk j + n
    c0 = j < n ? j : 2 * j;
    c1 = j < n ? j + n : 2 * j + 1;
  }
}

// What a lane does with its 16 channels of a row: the angles of its pairs (cos 1, sin 0 where it
// rotates nothing), norm, rotation.
__device__ inline void angles(const RopeRows& a, int j, int64_t position, float (&cs)[8], float (&sn)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    cs[i] = 1.0f;
    sn[i] = 0.0f;
  }
  if (j >= a.rotary / 16) return;
  const double pos = (double)position * 0.15915494309189533577;  // 1 / 2 pi
  const float4* fp = reinterpret_cast<const float4*>(a.freq + 8 * j);
  const float4 f0 = fp[0], f1 = fp[1];
  const float fr[8] = {f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double turns = pos * (double)fr[i];
    const float t = (float)(turns - __builtin_rint(turns));
    cs[i] = __builtin_amdgcn_cosf(t) * a.factor;
    sn[i] = __builtin_amdgcn_sinf(t) * a.factor;
  }
}
// A row divided by a power of two that brings its largest magnitude, or the root of eps, near 1; what
// eps is there.
__device__ inline float rescale(float (&x)[16], float eps) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
  for (int m = 1; m < 8; m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m, 8));
  const int e_eps = eps > 0.0f ? (int)(__float_as_uint(eps) >> 23) - 127 : -400;
  const int e = max((int)(top >> 23) - 127, e_eps >> 1);
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = ldexpf(x[i], -e);
  return ldexpf(eps, -2 * e);
}
__device__ inline void norm_rotate(const RopeRows& a, const uint16_t* weight, int j, int c0, int c1,
                                   const float (&cs)[8], const float (&sn)[8], u4v& w0, u4v& w1) {
  float x[16];
  unpack8(w0, x);
  unpack8(w1, x + 8);
  if (weight) {
    auto mean_square = [&]() {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) s = fmaf(x[i], x[i], s);
      return sum8(s) * (1.0f / kD);
    };
    float mean = mean_square() + a.eps;
    if (!(mean >= 0x1p-100f && mean <= 0x1p100f)) mean = rescale(x, a.eps) + mean_square();
    const float r = 1.0f / sqrtf(mean);
    float g[16];
    unpack8(*reinterpret_cast<const u4v*>(weight + 8 * c0), g);
    unpack8(*reinterpret_cast<const u4v*>(weight + 8 * c1), g + 8);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = x[i] * r * g[i];
  }
  if (j < a.rotary / 16) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float& p = a.interleaved ? x[2 * i] : x[i];
      float& q = a.interleaved ? x[2 * i + 1] : x[8 + i];
      const float y = p * cs[i] - q * sn[i], v = q * cs[i] + p * sn[i];
      p = y;
      q = v;
    }
  }
  w0 = pack8(x);
  w1 = pack8(x + 8);
}

// A wave takes up to `units` units of a token, 8 of its query and (without pages) key heads each,
// with the sines and cosines in registers.
template <bool PAGES>
__device__ inline void rows_units(const RopeRows& a, int64_t item, int units, int per_tok) {
  const int l = threadIdx.x & 63, j = l & 7;
  const int parts = (per_tok + units - 1) / units;
  const int64_t tok = item / parts;
  const int u0 = (int)(item - tok * parts) * units, u1 = min(u0 + units, per_tok);
  const int heads = a.Hq + (PAGES ? 0 : a.Hkv);
  int c0, c1;
  lane_chunks(j, a.rotary, a.interleaved, c0, c1);
  u4v w0{0, 0, 0, 0}, w1{0, 0, 0, 0};
  auto load = [&](int u) {
    const int head = u * kUnitHeads + (l >> 3);
    if (head >= heads) return;
    const uint16_t* src = !PAGES && head >= a.Hq ? a.k + (size_t)tok * a.k_stride + (size_t)(head - a.Hq) * kD
                                                 : a.q + (size_t)tok * a.q_stride + (size_t)head * kD;
    w0 = *reinterpret_cast<const u4v*>(src + 8 * c0);
    w1 = *reinterpret_cast<const u4v*>(src + 8 * c1);
  };
  load(u0);
  float cs[8], sn[8];
  angles(a, j, a.positions[tok], cs, sn);
  for (int u = u0; u < u1; ++u) {
    const int head = u * kUnitHeads + (l >> 3);
    const bool is_k = !PAGES && head >= a.Hq;
    u4v y0 = w0, y1 = w1;
    if (u + 1 < u1) load(u + 1);
    norm_rotate(a, is_k ? a.k_weight : a.q_weight, j, c0, c1, cs, sn, y0, y1);
    if (head >= heads) continue;
    uint16_t* dst = is_k ? a.k_out + ((size_t)tok * a.Hkv + head - a.Hq) * kD
                         : a.q_out + ((size_t)tok * a.Hq + head) * kD;
    *reinterpret_cast<u4v*>(dst + 8 * c0) = y0;
    *reinterpret_cast<u4v*>(dst + 8 * c1) = y1;
  }
}

// Keys of TOK tokens of one KV head into the pages, eight tokens a wave at a time.  A page's 128
// bytes hold 16 of eight slots each (every fourth slot): from one block, and so one L2, they go to
// memory as whole lines (a token's heads in one wave: 16503 tokens of 64 + 8 heads took 154 us, 147 now).
template <int TOK>
__device__ inline void keys_tile(const RopeRows& a, int64_t tile) {
  const int kvh = (int)(tile % a.Hkv);
  const int64_t tok0 = tile / a.Hkv * TOK;
  const int l = threadIdx.x & 63, j = l & 7;
  int c0, c1;
  lane_chunks(j, a.rotary, a.interleaved, c0, c1);
  for (int r = (threadIdx.x >> 6) * 8 + (l >> 3); r < TOK; r += 32) {
    const bool live = tok0 + r < a.n_tok;
    const int64_t tok = live ? tok0 + r : a.n_tok - 1;
    const uint16_t* src = a.k + (size_t)tok * a.k_stride + (size_t)kvh * kD;
    u4v w0 = *reinterpret_cast<const u4v*>(src + 8 * c0), w1 = *reinterpret_cast<const u4v*>(src + 8 * c1);
    float cs[8], sn[8];
    angles(a, j, a.positions[tok], cs, sn);
    norm_rotate(a, a.k_weight, j, c0, c1, cs, sn, w0, w1);
    const int64_t slot = a.slots[tok];
    if (!live || slot < 0) continue;
    const int t = (int)(slot % kP);
    u4v* blk = reinterpret_cast<u4v*>(a.pages + ((size_t)(slot / kP) * a.Hkv + kvh) * kBlockElems);
    // chunk c: channels 32 hi + 8 kc of slot 4 lo + u
    blk[((t & 3) * 4 + (c0 & 3)) * 64 + (t >> 2) + 16 * (c0 >> 2)] = w0;
    blk[((t & 3) * 4 + (c1 & 3)) * 64 + (t >> 2) + 16 * (c1 >> 2)] = w1;
  }
}

// Values of TOK tokens of one KV head into the pages.  A page holds eight slots of a
// channel in 16 bytes: eight tokens of the call in such slots are stored together (through
// LDS), the others two bytes each.
template <int TOK>
__device__ inline void values_tile(const RopeRows& a, int64_t tile, uint8_t* smem) {
  constexpr int kPitch = kD + 2;  // elements: tokens of one channel fall in different banks
  uint16_t* vs = reinterpret_cast<uint16_t*>(smem);
  int64_t* slot = reinterpret_cast<int64_t*>(smem + (size_t)TOK * kPitch * 2);
  int* lead = reinterpret_cast<int*>(slot + TOK);  // per token: its run's first token, -1: alone, -2: skipped
  const int kvh = (int)(tile % a.Hkv);
  const int64_t tok0 = tile / a.Hkv * TOK;
  const int n = (int)(a.n_tok - tok0 < TOK ? a.n_tok - tok0 : TOK);
  const int t = threadIdx.x;
  if (t < TOK) slot[t] = t < n ? a.slots[tok0 + t] : -1;
  for (int i = t; i < n * (kD / 8); i += 256) {
    const int r = i / (kD / 8), c = i % (kD / 8);
    const u4v w = *reinterpret_cast<const u4v*>(a.v + (size_t)(tok0 + r) * a.v_stride + (size_t)kvh * kD + 8 * c);
    uint32_t* d = reinterpret_cast<uint32_t*>(vs + r * kPitch + 8 * c);
    d[0] = w.x; d[1] = w.y; d[2] = w.z; d[3] = w.w;
  }
  __syncthreads();
  if (t < TOK) {
    const int64_t s = slot[t];
    int v = -2;
    if (s >= 0) {
      const int f = t - (int)(s & 7);
      bool run = f >= 0 && f + 8 <= TOK;
      if (run)
#pragma unroll
        for (int i = 0; i < 8; ++i) run = run && slot[f + i] == s - (s & 7) + i;
      v = run ? f : -1;
    }
    lead[t] = v;
  }
  __syncthreads();
  // element of channel c, slot s: ((ct 2 + kt) 64 + lo + 16 hi) 8 + e
  auto at = [&](int64_t s, int c) {
    const int ts = (int)(s % kP);
    return ((size_t)(s / kP) * a.Hkv + kvh) * kBlockElems + kP * kD +
           (size_t)(((c >> 4) * 2 + ((ts >> 3) & 1)) * 64 + (c & 15) + 16 * (ts >> 4)) * 8 + (ts & 7);
  };
  for (int i = t; i < TOK * kD; i += 256) {
    const int r = i / kD, c = i % kD, ld = lead[r];
    if (ld == r) {
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[k] = vs[(r + 2 * k) * kPitch + c] | (uint32_t)vs[(r + 2 * k + 1) * kPitch + c] << 16;
      *reinterpret_cast<u4v*>(a.pages + at(slot[r], c)) = u4v{w[0], w[1], w[2], w[3]};
    } else if (ld == -1) {
      a.pages[at(slot[r], c)] = vs[r * kPitch + c];
    }
  }
}

template <bool PAGES, int TOK>
__global__ __launch_bounds__(256) void rope_kernel(RopeRows a, int64_t row_blocks, int units, int per_tok) {
  __shared__ __align__(16) uint8_t smem[PAGES ? TOK * (kD + 2) * 2 + TOK * 8 + TOK * 4 : 16];
  if (!PAGES || blockIdx.x < row_blocks) {
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (item < (int64_t)a.n_tok * ((per_tok + units - 1) / units)) rows_units<PAGES>(a, item, units, per_tok);
    return;
  }
  if (PAGES) {
    keys_tile<TOK>(a, (int64_t)blockIdx.x - row_blocks);
    values_tile<TOK>(a, (int64_t)blockIdx.x - row_blocks, smem);
  }
}

template <bool PAGES, int TOK>
hipError_t launch(const RopeRows& a, hipStream_t st) {
  // a launch holds fewer than 2^32 threads: the tokens in parts where they need more
  const int per_tok = (a.Hq + (PAGES ? 0 : a.Hkv) + kUnitHeads - 1) / kUnitHeads;
  const int64_t per = (int64_t)per_tok + (PAGES ? a.Hkv : 0);
  int64_t most = ((int64_t)1 << 23) / per / 64 * 64;
  if (most < 64) most = 64;
  for (int64_t t0 = 0; t0 < a.n_tok; t0 += most) {
    RopeRows p = a;
    p.n_tok = (int)(a.n_tok - t0 < most ? a.n_tok - t0 : most);
    if (p.q) p.q += t0 * a.q_stride;
    if (p.q_out) p.q_out += t0 * a.Hq * kD;
    p.k += t0 * a.k_stride;
    if (p.k_out) p.k_out += t0 * a.Hkv * kD;
    if (p.v) p.v += t0 * a.v_stride;
    p.positions += t0;
    if (p.slots) p.slots += t0;
    // Two units a wave where that leaves each SIMD eight waves.  8191 tokens of 32 + 8 heads that the
    // last-level cache holds take 35 us with one, 30 with two, 29 with all five; from memory 35.5, 35.5
    // and 38.7; 16503 of 64 heads into pages 144, 145 and, with eight, 154.
    const int units = (int64_t)p.n_tok * per_tok >= 64 * device_cus() ? 2 : 1;
    const int64_t rows = per_tok ? ((int64_t)p.n_tok * ((per_tok + units - 1) / units) + 3) / 4 : 0;
    const int64_t tiles = PAGES ? (int64_t)((p.n_tok + TOK - 1) / TOK) * a.Hkv : 0;
    hipLaunchKernelGGL((rope_kernel<PAGES, TOK>), dim3((unsigned)(rows + tiles)), dim3(256), 0, st, p, rows,
                       units, per_tok);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_rope(const RopeRows& a, hipStream_t st) {
  if (!a.pages) return launch<false, 8>(a, st);
  const bool few = (int64_t)a.n_tok * a.Hkv < (int64_t)64 * 2 * device_cus();
  return few ? launch<true, 8>(a, st) : launch<true, 64>(a, st);
}

}  // namespace oscar
