// Queries and keys of new tokens on their way from the projection: RMS norm per head and
// rotation by position, into rows of their own or (keys, with the values) into the bf16
// cache's pages.
//   x^_c = x_c / sqrt(mean_c x_c^2 + eps) w_c             (without weights: x^ = x)
//   pair (a, b) of x^ -> f (a cos t - b sin t, b cos t + a sin t),  t = pos * freq_i
// for the rotary / 2 pairs of the head's first channels, the others as they are.
// All steps in fp32 and one rounding to bf16 at the end, but for the angle: pos * freq is
// the exact fp64 product of an integer and an fp32 number, brought to turns and reduced to
// its fraction in fp64, since an fp32 angle of position 10^5 is off by 0.004 already.  The
// hardware's sine and cosine take turns.
// Eight lanes hold a (token, head) row, two chunks of 8 channels each, so chosen that a
// lane has both channels of its pairs; the norm's sum is three DPP steps.
#include "internal.h"

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

// One wave's unit: heads [8 u, 8 u + 8) of the Hq + Hkv query and key heads of a token.
template <bool PAGES>
__device__ inline void rows_unit(const RopeRows& a, int64_t unit, int per_tok) {
  const int l = threadIdx.x & 63, j = l & 7;
  const int64_t tok = unit / per_tok;
  const int head = (int)(unit - tok * per_tok) * kUnitHeads + (l >> 3);
  const int heads = a.Hq + a.Hkv;
  const bool is_k = head >= a.Hq, live = head < heads;
  const int kvh = head - a.Hq;
  const uint16_t* src = is_k ? a.k + (size_t)tok * a.k_stride + (size_t)kvh * kD
                             : a.q + (size_t)tok * a.q_stride + (size_t)head * kD;
  int c0, c1;
  lane_chunks(j, a.rotary, a.interleaved, c0, c1);
  u4v w0{0, 0, 0, 0}, w1{0, 0, 0, 0};
  if (live) {
    w0 = *reinterpret_cast<const u4v*>(src + 8 * c0);
    w1 = *reinterpret_cast<const u4v*>(src + 8 * c1);
  }
  float x[16];
  unpack8(w0, x);
  unpack8(w1, x + 8);
  const uint16_t* wt = is_k ? a.k_weight : a.q_weight;
  if (wt) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s = fmaf(x[i], x[i], s);
    const float r = 1.0f / sqrtf(sum8(s) * (1.0f / kD) + a.eps);
    float g[16];
    unpack8(*reinterpret_cast<const u4v*>(wt + 8 * c0), g);
    unpack8(*reinterpret_cast<const u4v*>(wt + 8 * c1), g + 8);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = x[i] * r * g[i];
  }
  if (j < a.rotary / 16) {
    const double pos = (double)a.positions[tok] * 0.15915494309189533577;  // 1 / 2 pi
    float fr[8];  // frequencies of the lane's pairs
    const float4* fp = reinterpret_cast<const float4*>(a.freq + 8 * j);
    const float4 f0 = fp[0], f1 = fp[1];
    fr[0] = f0.x; fr[1] = f0.y; fr[2] = f0.z; fr[3] = f0.w;
    fr[4] = f1.x; fr[5] = f1.y; fr[6] = f1.z; fr[7] = f1.w;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double turns = pos * (double)fr[i];
      const float t = (float)(turns - __builtin_rint(turns));
      const float c = __builtin_amdgcn_cosf(t) * a.factor, s = __builtin_amdgcn_sinf(t) * a.factor;
      float& p = a.interleaved ? x[2 * i] : x[i];
      float& q = a.interleaved ? x[2 * i + 1] : x[8 + i];
      const float u = p * c - q * s, v = q * c + p * s;
      p = u;
      q = v;
    }
  }
  w0 = pack8(x);
  w1 = pack8(x + 8);
  if (!live) return;
  if (PAGES && is_k) {
    const int64_t slot = a.slots[tok];
    if (slot < 0) return;
    const int t = (int)(slot % kP);
    u4v* blk = reinterpret_cast<u4v*>(a.pages + ((size_t)(slot / kP) * a.Hkv + kvh) * kBlockElems);
    // chunk c: channels 32 hi + 8 kc of slot 4 lo + u
    blk[((t & 3) * 4 + (c0 & 3)) * 64 + (t >> 2) + 16 * (c0 >> 2)] = w0;
    blk[((t & 3) * 4 + (c1 & 3)) * 64 + (t >> 2) + 16 * (c1 >> 2)] = w1;
    return;
  }
  uint16_t* dst = is_k ? a.k_out + ((size_t)tok * a.Hkv + kvh) * kD : a.q_out + ((size_t)tok * a.Hq + head) * kD;
  *reinterpret_cast<u4v*>(dst + 8 * c0) = w0;
  *reinterpret_cast<u4v*>(dst + 8 * c1) = w1;
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
__global__ __launch_bounds__(256) void rope_kernel(RopeRows a, int64_t row_blocks, int per_tok) {
  __shared__ __align__(16) uint8_t smem[PAGES ? TOK * (kD + 2) * 2 + TOK * 8 + TOK * 4 : 16];
  if (!PAGES || blockIdx.x < row_blocks) {
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit < (int64_t)a.n_tok * per_tok) rows_unit<PAGES>(a, unit, per_tok);
    return;
  }
  if (PAGES) values_tile<TOK>(a, (int64_t)blockIdx.x - row_blocks, smem);
}

template <bool PAGES, int TOK>
hipError_t launch(const RopeRows& a, hipStream_t st) {
  // a launch holds fewer than 2^32 threads: the tokens in parts where they need more
  const int per_tok = (a.Hq + a.Hkv + kUnitHeads - 1) / kUnitHeads;
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
    const int64_t rows = ((int64_t)p.n_tok * per_tok + 3) / 4;
    const int64_t tiles = PAGES ? (int64_t)((p.n_tok + TOK - 1) / TOK) * a.Hkv : 0;
    hipLaunchKernelGGL((rope_kernel<PAGES, TOK>), dim3((unsigned)(rows + tiles)), dim3(256), 0, st, p, rows,
                       per_tok);
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
