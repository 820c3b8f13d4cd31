// Rows of the 4-bit cache read back as values, and eviction from it.
#include <hip/hip_fp16.h>

#include <algorithm>

#include "internal.h"

namespace oscar {
namespace {

__device__ inline uint16_t bf16_rne(float f) {  // finite values
  const uint32_t u = __float_as_uint(f);
  return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

// ---------------------------------------------------------------------------
// gather: value s (n - z) of every channel of the rows at `slots`, in fp32 steps (the
// bf16 output rounds the product once).  32 threads per (token, head, tensor), 4
// channels each.  Bound: HBM writes.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void kv4_gather_kernel(const uint8_t* __restrict__ pages, int Hkv,
                                                         const int64_t* __restrict__ slots, int64_t n_rows,
                                                         void* __restrict__ k, void* __restrict__ v,
                                                         int out_f32, int meta_bf16, int ng) {
  const int c = threadIdx.x & 31, is_v = (threadIdx.x >> 5) & 1;
  for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < n_rows; row += (int64_t)gridDim.x * 4) {
    const int64_t tok = row / Hkv;
    const int h = (int)(row - tok * Hkv);
    const int64_t slot = slots[tok];
    if (slot < 0) continue;
    const int64_t page = slot / kP;
    const int t = (int)(slot - page * kP);
    const uint8_t* blk = pages + ((size_t)page * Hkv + h) * kv4_block_bytes(ng);
    const uint32_t e = *reinterpret_cast<const uint32_t*>(blk + kv4_sz_off(ng, is_v) + (t * ng + c * ng / 32) * 4);
    const float s = meta_bf16 ? __uint_as_float(e << 16) : __half2float(__ushort_as_half((unsigned short)e));
    const float z = meta_bf16 ? __uint_as_float(e & 0xffff0000u)
                              : __half2float(__ushort_as_half((unsigned short)(e >> 16)));
    float x[4];
    if (is_v) {
      const uint8_t* b = blk + kv4_v_off(4 * c - 16 * (c >> 2 & 1), t);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = s * ((float)((b[16 * i] >> (c & 4)) & 15) - z);
    } else {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(blk + kv4_k_off(4 * c, t)) >> (8 * (c & 1));
      x[0] = s * ((float)(w & 15) - z);
      x[1] = s * ((float)((w >> 16) & 15) - z);
      x[2] = s * ((float)((w >> 4) & 15) - z);
      x[3] = s * ((float)((w >> 20) & 15) - z);
    }
    void* out = is_v ? v : k;
    if (out_f32)
      reinterpret_cast<float4*>(out)[row * 32 + c] = make_float4(x[0], x[1], x[2], x[3]);
    else
      reinterpret_cast<uint2*>(out)[row * 32 + c] =
          make_uint2(bf16_rne(x[0]) | ((uint32_t)bf16_rne(x[1]) << 16),
                     bf16_rne(x[2]) | ((uint32_t)bf16_rne(x[3]) << 16));
  }
}

// ---------------------------------------------------------------------------
// Eviction.  A (sequence, KV head) row keeps its m = min(len, budget) slots of largest
// rank: protected tokens first, then by weight, equal ranks from the lowest slot on.
// Kept slots below m stay; the i-th kept slot at or past m moves to the i-th free slot
// below m, so that only rows that must move do, sources and destinations are disjoint,
// and the moves can run in any order, in place.
//
//   select: one block per row.  The m-th largest rank by radix selection on ordered
//           32-bit keys (4 histograms of 8 bits), then one pass in slot order that marks
//           what is kept, with block-wide counts for ties, holes and movers.
//   move:   the moved rows' bytes (codes, scales, zeros) from page to page.
// ---------------------------------------------------------------------------
constexpr int kSel = 1024;  // threads of a select block

// Larger key, larger rank: finite weights in order (-0 as 0), NaN below all, protected
// tokens above all.
__device__ inline uint32_t rank_key(float w, bool safe) {
  if (safe) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w == 0.0f ? 0.0f : w);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// Exclusive prefix sum over the block's threads in order, and the total.
__device__ inline int block_scan(int v, int* part, int& total) {
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const int y = __shfl_up(x, k, 64);
    if (l >= k) x += y;
  }
  __syncthreads();  // earlier reads of part
  if (l == 63) part[w] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int k = 0; k < kSel / 64; ++k) {
    before += k < w ? part[k] : 0;
    total += part[k];
  }
  return before + x - v;
}

__global__ __launch_bounds__(kSel) void kv4_evict_select_kernel(
    int Hkv, int64_t S, int max_pages, const int32_t* __restrict__ seq_lens, const float* weights,
    float* weights_out, const int32_t* pos, int32_t* pos_out, const int32_t* __restrict__ seen_all,
    int budget, int sink, int recent, int32_t* __restrict__ new_lens, int32_t* __restrict__ counts,
    int2* __restrict__ moves, int64_t row0) {
  __shared__ int hist[256];
  __shared__ int part[kSel / 64];
  __shared__ uint32_t found;
  __shared__ int left;
  const int64_t row = row0 + blockIdx.x;
  const int b = (int)(row / Hkv), h = (int)(row - (int64_t)b * Hkv), t = threadIdx.x;
  const int n = min(max(seq_lens[b], 0), max_pages * kP), m = min(n, budget), seen = seen_all[b];
  const float* w_in = weights + row * S;
  const int32_t* p_in = pos + row * S;
  float* w_out = weights_out + row * S;
  int32_t* p_out = pos_out + row * S;
  if (h == 0 && t == 0) new_lens[b] = m;
  auto pos_of = [&](int i) {
    const int p = p_in[i];
    return p >= 0 ? p : seen - (n - i);
  };
  auto key_of = [&](int i) {
    const int p = pos_of(i);
    return rank_key(w_in[i], p < sink || p >= seen - recent);
  };
  int n_moves = 0;
  if (n <= budget) {
    for (int i = t; i < n; i += kSel) {
      w_out[i] = w_in[i];
      p_out[i] = pos_of(i);
    }
  } else {
    uint32_t prefix = 0;
    int need = m;  // slots still to be kept among the keys that share the prefix
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (t < 256) hist[t] = 0;
      __syncthreads();
      for (int i = t; i < n; i += kSel) {
        const uint32_t k = key_of(i);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);
      }
      __syncthreads();
      if (t < 64) {  // digits 4 t .. 4 t + 3, counted from the top
        int c[4], sum = 0;
#pragma unroll
        for (int i = 3; i >= 0; --i) sum += c[i] = hist[4 * t + i];
        int above = sum;  // inclusive sum over the lanes from t up
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) {
          const int y = __shfl_down(above, k, 64);
          if (t + k < 64) above += y;
        }
        above -= sum;
#pragma unroll
        for (int i = 3; i >= 0; --i) {
          if (above < need && above + c[i] >= need) {
            found = (uint32_t)(4 * t + i);
            left = need - above;
          }
          above += c[i];
        }
      }
      __syncthreads();
      prefix |= found << shift;
      need = left;
      __syncthreads();
    }
    // kept: keys above the prefix, and the first `need` slots of equal key
    int2* mv = moves + row * (S / 2);
    int n_equal = 0, holes = 0, movers = 0;
    for (int base = 0; base < n; base += kSel) {
      const int i = base + t;
      uint32_t k = 0;
      bool equal = false;
      if (i < n) {
        k = key_of(i);
        equal = k == prefix;
      }
      int total;
      const int before = n_equal + block_scan(equal, part, total);
      n_equal += total;
      const bool kept = i < n && (k > prefix || (equal && before < need));
      const bool hole = i < m && !kept, mover = kept && i >= m;
      const int at = block_scan(hole ? 1 : mover ? 1 << 16 : 0, part, total);
      if (hole) mv[holes + (at & 0xffff)].y = i;
      if (mover) mv[movers + (at >> 16)].x = i;
      holes += total & 0xffff;
      movers += total >> 16;
      if (kept && !mover) {
        w_out[i] = w_in[i];
        p_out[i] = pos_of(i);
      }
    }
    n_moves = movers;
    __syncthreads();
    for (int i = t; i < n_moves; i += kSel) {
      const int2 x = mv[i];
      w_out[x.y] = w_in[x.x];
      p_out[x.y] = pos_of(x.x);
    }
    __syncthreads();
  }
  for (int64_t i = m + t; i < S; i += kSel) {
    w_out[i] = 0.0f;
    p_out[i] = -1;
  }
  if (t == 0) counts[row] = n_moves;
}

// One wave per moved row: 16 dwords of K codes, 64 bytes of V codes, 2 ng metadata entries.
__global__ __launch_bounds__(256) void kv4_evict_move_kernel(uint8_t* __restrict__ pages, int Hkv, int64_t S,
                                                             int ng, const int32_t* __restrict__ block_table,
                                                             int max_pages, const int32_t* __restrict__ counts,
                                                             const int2* __restrict__ moves, int64_t row0) {
  const int64_t row = row0 + blockIdx.y;
  const int b = (int)(row / Hkv), h = (int)(row - (int64_t)b * Hkv), l = threadIdx.x & 63;
  const int n = counts[row];
  const int2* mv = moves + row * (S / 2);
  const int32_t* bt = block_table + (size_t)b * max_pages;
  for (int i = blockIdx.x * 4 + (threadIdx.x >> 6); i < n; i += gridDim.x * 4) {
    const int2 x = mv[i];
    const int ts = x.x % kP, td = x.y % kP;
    const uint8_t* from = pages + ((size_t)bt[x.x / kP] * Hkv + h) * kv4_block_bytes(ng);
    uint8_t* to = pages + ((size_t)bt[x.y / kP] * Hkv + h) * kv4_block_bytes(ng);
    const int cv = 32 * (l >> 4) + (l & 15);
    const uint8_t v = from[kv4_v_off(cv, ts)];
    uint32_t d = 0;
    const int sz = l - 16;  // lanes 16 ..: metadata entries of K, then of V
    if (l < 16) d = *reinterpret_cast<const uint32_t*>(from + kv4_k_off(8 * l, ts));
    else if (sz < 2 * ng)
      d = *reinterpret_cast<const uint32_t*>(from + kv4_sz_off(ng, sz >= ng) + (ts * ng + sz % ng) * 4);
    to[kv4_v_off(cv, td)] = v;
    if (l < 16) *reinterpret_cast<uint32_t*>(to + kv4_k_off(8 * l, td)) = d;
    else if (sz < 2 * ng)
      *reinterpret_cast<uint32_t*>(to + kv4_sz_off(ng, sz >= ng) + (td * ng + sz % ng) * 4) = d;
  }
}

}  // namespace

hipError_t launch_kv4_gather(const uint8_t* pages, int Hkv, const int64_t* slots, int64_t n_tok,
                             void* k, void* v, int out_f32, int meta_bf16, int ng, hipStream_t st) {
  const int64_t rows = n_tok * Hkv;
  const unsigned blocks = (unsigned)std::min<int64_t>((rows + 3) / 4, 1 << 20);
  hipLaunchKernelGGL(kv4_gather_kernel, dim3(blocks), dim3(256), 0, st, pages, Hkv, slots, rows, k, v,
                     out_f32, meta_bf16, ng);
  return hipGetLastError();
}

namespace {
struct EvictWs {
  size_t moves_off, total;
};
EvictWs evict_ws(int Hkv, int B, int max_pages) {
  const size_t rows = (size_t)B * Hkv;
  EvictWs w;
  w.moves_off = align256(rows * sizeof(int32_t));
  w.total = align256(w.moves_off + rows * ((size_t)max_pages * kP / 2) * sizeof(int2));
  return w;
}
}  // namespace

size_t kv4_evict_ws_bytes(int Hkv, int B, int max_pages) { return evict_ws(Hkv, B, max_pages).total; }

hipError_t launch_kv4_evict(const EvictArgs& a, hipStream_t st) {
  const int64_t rows = (int64_t)a.B * a.Hkv, S = (int64_t)a.max_pages * kP;
  int32_t* counts = static_cast<int32_t*>(a.ws);
  int2* moves = reinterpret_cast<int2*>(static_cast<uint8_t*>(a.ws) +
                                        evict_ws(a.Hkv, a.B, a.max_pages).moves_off);
  for (int64_t r0 = 0; r0 < rows; r0 += 1 << 20) {  // a launch holds fewer than 2^32 threads
    hipLaunchKernelGGL(kv4_evict_select_kernel, dim3((unsigned)std::min<int64_t>(rows - r0, 1 << 20)),
                       dim3(kSel), 0, st, a.Hkv, S, a.max_pages, a.seq_lens, a.weights, a.weights_out, a.pos,
                       a.pos_out, a.seen, a.budget, a.sink, a.recent, a.new_lens, counts, moves, r0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t most = std::min<int64_t>(a.budget, S / 2);  // moves of a row
  const unsigned gx = (unsigned)std::max<int64_t>(
      1, std::min((most + 3) / 4, (16 * (int64_t)device_cus() + rows - 1) / rows));
  for (int64_t r0 = 0; r0 < rows; r0 += 65535) {
    hipLaunchKernelGGL(kv4_evict_move_kernel, dim3(gx, (unsigned)std::min<int64_t>(rows - r0, 65535)),
                       dim3(256), 0, st, a.pages, a.Hkv, S, a.ng, a.block_table, a.max_pages, counts, moves,
                       r0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace oscar
