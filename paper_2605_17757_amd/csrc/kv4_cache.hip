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

// Scale and zero of a metadata entry.
__device__ inline float2 meta_of(uint32_t e, int bf16) {
  return bf16 ? make_float2(__uint_as_float(e << 16), __uint_as_float(e & 0xffff0000u))
              : make_float2(__half2float(__ushort_as_half((unsigned short)e)),
                            __half2float(__ushort_as_half((unsigned short)(e >> 16))));
}
// Value of code (x >> sh) & 15.
__device__ inline float value_of(uint32_t x, int sh, float2 m) { return m.x * ((float)((x >> sh) & 15u) - m.y); }

// ---------------------------------------------------------------------------
// gather: value s (n - z) of every channel of the rows at `slots`, in fp32 steps (the
// bf16 output rounds the product once).  Bound: HBM writes (fp32: 1024 bytes per token
// and head against 128 + 8 ng read).
//
// Row by row (half a wave per tensor, 4 channels a lane) a V row is 64 single bytes of 8
// cache lines.  Calls of more than kRowsMost rows take tiles of 64 tokens, one block per
// (tile, head): the tile's slots are grouped by page, and of a page with kPageRows members
// or more the block reads the whole page-head block in its 16-byte units, a quarter per
// wave, and stores the members' rows from registers; rows of other pages go one by one.
// Row by row against tiles, 8 heads: 1000 tokens in order 6.1 us against 6.9, 2048 8.0
// against 7.2, 4200 13.2 against 10.2; of as many pages (a step's new tokens) 97 tokens 6.2
// against 20, 4200 15 against 25, 131072 513 against 646.
// 131072 tokens x 8 heads, fp32 (1.24 GB): 539 us row by row, 224 us (5.5 TB/s) by tiles
// at three waves per SIMD; at eight, whose half-written output lines do not fit the L2,
// 307, at two 245, with non-temporal stores 450.
// ---------------------------------------------------------------------------
struct GatherArgs {
  const uint8_t* pages;
  int Hkv;
  const int64_t* slots;
  int64_t n_tok;
  void* k;
  void* v;
  int meta_bf16, ng;
};

template <bool F32>
__device__ inline void put4(void* out, size_t at, float a, float b, float c, float d) {  // at: element, % 4 == 0
  if (F32) *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(a, b, c, d);
  else
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) =
        make_uint2(bf16_rne(a) | ((uint32_t)bf16_rne(b) << 16), bf16_rne(c) | ((uint32_t)bf16_rne(d) << 16));
}
template <bool F32>
__device__ inline void put1(void* out, size_t at, float x) {
  if (F32) static_cast<float*>(out)[at] = x;
  else static_cast<uint16_t*>(out)[at] = bf16_rne(x);
}

// One row by one wave: lanes 0 .. 31 K, 32 .. 63 V, channels 4 (l % 32) ..
struct RowPart {
  uint32_t codes, meta;  // codes: value i in nibble i of the lane's order
};
__device__ inline RowPart load_row(const GatherArgs& a, int h, int64_t slot, int l) {
  const int c = l & 31, is_v = l >> 5;
  const int64_t page = slot / kP;
  const int t = (int)(slot - page * kP);
  const uint8_t* blk = a.pages + ((size_t)page * a.Hkv + h) * kv4_block_bytes(a.ng);
  RowPart r;
  r.meta = *reinterpret_cast<const uint32_t*>(blk + kv4_sz_off(a.ng, is_v) + (t * a.ng + c * a.ng / 32) * 4);
  if (is_v) {
    const uint8_t* b = blk + kv4_v_off(4 * c - 16 * (c >> 2 & 1), t);
    r.codes = (b[0] | (uint32_t)b[16] << 8 | (uint32_t)b[32] << 16 | (uint32_t)b[48] << 24) >> (c & 4);
  } else {
    r.codes = *reinterpret_cast<const uint32_t*>(blk + kv4_k_off(4 * c, t)) >> (8 * (c & 1));
  }
  return r;
}
template <bool F32>
__device__ inline void store_row(const GatherArgs& a, int64_t tok, int h, int l, const RowPart& r) {
  const size_t at = ((size_t)tok * a.Hkv + h) * kD + 4 * (l & 31);
  const float2 m = meta_of(r.meta, a.meta_bf16);
  const uint32_t x = r.codes;
  if (l >> 5) put4<F32>(a.v, at, value_of(x, 0, m), value_of(x, 8, m), value_of(x, 16, m), value_of(x, 24, m));
  else put4<F32>(a.k, at, value_of(x, 0, m), value_of(x, 16, m), value_of(x, 4, m), value_of(x, 20, m));
}

template <bool F32>
__global__ __launch_bounds__(256) void kv4_gather_rows_kernel(GatherArgs a) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.n_tok * a.Hkv) return;
  const int64_t tok = row / a.Hkv, slot = a.slots[tok];
  const int h = (int)(row - tok * a.Hkv), l = threadIdx.x & 63;
  if (slot >= 0) store_row<F32>(a, tok, h, l, load_row(a, h, slot, l));
}

constexpr int kRowsMost = 12 << 10;  // (token, head) rows up to which they are read one by one
constexpr int kPageRows = 8;        // members of a page from which on it is read whole
constexpr int kSmallPages = 8;      // pages with fewer after which the rest of a tile is read row by row

template <bool F32>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3, 3))) void kv4_gather_kernel(GatherArgs a) {
  __shared__ int idx_all[4][kP];  // per wave, of a page's slots: the tile's token, or -1
  __shared__ uint32_t vsz_all[4][kP];
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63, lo = l & 15, hi = l >> 4, ng = a.ng;
  // Blocks go to the 8 XCDs in turn: the heads of a tile, whose output rows are
  // neighbours, to the same one.
  const unsigned turn = blockIdx.x / 8;
  const int64_t tok0 = ((int64_t)(turn / (unsigned)a.Hkv) * 8 + blockIdx.x % 8) * 64;
  const int h = (int)(turn % (unsigned)a.Hkv);
  if (tok0 >= a.n_tok) return;
  int* idx = idx_all[w];
  uint32_t* vsz = vsz_all[w];
  const int64_t slot = tok0 + l < a.n_tok ? a.slots[tok0 + l] : -1;
  const int64_t page = slot >= 0 ? slot / kP : -1;
  const int t = (int)(slot - page * kP);
  uint64_t open = __ballot(slot >= 0), loose = 0;
  int small = 0;  // pages of fewer members
  while (open) {  // one page per turn, the same in the four waves
    const int first = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)open) - 1);
    const int64_t p = ((int64_t)(uint32_t)__builtin_amdgcn_readlane((int)(page >> 32), first) << 32) |
                      (uint32_t)__builtin_amdgcn_readlane((int)page, first);
    const bool member = (open >> l & 1) && page == p;
    const uint64_t members = __ballot(member);
    if (__popcll(members) < kPageRows) {
      const uint64_t rest = ++small < kSmallPages ? members : open;  // (then the others hardly have more)
      loose |= rest;
      open &= ~rest;
      continue;
    }
    // the wave's quarter, whole rows: K of slots 16 w .. + 15 (lane: slot 16 w + l / 4,
    // channels 32 kc + 8 (l % 4) ..), V of slots 8 w .. + 7 and 32 more (lane: channels
    // 32 hi + lo, + 16)
    const uint8_t* blk = a.pages + ((size_t)p * a.Hkv + h) * kv4_block_bytes(ng);
    const int tk = 16 * w + (l >> 2), c8 = l & 3;
    const uint4 kr = reinterpret_cast<const uint4*>(blk)[64 * (tk & 3) + 16 * c8 + (tk >> 2)];
    const uint4 vr = reinterpret_cast<const uint4*>(blk + kKv4CodeBytes)[64 * hi + 16 * w + lo];
    uint32_t zk[4];
#pragma unroll
    for (int kc = 0; kc < 4; ++kc)
      zk[kc] = reinterpret_cast<const uint32_t*>(blk + kv4_sz_off(ng, 0))[tk * ng + kc * ng / 4];
    // V entries of the wave's slots: lane (slot 32 (l / 32) + 8 w + l / 4 % 8, block l % 4)
    const uint32_t zv = reinterpret_cast<const uint32_t*>(
        blk + kv4_sz_off(ng, 1))[(32 * (l >> 5) + 8 * w + (l >> 2 & 7)) * ng + (l & 3) * ng / 4];
    lane_exchange();  // the last turn's reads come first
    idx[l] = -1;
    vsz[l] = zv;
    lane_exchange();
    // Of tokens of the same slot the last one goes first and the others wait.  (The waves
    // must take the same one, as each stores its part of the row, and which of several
    // stores to one LDS word remains is not defined: a maximum is.)
    if (member) atomicMax(&idx[t], l);
    lane_exchange();
    open &= ~__ballot(member && idx[t] == l);
    if (const int i = idx[tk]; i >= 0) {
      const size_t at = ((size_t)(tok0 + i) * a.Hkv + h) * kD + 8 * c8;
      const uint32_t d[4] = {kr.x, kr.y, kr.z, kr.w};
#pragma unroll
      for (int kc = 0; kc < 4; ++kc) {
        const float2 m = meta_of(zk[kc], a.meta_bf16);
        put4<F32>(a.k, at + 32 * kc, value_of(d[kc], 0, m), value_of(d[kc], 16, m), value_of(d[kc], 4, m),
                  value_of(d[kc], 20, m));
        put4<F32>(a.k, at + 32 * kc + 4, value_of(d[kc], 8, m), value_of(d[kc], 24, m), value_of(d[kc], 12, m),
                  value_of(d[kc], 28, m));
      }
    }
    const uint32_t d[4] = {vr.x, vr.y, vr.z, vr.w};
#pragma unroll
    for (int k = 0; k < 16; ++k) {  // slot 32 kt + 8 w + 4 f + x
      const int kt = k >> 3, f = k >> 2 & 1, x = k & 3;
      const int i = __builtin_amdgcn_readfirstlane(idx[32 * kt + 8 * w + 4 * f + x]);
      if (i < 0) continue;
      const float2 m = meta_of(vsz[4 * k + hi], a.meta_bf16);
      const uint32_t b = d[2 * kt + f] >> (8 * (x / 2 + 2 * (x % 2)));
      const size_t at = ((size_t)(tok0 + i) * a.Hkv + h) * kD + 32 * hi + lo;
      put1<F32>(a.v, at, value_of(b, 0, m));
      put1<F32>(a.v, at + 16, value_of(b, 4, m));
    }
  }
  // rows of the other pages: every fourth token of the tile (four at a time, whose
  // half-written lines leave the L2: 131072 tokens of as many pages 712 us for 646)
  for (uint64_t mine = loose & (0x1111111111111111ull << w); mine; mine &= mine - 1) {
    const int i = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)mine) - 1);
    const int64_t at = ((int64_t)(uint32_t)__builtin_amdgcn_readlane((int)(slot >> 32), i) << 32) |
                       (uint32_t)__builtin_amdgcn_readlane((int)slot, i);
    store_row<F32>(a, tok0 + i, h, l, load_row(a, h, at, l));
  }
}

// ---------------------------------------------------------------------------
// Eviction.  A (sequence, KV head) row keeps its m = min(len, budget) slots of largest
// rank: protected tokens first, then by weight, equal ranks from the lowest slot on.
// Kept slots below m stay; the i-th kept slot at or past m moves to the i-th free slot
// below m, so that only rows that must move do, sources and destinations are disjoint,
// and the moves can run in any order, in place.
//
//   select: one block of 16 waves per row, each wave a contiguous part of the slots.  The
//           m-th largest rank by radix selection on ordered 32-bit keys (3 histograms of
//           11, 11 and 10 bits), kept in registers up to 32 slots a thread; then every
//           wave counts what it keeps, one block-wide sum gives it its places in the
//           lists of holes and movers, and a last pass fills them and pairs them off.  Rows
//           of more than 32768 slots take several blocks each (kv4_evict_part_kernel).
//   move:   the moved rows' bytes (codes, scales, zeros) from page to page, one block per
//           page that receives any.
// Bounds: select the latency of its passes, one block per row: 32 x 8 rows of 8k to 16k
// slots 33 us, 13 of them the two streams' bytes at the copy rate; 8 rows of 2k slots 9 us
// (40 and 11.4 with the lists in the workspace and every wave copying its own kept slots;
// 73 with keys formed anew in every pass, two block-wide sums per 1024 slots).  Move the
// cache lines of the sources' V codes, 64 bytes of a row in 8 lines: the same rows to 1024
// slots, 240000 moves, 82 us for about 250 MB of lines (116 a wave per row).
// ---------------------------------------------------------------------------
constexpr int kSel = 1024;            // threads of a select block
constexpr int kSelLds = 32 * kSel;    // slots up to which they fit into its registers and LDS

// Larger key, larger rank: finite weights in order (-0 as 0), NaN below all, protected
// tokens above all.
__device__ inline uint32_t rank_key(float w, bool safe) {
  if (safe) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w == 0.0f ? 0.0f : w);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// The select in one block per row.  ITEMS: slots per thread at most; their keys are kept in
// registers, the lists of holes and movers (at most S / 2 of each) in LDS.
template <int ITEMS>
__global__ __launch_bounds__(kSel) void kv4_evict_select_kernel(
    int Hkv, int64_t S, int max_pages, const int32_t* __restrict__ seq_lens, const float* weights,
    float* weights_out, const int32_t* pos, int32_t* pos_out, const int32_t* __restrict__ seen_all,
    int budget, int sink, int recent, int32_t* __restrict__ new_lens, int32_t* __restrict__ counts,
    int32_t* __restrict__ source, int64_t row0) {
  constexpr int kW = kSel / 64, kB = ITEMS % 6 == 0 ? 6 : 4;  // kB: slots per thread whose loads are issued together
  __shared__ int2 hist[kSel];  // entry i of the ints: keys whose digit is 2047 - i
  __shared__ int3 part[kW];    // per wave: keys equal to the last kept one, holes, movers
  __shared__ int above_all[kW];
  __shared__ uint32_t found;
  __shared__ int left, same_all;
  __shared__ uint16_t list[2][ITEMS * kSel / 2];  // holes, movers, ascending
  __shared__ uint64_t stays[ITEMS * kSel / 64];   // bit per slot: kept, and below m
  const int64_t row = row0 + blockIdx.x;
  const int b = (int)(row / Hkv), h = (int)(row - (int64_t)b * Hkv), t = threadIdx.x, w = t >> 6, l = t & 63;
  const int n = min(max(seq_lens[b], 0), max_pages * kP), m = min(n, budget), seen = seen_all[b];
  const float* w_in = weights + row * S;
  const int32_t* p_in = pos + row * S;
  float* w_out = weights_out + row * S;
  int32_t* p_out = pos_out + row * S;
  int32_t* src = source + row * S;
  if (h == 0 && t == 0) new_lens[b] = m;
  auto pos_of = [&](int i) {
    const int p = p_in[i];
    return p >= 0 ? p : seen - (n - i);
  };
  int n_moves = 0;
  if (n <= budget) {
    for (int i = t; i < n; i += kSel) {
      w_out[i] = w_in[i];
      p_out[i] = pos_of(i);
    }
  } else {
    // the wave's slots: [s0, s1), s0 + 64 i + lane for i < reps
    const int reps = (n + kSel - 1) / kSel, s0 = w * 64 * reps, s1 = min(n, s0 + 64 * reps);
    // kB keys from item i0 on, all loads first (keys past s1 are not used)
    auto load_keys = [&](int i0, uint32_t* key) {
      int p[kB];
      float x[kB];
#pragma unroll
      for (int i = 0; i < kB; ++i) {
        const int at = min(s0 + 64 * (i0 + i) + l, n - 1);
        p[i] = p_in[at];
        x[i] = w_in[at];
      }
#pragma unroll
      for (int i = 0; i < kB; ++i) {
        const int at = min(s0 + 64 * (i0 + i) + l, n - 1), q = p[i] >= 0 ? p[i] : seen - (n - at);
        key[i] = rank_key(x[i], q < sink || q >= seen - recent);
      }
    };
    hist[t] = make_int2(0, 0);
    uint32_t keys[ITEMS];
#pragma unroll
    for (int i0 = 0; i0 < ITEMS; i0 += kB)
      if (i0 < reps) load_keys(i0, keys + i0);
    // f(i, key, valid) of the wave's slots in order
    auto each = [&](auto&& f) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
        if (i < reps) f(i, keys[i], s0 + 64 * i + l < s1);
    };
    uint32_t prefix = 0;
    int need = m;  // slots still to be kept among the keys that share the prefix
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
      each([&](int, uint32_t k, bool valid) {
        if (valid && (pass == 0 || (k >> (shift + bits)) == (prefix >> (shift + bits))))
          atomicAdd(&reinterpret_cast<int*>(hist)[2047 - ((k >> shift) & ((1u << bits) - 1))], 1);
      });
      __syncthreads();
      const int2 c = hist[t];  // digits 2047 - 2 t, 2046 - 2 t
      hist[t] = make_int2(0, 0);
      int above = wave_prefix(c.x + c.y);  // of the wave's keys, those of digits from 2046 - 2 t up
      if (l == 63) above_all[w] = above;
      __syncthreads();
      above -= c.x + c.y;
#pragma unroll
      for (int i = 0; i < kW; ++i) above += i < w ? above_all[i] : 0;
      if (above < need && above + c.x >= need) {
        found = 2047 - 2 * t;
        left = need - above;
        same_all = c.x;
      } else if (above + c.x < need && above + c.x + c.y >= need) {
        found = 2046 - 2 * t;
        left = need - above - c.x;
        same_all = c.y;
      }
      __syncthreads();
      prefix |= found << shift;
      need = left;
      if (same_all == need) break;  // every key of the prefix is kept: the lower digits do not matter
    }
    // kept: keys from the prefix up, or, where more keys are equal to it than can be kept
    // (all 32 bits then), those above it and the first `need` slots of equal key
    const bool ties = same_all > need;
    const uint64_t below = (1ull << l) - 1;
    int eq0 = 0;  // equal keys of the waves before
    if (ties) {
      int eq = 0;
      each([&](int, uint32_t k, bool valid) { eq += __popcll(__ballot(valid && k == prefix)); });
      if (l == 0) part[w].x = eq;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kW; ++i) eq0 += i < w ? part[i].x : 0;
    }
    auto kept_of = [&](uint32_t k, bool valid, int& e) {
      if (!ties) return valid && k >= prefix;
      const uint64_t same = __ballot(valid && k == prefix);
      const bool kept = valid && (k > prefix || (k == prefix && e + __popcll(same & below) < need));
      e += __popcll(same);
      return kept;
    };
    int e = eq0, holes = 0, movers = 0;
    each([&](int i, uint32_t k, bool valid) {
      const int at = s0 + 64 * i + l;
      const bool kept = kept_of(k, valid, e);
      holes += __popcll(__ballot(valid && at < m && !kept));
      movers += __popcll(__ballot(kept && at >= m));
    });
    if (l == 0) {
      part[w].y = holes;
      part[w].z = movers;
    }
    __syncthreads();
    holes = movers = 0;
#pragma unroll
    for (int i = 0; i < kW; ++i) {
      holes += i < w ? part[i].y : 0;
      movers += i < w ? part[i].z : 0;
      n_moves += part[i].z;
    }
    e = eq0;
    each([&](int i, uint32_t k, bool valid) {
      const int at = s0 + 64 * i + l;
      const bool kept = kept_of(k, valid, e);
      const bool hole = valid && at < m && !kept, mover = kept && at >= m;
      const uint64_t hs = __ballot(hole), ms = __ballot(mover);
      const int ih = holes + __popcll(hs & below), im = movers + __popcll(ms & below);
      if (hole) list[0][ih] = (uint16_t)at;
      if (mover) list[1][im] = (uint16_t)at;
      const uint64_t st = __ballot(kept && at < m);
      if (l == 0) stays[s0 / 64 + i] = st;
      holes += __popcll(hs);
      movers += __popcll(ms);
    });
    __syncthreads();
    for (int i = t; i < m; i += kSel)  // over all threads, whichever wave the slots are
      if (stays[i / 64] >> (i & 63) & 1) {
        w_out[i] = w_in[i];
        p_out[i] = pos_of(i);
        src[i] = -1;
      }
    for (int i = t; i < n_moves; i += kSel) {
      const int x = list[1][i], y = list[0][i];
      w_out[y] = w_in[x];
      p_out[y] = pos_of(x);
      src[y] = x;
    }
    __syncthreads();  // in place, the sources lie in what is cleared now
  }
  for (int64_t i = m + t; i < S; i += kSel) {
    w_out[i] = 0.0f;
    p_out[i] = -1;
  }
  if (t == 0) counts[row] = n_moves;
}

// ---------------------------------------------------------------------------
// The select over several blocks per row, part `c` of `parts` each, for rows that do not fit
// into one block or are too few to fill the device with one: a launch per histogram, every
// block writing its own and, in the next launch, adding up the row's; then one that places.
// With the counts of the parts before its own a block knows, slot by slot, how many kept
// slots come before: a hole at slot s is the (s - before)-th, a mover the (before - kept
// slots below m)-th.  (A pass whose digit settles the selection ends the histograms.)  Bound:
// two to four reads of the row's weights and positions, 8 bytes a slot, and five launches: 256
// rows of 100000 slots 402 us with the moved rows' reading back, 8 rows of 70000 44 us.  Holes
// leave their number in `source`, movers their slot, position and
// weight in a list, counted from its end (m - 1 - before), and the move kernel pairs them.
// ---------------------------------------------------------------------------
struct Found {        // after a pass
  uint32_t prefix;    // of the key of the last kept slot
  int need;           // slots still to be kept among those that share it; 0: all above it are kept, and no more
  int same;           // how many share it
  int before;         // kept slots of the row's parts before, by the digits so far
};
struct Mover {
  int slot, pos;
  float w;
};
struct Parts {
  int Hkv;
  int64_t S;
  int max_pages;
  const int32_t* __restrict__ seq_lens;
  const float* weights;
  float* weights_out;
  const int32_t* pos;
  int32_t* pos_out;
  const int32_t* __restrict__ seen;
  int budget, sink, recent;
  int32_t* __restrict__ new_lens;
  int32_t* __restrict__ counts;
  Mover* __restrict__ movers;    // [row][S / 2]
  int32_t* __restrict__ source;  // [row][S]
  int2* __restrict__ hist;       // [row][part][3][kSel]
  Found* __restrict__ found;     // [row][part][2]
  int parts;
};
constexpr int kMaxParts = 16;

// PASS 0 .. 2: histogram of that digit of the keys; 3: place.
template <int PASS>
__global__ __launch_bounds__(kSel) void kv4_evict_part_kernel(Parts a, int64_t row0) {
  constexpr int kW = kSel / 64, kB = 4;
  __shared__ int2 hist[kSel];
  __shared__ int2 sums[kW];
  __shared__ Found got;
  __shared__ int got_same_before;
  const int64_t row = row0 + blockIdx.x / a.parts;
  const int c = (int)(blockIdx.x % a.parts), t = threadIdx.x, w = t >> 6, l = t & 63;
  const int b = (int)(row / a.Hkv), h = (int)(row - (int64_t)b * a.Hkv);
  const int n = min(max(a.seq_lens[b], 0), a.max_pages * kP), m = min(n, a.budget), seen = a.seen[b];
  const float* w_in = a.weights + row * a.S;
  const int32_t* p_in = a.pos + row * a.S;
  float* w_out = a.weights_out + row * a.S;
  int32_t* p_out = a.pos_out + row * a.S;
  if (PASS < 3 && n <= a.budget) return;
  // the wave's slots: [s0, s1), s0 + 64 i + lane for i < reps
  const int reps = (int)(((int64_t)n + a.parts * kSel - 1) / (a.parts * kSel));
  const int64_t first = ((int64_t)c * kW + w) * 64 * reps;
  const int s0 = (int)min((int64_t)n, first), s1 = (int)min((int64_t)n, first + 64 * reps);
  // f(slot, key, weight, position, valid) of the wave's slots in order
  auto each = [&](auto&& f) {
    for (int i0 = 0; i0 < reps && s0 + 64 * i0 < s1; i0 += kB) {
      int p[kB];
      float x[kB];
#pragma unroll
      for (int i = 0; i < kB; ++i) {
        const int at = min(s0 + 64 * (i0 + i) + l, n - 1);
        p[i] = p_in[at];
        x[i] = w_in[at];
      }
#pragma unroll
      for (int i = 0; i < kB; ++i) {
        const int at = s0 + 64 * (i0 + i) + l, q = p[i] >= 0 ? p[i] : seen - (n - at);
        f(at, rank_key(x[i], q < a.sink || q >= seen - a.recent), x[i], q, at < s1);
      }
    }
  };
  const int64_t part = row * a.parts + c;
  if (PASS == 3) {
    if (h == 0 && c == 0 && t == 0) a.new_lens[b] = m;
    for (int64_t i = n + (int64_t)c * kSel + t; i < a.S; i += (int64_t)a.parts * kSel) {
      w_out[i] = 0.0f;
      p_out[i] = -1;
    }
    if (n <= a.budget) {
      if (c == 0 && t == 0) a.counts[row] = 0;
      each([&](int at, uint32_t, float x, int q, bool valid) {
        if (!valid) return;
        w_out[at] = x;
        p_out[at] = q;
      });
      return;
    }
  }
  Found f{0u, m, 0, 0};
  int same_before = 0;
  if (PASS > 1) f = a.found[part * 2 + PASS - 2];
  if (PASS > 0 && f.need > 0) {  // the digit of the pass before
    constexpr int kShift = PASS == 1 ? 21 : PASS == 2 ? 10 : 0;
    int2 all = make_int2(0, 0), bef = make_int2(0, 0);  // digits 2047 - 2 t, 2046 - 2 t: of the row, of the parts before
#pragma unroll 4
    for (int k = 0; k < a.parts; ++k) {
      const int2 x = a.hist[((row * a.parts + k) * 3 + PASS - 1) * kSel + t];
      all.x += x.x;
      all.y += x.y;
      bef.x += k < c ? x.x : 0;
      bef.y += k < c ? x.y : 0;
    }
    int above = wave_prefix(all.x + all.y), above_bef = wave_prefix(bef.x + bef.y);
    if (l == 63) sums[w] = make_int2(above, above_bef);
    __syncthreads();
    above -= all.x + all.y;
    above_bef -= bef.x + bef.y;
#pragma unroll
    for (int i = 0; i < kW; ++i) {
      above += i < w ? sums[i].x : 0;
      above_bef += i < w ? sums[i].y : 0;
    }
    auto set = [&](int digit, int ab, int ab_bef, int same, int same_bef) {
      if (ab < f.need && ab + same >= f.need) {
        got = Found{f.prefix | (uint32_t)digit << kShift, f.need - ab, same, f.before + ab_bef};
        got_same_before = same_bef;
      }
    };
    set(2047 - 2 * t, above, above_bef, all.x, bef.x);
    set(2046 - 2 * t, above + all.x, above_bef + bef.x, all.y, bef.y);
    __syncthreads();
    f = got;
    same_before = got_same_before;
    if (f.same == f.need) {  // all of them are kept: those above prefix - 1, and the lower digits do not matter
      f.prefix -= 1;
      f.before += same_before;
      f.need = same_before = 0;
    }
  }
  if (PASS > 0 && PASS < 3) {
    if (t == 0) a.found[part * 2 + PASS - 1] = f;
    if (f.need == 0) return;
  }
  if (PASS < 3) {
    constexpr int kShift = PASS == 0 ? 21 : PASS == 1 ? 10 : 0, kBits = PASS == 2 ? 10 : 11;
    hist[t] = make_int2(0, 0);
    __syncthreads();
    each([&](int, uint32_t k, float, int, bool valid) {
      if (valid && (PASS == 0 || (k >> ((kShift + kBits) & 31)) == (f.prefix >> ((kShift + kBits) & 31))))
        atomicAdd(&reinterpret_cast<int*>(hist)[2047 - ((k >> kShift) & ((1u << kBits) - 1))], 1);
    });
    __syncthreads();
    a.hist[(part * 3 + PASS) * kSel + t] = hist[t];
    return;
  }
  // place: kept are the keys above the prefix and the first f.need slots of equal key
  int more = 0, same = 0;
  each([&](int, uint32_t k, float, int, bool valid) {
    more += __popcll(__ballot(valid && k > f.prefix));
    same += __popcll(__ballot(valid && k == f.prefix));
  });
  if (l == 0) sums[w] = make_int2(more, same);
  __syncthreads();
  more = f.before;
  same = same_before;
#pragma unroll
  for (int i = 0; i < kW; ++i) {
    more += i < w ? sums[i].x : 0;
    same += i < w ? sums[i].y : 0;
  }
  Mover* movers = a.movers + row * (a.S / 2);
  int32_t* src = a.source + row * a.S;
  const uint64_t below = (1ull << l) - 1;
  each([&](int at, uint32_t k, float x, int q, bool valid) {
    const uint64_t gt = __ballot(valid && k > f.prefix), eq = __ballot(valid && k == f.prefix);
    const int same_at = same + __popcll(eq & below);
    const int before = more + __popcll(gt & below) + min(same_at, f.need);  // kept slots below this one
    const bool kept = valid && (k > f.prefix || (k == f.prefix && same_at < f.need));
    more += __popcll(gt);
    same += __popcll(eq);
    if (!valid) return;
    if (at == m) a.counts[row] = m - before;
    if (at < m) {
      src[at] = kept ? -1 : -2 - (at - before);
      if (kept) {
        w_out[at] = x;
        p_out[at] = q;
      }
    } else {
      if (kept) movers[m - 1 - before] = Mover{at, q, x};
      w_out[at] = 0.0f;
      p_out[at] = -1;
    }
  });
}

// Rows that move into destination page blockIdx.x of row blockIdx.y, by source slot.
// Fewer than kPageRows of them go one at a time, a wave each: 16 dwords of K codes, 64
// bytes of V codes, 2 ng metadata entries.  More are put together in the page's own units: wave
// w takes the K units of slots 4 lo + w (16 bytes of one slot per lane) and the V units
// of channels 32 w .. (16 slots of a channel pair per lane: 16 byte loads, of which 16
// lanes share two cache lines, and one store; a wave per row moved 64 single bytes both
// ways: 32 x 8 rows of 16k to 1024 slots, 116 us).
__global__ __launch_bounds__(256) void kv4_evict_move_kernel(uint8_t* __restrict__ pages, int Hkv, int64_t S,
                                                             int ng, const int32_t* __restrict__ block_table,
                                                             int max_pages, const int32_t* __restrict__ counts,
                                                             const int32_t* __restrict__ source,
                                                             const Mover* __restrict__ movers,
                                                             float* __restrict__ weights_out,
                                                             int32_t* __restrict__ pos_out, int budget,
                                                             int64_t row0) {
  __shared__ const uint8_t* from_all[4][kP];  // per wave, of a page's slots: the source's block
  __shared__ int src_all[4][kP];              // and its slot in it, or -1
  const int64_t row = row0 + blockIdx.y;
  const int n_moves = counts[row];
  if (n_moves == 0) return;  // then source is not written
  const int b = (int)(row / Hkv), h = (int)(row - (int64_t)b * Hkv);
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63, lo = l & 15, hi = l >> 4;
  const int32_t* bt = block_table + (size_t)b * max_pages;
  const int slot = blockIdx.x * kP + l;
  int from = slot < budget ? source[row * S + slot] : -1;  // (moves: the row has more than budget slots)
  if (from < -1) {  // hole -2 - from, of the select in parts
    const Mover e = movers[row * (S / 2) + n_moves + 1 + from];
    from = e.slot;
    if (w == 0) {
      weights_out[row * S + slot] = e.w;
      pos_out[row * S + slot] = e.pos;
    }
  }
  const uint64_t moved = __ballot(from >= 0);
  if (!moved) return;
  const uint8_t* src = nullptr;
  if (from >= 0) src = pages + ((size_t)bt[from / kP] * Hkv + h) * kv4_block_bytes(ng);
  uint8_t* to = pages + ((size_t)bt[blockIdx.x] * Hkv + h) * kv4_block_bytes(ng);
  const uint8_t** from_of = from_all[w];
  int* src_of = src_all[w];
  from_of[l] = src;
  src_of[l] = from >= 0 ? from % kP : -1;
  lane_exchange();
  if (__popcll(moved) < kPageRows) {
    const int cv = 32 * (l >> 4) + (l & 15), sz = l - 16;  // lanes 16 ..: metadata entries of K, then of V
    int n = 0;
    for (uint64_t todo = moved; todo; todo &= todo - 1, ++n) {
      if ((n & 3) != w) continue;
      const int td = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)todo) - 1), ts = src_of[td];
      const uint8_t* f = from_of[td];
      const uint8_t v = f[kv4_v_off(cv, ts)];
      uint32_t d = 0;
      if (l < 16) d = *reinterpret_cast<const uint32_t*>(f + kv4_k_off(8 * l, ts));
      else if (sz < 2 * ng)
        d = *reinterpret_cast<const uint32_t*>(f + kv4_sz_off(ng, sz >= ng) + (ts * ng + sz % ng) * 4);
      to[kv4_v_off(cv, td)] = v;
      if (l < 16) *reinterpret_cast<uint32_t*>(to + kv4_k_off(8 * l, td)) = d;
      else if (sz < 2 * ng)
        *reinterpret_cast<uint32_t*>(to + kv4_sz_off(ng, sz >= ng) + (td * ng + sz % ng) * 4) = d;
    }
    return;
  }
  // V units: the bytes of slots that do not move come from the page itself
  uint4* vu = reinterpret_cast<uint4*>(to + kKv4CodeBytes) + 64 * w + l;
  const uint4 old = *vu;
  uint32_t got[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) {  // slot 32 kt + 8 hi + 4 f + x
    const int kt = k >> 3, f = k >> 2 & 1, x = k & 3, ts = 32 * kt + 8 * hi + 4 * f + x;
    const int s = src_of[ts];
    got[k] = s < 0 ? 256u : from_of[ts][kv4_v_off(32 * w + lo, s)];
  }
  const int tk = 4 * lo + w, sk = src_of[tk];
  uint4 kd = make_uint4(0, 0, 0, 0);
  if (sk >= 0) kd = reinterpret_cast<const uint4*>(from_of[tk])[64 * (sk % 4) + 16 * hi + sk / 4];
  uint32_t zd[2] = {0, 0};  // metadata entries of slot l: group w of K and of V
  const int sl = src_of[l];
  if (sl >= 0 && w < ng) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      zd[i] = *reinterpret_cast<const uint32_t*>(from_of[l] + kv4_sz_off(ng, i) + (sl * ng + w) * 4);
  }
  uint32_t d[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int x = k & 3, sh = 8 * (x / 2 + 2 * (x % 2));
    d[k >> 2] = got[k] > 255u ? d[k >> 2] : (d[k >> 2] & ~(255u << sh)) | (got[k] << sh);
  }
  *vu = make_uint4(d[0], d[1], d[2], d[3]);
  if (sk >= 0) reinterpret_cast<uint4*>(to)[64 * (tk % 4) + 16 * hi + tk / 4] = kd;
  if (sl >= 0 && w < ng) {
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<uint32_t*>(to + kv4_sz_off(ng, i) + (l * ng + w) * 4) = zd[i];
  }
}

}  // namespace

hipError_t launch_kv4_gather(const uint8_t* pages, int Hkv, const int64_t* slots, int64_t n_tok,
                             void* k, void* v, int out_f32, int meta_bf16, int ng, hipStream_t st) {
  // a launch holds fewer than 2^32 threads: 2^24 (token, head) rows at a time
  const int64_t most = std::max<int64_t>(64, (1 << 24) / Hkv / 64 * 64);  // (at most 2^18 blocks)
  for (int64_t t0 = 0; t0 < n_tok; t0 += most) {
    const int64_t n = std::min(most, n_tok - t0), at = t0 * Hkv * kD * (out_f32 ? 4 : 2);
    const GatherArgs a{pages, Hkv, slots + t0, n, static_cast<char*>(k) + at, static_cast<char*>(v) + at,
                       meta_bf16, ng};
    const bool by_row = n * Hkv <= kRowsMost;
    const int64_t blocks = by_row ? (n * Hkv + 3) / 4 : (n + 511) / 512 * 8 * Hkv;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, a); };
    if (by_row) {
      if (out_f32) go(kv4_gather_rows_kernel<true>);
      else go(kv4_gather_rows_kernel<false>);
    } else {
      if (out_f32) go(kv4_gather_kernel<true>);
      else go(kv4_gather_kernel<false>);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

namespace {
// Parts of a row's select, or 0: in one block per row, which takes up to 32768 slots.  (Of
// full tables in parts would be the faster way from 24000 slots on where rows are few, 8 rows
// of 32000 slots 37 us for 46, of short sequences in such tables one block is.)  About one
// part for each of 256 CUs: at two 64 rows of 49000 slots take 107 us for 93, since every block adds up
// its row's histograms.  In one block each, keys formed anew in every pass, they took 140; 8
// rows of 70000 slots 114 for 43.
int evict_parts(int64_t rows, int64_t S) {
  return S <= kSelLds ? 0 : (int)std::max<int64_t>(2, std::min<int64_t>(kMaxParts, 256 / rows));
}
// Moves per row, the source of every slot below the budget, and for a select in parts the
// lists of movers, the histograms and what was found in them.
struct EvictWs {
  size_t source_off, movers_off, hist_off, found_off, total;
};
EvictWs evict_ws(int Hkv, int B, int max_pages) {
  const size_t rows = (size_t)B * Hkv, S = (size_t)max_pages * kP;
  const size_t parts = evict_parts(rows, S), many = parts ? rows : 0;
  EvictWs w;
  w.source_off = align256(rows * sizeof(int32_t));
  w.movers_off = align256(w.source_off + rows * S * sizeof(int32_t));
  w.hist_off = align256(w.movers_off + many * (S / 2) * sizeof(Mover));
  w.found_off = align256(w.hist_off + many * parts * 3 * kSel * sizeof(int2));
  w.total = align256(w.found_off + many * parts * 2 * sizeof(Found));
  return w;
}
}  // namespace

size_t kv4_evict_ws_bytes(int Hkv, int B, int max_pages) { return evict_ws(Hkv, B, max_pages).total; }

hipError_t launch_kv4_evict(const EvictArgs& a, hipStream_t st) {
  const int64_t rows = (int64_t)a.B * a.Hkv, S = (int64_t)a.max_pages * kP;
  const EvictWs ws = evict_ws(a.Hkv, a.B, a.max_pages);
  uint8_t* base = static_cast<uint8_t*>(a.ws);
  int32_t* counts = reinterpret_cast<int32_t*>(base);
  int32_t* source = reinterpret_cast<int32_t*>(base + ws.source_off);
  Mover* movers = reinterpret_cast<Mover*>(base + ws.movers_off);
  const int parts = evict_parts(rows, S);
  const int64_t step = (1 << 20) / std::max(parts, 1);  // rows per launch, which holds fewer than 2^32 threads
  for (int64_t r0 = 0; r0 < rows; r0 += step) {
    const unsigned nr = (unsigned)std::min<int64_t>(rows - r0, step);
    if (parts) {
      const Parts p{a.Hkv, S, a.max_pages, a.seq_lens, a.weights, a.weights_out, a.pos, a.pos_out, a.seen,
                    a.budget, a.sink, a.recent, a.new_lens, counts, movers, source,
                    reinterpret_cast<int2*>(base + ws.hist_off), reinterpret_cast<Found*>(base + ws.found_off),
                    parts};
      auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(nr * parts), dim3(kSel), 0, st, p, r0); };
      go(kv4_evict_part_kernel<0>);
      go(kv4_evict_part_kernel<1>);
      go(kv4_evict_part_kernel<2>);
      go(kv4_evict_part_kernel<3>);
    } else {
      auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(nr), dim3(kSel), 0, st, a.Hkv, S, a.max_pages, a.seq_lens, a.weights,
                           a.weights_out, a.pos, a.pos_out, a.seen, a.budget, a.sink, a.recent, a.new_lens,
                           counts, source, r0);
      };
      if (S <= 4 * kSel) go(kv4_evict_select_kernel<4>);
      else if (S <= 12 * kSel) go(kv4_evict_select_kernel<12>);
      else go(kv4_evict_select_kernel<32>);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t pages = std::min<int64_t>(a.max_pages, ((int64_t)a.budget + kP - 1) / kP);  // that keep rows
  const int64_t most = std::min<int64_t>(65535, std::max<int64_t>(1, (1 << 23) / pages));
  for (int64_t r0 = 0; r0 < rows; r0 += most) {
    hipLaunchKernelGGL(kv4_evict_move_kernel, dim3((unsigned)pages, (unsigned)std::min(rows - r0, most)),
                       dim3(256), 0, st, a.pages, a.Hkv, S, a.ng, a.block_table, a.max_pages, counts, source,
                       movers, a.weights_out, a.pos_out, a.budget, r0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace oscar
