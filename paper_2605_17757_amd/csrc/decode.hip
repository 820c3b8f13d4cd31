// Decode attention over the INT2 paged cache (Alg. 1 DecodeStep; Sec. 4
// "Decoding Attention Kernel"), in three kernels:
//   prepare : q~ = q R_k * (sm_scale * log2 e)                    [B*Hq, 128] fp32
//             (in append.hip, where it can share a launch with the cache update)
//   split   : online softmax over page ranges in the rotated basis, unnormalized
//             o~ and (m, l) per piece (decode_mfma.hip)
//   reduce  : log-sum-exp merge of the pieces, o = o~ R_v^T, bf16/fp32 store
//             (this file; the body in reduce_body.h)
//
// Rotated-basis identities used (Sec. 2, K^ = Q(K~) R^T with R orthogonal):
//   q k^T = (q R_k) Q(k~)^T,   sum_t p_t v^_t = (sum_t p_t Q(v~_t)) R_v^T,
// and per group g of 32 channels, with Q(x~)_c = s_g (code_c - z_g):
//   q~ . Q(k~) = sum_g s_g (sum_{c in g} q~_c code_c - z_g sum_{c in g} q~_c).
// Scores are kept in log2 units (q~ carries log2 e) so the softmax uses exp2.
#include <hip/hip_fp16.h>

#include <type_traits>

#include "reduce_body.h"

namespace oscar {
namespace {

template <bool MIXED, int RB>
__global__ __launch_bounds__(kRedThreads) void reduce_kernel(int rows, int num_splits,
                                                     const float* __restrict__ part_o,
                                                     const float* __restrict__ part_ml,
                                                     const float* __restrict__ Rv,
                                                     void* __restrict__ out, int out_f32, int rph,
                                                     int Hq, int Hkv) {
  reduce_body<MIXED, RB>(blockIdx.x, rows, num_splits, part_o, part_ml, Rv, out, out_f32, rph, Hq, Hkv);
}

}  // namespace

hipError_t launch_decode_split(const uint8_t* pages, int Hkv, int B, int Hq,
                               const int32_t* block_table, int max_pages,
                               const int32_t* seq_lens, int num_splits, const float* qt,
                               float* part_o, float* part_ml, hipStream_t st, int meta_bf16,
                               int ng, const MixedSpec* mixed) {
  // (with more splits the grid does not grow with the sequences)
  return by_seqs(B, num_splits == 1 ? launch_seqs(Hq) : B, [&](int b0, int nb) {
    const size_t row = (size_t)b0 * Hq, part = row * (mixed ? mixed->row_stride : num_splits);
    return launch_decode_split_mfma(pages, Hkv, nb, Hq, block_table + (size_t)b0 * max_pages, max_pages,
                                    seq_lens + b0, num_splits, device_cus(), qt + row * kD,
                                    part_o + part * kD, part_ml + part * 2, st, meta_bf16, ng, mixed);
  });
}

hipError_t launch_decode_reduce(int B, int Hq, int num_splits, const float* part_o,
                                const float* part_ml, const float* Rv, void* out, int out_f32,
                                hipStream_t st, const MixedSpec* mixed, int rph, int Hkv) {
  if (const int most = launch_seqs(Hq); B > most)
    return by_seqs(B, most, [&](int b0, int nb) {
      const size_t row = (size_t)b0 * Hq, part = row * (mixed ? num_splits + 1 : num_splits);
      return launch_decode_reduce(nb, Hq, num_splits, part_o + part * kD, part_ml + part * 2, Rv,
                                  static_cast<char*>(out) + row * kD * (out_f32 ? 4 : 2), out_f32, st,
                                  mixed, rph, Hkv);
    });
  const int rows = B * Hq;
  const int rb = reduce_rows(rows);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(query_blocks(B, Hq, Hkv, rph, rb)), dim3(kRedThreads), 0, st, rows,
                       num_splits, part_o, part_ml, Rv, out, out_f32, rph, Hq, Hkv);
  };
  auto by_rows = [&](auto mixed_c) {
    constexpr bool M = decltype(mixed_c)::value;
    if (rb == 16) go(reduce_kernel<M, 16>);
    else if (rb == 8) go(reduce_kernel<M, 8>);
    else if (rb == 4) go(reduce_kernel<M, 4>);
    else go(reduce_kernel<M, 2>);
  };
  if (mixed) by_rows(std::true_type{});
  else by_rows(std::false_type{});
  return hipGetLastError();
}

}  // namespace oscar
