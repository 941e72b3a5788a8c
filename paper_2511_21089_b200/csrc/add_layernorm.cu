// Residual addition + LayerNorm + (optionally) 8-bit output with scales in one pass (mlpmoe_add_layernorm):
//     s = x + r,  x_out = s,  v = (s - mean(s)) / sqrt(var(s) + eps) * gain + bias,  out = v | e4m3(v / scale).
// The kernel of mlpmoe_add_rmsnorm with one sum over the row more: HBM-bound, a row in registers between its one load and its one store.
// 16384 x 4096 fp32 + bf16 to fp32 and bf16: 805 MB in 121 us in short runs, 127 to 136 over seconds (92 to 98 % of a copy); to e4m3 738 MB in 137 to 148
// (78 to 84 %: a reduction more).  Rows that start anywhere, to bf16: 12288 x 4096 114 us (82 %), 16384 x 901 37 to 39 (71 to 75 %), 12285 x 4097 165 (57 %), 16384 x 201 14 (44 %).
#include "add_norm.cuh"

extern "C" mlpmoe_status_t mlpmoe_add_layernorm(const void* x, mlpmoe_dtype_t x_dtype, int64_t x_stride, const void* r,
                                                mlpmoe_dtype_t r_dtype, int64_t r_stride, const float* gain, const float* bias, void* x_out,
                                                int64_t x_out_stride, void* out, mlpmoe_dtype_t out_dtype, int64_t out_stride,
                                                float* scales, int64_t group, int64_t n_tokens, int64_t d_model, float eps, void* stream) {
  return mlpmoe::add_norm<true>(x, x_dtype, x_stride, r, r_dtype, r_stride, gain, bias, x_out, x_out_stride, out, out_dtype, out_stride, scales,
                                group, n_tokens, d_model, eps, stream);
}
