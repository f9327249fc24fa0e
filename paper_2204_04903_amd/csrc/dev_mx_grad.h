// dW (+)= dY^T X, X an 8-bit checkpoint.
// Part of pk_mx.hip: included there, in this order, inside its anonymous namespace.

template <bool BF16>
__global__ void __launch_bounds__(NT)
mx_weight_grad_kernel(const char* __restrict__ dy, int64_t dy_stride, const uint8_t* __restrict__ xq, int64_t x_stride, int64_t B, int64_t K,
                      int64_t items, float* __restrict__ dw, int64_t dw_stride, int accumulate)
{
    const int64_t words = (K + 3) / 4;
    for (int64_t it = (int64_t)blockIdx.x * NT + threadIdx.x; it < items; it += (int64_t)gridDim.x * NT) {
        const int64_t n = it / K, k = it - n * K;
        float acc = 0.f;
        for (int64_t b = 0; b < B; ++b) {
            const char* d = dy + b * dy_stride;
            const uint8_t* row = xq + b * x_stride;
            const float g = BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t*>(d)[n]) : reinterpret_cast<const float*>(d)[n];
            const f32x2v x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(row[k], mx_scale(row[words * 4 + k / 32]), false);
            acc += g * x.x;
        }
        float* o = dw + n * dw_stride + k;
        *o = accumulate ? *o + acc : acc;
    }
}
