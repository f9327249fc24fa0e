// y = Q(x) W^T + bias, both operands in 4 bits.
// Part of pk_mx.hip: included there, in this order, inside its anonymous namespace.

struct LinearLayout { int64_t x_stride; size_t total; };
inline LinearLayout linear_layout(int64_t M, int64_t N, int64_t K)
{
    LinearLayout L;
    (void)N;
    L.x_stride = (mx_row_bytes(PK_MXFP4, K) + 15) / 16 * 16;
    L.total = std::max<size_t>(kAlign, (size_t)(M * L.x_stride) + kAlign);
    return L;
}

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4m __attribute__((ext_vector_type(4)));

// block kb of a row: its 32 codes (what lies behind the last word is zero) and its scale (1 behind the last block)
__device__ __forceinline__ void mx_load_block(const uint8_t* row, int words, int blocks, int kb, i32x8& v, int& scale)
{
    const uint32_t* at = reinterpret_cast<const uint32_t*>(row) + 4 * kb;
    v = i32x8{0, 0, 0, 0, 0, 0, 0, 0};
    if (4 * kb + 4 <= words) {
        uint32_t u[4];
        load_u32<4>(at, u);
        v[0] = (int)u[0]; v[1] = (int)u[1]; v[2] = (int)u[2]; v[3] = (int)u[3];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * kb + i < words) v[i] = (int)at[i];
    }
    scale = kb < blocks ? (int)row[words * 4 + kb] : 127;
}

// A wavefront takes 16 rows and 64 columns of y: one scaled product of 16 x 16 x 128 per 16 columns and 128 of K.  Lane l holds
// row (and column) l % 16 and of the 128 the block l / 16, so that its operand is 16 bytes and one scale byte.
template <bool BF16>
__global__ void __launch_bounds__(256)
mx_linear_kernel(const uint8_t* __restrict__ xq, int64_t x_stride, const uint8_t* __restrict__ wq, int64_t w_stride, int M, int N, int K,
                 const float* __restrict__ bias, char* __restrict__ y, int64_t y_stride)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * 64, words = (K + 7) / 8, blocks = (K + 31) / 32;
    for (int64_t m0 = (int64_t)blockIdx.y * 64 + wave * 16; m0 < M; m0 += (int64_t)gridDim.y * 64) {
        const uint8_t* xr = xq + min(m0 + r, (int64_t)M - 1) * x_stride;
        f32x4m acc[4] = {};
        for (int kb = 0; kb < blocks; kb += 4) {
            i32x8 a; int sa;
            mx_load_block(xr, words, blocks, kb + q, a, sa);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                i32x8 b; int sb;
                mx_load_block(wq + (int64_t)min(n0 + 16 * t + r, N - 1) * w_stride, words, blocks, kb + q, b, sb);
                acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[t], 4, 4, 0, sa, 0, sb);
            }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int n = n0 + 16 * t + r;
            if (n >= N) continue;
            const float add = bias ? bias[n] : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t m = m0 + 4 * q + i;
                if (m >= M) continue;
                const float v = acc[t][i] + add;
                if constexpr (BF16) reinterpret_cast<uint16_t*>(y)[m * y_stride + n] = (uint16_t)pack_bf16(v, 0.f);
                else reinterpret_cast<float*>(y)[m * y_stride + n] = v;
            }
        }
    }
}
