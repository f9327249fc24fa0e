// dW (+)= dY^T X, X an 8-bit checkpoint.
// Part of pk_mx.hip: included there, in this order, inside its anonymous namespace.

// ---------------------------------------------------------------------------
// The sum runs over the samples, which are the rows of both operands, while a lane of a matrix instruction wants eight
// consecutive samples of one column: a thread loads eight rows of four columns, and turns them over in registers on the way to
// LDS.  X's elements become bf16 there (four digits and a power of two: exact); of an fp32 dY every element becomes three
// bf16 numbers whose sum it is (8 + 8 + 8 digits, cut off, not rounded), so that all products are exact and what is
// lost is what fp32 additions lose.
// A block takes kGradN x kGradK elements of dW and a stretch of the samples, kGradB a step; the stretches' sums meet in a
// second launch in their order, so that a result does not depend on which block came first.
// ---------------------------------------------------------------------------
constexpr int kGradN = 128, kGradK = 128, kGradB = 64;
constexpr int64_t kGradBlocks = 512;             // two blocks a compute unit
constexpr int kGradRow = kGradB * 2;             // bytes of a column's samples in LDS

struct GradLayout { int64_t tiles_n, tiles, steps, splits, ld; size_t total; };
inline GradLayout grad_layout(int64_t B, int64_t N, int64_t K)
{
    GradLayout L;
    L.tiles_n = (N + kGradN - 1) / kGradN;
    L.steps = (B + kGradB - 1) / kGradB;
    L.tiles = L.tiles_n * ((K + kGradK - 1) / kGradK);
    L.splits = std::max<int64_t>(1, std::min<int64_t>(L.steps / 4, kGradBlocks / L.tiles));
    L.ld = (K + 3) / 4 * 4;
    L.total = L.splits > 1 ? (size_t)(L.splits * N * L.ld * 4) : kAlign;
    return L;
}

// Where 16 bytes (samples 8 c .. 8 c + 7) of column r stand: neighbouring columns, which lanes read together, and every fourth,
// which they write together, fall on different banks.
__device__ __forceinline__ int grad_at(int r, int c) { return r * kGradRow + ((c ^ (r >> 2) ^ (r >> 1 & 1) << 2) & 7) * 16; }

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

// what a thread brings of a step: eight samples of four columns of dY and of X, and their scale words
template <bool F32>
struct GradBrought { uint32_t a[8][F32 ? 4 : 2], x[8], s[8]; };

template <bool F32>
__global__ void __launch_bounds__(256, 2)
mx_grad_kernel(const char* __restrict__ dy, int64_t dy_stride, const uint8_t* __restrict__ xq, int64_t x_stride, int64_t B, int N, int K,
               int tiles_n, int tiles, int steps, int splits, float* __restrict__ out, int64_t out_stride, int64_t split_stride, int accumulate)
{
    constexpr int P = F32 ? 3 : 1, E = F32 ? 4 : 2, A = F32 ? 4 : 2;       // parts of an element of dY, its bytes, words of four of them
    __shared__ __attribute__((aligned(16))) char s_a[P * kGradN * kGradRow];
    __shared__ __attribute__((aligned(16))) char s_b[kGradK * kGradRow];
    // an XCD takes neighbouring pieces of the work: those of one stretch of samples share dY and X in its L2
    const int n_work = tiles * splits, per = (n_work + 7) / 8, work = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || work >= n_work) return;
    const int split = work / tiles, tile = work - split * tiles, tk = tile / tiles_n, tn = tile - tk * tiles_n;
    const int step0 = (int)((int64_t)steps * split / splits), step1 = (int)((int64_t)steps * (split + 1) / splits);
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, wn = wave & 1, wk = wave >> 1;
    const int c4 = (t & 31) * 4, bg = t >> 5;    // this thread's columns and its eight samples of a step
    const int n = tn * kGradN + c4, code_bytes = (K + 3) / 4 * 4, kw = min(tk * kGradK + c4, code_bytes - 4);
    // the scales of the tile's four blocks of columns are a whole word of the row (scales and zeros fill whole words)
    const int scale_word = code_bytes + tk * (kGradK / 32), scale_shift = (c4 >> 5) * 8;
    const bool whole_n = tn * kGradN + kGradN <= N;
    using Brought = GradBrought<F32>;
    auto load = [&](Brought& v, int step) {
        const int64_t b0 = (int64_t)step * kGradB;
        if (b0 + kGradB <= B && whole_n) {
            const char* d = dy + (b0 + bg * 8) * dy_stride + (int64_t)n * E;
            const uint8_t* row = xq + (b0 + bg * 8) * x_stride;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (F32) load_u32<4>(reinterpret_cast<const uint32_t*>(d + i * dy_stride), v.a[i]);
                else { const u32x2_any u = *reinterpret_cast<const u32x2_any*>(d + i * dy_stride); v.a[i][0] = u.x; v.a[i][1] = u.y; }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v.x[i] = *reinterpret_cast<const uint32_t*>(row + i * x_stride + kw);
                v.s[i] = *reinterpret_cast<const uint32_t*>(row + i * x_stride + scale_word);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t b = b0 + bg * 8 + i;
                const char* d = dy + min(b, B - 1) * dy_stride + (int64_t)n * E;
                const uint8_t* row = xq + min(b, B - 1) * x_stride;
                v.x[i] = *reinterpret_cast<const uint32_t*>(row + kw);
                v.s[i] = *reinterpret_cast<const uint32_t*>(row + scale_word);
                if (b >= B) v.x[i] = v.s[i] = 0;           // samples and columns that are not there: zeros
#pragma unroll
                for (int j = 0; j < A; ++j) v.a[i][j] = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (b < B && n + j < N) {
                        if constexpr (F32) v.a[i][j] = reinterpret_cast<const uint32_t*>(d)[j];
                        else v.a[i][j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(d)[j] << (j & 1 ? 16 : 0);
                    }
            }
        }
    };
    // X's elements as bf16 numbers, two columns of a sample to a word (in place of the codes and the scales)
    auto scale_x = [&](Brought& v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float sc = mx_scale(v.s[i] >> scale_shift & 255u);
            const uint32_t x = v.x[i];
            v.x[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, sc, false));
            v.s[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, sc, true));
        }
    };
    // column j of this thread's, its eight samples in a row
    auto turn = [](char* at, uint32_t u0, uint32_t u1, uint32_t u2, uint32_t u3, uint32_t u4, uint32_t u5, uint32_t u6, uint32_t u7, uint32_t sel) {
        uint4 w;
        w.x = __builtin_amdgcn_perm(u1, u0, sel);
        w.y = __builtin_amdgcn_perm(u3, u2, sel);
        w.z = __builtin_amdgcn_perm(u5, u4, sel);
        w.w = __builtin_amdgcn_perm(u7, u6, sel);
        *reinterpret_cast<uint4*>(at) = w;
    };
    // a quarter of a step's columns
    auto store = [&](Brought& v, int j) {
        const int at = grad_at(c4 + j, bg);
        const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
        if (j < 2) turn(s_b + at, v.x[0], v.x[1], v.x[2], v.x[3], v.x[4], v.x[5], v.x[6], v.x[7], sel);
        else turn(s_b + at, v.s[0], v.s[1], v.s[2], v.s[3], v.s[4], v.s[5], v.s[6], v.s[7], sel);
        if constexpr (!F32) {
            turn(s_a + at, v.a[0][j >> 1], v.a[1][j >> 1], v.a[2][j >> 1], v.a[3][j >> 1], v.a[4][j >> 1], v.a[5][j >> 1], v.a[6][j >> 1], v.a[7][j >> 1],
                 sel);
        } else {
#pragma unroll
            for (int p = 0; p < 3; ++p) {                  // the upper half of what is left: its next eight digits
                turn(s_a + p * kGradN * kGradRow + at, v.a[0][j], v.a[1][j], v.a[2][j], v.a[3][j], v.a[4][j], v.a[5][j], v.a[6][j], v.a[7][j], 0x07060302u);
#pragma unroll
                for (int i = 0; i < 8 && p < 2; ++i) v.a[i][j] = __float_as_uint(__uint_as_float(v.a[i][j]) - __uint_as_float(v.a[i][j] & 0xFFFF0000u));
            }
        }
    };
    f32x16 acc[2][2] = {};
    const int row_a = wn * 64 + (lane & 31), row_b = wk * 64 + (lane & 31);
    auto multiply = [&](int kk) {
        const int c = kk * 2 + (lane >> 5);
        bf16x8 fb[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) fb[j] = *reinterpret_cast<const bf16x8*>(s_b + grad_at(row_b, c) + j * 32 * kGradRow);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bf16x8 fa = *reinterpret_cast<const bf16x8*>(s_a + p * kGradN * kGradRow + grad_at(row_a, c) + i * 32 * kGradRow);
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa, fb[j], acc[i][j], 0, 0, 0);
            }
    };
    // a step on its way while one is multiplied; the other blocks of the compute unit fill the pauses
    Brought v;
    if (step0 < step1) load(v, step0);
    for (int step = step0; step < step1; ++step) {
        scale_x(v);
#pragma unroll
        for (int j = 0; j < 4; ++j) store(v, j);
        __syncthreads();
        if (step + 1 < step1) load(v, step + 1);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) multiply(kk);
        __syncthreads();
    }
    float* o = out + split * split_stride;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int kc = tk * kGradK + wk * 64 + j * 32 + (lane & 31);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int nr = tn * kGradN + wn * 64 + i * 32 + (e >> 2) * 8 + (lane >> 5) * 4 + (e & 3);
                if (nr < N && kc < K) {
                    float* at = o + (int64_t)nr * out_stride + kc;
                    *at = accumulate ? *at + acc[i][j][e] : acc[i][j][e];
                }
            }
        }
}

// the stretches' sums, added up in their order
__global__ void __launch_bounds__(NT)
mx_grad_join_kernel(const float* __restrict__ part, int64_t ld, int64_t split_stride, int splits, int K, int64_t items, float* __restrict__ dw,
                    int64_t dw_stride, int accumulate)
{
    const int64_t per_row = ld / 4;
    for (int64_t it = (int64_t)blockIdx.x * NT + threadIdx.x; it < items; it += (int64_t)gridDim.x * NT) {
        const int64_t n = it / per_row;
        const int k = (int)(it - n * per_row) * 4;
        const float* p = part + n * ld + k;
        f32x4 v = *reinterpret_cast<const f32x4*>(p);
#pragma unroll 8
        for (int s = 1; s < splits; ++s) v += *reinterpret_cast<const f32x4*>(p + s * split_stride);
        float* o = dw + n * dw_stride + k;
        const int m = K - k;
        if (m >= 4) {
            if (accumulate) v += *reinterpret_cast<const f32x4*>(o);
            *reinterpret_cast<f32x4*>(o) = v;
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (j < m) o[j] = accumulate ? o[j] + v[j] : v[j];
        }
    }
}
