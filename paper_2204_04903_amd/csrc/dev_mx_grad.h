// dW (+)= dY^T X, X an 8-bit checkpoint.
// Part of pk_mx.hip: included there, in this order, inside its anonymous namespace.

// ---------------------------------------------------------------------------
// The sum runs over the samples, which are the rows of both operands, while a lane of a matrix instruction wants eight
// consecutive samples of one column: a thread loads eight rows of four columns, and turns them over in registers on the way to
// LDS.  X's elements become bf16 there (four digits and a power of two: exact, from 2^-133 on, the smallest bf16 number); of an
// fp32 dY every element becomes three bf16 numbers whose sum it is (8 + 8 + 8 digits, cut off, not rounded; digits below
// 2^-133 are lost), so that all products are exact and what is lost is what fp32 additions lose.
// A block takes kGradN x kGradK elements of dW and a stretch of the samples, kGradB a step; the stretches' sums meet in a
// second launch in their order, so that a result does not depend on which block came first.
// bf16, 8192 samples, 832 x 1024: 29 us (0.48 PFLOP/s: narrow loads, turning over and LDS, the matrix unit would take 10) and 6.3 to
// join nine stretches.  fp32, 512 samples, 12000 x 1024, added to dW: 45 us (0.84 PFLOP/s of bf16 products).
// ---------------------------------------------------------------------------
constexpr int kGradN = 128, kGradK = 128, kGradB = 64;
// Blocks that the stretches are cut for, two a compute unit: 8192 samples, 832 x 1024, bf16, 39.9 us; 256 blocks 47.8, one stretch 140.
constexpr int64_t kGradBlocks = 512;
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

struct GradJob {
    const char* dy; int64_t dy_stride; const uint8_t* xq; int64_t x_stride, B; int N, K, tiles_n, tiles, steps, splits;
    float* out; int64_t out_stride, split_stride; int accumulate;
};
// A block's work.  An XCD takes neighbouring pieces: those of one stretch of samples share dY and X in its L2.
struct GradWork {
    int split, tk, tn, step0, step1;
    __device__ __forceinline__ explicit GradWork(const GradJob& g)
    {
        const int n_work = g.tiles * g.splits, per = (n_work + 7) / 8, work = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
        if ((int)(blockIdx.x >> 3) >= per || work >= n_work) { split = -1; return; }
        split = work / g.tiles;
        const int tile = work - split * g.tiles;
        tk = tile / g.tiles_n; tn = tile - tk * g.tiles_n;
        step0 = (int)((int64_t)g.steps * split / g.splits); step1 = (int)((int64_t)g.steps * (split + 1) / g.splits);
    }
};

// eight samples of one column, a word holds it and a neighbour of each: as the matrix unit wants them
__device__ __forceinline__ uint4 grad_turn(uint32_t u0, uint32_t u1, uint32_t u2, uint32_t u3, uint32_t u4, uint32_t u5, uint32_t u6, uint32_t u7, uint32_t sel)
{
    return make_uint4(__builtin_amdgcn_perm(u1, u0, sel), __builtin_amdgcn_perm(u3, u2, sel), __builtin_amdgcn_perm(u5, u4, sel), __builtin_amdgcn_perm(u7, u6, sel));
}
constexpr uint32_t kLowHalves = 0x05040100u, kHighHalves = 0x07060302u;

// A matrix from row b0 on as a buffer: a row's distance is then a scalar of the access (as plain loads, the addresses of a step's
// forty accesses took 160 registers).  Nothing is read behind the last row: its end is not what keeps an access inside.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t grad_rows(const void* p, int64_t stride, int64_t b0)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(p) + b0 * stride), 0, 0x7FFFFFFF, 0x00020000);
}
// words of eight rows from `first` on, at byte `at` of each, zeros for rows that are not among the n there
__device__ __forceinline__ void grad_words(__amdgpu_buffer_rsrc_t rows, int first, int at, int stride, int64_t n, bool whole, uint32_t (&v)[8])
{
    if (whole) {
        const int place = first * stride + at;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_amdgcn_raw_buffer_load_b32(rows, place, i * stride, 0);
    } else {
        asm volatile("" : "+v"(first));                    // (formed here, where it is wanted once, not kept in registers all along)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = 0;
            if (first + i < n) v[i] = __builtin_amdgcn_raw_buffer_load_b32(rows, (first + i) * stride + at, 0, 0);
        }
    }
}

// What a thread brings of X in a step: eight samples of four columns and their scale words.
struct GradX {
    uint32_t x[8], s[8];
    __device__ __forceinline__ void load(const GradJob& g, const GradWork& w, int step)
    {
        const int t = threadIdx.x, code_bytes = (g.K + 3) / 4 * 4;
        const int64_t b0 = (int64_t)step * kGradB, n = g.B - b0;
        const auto rows = grad_rows(g.xq, g.x_stride, b0);
        // (columns that are not there: any that are; the scales of the tile's four blocks are a whole word of the row)
        grad_words(rows, (t >> 5) * 8, min(w.tk * kGradK + (t & 31) * 4, code_bytes - 4), (int)g.x_stride, n, n >= kGradB, x);
        grad_words(rows, (t >> 5) * 8, code_bytes + w.tk * (kGradK / 32), (int)g.x_stride, n, n >= kGradB, s);
    }
    // the elements as bf16 numbers, two columns of a sample to a word (in place of the codes and the scales)
    __device__ __forceinline__ void scale()
    {
        const int shift = ((threadIdx.x & 31) >> 3) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float sc = mx_scale(s[i] >> shift & 255u);
            const uint32_t v = x[i];
            x[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, sc, false));
            s[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, sc, true));
        }
    }
    // column j of the thread's four
    __device__ __forceinline__ void store(char* lds, int j) const
    {
        const uint32_t(&u)[8] = j < 2 ? x : s;
        *reinterpret_cast<uint4*>(lds + grad_at((threadIdx.x & 31) * 4 + j, threadIdx.x >> 5)) =
            grad_turn(u[0], u[1], u[2], u[3], u[4], u[5], u[6], u[7], j & 1 ? kHighHalves : kLowHalves);
    }
};

// 32 x 32 of the result: lane l has column l % 32, rows 8 (e / 4) + 4 (l / 32) + e % 4
__device__ __forceinline__ void grad_write(const GradJob& g, const GradWork& w, int n0, int k0, const f32x16& acc)
{
    const int lane = threadIdx.x & 63, kc = k0 + (lane & 31);
    float* o = g.out + w.split * g.split_stride + kc;
    f32x16 old = {};
    if (kc >= g.K) return;
    if (g.accumulate) {                                    // (all asked for before the first is written: they are not known to be apart)
#pragma unroll
        for (int e = 0; e < 16; ++e) old[e] = o[(int64_t)min(n0 + (e >> 2) * 8 + (lane >> 5) * 4 + (e & 3), g.N - 1) * g.out_stride];
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int nr = n0 + (e >> 2) * 8 + (lane >> 5) * 4 + (e & 3);
        if (nr < g.N) o[(int64_t)nr * g.out_stride] = acc[e] + old[e];
    }
}

// dY in bf16: both operands by way of LDS, a wavefront takes 64 x 64.  A step on its way while one is multiplied; the other block
// of the compute unit fills the pauses.  (dY from memory to registers, as below, takes 46.9 us instead of 40.5 with the joining: with one
// product instead of three for what a lane has read, its loads are what is waited for.)
__global__ void __launch_bounds__(256, 2)
mx_grad_bf16_kernel(GradJob g)
{
    __shared__ __attribute__((aligned(16))) char s_a[kGradN * kGradRow], s_b[kGradK * kGradRow];
    const GradWork w(g);
    if (w.split < 0) return;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, wn = wave & 1, wk = wave >> 1;
    const int c4 = (t & 31) * 4, bg = t >> 5, n = w.tn * kGradN + c4;      // this thread's columns and its eight samples of a step
    const bool whole_n = w.tn * kGradN + kGradN <= g.N;
    GradX x;
    uint32_t a[8][2];
    auto load = [&](int step) {
        const int64_t b0 = (int64_t)step * kGradB;
        if (b0 + kGradB <= g.B && whole_n) {
            const char* d = g.dy + (b0 + bg * 8) * g.dy_stride + (int64_t)n * 2;
#pragma unroll
            for (int i = 0; i < 8; ++i) { const u32x2_any u = *reinterpret_cast<const u32x2_any*>(d + i * g.dy_stride); a[i][0] = u.x; a[i][1] = u.y; }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t b = b0 + bg * 8 + i;
                const char* d = g.dy + min(b, g.B - 1) * g.dy_stride + (int64_t)n * 2;
                a[i][0] = a[i][1] = 0;                     // samples and columns that are not there: zeros
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (b < g.B && n + j < g.N) a[i][j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(d)[j] << (j & 1 ? 16 : 0);
            }
        }
        x.load(g, w, step);
    };
    f32x16 acc[2][2] = {};
    if (w.step0 < w.step1) load(w.step0);
    for (int step = w.step0; step < w.step1; ++step) {
        x.scale();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x.store(s_b, j);
            const int h = j >> 1;
            *reinterpret_cast<uint4*>(s_a + grad_at(c4 + j, bg)) =
                grad_turn(a[0][h], a[1][h], a[2][h], a[3][h], a[4][h], a[5][h], a[6][h], a[7][h], j & 1 ? kHighHalves : kLowHalves);
        }
        __syncthreads();
        if (step + 1 < w.step1) load(step + 1);
#pragma unroll
        for (int kk = 0; kk < kGradB / 16; ++kk) {
            const int c = kk * 2 + (lane >> 5);
            bf16x8 fb[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) fb[j] = *reinterpret_cast<const bf16x8*>(s_b + grad_at(wk * 64 + (lane & 31), c) + j * 32 * kGradRow);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bf16x8 fa = *reinterpret_cast<const bf16x8*>(s_a + grad_at(wn * 64 + (lane & 31), c) + i * 32 * kGradRow);
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa, fb[j], acc[i][j], 0, 0, 0);
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) grad_write(g, w, w.tn * kGradN + wn * 64 + i * 32, w.tk * kGradK + wk * 64 + j * 32, acc[i][j]);
}

// dY in fp32: only X goes by way of LDS.  A wavefront takes 32 columns of dY and all of X's 128, so that no two read the same of dY, and a
// lane reads just what it holds as an operand, eight samples of one column: 32 lanes a line.  The three parts are made in
// registers; a quarter of a step is asked for again, for the next step, as soon as its parts are made.
__global__ void __launch_bounds__(256, 3)
mx_grad_f32_kernel(GradJob g)
{
    __shared__ __attribute__((aligned(16))) char s_b[2][kGradK * kGradRow];
    const GradWork w(g);
    if (w.split < 0) return;
    const int lane = threadIdx.x & 63, n0 = w.tn * kGradN + (threadIdx.x >> 6) * 32, h8 = (lane >> 5) * 8;
    const int at = 4 * min(n0 + (lane & 31), g.N - 1);
    GradX x;
    uint32_t a[4][8];
    auto load = [&](int step, int kk) {
        const int64_t b0 = (int64_t)step * kGradB + kk * 16, n = g.B - b0;
        grad_words(grad_rows(g.dy, g.dy_stride, b0), h8, at, (int)g.dy_stride, n, n >= 16, a[kk]);
    };
    f32x16 acc[4] = {};
    if (w.step0 < w.step1) {
        x.load(g, w, w.step0);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) load(w.step0, kk);
    }
    for (int step = w.step0; step < w.step1; ++step) {
        char* lds = s_b[(step - w.step0) & 1];             // (two steps in LDS: one barrier is enough)
        x.scale();
#pragma unroll
        for (int j = 0; j < 4; ++j) x.store(lds, j);
        __syncthreads();
        const bool more = step + 1 < w.step1;
        if (more) x.load(g, w, step + 1);
#pragma unroll
        for (int kk = 0; kk < kGradB / 16; ++kk) {
            bf16x8 fa[3];
#pragma unroll
            for (int p = 0; p < 3; ++p) {                  // the upper half of what is left: its next eight digits
                fa[p] = __builtin_bit_cast(bf16x8, grad_turn(a[kk][0], a[kk][1], a[kk][2], a[kk][3], a[kk][4], a[kk][5], a[kk][6], a[kk][7], kHighHalves));
#pragma unroll
                for (int i = 0; i < 8 && p < 2; ++i) {
                    const float v = __uint_as_float(a[kk][i]), rest = v - __uint_as_float(a[kk][i] & 0xFFFF0000u);
                    a[kk][i] = __float_as_uint(p == 0 && __builtin_isinf(v) ? 0.f : rest);   // (nothing is left of an infinity)
                }
            }
            if (more) load(step + 1, kk);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x8 fb = *reinterpret_cast<const bf16x8*>(lds + grad_at(lane & 31, kk * 2 + (lane >> 5)) + j * 32 * kGradRow);
#pragma unroll
                for (int p = 0; p < 3; ++p) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[p], fb, acc[j], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);             // (else all quarters' parts are made first, in registers that are not there)
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) grad_write(g, w, n0, w.tk * kGradK + j * 32, acc[j]);
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
