// y = Q(x) W^T + bias, both operands in 4 bits.
// Part of pk_mx.hip: included there, in this order, inside its anonymous namespace.

// ---------------------------------------------------------------------------
// x is rounded first, into the workspace, in the product's own layout: codes [M][kp / 2] and scale bytes [M][kp / 32], K filled up
// with zeros (scale 1) to whole steps kp.  A block then takes kLinM x kLinN of y, kLinK of K a step: codes and scales go to
// LDS through registers, the next step's on their way while this one is multiplied.  A scaled product of 16 x 16 x 128 takes of every
// lane 16 bytes and a scale: row (column) l % 16 and of the 128 the block l / 16.  W is its first operand, so that a lane's four results are
// neighbours in a row of y.  Where the tiles are too few for the chip, K is cut into stretches whose sums meet in a second
// launch, in their order.
// 2048 x 12000 -> 1024: rounding 17.5 us (98 MB read, 13 written: 6.3 TB/s), product 24.6 (2.0 PFLOP/s: a step's stores to LDS and its
// barriers, not the matrix unit), joining four stretches 9.2.  8192 x 832 -> 1024: rounding 7.0, product 14.7 (four steps a tile: its first
// loads and 17 MB of y).
// ---------------------------------------------------------------------------
constexpr int kLinM = 128, kLinN = 128, kLinK = 256;
constexpr int kLinRow = kLinK / 2;               // bytes of a row's codes in LDS
constexpr int kLinScales = 16;                   // steps whose scales are in LDS at a time: 128 bytes a row
// Steps of a stretch, at least: its tile is written and read once more.  2048 x 12000 -> 1024 takes 53 us in four stretches and 68 in one,
// 512 x 12000 -> 256 23 and 54; stretches of two steps cost 2048 x 2048 -> 1024 26 us instead of 18.
constexpr int kLinStretch = 6;

// Few rows of x, up to 16 of kLinFew elements together, take one launch (K 832, N 1024, 1 and 16 rows: 4.2 and 5.1 us, by tiles 10.5 and
// 10.8; K 3840, 16 rows 10.7 and 15.0; K 6000 and 16 rows 15.3 both; K 12000, N 1024, 1, 4, 8 rows 13.8 17.7 21.5, by tiles 16.3 16.4 16.7:
// each block reads all of x).  What would be 2^32 threads and more goes by tiles too.
constexpr int64_t kLinFew = 1 << 16;
inline int linear_few_waves(int64_t K) { return (int)std::min<int64_t>(16, std::max<int64_t>(1, (K + 255) / 256)); }
inline bool linear_few(int64_t M, int64_t N, int64_t K)
{
    return M <= 16 && M * K <= kLinFew && (N + 15) / 16 * (64 * linear_few_waves(K)) < kLaunchThreads;
}
struct LinearLayout { int64_t kp, tiles_m, tiles_n, steps, splits, ld; size_t scales, parts, total; };
inline LinearLayout linear_layout(int64_t M, int64_t N, int64_t K)
{
    auto pad = [](int64_t b) { return (size_t)((b + 255) / 256 * 256); };
    LinearLayout L;
    L.steps = (K + kLinK - 1) / kLinK;
    L.kp = L.steps * kLinK;
    L.tiles_m = (M + kLinM - 1) / kLinM;
    L.tiles_n = (N + kLinN - 1) / kLinN;
    const int64_t tiles = std::max<int64_t>(1, L.tiles_m * L.tiles_n);
    L.splits = std::max<int64_t>(1, std::min<int64_t>(L.steps / kLinStretch, 512 / tiles));
    L.ld = (N + 3) / 4 * 4;
    L.scales = pad(M * (L.kp / 2));
    L.parts = L.scales + pad(M * (L.kp / 32));
    L.total = linear_few(M, N, K) ? kAlign : std::max<size_t>(kAlign, L.parts + (L.splits > 1 ? pad(L.splits * M * L.ld * 4) : 0));
    return L;
}

// x's rows in the layout above; a thread takes eight columns as in mx_quantize_kernel, groups: of kp columns
template <bool BF16>
__global__ void __launch_bounds__(NT)
mx_linear_round_kernel(const char* __restrict__ src, int64_t src_stride, uint32_t cols, RowGroups groups, uint32_t* __restrict__ codes,
                       uint8_t* __restrict__ scales, int64_t items)
{
    for (int64_t base = (int64_t)blockIdx.x * NT; base < items; base += (int64_t)gridDim.x * NT) {
        if (base + threadIdx.x >= items) break;
        uint32_t g;
        const int64_t r = groups.row(base, threadIdx.x, g);
        float x[8];
        load_f8<BF16>(src + r * src_stride + (int64_t)g * (BF16 ? 16 : 32), (int)cols - (int)(8 * g), x);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
        m = max(m, (uint32_t)__shfl_xor((int)m, 1));
        m = max(m, (uint32_t)__shfl_xor((int)m, 2));
        const uint32_t s = mx_scale_byte<PK_MXFP4>(m);
        uint32_t w[1];
        mx_encode8<PK_MXFP4>(x, s, w);
        const int64_t at = base + threadIdx.x;             // (rows follow one another without gaps)
        codes[at] = w[0];
        if ((g & 3) == 0) scales[at >> 2] = (uint8_t)s;
    }
}

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4m __attribute__((ext_vector_type(4)));

// where chunk c (16 bytes) of row r stands: the eight chunks of a row trade places, so that neighbouring rows' are on different banks
__device__ __forceinline__ int lin_at(int r, int c) { return r * kLinRow + ((c ^ r) & 7) * 16; }

// four neighbours in a row of y
template <bool BF16>
__device__ __forceinline__ void lin_store(char* y, int64_t at, int left, const f32x4m& v)
{
    if constexpr (BF16) {
        uint16_t* o = reinterpret_cast<uint16_t*>(y) + at;
        const uint32_t a = pack_bf16(v[0], v[1]), b = pack_bf16(v[2], v[3]);
        if (left >= 4) {
            u32x2_b2 u;
            u.x = a; u.y = b;
            *reinterpret_cast<u32x2_b2*>(o) = u;
        } else {
            o[0] = (uint16_t)a;
            if (left > 1) o[1] = (uint16_t)(a >> 16);
            if (left > 2) o[2] = (uint16_t)b;
        }
    } else {
        float* o = reinterpret_cast<float*>(y) + at;
        if (left >= 4) {
            f32x4 u;
            u.x = v[0]; u.y = v[1]; u.z = v[2]; u.w = v[3];
            *reinterpret_cast<f32x4*>(o) = u;
        } else {
            o[0] = v[0];
            if (left > 1) o[1] = v[1];
            if (left > 2) o[2] = v[2];
        }
    }
}

template <bool BF16>
__global__ void __launch_bounds__(256)
mx_linear_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const uint8_t* __restrict__ wq, int64_t w_stride, int M, int N, int K,
                 int tiles_n, int tiles, int steps, int splits, const float* __restrict__ bias, char* __restrict__ y, int64_t y_stride, int64_t split_stride)
{
    __shared__ __attribute__((aligned(16))) char s_all[4][128 * 128];
    static_assert(kLinM == 128 && kLinN == 128 && kLinRow == 128 && 8 * kLinScales == 128, "a row's codes and its scales are 128 bytes each");
    char *s_x = s_all[0], *s_w = s_all[1], *s_sx = s_all[2], *s_sw = s_all[3];
    // an XCD takes neighbouring pieces of the work: those of one stretch and one stretch of rows share x in its L2
    const int n_work = tiles * splits, per = (n_work + 7) / 8, work = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || work >= n_work) return;
    const int split = work / tiles, tile = work - split * tiles, tm = tile / tiles_n, tn = tile - tm * tiles_n;
    const int step0 = (int)((int64_t)steps * split / splits), step1 = (int)((int64_t)steps * (split + 1) / splits);
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, wm = wave & 1, wn = wave >> 1, r = lane & 15, q = lane >> 4;
    const int kp = steps * kLinK, words = (K + 7) / 8, blocks = (K + 31) / 32;
    // what this thread brings of a step: chunk c of rows t / 8, t / 8 + 32 ...
    const int c = t & 7, row = t >> 3;
    uint32_t x[4][4], w[4][4];
    // (a tile's rows are less than 2^31 bytes apart: kMxDepthMax)
    const uint8_t* xt = codes + (int64_t)tm * kLinM * (kp / 2);
    const uint8_t* wt = wq + (int64_t)tn * kLinN * w_stride;
    uint32_t xo[4], wo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        xo[i] = (uint32_t)min(row + 32 * i, M - 1 - tm * kLinM) * (uint32_t)(kp / 2) + 16 * c;
        wo[i] = (uint32_t)min(row + 32 * i, N - 1 - tn * kLinN) * (uint32_t)w_stride + 16 * c;
    }
    auto load = [&](int step) {
        const uint8_t *xb = xt + (int64_t)step * kLinRow, *wb = wt + (int64_t)step * kLinRow;
#pragma unroll
        for (int i = 0; i < 4; ++i) load_u32<4>(reinterpret_cast<const uint32_t*>(xb + xo[i]), x[i]);
        if ((step + 1) * (kLinK / 8) <= words) {
#pragma unroll
            for (int i = 0; i < 4; ++i) load_u32<4>(reinterpret_cast<const uint32_t*>(wb + wo[i]), w[i]);
        } else {                                           // the last step of a row that does not fill it
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    w[i][j] = 0;
                    if (step * (kLinK / 8) + 4 * c + j < words) w[i][j] = reinterpret_cast<const uint32_t*>(wb + wo[i])[j];
                }
        }
    };
    auto store = [&]() {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<uint4*>(s_x + lin_at(row + 32 * i, c)) = make_uint4(x[i][0], x[i][1], x[i][2], x[i][3]);
            *reinterpret_cast<uint4*>(s_w + lin_at(row + 32 * i, c)) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
        }
    };
    // The scales of kLinScales steps, in whole lines: eight bytes of a row a step are a request each, and an L1 has few on their way.
    // Step i's eight bytes of row r stand at place i ^ r of the row.
    auto load_scales = [&](int first) {
        const int word = 2 * first + (t & 31);
        const bool in_x = word < kp / 128, in_w = 4 * word < blocks;
#pragma nounroll
        for (int h = 0; h < 16; h += 8) {
            uint32_t v[8], u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int rr = (t >> 5) + 8 * (h + i);
                v[i] = u[i] = 0;
                if (in_x) v[i] = *reinterpret_cast<const uint32_t*>(scales + (int64_t)min(tm * kLinM + rr, M - 1) * (kp / 32) + 4 * word);
                if (in_w) u[i] = *reinterpret_cast<const uint32_t*>(wt + (uint32_t)min(rr, N - 1 - tn * kLinN) * (uint32_t)w_stride + 4 * (words + word));
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int rr = (t >> 5) + 8 * (h + i), at = rr * 8 * kLinScales + ((((t & 31) >> 1) ^ rr) & (kLinScales - 1)) * 8 + (t & 1) * 4;
                *reinterpret_cast<uint32_t*>(s_sx + at) = v[i];
                *reinterpret_cast<uint32_t*>(s_sw + at) = u[i];
            }
        }
    };
    f32x4m acc[4][4] = {};                                 // [columns of y][rows of y]
    if (step0 < step1) load(step0);
    for (int step = step0; step < step1; ++step) {
        const int place = (step - step0) & (kLinScales - 1);
        if (place == 0) load_scales(step);
        store();
        __syncthreads();
        if (step + 1 < step1) load(step + 1);
        uint2 fsx[4], fsw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fsx[i] = *reinterpret_cast<const uint2*>(s_sx + (wm * 64 + i * 16 + r) * 8 * kLinScales + (place ^ r) * 8);
            fsw[i] = *reinterpret_cast<const uint2*>(s_sw + (wn * 64 + i * 16 + r) * 8 * kLinScales + (place ^ r) * 8);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x8 fx[4], fw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 a = *reinterpret_cast<const uint4*>(s_x + lin_at(wm * 64 + i * 16 + r, 4 * h + q));
                const uint4 b = *reinterpret_cast<const uint4*>(s_w + lin_at(wn * 64 + i * 16 + r, 4 * h + q));
                fx[i] = i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
                fw[i] = i32x8{(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[i], fx[j], acc[i][j], 4, 4, 0, (int)((h ? fsw[i].y : fsw[i].x) >> (8 * q)),
                                                                                0, (int)((h ? fsx[j].y : fsx[j].x) >> (8 * q)));
        }
        __syncthreads();
    }
    // y by way of LDS, so that a wavefront writes whole rows of the tile (16 rows of 32 bytes at a time: 6 us more for 17 MB); the
    // 32 chunks of a row trade places
    y += split * split_stride;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int m = wm * 64 + j * 16 + r, chunk = wn * 16 + i * 4 + q;
            *reinterpret_cast<f32x4m*>(s_all[0] + m * 512 + (chunk ^ (m & 31)) * 16) = acc[i][j];
        }
    __syncthreads();
    const int chunk = t & 31, n = tn * kLinN + 4 * chunk;
    if (n >= N) return;
    f32x4m add = {0.f, 0.f, 0.f, 0.f};
    if (bias)
#pragma unroll
        for (int e = 0; e < 4; ++e) add[e] = bias[min(n + e, N - 1)];
#pragma unroll 4
    for (int k = 0; k < 16; ++k) {
        const int row_y = (t >> 5) + 8 * k, m = tm * kLinM + row_y;
        if (m < M) lin_store<BF16>(y, m * y_stride + n, N - n, *reinterpret_cast<const f32x4m*>(s_all[0] + row_y * 512 + (chunk ^ (row_y & 31)) * 16) + add);
    }
}

// the stretches' sums, added up in their order, and the bias
template <bool BF16>
__global__ void __launch_bounds__(NT)
mx_linear_join_kernel(const float* __restrict__ part, int64_t ld, int64_t split_stride, int splits, int N, int64_t items, const float* __restrict__ bias,
                      char* __restrict__ y, int64_t y_stride)
{
    const int64_t per_row = ld / 4;
    for (int64_t it = (int64_t)blockIdx.x * NT + threadIdx.x; it < items; it += (int64_t)gridDim.x * NT) {
        const int64_t m = it / per_row;
        const int n = (int)(it - m * per_row) * 4;
        const float* p = part + m * ld + n;
        f32x4 v = *reinterpret_cast<const f32x4*>(p);
        for (int s = 1; s < splits; ++s) v += *reinterpret_cast<const f32x4*>(p + s * split_stride);
        f32x4m u = {v.x, v.y, v.z, v.w};
        if (bias)
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] += bias[min(n + e, N - 1)];
        lin_store<BF16>(y, m * y_stride + n, N - n, u);
    }
}

// Few rows of x: a block takes 16 columns of y and all of K, its wavefronts a stretch each; x is rounded in registers, a lane
// a block of 32 of its row, just as the product wants it.  The stretches' sums meet in LDS, in their order.
template <bool XBF, bool YBF>
__global__ void __launch_bounds__(1024)
mx_linear_few_kernel(const char* __restrict__ x, int64_t x_stride, int M, const uint8_t* __restrict__ wq, int64_t w_stride, int N, int K,
                     const float* __restrict__ bias, char* __restrict__ y, int64_t y_stride)
{
    __shared__ float s_part[16][16][17];                   // [wavefront][row of x][column]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, r = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * 16, words = (K + 7) / 8, blocks = (K + 31) / 32, steps = (blocks + 3) / 4;
    const uint8_t* wr = wq + (int64_t)min(n0 + r, N - 1) * w_stride;
    const char* xr = x + (int64_t)min(r, M - 1) * x_stride;
    f32x4m acc = {0.f, 0.f, 0.f, 0.f};
    struct Step { uint32_t w[4], s; float x[4][8]; };
    // WHOLE: the step lies inside the rows.  (Lanes of rows that are not there read the last one; what they give is not written.)
    auto load = [&](Step& v, int step, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        const int kb = 4 * step + q;
        if (WHOLE || 4 * kb + 4 <= words) {
            load_u32<4>(reinterpret_cast<const uint32_t*>(wr) + 4 * kb, v.w);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) { v.w[i] = 0; if (4 * kb + i < words) v.w[i] = reinterpret_cast<const uint32_t*>(wr)[4 * kb + i]; }
        }
        v.s = 127;
        if (WHOLE || kb < blocks) v.s = wr[4 * words + kb];
#pragma unroll
        for (int i = 0; i < 4; ++i) load_f8<XBF>(xr + (int64_t)(32 * kb + 8 * i) * (XBF ? 2 : 4), WHOLE ? 8 : K - 32 * kb - 8 * i, v.x[i]);
    };
    auto multiply = [&](const Step& v) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v.x[i][j]) & 0x7FFFFFFFu);
        const uint32_t s = mx_scale_byte<PK_MXFP4>(m);
        const i32x8 a = {(int)v.w[0], (int)v.w[1], (int)v.w[2], (int)v.w[3], 0, 0, 0, 0};
        i32x8 b = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t w[1];
            mx_encode8<PK_MXFP4>(v.x[i], s, w);
            b[i] = (int)w[0];
        }
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, 0, (int)v.s, 0, (int)s);
    };
    const int first = steps * wave / waves, end = steps * (wave + 1) / waves, whole = min(end, K / 128);
    int step = first;
    for (; step + 2 <= whole; step += 2) {
        Step v0, v1;
        load(v0, step, std::true_type{});
        load(v1, step + 1, std::true_type{});
        multiply(v0);
        multiply(v1);
    }
    for (; step < end; ++step) {
        Step v;
        load(v, step, std::false_type{});
        multiply(v);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s_part[wave][r][4 * q + i] = acc[i];
    __syncthreads();
    for (int at = threadIdx.x; at < 16 * 16; at += blockDim.x) {
        const int m = at >> 4, c = at & 15, n = n0 + c;
        if (m >= M || n >= N) continue;
        float v = s_part[0][m][c];
        for (int w = 1; w < waves; ++w) v += s_part[w][m][c];
        if (bias) v += bias[n];
        if constexpr (YBF) reinterpret_cast<uint16_t*>(y)[m * y_stride + n] = (uint16_t)pack_bf16(v, 0.f);
        else reinterpret_cast<float*>(y)[m * y_stride + n] = v;
    }
}
