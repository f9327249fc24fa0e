// Rounding to microscaled rows and reading them back.
// Part of pk_mx.hip: included there, in this order, inside its anonymous namespace.

// ---------------------------------------------------------------------------
// A thread takes eight columns, so that a block of 32 is four neighbouring lanes: the largest magnitude of the block is two
// exchanges away.  Both kernels move bytes and little else: what bounds them is HBM and the cache behind it.  2048 x 12000 fp32 to 8
// bits 18.8 us (6.6 TB/s), back to bf16 12.6 (6.0); 1 M x 32 bf16 to 4 bits 19.7 (4.2), back to fp32 24.2 (6.1).
// ---------------------------------------------------------------------------
struct RowGroups {                   // a row's groups of eight columns, whole blocks of four
    uint32_t n, magic;               // magic: floor(2^32 / n) + 1, exact for the quotients below 512 / n that are asked of it
    explicit RowGroups(int64_t cols) : n((uint32_t)((cols + 31) / 32 * 4)), magic((uint32_t)(((uint64_t)1 << 32) / n) + 1) {}
    // item base + i (i < 256, base uniform): its row, and its group in g
    __device__ __forceinline__ int64_t row(int64_t base, uint32_t i, uint32_t& g) const
    {
        const int64_t row0 = (int64_t)((uint64_t)base / n);
        const uint32_t off = (uint32_t)(base - row0 * n) + i;
        const uint32_t dr = n >= 256 ? (off >= n ? 1u : 0u) : __umulhi(off, magic);
        g = off - dr * n;
        return row0 + dr;
    }
};
// a launch has fewer threads than this; blocks of 256, dealt out in eights
constexpr int64_t kLaunchThreads = (int64_t)1 << 32, kLaunchBlocks = kLaunchThreads / 256 - 8;
inline unsigned mx_blocks_for(int64_t items)
{
    return (unsigned)std::min<int64_t>((items + NT - 1) / NT, (int64_t)1 << 20);
}

template <int FMT, bool BF16>
__global__ void __launch_bounds__(NT)
mx_quantize_kernel(const char* __restrict__ src, int64_t src_stride, uint32_t cols, RowGroups groups, uint8_t* __restrict__ rows,
                   int64_t row_stride, int64_t items)
{
    constexpr int W = FMT == PK_MXFP4 ? 1 : 2;             // words of eight columns
    for (int64_t base = (int64_t)blockIdx.x * NT; base < items; base += (int64_t)gridDim.x * NT) {
        if (base + threadIdx.x >= items) break;            // (items are whole blocks: a block's four lanes go together)
        uint32_t g;
        const int64_t r = groups.row(base, threadIdx.x, g);
        const int n = (int)cols - (int)(8 * g);
        float x[8];
        load_f8<BF16>(src + r * src_stride + (int64_t)g * (BF16 ? 16 : 32), n, x);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
        m = max(m, (uint32_t)__shfl_xor((int)m, 1));
        m = max(m, (uint32_t)__shfl_xor((int)m, 2));
        const uint32_t s = mx_scale_byte<FMT>(m);
        uint32_t w[W];
        mx_encode8<FMT>(x, s, w);
        if (FMT == PK_MXFP8 && n < 8) {                    // (a bad block's codes are not zeros: none behind the last column)
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = n >= 4 * i + 4 ? w[i] : n > 4 * i ? w[i] & ((1u << 8 * (n - 4 * i)) - 1u) : 0u;
        }
        uint8_t* row = rows + r * row_stride;
        const uint32_t words = FMT == PK_MXFP4 ? (cols + 7) / 8 : (cols + 3) / 4;
        uint32_t* at = reinterpret_cast<uint32_t*>(row);
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (g * W + i < words) at[g * W + i] = w[i];
        if ((g & 3) == 0) {
            const uint32_t blocks = groups.n / 4, b = g / 4;
            uint8_t* sc = row + words * 4;
            sc[b] = (uint8_t)s;
            if (b + 1 == blocks)
                for (uint32_t i = blocks; i & 3; ++i) sc[i] = 0;       // the row's last word
        }
    }
}

template <int FMT, bool BF16>
__global__ void __launch_bounds__(NT)
mx_dequantize_kernel(const uint8_t* __restrict__ rows, int64_t row_stride, uint32_t cols, RowGroups groups, char* __restrict__ dst,
                     int64_t dst_stride, int64_t items)
{
    constexpr int W = FMT == PK_MXFP4 ? 1 : 2;
    for (int64_t base = (int64_t)blockIdx.x * NT; base < items; base += (int64_t)gridDim.x * NT) {
        if (base + threadIdx.x >= items) break;
        uint32_t g;
        const int64_t r = groups.row(base, threadIdx.x, g);
        const int n = (int)cols - (int)(8 * g);
        if (n <= 0) continue;
        const uint8_t* row = rows + r * row_stride;
        const uint32_t words = FMT == PK_MXFP4 ? (cols + 7) / 8 : (cols + 3) / 4;
        const uint32_t* at = reinterpret_cast<const uint32_t*>(row);
        uint32_t w[W];
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = at[min(g * W + i, words - 1)];
        float x[8];
        mx_decode8<FMT>(w, row[words * 4 + g / 4], x);
        store_f8<BF16>(dst + r * dst_stride + (int64_t)g * (BF16 ? 16 : 32), n, x);
    }
}
