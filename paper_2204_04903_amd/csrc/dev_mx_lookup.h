// Pooled lookup from tables of microscaled 4-bit rows.
// Part of pk_device.hip: included there, in this order, inside its anonymous namespace.

// ---------------------------------------------------------------------------
// out[b, field's columns] = (1/L) sum over the bag's IDs of s * e, the elements e of the ID's row times their blocks'
// scales; Gather and SegmentReduction (Sec. II-D) of all packs in one launch, keys formed from the IDs as the pooling of
// small batches does.
//
// A lane holds up to 32 columns of a row, one block, which is one wide access and, from 25 columns on, one for the scale; a
// row of more columns is a group of 2, 4 or 8 lanes.  A block of the launch takes the bags of one field that its groups can
// hold, one each, and deals them out by their number of rounds of R rows, longest first, so that the groups of a wavefront
// have about as many (bags of 1 to 50 IDs in their own order: half of the lanes wait).  R rows and the next R IDs are in flight together;
// a round's rows are added as a tree in fp32 (two digits each: exact unless the scales are far apart), the rounds in
// double.  Fields of sequences (kMxSeqAvg IDs per bag on average and more) go to wavefronts of their own, which start first: there the groups of a
// wavefront share a bag, and their sums meet by halves, every lane giving away half of its columns a step.
// ---------------------------------------------------------------------------
constexpr int kMxPacks = 16;     // packs of one launch
constexpr int kMxRound = 8;
constexpr int kMxSeqAvg = 64;
constexpr int kMxBins = 32;      // numbers of rounds that are told apart
struct MxPack {
    const uint8_t* T; const int32_t* slot_field;
    int32_t D, sh, kind, stride, code_bytes;     // dimension; log2 of the lanes per row; 1 to 4: words of a row of one lane, 5: whole blocks, 6: others
    int32_t n_fields, tiles, item_begin;         // fields; blocks per field; first block of the pack among the launch's
};
struct MxJob {
    MxPack pack[kMxPacks];
    int32_t n_packs, B, n_fields, n_items, seq_blocks; int64_t nnz;
    const FieldMeta* fmeta; const int64_t* ids; const int32_t* offsets;
    float* out; int64_t out_stride; int32_t* error_word;
};

// what a lane holds of a row: W words of codes and the scale
template <int W, bool MULTI, bool RAGGED>
struct MxPiece {
    uint32_t w[W], s;
    __device__ __forceinline__ void load(const uint8_t* row, int li, int code_bytes)
    {
        const uint32_t* at = reinterpret_cast<const uint32_t*>(row);
        if constexpr (RAGGED) {
            const int words = code_bytes >> 2, blk = min(li, (words - 1) >> 2);
#pragma unroll
            for (int j = 0; j < W; ++j) w[j] = at[min(4 * blk + j, words - 1)];
            s = row[code_bytes + blk];
        } else if constexpr (MULTI) {
            load_u32<4>(at + 4 * li, w);
            s = row[code_bytes + li];
        } else if constexpr (W == 1) {
            uint32_t v[2];
            load_u32<2>(at, v);
            w[0] = v[0]; s = v[1];
        } else if constexpr (W == 2) {
            typedef uint32_t u32x3 __attribute__((ext_vector_type(3), aligned(4)));
            const u32x3 v = *reinterpret_cast<const u32x3*>(at);
            w[0] = v.x; w[1] = v.y; s = v.z;
        } else if constexpr (W == 3) {
            uint32_t v[4];
            load_u32<4>(at, v);
            w[0] = v[0]; w[1] = v[1]; w[2] = v[2]; s = v[3];
        } else {
            load_u32<4>(at, w);
            s = at[4];
        }
    }
};

struct MxField {
    const uint8_t* T; const int64_t* ids; int64_t nnz;
    uint32_t base, rows, stride; uint64_t magic;
    int code_bytes;
    __device__ __forceinline__ MxField(const MxJob& job, const MxPack& k, const FieldMeta& m)
        : T(as_global(k.T)), ids(as_global(job.ids)), nnz(job.nnz), base(m.base_row), rows(m.rows), stride((uint32_t)k.stride), magic(m.magic),
          code_bytes(k.code_bytes) {}
    // R IDs from q on, those from e (> q) on replaced by the last one before it
    template <int R>
    __device__ __forceinline__ void load_ids(int q, int e, int64_t (&id)[R]) const
    {
#pragma unroll
        for (int i = 0; i < R; ++i) id[i] = ids[min(q + i, e - 1)];
    }
    template <int W, bool MULTI, bool RAGGED, int R>
    __device__ __forceinline__ void add_rows(const int64_t (&id)[R], int left, int li, double (&acc)[8 * W]) const
    {
        MxPiece<W, MULTI, RAGGED> v[R];
#pragma unroll
        for (int i = 0; i < R; ++i) v[i].load(T + (size_t)(base + fold_id(id[i], rows, magic)) * stride, li, code_bytes);
        float sc[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            sc[i] = mx_scale(v[i].s & 255u);
            if (i > 0 && i >= left) {                      // past the bag's end: nothing
                sc[i] = 0.f;
#pragma unroll
                for (int j = 0; j < W; ++j) v[i].w[j] = 0;
            }
        }
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                f32x2v x[R];
#pragma unroll
                for (int i = 0; i < R; ++i)
                    x[i] = c == 0 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v[i].w[j], sc[i], 0)
                         : c == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v[i].w[j], sc[i], 1)
                         : c == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v[i].w[j], sc[i], 2)
                                  : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v[i].w[j], sc[i], 3);
#pragma unroll
                for (int d = 1; d < R; d *= 2)
#pragma unroll
                    for (int i = 0; i + d < R; i += 2 * d) { x[i].x += x[i + d].x; x[i].y += x[i + d].y; }
                acc[8 * j + 2 * c] += (double)x[0].x;
                acc[8 * j + 2 * c + 1] += (double)x[0].y;
            }
    }
};

__device__ __forceinline__ bool mx_is_seq(const MxJob& job, int f)
{
    const int32_t* o = as_global(job.offsets) + (int64_t)f * job.B;
    return job.seq_blocks && (int64_t)o[job.B] - o[0] >= (int64_t)kMxSeqAvg * job.B;
}
// bag b of a field: its positions, none and the error raised where its offsets are no range of the IDs
__device__ __forceinline__ void mx_bag(const MxJob& job, const int32_t* offs, int b, bool report, int& q, int& e)
{
    q = offs[b]; e = offs[b + 1];
    if (q < 0 || e < q || e > job.nnz) {
        if (report) atomicOr(job.error_word, 1);
        q = e = 0;
    }
}

// a block's tile of a field: s_bin [kMxBins], s_bag [256]
template <int W, bool MULTI, bool RAGGED>
__device__ __forceinline__ void mx_tile(const MxJob& job, const MxPack& k, const FieldMeta& m, const int32_t* offs, int tile, int* s_bin, int* s_bag)
{
    constexpr int R = kMxRound;
    const int t = threadIdx.x, sh = MULTI ? k.sh : 0, n_groups = NT >> sh, b0 = tile * n_groups, nb = min(n_groups, job.B - b0);
    const MxField src(job, k, m);
    {
        if (t < kMxBins) s_bin[t] = 0;
        __syncthreads();
        int pos = 0, bin = 0;
        if (t < nb) {
            int q, e;
            mx_bag(job, offs, b0 + t, true, q, e);
            bin = kMxBins - 1 - min((e - q + R - 1) / R, kMxBins - 1);
            pos = atomicAdd(&s_bin[bin], 1);
        }
        __syncthreads();
        if (t < 64) {                                      // bins to places (the first wavefront, half of it idle)
            int v = t < kMxBins ? s_bin[t] : 0;
            const int own = v;
#pragma unroll
            for (int o = 1; o < kMxBins; o <<= 1) { const int u = __shfl_up(v, o, 64); if (t >= o) v += u; }
            if (t < kMxBins) s_bin[t] = v - own;
        }
        __syncthreads();
        if (t < nb) s_bag[s_bin[bin] + pos] = b0 + t;
        __syncthreads();
    }
    const int g = t >> sh, li = t & ((1 << sh) - 1);
    if (g >= nb) return;
    const int b = s_bag[g];
    int q, e;
    mx_bag(job, offs, b, false, q, e);
    const int len = e - q;
    double acc[8 * W] = {};
    int64_t id[R], next[R];
    if (q < e) src.template load_ids<R>(q, e, id);
    while (q < e) {
        src.template load_ids<R>(min(q + R, e - 1), e, next);
        src.template add_rows<W, MULTI, RAGGED, R>(id, e - q, li, acc);
#pragma unroll
        for (int i = 0; i < R; ++i) id[i] = next[i];
        q += R;
    }
    const double scale = m.pool == PK_MEAN && len > 0 ? 1.0 / (double)len : 1.0;
    float* o = as_global(job.out) + (size_t)b * (size_t)job.out_stride + m.col + 32 * li;
#pragma unroll
    for (int j = 0; j < W; ++j) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = (float)(acc[8 * j + i] * scale);
        store_f8<false>(reinterpret_cast<char*>(o + 8 * j), k.D - 32 * li - 8 * j, y);
    }
}

// a step of the meeting sums: with the lane `o` away, N columns of which each keeps half, the lane with the bit the upper one
template <int N>
__device__ __forceinline__ void mx_halve(double* acc, int o, bool upper)
{
    if constexpr (N > 1) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const double give = upper ? acc[i] : acc[i + N / 2], keep = upper ? acc[i + N / 2] : acc[i];
            acc[i] = keep + __shfl_xor(give, o, 64);
        }
    } else {
        acc[0] += __shfl_xor(acc[0], o, 64);
    }
}

template <int W, bool MULTI, bool RAGGED>
__device__ __forceinline__ void mx_seq_bag(const MxJob& job, const MxPack& k, const FieldMeta& m, const int32_t* offs, int b)
{
    constexpr int R = kMxRound;
    const int lane = threadIdx.x & 63, sh = MULTI ? k.sh : 0, g = lane >> sh, li = lane & ((1 << sh) - 1), n_groups = 64 >> sh;
    const MxField src(job, k, m);
    int q0, e;
    mx_bag(job, offs, b, lane == 0, q0, e);
    double acc[8 * W] = {};
    int64_t id[R], next[R];
    int q = q0 + g * R;
    if (q < e) src.template load_ids<R>(q, e, id);
    while (q < e) {
        src.template load_ids<R>(min(q + R * n_groups, e - 1), e, next);
        src.template add_rows<W, MULTI, RAGGED, R>(id, e - q, li, acc);
#pragma unroll
        for (int i = 0; i < R; ++i) id[i] = next[i];
        q += R * n_groups;
    }
    // six steps less the row's lanes; W == 3 has no halves: its last word is zeros
    constexpr int C = W == 3 ? 32 : 8 * W;
    double a[C];
#pragma unroll
    for (int i = 0; i < C; ++i) a[i] = i < 8 * W ? acc[i] : 0.0;
    int col = 0, n = C, o = 1 << sh;
    auto step = [&](auto N) {
        if (o < 64) {
            const bool upper = (lane & o) != 0;
            mx_halve<decltype(N)::value>(a, o, upper);
            if constexpr (decltype(N)::value > 1) { n /= 2; col += upper ? n : 0; }
            o *= 2;
        }
    };
    step(std::integral_constant<int, C>{});
    step(std::integral_constant<int, C / 2>{});
    step(std::integral_constant<int, C / 4>{});
    step(std::integral_constant<int, (C >= 16 ? C / 8 : 1)>{});
    step(std::integral_constant<int, (C >= 32 ? C / 16 : 1)>{});
    step(std::integral_constant<int, 1>{});
    // n columns are left in a lane: from col on of the row's lane li (several lanes may hold the same ones)
    const double scale = m.pool == PK_MEAN && e > q0 ? 1.0 / (double)(e - q0) : 1.0;
    float* out = as_global(job.out) + (size_t)b * (size_t)job.out_stride + m.col;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n && 32 * li + col + i < k.D) out[32 * li + col + i] = (float)(a[i] * scale);
}

#define MX_KINDS(call)                                              \
    switch (k.kind) {                                               \
        case 1: call(1, false, false); break;                       \
        case 2: call(2, false, false); break;                       \
        case 3: call(3, false, false); break;                       \
        case 4: call(4, false, false); break;                       \
        case 5: call(4, true, false); break;                        \
        default: call(4, true, true); break;                        \
    }

__global__ void __launch_bounds__(NT)
mx_lookup_kernel(MxJob job)
{
    __shared__ int s_bin[kMxBins], s_bag[NT];
    const int item = (int)blockIdx.x - job.seq_blocks;
    if (item < 0) {
        // the bags of all sequence fields, one after the other, dealt to the wavefronts
        const int lane = threadIdx.x & 63, n_waves = job.seq_blocks * (NT / 64);
        int64_t base = 0, next = (int)blockIdx.x * (NT / 64) + (threadIdx.x >> 6);
        for (int p = 0; p < job.n_packs; ++p) {
            const MxPack& k = job.pack[p];
            for (int j0 = 0; j0 < k.n_fields; j0 += 64) {
                bool seq = false;
                if (j0 + lane < k.n_fields) seq = mx_is_seq(job, as_global(k.slot_field)[j0 + lane]);
                for (uint64_t todo = __ballot(seq); todo; todo &= todo - 1) {
                    const int f = as_global(k.slot_field)[j0 + __ffsll((unsigned long long)todo) - 1];
                    const FieldMeta m = as_global(job.fmeta)[f];
                    const int32_t* offs = as_global(job.offsets) + (int64_t)f * job.B;
                    for (; next < base + job.B; next += n_waves) {
                        const int b = (int)(next - base);
#define MX_SEQ(W, M, G) mx_seq_bag<W, M, G>(job, k, m, offs, b)
                        MX_KINDS(MX_SEQ)
                    }
                    base += job.B;
                }
            }
        }
        return;
    }
    if (item == 0 && threadIdx.x == 0) {
        const int32_t* o = as_global(job.offsets);
        if (o[0] != 0 || o[(int64_t)job.n_fields * job.B] != job.nnz) atomicOr(job.error_word, 1);
    }
    int p = 0;
    while (p + 1 < job.n_packs && item >= job.pack[p + 1].item_begin) ++p;
    const MxPack& k = job.pack[p];
    const int j = (item - k.item_begin) / k.tiles, tile = item - k.item_begin - j * k.tiles;
    const int f = as_global(k.slot_field)[j];
    if (mx_is_seq(job, f)) return;
    const FieldMeta m = as_global(job.fmeta)[f];
    const int32_t* offs = as_global(job.offsets) + (int64_t)f * job.B;
#define MX_TILE(W, M, G) mx_tile<W, M, G>(job, k, m, offs, tile, s_bin, s_bag)
    MX_KINDS(MX_TILE)
}
