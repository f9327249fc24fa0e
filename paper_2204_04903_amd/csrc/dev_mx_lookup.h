// Pooled lookup from tables of microscaled 4-bit rows.
// Part of pk_device.hip: included there, in this order, inside its anonymous namespace.

// ---------------------------------------------------------------------------
// out[b, field's columns] = (1/L) sum over the bag's IDs of s * e, the elements e of the ID's row times their blocks'
// scales; Gather and SegmentReduction (Sec. II-D) of all packs in one launch, keys formed from the IDs as the pooling of
// small batches does.
//
// What a lookup costs is its requests: from an L2 246 G of them a second (row of 20 bytes, one access), and 135 G rows where codes and scale
// are two accesses, because the second one finds the line not there yet either.  So a lane holds two words of codes, 16
// columns, and the word behind them; the last lane of a row has the row's scales there and hands them to the others.
// A wavefront, a block of its own, takes two bags per lane group, those with many rounds of R rows
// together with those with few.  A round's IDs are read by all lanes, R of them next to one another per bag, each ID once; its keys
// go through LDS; its rows are in flight together with the next round's IDs.  A round's rows are added as a tree in fp32 (two digits each: exact unless the
// scales are far apart), the rounds in double.  Fields of sequences (kMxSeqAvg IDs per bag on average and more) go to
// wavefronts of their own, which start first: there the groups of a wavefront share a bag, and their sums meet by halves, every
// lane giving away half of its columns a step.
// 200 fields of 8 to 64 columns, 20.9 M IDs: 215 us, 97 G rows/s, 763 MB past the L2s (an earlier form took 240: 135 with all rows in the
// L2s, 185 without the output's writes); 10 sequence fields of 100 to 1000 IDs, 64 columns, 1024 samples: 53 us, 107 G; 26 one-hot
// fields, 64 samples: 5.
// ---------------------------------------------------------------------------
constexpr int kMxPacks = 16;     // packs of one launch
// From which average a field's bags go to wavefronts of their own, by the number of bags.  Few bags are too few tiles for the chip: one sample
// of 26 fields of 32 columns takes 5.6 us at 6 IDs a bag by tiles and 5.7 by bags, 6.7 and 6.0 at 8, 12.6 and 6.1 at 50; 128 samples of 30
// fields 13.0 and 12.7 at 8, 27 and 13.4 at 50.  Many keep the tiles busy: 1024 samples of 26 fields 32.8 and 56 at 63 IDs a bag.  Where the two
// meet depends on more than the bags: 30 fields of 50 IDs take 28.7 by tiles and 13.1 by bags with 4110 bags, 31.2 and 20.4 with 7680, 32.8 and
// 36.6 with 15 360 (of 25 IDs 17.3 and 12.7, 18.0 and 19.0, 21.0 and 36.0); 200 fields of 25 IDs 17.0 and 73 with 12 800, since every wavefront
// walks the list of fields.  It is a field's average that counts: a long bag among short ones is one lane group's.
constexpr int kMxSeqAvg = 64, kMxSeqAvgFew = 8;
constexpr int64_t kMxFewBags = 4096;
constexpr int64_t kMxSeqBlocks = 8192, kMxSeqIds = 512;      // wavefronts for their bags, at most (half as many: sequences of 550 IDs 63 us instead of 57), and IDs that there should be for each
// Fields from which every one has its XCD.  8192 samples, 32 columns, 5 IDs: 32 fields 22.7 us so and 26.8 without, 33 25.2 and 27.6, 41 30.9 and 33.6, 64
// 37.4 and 45.4.  3001 samples of four widths, where the XCDs' shares are less even: 32 fields 15.9 and 20.0, 33 19.1 and 20.3, 37 21.4 and 20.7, 41 22.0
// both, 64 27.3 and 30.1; bags of 0 to 19 IDs in 37 fields 30.0 and 28.5.
constexpr int kMxXcdFields = 32;
// One-hot bags of this many samples and more are written by tiles too: 26 fields of 32 columns, 8192 samples, 17.2 us bag by bag, 15.3 so;
// 100 of 16 columns and 2 IDs, 1024 samples, 10.2 and 10.9; 26 of 32, 64 samples, 4.8 and 5.6.
constexpr int kMxStagedBags = 4096;
constexpr int kMxBins = 32;      // numbers of rounds that are told apart
struct MxPack {
    const uint8_t* T; const int32_t* slot_field;
    int32_t D, kind, stride, code_bytes;         // dimension; MxKind; bytes of a row and of its codes
    int32_t n_fields, tiles, item_begin, turn, p;   // fields; blocks per field; first block of the pack among the launch's; its first field's XCD; pack
};
struct MxJob {
    MxPack pack[kMxPacks];
    int32_t n_packs, B, n_fields, by_xcd, seq_avg, seq_blocks; int64_t nnz;
    const FieldMeta* fmeta; const int64_t* ids; const int32_t* offsets;
    float* out; int64_t out_stride; int32_t* error_word;
};

// Kinds of rows: 0: up to 8 columns, one lane with the row's one word and its scale; k: up to 2^(k + 3) columns, 2^(k - 1)
// lanes of two words each, the last ones ending with the row; 5: more than 128 columns, 16 lanes, scales in more than one word.
constexpr int kMxKinds = 6;
constexpr int mx_lanes_shift(int kind) { return kind == 0 ? 0 : kind - 1; }
inline int mx_kind(int dim) { int k = 0; while ((8 << k) < dim) ++k; return k; }

struct MxSrc {
    const uint8_t* T; const int64_t* ids;
    uint32_t base, rows, stride; uint64_t magic;
    int code_bytes;
    __device__ __forceinline__ MxSrc(const MxJob& job, const MxPack& k, const FieldMeta& m)
        : T(as_global(k.T)), ids(as_global(job.ids)), base(m.base_row), rows(m.rows), stride((uint32_t)k.stride), magic(m.magic), code_bytes(k.code_bytes) {}
    __device__ __forceinline__ uint32_t key(int64_t id) const { return base + fold_id(id, rows, magic); }
};

template <int KIND>
struct MxLane {
    static constexpr int W = KIND == 0 ? 1 : 2, SH = mx_lanes_shift(KIND), L = 1 << SH, G = 64 >> SH;
    int c;                                                 // first word
    uint32_t turn0, turn1;                                 // the words' scales, turned to where a number has its exponent
    const uint8_t *at, *scale_at;
    __device__ __forceinline__ explicit MxLane(const MxSrc& src)
    {
        c = KIND == 0 ? 0 : min(2 * (int)(threadIdx.x & (L - 1)), (src.code_bytes >> 2) - 2);
        turn0 = ((c >> 2) * 8 + 9) & 31; turn1 = (((c + 1) >> 2) * 8 + 9) & 31;
        at = src.T + 4 * c; scale_at = src.T + src.code_bytes;
    }
    // the rows of R keys in LDS, of which `left` count
    template <int R>
    __device__ __forceinline__ void add_rows(const MxSrc& src, const uint32_t* s_key, int left, double (&acc)[8 * W]) const
    {
        uint32_t w[R][W], s[R], s2[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const uint64_t row = (uint64_t)s_key[i] * src.stride;
            const uint32_t* p = reinterpret_cast<const uint32_t*>(at + row);
            if constexpr (W == 1) {
                uint32_t v[2];
                load_u32<2>(p, v);
                w[i][0] = v[0]; s[i] = v[1];
            } else if constexpr (KIND == 5) {
                uint32_t v[2];
                load_u32<2>(p, v);
                w[i][0] = v[0]; w[i][1] = v[1];
                s[i] = scale_at[row + (c >> 2)]; s2[i] = scale_at[row + ((c + 1) >> 2)];
            } else {
                typedef uint32_t u32x3 __attribute__((ext_vector_type(3), aligned(4)));
                const u32x3 v = *reinterpret_cast<const u32x3*>(p);
                w[i][0] = v.x; w[i][1] = v.y; s[i] = v.z;
            }
        }
        // (of a scale operand the exponent is all that is read: what else the word holds may stay)
        float f0[R], f1[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if constexpr (KIND == 2) s[i] = (uint32_t)__builtin_amdgcn_mov_dpp((int)s[i], 0xF5, 0xF, 0xF, true);        // lanes 1 1 3 3
            if constexpr (KIND == 3) s[i] = (uint32_t)__builtin_amdgcn_mov_dpp((int)s[i], 0xFF, 0xF, 0xF, true);        // lane 3
            if constexpr (KIND == 4) s[i] = (uint32_t)__shfl((int)s[i], threadIdx.x | 7, 64);
            if constexpr (KIND == 5) {
                f0[i] = mx_scale(s[i]); f1[i] = mx_scale(s2[i]);
            } else if constexpr (KIND <= 1) {
                f0[i] = f1[i] = mx_scale(s[i]);
            } else {
                f0[i] = __uint_as_float(__builtin_amdgcn_alignbit(s[i], s[i], turn0));
                f1[i] = __uint_as_float(__builtin_amdgcn_alignbit(s[i], s[i], turn1));
            }
        }
        if (__any(left < R)) {                             // past the bag's end: nothing (its last row again, whose scale does no harm)
#pragma unroll
            for (int i = 1; i < R; ++i)
#pragma unroll
                for (int j = 0; j < W; ++j) w[i][j] = i < left ? w[i][j] : 0;
        }
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                f32x2v x[R];
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const float f = j ? f1[i] : f0[i];
                    x[i] = h == 0 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i][j], f, 0)
                         : h == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i][j], f, 1)
                         : h == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i][j], f, 2)
                                  : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i][j], f, 3);
                }
#pragma unroll
                for (int d = 1; d < R; d *= 2)
#pragma unroll
                    for (int i = 0; i + d < R; i += 2 * d) { x[i].x += x[i + d].x; x[i].y += x[i + d].y; }
                acc[8 * j + 2 * h] += (double)x[0].x;
                acc[8 * j + 2 * h + 1] += (double)x[0].y;
            }
    }
};

__device__ __forceinline__ void mx_wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ bool mx_is_seq(const MxJob& job, int64_t field_ids)
{
    return job.seq_blocks && field_ids >= (int64_t)job.seq_avg * job.B;
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

// A wavefront's tile of a field.  s_bin [kMxBins], s_bag [128], s_key [2][64 * 8], s_out [128 * 16]
template <int KIND, int R>
__device__ __forceinline__ void mx_tile(const MxJob& job, const MxPack& k, const FieldMeta& m, const int32_t* offs, int tile, int* s_bin, int* s_bag,
                                        uint32_t (*s_key)[512], float* s_out)
{
    using Lane = MxLane<KIND>;
    constexpr int G = Lane::G, W = Lane::W, SH = Lane::SH, COLS = 8 * W * Lane::L;
    const bool staged = R > 1 || job.B >= kMxStagedBags;   // sums go out together, else each as it is done
    const int lane = threadIdx.x, b0 = tile * 2 * G, nb = min(2 * G, job.B - b0);
    const MxSrc src(job, k, m);
    // the bags by their number of rounds, most first
    if (R > 1) {
        if (lane < kMxBins) s_bin[lane] = 0;
        mx_wave_order();
        int bin[2] = {0, 0}, pos[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = lane + 64 * h;
            if (i < nb) {
                int q, e;
                mx_bag(job, offs, b0 + i, true, q, e);
                bin[h] = kMxBins - 1 - min((int)((unsigned)(e - q + R - 1) / R), kMxBins - 1);
                pos[h] = atomicAdd(&s_bin[bin[h]], 1);
            }
        }
        mx_wave_order();
        int v = lane < kMxBins ? s_bin[lane] : 0;
        const int own = v;
#pragma unroll
        for (int o = 1; o < kMxBins; o <<= 1) { const int u = __shfl_up(v, o, 64); if (lane >= o) v += u; }
        mx_wave_order();
        if (lane < kMxBins) s_bin[lane] = v - own;
        mx_wave_order();
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (lane + 64 * h < nb) s_bag[s_bin[bin[h]] + pos[h]] = b0 + lane + 64 * h;
        mx_wave_order();
    }
    const int g = lane >> SH, i1 = min(g, nb - 1), i2 = min(2 * G - 1 - g, nb - 1);
    int bag = R > 1 ? s_bag[i1] : b0 + i1, bag2 = R > 1 ? s_bag[i2] : b0 + i2;
    int q, e, q2, e2;
    mx_bag(job, offs, bag, R == 1 && g < nb, q, e);
    mx_bag(job, offs, bag2, R == 1 && 2 * G - 1 - g < nb, q2, e2);
    int todo = (g < nb) + (g < nb && 2 * G - 1 - g < nb);  // bags that this group has left to write
    if (todo == 0) q = e = 0;
    const Lane me(src);
    int q0 = q;                                            // where the bag begins
    double acc[8 * W] = {};
    // the IDs of a round: lane l reads number l % R of groups l / R, l / R + 64 / R ...
    constexpr int N = G * R <= 64 ? 1 : G * R / 64;
    int64_t id[N];
    auto ask = [&](int at, int end) {                      // (a group's first position and its bag's end)
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int from = ((lane + 64 * n) / R) << SH, p = __shfl(at, from, 64), z = __shfl(end, from, 64);
            id[n] = 0;
            if (lane + 64 * n < G * R && p < z) id[n] = src.ids[min(p + lane % R, z - 1)];
        }
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int n = 0; n < N; ++n) s_key[buf][lane + 64 * n] = src.key(id[n]);
        mx_wave_order();
    };
    auto write = [&]() {
        const double scale = m.pool == PK_MEAN && e > q0 ? 1.0 / (double)(e - q0) : 1.0;
        float y[8 * W];
#pragma unroll
        for (int i = 0; i < 8 * W; ++i) { y[i] = (float)(acc[i] * scale); acc[i] = 0.0; }
        if (staged) {
            float* o = s_out + (bag - b0) * COLS + 8 * me.c;
#pragma unroll
            for (int i = 0; i < 8 * W; i += 4) { f32x4 v; v.x = y[i]; v.y = y[i + 1]; v.z = y[i + 2]; v.w = y[i + 3]; *reinterpret_cast<f32x4*>(o + i) = v; }
        } else {
            float* o = as_global(job.out) + (size_t)bag * (size_t)job.out_stride + m.col + 8 * me.c;
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float z[8] = {y[8 * j], y[8 * j + 1], y[8 * j + 2], y[8 * j + 3], y[8 * j + 4], y[8 * j + 5], y[8 * j + 6], y[8 * j + 7]};
                store_f8<false>(reinterpret_cast<char*>(o + 8 * j), k.D - 8 * (me.c + j), z);
            }
        }
        --todo;
        bag = bag2;
        q = q0 = todo ? q2 : 0;
        e = todo ? e2 : 0;
    };
    ask(q, e);
    put(0);
    for (int buf = 0; __any(todo > 0); buf ^= 1) {
        // (a bag without positions still takes a round, of which nothing counts: it is written after it)
        const bool ends = q + R >= e;
        const int nq = ends ? (todo > 1 ? q2 : 0) : q + R, ne = ends ? (todo > 1 ? e2 : 0) : e;
        ask(nq, ne);
        if (q < e) me.template add_rows<R>(src, s_key[buf] + g * R, e - q, acc);
        put(buf ^ 1);
        if (todo > 0) {
            if (ends) write();
            else q += R;
        }
    }
    if (!staged) return;
    mx_wave_order();
    // rows of the output in whole, 16 bytes a lane
    constexpr int PER = COLS / 4;
    const int col = 4 * (lane % PER), left = k.D - col;
#pragma unroll
    for (int r = lane / PER; r < 2 * G; r += 64 / PER) {
        if (r >= nb || left <= 0) continue;
        const f32x4 y = *reinterpret_cast<const f32x4*>(s_out + r * COLS + col);
        float* o = as_global(job.out) + (size_t)(b0 + r) * (size_t)job.out_stride + m.col + col;
        if (left >= 4) {
            *reinterpret_cast<f32x4*>(o) = y;
        } else {
            o[0] = y.x;
            if (left > 1) o[1] = y.y;
            if (left > 2) o[2] = y.z;
        }
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

template <int KIND>
__device__ __forceinline__ void mx_seq_bag(const MxJob& job, const MxPack& k, const FieldMeta& m, const int32_t* offs, int b, uint32_t (*s_key)[512])
{
    using Lane = MxLane<KIND>;
    constexpr int R = 8, G = Lane::G, W = Lane::W, SH = Lane::SH, C = 8 * W, N = G * R / 64 > 0 ? G * R / 64 : 1;
    const int lane = threadIdx.x, g = lane >> SH;
    const MxSrc src(job, k, m);
    int q0, e;
    mx_bag(job, offs, b, lane == 0, q0, e);
    const Lane me(src);
    double acc[C] = {};
    int64_t id[N];
    auto ask = [&](int at) {
#pragma unroll
        for (int n = 0; n < N; ++n)
            if (lane + 64 * n < G * R) id[n] = src.ids[min(at + lane + 64 * n, e - 1)];
    };
    int buf = 0;
    if (q0 < e) ask(q0);
    for (int q = q0; q < e; q += G * R) {
#pragma unroll
        for (int n = 0; n < N; ++n)
            if (lane + 64 * n < G * R) s_key[buf][lane + 64 * n] = src.key(id[n]);
        mx_wave_order();
        if (q + G * R < e) ask(q + G * R);
        if (q + g * R < e) me.template add_rows<R>(src, s_key[buf] + g * R, e - q - g * R, acc);
        buf ^= 1;
    }
    int col = 0, n = C, o = 1 << SH;
    auto step = [&](auto H) {
        constexpr int have = decltype(H)::value;
        if (o < 64) {
            const bool upper = (lane & o) != 0;
            mx_halve<have>(acc, o, upper);
            if constexpr (have > 1) { n /= 2; col += upper ? n : 0; }
            o *= 2;
        }
    };
    step(std::integral_constant<int, C>{});
    step(std::integral_constant<int, C / 2>{});
    step(std::integral_constant<int, C / 4>{});
    step(std::integral_constant<int, (C >= 16 ? C / 8 : 1)>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 1>{});
    // n columns are left in a lane: from col on of its 16 (several lanes may hold the same ones)
    const double scale = m.pool == PK_MEAN && e > q0 ? 1.0 / (double)(e - q0) : 1.0;
    float* out = as_global(job.out) + (size_t)b * (size_t)job.out_stride + m.col;
    col += 8 * me.c;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n && col + i < k.D) out[col + i] = (float)(acc[i] * scale);
}

#define MX_KINDS(call)                     \
    switch (k.kind) {                      \
        case 0: call(0); break;            \
        case 1: call(1); break;            \
        case 2: call(2); break;            \
        case 3: call(3); break;            \
        case 4: call(4); break;            \
        default: call(5); break;           \
    }

__global__ void __launch_bounds__(64)
mx_lookup_kernel(MxJob job)
{
    __shared__ int s_bin[kMxBins], s_bag[128];
    __shared__ __attribute__((aligned(16))) uint32_t s_key[2][512];
    __shared__ __attribute__((aligned(16))) float s_out[128 * 16];     // a tile's sums
    const int item = (int)blockIdx.x - job.seq_blocks, lane = threadIdx.x;
    const int32_t* offsets = as_global(job.offsets);
    if (item < 0) {
        // the bags of all sequence fields, one after the other, dealt to the wavefronts (four looks at 64 fields at a time)
        int64_t base = 0, next = blockIdx.x;
        for (int f0 = 0; f0 < job.n_fields; f0 += 256) {
            int lo[4], hi[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int32_t* o = offsets + (int64_t)min(f0 + 64 * i + lane, job.n_fields - 1) * job.B;
                lo[i] = o[0]; hi[i] = o[job.B];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int f1 = f0 + 64 * i;
                for (uint64_t todo = __ballot(f1 + lane < job.n_fields && mx_is_seq(job, (int64_t)hi[i] - lo[i])); todo; todo &= todo - 1) {
                    if (next < base + job.B) {             // (a field's metadata only where one of its bags is this wavefront's)
                        const int f = f1 + __ffsll((unsigned long long)todo) - 1;
                        const FieldMeta m = as_global(job.fmeta)[f];
                        int p = 0;
                        while (p < job.n_packs && job.pack[p].p != m.pack) ++p;
                        const MxPack& k = job.pack[min(p, job.n_packs - 1)];
                        const int32_t* offs = offsets + (int64_t)f * job.B;
                        for (; next < base + job.B; next += job.seq_blocks) {
                            if (p == job.n_packs) continue;        // another launch's
                            const int b = (int)(next - base);
#define MX_SEQ(K) mx_seq_bag<K>(job, k, m, offs, b, s_key)
                            MX_KINDS(MX_SEQ)
                        }
                    }
                    base += job.B;
                }
            }
        }
        return;
    }
    if (item == 0 && lane == 0) {
        if (offsets[0] != 0 || offsets[(int64_t)job.n_fields * job.B] != job.nnz) atomicOr(job.error_word, 1);
    }
    int p = 0;
    while (p + 1 < job.n_packs && item >= job.pack[p + 1].item_begin) ++p;
    const MxPack& k = job.pack[p];
    int j, tile;
    if (job.by_xcd) {                                      // a field's tiles on one XCD (blocks go to them in turn)
        const int x = item & 7, i = (item - k.item_begin) >> 3, h = i / k.tiles;
        j = 8 * h + ((x - k.turn) & 7); tile = i - h * k.tiles;
        if (j >= k.n_fields) return;
    } else {
        j = (item - k.item_begin) / k.tiles; tile = item - k.item_begin - j * k.tiles;
    }
    const int f = as_global(k.slot_field)[j];
    const int32_t* offs = offsets + (int64_t)f * job.B;
    const int64_t field_ids = (int64_t)offs[job.B] - offs[0];
    if (mx_is_seq(job, field_ids)) return;
    const FieldMeta m = as_global(job.fmeta)[f];
#define MX_TILE8(K) mx_tile<K, 8>(job, k, m, offs, tile, s_bin, s_bag, s_key, s_out)
#define MX_TILE1(K) mx_tile<K, 1>(job, k, m, offs, tile, s_bin, s_bag, s_key, s_out)
    // (rounds of eight rows from two and a half IDs a bag on: 40 fields of 64 columns, 2048 samples, 3 IDs a bag 14.1 us so and 16.4 row by
    // row, 6 15.2 and 20.1; 100 of 16 columns 17.1 and 15.9 at 3, 21.8 both at 6)
    if (2 * field_ids > 5 * (int64_t)job.B) { MX_KINDS(MX_TILE8) }
    else { MX_KINDS(MX_TILE1) }
}
