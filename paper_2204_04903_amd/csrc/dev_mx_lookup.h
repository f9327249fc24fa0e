// Pooled lookup from tables of microscaled 4-bit rows.
// Part of pk_device.hip: included there, in this order, inside its anonymous namespace.

// ---------------------------------------------------------------------------
// out[b, field's columns] = (1/L) sum over the bag's IDs of s * e, the elements e of the ID's row times their blocks'
// scales; Gather and SegmentReduction (Sec. II-D) of all packs in one launch, keys formed from the IDs as the pooling of
// small batches does.  A thread holds eight columns of a bag and goes through the bag's IDs; sums in double, rounded once.
// ---------------------------------------------------------------------------
constexpr int kMxPacks = 16;     // packs of one launch
struct MxPack {
    const uint8_t* T; const int32_t* slot_field;
    int32_t D, chunks, stride, code_bytes;       // dimension; eight columns each; bytes of a row and of its codes
    int64_t item_begin;                          // (slot, bag, chunk) items of the packs before
};
struct MxJob {
    MxPack pack[kMxPacks];
    int32_t n_packs, B, n_fields; int64_t n_items, nnz;
    const FieldMeta* fmeta; const int64_t* ids; const int32_t* offsets;
    float* out; int64_t out_stride; int32_t* error_word;
};

__global__ void __launch_bounds__(NT)
mx_lookup_kernel(MxJob job)
{
    const int64_t item = (int64_t)blockIdx.x * NT + threadIdx.x;
    if (item == 0) {
        const int32_t* o = as_global(job.offsets);
        if (o[0] != 0 || o[(int64_t)job.n_fields * job.B] != job.nnz) atomicOr(job.error_word, 1);
    }
    if (item >= job.n_items) return;
    int p = 0;
    while (p + 1 < job.n_packs && item >= job.pack[p + 1].item_begin) ++p;
    const MxPack& k = job.pack[p];
    const int64_t at = item - k.item_begin, bag = at / k.chunks;
    const int c = (int)(at - bag * k.chunks), j = (int)(bag / job.B), b = (int)(bag - (int64_t)j * job.B);
    const int f = as_global(k.slot_field)[j];
    const FieldMeta m = as_global(job.fmeta)[f];
    const int32_t* offs = as_global(job.offsets) + (int64_t)f * job.B + b;
    const int64_t* ids = as_global(job.ids);
    int q0 = offs[0], q1 = offs[1];
    if (q0 < 0 || q1 < q0 || q1 > job.nnz) {               // a rejected bag pools to zeros, nothing is read for it
        if (c == 0) atomicOr(job.error_word, 1);
        q1 = q0;
    }
    const uint8_t* T = as_global(k.T);
    double acc[8] = {};
    for (int q = q0; q < q1; ++q) {
        const uint8_t* row = T + (size_t)(m.base_row + fold_id(ids[q], m.rows, m.magic)) * (uint32_t)k.stride;
        const uint32_t w[1] = {reinterpret_cast<const uint32_t*>(row)[c]};
        float x[8];
        mx_decode8<PK_MXFP4>(w, row[k.code_bytes + (c >> 2)], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += (double)x[i];
    }
    const double scale = m.pool == PK_MEAN && q1 > q0 ? 1.0 / (double)(q1 - q0) : 1.0;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (float)(acc[i] * scale);
    store_f8<false>(reinterpret_cast<char*>(as_global(job.out) + (size_t)b * (size_t)job.out_stride + m.col + 8 * c), k.D - 8 * c, y);
}
