// Microscaled rows (OCP element formats E2M1 and E4M3 with one E8M0 scale per 32 columns): device side.
// Part of pk_device.hip and pk_mx.hip: included there inside their anonymous namespaces, after dev_rows.h.

// ---------------------------------------------------------------------------
// A block of 32 columns with largest magnitude m has the scale 2^t, t the smallest integer with m <= MAX * 2^t (MAX: 6 of
// E2M1, 448 of E4M3), so that every element is off by at most half a step of its format; the scale byte is t + 127, from 1
// (2^-126, also of a block of zeros) on.  One code is not used: what is nearest to 2^128, which fp32 does not hold, gets the
// code below (1.5 and 1.875 times 2^127), still within 2^-2 and 2^-4 of itself.  A block that holds an infinity or a NaN has the
// scale byte 255 and reads back as NaN.  (With the other usual rule, t = floor(log2 m) less the exponent of MAX, the
// elements between MAX and the next power of two saturate: 32 normal columns in 8 bits 2.9 % off instead of 2.7, in 4 bits 11.5 both.)
// ---------------------------------------------------------------------------
template <int FMT>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t max_bits)       // bits of the largest magnitude
{
    const int e = (int)(max_bits >> 23), m = (int)(max_bits & 0x7FFFFFu);
    if (e == 255) return 255u;
    const int t = FMT == PK_MXFP4 ? e - 2 + (m > 0x400000)                 // 6 = 1.5 * 2^2
                                  : e - 8 + (m > 0x600000);                // 448 = 1.75 * 2^8
    return (uint32_t)max(t, 1);
}
// the scale byte of the blocks that hold numbers so large, and the largest that is held
template <int FMT> constexpr uint32_t kMxTopByte = FMT == PK_MXFP4 ? 126 + 127 : 120 + 127;
template <int FMT> constexpr float kMxTop = FMT == PK_MXFP4 ? 0x1.8p127f : 0x1.Ep127f;
// the scale as the number that the conversions take (they read its exponent; byte 255: NaN)
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

typedef float f32x2v __attribute__((ext_vector_type(2)));
typedef short s16x2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

// eight columns of a block, first column in the lowest bits
template <int FMT>
__device__ __forceinline__ void mx_encode8(const float (&v)[8], uint32_t byte, uint32_t (&w)[FMT == PK_MXFP4 ? 1 : 2])
{
    const float s = mx_scale(byte);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v[i];
    if (byte == kMxTopByte<FMT>) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_fmed3f(x[i], -kMxTop<FMT>, kMxTop<FMT>);
    }
    if constexpr (FMT == PK_MXFP4) {
        uint32_t u = 0;
        u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[0], x[1], s, 0);
        u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[2], x[3], s, 1);
        u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[4], x[5], s, 2);
        u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[6], x[7], s, 3);
        w[0] = byte == 255u ? 0u : u;
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s16x2v u = {0, 0};
            u = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(u, x[4 * h], x[4 * h + 1], s, false);
            u = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(u, x[4 * h + 2], x[4 * h + 3], s, true);
            w[h] = byte == 255u ? 0x7F7F7F7Fu : __builtin_bit_cast(uint32_t, u);
        }
    }
}

template <int FMT>
__device__ __forceinline__ void mx_decode8(const uint32_t (&w)[FMT == PK_MXFP4 ? 1 : 2], uint32_t byte, float (&x)[8])
{
    const float s = mx_scale(byte);
    f32x2v v[4];
    if constexpr (FMT == PK_MXFP4) {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], s, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], s, 1);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], s, 2);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], s, 3);
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v[2 * h] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[h], s, false);
            v[2 * h + 1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[h], s, true);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = v[i].x; x[2 * i + 1] = v[i].y; }
}

// two fp32 numbers as bf16, to nearest, ties to even; NaN stays NaN
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    bf16x2v v;
    v.x = (__bf16)a;
    v.y = (__bf16)b;
    return __builtin_bit_cast(uint32_t, v);
}

// Up to eight elements from p on, n of them there (n >= 8: two or one wide accesses; elements may be anywhere their own
// alignment allows), zeros for the others.
template <bool BF16>
__device__ __forceinline__ void load_f8(const char* p, int n, float (&x)[8])
{
    if (n >= 8) {
        if constexpr (!BF16) {
            const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        } else {
            typedef uint32_t u32x4_b2 __attribute__((ext_vector_type(4), aligned(2)));
            const u32x4_b2 a = *reinterpret_cast<const u32x4_b2*>(p);
            const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_to_f32(u[i] & 0xFFFFu); x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u); }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = 0.f;
            if (i < n) x[i] = BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t*>(p)[i]) : reinterpret_cast<const float*>(p)[i];
        }
    }
}
template <bool BF16>
__device__ __forceinline__ void store_f8(char* p, int n, const float (&x)[8])
{
    if (n >= 8) {
        if constexpr (!BF16) {
            f32x4 a, b;
            a.x = x[0]; a.y = x[1]; a.z = x[2]; a.w = x[3]; b.x = x[4]; b.y = x[5]; b.z = x[6]; b.w = x[7];
            reinterpret_cast<f32x4*>(p)[0] = a; reinterpret_cast<f32x4*>(p)[1] = b;
        } else {
            typedef uint32_t u32x4_b2 __attribute__((ext_vector_type(4), aligned(2)));
            u32x4_b2 a;
            a.x = pack_bf16(x[0], x[1]); a.y = pack_bf16(x[2], x[3]); a.z = pack_bf16(x[4], x[5]); a.w = pack_bf16(x[6], x[7]);
            *reinterpret_cast<u32x4_b2*>(p) = a;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i >= n) break;
            if constexpr (BF16) reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)pack_bf16(x[i], 0.f);
            else reinterpret_cast<float*>(p)[i] = x[i];
        }
    }
}
