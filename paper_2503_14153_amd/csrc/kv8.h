// Cache rows in 8 bits: layout and conversions.
//
// A block is 32 rows of one head, keys and values apart. It has ONE exponent e, the least whole number with max|x| <= 448 * 2^e
// over its rows (448 is the largest e4m3 number; a block of zeros has e = 0; -100 <= e <= 120), and holds every x / 2^e rounded
// to e4m3 (OCP: 4 exponent bits, bias 7, 3 mantissa bits, no infinity), ties to even. The scale is a power of two because a
// floating format gains nothing from the bits in between, and a power of two costs nothing: the instruction that widens codes to
// bfloat16 multiplies by it, a value is exact in bfloat16, and moving a code to a block of another exponent is exact down to
// e4m3's subnormals (2^-15 of the block's largest). Infinities and NaN become the format's NaN and have no say in e.
//
// Codes lie as the attention's matrix operands (32x32x16, bfloat16) take them after widening, two contraction steps to a 16-byte
// unit, so that a wave's load instruction fetches one contiguous KiB of a block:
//   keys    K[i][lane][16]: row c, dim e: i = e/32, lane = c%32 + 32*((e/8)&1), byte 8*((e/16)&1) + e%8
//   values  V[eb][lane][16]: row c, dim e: eb = e/32, lane = e%32 + 32*((c/4)&1), byte 8*((c%32)/16) + 4*((c/8)&1) + c%4
// Exponents: two int8 per block (keys', values'), [layer][seq][head][block], a head's filled up to whole 4-byte words.
#pragma once
#include "sd_internal.h"

#define KV8_E_MIN (-100)
#define KV8_E_MAX 120

static __host__ __device__ inline size_t k8_index(int c, int e, int HD) {
    return (size_t)(c >> 5) * (32 * HD) + (((e >> 5) * 64 + (c & 31) + 32 * ((e >> 3) & 1)) << 4) + 8 * ((e >> 4) & 1) + (e & 7);
}
static __host__ __device__ inline size_t v8_index(int c, int e, int HD) {
    return (size_t)(c >> 5) * (32 * HD) + (((e >> 5) * 64 + (e & 31) + 32 * ((c >> 2) & 1)) << 4) + 8 * ((c >> 4) & 1) + 4 * ((c >> 3) & 1) +
           (c & 3);
}
// byte s of a value unit of lane half g is row v8_row(s, g) of its block
static __host__ __device__ inline int v8_row(int s, int g) { return (s >> 3) * 16 + ((s >> 2) & 1) * 8 + 4 * g + (s & 3); }

static __host__ __device__ inline size_t kv8_ex_head(int cap_blocks) { return (size_t)((cap_blocks + 1) / 2) * 4; }   // bytes

// One layer of a cache in 8 bits, or (with the strides between layers) all of them.
struct Kv8 {
    uint8_t *k, *v;
    int8_t* ex;
    int cap_blocks;
    size_t code_stride, ex_stride;       // bytes between layers
};

#ifdef __HIPCC__
// 2^e for KV8_E_MIN <= e <= KV8_E_MAX (and their negatives)
static __device__ __forceinline__ float kv8_scale(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// the exponent of a block whose largest finite magnitude is `most`
static __device__ __forceinline__ int kv8_exponent(float most) {
    const uint32_t b = __float_as_uint(most);
    if (b == 0) return 0;
    // most = 1.m * 2^x; 448 = 1.75 * 2^8 (a subnormal `most` has x far below KV8_E_MIN either way)
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return min(max(e, KV8_E_MIN), KV8_E_MAX);
}
// Four values to codes of a block whose exponent counts them: none is beyond 448 units, and what is not finite becomes NaN.
static __device__ __forceinline__ uint32_t kv8_codes(const float (&f)[4], float scale) {
    typedef __attribute__((ext_vector_type(2))) short s16x2;
    s16x2 q = {0, 0};
    q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, f[0], f[1], scale, false);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, f[2], f[3], scale, true);
    return __builtin_bit_cast(uint32_t, q);
}
// The same of rows that have no say in it (past the sequence's end): held at 448 units.
static __device__ __forceinline__ float kv8_held(float f, float scale) {
    const float most = 448.f * scale;
    return fabsf(f) < __builtin_inff() ? fminf(fmaxf(f, -most), most) : f;
}
// four codes to their values
static __device__ __forceinline__ void kv8_values(uint32_t codes, float scale, float (&f)[4]) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, true);
    f[0] = lo.x; f[1] = lo.y; f[2] = hi.x; f[3] = hi.y;
}
// eight codes to eight bfloat16 values: a matrix operand
static __device__ __forceinline__ bf16x8 kv8_widen(uint32_t c0, uint32_t c1, float scale) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    union { bf16x2 p[4]; bf16x8 v; } u;
    u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, scale, false);
    u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, scale, true);
    u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, scale, false);
    u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, scale, true);
    return u.v;
}
#endif

// ---- launchers (kv8.hip)
// natural rows [layer][nrows][nh][hd] of bfloat16 <-> one sequence's blocks, `layers` of them from c's own on
void launch_kv8_rows(const Kv8& c, void* k_rows, void* v_rows, int row0, int nrows, int nh, int hd, int seq, int layers, int to_cache,
                     hipStream_t s);
// arguments as launch_kv_commit's
void launch_kv8_commit(const void* kt_all, const void* vt_all, const Kv8& c, const int32_t* src_slots, const int32_t* n_accept,
                       const int32_t* n_old, const RowMap& rm, int L, int B, int nh, int hd, int TB, int W, hipStream_t s);
