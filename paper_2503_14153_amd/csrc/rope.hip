// Rotary embedding of natural rows (queries, keys; or, inverse, their gradients): every pair of dims of a head turned by
// position * frequency. Bound by reading and writing the rows: the angles, taken in float64 (turns, reduced before they are
// rounded), are made once per row and workgroup, in LDS, and serve all heads of the row. 16384 rows of 32 heads of 128 dims in bfloat16,
// out of place: 268 MB read, 268 MB written in 98 us, 5.5 TB/s (a large copy: 5.2); up to some 64 rows it is one launch, 3.5 us.
#include "rope.h"
#include "row_ops.h"

#include <algorithm>

// how a workgroup's rows and heads are cut: enough workgroups to fill the chip, and rows enough to share the angles' set-up
#define ROPE_ROWS 4

template <class T> struct RopeIo;
template <> struct RopeIo<float> {
    static __device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
        const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    static __device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
        *(float4*)p = make_float4(f[0], f[1], f[2], f[3]);
        *(float4*)(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
    }
    static __device__ __forceinline__ float load(const float* p) { return *p; }
    static __device__ __forceinline__ void store(float* p, float f) { *p = f; }
};
template <> struct RopeIo<uint16_t> {
    typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ void load8(const uint16_t* p, float (&f)[8]) {
        const u16x8 v = *(const u16x8*)p;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = bf16_bits_to_float(v[i]);
    }
    static __device__ __forceinline__ void store8(uint16_t* p, const float (&f)[8]) {
        u16x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(uint16_t, (__bf16)f[i]);
        *(u16x8*)p = v;
    }
    static __device__ __forceinline__ float load(const uint16_t* p) { return bf16_bits_to_float(*p); }
    static __device__ __forceinline__ void store(uint16_t* p, float f) { *p = __builtin_bit_cast(uint16_t, (__bf16)f); }
};

// (a, b) -> (a cos - b sin, a sin + b cos)
static __device__ __forceinline__ void turn(float& a, float& b, float2 w) {
    const float x = a * w.x - b * w.y, y = a * w.y + b * w.x;
    a = x;
    b = y;
}

// grid (row groups of `per`, head groups of `heads_per`). VEC: eight dims at a time (the launcher has looked at alignment and sizes)
template <class T, bool INTERLEAVED, bool VEC>
__global__ __launch_bounds__(256) void k_rope_rows(const T* x, T* y, const int32_t* __restrict__ pos, RopeTable f, int n, int heads,
                                                   int heads_per, int hd, int64_t ldx, int64_t ldy, int per) {
    __shared__ float2 cs[ROPE_ROWS][ROPE_MAX_DIM / 2];
    typedef RopeIo<T> Io;
    const int tid = threadIdx.x, rd = f.rotary, half = rd / 2, r0 = blockIdx.x * per, rows = min(per, n - r0);
    const int h0 = blockIdx.y * heads_per, nh = min(heads_per, heads - h0);
    for (int i = tid; i < rows * half; i += 256) {
        const int r = i / half, k = i - r * half;
        const double t = (double)pos[r0 + r] * f.turns[k];
        float s, c;
        sincospif(2.f * (float)(t - rint(t)), &s, &c);
        cs[r][k] = make_float2(c * f.magnitude, s * f.magnitude);
    }
    __syncthreads();
    // a head's items: its rotated pairs, eight or one at a time, then (unless in place) the dims that pass through
    const int W = VEC ? 8 : 1, turned = INTERLEAVED && VEC ? rd / 8 : half / W, items = turned + (x == y ? 0 : (hd - rd) / W);
    for (int i = tid; i < rows * nh * items; i += 256) {
        const int rh = i / items, it = i - rh * items, r = rh / nh, h = h0 + rh - r * nh;
        const T* px = x + (r0 + r) * ldx + (int64_t)h * hd;
        T* py = y + (r0 + r) * ldy + (int64_t)h * hd;
        if constexpr (VEC) {
            float a[8], b[8];
            if (it >= turned) {
                const int e = rd + (it - turned) * 8;
                Io::load8(px + e, a);
                Io::store8(py + e, a);
            } else if constexpr (INTERLEAVED) {
                Io::load8(px + it * 8, a);
#pragma unroll
                for (int k = 0; k < 4; ++k) turn(a[2 * k], a[2 * k + 1], cs[r][it * 4 + k]);
                Io::store8(py + it * 8, a);
            } else {
                Io::load8(px + it * 8, a);
                Io::load8(px + half + it * 8, b);
#pragma unroll
                for (int k = 0; k < 8; ++k) turn(a[k], b[k], cs[r][it * 8 + k]);
                Io::store8(py + it * 8, a);
                Io::store8(py + half + it * 8, b);
            }
        } else if (it >= turned) {
            const int e = rd + it - turned;
            py[e] = px[e];
        } else {
            const int ea = INTERLEAVED ? 2 * it : it, eb = INTERLEAVED ? ea + 1 : half + it;
            float a = Io::load(px + ea), b = Io::load(px + eb);
            turn(a, b, cs[r][it]);
            Io::store(py + ea, a);
            Io::store(py + eb, b);
        }
    }
}

void launch_rope_rows(const void* x, void* y, const int32_t* pos, const RopeTable& f, int f32, int interleaved, int n, int heads, int hd,
                      int64_t ldx, int64_t ldy, hipStream_t s) {
    const int align = f32 ? 4 : 8, rd = f.rotary;      // elements of 16 bytes
    const bool vec = ((((uintptr_t)x) | ((uintptr_t)y)) & 15) == 0 && ldx % align == 0 && ldy % align == 0 && hd % 8 == 0 &&
                     rd % (interleaved ? 8 : 16) == 0;
    // A workgroup's (row, head) pairs: 32 or so pay for its angles (16384 rows of 8 heads, 128 dims of bfloat16: four rows 12.2 us, one
    // 14.8; of 64 heads: four 104, one 94), where rows fill the chip that way; else one row, its heads dealt out (64 rows of 64 heads: 3.6
    // us, 3.9 in a workgroup).
    const int most = heads >= 32 ? 1 : heads >= 16 ? 2 : ROPE_ROWS, per = n >= 512 * most ? most : 1, groups = (n - 1) / per + 1;
    const int hg = groups >= 512 ? 1 : 512 / groups, hp = (heads + hg - 1) / hg;
    const int step = 1 << 20;                          // rows a launch (a grid's limit)
#define ROPE(T_, I_, V_)                                                                                               \
    for (int r = 0; r < n; r += std::min(step, n - r)) {                                                               \
        const int some = std::min(step, n - r);                                                                        \
        hipLaunchKernelGGL((k_rope_rows<T_, I_, V_>), dim3((some - 1) / per + 1, (heads + hp - 1) / hp), dim3(256), 0, s, \
                           (const T_*)x + r * ldx, (T_*)y + r * ldy, pos + r, f, some, heads, hp, hd, ldx, ldy, per);   \
    }
#define ROPE2(T_, I_) do { if (vec) { ROPE(T_, I_, true) } else { ROPE(T_, I_, false) } } while (0)
    if (f32) { if (interleaved) ROPE2(float, true); else ROPE2(float, false); }
    else     { if (interleaved) ROPE2(uint16_t, true); else ROPE2(uint16_t, false); }
#undef ROPE2
#undef ROPE
}

// the model's own table: its steps' frequencies, and behind them the magnitude
__global__ void k_set_rope(RopeTable f, double* __restrict__ freq) {
    const int i = threadIdx.x;
    if (i < f.rotary / 2) freq[i] = f.turns[i];
    else if (i == f.rotary / 2) freq[i] = (double)f.magnitude;
}
void launch_set_rope(const RopeTable& f, double* freq, hipStream_t s) {
    hipLaunchKernelGGL(k_set_rope, dim3(1), dim3(ROPE_MAX_DIM / 2 + 64), 0, s, f, freq);
}
