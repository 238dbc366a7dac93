// Sequences of a cache that branch (fork) or lose rows (drop), in the three storage formats: float32 rows, bfloat16 fragments
// (sd_internal.h), e4m3 blocks (kv8.h).
#include "kv_seq.h"
#include "row_ops.h"

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// ------------------------------------------------------------------------------------------
// Fork: the source's blocks, which are contiguous per (layer, plane, head), read once and written to every copy as they are. A
// pure copy: one 16-byte load and n_dst stores per lane, FORK_U of them in flight.
// grid (pieces of a run, heads x 2 planes, layers); the run's length is the device's, the grid the host's bound.
#define FORK_U 4
__global__ __launch_bounds__(256) void k_kv_fork(KvPlanes src, KvPlanes dst, SeqList to, int n_dst, const int32_t* __restrict__ kv_len,
                                                 int src_seq, int heads, KvCarried from, KvCarried into, int n_cand) {
    const int h = blockIdx.y >> 1, plane = blockIdx.y & 1, tid = threadIdx.x;
    const int len = kv_len[src_seq];
    const int units = (len + src.unit_rows - 1) / src.unit_rows;
    const size_t run = (size_t)units * src.unit_bytes, at0 = (size_t)blockIdx.x * (256 * 16 * FORK_U) + tid * 16;
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0)
        for (int i = 0; i < n_dst; ++i) {              // what the copies carry into their next step
            const int b = to.seq[i];
            if (tid == 0) { into.kv_len[b] = len; into.root_tok[b] = from.root_tok[src_seq]; }
            for (int c = tid; c < n_cand; c += 256) into.cand[(size_t)b * n_cand + c] = from.cand[(size_t)src_seq * n_cand + c];
        }
    if (src.ex && plane == 0 && blockIdx.x == 0) {     // both planes' exponents
        const uint16_t* es = (const uint16_t*)(src.ex + blockIdx.z * src.ex_layer + ((size_t)src_seq * heads + h) * src.ex_head);
        for (int u = tid; u < units; u += 256) {
            const uint16_t v = es[u];
            for (int i = 0; i < n_dst; ++i)
                ((uint16_t*)(dst.ex + blockIdx.z * dst.ex_layer + ((size_t)to.seq[i] * heads + h) * dst.ex_head))[u] = v;
        }
    }
    const char* s = src.p[plane] + blockIdx.z * src.layer + ((size_t)src_seq * heads + h) * src.head;
    u32x4 v[FORK_U];
#pragma unroll
    for (int u = 0; u < FORK_U; ++u) {
        const size_t at = at0 + u * (256 * 16);
        if (at < run) v[u] = *(const u32x4*)(s + at);
    }
    for (int i = 0; i < n_dst; ++i) {
        char* d = dst.p[plane] + blockIdx.z * dst.layer + ((size_t)to.seq[i] * heads + h) * dst.head;
#pragma unroll
        for (int u = 0; u < FORK_U; ++u) {
            const size_t at = at0 + u * (256 * 16);
            if (at < run) *(u32x4*)(d + at) = v[u];
        }
    }
}

void launch_kv_fork(const KvPlanes& src, const KvPlanes& dst, const SeqList& to, int n_dst, const int32_t* kv_len, int src_seq,
                    int len_hi, int heads, int layers, const KvCarried& from, const KvCarried& into, int n_cand, hipStream_t s) {
    const size_t run = (size_t)((len_hi + src.unit_rows - 1) / src.unit_rows) * src.unit_bytes, piece = 256 * 16 * FORK_U;
    const unsigned x = (unsigned)((run + piece - 1) / piece);
    hipLaunchKernelGGL(k_kv_fork, dim3(x ? x : 1, heads * 2, layers), dim3(256), 0, s, src, dst, to, n_dst, kv_len, src_seq, heads, from,
                       into, n_cand);
}

// ------------------------------------------------------------------------------------------
// Drop: row j of what is left was row j + (dropped before it). Keys are rotated for the new position: R(p') = R(p' - p) R(p), one
// angle per dim pair and segment between two gaps (table[segment - 1][pair], made by k_drop_setup). The rotation is taken in
// float64 and reaches the storage format in ONE rounding (via float32 rounded to odd), so where a result lies next to a border
// of the format does not hang on how the products were taken; 4 multiply-adds per pair beside 2 loads and 2 stores do not count.
//
// Everything in place: dest rows 32 d .. of a block come from rows at or behind them, so a workgroup that walks the blocks of a
// (layer, head, plane) in order reads every row before it is overwritten (a barrier between a block's reads and its writes). That
// is one workgroup per (layer, head, plane): enough where a model has some thousand of them. Where it has fewer, `gridDim.x / nh`
// workgroups share the blocks of [d0, d1), which the host makes no longer than the shortest shift: none of them then writes what
// another one still has to read, and the launches follow one another.
static __device__ __forceinline__ float odd_float(double d) {
    const float f = (float)d;
    if ((double)f == d) return f;
    uint32_t b = __float_as_uint(f);
    if (fabs((double)f) > fabs(d)) --b;
    return __uint_as_float(b | 1u);
}
static __device__ __forceinline__ int source_row(const DropRanges& R, int j, int& segment) {
    int s = j, i = 0;
    for (; i < R.n && R.first[i] <= s; ++i) s += R.count[i];
    segment = i;
    return s;
}

__global__ void k_drop_setup(DropRanges R, const double* __restrict__ freq, int half, int32_t* __restrict__ kv_len, int seq,
                             DropState* __restrict__ st) {
    const int seg = blockIdx.x, i = threadIdx.x;
    int shift = 0;
    for (int r = 0; r <= seg; ++r) shift += R.count[r];
    if (i < half) sincos(-(double)shift * freq[i], &st->table[seg][i].y, &st->table[seg][i].x);
    if (seg == 0 && i == 0) {
        const int len = kv_len[seq];
        int gone = 0;
        for (int r = 0; r < R.n; ++r) gone += max(0, min(R.count[r], len - R.first[r]));
        st->old_len = len;
        st->new_len = len - gone;
        kv_len[seq] = len - gone;
    }
}

// ST: 0 float32, 1 bfloat16, 2 e4m3
template <int ST> struct Eight { float f[8]; };
template <int ST, int HD>
static __device__ __forceinline__ void load_row8(const char* p, int row, int e, int nh, float sc, float (&f)[8]) {
    if constexpr (ST == 0) {
        const float4 a = *(const float4*)((const float*)p + (size_t)row * nh * HD + e), b = *(const float4*)((const float*)p + (size_t)row * nh * HD + e + 4);
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    } else if constexpr (ST == 1) {
        const u16x8 v = *(const u16x8*)((const uint16_t*)p + kblk_index(row, e, HD));
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = bf16_bits_to_float(v[i]);
    } else {
        const u32x2 q = *(const u32x2*)(p + k8_index(row, e, HD));
        float a[4], b[4];
        kv8_values(q.x, sc, a);
        kv8_values(q.y, sc, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[i] = a[i]; f[4 + i] = b[i]; }
    }
}
template <int ST, int HD>
static __device__ __forceinline__ void store_row8(char* p, int row, int e, int nh, float inv, const float (&f)[8]) {
    if constexpr (ST == 0) {
        *(float4*)((float*)p + (size_t)row * nh * HD + e) = make_float4(f[0], f[1], f[2], f[3]);
        *(float4*)((float*)p + (size_t)row * nh * HD + e + 4) = make_float4(f[4], f[5], f[6], f[7]);
    } else if constexpr (ST == 1) {
        u16x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(uint16_t, (__bf16)f[i]);
        *(u16x8*)((uint16_t*)p + kblk_index(row, e, HD)) = v;
    } else {
        const float a[4] = {f[0], f[1], f[2], f[3]}, b[4] = {f[4], f[5], f[6], f[7]};
        u32x2 q;
        q.x = kv8_four(a, inv);
        q.y = kv8_four(b, inv);
        *(u32x2*)(p + k8_index(row, e, HD)) = q;
    }
}
static __device__ __forceinline__ uint32_t finite_bits(float f) {
    const uint32_t a = __float_as_uint(f) & 0x7fffffffu;
    return a < 0x7f800000u ? a : 0u;
}

template <int ST, int HD>
__global__ __launch_bounds__(256) void k_kv_drop(KvPlanes c, int seq, int nh, DropRanges R, const DropState* __restrict__ st, int d0, int d1) {
    constexpr int A = HD / 16;                         // pieces of 8 dims + their rotary partners per row
    constexpr int TW = 32 * A;                         // threads that have one
    __shared__ uint32_t most[2][4];
    __shared__ __attribute__((aligned(16))) uint16_t tile[32][HD + 8];
    const int h = blockIdx.x % nh, lanes = gridDim.x / nh, plane = blockIdx.z, tid = threadIdx.x;
    const int len = st->old_len, left = st->new_len;
    if (left == len) return;                           // nothing of it is in the ranges
    const int end = min(d1, (left + 31) >> 5);
    const int heads = ST == 0 ? 1 : nh;                // (float32: a row holds all heads)
    char* p = c.p[plane] + blockIdx.y * c.layer + ((size_t)seq * heads + (ST == 0 ? 0 : h)) * c.head + (ST == 0 ? (size_t)h * HD * 4 : 0);
    int8_t* ex = ST == 2 ? (int8_t*)(c.ex + blockIdx.y * c.ex_layer + ((size_t)seq * nh + h) * c.ex_head) + plane : nullptr;
    int turn = 0;
    for (int d = d0 + (int)blockIdx.x / nh; d < end; d += lanes, turn ^= 1) {
        const bool natural = plane == 0 || ST == 0;    // rows as pieces of dims
        float lo[8], hi[8];
        uint32_t m = 0;
        const int r = tid & 31, a = tid >> 5, j = d * 32 + r;
        if (natural) {
            const bool live = tid < TW && j < left;
#pragma unroll
            for (int i = 0; i < 8; ++i) { lo[i] = 0.f; hi[i] = 0.f; }
            if (live) {
                int seg;
                const int s = source_row(R, j, seg);
                const float sc = ST == 2 ? kv8_scale(ex[2 * (s >> 5)]) : 1.f;
                load_row8<ST, HD>(p, s, a * 8, nh, sc, lo);
                load_row8<ST, HD>(p, s, HD / 2 + a * 8, nh, sc, hi);
                if (plane == 0 && seg) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const double2 w = st->table[seg - 1][a * 8 + i];
                        const double x = lo[i], y = hi[i], u = x * w.x - y * w.y, v = x * w.y + y * w.x;
                        lo[i] = ST == 0 ? (float)u : odd_float(u);
                        hi[i] = ST == 0 ? (float)v : odd_float(v);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, max(finite_bits(lo[i]), finite_bits(hi[i])));
        } else {
            // values: a stored piece holds one dim of several rows, so the block is put together in LDS, segment by segment
            __syncthreads();                           // the tile's last readers are done
            for (int r0 = 0; r0 < 32 && d * 32 + r0 < left;) {
                int seg;
                const int s0 = source_row(R, d * 32 + r0, seg);
                int r1 = min(32, left - d * 32);       // rows [r0, r1) lie in one segment: s0 + r - r0
                if (seg < R.n) r1 = min(r1, r0 + R.first[seg] - s0);
                for (int sb = s0 >> 5; sb <= (s0 + r1 - r0 - 1) >> 5; ++sb) {
                    const int off = sb * 32 - s0 + r0;   // row c of the source block is row c + off here
                    if constexpr (ST == 2) {
                        const float sc = kv8_scale(ex[2 * sb]);
                        for (int u = tid; u < HD * 2; u += 256) {
                            const int lane = u & 63, g = lane >> 5, e = (u >> 6) * 32 + (lane & 31);
                            const u32x4 q = *(const u32x4*)(p + (size_t)sb * (32 * HD) + u * 16);
#pragma unroll
                            for (int x = 0; x < 4; ++x) {
                                float f[4];
                                kv8_values(q[x], sc, f);
#pragma unroll
                                for (int y = 0; y < 4; ++y) {
                                    const int to = v8_row(x * 4 + y, g) + off;
                                    if (to >= r0 && to < r1) tile[to][e] = __builtin_bit_cast(uint16_t, (__bf16)f[y]);
                                }
                            }
                        }
                    } else {
                        for (int u = tid; u < HD * 4; u += 256) {
                            const int lane = u & 63, g = lane >> 5, pe = u >> 6, e = (pe % (HD / 32)) * 32 + (lane & 31), half = pe / (HD / 32);
                            const u16x8 q = *(const u16x8*)((const uint16_t*)p + (size_t)sb * (32 * HD) + u * 8);
#pragma unroll
                            for (int x = 0; x < 8; ++x) {
                                const int to = half * 16 + g * 4 + (x >> 2) * 8 + (x & 3) + off;
                                if (to >= r0 && to < r1) tile[to][e] = q[x];
                            }
                        }
                    }
                }
                r0 = r1;
            }
            __syncthreads();
            if constexpr (ST == 2)
                for (int i = tid; i < min(32, left - d * 32) * (HD / 8); i += 256) {
                    const u16x8 v = *(const u16x8*)&tile[i / (HD / 8)][(i % (HD / 8)) * 8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) m = max(m, finite_bits(bf16_bits_to_float(v[x])));
                }
        }
        int e = 0;
        if constexpr (ST == 2) {
#pragma unroll
            for (int o = 32; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
            if ((tid & 63) == 0) most[turn][tid >> 6] = m;
        }
        __syncthreads();                               // every row of this block has been read
        if constexpr (ST == 2) {
            e = kv8_exponent(__uint_as_float(max(max(most[turn][0], most[turn][1]), max(most[turn][2], most[turn][3]))));
            if (tid == 0) ex[2 * d] = (int8_t)e;
        }
        const float inv = kv8_scale(-e);
        if (natural) {
            // (rows past the end: e4m3 zeros, as their block has a new exponent; the other formats leave them as they are)
            if (tid < TW && (ST == 2 || j < left)) {
                store_row8<ST, HD>(p, j, a * 8, nh, inv, lo);
                store_row8<ST, HD>(p, j, HD / 2 + a * 8, nh, inv, hi);
            }
        } else if constexpr (ST == 2) {
            for (int u = tid; u < HD * 2; u += 256) {
                const int lane = u & 63, g = lane >> 5, dim = (u >> 6) * 32 + (lane & 31);
                u32x4 q;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    float f[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const int row = v8_row(x * 4 + y, g);
                        f[y] = d * 32 + row < left ? bf16_bits_to_float(tile[row][dim]) : 0.f;
                    }
                    q[x] = kv8_four(f, inv);
                }
                *(u32x4*)(p + (size_t)d * (32 * HD) + u * 16) = q;
            }
        } else if constexpr (ST == 1) {
            for (int u = tid; u < HD * 4; u += 256) {
                const int lane = u & 63, g = lane >> 5, pe = u >> 6, dim = (pe % (HD / 32)) * 32 + (lane & 31), half = pe / (HD / 32);
                u16x8* to = (u16x8*)((uint16_t*)p + (size_t)d * (32 * HD) + u * 8);
                u16x8 q = *to;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int row = half * 16 + g * 4 + (x >> 2) * 8 + (x & 3);
                    if (d * 32 + row < left) q[x] = tile[row][dim];
                }
                *to = q;
            }
        }
    }
}

void launch_kv_drop(int storage, const KvPlanes& c, int seq, int nh, int hd, int layers, const DropRanges& R, const double* freq,
                    int32_t* kv_len, int len_hi, DropState* st, hipStream_t s) {
    hipLaunchKernelGGL(k_drop_setup, dim3(R.n), dim3(64), 0, s, R, freq, hd / 2, kv_len, seq, st);
    int left = len_hi;                                 // the host's bound: what is left of the longest it may be
    for (int i = 0; i < R.n; ++i) left -= R.count[i] < len_hi - R.first[i] ? R.count[i] : (len_hi > R.first[i] ? len_hi - R.first[i] : 0);
    const int d0 = R.first[0] >> 5, d1 = (left + 31) >> 5, shift = R.count[0] >> 5;
    // Runs of `shift` blocks, all at once in each, where one workgroup per (layer, head, plane) would leave the chip half empty and
    // the runs are few; else one launch in which every workgroup walks its blocks in order.
    const int walkers = layers * nh * 2;
    const bool runs = shift > 1 && walkers < 2048 && (d1 - d0 + shift - 1) / shift <= 32;
    for (int d = d0; d < d1; d += runs ? shift : d1 - d0) {
        const int e = runs ? (d + shift < d1 ? d + shift : d1) : d1;
        const dim3 grid(nh * (runs ? e - d : 1), layers, 2);
#define DROP(ST_, HD_) hipLaunchKernelGGL((k_kv_drop<ST_, HD_>), grid, dim3(256), 0, s, c, seq, nh, R, st, d, e)
#define DROP2(ST_) do { if (hd == 128) DROP(ST_, 128); else DROP(ST_, 64); } while (0)
        if (storage == 0) DROP2(0);
        else if (storage == 1) DROP2(1);
        else DROP2(2);
#undef DROP2
#undef DROP
    }
}
