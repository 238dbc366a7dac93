// Rows into and out of a cache of 8 bits (layout and rounding: kv8.h). One workgroup owns one block of one head, keys and values.
// All of it is a stream: bfloat16 rows in, half their bytes out, or the other way round; a block that keeps some of its rows is
// widened, patched and rounded again, which changes no kept value (kv8.h), so appending never loses anything by degrees.
//
// Rows pass through LDS as bfloat16, which holds old and new values exactly: natural rows are read and written as whole 16-byte
// pieces of 2 * head_dim contiguous bytes, codes as 16-byte units, and the value units (sixteen rows of one dim) are turned there.
// 16384 rows of 32 heads of 128 dims, 402 MB read and written: into the cache 84 - 87 us, out of it 67 - 71 (a copy of as many bytes: 77).
#include "kv8.h"
#include "row_ops.h"

#include <algorithm>

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

static __device__ __forceinline__ uint16_t bf16_bits(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

template <int HD>
struct RowTile { uint16_t t[2][32][HD + 8]; };         // keys, values; rows padded by 16 bytes: columns spread over the banks

// Rows of the block that keep() to the tile, from their codes.
template <int HD, class Keep>
static __device__ __forceinline__ void kept_rows(RowTile<HD>& tile, const uint8_t* kb, const uint8_t* vb, int ek, int ev, Keep&& keep) {
    constexpr int U = HD * 2;                          // 16-byte units of a block
    for (int u = threadIdx.x; u < 2 * U; u += 256) {
        const int plane = u / U, w = u - plane * U, i = w >> 6, lane = w & 63, g = lane >> 5;
        const u32x4 q = *(const u32x4*)((plane ? vb : kb) + (size_t)w * 16);
        const float sc = kv8_scale(plane ? ev : ek);
        if (plane == 0 && !keep(lane & 31)) continue;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            float f[4];
            kv8_values(q[d], sc, f);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int s = d * 4 + x;
                if (plane == 0) tile.t[0][lane & 31][i * 32 + 16 * (s >> 3) + 8 * g + (s & 7)] = bf16_bits(f[x]);
                else if (keep(v8_row(s, g))) tile.t[1][v8_row(s, g)][i * 32 + (lane & 31)] = bf16_bits(f[x]);
            }
        }
    }
}

static __device__ __forceinline__ uint32_t largest_of(const u16x8& v) {
    uint32_t m = v[0];
#pragma unroll
    for (int x = 1; x < 8; ++x) m = max(m, (uint32_t)v[x]);
    return m;
}

// The tile's exponents from its first `valid` rows (those that count), the codes of all 32. Every thread of the workgroup calls it.
template <int HD>
static __device__ __forceinline__ void encode_block(const RowTile<HD>& tile, uint8_t* kb, uint8_t* vb, int8_t* ex, int valid) {
    constexpr int U = HD * 2, PC = HD / 8;
    __shared__ uint32_t most[2][4];
    const int tid = threadIdx.x;
    __syncthreads();                                   // the tile is whole
    uint32_t m[2];                                     // largest finite magnitude, as bits: they order like the numbers
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        u16x8 v8 = {0, 0, 0, 0, 0, 0, 0, 0};
        for (int i = tid; i < valid * PC; i += 256)
            v8 = __builtin_elementwise_max(v8, *(const u16x8*)&tile.t[p][i / PC][(i % PC) * 8] & (u16x8)(0x7fff));
        m[p] = largest_of(v8);
        if (__any(m[p] >= 0x7f80u)) {                  // infinities or NaN among them (rare): without those
            u16x8 f8 = {0, 0, 0, 0, 0, 0, 0, 0};
            for (int i = tid; i < valid * PC; i += 256) {
                const u16x8 v = *(const u16x8*)&tile.t[p][i / PC][(i % PC) * 8] & (u16x8)(0x7fff);
#pragma unroll
                for (int x = 0; x < 8; ++x) f8[x] = v[x] < 0x7f80u && v[x] > f8[x] ? v[x] : f8[x];
            }
            m[p] = largest_of(f8);
        }
#pragma unroll
        for (int o = 32; o; o >>= 1) m[p] = max(m[p], (uint32_t)__shfl_xor((int)m[p], o));
        if ((tid & 63) == 0) most[p][tid >> 6] = m[p];
    }
    __syncthreads();
    int e[2];
#pragma unroll
    for (int p = 0; p < 2; ++p)
        e[p] = kv8_exponent(__uint_as_float(max(max(most[p][0], most[p][1]), max(most[p][2], most[p][3])) << 16));
    if (tid < 2) ex[tid] = (int8_t)e[tid];
    for (int u = tid; u < 2 * U; u += 256) {
        const int p = u / U, w = u - p * U, i = w >> 6, lane = w & 63, g = lane >> 5;
        const float unit = kv8_scale(e[p]);
        u32x4 q;
        if (p == 0) {
            const u16x8 a = *(const u16x8*)&tile.t[0][lane & 31][i * 32 + 8 * g], b = *(const u16x8*)&tile.t[0][lane & 31][i * 32 + 16 + 8 * g];
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                float f[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) f[x] = bf16_bits_to_float(d < 2 ? a[d * 4 + x] : b[(d - 2) * 4 + x]);
                if (valid < 32)
#pragma unroll
                    for (int x = 0; x < 4; ++x) f[x] = (lane & 31) < valid ? f[x] : kv8_held(f[x], unit);
                q[d] = kv8_codes(f, unit);
            }
        } else {
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                float f[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) f[x] = bf16_bits_to_float(tile.t[1][v8_row(d * 4 + x, g)][i * 32 + (lane & 31)]);
                if (valid < 32)
#pragma unroll
                    for (int x = 0; x < 4; ++x) f[x] = v8_row(d * 4 + x, g) < valid ? f[x] : kv8_held(f[x], unit);
                q[d] = kv8_codes(f, unit);
            }
        }
        *(u32x4*)((p ? vb : kb) + (size_t)w * 16) = q;
    }
}

// ------------------------------------------------------------------------------------------
// Natural rows [layer][nrows][nh][hd] <-> one sequence's blocks, grid (heads, blocks, layers): the heads of a row lie side by side in
// natural memory, so they are taken side by side (blocks first: 115 us into the cache instead of 87). VEC: the caller's arrays are
// 16-byte aligned; else they are read and written by elements.
template <bool VEC>
static __device__ __forceinline__ u16x8 piece_from(const uint16_t* p) {
    if constexpr (VEC) return *(const u16x8*)p;
    u16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[i];
    return v;
}
template <bool VEC>
static __device__ __forceinline__ void piece_to(uint16_t* p, const u16x8& v) {
    if constexpr (VEC) { *(u16x8*)p = v; return; }
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = v[i];
}
template <int HD, bool TO_CACHE, bool VEC>
__global__ __launch_bounds__(256) void k_kv8_rows(Kv8 c, uint16_t* __restrict__ k_rows, uint16_t* __restrict__ v_rows, int row0, int nrows,
                                                  int nh, int seq, int b0) {
    constexpr int PC = HD / 8;
    __shared__ __attribute__((aligned(16))) RowTile<HD> tile;
    const int blk = (row0 >> 5) + b0 + blockIdx.y, h = blockIdx.x, tid = threadIdx.x;
    const size_t at = ((size_t)seq * nh + h) * c.cap_blocks + blk;
    uint8_t* kb = c.k + blockIdx.z * c.code_stride + at * (32 * HD);
    uint8_t* vb = c.v + blockIdx.z * c.code_stride + at * (32 * HD);
    int8_t* ex = c.ex + blockIdx.z * c.ex_stride + ((size_t)seq * nh + h) * kv8_ex_head(c.cap_blocks) + blk * 2;
    const int first = blk * 32 - row0;                 // natural row of the block's row 0 (negative: before the range)
    const size_t layer = (size_t)blockIdx.z * nrows;
    auto asked = [&](int r) { return first + r >= 0 && first + r < nrows; };
    auto nat = [&](int r) { return ((layer + first + r) * nh + h) * HD; };
    const bool all = first >= 0 && first + 32 <= nrows;
    if constexpr (TO_CACHE) {
        for (int i = tid; i < 2 * 32 * PC; i += 256) {
            const int p = i / (32 * PC), r = (i / PC) & 31, e = (i % PC) * 8;
            if (asked(r)) *(u16x8*)&tile.t[p][r][e] = piece_from<VEC>((p ? v_rows : k_rows) + nat(r) + e);
        }
        if (!all) kept_rows<HD>(tile, kb, vb, ex[0], ex[1], [&](int r) { return !asked(r); });
        encode_block<HD>(tile, kb, vb, ex, 32);        // (its first barrier: nobody writes codes before everybody has read them)
    } else {
        kept_rows<HD>(tile, kb, vb, ex[0], ex[1], asked);
        __syncthreads();
        for (int i = tid; i < 2 * 32 * PC; i += 256) {
            const int p = i / (32 * PC), r = (i / PC) & 31, e = (i % PC) * 8;
            if (asked(r)) piece_to<VEC>((p ? v_rows : k_rows) + nat(r) + e, *(const u16x8*)&tile.t[p][r][e]);
        }
    }
}

void launch_kv8_rows(const Kv8& c, void* k_rows, void* v_rows, int row0, int nrows, int nh, int hd, int seq, int layers, int to_cache,
                     hipStream_t s) {
    const int blocks = (row0 + nrows - 1) / 32 - row0 / 32 + 1, step = 32768;      // (a grid's second axis has 65535)
    const bool vec = ((((uintptr_t)k_rows) | ((uintptr_t)v_rows)) & 15) == 0;
#define KV8_ROWS(HD_, TO_, VEC_)                                                                                       \
    for (int b0 = 0; b0 < blocks; b0 += step)                                                                          \
        hipLaunchKernelGGL((k_kv8_rows<HD_, TO_, VEC_>), dim3(nh, std::min(step, blocks - b0), layers), dim3(256), 0, s, c, \
                           (uint16_t*)k_rows, (uint16_t*)v_rows, row0, nrows, nh, seq, b0)
#define KV8_ROWS2(HD_, TO_) do { if (vec) KV8_ROWS(HD_, TO_, true); else KV8_ROWS(HD_, TO_, false); } while (0)
    if (hd == 128) { if (to_cache) KV8_ROWS2(128, true); else KV8_ROWS2(128, false); }
    else           { if (to_cache) KV8_ROWS2(64, true);  else KV8_ROWS2(64, false); }
#undef KV8_ROWS2
#undef KV8_ROWS
}

// ------------------------------------------------------------------------------------------
// Commit: the accepted rows of the tree scratch (bfloat16 fragments, as k_kv_commit takes them) appended to every sequence.
// grid (heads, sequences of the pass, layers * blocks that the widest commit can touch); rows past the new length have no say in
// the exponent.
template <int HD>
__global__ __launch_bounds__(256) void k_kv8_commit(const uint16_t* __restrict__ kt, const uint16_t* __restrict__ vt, Kv8 c,
                                                    const int32_t* __restrict__ src_slots, const int32_t* __restrict__ n_accept,
                                                    const int32_t* __restrict__ n_old, RowMap rm, int nh, int TB, int W, int nb,
                                                    size_t layer_stride_t) {
    constexpr int PC = HD / 8;
    __shared__ __attribute__((aligned(16))) RowTile<HD> tile;
    const int h = blockIdx.x, b = blockIdx.y, l = blockIdx.z / nb, tid = threadIdx.x;
    const int lst = rm.off[b] & 255, last = rm.off[b] >> 8;        // whose list, count and old length these are; its last row
    const int a = min(n_accept[lst], W), n = n_old[lst];
    const int blk = (n >> 5) + blockIdx.z % nb, lo = n - blk * 32, hi = n + a - blk * 32;      // new rows of the block: lo <= r < hi
    if (a <= 0 || hi <= 0 || blk >= c.cap_blocks) return;
    const size_t at = ((size_t)rm.seq[b] * nh + h) * c.cap_blocks + blk;
    uint8_t* kb = c.k + l * c.code_stride + at * (32 * HD);
    uint8_t* vb = c.v + l * c.code_stride + at * (32 * HD);
    int8_t* ex = c.ex + l * c.ex_stride + ((size_t)rm.seq[b] * nh + h) * kv8_ex_head(c.cap_blocks) + blk * 2;
    const size_t src = l * layer_stride_t + ((size_t)b * nh + h) * TB * (32 * HD);
    auto fresh = [&](int r) { return r >= lo && r < hi; };
    auto slot = [&](int r) { return min(max(src_slots[(size_t)lst * W + r - lo], 0), last); };
    for (int i = tid; i < 32 * PC; i += 256) {         // keys: 16-byte pieces, neighbouring rows 16 bytes apart
        const int r = i & 31, e = (i >> 5) * 8;
        if (fresh(r)) *(u16x8*)&tile.t[0][r][e] = *(const u16x8*)(kt + src + kblk_index(slot(r), e, HD));
    }
    for (int i = tid; i < 32 * HD; i += 256) {         // values: one dim of eight rows to a piece, of which any may be wanted
        const int r = i / HD, e = i % HD;
        if (fresh(r)) tile.t[1][r][e] = vt[src + vblk_index(slot(r), e, HD)];
    }
    if (lo > 0 || hi < 32) kept_rows<HD>(tile, kb, vb, ex[0], ex[1], [&](int r) { return !fresh(r); });
    encode_block<HD>(tile, kb, vb, ex, min(hi, 32));
}

void launch_kv8_commit(const void* kt_all, const void* vt_all, const Kv8& c, const int32_t* src_slots, const int32_t* n_accept,
                       const int32_t* n_old, const RowMap& rm, int L, int B, int nh, int hd, int TB, int W, hipStream_t s) {
    const size_t lst = (size_t)B * nh * TB * 32 * hd;
    const int nb = (W + 30) / 32 + 1;                  // blocks that W rows can lie in
#define KV8_COMMIT(HD_)                                                                                                \
    hipLaunchKernelGGL((k_kv8_commit<HD_>), dim3(nh, B, L * nb), dim3(256), 0, s, (const uint16_t*)kt_all, (const uint16_t*)vt_all, c, \
                       src_slots, n_accept, n_old, rm, nh, TB, W, nb, lst)
    if (hd == 128) KV8_COMMIT(128); else KV8_COMMIT(64);
#undef KV8_COMMIT
}
