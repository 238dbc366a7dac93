// Sequences of a cache that branch (fork) or lose rows (drop), in the three storage formats: float32 rows, bfloat16 fragments
// (sd_internal.h), e4m3 blocks (kv8.h).
#include "kv_seq.h"
#include "row_ops.h"

#include <algorithm>

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// ------------------------------------------------------------------------------------------
// Fork: the source's blocks, which are contiguous per (layer, plane, head), read once and written to every copy as they are. A
// pure copy: one 16-byte load and n_dst stores per lane, FORK_U of them in flight. 16384 rows of 4 layers, 32 heads of 128 dims, in 8
// bits, to one sequence: 537 MB read and as many written in 190 - 205 us, 5.2 - 5.6 TB/s, what a large copy reaches.
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
// float64 and reaches the storage format in ONE rounding (via float32 rounded to odd where that matters), so where a result lies next
// to a border of the format does not hang on how the products were taken.
//
// Everything in place: dest rows 32 d .. of a block come from rows at or behind them, so a workgroup that walks the blocks of a
// (layer, head, plane) in order, G at a time, has read every row before it is overwritten (a barrier between the reads of G
// blocks and their writes). That is one workgroup per (layer, head, plane): enough where a model has a thousand of them.
// Where it has fewer, the blocks go in runs of [d0, d1), which the host makes no longer than the shortest shift: a run has a
// workgroup for every turn of G blocks, none of which then writes what another one still has to read, and the runs' launches follow
// one another.
//
// Bound: a run by loads, stores and some 350 vector instructions a wave and block together (the float64 turn is a third of them): 128
// blocks of 4 layers, 32 heads of 128 dims, 268 MB in 85 - 92 us, 51 at the copy rate. A walk by its turns, each a chain of memory round
// trips and the conversions of one workgroup, some 4 us: 130 of 700 rows of the same, 18 blocks, four at a time, 27 us. A walk's V blocks
// of several shifts go by themselves, through LDS (a whole turn of four that way: 3 us more).
// d rounded to odd: cut to 24 bits, the last one set if anything was cut, so that a later rounding to fewer bits sees on which side
// of a border d lies. (From the bits: below 29 bits of a float64's fraction, a float32's ends.)
static __device__ __forceinline__ float odd_float(double d) {
    const uint64_t b = (uint64_t)__double_as_longlong(d);
    const uint32_t lo = (uint32_t)b, cut = lo & 0x1fffffffu;
    const uint32_t kept = (lo & 0xe0000000u) | ((cut + 0x1fffffffu) & 0x20000000u);
    return (float)__longlong_as_double((long long)((b & 0xffffffff00000000ull) | kept));
}
// Where rows come from. Lane i has the first row of what is left that comes from behind range i (none: INT_MAX), and how many rows are
// gone by then, so a row that is the same for the whole wave takes a ballot, and one per lane a compare for each range.
struct Gaps { int from, gone; };
static __device__ __forceinline__ Gaps gaps_of(const DropRanges& R) {
    const int lane = threadIdx.x & 63;
    Gaps g = {0x7fffffff, 0};
    int before = 0;
    for (int i = 0; i < R.n; ++i) {
        if (lane == i) g = {R.first[i] - before, before + R.count[i]};
        before += R.count[i];
    }
    return g;
}
static __device__ __forceinline__ int segment_at(const Gaps& g, int j) {
    return (int)__popcll(__ballot(g.from <= __builtin_amdgcn_readfirstlane(j)));
}
static __device__ __forceinline__ int gone_before(const Gaps& g, int segment) {
    return segment ? __builtin_amdgcn_readlane(g.gone, segment - 1) : 0;
}
static __device__ __forceinline__ int source_row(const Gaps& g, int n, int j, int& segment) {      // (all lanes of the wave)
    segment = 0;
    int s = j;
    for (int i = 0; i < n; ++i) {
        const bool behind = __builtin_amdgcn_readlane(g.from, i) <= j;
        const int gone = __builtin_amdgcn_readlane(g.gone, i);
        segment += behind ? 1 : 0;
        s = behind ? j + gone : s;
    }
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

// ST: 0 float32, 1 bfloat16, 2 e4m3. Eight dims of a row as the first two store them.
template <int ST> struct Raw { u32x4 a, b; };
template <> struct Raw<1> { u16x8 a; };
template <int ST, int HD>
static __device__ __forceinline__ Raw<ST> load_row8(const char* p, int row, int e, int nh) {
    Raw<ST> r;
    if constexpr (ST == 0) {
        r.a = *(const u32x4*)((const float*)p + (size_t)row * nh * HD + e);
        r.b = *(const u32x4*)((const float*)p + (size_t)row * nh * HD + e + 4);
    } else if constexpr (ST == 1) {
        r.a = *(const u16x8*)((const uint16_t*)p + kblk_index(row, e, HD));
    }
    return r;
}
template <int ST>
static __device__ __forceinline__ void row8_values(const Raw<ST>& r, float (&f)[8]) {
    if constexpr (ST == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[i] = __uint_as_float(r.a[i]); f[4 + i] = __uint_as_float(r.b[i]); }
    } else if constexpr (ST == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = bf16_bits_to_float(r.a[i]);
    }
}
template <int ST, int HD>
static __device__ __forceinline__ void store_row8(char* p, int row, int e, int nh, const float (&f)[8]) {
    if constexpr (ST == 0) {
        *(float4*)((float*)p + (size_t)row * nh * HD + e) = make_float4(f[0], f[1], f[2], f[3]);
        *(float4*)((float*)p + (size_t)row * nh * HD + e + 4) = make_float4(f[4], f[5], f[6], f[7]);
    } else if constexpr (ST == 1) {
        u16x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(uint16_t, (__bf16)f[i]);
        *(u16x8*)((uint16_t*)p + kblk_index(row, e, HD)) = v;
    }
}
// Eight pairs turned by the table's angles. A border between two numbers of a narrower format has its last 15 bits clear (bfloat16;
// e4m3 19, of which 16 are looked at): where a float32 result has not, its own rounding decided nothing.
template <int ST>
static __device__ __forceinline__ void turn_pairs(const double2* __restrict__ table, float (&x)[8], float (&y)[8]) {
    const uint32_t keep = ST == 1 ? 0x7fffu : 0xffffu;
    uint16_t low = 0xffffu;
    float u[8], v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const double2 w = table[k];
        u[k] = (float)(x[k] * w.x - y[k] * w.y);
        v[k] = (float)(x[k] * w.y + y[k] * w.x);
        const uint16_t lu = (uint16_t)(__float_as_uint(u[k]) & keep), lv = (uint16_t)(__float_as_uint(v[k]) & keep);
        low = low < lu ? low : lu;
        low = low < lv ? low : lv;
    }
    if (ST != 0 && low == 0) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const double2 w = table[k];
            u[k] = odd_float(x[k] * w.x - y[k] * w.y);
            v[k] = odd_float(x[k] * w.y + y[k] * w.x);
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) { x[k] = u[k]; y[k] = v[k]; }
}
// Values that come from codes are finite or NaN, and a maximum of floats takes no NaN: the plain instruction does.
static __device__ __forceinline__ float larger(float m, float a, float b) { return fmaxf(fmaxf(m, fabsf(a)), fabsf(b)); }
// The largest of the workgroup's magnitudes for each of G blocks -> exponents. One barrier, which also ends the reads of
// those blocks. `most` alternates between turns: the one before it may still be read.
template <int G, int W>
static __device__ __forceinline__ void exponents_of(float (&m)[G], float (*most)[W], int (&e)[G]) {
#pragma unroll
    for (int i = 0; i < G; ++i) {
#pragma unroll
        for (int o = 32; o; o >>= 1) m[i] = fmaxf(m[i], __shfl_xor(m[i], o));
        if ((threadIdx.x & 63) == 0) most[i][threadIdx.x >> 6] = m[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < G; ++i) {
        float x = most[i][0];
#pragma unroll
        for (int w = 1; w < W; ++w) x = fmaxf(x, most[i][w]);
        e[i] = kv8_exponent(x);
    }
}

// Does block b lie in one segment?
static __device__ __forceinline__ bool one_shift(const Gaps& g, int b, int left) {
    return segment_at(g, b * 32) == segment_at(g, min(b * 32 + 31, left - 1));
}

// Blocks a turn. Codes: as many as give every thread two units (one dim's rows). The others: two, for registers (16384 rows of bfloat16 less 4096: 468 us
// with two, 542 with four).
static constexpr int drop_blocks(int storage, int HD, int threads) { return storage == 2 ? threads / HD : 2; }

template <int ST, int HD, int G, int TH>
__global__ __launch_bounds__(TH, 4) void k_kv_drop(KvPlanes c, int seq, int nh, DropRanges R, const DropState* __restrict__ st, int d0, int d1) {
    constexpr int A = HD / 16;                         // pieces of 8 dims + their rotary partners per row
    constexpr int TW = 32 * A;                         // threads that have one
    constexpr bool TILES = ST != 0;                    // values are stored turned: several rows of one dim to a piece
    __shared__ float most[2][G][TH / 64];
    __shared__ __attribute__((aligned(16))) uint16_t tile[TILES ? G : 1][32][HD + 8];
    const int h = blockIdx.x % nh, walkers = gridDim.x / nh, plane = blockIdx.z, tid = threadIdx.x;
    const int len = st->old_len, left = st->new_len;
    if (left == len) return;                           // nothing of it is in the ranges
    const int end = min(d1, (left + 31) >> 5);
    const int heads = ST == 0 ? 1 : nh;                // (float32: a row holds all heads)
    char* p = c.p[plane] + blockIdx.y * c.layer + ((size_t)seq * heads + (ST == 0 ? 0 : h)) * c.head + (ST == 0 ? (size_t)h * HD * 4 : 0);
    int8_t* ex = ST == 2 ? (int8_t*)(c.ex + blockIdx.y * c.ex_layer + ((size_t)seq * nh + h) * c.ex_head) + plane : nullptr;
    const Gaps gaps = gaps_of(R);
    int turn = 0, d = d0 + ((int)blockIdx.x / nh) * G, last = min(d + G, end);
    for (int stop; d < end; turn ^= 1, d = stop) {     // blocks [d, stop) of this workgroup's [.., last)
        if (d == last) {
            d += (walkers - 1) * G;
            last = min(d + G, end);
            if (d >= end) break;
        }
        asm("" : "+s"(d));                             // (else every row's distance from the end is a register that is counted along)
        stop = last;
        if (ST == 2 && plane == 1) {                   // blocks of one shift each, or one of several
            stop = d + 1;
            if (one_shift(gaps, d, left))
                while (stop < last && one_shift(gaps, stop, left)) ++stop;
        }
        float m[G] = {};
        int e[G] = {};
        if (ST != 2 && (plane == 0 || !TILES)) {       // rows as pieces of dims
            const int r = tid & 31, a = tid >> 5;
            Raw<ST> lo[G], hi[G];
            int seg[G];
#pragma unroll
            for (int i = 0; i < G; ++i) {
                const int j = (d + i) * 32 + r;
                const int s = source_row(gaps, R.n, j, seg[i]);
                if (!(tid < TW && d + i < stop && j < left)) seg[i] = -1;
                else {
                    lo[i] = load_row8<ST, HD>(p, s, a * 8, nh);
                    hi[i] = load_row8<ST, HD>(p, s, HD / 2 + a * 8, nh);
                }
            }
            float f[G][16];
#pragma unroll
            for (int i = 0; i < G; ++i) {
                float x[8], y[8];
                if (seg[i] >= 0) {
                    row8_values<ST>(lo[i], x);
                    row8_values<ST>(hi[i], y);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) { x[k] = 0.f; y[k] = 0.f; }
                }
                if (plane == 0 && seg[i] > 0) turn_pairs<ST>(st->table[seg[i] - 1] + a * 8, x, y);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    f[i][k] = x[k];
                    f[i][8 + k] = y[k];
                }
            }
            __syncthreads();                           // every row of these blocks has been read
#pragma unroll
            for (int i = 0; i < G; ++i) {
                const int j = (d + i) * 32 + r;
                if (tid < TW && d + i < stop && j < left) {
                    const float x[8] = {f[i][0], f[i][1], f[i][2], f[i][3], f[i][4], f[i][5], f[i][6], f[i][7]};
                    const float y[8] = {f[i][8], f[i][9], f[i][10], f[i][11], f[i][12], f[i][13], f[i][14], f[i][15]};
                    store_row8<ST, HD>(p, j, a * 8, nh, x);
                    store_row8<ST, HD>(p, j, HD / 2 + a * 8, nh, y);
                }
            }
        } else if (ST == 2 && plane == 0) {
            // Keys: thread = one row of one block and two 16-byte units of it, sixteen dims and their rotary partners: a wave reads and
            // writes whole runs of 512 bytes. (With eight dims to a thread, half units, the launch wrote 2.5 times its bytes.)
            constexpr int NB = TH / HD < G ? TH / HD : G, ROUNDS = G / NB;
            const int r = tid & 31, at = (((tid % HD) >> 6) * 64 + r + 32 * (((tid % HD) >> 5) & 1)) * 16;
            const int pair = ((tid % HD) >> 6) * 32 + 8 * (((tid % HD) >> 5) & 1);     // first dim; the others: + 1 .. 7, + 16 .. 23
            u32x4 lo[ROUNDS], hi[ROUNDS];
            int seg[ROUNDS];
            float sc[ROUNDS];
#pragma unroll
            for (int k = 0; k < ROUNDS; ++k) {
                const int i = k * NB + tid / HD, j = (d + i) * 32 + r;
                lo[k] = hi[k] = u32x4{0, 0, 0, 0};
                sc[k] = 1.f;
                const int s = source_row(gaps, R.n, j, seg[k]);
                if (!(tid < NB * HD && d + i < stop && j < left)) seg[k] = 0;
                else {
                    const char* q = p + (size_t)(s >> 5) * (32 * HD) + at + ((s & 31) - r) * 16;
                    lo[k] = *(const u32x4*)q;
                    hi[k] = *(const u32x4*)(q + HD * 16);
                    sc[k] = kv8_scale(ex[2 * (s >> 5)]);
                }
            }
            float f[ROUNDS][2][2][8];                  // [unit][half][dim]
#pragma unroll
            for (int k = 0; k < ROUNDS; ++k) {
                float mk = 0.f;
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    float (&x)[8] = f[k][0][hf], (&y)[8] = f[k][1][hf];
                    float t[4];
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        kv8_values(lo[k][hf * 2 + q], sc[k], t);
#pragma unroll
                        for (int z = 0; z < 4; ++z) x[q * 4 + z] = t[z];
                        kv8_values(hi[k][hf * 2 + q], sc[k], t);
#pragma unroll
                        for (int z = 0; z < 4; ++z) y[q * 4 + z] = t[z];
                    }
                    if (seg[k] > 0) turn_pairs<ST>(st->table[seg[k] - 1] + pair + 16 * hf, x, y);
#pragma unroll
                    for (int z = 0; z < 8; ++z) mk = larger(mk, x[z], y[z]);
                }
#pragma unroll
                for (int b = 0; b < NB; ++b) m[k * NB + b] = tid / HD == b ? mk : 0.f;
            }
            exponents_of(m, most[turn], e);
#pragma unroll
            for (int k = 0; k < ROUNDS; ++k) {
                const int i = k * NB + tid / HD;
                int mine = e[k * NB];
#pragma unroll
                for (int b = 1; b < NB; ++b) mine = tid / HD == b ? e[k * NB + b] : mine;
                const float unit = kv8_scale(mine);
                u32x4 q[2];
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int z = 0; z < 4; ++z) {
                        const float (&x)[8] = f[k][u][z >> 1];
                        const float t[4] = {x[(z & 1) * 4], x[(z & 1) * 4 + 1], x[(z & 1) * 4 + 2], x[(z & 1) * 4 + 3]};
                        q[u][z] = kv8_codes(t, unit);
                    }
                if (tid < NB * HD && d + i < stop) {    // (rows past the end: zeros, as their block has a new exponent)
                    *(u32x4*)(p + (size_t)(d + i) * (32 * HD) + at) = q[0];
                    *(u32x4*)(p + (size_t)(d + i) * (32 * HD) + at + HD * 16) = q[1];
                }
            }
        } else if (ST == 2 && one_shift(gaps, d, left)) {
            // Values of blocks whose rows all have one shift: thread = one dim of one block, whose 32 rows are eight words, every one cut
            // from two neighbouring words of the source (four rows each; word w of a dim: unit w % 2, word w / 2 of it, in block w / 8).
            constexpr int NB = TH / HD < G ? TH / HD : G, ROUNDS = G / NB;      // (two blocks of 64 dims: half the threads)
            const int dim = tid % HD, at = ((dim >> 5) * 64 + (dim & 31)) * 16, lastw = (len - 1) >> 2;
            float f[ROUNDS][8][4];
            uint32_t word[ROUNDS][9];
            int s0[ROUNDS], ev[ROUNDS];
#pragma unroll
            for (int k = 0; k < ROUNDS; ++k) {
                const int i = __builtin_amdgcn_readfirstlane(min(k * NB + tid / HD, G - 1));     // (whole waves have one block)
                const int j = min(d + i, stop - 1) * 32;
                s0[k] = j + gone_before(gaps, segment_at(gaps, j));
                ev[k] = ex[2 * min((s0[k] >> 5) + (tid & 1), (len - 1) >> 5)];      // of the block and the one behind it
#pragma unroll
                for (int x = 0; x < 9; ++x) {
                    const int wi = min((s0[k] >> 2) + x, lastw);
                    word[k][x] = *(const uint32_t*)(p + (size_t)(wi >> 3) * (32 * HD) + (wi & 1) * 512 + ((wi & 7) >> 1) * 4 + at);
                }
            }
#pragma unroll
            for (int k = 0; k < ROUNDS; ++k) {
                const int i = __builtin_amdgcn_readfirstlane(min(k * NB + tid / HD, G - 1));
                const float sa = kv8_scale(__builtin_amdgcn_readlane(ev[k], 0)), sb = kv8_scale(__builtin_amdgcn_readlane(ev[k], 1));
                const int live = d + i < stop ? left - (d + i) * 32 : 0;      // rows of it that are not past the end
                float mk = 0.f;
#pragma unroll
                for (int x = 0; x < 8; ++x) {          // rows 4 x ..
                    kv8_values(__builtin_amdgcn_alignbyte(word[k][x + 1], word[k][x], s0[k] & 3), 1.f, f[k][x]);
#pragma unroll
                    for (int y = 0; y < 4; ++y) f[k][x][y] *= (s0[k] & 31) + 4 * x + y < 32 ? sa : sb;
                }
                if (live < 32)
#pragma unroll
                    for (int x = 0; x < 8; ++x)
#pragma unroll
                        for (int y = 0; y < 4; ++y) f[k][x][y] = 4 * x + y < live ? f[k][x][y] : 0.f;
#pragma unroll
                for (int x = 0; x < 8; ++x) mk = larger(larger(mk, f[k][x][0], f[k][x][1]), f[k][x][2], f[k][x][3]);
#pragma unroll
                for (int b = 0; b < NB; ++b) m[k * NB + b] = tid / HD == b ? mk : 0.f;
            }
            exponents_of(m, most[turn], e);
#pragma unroll
            for (int k = 0; k < ROUNDS; ++k) {
                const int i = k * NB + tid / HD;
                int mine = e[k * NB];
#pragma unroll
                for (int b = 1; b < NB; ++b) mine = tid / HD == b ? e[k * NB + b] : mine;
                const float unit = kv8_scale(mine);
                u32x4 q[2];
#pragma unroll
                for (int x = 0; x < 8; ++x) q[x & 1][x >> 1] = kv8_codes(f[k][x], unit);
                if (tid < NB * HD && d + i < stop) {
                    *(u32x4*)(p + (size_t)(d + i) * (32 * HD) + at) = q[0];
                    *(u32x4*)(p + (size_t)(d + i) * (32 * HD) + at + 512) = q[1];
                }
            }
        } else if constexpr (TILES) {
            // the blocks are put together in LDS, segment by segment of rows with one shift
            __syncthreads();                           // the tiles' last readers are done
            for (int i = 0; i < G && d + i < stop; ++i)
                for (int r0 = 0; r0 < 32 && (d + i) * 32 + r0 < left;) {
                    const int seg = segment_at(gaps, (d + i) * 32 + r0), s0 = (d + i) * 32 + r0 + gone_before(gaps, seg);
                    int r1 = min(32, left - (d + i) * 32);     // rows [r0, r1) lie in one segment: s0 + r - r0
                    if (seg < R.n) r1 = min(r1, __builtin_amdgcn_readlane(gaps.from, seg) - (d + i) * 32);
                    for (int sb = s0 >> 5; sb <= (s0 + r1 - r0 - 1) >> 5; ++sb) {
                        const int off = sb * 32 - s0 + r0;       // row c of the source block is row c + off here
                        if constexpr (ST == 2) {
                            const float sc = kv8_scale(ex[2 * sb]);
                            for (int u = tid; u < HD * 2; u += TH) {
                                const int lane = u & 63, g = lane >> 5, dim = (u >> 6) * 32 + (lane & 31);
                                const u32x4 q = *(const u32x4*)(p + (size_t)sb * (32 * HD) + u * 16);
#pragma unroll
                                for (int x = 0; x < 4; ++x) {
                                    float f[4];
                                    kv8_values(q[x], sc, f);
#pragma unroll
                                    for (int y = 0; y < 4; ++y) {
                                        const int to = v8_row(x * 4 + y, g) + off;
                                        if (to >= r0 && to < r1) tile[i][to][dim] = __builtin_bit_cast(uint16_t, (__bf16)f[y]);
                                    }
                                }
                            }
                        } else {
                            for (int u = tid; u < HD * 4; u += TH) {
                                const int lane = u & 63, g = lane >> 5, pe = u >> 6, dim = (pe % (HD / 32)) * 32 + (lane & 31), half = pe / (HD / 32);
                                const u16x8 q = *(const u16x8*)((const uint16_t*)p + (size_t)sb * (32 * HD) + u * 8);
#pragma unroll
                                for (int x = 0; x < 8; ++x) {
                                    const int to = half * 16 + g * 4 + (x >> 2) * 8 + (x & 3) + off;
                                    if (to >= r0 && to < r1) tile[i][to][dim] = q[x];
                                }
                            }
                        }
                    }
                    r0 = r1;
                }
            __syncthreads();
            if constexpr (ST == 2) {
#pragma unroll
                for (int i = 0; i < G; ++i)
                    for (int k = tid; k < min(32, d + i < stop ? left - (d + i) * 32 : 0) * (HD / 8); k += TH) {
                        const u16x8 v = *(const u16x8*)&tile[i][k / (HD / 8)][(k % (HD / 8)) * 8];
#pragma unroll
                        for (int x = 0; x < 8; x += 2) m[i] = larger(m[i], bf16_bits_to_float(v[x]), bf16_bits_to_float(v[x + 1]));
                    }
                exponents_of(m, most[turn], e);
            }
#pragma unroll
            for (int i = 0; i < G; ++i) {
                if (d + i >= stop) break;
                for (int u = tid; u < HD * (ST == 2 ? 2 : 4); u += TH) {
                    const int lane = u & 63, g = lane >> 5, pe = u >> 6, dim = (pe % (HD / 32)) * 32 + (lane & 31), half = pe / (HD / 32);
                    if constexpr (ST == 2) {
                        u32x4 q;
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            float f[4];
#pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                const int row = v8_row(x * 4 + y, g);
                                f[y] = (d + i) * 32 + row < left ? bf16_bits_to_float(tile[i][row][dim]) : 0.f;
                            }
                            q[x] = kv8_codes(f, kv8_scale(e[i]));
                        }
                        *(u32x4*)(p + (size_t)(d + i) * (32 * HD) + u * 16) = q;
                    } else {
                        u16x8* to = (u16x8*)((uint16_t*)p + (size_t)(d + i) * (32 * HD) + u * 8);
                        u16x8 q = *to;
#pragma unroll
                        for (int x = 0; x < 8; ++x) {
                            const int row = half * 16 + g * 4 + (x >> 2) * 8 + (x & 3);
                            if ((d + i) * 32 + row < left) q[x] = tile[i][row][dim];
                        }
                        *to = q;
                    }
                }
            }
        }
        if constexpr (ST == 2)
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (tid == i && d + i < stop) ex[2 * (d + i)] = (int8_t)e[i];
    }
}

void launch_kv_drop(int storage, const KvPlanes& c, int seq, int nh, int hd, int layers, const DropRanges& R, const double* freq,
                    int32_t* kv_len, int len_hi, DropState* st, hipStream_t s) {
    hipLaunchKernelGGL(k_drop_setup, dim3(R.n), dim3(64), 0, s, R, freq, hd / 2, kv_len, seq, st);
    // Runs where one workgroup per (layer, head, plane) would leave the chip half empty, and the shift is long enough to pay for a
    // launch. us, runs / walks; 256 triples of 128 dims: 16384 rows of 8 bits less 4096 283 / 456, less 512 (16 blocks a run) 512 / 501, less
    // 300 697 / 497; of bfloat16 less 4096 466 / 1288, less 512 775 / 1483, less 300 1117 / 1759, 700 rows less 130 (four blocks) 53 / 60.
    // 1024 triples of 64 dims, 8000 rows less 600: 8 bits 508 / 324, bfloat16 766 / 700.
    // A walk of codes where walkers are few takes 512 threads: less 300 of 16384 rows 497, with 256 648; 130 of 700 31.4 / 32.2, with 1024
    // 38.9.
    int left = len_hi;                                 // the host's bound: what is left of the longest it may be
    for (int i = 0; i < R.n; ++i) left -= R.count[i] < len_hi - R.first[i] ? R.count[i] : (len_hi > R.first[i] ? len_hi - R.first[i] : 0);
    const int d0 = R.first[0] >> 5, d1 = (left + 31) >> 5, shift = std::min(R.count[0] >> 5, 32768);   // (a grid's limit)
    const int walkers = layers * nh * 2, least = storage == 2 ? 24 : 8;
    const bool runs = shift >= least && walkers < 1024;
    for (int d = d0; d < d1; d += runs ? shift : d1 - d0) {
        const int e = runs ? (d + shift < d1 ? d + shift : d1) : d1;
#define DROP_T(ST_, HD_, TH_)                                                                                          \
    do {                                                                                                               \
        constexpr int G_ = drop_blocks(ST_, HD_, TH_);                                                                 \
        hipLaunchKernelGGL((k_kv_drop<ST_, HD_, G_, TH_>), dim3(nh * (runs ? (e - d + G_ - 1) / G_ : 1), layers, 2), dim3(TH_), 0, s, c, \
                           seq, nh, R, st, d, e);                                                                      \
    } while (0)
#define DROP(ST_, HD_) do { if (ST_ == 2 && !runs && walkers < 1024) DROP_T(ST_, HD_, ST_ == 2 ? 512 : 256); else DROP_T(ST_, HD_, 256); } while (0)
#define DROP2(ST_) do { if (hd == 128) DROP(ST_, 128); else DROP(ST_, 64); } while (0)
        if (storage == 0) DROP2(0);
        else if (storage == 1) DROP2(1);
        else DROP2(2);
#undef DROP2
#undef DROP
#undef DROP_T
    }
}
