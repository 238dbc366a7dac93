// Tree-masked attention over a cache in 8 bits (layout: kv8.h). As in attn.hip a head's K and V are a stream that all query rows
// share, split over workgroups and waves and joined by (max, sum, O) triples; what differs:
//   * half the bytes: 16 KiB of bfloat16 per block become 8 KiB of codes, and one instruction per two values widens them to
//     bfloat16 operands, the block's power-of-two scale included. Widened values are exact, so nothing else is rounded for it;
//   * queries and probabilities enter as ONE bfloat16 term, not two (attn.hip): their rounding, 2^-9 of a value, is far below
//     that of the codes they meet, 2^-4. Scores, maxima, sums and outputs stay float32;
//   * so the queries of a workgroup fit its registers, and nothing but the loads of the stream is left in the loop.
// S^T = K Q^T puts query t in lane t % 32; exp(S) in its accumulator registers is the next product's operand (values are stored
// with their rows in that order).
#include "attn8.h"
#include "row_ops.h"

#define NEG_INF (-__builtin_inff())
#define LAZY_MAX 8.0f                  // the running maximum is raised only past 2^8 of itself (see attn.hip)
// blocks of K and V that a wave has in flight or in registers
#define RING 2

// x *= alpha for an accumulator in an AGPR (see attn.hip)
static __device__ __forceinline__ void acc_scale(float& x, float alpha) {
    float t;
    asm volatile("v_accvgpr_read_b32 %1, %0\n\tv_mul_f32 %1, %1, %2\n\tv_accvgpr_write_b32 %0, %1"
                 : "+a"(x), "=&v"(t) : "v"(alpha));
}

struct Attn8Args {
    const uint8_t *kc, *vc; const int8_t* ex; int cap_blocks;
    const int32_t* kv_len;
    RowRef rr;
    int nh, Tp, TG, nparts;
    float scale_log2;
    float* opart; float2* mlpart;
    const bf16x8 *qp, *kt, *vt; const uint32_t* anc;
    const uint16_t *q, *k, *v; int ld, T; const int32_t* parent;
    uint16_t* out; int ldo;
    AttnSplit split;
};

// grid (head, entry of the split x query group): the workgroups of a head share an XCD where heads are a multiple of eight.
// NAT: natural rows; else packed ones. TBW: query blocks of 32 rows per workgroup.
template <int HD, int TBW, bool NAT>
__global__ __launch_bounds__(256, TBW == 1 ? 2 : 1) void k_attn8(Attn8Args a) {
    constexpr int KK = HD / 16, EB = HD / 32, NU = HD / 32;        // contraction steps, output blocks, 16-byte units of a block per lane
    constexpr int BLK = 32 * HD;                                   // bytes of a block
    constexpr int NT = TBW * EB;                                   // 32x32 output tiles of one wave
    constexpr int VROW = HD + 8;                                   // LDS row of the tree's values (NAT)
    __shared__ __attribute__((aligned(16))) float4 lds_o[4 * NT * 4 * 64];      // the waves' O; before that the tree's values
    __shared__ float lds_ml[4 * TBW * 2 * 64];
    static_assert(32 * VROW * 2 <= NT * 4 * 64 * 16, "a wave's tree values fit its part of the merge area");
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, g = lane >> 5, tl = lane & 31;
    const int h = blockIdx.x, nh = a.nh, Tp = a.Tp, TB = Tp >> 5;
    const int en = blockIdx.y / a.TG, tg = blockIdx.y - en * a.TG;
    const uint32_t entry = a.split.slot[en];
    const int b = entry & 255, part = (entry >> 8) & 255, own = entry >> 16;
    const bool MAP = !NAT && a.rr.map != nullptr;
    const int rows = NAT ? a.T : a.rr.len(b);
    if (tg * TBW * 32 >= rows) return;
    const int sq = NAT ? b : a.rr.seq(b);
    const int n = MAP ? a.rr.map->ctx[b] : a.kv_len[sq];
    const int nblk = (n + 31) >> 5;
    const int ntree = min(tg * TBW + TBW, (rows + 31) >> 5);       // tree blocks that the rows can see into
    // this part's items [i0, i1) of the sequence's cache blocks and, behind them, tree blocks
    const int total = nblk + ntree, each = (total + own - 1) / own;
    const int i0 = min(part * each, total), i1 = min(i0 + each, total);
    const int c0 = min(i0, nblk), c1 = min(i1, nblk);              // its cache blocks
    const int t0 = max(i0, nblk) - nblk, t1 = max(i1, nblk) - nblk;   // its tree blocks
    const int share = (c1 - c0 + 3) >> 2;
    const int jw = __builtin_amdgcn_readfirstlane(min(c0 + wave * share, c1));
    const int je = __builtin_amdgcn_readfirstlane(min(jw + share, c1));          // this wave's cache blocks [jw, je)
    const size_t head = ((size_t)sq * nh + h) * a.cap_blocks;
    const uint8_t* kcb = a.kc + head * BLK + lane * 16;
    const uint8_t* vcb = a.vc + head * BLK + lane * 16;
    const uint16_t* exb = (const uint16_t*)(a.ex + head * 2);

    u32x4 kr[RING][NU], vr[RING][NU];
    uint32_t er[RING];
    auto block_of = [&](int j) { return max(min(j, je - 1), 0); };   // (past the wave's last: that block again; in bounds for a wave without any)
    auto request_k = [&](int r, int j) {
        const uint8_t* p = kcb + (size_t)block_of(j) * BLK;
        er[r] = exb[block_of(j)];
#pragma unroll
        for (int i = 0; i < NU; ++i) kr[r][i] = __builtin_nontemporal_load((const u32x4*)(p + i * 1024));
    };
    auto request_v = [&](int r, int j) {
        const uint8_t* p = vcb + (size_t)block_of(j) * BLK;
#pragma unroll
        for (int i = 0; i < NU; ++i) vr[r][i] = __builtin_nontemporal_load((const u32x4*)(p + i * 1024));
    };
    // queries: B operands of all contraction steps, kept in registers
    bf16x8 qf[TBW][KK];
#pragma unroll
    for (int tb = 0; tb < TBW; ++tb) {
        const int blk = min(tg * TBW + tb, TB - 1);
        if constexpr (NAT) {
            const int t = min(blk * 32 + tl, a.T - 1);
            const uint16_t* p = a.q + ((size_t)b * a.T + t) * a.ld + h * HD + g * 8;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) qf[tb][kk] = *(const bf16x8*)(p + kk * 16);
        } else {                                       // (the first of the two terms that the rotary stage leaves)
            const bf16x8* p = a.qp + (((size_t)b * nh + h) * TB + blk) * (KK * 2 * 64) + lane;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) qf[tb][kk] = p[kk * 128];
        }
    }
#pragma unroll
    for (int r = 0; r < RING; ++r) { request_k(r, jw + r); request_v(r, jw + r); }

    f32x16 O[TBW][EB];
    float mrun[TBW], lrun[TBW];
#pragma unroll
    for (int tb = 0; tb < TBW; ++tb) {
        mrun[tb] = NEG_INF;
        lrun[tb] = 0.f;
#pragma unroll
        for (int eb = 0; eb < EB; ++eb)
#pragma unroll
            for (int v = 0; v < 16; ++v) O[tb][eb][v] = 0.f;
    }
    // softmax of a block's scores; vis: which of the block's rows this lane's query row sees (bit = row), where `masked`
    auto softmax = [&](f32x16& S, int tb, bool masked, uint32_t vis, bf16x8 (&pf)[2]) {
        if (masked) {
            vis >>= 4 * g;                             // lane (t = tl, g) holds rows 8*(v/4) + 4*g + v%4 of the block
#pragma unroll
            for (int v = 0; v < 16; ++v) S[v] = (vis & (1u << (8 * (v >> 2) + (v & 3)))) ? S[v] : NEG_INF;
        }
        float mx = S[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) mx = fmaxf(mx, S[v]);
        mx = fmaxf(mx, __shfl_xor(mx, 32)) * a.scale_log2;
        const bool upd = mx > mrun[tb] + LAZY_MAX;
        if (__any(upd)) {
            const float alpha = upd ? __builtin_amdgcn_exp2f(mrun[tb] - mx) : 1.f;
            mrun[tb] = upd ? mx : mrun[tb];
            lrun[tb] *= alpha;
            asm volatile("s_nop 7\n\ts_nop 7");
#pragma unroll
            for (int eb = 0; eb < EB; ++eb)
#pragma unroll
                for (int v = 0; v < 16; ++v) { float x = O[tb][eb][v]; acc_scale(x, alpha); O[tb][eb][v] = x; }
            asm volatile("s_nop 7");
        }
        const float muse = (mrun[tb] == NEG_INF) ? 0.f : mrun[tb];
        float psum = 0.f;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const float pv = __builtin_amdgcn_exp2f(__builtin_fmaf(S[8 * p + s], a.scale_log2, -muse));
                psum += pv;
                pf[p][s] = (__bf16)pv;
            }
        lrun[tb] += psum;
    };

    for (int j = jw; j < je; j += RING) {
#pragma unroll
        for (int r = 0; r < RING; ++r) {
            const bool live = j + r < je;
            f32x16 S[TBW];
            const float vs = kv8_scale((int)(int8_t)(er[r] >> 8));
            if (live) {
                const float ks = kv8_scale((int)(int8_t)er[r]);
#pragma unroll
                for (int tb = 0; tb < TBW; ++tb)
#pragma unroll
                    for (int v = 0; v < 16; ++v) S[tb][v] = 0.f;
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    const bf16x8 k0 = kv8_widen(kr[r][i].x, kr[r][i].y, ks), k1 = kv8_widen(kr[r][i].z, kr[r][i].w, ks);
#pragma unroll
                    for (int tb = 0; tb < TBW; ++tb) S[tb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0, qf[tb][2 * i], S[tb], 0, 0, 0);
#pragma unroll
                    for (int tb = 0; tb < TBW; ++tb) S[tb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1, qf[tb][2 * i + 1], S[tb], 0, 0, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            request_k(r, j + r + RING);
            __builtin_amdgcn_sched_barrier(0);
            if (live) {
                const int left = n - (j + r) * 32;
                const bool ragged = left < 32;                     // wave-uniform
                bf16x8 pf[TBW][2];
#pragma unroll
                for (int tb = 0; tb < TBW; ++tb) softmax(S[tb], tb, ragged, ragged ? (1u << left) - 1u : 0u, pf[tb]);
                if (ragged)                            // rows past the end may hold NaN codes, and 0 * NaN is NaN
#pragma unroll
                    for (int i = 0; i < NU; ++i)
#pragma unroll
                        for (int d = 0; d < 4; ++d) {
                            const int keep = min(max(left - v8_row(4 * d, g), 0), 4);      // leading bytes of this word that are rows
                            vr[r][i][d] &= keep == 4 ? 0xffffffffu : (1u << (8 * keep)) - 1u;
                        }
#pragma unroll
                for (int eb = 0; eb < EB; ++eb) {
                    const bf16x8 v0 = kv8_widen(vr[r][eb].x, vr[r][eb].y, vs), v1 = kv8_widen(vr[r][eb].z, vr[r][eb].w, vs);
#pragma unroll
                    for (int tb = 0; tb < TBW; ++tb) O[tb][eb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v0, pf[tb][0], O[tb][eb], 0, 0, 0);
#pragma unroll
                    for (int tb = 0; tb < TBW; ++tb) O[tb][eb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v1, pf[tb][1], O[tb][eb], 0, 0, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            request_v(r, j + r + RING);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // ---- the tree's blocks, dealt to the waves one by one: bfloat16 rows, masked by the ancestor sets
    for (int tblk = t0 + wave; tblk < t1; tblk += 4) {
        bf16x8 kf[KK], vf[2 * EB];
        uint32_t vis[TBW];
        if constexpr (NAT) {
            const int row = min(tblk * 32 + tl, a.T - 1);
            const uint16_t* kp = a.k + ((size_t)b * a.T + row) * a.ld + h * HD + g * 8;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) kf[kk] = *(const bf16x8*)(kp + kk * 16);
            // values through this wave's part of the merge area: whole rows in, columns out
            uint16_t* tv = (uint16_t*)(lds_o + wave * NT * 4 * 64);
            constexpr int PC = HD / 8;
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < 32 * PC / 64; ++i) {
                const int rr = (i * 64 + lane) / PC, e = ((i * 64 + lane) % PC) * 8, t = tblk * 32 + rr;
                u32x4 x = *(const u32x4*)(a.v + ((size_t)b * a.T + min(t, a.T - 1)) * a.ld + h * HD + e);
                if (t >= a.T) x = u32x4{0, 0, 0, 0};
                *(u32x4*)(tv + rr * VROW + e) = x;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int eb = 0; eb < EB; ++eb)
#pragma unroll
                    for (int s = 0; s < 8; ++s)
                        vf[p * EB + eb][s] = __builtin_bit_cast(__bf16, tv[(p * 16 + 4 * g + 8 * (s >> 2) + (s & 3)) * VROW + eb * 32 + tl]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int tb = 0; tb < TBW; ++tb) {         // (a node's depth is at most SD_MAX_MEDUSA)
                const int t = (tg * TBW + tb) * 32 + tl;
                vis[tb] = 0;
                for (int i = t < a.T ? t : -1, guard = 0; i >= 0 && guard <= SD_MAX_MEDUSA; i = a.parent[i], ++guard)
                    if ((i >> 5) == tblk) vis[tb] |= 1u << (i & 31);
            }
        } else {
            const bf16x8* kp = a.kt + ((((size_t)b * nh + h) * TB + tblk) * BLK >> 3) + lane;
            const bf16x8* vp = a.vt + ((((size_t)b * nh + h) * TB + tblk) * BLK >> 3) + lane;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) kf[kk] = kp[kk * 64];
#pragma unroll
            for (int i = 0; i < 2 * EB; ++i) vf[i] = vp[i * 64];
#pragma unroll
            for (int tb = 0; tb < TBW; ++tb)
                vis[tb] = a.anc[((size_t)b * Tp + min((tg * TBW + tb) * 32 + tl, Tp - 1)) * SD_ANC_WORDS + tblk];
        }
#pragma unroll
        for (int tb = 0; tb < TBW; ++tb) {
            f32x16 S;
            bf16x8 pf[2];
#pragma unroll
            for (int v = 0; v < 16; ++v) S[v] = 0.f;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk], qf[tb][kk], S, 0, 0, 0);
            softmax(S, tb, true, vis[tb], pf);
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int eb = 0; eb < EB; ++eb) O[tb][eb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[p * EB + eb], pf[p], O[tb][eb], 0, 0, 0);
        }
    }

    // ---- the four waves meet in LDS; each writes a quarter of the output tiles
    __syncthreads();                                   // (the tree's values of every wave have been read)
#pragma unroll
    for (int tb = 0; tb < TBW; ++tb) {
#pragma unroll
        for (int eb = 0; eb < EB; ++eb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                lds_o[(wave * NT + tb * EB + eb) * 4 * 64 + i * 64 + lane] =
                    make_float4(O[tb][eb][4 * i], O[tb][eb][4 * i + 1], O[tb][eb][4 * i + 2], O[tb][eb][4 * i + 3]);
        lds_ml[((wave * TBW + tb) * 2 + 0) * 64 + lane] = mrun[tb];
        lds_ml[((wave * TBW + tb) * 2 + 1) * 64 + lane] = lrun[tb];
    }
    __syncthreads();
    for (int ti = wave; ti < NT; ti += 4) {
        const int tb = ti / EB, eb = ti % EB;
        float mw[4], lw[4], M = NEG_INF;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            mw[w] = lds_ml[((w * TBW + tb) * 2 + 0) * 64 + lane];
            lw[w] = lds_ml[((w * TBW + tb) * 2 + 1) * 64 + lane];
            M = fmaxf(M, mw[w]);
        }
        const float Muse = (M == NEG_INF) ? 0.f : M;
        float L = 0.f, sc[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            sc[w] = exp2f(mw[w] - Muse);               // exp2(-inf) = 0 for a wave that saw nothing
            L += sc[w] * lw[w];
        }
        const float ltot = L + __shfl_xor(L, 32);
        const int t = (tg * TBW + tb) * 32 + tl;
        if (t >= rows) continue;                       // a padding row: nobody reads it
        const bool done = NAT && a.nparts == 1;        // nothing to merge
        const size_t row = (((size_t)b * nh + h) * a.nparts + part) * Tp + t;
        if (eb == 0 && g == 0 && !done) a.mlpart[row] = make_float2(M, ltot);
        const float inv = 1.f / ltot;                  // (every row sees at least itself)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float4 x = lds_o[(w * NT + ti) * 4 * 64 + i * 64 + lane];
                acc.x += sc[w] * x.x; acc.y += sc[w] * x.y; acc.z += sc[w] * x.z; acc.w += sc[w] * x.w;
            }
            const int e = eb * 32 + 8 * i + 4 * g;
            if (done) {
                union { __bf16 f[4]; uint64_t u; } o;
                o.f[0] = (__bf16)(acc.x * inv); o.f[1] = (__bf16)(acc.y * inv); o.f[2] = (__bf16)(acc.z * inv); o.f[3] = (__bf16)(acc.w * inv);
                *(uint64_t*)(a.out + ((size_t)b * a.T + t) * a.ldo + h * HD + e) = o.u;
            } else {
                *(float4*)(a.opart + row * HD + e) = acc;
            }
        }
    }
}

// The parts of natural rows, merged: one thread per (row, head, 8 dims)
__global__ __launch_bounds__(256) void k_attn8_merge(Attn8Args a, int hd, int e8_shift) {
    const int idx = blockIdx.x * blockDim.x + threadIdx.x;
    const int e8 = idx & ((1 << e8_shift) - 1), t = idx >> e8_shift, h = blockIdx.y, b = blockIdx.z;
    if (t >= a.T) return;
    int own = 1;
    for (int i = 0; i < a.split.n; ++i)
        if ((int)(a.split.slot[i] & 255) == b) own = a.split.slot[i] >> 16;
    float o[8];
    attn_merge_values(a.opart, a.mlpart, a.nh, hd, a.Tp, a.nparts, own, b, h, t, e8, o);
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (__bf16)o[i];
    *(bf16x8*)(a.out + ((size_t)b * a.T + t) * a.ldo + h * hd + e8 * 8) = r;
}

void launch_attn8(const Attn8& a, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1) {
    const int TB = a.Tp / 32, TBW = attn8_tbw(TB), TG = (TB + TBW - 1) / TBW;
    const bool nat = a.q != nullptr;
    Attn8Args r;
    r.kc = a.c.k; r.vc = a.c.v; r.ex = a.c.ex; r.cap_blocks = a.c.cap_blocks; r.kv_len = a.kv_len; r.rr = a.rr;
    r.nh = a.nh; r.Tp = a.Tp; r.TG = TG; r.nparts = a.split.max_parts;
    r.scale_log2 = 1.4426950408889634f / sqrtf((float)a.hd);
    r.opart = a.opart; r.mlpart = a.mlpart; r.qp = a.qp; r.kt = a.kt; r.vt = a.vt; r.anc = a.anc;
    r.q = a.q; r.k = a.k; r.v = a.v; r.ld = a.ld; r.T = a.T; r.parent = a.parent; r.out = a.out; r.ldo = a.ldo;
    r.split = a.split;
    const dim3 grid(a.nh, a.split.n * TG);
#define ATT8(HD_, TBW_, NAT_)                                                                                          \
    do {                                                                                                               \
        if (ev0 || ev1) hipExtLaunchKernelGGL((k_attn8<HD_, TBW_, NAT_>), grid, dim3(256), 0, s, ev0, ev1, 0, r);       \
        else hipLaunchKernelGGL((k_attn8<HD_, TBW_, NAT_>), grid, dim3(256), 0, s, r);                                  \
    } while (0)
#define ATT8_T(HD_, NAT_) do { if (TBW == 2) ATT8(HD_, 2, NAT_); else ATT8(HD_, 1, NAT_); } while (0)
    if (a.hd == 128) { if (nat) ATT8_T(128, true); else ATT8_T(128, false); }
    else             { if (nat) ATT8_T(64, true);  else ATT8_T(64, false); }
#undef ATT8_T
#undef ATT8
    if (nat && r.nparts > 1)
        hipLaunchKernelGGL(k_attn8_merge, dim3((a.T * (a.hd / 8) + 255) / 256, a.nh, a.B), dim3(256), 0, s, r, a.hd, a.hd == 128 ? 4 : 3);
}
