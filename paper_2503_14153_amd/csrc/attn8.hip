// Tree-masked attention over a cache in 8 bits (layout: kv8.h). As in attn.hip a head's K and V are a stream that all query rows
// share, split over workgroups and waves and joined by (max, sum, O) triples; what differs:
//   * half the bytes: 16 KiB of bfloat16 per block become 8 KiB of codes, and one instruction per two values widens them to
//     bfloat16 operands, the block's power-of-two scale included. Widened values are exact, so nothing else is rounded for it;
//   * queries and probabilities enter as ONE bfloat16 term, not two (attn.hip): their rounding, 2^-8 of a value at most, is far below
//     that of the codes they meet, 2^-4. Scores, maxima, sums and partial outputs stay float32, natural outputs are rounded once;
//   * what that saves in registers holds two blocks of keys and values per wave, each requested again as soon as it has been used. A wave
//     counts its loads in flight (nothing may wait for all of them: see the exponents), and they are under way before the length is known.
//     Three blocks spill, or share their registers with the accumulators in moves (64 rows over 16873: 47 us, 41 with two); with 64
//     dims there is room for four, which are not faster (24.8 us, 24.6: eight ragged sequences of 32 rows).
// Bound by the codes' stream where they are many: 134 MB in 32 us (one row over 16384, 32 heads of 128 dims; the same card streams a
// plain read in 19), 176 MB in 43 (eight ragged sequences of 32 rows, whose parts are whole blocks of work: the longest part has 51, the
// mean 40), 140 MB in 39 - 42 (64 rows over 16873). Some 7 us are fixed: launch, first loads, the waves' and the parts' merges.
// S^T = K Q^T puts query t in lane t % 32; exp(S) in its accumulator registers is the next product's operand (values are stored
// with their rows in that order).
#include "attn8.h"
#include "row_ops.h"

#define NEG_INF (-__builtin_inff())
#define LAZY_MAX 8.0f                  // the running maximum is raised only past 2^8 of itself (see attn.hip)

struct Attn8Args {
    const uint8_t *kc, *vc; const int8_t* ex; int cap_blocks; size_t ex_head;
    const int32_t* kv_len;
    RowRef rr;
    int nh, Tp, nparts;
    float scale_log2;
    float* opart; float2* mlpart;
    const uint32_t* anc; const bf16x8 *qp, *kt, *vt;
    const uint16_t *q, *k, *v; int ld, T;
    uint16_t* out; int ldo; int32_t* arrived;
    Attn8Split split;
};

// grid (head, entry of the split x block of 32 query rows): the workgroups of a head share an XCD where heads are a multiple of eight, and
// the query blocks of a part follow one another, so that all but the first find its rows in the caches. (Two query blocks a workgroup,
// eight waves, and a launch that merges: 64 rows over 1280 / 16873 17.5 / 39.1 us, here 15.8 - 16.4 / 39.3 - 42; in a step's own launch, 64 rows
// over some 600, 10.3 us, here 8.9.) Wave w has wave w of the part's blocks. NAT: natural rows; else packed ones.
template <int HD, bool NAT>
__global__ __launch_bounds__(256, 2) void k_attn8(Attn8Args a) {
    constexpr int KK = HD / 16, EB = HD / 32, NU = HD / 32;        // contraction steps, output blocks, 16-byte units of a block per lane
    constexpr int BLK = 32 * HD;                                   // bytes of a block
    constexpr int VROW = HD + 8;                                   // LDS row of the tree's values (NAT)
    constexpr int RING = 2;                                        // blocks of K and V that a wave has in flight or in registers
    constexpr int TURNS = 64 / RING * RING;                        // blocks between two loads of exponents
    __shared__ __attribute__((aligned(16))) float4 lds_o[4 * EB * 4 * 64];      // the waves' O; before that the tree's values
    __shared__ float lds_ml[4 * 2 * 64];
    static_assert(32 * VROW * 2 <= EB * 4 * 64 * 16, "a wave's tree values fit its part of the merge area");
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, g = lane >> 5, tl = lane & 31;
    const int h = blockIdx.x, nh = a.nh, Tp = a.Tp, TB = Tp >> 5;
    const int en = blockIdx.y / TB, qb = blockIdx.y - en * TB;      // entry, block of query rows
    const uint32_t entry = a.split.slot[en];
    const int b = entry & 255, part = (entry >> 8) & 255, own = entry >> 16;
    const bool MAP = !NAT && a.rr.map != nullptr;
    const int rows = NAT ? a.T : a.rr.len(b);
    if (qb * 32 >= rows) return;
    const int sq = NAT ? b : a.rr.seq(b);
    const int jw = __builtin_amdgcn_readfirstlane(part * a.split.each[en] + wave * a.split.share[en]);    // its first cache block
    const size_t head = ((size_t)sq * nh + h) * a.cap_blocks;
    const uint8_t* kcb = a.kc + head * BLK + lane * 16;
    const uint8_t* vcb = a.vc + head * BLK + lane * 16;
    u32x4 kr[RING][NU], vr[RING][NU];
    auto request_k = [&](int r, int blk) {
        const uint8_t* p = kcb + (size_t)blk * BLK;
#pragma unroll
        for (int i = 0; i < NU; ++i) kr[r][i] = *(const u32x4*)(p + i * 1024);
    };
    auto request_v = [&](int r, int blk) {
        const uint8_t* p = vcb + (size_t)blk * BLK;
#pragma unroll
        for (int i = 0; i < NU; ++i) vr[r][i] = *(const u32x4*)(p + i * 1024);
    };
    int n = MAP ? a.rr.map->ctx[b] : a.kv_len[sq];
    // Exponents of the wave's next 64 blocks, one per lane: a load for each block in the loop would have to be waited for where its
    // value moves to a scalar register, and with it everything requested before it. (The empty asm below is the place of the wait:
    // not the head of the loop.)
    const uint16_t* const exb = (const uint16_t*)(a.ex + ((size_t)sq * nh + h) * a.ex_head);
    uint32_t ev = exb[min(jw + lane, a.cap_blocks - 1)];
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 qf[KK];                                     // queries: B operands of all contraction steps
    {
        if constexpr (NAT) {
            const uint16_t* p = a.q + ((size_t)b * a.T + min(qb * 32 + tl, a.T - 1)) * a.ld + h * HD + g * 8;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) qf[kk] = *(const bf16x8*)(p + kk * 16);
        } else {                                       // (the first of the two terms that the rotary stage leaves)
            const bf16x8* p = a.qp + (((size_t)b * nh + h) * TB + qb) * (KK * 2 * 64) + lane;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) qf[kk] = p[kk * 128];
        }
    }
#pragma unroll
    for (int r = 0; r < RING; ++r) {
        const int blk = min(jw + r, a.cap_blocks - 1);  // (in bounds, whatever the length is; unused past the wave's last block)
        __builtin_amdgcn_sched_barrier(0);             // (the order that the loop repeats, so that it can count what is in flight)
        request_k(r, blk);
        __builtin_amdgcn_sched_barrier(0);
        request_v(r, blk);
    }
    __builtin_amdgcn_sched_barrier(0);
    // All of these are under way before the length is known.
    n = __builtin_amdgcn_readfirstlane(n);
    asm volatile("" : "+s"(n));
    const int nblk = (n + 31) >> 5;
    const int ntree = part == own - 1 ? qb + 1 : 0;                // tree blocks that the rows can see into: no node before its parent
    const int pend = part == own - 1 ? nblk : min(nblk, (part + 1) * a.split.each[en]);
    const int je = __builtin_amdgcn_readfirstlane(wave == 3 ? pend : min(pend, jw + a.split.share[en]));   // this wave's blocks [jw, je)
    auto block_of = [&](int j) { return max(min(j, je - 1), 0); };   // (past the wave's last: that block again)

    f32x16 O[EB];
    float mrun = NEG_INF, lrun = 0.f;
#pragma unroll
    for (int eb = 0; eb < EB; ++eb)
#pragma unroll
        for (int v = 0; v < 16; ++v) O[eb][v] = 0.f;
    // softmax of a block's scores; vis: which of the block's rows this lane's query row sees (bit = row), where `masked`
    auto softmax = [&](f32x16& S, bool masked, uint32_t vis, bf16x8 (&pf)[2]) {
        if (masked) {
            vis >>= 4 * g;                             // lane (t = tl, g) holds rows 8*(v/4) + 4*g + v%4 of the block
#pragma unroll
            for (int v = 0; v < 16; ++v) S[v] = (vis & (1u << (8 * (v >> 2) + (v & 3)))) ? S[v] : NEG_INF;
        }
        float mx = S[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) mx = fmaxf(mx, S[v]);
        mx = fmaxf(mx, __shfl_xor(mx, 32)) * a.scale_log2;
        const bool upd = mx > mrun + LAZY_MAX;
        if (__any(upd)) {
            const float alpha = upd ? __builtin_amdgcn_exp2f(mrun - mx) : 1.f;
            mrun = upd ? mx : mrun;
            lrun *= alpha;
#pragma unroll
            for (int eb = 0; eb < EB; ++eb)
#pragma unroll
                for (int v = 0; v < 16; ++v) O[eb][v] *= alpha;
        }
        const float muse = (mrun == NEG_INF) ? 0.f : mrun;
        float psum = 0.f;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const float pv = __builtin_amdgcn_exp2f(__builtin_fmaf(S[8 * p + s], a.scale_log2, -muse));
                psum += pv;
                pf[p][s] = (__bf16)pv;
            }
        lrun += psum;
    };

    asm volatile("" ::"v"(ev));
    // one block: scores, softmax, values
    auto scores = [&](const u32x4(&k)[NU], float ks, f32x16& S) {
#pragma unroll
        for (int v = 0; v < 16; ++v) S[v] = 0.f;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv8_widen(k[i].x, k[i].y, ks), qf[2 * i], S, 0, 0, 0);
            S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv8_widen(k[i].z, k[i].w, ks), qf[2 * i + 1], S, 0, 0, 0);
        }
    };
    auto values = [&](u32x4(&v)[NU], float vs, f32x16& S, int left) {
        const bool ragged = left < 32;                 // wave-uniform
        bf16x8 pf[2];
        softmax(S, ragged, ragged ? (1u << left) - 1u : 0u, pf);
        if (ragged)                                    // rows past the end may hold NaN codes, and 0 * NaN is NaN
#pragma unroll
            for (int i = 0; i < NU; ++i)
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const int keep = min(max(left - v8_row(4 * d, g), 0), 4);      // leading bytes of this word that are rows
                    v[i][d] &= keep == 4 ? 0xffffffffu : (1u << (8 * keep)) - 1u;
                }
#pragma unroll
        for (int eb = 0; eb < EB; ++eb) {
            O[eb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv8_widen(v[eb].x, v[eb].y, vs), pf[0], O[eb], 0, 0, 0);
            O[eb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv8_widen(v[eb].z, v[eb].w, vs), pf[1], O[eb], 0, 0, 0);
        }
    };
    for (int j0 = jw; j0 < je; j0 += TURNS) {
        for (int j = j0; j < min(j0 + TURNS, je); j += RING) {
#pragma unroll
            for (int r = 0; r < RING; ++r) {
                const bool live = j + r < je;
                f32x16 S;
                const uint32_t e2 = (uint32_t)__builtin_amdgcn_readlane((int)ev, j + r - j0);
                if (live) scores(kr[r], kv8_scale((int)(int8_t)e2), S);
                __builtin_amdgcn_sched_barrier(0);
                request_k(r, block_of(j + r + RING));
                __builtin_amdgcn_sched_barrier(0);
                if (live) values(vr[r], kv8_scale((int)(int8_t)(e2 >> 8)), S, n - (j + r) * 32);
                __builtin_amdgcn_sched_barrier(0);
                request_v(r, block_of(j + r + RING));
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (j0 + TURNS < je) {
            ev = exb[block_of(j0 + TURNS + lane)];
            asm volatile("" ::"v"(ev));
        }
    }

    // ---- the tree's blocks, dealt to the waves one by one: bfloat16 rows, masked by the ancestor sets
    for (int tblk = wave; tblk < ntree; tblk += 4) {
        bf16x8 kf[KK], vf[2 * EB];
        uint32_t vis = 0;
        if constexpr (NAT) {
            const int row = min(tblk * 32 + tl, a.T - 1);
            const uint16_t* kp = a.k + ((size_t)b * a.T + row) * a.ld + h * HD + g * 8;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) kf[kk] = *(const bf16x8*)(kp + kk * 16);
            // values through this wave's part of the merge area: whole rows in, columns out
            uint16_t* tv = (uint16_t*)(lds_o + wave * EB * 4 * 64);
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
            vis = a.anc[(size_t)(qb * 32 + tl) * SD_ANC_WORDS + tblk];
        } else {
            const bf16x8* kp = a.kt + ((((size_t)b * nh + h) * TB + tblk) * BLK >> 3) + lane;
            const bf16x8* vp = a.vt + ((((size_t)b * nh + h) * TB + tblk) * BLK >> 3) + lane;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) kf[kk] = kp[kk * 64];
#pragma unroll
            for (int i = 0; i < 2 * EB; ++i) vf[i] = vp[i * 64];
            vis = a.anc[((size_t)b * Tp + (qb * 32 + tl)) * SD_ANC_WORDS + tblk];
        }
        f32x16 S;
        bf16x8 pf[2];
#pragma unroll
        for (int v = 0; v < 16; ++v) S[v] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk], qf[kk], S, 0, 0, 0);
        softmax(S, true, vis, pf);
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int eb = 0; eb < EB; ++eb) O[eb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[p * EB + eb], pf[p], O[eb], 0, 0, 0);
    }

    // ---- the four waves meet in LDS; the output tiles are shared out over them
    __syncthreads();                                   // (the tree's values of every wave have been read)
#pragma unroll
    for (int eb = 0; eb < EB; ++eb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            lds_o[(wave * EB + eb) * 4 * 64 + i * 64 + lane] = make_float4(O[eb][4 * i], O[eb][4 * i + 1], O[eb][4 * i + 2], O[eb][4 * i + 3]);
    lds_ml[(wave * 2 + 0) * 64 + lane] = mrun;
    lds_ml[(wave * 2 + 1) * 64 + lane] = lrun;
    __syncthreads();
    const int t = qb * 32 + tl, eb = wave;
    if (eb < EB && t < rows) {                         // (a padding row: nobody reads it)
        float mw[4], lw[4], M = NEG_INF;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            mw[w] = lds_ml[w * 2 * 64 + lane];
            lw[w] = lds_ml[(w * 2 + 1) * 64 + lane];
            M = fmaxf(M, mw[w]);
        }
        const float Muse = (M == NEG_INF) ? 0.f : M;
        float L = 0.f, sc[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            sc[w] = exp2f(mw[w] - Muse);               // exp2(-inf) = 0 for a wave that saw nothing
            L += sc[w] * lw[w];
        }
        const float ltot = L + __shfl_xor(L, 32);      // (the other half of the same row)
        const bool done = NAT && own == 1;             // nothing to merge
        const size_t row = (((size_t)b * nh + h) * a.nparts + part) * Tp + t;
        if (eb == 0 && g == 0 && !done) {
            union { float f[2]; uint64_t u; } ml;
            ml.f[0] = M; ml.f[1] = ltot;
            if constexpr (NAT) __hip_atomic_store((uint64_t*)&a.mlpart[row], ml.u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            else a.mlpart[row] = make_float2(M, ltot);
        }
        const float inv = 1.f / ltot;                  // (every row sees at least itself)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float4 x = lds_o[(w * EB + eb) * 4 * 64 + i * 64 + lane];
                acc.x += sc[w] * x.x; acc.y += sc[w] * x.y; acc.z += sc[w] * x.z; acc.w += sc[w] * x.w;
            }
            const int e = eb * 32 + 8 * i + 4 * g;
            if (done) {
                union { __bf16 f[4]; uint64_t u; } o;
                o.f[0] = (__bf16)(acc.x * inv); o.f[1] = (__bf16)(acc.y * inv); o.f[2] = (__bf16)(acc.z * inv); o.f[3] = (__bf16)(acc.w * inv);
                *(uint64_t*)(a.out + ((size_t)b * a.T + t) * a.ldo + h * HD + e) = o.u;
            } else {
                store_frag16<NAT>((bf16x8*)(a.opart + row * HD + e), __builtin_bit_cast(bf16x8, acc));
            }
        }
    }

    // ---- natural rows: whichever part of this (sequence, head, query block) ends last merges them all, always in the order of their
    // numbers (one row over 16384: 35.6 us with a launch for it, 32.2 here). The parts were stored past this XCD's L2 (row_ops.h:
    // write-through), and have arrived when this workgroup counts itself; the last one puts the count back to zero for the next launch.
    if constexpr (NAT) {
        if (own == 1) return;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        int* last = (int*)lds_ml;
        if (tid == 0) {
            int32_t* count = a.arrived + ((size_t)b * nh + h) * TB + qb;
            const int before = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (before == own - 1) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            *last = before == own - 1;
        }
        __syncthreads();
        if (!*last) return;                            // (workgroup-uniform)
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        const int first = qb * 32, here = min(32, rows - first);
        for (int i = tid; i < here * (HD / 8); i += 256) {
            const int r = first + i / (HD / 8), e8 = i % (HD / 8);
            float o[8];
            attn_merge_values(a.opart, a.mlpart, nh, HD, Tp, a.nparts, own, b, h, r, e8, o);
            bf16x8 v;
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x] = (__bf16)o[x];
            *(bf16x8*)(a.out + ((size_t)b * a.T + r) * a.ldo + h * HD + e8 * 8) = v;
        }
    }
}

void launch_attn8(const Attn8& a, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1) {
    const bool nat = a.q != nullptr;
    Attn8Args r;
    r.kc = a.c.k; r.vc = a.c.v; r.ex = a.c.ex; r.cap_blocks = a.c.cap_blocks; r.ex_head = kv8_ex_head(a.c.cap_blocks); r.kv_len = a.kv_len; r.rr = a.rr;
    r.nh = a.nh; r.Tp = a.Tp; r.nparts = a.split.max_parts;
    r.scale_log2 = 1.4426950408889634f / sqrtf((float)a.hd);
    r.opart = a.opart; r.mlpart = a.mlpart; r.qp = a.qp; r.kt = a.kt; r.vt = a.vt; r.anc = a.anc;
    r.q = a.q; r.k = a.k; r.v = a.v; r.ld = a.ld; r.T = a.T; r.out = a.out; r.ldo = a.ldo; r.arrived = a.arrived;
    r.split = a.split;
    const dim3 grid(a.nh, a.split.n * (a.Tp / 32));
#define ATT8(HD_, NAT_)                                                                                                \
    do {                                                                                                               \
        if (ev0 || ev1) hipExtLaunchKernelGGL((k_attn8<HD_, NAT_>), grid, dim3(256), 0, s, ev0, ev1, 0, r);            \
        else hipLaunchKernelGGL((k_attn8<HD_, NAT_>), grid, dim3(256), 0, s, r);                                       \
    } while (0)
    if (a.hd == 128) { if (nat) ATT8(128, true); else ATT8(128, false); }
    else             { if (nat) ATT8(64, true);  else ATT8(64, false); }
#undef ATT8
}
