// Attention over a cache in 8 bits: how a pass is cut into workgroups, and its launch (attn8.hip).
#pragma once
#include "kv8.h"
#include "attn_geom.h"

struct Attn8 {
    Kv8 c;                               // one layer
    const int32_t* kv_len;
    RowRef rr;
    int B, nh, hd, Tp;
    Attn8Split split;
    float* opart; float2* mlpart;        // [seq][head][split.max_parts][Tp][hd], as launch_attn_merge takes them
    const uint32_t* anc;                 // ancestor sets [Tp][SD_ANC_WORDS] (inside a pass: of every sequence)
    // inside a pass: queries, tree keys and values as the rotary stage leaves them
    const bf16x8 *qp, *kt, *vt;
    // or the stage alone: natural rows [seq][T] of bfloat16, `ld` apart
    const uint16_t *q, *k, *v;
    int ld, T;
    uint16_t* out; int ldo;
    int32_t* arrived;                    // zeros, one per (seq, head, query block): see k_attn8
};
// natural rows: the launch merges its parts into `out`
void launch_attn8(const Attn8& a, hipStream_t s, hipEvent_t ev0 = nullptr, hipEvent_t ev1 = nullptr);
