// What the copying and compacting kernels (kv_seq.hip) know of a cache, whatever its storage format.
#pragma once
#include "kv8.h"

// Byte strides of the key plane p[0] and the value plane p[1]: between layers, and between heads (sequence b's head h starts at
// (b * heads + h) * head; float32 caches count one head that holds whole rows). A unit (32 rows, or one float32 row) is
// unit_bytes and units of a head are contiguous. ex: exponents of an 8-bit cache, or NULL.
struct KvPlanes {
    char* p[2];
    size_t layer, head;
    char* ex;
    size_t ex_layer, ex_head;
    int unit_rows, unit_bytes;
};
struct KvCarried { int32_t *kv_len, *root_tok, *cand; };

// Rows to drop: ascending, apart from one another, each at least one row.
#define DROP_MAX SD_MAX_DROP_RANGES
struct DropRanges { int32_t first[DROP_MAX], count[DROP_MAX]; int n; };
// In device memory, per cache: (cos, sin) of the turn of every segment and dim pair, and the lengths before and after.
struct DropState { double2 table[DROP_MAX][64]; int32_t old_len, new_len; };

// read: rows of the source up to its device length; len_hi bounds it
void launch_kv_fork(const KvPlanes& src, const KvPlanes& dst, const SeqList& to, int n_dst, const int32_t* kv_len, int src_seq,
                    int len_hi, int heads, int layers, const KvCarried& from, const KvCarried& into, int n_cand, hipStream_t s);
// storage: 0 float32, 1 bfloat16, 2 e4m3; also sets the sequence's new length
void launch_kv_drop(int storage, const KvPlanes& c, int seq, int nh, int hd, int layers, const DropRanges& R, const double* freq,
                    int32_t* kv_len, int len_hi, DropState* st, hipStream_t s);
