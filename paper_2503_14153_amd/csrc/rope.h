// Rotary embedding: frequencies, which travel with the launch (rope.hip).
#pragma once
#include "sd_internal.h"

#define ROPE_MAX_DIM 256
struct RopeTable {
    double turns[ROPE_MAX_DIM / 2];      // per pair: turns per position, negative for the inverse (launch_set_rope: radians)
    float magnitude;
    int rotary;
};
// f32: float32 rows, else bfloat16; rows ldx / ldy elements apart, heads contiguous within them; y may be x
void launch_rope_rows(const void* x, void* y, const int32_t* pos, const RopeTable& f, int f32, int interleaved, int n, int heads, int hd,
                      int64_t ldx, int64_t ldy, hipStream_t s);
// freq [rotary / 2 + 1]: the frequencies in radians per position, then the magnitude
void launch_set_rope(const RopeTable& f, double* freq, hipStream_t s);
