// Sums that workgroups leave in slots, added up in a fixed order.
#pragma once
#include "model_ops.h"

namespace bm {

// out[vector][c] = sum over i < count of slots[vector][i][c], for up to two such arrays at a time.  The slots are used up.
struct SlotSumArgs {
    float* slots[2];         // element (vector, i, c) at vector * count * pitch + i * pitch + c
    float* out[2];           // null: not wanted
    long long count, pitch;
    int d;
};
void launch_slot_sum(SlotSumArgs a, int vectors, hipStream_t st);

}  // namespace bm
