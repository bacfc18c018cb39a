#include "slot_sums.h"

namespace bm {

// 32 channels to a workgroup, each of its rows of threads a share of the slots.
constexpr int kSlotChannels = 32;
template <int kRows>
__global__ __launch_bounds__(kRows * kSlotChannels) void slot_sum_kernel(const SlotSumArgs a)
{
    float* const out = a.out[blockIdx.z];
    if (!out) return;
    const int c = threadIdx.x % kSlotChannels, r = threadIdx.x / kSlotChannels, col = blockIdx.x * kSlotChannels + c;
    __shared__ float sum[kRows][kSlotChannels];
    float s = 0.0f;
    const float* const from = a.slots[blockIdx.z] + blockIdx.y * a.count * a.pitch + col;
    if (col < a.d)
#pragma unroll 8
        for (long long i = r; i < a.count; i += kRows) s += from[i * a.pitch];
    sum[r][c] = s;
    __syncthreads();
    if (r == 0 && col < a.d) {
#pragma unroll
        for (int k = 1; k < kRows; k++) s += sum[k][c];
        out[(long long)blockIdx.y * a.d + col] = s;
    }
}
void launch_slot_sum(const SlotSumArgs& a, int vectors, hipStream_t st)
{
    const dim3 grid((a.d + kSlotChannels - 1) / kSlotChannels, vectors, a.out[1] ? 2 : 1);
    if (a.count <= 64) hipLaunchKernelGGL(slot_sum_kernel<8>, grid, dim3(8 * kSlotChannels), 0, st, a);
    else hipLaunchKernelGGL(slot_sum_kernel<32>, grid, dim3(32 * kSlotChannels), 0, st, a);
}

}  // namespace bm
