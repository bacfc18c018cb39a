#include "slot_sums.h"

namespace bm {

// More than 2048 slots are added in two steps, others in the second alone, whose time is that of one row of threads' loads.  First: 64 lanes of
// four channels, four waves of eight slots each, all of them asked for together; the sum goes to the first of the 32 slots, which no other
// workgroup reads.  (Just written, of 2 x 256 channels: 512 slots both steps 5.1 us, one 2.4; 2048 5.2, 5.5; 16384 18.9, 38.9; of 2 x 4096:
// 512 12.0, 8.4; 4096 28.9, 26.2; of 2 x 4: 65536 12.5, 122.)
constexpr int kSlots = 32, kWide = 256, kOneStep = 2048;
__global__ __launch_bounds__(256) void slot_merge_kernel(const SlotSumArgs a, int arrays)
{
    const int which = blockIdx.z % arrays, vector = blockIdx.z / arrays;
    if (!a.out[which]) return;
    const int lane = threadIdx.x % 64, w = threadIdx.x / 64, c = blockIdx.x * kWide + lane * 4;
    const long long first = (long long)blockIdx.y * kSlots;
    float* const from = a.slots[which] + (vector * a.count + first) * a.pitch;
    const int n = (int)min((long long)kSlots, a.count - first);
    __shared__ float sum[4][kWide];
    float s[4] = {};
    if (a.d >= 4) {
        Piece<IoF32, 4> p[8];
#pragma unroll
        for (int i = 0; i < 8; i++) p[i] = load_clamped<IoF32, 4>(from + min(w * 8 + i, n - 1) * a.pitch, c, a.d);
#pragma unroll
        for (int i = 0; i < 8; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) s[j] += w * 8 + i < n ? p[i][j] : 0.0f;
    } else {
        for (int i = w * 8; i < min(w * 8 + 8, n); i++)
            for (int j = 0; j < 4; j++)
                if (c + j < a.d) s[j] += from[i * a.pitch + c + j];
    }
    // (a row's last piece was taken whole: its channels are those from d - 4 on)
    const int at = a.d >= 4 ? min(c, a.d - 4) : c;
#pragma unroll
    for (int j = 0; j < 4; j++) sum[w][lane * 4 + j] = s[j];
    __syncthreads();
    if (w == 0)
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (at + j >= c && at + j < a.d) from[at + j] = (sum[0][lane * 4 + j] + sum[1][lane * 4 + j]) + (sum[2][lane * 4 + j] + sum[3][lane * 4 + j]);
}
// 32 channels to a workgroup, each of its rows of threads a share of the slots.
constexpr int kSlotChannels = 32;
template <int kRows>
__global__ __launch_bounds__(kRows * kSlotChannels) void slot_sum_kernel(const SlotSumArgs a, long long per_vector)
{
    float* const out = a.out[blockIdx.z];
    if (!out) return;
    const int c = threadIdx.x % kSlotChannels, r = threadIdx.x / kSlotChannels, col = blockIdx.x * kSlotChannels + c;
    __shared__ float sum[kRows][kSlotChannels];
    float s = 0.0f;
    const float* const from = a.slots[blockIdx.z] + blockIdx.y * per_vector + col;
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
void launch_slot_sum(SlotSumArgs a, int vectors, hipStream_t st)
{
    const int arrays = a.out[1] ? 2 : 1;
    const long long per_vector = a.count * a.pitch;
    if (a.count > kOneStep && a.count <= 65535ll * kSlots && vectors * arrays <= 65535) {
        const long long heads = (a.count + kSlots - 1) / kSlots;
        hipLaunchKernelGGL(slot_merge_kernel, dim3((a.d + kWide - 1) / kWide, (unsigned)heads, vectors * arrays), dim3(256), 0, st, a, arrays);
        a.count = heads, a.pitch *= kSlots;
    }
    const dim3 grid((a.d + kSlotChannels - 1) / kSlotChannels, vectors, arrays);
    if (a.count <= 64) hipLaunchKernelGGL(slot_sum_kernel<8>, grid, dim3(8 * kSlotChannels), 0, st, a, per_vector);
    else hipLaunchKernelGGL(slot_sum_kernel<32>, grid, dim3(32 * kSlotChannels), 0, st, a, per_vector);
}

}  // namespace bm
