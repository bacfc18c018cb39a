// Kernels of the norm of groups of channels, for one activation (BM_ACT).
#include "group_norm.h"

namespace bm {

// A token's group stays in registers: 2^k lanes hold it in pieces of 16 bytes, up to 16 elements a lane, so a wave has 64 / lanes neighbouring
// groups of a row in hand (beyond 1024 channels four or eight waves share one).  It takes a few rows one after the other with
// weight and bias in registers; the gradients' sums for these two stay there as well and are left in a slot at the end.  The statistics are
// taken over the registers, the mean before the squares around it, so that a large mean costs no digits.  All arithmetic is fp32,
// each output is rounded once.
//
// What bounds it are the bytes, with the vector pipe beside them (busy all of the time with a gate and a mean, two thirds in the gradients, where all
// lanes hold elements), and in which order the memory sees them: a wave takes four rows and goes, so that all waves in hand
// work on neighbouring rows.  65536 rows of 4096 in groups of 64, gated, past the caches: 4 rows 250 us (6.45 TB/s; two tensors added to a
// third reach 6.0, past the caches 6.55), 1 row 284, 8 rows 274; through the caches 280; gradients 433 us (6.2 TB/s), 2 rows 461, 8 rows 463,
// through the caches 478.  Groups that waves share wait at a barrier in each row: their gradients read a row ahead (65536 groups of
// 4096 511 us, 541 without).  Lanes, pieces and waves come in powers of two: groups between them leave lanes empty, whose vector work the bytes
// no longer hide (65536 rows, gated before: one group of 2048 133 us, 6.05 TB/s; of 1536 138, 4.4; of 2560 233, 4.3; of 5120 529, 3.8; 20 of 100 191,
// 4.1; 55 of 37 276, 2.9; gradients 268, 223, 536, 1039, 340, 490).
enum Act { kPlain = BIMAMBA_ACT_NONE, kSilu = BIMAMBA_ACT_SILU, kBefore = BIMAMBA_ACT_GATE_BEFORE, kAfter = BIMAMBA_ACT_GATE_AFTER };

__device__ __forceinline__ float sigmoid_of(float v) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * v)); }

// Values summed over each run of `lanes` lanes, the same in all of a run.
template <int kN>
__device__ __forceinline__ void run_sum(float (&v)[kN], int lanes)
{
#define BM_DPP(ctrl) \
    for (int i = 0; i < kN; i++) v[i] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v[i]), ctrl, 0xf, 0xf, true))
    if (lanes < 2) return;
#pragma unroll
    BM_DPP(0xB1);    // quad_perm 1 0 3 2
    if (lanes < 4) return;
#pragma unroll
    BM_DPP(0x4E);    // quad_perm 2 3 0 1
    if (lanes < 8) return;
#pragma unroll
    BM_DPP(0x141);   // row_half_mirror
    if (lanes < 16) return;
#pragma unroll
    BM_DPP(0x140);   // row_mirror
#undef BM_DPP
    if (lanes < 32) return;
#pragma unroll
    for (int i = 0; i < kN; i++) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i]), false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (lanes < 64) return;
#pragma unroll
    for (int i = 0; i < kN; i++) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i]), false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
}

// The sums of a group from those of its lanes, and over its waves.  (Two turns: a part is written again only after the barrier of the sum
// between, which no wave passes before it has read this one's.)
template <int kWaves, int kN>
struct GroupSum {
    float part[2][kWaves][kN];
    __device__ __forceinline__ void operator()(float (&v)[kN], int lanes, int wave, int& turn)
    {
        run_sum(v, lanes);
        if constexpr (kWaves > 1) {
#pragma unroll
            for (int i = 0; i < kN; i++) part[turn][wave][i] = v[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kN; i++) {
                v[i] = part[turn][0][i];
#pragma unroll
                for (int k = 1; k < kWaves; k++) v[i] += part[turn][k][i];
            }
            turn ^= 1;
        }
    }
};

// Where a lane's elements lie and which rows its wave takes.
template <int kWaves, int kPieces, int kPiece, int kTeam, bool kPast, bool kMany>
struct GroupPlace {
    int g, in, n, stride;
    bool real, whole;   // whether the lane's group exists; (wave-uniform) every piece of every lane lies within its group
    bool in_group;      // (wave-uniform) every piece lies within its group, whether or not there is one for each lane
    unsigned run, r0, r1;   // the lane's row among those that the wave takes at once; the first of them, the end
    __device__ __forceinline__ GroupPlace(const GroupNormArgs& a, int lane, int wave) : n(a.n)
    {
        const int runs = 64 / a.lanes / (kMany ? a.at_once : 1), first = blockIdx.x * runs, k = lane / a.lanes;   // (groups of a row)
        run = kMany ? k / runs : 0;
        g = first + (kMany ? k % runs : k);
        real = g < a.G;
        g = min(g, a.G - 1);
        in = (lane % a.lanes + (kWaves > 1 ? wave * kPieces * 64 : 0)) * kPiece;
        stride = a.lanes * kPiece;
        whole = !kMany && first + runs <= a.G && a.n == kWaves * kPieces * stride;
        in_group = a.n == kWaves * kPieces * stride;
        const unsigned group = kWaves == 1 ? blockIdx.y * kTeam + wave : blockIdx.y;
        const unsigned step = a.per_wave * at_once(a);
        r0 = (unsigned)min((unsigned long long)a.rows, (unsigned long long)group * step);
        r1 = min(r0 + step, a.rows);
    }
    static __device__ __forceinline__ unsigned at_once(const GroupNormArgs& a) { return kMany ? a.at_once : 1; }
    // The row that a lane takes of those from r on: beyond the last one that one, and then it stores nothing.
    struct Row {
        unsigned r, b, t;
        bool real;
    };
    __device__ __forceinline__ Row row(const GroupNormArgs& a, unsigned r) const
    {
        if constexpr (kMany) r += run;   // (else the same in all lanes)
        Row x;
        x.real = real && r < r1;
        x.r = min(r, r1 - 1);
        x.b = x.r / a.L;
        x.t = x.r - x.b * a.L;
        return x;
    }
    __device__ __forceinline__ int at(int k) const { return in + k * stride; }
    __device__ __forceinline__ int channel() const { return g * n; }
    template <typename IO>
    __device__ __forceinline__ void load(Piece<IO, kPiece> (&p)[kPieces], const RowView& v, const Row& x) const
    {
        const typename IO::T* const row = static_cast<const typename IO::T*>(v.p) + row_offset(v, x.b, x.t) + channel();
#pragma unroll
        for (int k = 0; k < kPieces; k++) p[k] = load_clamped<IO, kPiece, kPast>(row, at(k), n);
    }
    template <typename IO>
    __device__ __forceinline__ void settled(Piece<IO, kPiece> (&p)[kPieces]) const
    {
        if (in_group) return;
#pragma unroll
        for (int k = 0; k < kPieces; k++) settle(p[k], at(k), n, typename IO::T(0));
    }
    template <typename IO>
    __device__ __forceinline__ void store(const RowView& v, const Row& x, const float (&f)[kPieces][kPiece]) const
    {
        typename IO::T* const row = static_cast<typename IO::T*>(v.p) + row_offset(v, x.b, x.t) + channel();
#pragma unroll
        for (int k = 0; k < kPieces; k++) {
            if (whole) store_piece<IO, kPast>(row + at(k), f[k]);
            else if (x.real) store_piece_of<IO, kPast>(row, at(k), n, f[k]);
        }
    }
    __device__ __forceinline__ void params(float (&f)[kPieces][kPiece], const float* p, float missing) const
    {
#pragma unroll
        for (int k = 0; k < kPieces; k++) {
            if (p) load_floats(f[k], p + channel(), at(k), n, 0.0f);
            else
#pragma unroll
                for (int i = 0; i < kPiece; i++) f[k][i] = missing;
        }
    }
};

template <typename IO, int kAct, int kWaves, int kPieces, int kPiece, int kTeam, bool kPast, bool kMany>
__device__ __forceinline__ void group_norm_rows(const GroupNormArgs& a)
{
    __shared__ GroupSum<kWaves, 1> sum;
    constexpr bool kGated = kAct == kBefore || kAct == kAfter;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const GroupPlace<kWaves, kPieces, kPiece, kTeam, kPast, kMany> place(a, lane, wave);
    if (place.r0 >= place.r1) return;   // (with several waves to a group: the whole workgroup)
    float w[kPieces][kPiece], c[kPieces][kPiece];
    place.params(w, a.weight, 1.0f);
    place.params(c, a.bias, 0.0f);
    const float inv = 1.0f / a.n;
    Piece<IO, kPiece> px[kPieces], pz[kPieces];
    auto next = place.row(a, place.r0);
    place.template load<IO>(px, a.x, next);
    if constexpr (kGated) place.template load<IO>(pz, a.z, next);
    int turn = 0;
    for (unsigned r = place.r0; r < place.r1; r += place.at_once(a)) {
        float u[kPieces][kPiece], gate[kPieces][kPiece], total[1] = {0.0f}, mean = 0.0f;
        place.template settled<IO>(px);
        if constexpr (kGated) place.template settled<IO>(pz);
#pragma unroll
        for (int k = 0; k < kPieces; k++)
#pragma unroll
            for (int i = 0; i < kPiece; i++) {
                u[k][i] = px[k][i];
                if constexpr (kGated) gate[k][i] = pz[k][i] * sigmoid_of(pz[k][i]);
                if constexpr (kAct == kBefore) u[k][i] *= gate[k][i];
            }
        const auto row = next;
        if (place.r1 - r > place.at_once(a)) {
            next = place.row(a, r + place.at_once(a));
            place.template load<IO>(px, a.x, next);
            if constexpr (kGated) place.template load<IO>(pz, a.z, next);
        }
        if (a.centred) {
#pragma unroll
            for (int k = 0; k < kPieces; k++)
#pragma unroll
                for (int i = 0; i < kPiece; i++) total[0] += u[k][i];
            sum(total, a.lanes, wave, turn);
            mean = total[0] * inv;
            total[0] = 0.0f;
#pragma unroll
            for (int k = 0; k < kPieces; k++)
#pragma unroll
                for (int i = 0; i < kPiece; i++) u[k][i] -= mean;
            if (!place.in_group)
#pragma unroll
                for (int k = 0; k < kPieces; k++)
#pragma unroll
                    for (int i = 0; i < kPiece; i++) u[k][i] = place.at(k) + i < a.n ? u[k][i] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < kPieces; k++)
#pragma unroll
            for (int i = 0; i < kPiece; i++) total[0] += u[k][i] * u[k][i];
        sum(total, a.lanes, wave, turn);
        const float rstd = 1.0f / sqrtf(total[0] * inv + a.eps);
#pragma unroll
        for (int k = 0; k < kPieces; k++)
#pragma unroll
            for (int i = 0; i < kPiece; i++) {
                const float v = u[k][i] * rstd * w[k][i] + c[k][i];
                u[k][i] = kAct == kSilu ? v * sigmoid_of(v) : kAct == kAfter ? v * gate[k][i] : v;
            }
        place.template store<IO>(a.y, row, u);
        if (row.real && lane % a.lanes == 0 && (kWaves == 1 || wave == 0)) {
            if (a.mean) a.mean[(long long)row.r * a.G + place.g] = mean;
            if (a.rstd) a.rstd[(long long)row.r * a.G + place.g] = rstd;
        }
    }
}

template <typename IO, int kAct, int kWaves, int kPieces, int kPiece, int kTeam, bool kPast, bool kMany>
__device__ __forceinline__ void group_norm_bwd_rows(const GroupNormArgs& a)
{
    __shared__ GroupSum<kWaves, 2> sum;
    constexpr bool kGated = kAct == kBefore || kAct == kAfter;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const GroupPlace<kWaves, kPieces, kPiece, kTeam, kPast, kMany> place(a, lane, wave);   // (r0 >= r1: a wave without rows, which leaves zeros)
    float w[kPieces][kPiece], c[kPieces][kPiece], dw[kPieces][kPiece], db[kPieces][kPiece];
    place.params(w, a.weight, 1.0f);
    if constexpr (kAct == kSilu || kAct == kAfter) place.params(c, a.bias, 0.0f);
#pragma unroll
    for (int k = 0; k < kPieces; k++)
#pragma unroll
        for (int i = 0; i < kPiece; i++) dw[k][i] = db[k][i] = 0.0f;
    const float inv = 1.0f / a.n;
    int turn = 0;
    struct Read {
        Piece<IO, kPiece> x[kPieces], z[kPieces], d[kPieces];
        float mean, rstd;
    };
    const auto read = [&](const auto& row) {
        Read p;
        place.template load<IO>(p.x, a.x, row);
        if constexpr (kGated) place.template load<IO>(p.z, a.z, row);
        place.template load<IO>(p.d, a.dy, row);
        p.mean = a.centred ? a.mean[(long long)row.r * a.G + place.g] : 0.0f;
        p.rstd = a.rstd[(long long)row.r * a.G + place.g];
        return p;
    };
    Read ahead;
    if (kWaves > 1 && place.r0 < place.r1) ahead = read(place.row(a, place.r0));
    for (unsigned r = place.r0; r < place.r1; r += place.at_once(a)) {
        const auto row = place.row(a, r);
        Read now = kWaves > 1 ? ahead : read(row);
        if (kWaves > 1 && place.r1 - r > place.at_once(a)) ahead = read(place.row(a, r + place.at_once(a)));
        auto &px = now.x, &pz = now.z, &pd = now.d;
        const float mean = now.mean, rstd = now.rstd;
        place.template settled<IO>(px);
        if constexpr (kGated) place.template settled<IO>(pz);
        place.template settled<IO>(pd);
        // xh, and k = dv * weight; what dz needs beside them
        float xh[kPieces][kPiece], g[kPieces][kPiece], dz[kPieces][kPiece], gate[kPieces][kPiece], total[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kPieces; k++)
#pragma unroll
            for (int i = 0; i < kPiece; i++) {
                float u = px[k][i], dv = pd[k][i];
                if constexpr (kGated) {
                    const float z = pz[k][i], s = sigmoid_of(z);
                    gate[k][i] = z * s;
                    dz[k][i] = s * (1.0f + z * (1.0f - s));
                    if constexpr (kAct == kBefore) u *= gate[k][i];
                }
                xh[k][i] = (u - mean) * rstd;
                if constexpr (kAct == kSilu || kAct == kAfter) {
                    const float v = xh[k][i] * w[k][i] + c[k][i];
                    if constexpr (kAct == kSilu) {
                        const float s = sigmoid_of(v);
                        dv *= s * (1.0f + v * (1.0f - s));
                    } else {
                        dz[k][i] *= dv * v;
                        dv *= gate[k][i];
                    }
                }
                dw[k][i] += !kMany || row.real ? dv * xh[k][i] : 0.0f;
                db[k][i] += !kMany || row.real ? dv : 0.0f;
                g[k][i] = dv * w[k][i];
                total[0] += g[k][i];
                total[1] += g[k][i] * xh[k][i];
            }
        sum(total, a.lanes, wave, turn);
        const float c0 = a.centred ? total[0] * inv : 0.0f, c1 = total[1] * inv;
#pragma unroll
        for (int k = 0; k < kPieces; k++)
#pragma unroll
            for (int i = 0; i < kPiece; i++) {
                const float du = rstd * (g[k][i] - c0 - xh[k][i] * c1);
                if constexpr (kAct == kBefore) {
                    dz[k][i] *= du * px[k][i];
                    g[k][i] = du * gate[k][i];
                } else {
                    g[k][i] = du;
                }
            }
        place.template store<IO>(a.dx, row, g);
        if constexpr (kGated) place.template store<IO>(a.dz, row, dz);
    }
    if constexpr (kMany) {   // the rows that a wave took at once
        for (int x = 64 / a.at_once; x < 64; x *= 2)
#pragma unroll
            for (int i = 0; i < kPiece; i++) {
                dw[0][i] += __shfl_xor(dw[0][i], x);
                db[0][i] += __shfl_xor(db[0][i], x);
            }
    }
    const long long slot = (long long)blockIdx.y * a.slot + place.channel();
    if constexpr (kWaves > 1) {
#pragma unroll
        for (int k = 0; k < kPieces; k++) {
            if (a.dw) store_piece_of<IoF32>(a.dw + slot, place.at(k), a.n, dw[k]);
            if (a.db) store_piece_of<IoF32>(a.db + slot, place.at(k), a.n, db[k]);
        }
    } else {   // the waves' sums of the same channels: one of the two at a time through shared memory
        __shared__ float all[kTeam][kPieces * kPiece][64];
#pragma unroll
        for (int which = 0; which < 2; which++) {
            float* const to = which ? a.db : a.dw;
            if (!to) continue;   // (all threads)
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kPieces; k++)
#pragma unroll
                for (int i = 0; i < kPiece; i++) all[wave][k * kPiece + i][lane] = which ? db[k][i] : dw[k][i];
            __syncthreads();
            if (wave != 0 || !place.real || place.run != 0) continue;
#pragma unroll
            for (int k = 0; k < kPieces; k++) {
                float f[kPiece];
#pragma unroll
                for (int i = 0; i < kPiece; i++) {
                    f[i] = all[0][k * kPiece + i][lane];
#pragma unroll
                    for (int m = 1; m < kTeam; m++) f[i] += all[m][k * kPiece + i][lane];
                }
                store_piece_of<IoF32>(to + slot, place.at(k), a.n, f);
            }
        }
    }
}

template <typename IO, int kAct, int kWaves, int kPieces, int kTeam, bool kPast, bool kMany>
__global__ __launch_bounds__(64 * kTeam) void group_norm_kernel(const GroupNormArgs a)
{
    if constexpr (kWaves == 1 && kPieces == 1) {   // (groups smaller than a piece: an element a lane)
        if (a.n < kPieceOf<IO>) return group_norm_rows<IO, kAct, 1, 1, 1, kTeam, kPast, kMany>(a);
    }
    group_norm_rows<IO, kAct, kWaves, kPieces, kPieceOf<IO>, kTeam, kPast, kMany>(a);
}
template <typename IO, int kAct, int kWaves, int kPieces, int kTeam, bool kPast, bool kMany>
__global__ __launch_bounds__(64 * kTeam) void group_norm_bwd_kernel(const GroupNormArgs a)
{
    if constexpr (kWaves == 1 && kPieces == 1) {
        if (a.n < kPieceOf<IO>) return group_norm_bwd_rows<IO, kAct, 1, 1, 1, kTeam, kPast, kMany>(a);
    }
    group_norm_bwd_rows<IO, kAct, kWaves, kPieces, kPieceOf<IO>, kTeam, kPast, kMany>(a);
}

namespace {

template <typename IO, int kAct, int kWaves, int kPieces, int kTeam, bool kPast, bool kMany = false>
void launch_form(const GroupPlan& p, const GroupNormArgs& a, bool bwd, hipStream_t st)
{
    const dim3 grid(p.tiles, p.row_groups), wg(64 * kTeam);
    constexpr bool kOne = kWaves == 1 && kPieces == 1 && !kMany;   // (gradients in teams of eight, the norm in teams of four)
    if (bwd) {
        if constexpr (!kOne || kTeam == 8) hipLaunchKernelGGL((group_norm_bwd_kernel<IO, kAct, kWaves, kPieces, kTeam, kPast, kMany>), grid, wg, 0, st, a);
    } else {
        if constexpr (!kOne || kTeam == 4) hipLaunchKernelGGL((group_norm_kernel<IO, kAct, kWaves, kPieces, kTeam, kPast, kMany>), grid, wg, 0, st, a);
    }
}
template <typename IO, int kAct, bool kPast>
void launch_io(const GroupPlan& p, const GroupNormArgs& a, bool bwd, hipStream_t st)
{
    constexpr int kWide = sizeof(typename IO::T) == 4 ? 2 : 1;   // (twice the pieces for as many elements)
    if (p.waves == 8) {
        if (p.pieces <= kWide) launch_form<IO, kAct, 8, kWide, 8, kPast>(p, a, bwd, st);
        else launch_form<IO, kAct, 8, 2 * kWide, 8, kPast>(p, a, bwd, st);
    } else if (p.waves == 4) {
        launch_form<IO, kAct, 4, kWide, 4, kPast>(p, a, bwd, st);
    } else if (p.pieces == 1) {
        if (p.at_once > 1) launch_form<IO, kAct, 1, 1, 4, kPast, true>(p, a, bwd, st);
        else if (bwd) launch_form<IO, kAct, 1, 1, 8, kPast>(p, a, bwd, st);
        else launch_form<IO, kAct, 1, 1, 4, kPast>(p, a, bwd, st);
    } else if (p.pieces == 2) {
        launch_form<IO, kAct, 1, 2, 4, kPast>(p, a, bwd, st);
    } else if constexpr (kWide == 2) {
        launch_form<IO, kAct, 1, 4, 4, kPast>(p, a, bwd, st);
    }
}

}  // namespace

template <>
void launch_group_norm<BM_ACT>(const GroupPlan& p, const GroupNormArgs& a, bool bf16, bool past, bool bwd, hipStream_t st)
{
    if (bf16) past ? launch_io<IoBF16, BM_ACT, true>(p, a, bwd, st) : launch_io<IoBF16, BM_ACT, false>(p, a, bwd, st);
    else past ? launch_io<IoF32, BM_ACT, true>(p, a, bwd, st) : launch_io<IoF32, BM_ACT, false>(p, a, bwd, st);
}

}  // namespace bm
