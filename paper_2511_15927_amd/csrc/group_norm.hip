// The norm of groups of channels with an activation or a gate, and its gradients.
#include "slot_sums.h"

namespace bm {

// A token's group stays in registers: 2^k lanes hold it in pieces of 16 bytes, up to 32 elements a lane, so a wave has 64 / lanes
// neighbouring groups of a row in hand (one, with four waves to it, beyond 2048 channels).  It takes rows one after the other with weight
// and bias in registers; the gradients' sums for these two stay there as well and are left in a slot at the end.  The statistics are taken
// over the registers, the mean before the squares around it, so that a large mean costs no digits.  All arithmetic is fp32, each
// output is rounded once.
struct GroupNormArgs {
    RowView x, z, y, dy, dx, dz;
    const float *weight, *bias;   // null: 1, 0
    float *mean, *rstd;           // [rows][G]; forward: null, not wanted
    float *dw, *db;               // sums of a row group, null: not wanted
    long long slot;               // from one row group's to the next one's
    unsigned L, rows, per_wave;   // rows that a wave (or the four of a wide group) takes
    int G, n, d, lanes;           // groups, channels of one; lanes that hold one
    int centred;
    float eps;
};
enum Act { kPlain = BIMAMBA_ACT_NONE, kSilu = BIMAMBA_ACT_SILU, kBefore = BIMAMBA_ACT_GATE_BEFORE, kAfter = BIMAMBA_ACT_GATE_AFTER };

__device__ __forceinline__ float sigmoid_of(float v) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * v)); }

// Two values summed over each run of `lanes` lanes, the same in all of a run.
__device__ __forceinline__ void run_sum(float& u, float& v, int lanes)
{
#define BM_DPP(x, ctrl) __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl, 0xf, 0xf, true))
    if (lanes < 2) return;
    u += BM_DPP(u, 0xB1), v += BM_DPP(v, 0xB1);     // quad_perm 1 0 3 2
    if (lanes < 4) return;
    u += BM_DPP(u, 0x4E), v += BM_DPP(v, 0x4E);     // quad_perm 2 3 0 1
    if (lanes < 8) return;
    u += BM_DPP(u, 0x141), v += BM_DPP(v, 0x141);   // row_half_mirror
    if (lanes < 16) return;
    u += BM_DPP(u, 0x140), v += BM_DPP(v, 0x140);   // row_mirror
#undef BM_DPP
    if (lanes < 32) return;
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(u), __float_as_uint(u), false, false);
    u = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    if (lanes < 64) return;
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(u), __float_as_uint(u), false, false);
    u = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The sums of a group from those of its lanes; kWaves 4: over the waves as well, two barriers apart from the next use of the same turn.
template <int kWaves>
struct GroupSum {
    float2 part[2][kWaves];
    __device__ __forceinline__ void operator()(float& u, float& v, int lanes, int wave, int turn)
    {
        run_sum(u, v, lanes);
        if constexpr (kWaves > 1) {
            part[turn][wave] = make_float2(u, v);
            __syncthreads();
            u = part[turn][0].x, v = part[turn][0].y;
#pragma unroll
            for (int k = 1; k < kWaves; k++) u += part[turn][k].x, v += part[turn][k].y;
        }
    }
};

// Where a lane's elements lie and which rows its wave takes.
template <int kWaves, int kPieces, int kPiece>
struct GroupPlace {
    int g, in, n, stride;
    bool real, whole;   // whether the lane's group exists; (wave-uniform) every piece of every lane lies within its group
    unsigned r0, r1;
    __device__ __forceinline__ GroupPlace(const GroupNormArgs& a, int lane, int wave) : n(a.n)
    {
        const int runs = 64 / a.lanes, first = blockIdx.x * runs;
        g = first + lane / a.lanes;
        real = g < a.G;
        g = min(g, a.G - 1);
        in = (lane % a.lanes + (kWaves > 1 ? wave * kPieces * 64 : 0)) * kPiece;
        stride = a.lanes * kPiece;
        whole = first + runs <= a.G && a.n == kWaves * kPieces * stride;
        const unsigned group = kWaves == 1 ? blockIdx.y * 4 + wave : blockIdx.y;
        r0 = min(group * a.per_wave, a.rows);
        r1 = min(r0 + a.per_wave, a.rows);
    }
    __device__ __forceinline__ int at(int k) const { return in + k * stride; }
    __device__ __forceinline__ int channel() const { return g * n; }
    template <typename IO>
    __device__ __forceinline__ void load(Piece<IO, kPiece> (&p)[kPieces], const RowView& v, unsigned b, unsigned t) const
    {
        const typename IO::T* const row = static_cast<const typename IO::T*>(v.p) + row_offset(v, b, t) + channel();
#pragma unroll
        for (int k = 0; k < kPieces; k++) p[k] = load_clamped<IO, kPiece>(row, at(k), n);
    }
    template <typename IO>
    __device__ __forceinline__ void settled(Piece<IO, kPiece> (&p)[kPieces]) const
    {
        if (whole) return;
#pragma unroll
        for (int k = 0; k < kPieces; k++) settle(p[k], at(k), n, typename IO::T(0));
    }
    template <typename IO>
    __device__ __forceinline__ void store(const RowView& v, unsigned b, unsigned t, const float (&f)[kPieces][kPiece]) const
    {
        typename IO::T* const row = static_cast<typename IO::T*>(v.p) + row_offset(v, b, t) + channel();
#pragma unroll
        for (int k = 0; k < kPieces; k++) {
            if (whole) store_piece<IO>(row + at(k), f[k]);
            else if (real) store_piece_of<IO>(row, at(k), n, f[k]);
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

template <typename IO, int kAct, int kWaves, int kPieces, int kPiece>
__device__ __forceinline__ void group_norm_rows(const GroupNormArgs& a)
{
    __shared__ GroupSum<kWaves> sum;
    constexpr bool kGated = kAct == kBefore || kAct == kAfter;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const GroupPlace<kWaves, kPieces, kPiece> place(a, lane, wave);
    if (place.r0 >= place.r1) return;   // (with four waves to a group: the whole workgroup)
    float w[kPieces][kPiece], c[kPieces][kPiece];
    place.params(w, a.weight, 1.0f);
    place.params(c, a.bias, 0.0f);
    const float inv = 1.0f / a.n;
    unsigned b = place.r0 / a.L, t = place.r0 - b * a.L;
    Piece<IO, kPiece> px[kPieces], pz[kPieces];
    place.template load<IO>(px, a.x, b, t);
    if constexpr (kGated) place.template load<IO>(pz, a.z, b, t);
    for (unsigned r = place.r0; r < place.r1; r++) {
        float u[kPieces][kPiece], gate[kPieces][kPiece], s0 = 0.0f, s1 = 0.0f;
        place.template settled<IO>(px);
        if constexpr (kGated) place.template settled<IO>(pz);
#pragma unroll
        for (int k = 0; k < kPieces; k++)
#pragma unroll
            for (int i = 0; i < kPiece; i++) {
                u[k][i] = px[k][i];
                if constexpr (kGated) gate[k][i] = pz[k][i] * sigmoid_of(pz[k][i]);
                if constexpr (kAct == kBefore) u[k][i] *= gate[k][i];
                s0 += u[k][i];
                s1 += u[k][i] * u[k][i];
            }
        const unsigned b0 = b, t0 = t;
        if (++t == a.L) t = 0, b++;
        if (r + 1 < place.r1) {
            place.template load<IO>(px, a.x, b, t);
            if constexpr (kGated) place.template load<IO>(pz, a.z, b, t);
        }
        sum(s0, s1, a.lanes, wave, 0);
        float mean = 0.0f;
        if (a.centred) {
            mean = s0 * inv;
            s0 = s1 = 0.0f;
#pragma unroll
            for (int k = 0; k < kPieces; k++)
#pragma unroll
                for (int i = 0; i < kPiece; i++) {
                    u[k][i] -= mean;
                    s1 += place.whole || place.at(k) + i < a.n ? u[k][i] * u[k][i] : 0.0f;
                }
            sum(s0, s1, a.lanes, wave, 1);
        } else if constexpr (kWaves > 1) {
            __syncthreads();
        }
        const float rstd = 1.0f / sqrtf(s1 * inv + a.eps);
#pragma unroll
        for (int k = 0; k < kPieces; k++)
#pragma unroll
            for (int i = 0; i < kPiece; i++) {
                const float v = u[k][i] * rstd * w[k][i] + c[k][i];
                u[k][i] = kAct == kSilu ? v * sigmoid_of(v) : kAct == kAfter ? v * gate[k][i] : v;
            }
        place.template store<IO>(a.y, b0, t0, u);
        if (place.real && lane % a.lanes == 0 && (kWaves == 1 || wave == 0)) {
            if (a.mean) a.mean[(long long)r * a.G + place.g] = mean;
            if (a.rstd) a.rstd[(long long)r * a.G + place.g] = rstd;
        }
    }
}

template <typename IO, int kAct, int kWaves, int kPieces, int kPiece>
__device__ __forceinline__ void group_norm_bwd_rows(const GroupNormArgs& a)
{
    __shared__ GroupSum<kWaves> sum;
    constexpr bool kGated = kAct == kBefore || kAct == kAfter;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const GroupPlace<kWaves, kPieces, kPiece> place(a, lane, wave);   // (r0 >= r1: a wave without rows, which leaves zeros)
    float w[kPieces][kPiece], c[kPieces][kPiece], dw[kPieces][kPiece], db[kPieces][kPiece];
    place.params(w, a.weight, 1.0f);
    if constexpr (kAct == kSilu || kAct == kAfter) place.params(c, a.bias, 0.0f);
#pragma unroll
    for (int k = 0; k < kPieces; k++)
#pragma unroll
        for (int i = 0; i < kPiece; i++) dw[k][i] = db[k][i] = 0.0f;
    const float inv = 1.0f / a.n;
    unsigned b = place.r0 / a.L, t = place.r0 - b * a.L;
    for (unsigned r = place.r0; r < place.r1; r++) {
        Piece<IO, kPiece> px[kPieces], pz[kPieces], pd[kPieces];
        place.template load<IO>(px, a.x, b, t);
        if constexpr (kGated) place.template load<IO>(pz, a.z, b, t);
        place.template load<IO>(pd, a.dy, b, t);
        const float mean = a.centred ? a.mean[(long long)r * a.G + place.g] : 0.0f, rstd = a.rstd[(long long)r * a.G + place.g];
        place.template settled<IO>(px);
        if constexpr (kGated) place.template settled<IO>(pz);
        place.template settled<IO>(pd);
        // xh, and k = dv * weight; what dz needs beside them
        float xh[kPieces][kPiece], g[kPieces][kPiece], dz[kPieces][kPiece], gate[kPieces][kPiece], s0 = 0.0f, s1 = 0.0f;
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
                dw[k][i] += dv * xh[k][i];
                db[k][i] += dv;
                g[k][i] = dv * w[k][i];
                s0 += g[k][i];
                s1 += g[k][i] * xh[k][i];
            }
        sum(s0, s1, a.lanes, wave, (r - place.r0) & 1);
        const float c0 = a.centred ? s0 * inv : 0.0f, c1 = s1 * inv;
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
        place.template store<IO>(a.dx, b, t, g);
        if constexpr (kGated) place.template store<IO>(a.dz, b, t, dz);
        if (++t == a.L) t = 0, b++;
    }
    const long long slot = (long long)blockIdx.y * a.slot + place.channel();
    if constexpr (kWaves > 1) {
#pragma unroll
        for (int k = 0; k < kPieces; k++) {
            if (a.dw) store_piece_of<IoF32>(a.dw + slot, place.at(k), a.n, dw[k]);
            if (a.db) store_piece_of<IoF32>(a.db + slot, place.at(k), a.n, db[k]);
        }
    } else {   // four waves' sums of the same channels: one of the two at a time through shared memory
        __shared__ float all[4][kPieces * kPiece][64];
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
            if (wave != 0 || !place.real) continue;
#pragma unroll
            for (int k = 0; k < kPieces; k++) {
                float f[kPiece];
#pragma unroll
                for (int i = 0; i < kPiece; i++) {
                    const int e = k * kPiece + i;
                    f[i] = (all[0][e][lane] + all[1][e][lane]) + (all[2][e][lane] + all[3][e][lane]);
                }
                store_piece_of<IoF32>(to + slot, place.at(k), a.n, f);
            }
        }
    }
}

template <typename IO, int kAct, int kWaves, int kPieces>
__global__ __launch_bounds__(256) void group_norm_kernel(const GroupNormArgs a)
{
    if constexpr (kWaves == 1 && kPieces == 1) {   // (groups smaller than a piece: an element a lane)
        if (a.n < kPieceOf<IO>) return group_norm_rows<IO, kAct, 1, 1, 1>(a);
    }
    group_norm_rows<IO, kAct, kWaves, kPieces, kPieceOf<IO>>(a);
}
template <typename IO, int kAct, int kWaves, int kPieces>
__global__ __launch_bounds__(256) void group_norm_bwd_kernel(const GroupNormArgs a)
{
    if constexpr (kWaves == 1 && kPieces == 1) {
        if (a.n < kPieceOf<IO>) return group_norm_bwd_rows<IO, kAct, 1, 1, 1>(a);
    }
    group_norm_bwd_rows<IO, kAct, kWaves, kPieces, kPieceOf<IO>>(a);
}

namespace {

constexpr int kMaxWidth = 65536, kMaxGroup = 8192;

int check_group_norm(const bimamba_group_norm_desc* d)
{
    if (!d) return BIMAMBA_ERR_NULL_POINTER;
    if (d->struct_size != sizeof(bimamba_group_norm_desc) || d->d_inner < 1 || d->groups < 1 || d->d_inner % d->groups) return BIMAMBA_ERR_BAD_SHAPE;
    if (!(d->eps > 0.0f) || !std::isfinite(d->eps) || (d->centred != 0 && d->centred != 1)) return BIMAMBA_ERR_BAD_SHAPE;
    if (const int rc = check_rows(d->batch, d->seqlen)) return rc;
    if (!known_dtype(d->io_dtype) || d->act < BIMAMBA_ACT_NONE || d->act > BIMAMBA_ACT_GATE_AFTER) return BIMAMBA_ERR_UNSUPPORTED;
    return d->d_inner > kMaxWidth || d->d_inner / d->groups > kMaxGroup ? BIMAMBA_ERR_UNSUPPORTED : BIMAMBA_OK;
}
bool gated(const bimamba_group_norm_desc* d) { return d->act == BIMAMBA_ACT_GATE_BEFORE || d->act == BIMAMBA_ACT_GATE_AFTER; }

struct GroupPlan {
    int waves, pieces, lanes;
    unsigned tiles, row_groups, per_wave;
};
GroupPlan plan_group_norm(const bimamba_group_norm_desc* d, bool bwd)
{
    GroupPlan p{};
    const int n = d->d_inner / d->groups, piece = d->io_dtype == BIMAMBA_BF16 ? 8 : 4;
    const int pieces = n < piece ? n : (n + piece - 1) / piece;   // (of one element in small groups)
    p.waves = n > 64 * 32 ? 4 : 1;
    p.lanes = 1;
    while (p.lanes < 64 && p.lanes < pieces) p.lanes *= 2;
    p.pieces = 1;
    while (p.pieces * p.lanes * p.waves < pieces) p.pieces *= 2;
    const int runs = 64 / p.lanes;
    p.tiles = (d->groups + runs - 1) / runs;
    const unsigned rows = (unsigned)((long long)d->batch * d->seqlen), together = p.waves == 1 ? 4 : 1, want = (bwd ? 8u : 16u) * cu_count();
    unsigned groups = (want + p.tiles - 1) / p.tiles;
    if (bwd && groups > rows / 8) groups = rows / 8 ? rows / 8 : 1;   // (each leaves a slot as long as two rows)
    p.per_wave = (rows + groups * together - 1) / (groups * together);
    if (p.per_wave < 1) p.per_wave = 1;
    const unsigned long long step = (unsigned long long)p.per_wave * together;
    p.row_groups = (unsigned)((rows + step - 1) / step);
    return p;
}

template <typename IO, int kAct, int kWaves, int kPieces>
void launch_one(const GroupPlan& p, const GroupNormArgs& a, bool bwd, hipStream_t st)
{
    const dim3 grid(p.tiles, p.row_groups), wg(256);
    if (bwd) hipLaunchKernelGGL((group_norm_bwd_kernel<IO, kAct, kWaves, kPieces>), grid, wg, 0, st, a);
    else hipLaunchKernelGGL((group_norm_kernel<IO, kAct, kWaves, kPieces>), grid, wg, 0, st, a);
}
template <typename IO, int kAct>
void launch_act(const GroupPlan& p, const GroupNormArgs& a, bool bwd, hipStream_t st)
{
    constexpr bool kWide = sizeof(typename IO::T) == 4;   // (twice the pieces for as many elements)
    if (p.waves == 4) {
        if (kWide ? p.pieces <= 4 : p.pieces <= 2) launch_one<IO, kAct, 4, kWide ? 4 : 2>(p, a, bwd, st);
        else launch_one<IO, kAct, 4, kWide ? 8 : 4>(p, a, bwd, st);
        return;
    }
    switch (p.pieces) {
        case 1: launch_one<IO, kAct, 1, 1>(p, a, bwd, st); break;
        case 2: launch_one<IO, kAct, 1, 2>(p, a, bwd, st); break;
        case 4: launch_one<IO, kAct, 1, 4>(p, a, bwd, st); break;
        default: if constexpr (kWide) launch_one<IO, kAct, 1, 8>(p, a, bwd, st);
    }
}
template <typename IO>
void launch_io(const bimamba_group_norm_desc* d, const GroupPlan& p, const GroupNormArgs& a, bool bwd, hipStream_t st)
{
    switch (d->act) {
        case BIMAMBA_ACT_NONE: launch_act<IO, kPlain>(p, a, bwd, st); break;
        case BIMAMBA_ACT_SILU: launch_act<IO, kSilu>(p, a, bwd, st); break;
        case BIMAMBA_ACT_GATE_BEFORE: launch_act<IO, kBefore>(p, a, bwd, st); break;
        default: launch_act<IO, kAfter>(p, a, bwd, st);
    }
}
void launch(const bimamba_group_norm_desc* d, const GroupPlan& p, GroupNormArgs& a, bool bwd, hipStream_t st)
{
    a.L = d->seqlen, a.rows = (unsigned)((long long)d->batch * d->seqlen), a.per_wave = p.per_wave;
    a.G = d->groups, a.n = d->d_inner / d->groups, a.d = d->d_inner, a.lanes = p.lanes, a.centred = d->centred, a.eps = d->eps;
    if (d->io_dtype == BIMAMBA_BF16) launch_io<IoBF16>(d, p, a, bwd, st);
    else launch_io<IoF32>(d, p, a, bwd, st);
}

int check_params(const float* p, long long count, Bytes* r)
{
    *r = bytes_of(p, count, 4);
    return aligned_to(p, 4) ? BIMAMBA_OK : BIMAMBA_ERR_MISALIGNED;
}

}  // namespace
}  // namespace bm

using namespace bm;

extern "C" {

int bimamba_group_norm(const bimamba_group_norm_desc* d, const bimamba_tensor* x, const bimamba_tensor* z, const float* weight,
                       const float* bias, const bimamba_tensor* y, float* mean, float* rstd, void* hip_stream)
{
    int rc = check_group_norm(d);
    if (rc) return rc;
    if (!x || !y || (gated(d) && !z)) return BIMAMBA_ERR_NULL_POINTER;
    if ((z && !gated(d)) || (mean && !d->centred)) return BIMAMBA_ERR_UNSUPPORTED;
    if (d->batch == 0 || d->seqlen == 0) return BIMAMBA_OK;
    const int Bt = d->batch, L = d->seqlen, D = d->d_inner, io = d->io_dtype;
    const long long stats = (long long)Bt * L * d->groups;
    const size_t elem = dtype_bytes(io);
    Bytes bx, bz{}, by, bw, bb, bm_, br;
    if ((rc = check_view(x, Bt, L, D, io, false, &bx)) || (z && (rc = check_view(z, Bt, L, D, io, false, &bz))) ||
        (rc = check_view(y, Bt, L, D, io, true, &by)) || (rc = check_params(weight, D, &bw)) || (rc = check_params(bias, D, &bb)) ||
        (rc = check_params(mean, stats, &bm_)) || (rc = check_params(rstd, stats, &br)))
        return rc;
    if (views_meet(y, D, by, x, D, bx, Bt, elem, elem) || (z && views_meet(y, D, by, z, D, bz, Bt, elem, elem))) return BIMAMBA_ERR_ALIAS;
    const Bytes written[] = {by, bm_, br}, read[] = {bw, bb, bx, bz};
    for (int i = 0; i < 3; i++) {
        for (int j = 0; j < (i == 0 ? 2 : 4); j++)
            if (meet(written[i], read[j])) return BIMAMBA_ERR_ALIAS;
        for (int j = 0; j < i; j++)
            if (meet(written[i], written[j])) return BIMAMBA_ERR_ALIAS;
    }
    GroupNormArgs a{};
    a.x = row_view(x), a.y = row_view(y);
    if (z) a.z = row_view(z);
    a.weight = weight, a.bias = bias, a.mean = mean, a.rstd = rstd;
    const Launches launches;
    launch(d, plan_group_norm(d, false), a, false, reinterpret_cast<hipStream_t>(hip_stream));
    return launches.status();
}

size_t bimamba_group_norm_bwd_workspace_bytes(const bimamba_group_norm_desc* d)
{
    if (check_group_norm(d) || d->batch == 0 || d->seqlen == 0) return 0;
    const GroupPlan p = plan_group_norm(d, true);
    return p.row_groups > 1 ? (size_t)p.row_groups * 2 * d->d_inner * sizeof(float) : 0;
}

int bimamba_group_norm_bwd(const bimamba_group_norm_desc* d, const bimamba_tensor* x, const bimamba_tensor* z, const float* weight,
                           const float* bias, const float* mean, const float* rstd, const bimamba_tensor* dy, const bimamba_tensor* dx,
                           const bimamba_tensor* dz, float* dweight, float* dbias, void* workspace, size_t workspace_bytes,
                           void* hip_stream)
{
    int rc = check_group_norm(d);
    if (rc) return rc;
    const bool rows = d->batch && d->seqlen, sums = dweight || dbias;
    if (!x || !dy || !dx || (gated(d) && (!z || !dz))) return BIMAMBA_ERR_NULL_POINTER;
    if (((z || dz) && !gated(d)) || (mean && !d->centred)) return BIMAMBA_ERR_UNSUPPORTED;
    const int Bt = d->batch, L = d->seqlen, D = d->d_inner, io = d->io_dtype;
    Bytes bw, bb, bdw, bdb;
    if ((rc = check_params(weight, D, &bw)) || (rc = check_params(bias, D, &bb)) || (rc = check_params(dweight, D, &bdw)) || (rc = check_params(dbias, D, &bdb)))
        return rc;
    const size_t need = rows && sums ? bimamba_group_norm_bwd_workspace_bytes(d) : 0;
    Bytes bx{}, bz{}, by{}, bdx{}, bdz{}, bm_{}, br{};
    if (rows) {
        if (!rstd || (d->centred && !mean)) return BIMAMBA_ERR_NULL_POINTER;
        const long long stats = (long long)Bt * L * d->groups;
        if ((rc = check_view(x, Bt, L, D, io, false, &bx)) || (z && (rc = check_view(z, Bt, L, D, io, false, &bz))) ||
            (rc = check_view(dy, Bt, L, D, io, false, &by)) || (rc = check_view(dx, Bt, L, D, io, true, &bdx)) ||
            (dz && (rc = check_view(dz, Bt, L, D, io, true, &bdz))) || (rc = check_params(mean, stats, &bm_)) || (rc = check_params(rstd, stats, &br)))
            return rc;
        if ((rc = check_workspace(workspace, workspace_bytes, need))) return rc;
        const size_t elem = dtype_bytes(io);
        const bimamba_tensor *const in[] = {x, dy, z}, *const out[] = {dx, dz};
        const Bytes from[] = {bx, by, bz}, to[] = {bdx, bdz};
        for (int i = 0; i < (dz ? 2 : 1); i++)
            for (int j = 0; j < (z ? 3 : 2); j++)
                if (views_meet(out[i], D, to[i], in[j], D, from[j], Bt, elem, elem)) return BIMAMBA_ERR_ALIAS;
        if (dz && views_meet(dx, D, bdx, dz, D, bdz, Bt, elem, elem)) return BIMAMBA_ERR_ALIAS;
    }
    const Bytes ws = bytes_of(need ? workspace : nullptr, need, 1);
    const Bytes written[] = {bdx, bdz, bdw, bdb, ws}, read[] = {bw, bb, bm_, br, bx, by, bz};
    for (int i = 0; i < 5; i++) {
        for (int j = 0; j < (i < 2 ? 4 : 7); j++)
            if (meet(written[i], read[j])) return BIMAMBA_ERR_ALIAS;
        for (int j = 0; j < i; j++)
            if (meet(written[i], written[j]) && !(i == 1 && j == 0)) return BIMAMBA_ERR_ALIAS;
    }
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    const GroupPlan p = rows ? plan_group_norm(d, true) : GroupPlan{};
    const bool direct = rows && p.row_groups == 1;
    float* const slots = static_cast<float*>(workspace);
    if (rows) {
        GroupNormArgs a{};
        a.x = row_view(x), a.dy = row_view(dy), a.dx = row_view(dx);
        if (z) a.z = row_view(z), a.dz = row_view(dz);
        a.weight = weight, a.bias = bias, a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd);
        a.dw = dweight ? direct ? dweight : slots : nullptr;
        a.db = dbias ? direct ? dbias : slots + D : nullptr;
        a.slot = 2ll * D;
        launch(d, p, a, true, st);
    }
    if (sums && !direct) launch_slot_sum(SlotSumArgs{{slots, slots + D}, {dweight, dbias}, p.row_groups, 2ll * D, D}, 1, st);
    return launches.status();
}

}  // extern "C"
