// The gated linear recurrence h = a h + u, channel by channel, in either direction along the sequence, and its gradients.
#include "slot_sums.h"

namespace bm {

// A workgroup walks a segment of the sequence for the channels of one wave: in each step its kW waves take kT tokens each, which stay in
// registers.  A wave first runs its tokens from a state of zero, which gives the state E that they add and the factor P that they put
// on what enters; the pairs are exchanged through shared memory, each wave folds those before it onto the state that entered the step
// and runs its tokens again from there.  So the activations are read once, one barrier a step.  Where there are too few channels for
// the chip the sequence is cut into segments: a launch before this one leaves every segment's (P, E), and a segment starts from the fold
// of those before it; that reads the activations twice.  (The state that enters goes through the links too: it may be replaced by the one
// that leaves while other segments start.)
//
// Everything is in fp32: a, u, the states; y is rounded once.  1 - a is formed beside a from the same exponential, not as a difference, so
// that neither loses digits where the other is near 1: with e = exp(-|v|), sigmoid(|v|) = 1 - e / (1 + e) and sigmoid(-|v|) = e / (1 + e).
constexpr int kKeep = 64;   // tokens between two kept states

enum Gate { kLog, kSigmoid };

struct RecurArgs {
    RowView x, g, add, y;    // add.p null: none
    RowView dy, dx, dg;      // gradients
    const float* bias;       // null: 0
    const int64_t* lengths;  // null: L
    const float* enter;      // [batch][d], null: 0; the state before the first token (gradients: that of the state after the last)
    float* leave;            // [batch][d] or null: the state after the last (gradients: that of the state before the first)
    float* states;           // [batch][ceil(L / kKeep)][d] or null
    float* dbias;            // [batch * nseg][d] or null
    float* links;            // [batch][nseg][2][d] with several segments: 0 and `enter`, then P, E of the segments in walking order (gradients: P, Q)
    int L, d, nseg, seg_len, reverse;
};

// The tokens that the steps of a scan take.
struct Places {
    int len, reverse;
    __device__ __forceinline__ Places(const RecurArgs& a, int b) : len(a.L), reverse(a.reverse)
    {
        if (a.lengths) len = (int)max(0ll, min((long long)a.L, (long long)a.lengths[b]));
    }
    // One that may be read for step s: beyond the end some other one.
    __device__ __forceinline__ int readable(int s) const
    {
        const int k = min(s, len - 1);
        return max(0, reverse ? len - 1 - k : k);
    }
    // The one that step s writes.
    __device__ __forceinline__ int written(int s) const { return reverse && s < len ? len - 1 - s : s; }
};

template <typename IO, int kC>
struct Channels {
    int at, d;
    bool whole;   // (wave-uniform) all lanes' channels exist
    __device__ __forceinline__ Channels(int first, int lane, int d) : at(first + lane * kC), d(d), whole(first + 64 * kC <= d) {}
    typedef Piece<IO, kC> Raw;
    __device__ __forceinline__ Raw load(const RowView& v, int b, int t) const
    {
        return load_clamped<IO, kC>(static_cast<const typename IO::T*>(v.p) + row_offset(v, b, t), at, d);
    }
    __device__ __forceinline__ void settled(Raw& r) const
    {
        if (!whole) settle(r, at, d, typename IO::T(0));
    }
    __device__ __forceinline__ void store(const RowView& v, int b, int t, const float (&f)[kC]) const
    {
        typename IO::T* const row = static_cast<typename IO::T*>(v.p) + row_offset(v, b, t);
        if (whole) store_piece<IO>(row + at, f);
        else store_piece_of<IO>(row, at, d, f);
    }
    __device__ __forceinline__ void load_params(float (&f)[kC], const float* p) const
    {
#pragma unroll
        for (int k = 0; k < kC; k++) f[k] = p && at + k < d ? p[at + k] : 0.0f;
    }
    __device__ __forceinline__ void store_params(float* p, const float (&f)[kC]) const
    {
#pragma unroll
        for (int k = 0; k < kC; k++)
            if (at + k < d) p[at + k] = f[k];
    }
};

// a, and for a sigmoid gate 1 - a, for a log gate the factor that da / dg is (a, or 0 where g > 0 was cut).
template <int kGate>
__device__ __forceinline__ void gate_of(float g, float bias, float& a, float& q)
{
    if constexpr (kGate == kSigmoid) {
        const float v = g + bias, e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(v)), low = e * __builtin_amdgcn_rcpf(1.0f + e), high = 1.0f - low;
        a = v > 0.0f ? high : low;
        q = v > 0.0f ? low : high;
    } else {
        a = __builtin_amdgcn_exp2f(kLog2e * (g > 0.0f ? 0.0f : g));   // (a NaN stays one)
        q = g > 0.0f ? 0.0f : a;
    }
}

template <int kC>
struct Link {
    float p[kC], e[kC];
};

// What enters the segment that comes `turn` segments after the first one walked.
template <typename IO, int kC>
__device__ __forceinline__ void enter(float (&carry)[kC], const Channels<IO, kC>& ch, const RecurArgs& r, int b, int turn)
{
    if (r.nseg == 1) {
        ch.load_params(carry, r.enter ? r.enter + (long long)b * r.d : nullptr);
        return;
    }
    const float* link = r.links + (long long)b * r.nseg * 2 * r.d;
#pragma unroll
    for (int j = 0; j < kC; j++) carry[j] = 0.0f;
#pragma unroll 4
    for (int k = 0; k <= turn; k++, link += 2 * r.d) {
        float p[kC], e[kC];
        ch.load_params(p, link);
        ch.load_params(e, link + r.d);
#pragma unroll
        for (int j = 0; j < kC; j++) carry[j] = p[j] * carry[j] + e[j];
    }
}

template <typename IO, int kGate, int kC, int kT, int kW, int kV>
__global__ __launch_bounds__(64 * kW * kV) void recur_kernel(const RecurArgs r)
{
    __shared__ Link<kC> part[2][kW][kV * 64];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), w = wave % kW, v = wave / kW;
    const int tiles = (r.d + 64 * kC * kV - 1) / (64 * kC * kV), tile = blockIdx.x % tiles, seg = blockIdx.x / tiles, b = blockIdx.y;
    const Channels<IO, kC> ch((tile * kV + v) * 64 * kC, lane, r.d);
    const Places places(r, b);
    const int p0 = seg * r.seg_len, p1 = min(p0 + r.seg_len, r.L), column = v * 64 + lane;
    float bias[kC], carry[kC];
    ch.load_params(bias, r.bias);
    enter(carry, ch, r, b, seg);
    Piece<IO, kC> nx[kT], ng[kT], nadd[kT];
    const auto request = [&](int base) {
#pragma unroll
        for (int i = 0; i < kT; i++) {
            const int t = places.readable(base + w * kT + i);
            nx[i] = ch.load(r.x, b, t);
            ng[i] = ch.load(r.g, b, t);
        }
    };
    request(p0);
    int turn = 0;
    for (int base = p0; base < p1; base += kW * kT, turn ^= 1) {
        const int s0 = base + w * kT;
        float a[kT][kC], u[kT][kC];
        Link<kC> mine;
#pragma unroll
        for (int j = 0; j < kC; j++) mine.p[j] = 1.0f, mine.e[j] = 0.0f;
        if (r.add.p)
#pragma unroll
            for (int i = 0; i < kT; i++) nadd[i] = ch.load(r.add, b, places.readable(s0 + i));
#pragma unroll
        for (int i = 0; i < kT; i++) {
            ch.settled(nx[i]);
            ch.settled(ng[i]);
            const bool inside = s0 + i < places.len;
#pragma unroll
            for (int j = 0; j < kC; j++) {
                float q;
                gate_of<kGate>(ng[i][j], bias[j], a[i][j], q);
                u[i][j] = kGate == kSigmoid ? q * nx[i][j] : nx[i][j];
                if (!inside) a[i][j] = 1.0f, u[i][j] = 0.0f;
                mine.e[j] = a[i][j] * mine.e[j] + u[i][j];
                mine.p[j] *= a[i][j];
            }
        }
        if (base + kW * kT < p1) request(base + kW * kT);
        float h[kC];
#pragma unroll
        for (int j = 0; j < kC; j++) h[j] = carry[j];
        if constexpr (kW > 1) {
            part[turn][w][column] = mine;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kW; k++) {
                const Link<kC> link = part[turn][k][column];
#pragma unroll
                for (int j = 0; j < kC; j++) {
                    carry[j] = link.p[j] * carry[j] + link.e[j];
                    if (k + 1 == w) h[j] = carry[j];
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < kC; j++) carry[j] = mine.p[j] * carry[j] + mine.e[j];
        }
        if (r.states && s0 % kKeep == 0 && s0 < p1) ch.store_params(r.states + ((long long)b * ((r.L + kKeep - 1) / kKeep) + s0 / kKeep) * r.d, h);
#pragma unroll
        for (int i = 0; i < kT; i++) {
            const int s = s0 + i;
            float f[kC];
            if (r.add.p) ch.settled(nadd[i]);
#pragma unroll
            for (int j = 0; j < kC; j++) {
                h[j] = a[i][j] * h[j] + u[i][j];
                f[j] = s < places.len ? h[j] + (r.add.p ? nadd[i][j] : 0.0f) : 0.0f;
            }
            if (s < p1) ch.store(r.y, b, places.written(s), f);
        }
    }
    if (r.leave && seg == r.nseg - 1 && w == 0) ch.store_params(r.leave + (long long)b * r.d, carry);
}

// dh_s = dy_s + a_{s+1} dh_{s+1} is the same recurrence from the other end: what enters a wave's tokens is q = a dh of the token after
// them, and they leave Q + P q.  The states in front of a wave's tokens are folded from the kept one before them, so the walk reads x, g
// and dy once and writes dx and dg.  dbias is summed by lane over the segment, then over the waves and the slots in a fixed order.
template <typename IO, int kGate, int kC, int kT, int kW, int kV>
__global__ __launch_bounds__(64 * kW * kV) void recur_bwd_kernel(const RecurArgs r)
{
    static_assert((kW * kT) % kKeep == 0, "every step starts at a kept state");
    struct Links {
        float p[kC], e[kC], q[kC];
    };
    __shared__ Links part[2][kW][kV * 64];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), w = wave % kW, v = wave / kW;
    const int tiles = (r.d + 64 * kC * kV - 1) / (64 * kC * kV), tile = blockIdx.x % tiles, seg = blockIdx.x / tiles, b = blockIdx.y;
    const Channels<IO, kC> ch((tile * kV + v) * 64 * kC, lane, r.d);
    const Places places(r, b);
    const int p0 = seg * r.seg_len, p1 = min(p0 + r.seg_len, r.L), column = v * 64 + lane, kept = (r.L + kKeep - 1) / kKeep;
    float bias[kC], carry[kC], dbias[kC];
    ch.load_params(bias, r.bias);
    enter(carry, ch, r, b, r.nseg - 1 - seg);
#pragma unroll
    for (int j = 0; j < kC; j++) dbias[j] = 0.0f;
    Piece<IO, kC> nx[kT], ng[kT], nd[kT];
    const auto request = [&](int base) {
#pragma unroll
        for (int i = 0; i < kT; i++) {
            const int t = places.readable(base + w * kT + i);
            nx[i] = ch.load(r.x, b, t);
            ng[i] = ch.load(r.g, b, t);
            nd[i] = ch.load(r.dy, b, t);
        }
    };
    const int steps = (p1 - p0 + kW * kT - 1) / (kW * kT);
    request(p0 + (steps - 1) * kW * kT);
    int turn = 0;
    for (int base = p0 + (steps - 1) * kW * kT; base >= p0; base -= kW * kT, turn ^= 1) {
        const int s0 = base + w * kT;
        float a[kT][kC], q[kT][kC], x[kT][kC], dy[kT][kC], h[kC];
        const int first = min(s0 / kKeep, kept - 1);   // (waves beyond the end: any)
        ch.load_params(h, r.states + ((long long)b * kept + first) * r.d);
        Links mine;
#pragma unroll
        for (int j = 0; j < kC; j++) mine.p[j] = 1.0f, mine.e[j] = mine.q[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < kT; i++) {
            ch.settled(nx[i]);
            ch.settled(ng[i]);
            ch.settled(nd[i]);
            const bool inside = s0 + i < places.len;
#pragma unroll
            for (int j = 0; j < kC; j++) {
                gate_of<kGate>(ng[i][j], bias[j], a[i][j], q[i][j]);
                x[i][j] = nx[i][j], dy[i][j] = nd[i][j];
                if (!inside) a[i][j] = 1.0f, q[i][j] = x[i][j] = dy[i][j] = 0.0f;
                mine.e[j] = a[i][j] * mine.e[j] + (kGate == kSigmoid ? q[i][j] * x[i][j] : x[i][j]);
                mine.p[j] *= a[i][j];
            }
        }
#pragma unroll
        for (int i = kT - 1; i >= 0; i--)
#pragma unroll
            for (int j = 0; j < kC; j++) mine.q[j] = a[i][j] * (dy[i][j] + mine.q[j]);
        if (base > p0) request(base - kW * kT);
        float dh[kC];   // (q of the tokens behind)
#pragma unroll
        for (int j = 0; j < kC; j++) dh[j] = carry[j];
        if constexpr (kW > 1) {
            part[turn][w][column] = mine;
            __syncthreads();
            const int w0 = (first * kKeep - base) / kT;   // (the wave that starts at the kept state)
#pragma unroll
            for (int k = 0; k < kW; k++)
                if (k >= w0 && k < w) {
                    const Links link = part[turn][k][column];
#pragma unroll
                    for (int j = 0; j < kC; j++) h[j] = link.p[j] * h[j] + link.e[j];
                }
#pragma unroll
            for (int k = kW - 1; k >= 0; k--) {
                const Links link = part[turn][k][column];
#pragma unroll
                for (int j = 0; j < kC; j++) {
                    carry[j] = link.p[j] * carry[j] + link.q[j];
                    if (k - 1 == w) dh[j] = carry[j];
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < kC; j++) carry[j] = mine.p[j] * carry[j] + mine.q[j];
        }
        float before[kT][kC];
#pragma unroll
        for (int i = 0; i < kT; i++)
#pragma unroll
            for (int j = 0; j < kC; j++) {
                before[i][j] = h[j];
                h[j] = a[i][j] * h[j] + (kGate == kSigmoid ? q[i][j] * x[i][j] : x[i][j]);
            }
#pragma unroll
        for (int i = kT - 1; i >= 0; i--) {
            const int s = s0 + i;
            float dx[kC], dg[kC];
#pragma unroll
            for (int j = 0; j < kC; j++) {
                const float d = dy[i][j] + dh[j];
                dh[j] = a[i][j] * d;
                if (kGate == kSigmoid) {
                    dx[j] = d * q[i][j];
                    dg[j] = dx[j] * (before[i][j] - x[i][j]) * a[i][j];
                } else {
                    dx[j] = d;
                    dg[j] = d * before[i][j] * q[i][j];
                }
                if (s >= places.len) dx[j] = dg[j] = 0.0f;
                dbias[j] += dg[j];
            }
            if (s < p1) {
                const int t = places.written(s);
                ch.store(r.dx, b, t, dx);
                ch.store(r.dg, b, t, dg);
            }
        }
    }
    if (r.leave && seg == 0 && w == 0) ch.store_params(r.leave + (long long)b * r.d, carry);
    if (r.dbias) {
        float* const slot = r.dbias + ((long long)b * r.nseg + seg) * r.d;
        if constexpr (kW > 1) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kC; j++) part[0][w][column].p[j] = dbias[j];
            __syncthreads();
            if (w == 0)
#pragma unroll
                for (int k = 1; k < kW; k++)
#pragma unroll
                    for (int j = 0; j < kC; j++) dbias[j] += part[0][k][column].p[j];
        }
        if (w == 0) ch.store_params(slot, dbias);
    }
}

// The (P, E) of a segment, or with kBack its (P, Q): each wave takes a run of it, the runs are joined at the end.
template <typename IO, int kGate, int kC, int kT, int kW, bool kBack>
__global__ __launch_bounds__(64 * kW) void recur_ends_kernel(const RecurArgs r)
{
    __shared__ Link<kC> part[kW][64];
    const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int tiles = (r.d + 64 * kC - 1) / (64 * kC), tile = blockIdx.x % tiles, turn = blockIdx.x / tiles, b = blockIdx.y;
    const int seg = kBack ? r.nseg - 1 - turn : turn;   // (the last one walked leaves nothing that is wanted)
    const Channels<IO, kC> ch(tile * 64 * kC, lane, r.d);
    const Places places(r, b);
    const int run = r.seg_len / kW, p0 = seg * r.seg_len + w * run, p1 = min(p0 + run, r.L), steps = max(0, (p1 - p0 + kT - 1) / kT);
    float bias[kC];
    ch.load_params(bias, r.bias);
    Link<kC> mine;
#pragma unroll
    for (int j = 0; j < kC; j++) mine.p[j] = 1.0f, mine.e[j] = 0.0f;
    for (int k = 0; k < steps; k++) {
        const int s0 = p0 + (kBack ? steps - 1 - k : k) * kT;
        Piece<IO, kC> x[kT], g[kT];
#pragma unroll
        for (int i = 0; i < kT; i++) {
            const int t = places.readable(s0 + i);
            x[i] = ch.load(kBack ? r.dy : r.x, b, t);
            g[i] = ch.load(r.g, b, t);
        }
#pragma unroll
        for (int n = 0; n < kT; n++) {
            const int i = kBack ? kT - 1 - n : n;
            ch.settled(x[i]);
            ch.settled(g[i]);
            const bool inside = s0 + i < min(p1, places.len);
#pragma unroll
            for (int j = 0; j < kC; j++) {
                float a, q, u = x[i][j];
                gate_of<kGate>(g[i][j], bias[j], a, q);
                if (!inside) a = 1.0f, q = u = 0.0f;
                if constexpr (kBack) mine.e[j] = a * (u + mine.e[j]);
                else mine.e[j] = a * mine.e[j] + (kGate == kSigmoid ? q * u : u);
                mine.p[j] *= a;
            }
        }
    }
    part[w][lane] = mine;
    __syncthreads();
    if (w != 0) return;
    mine = part[kBack ? kW - 1 : 0][lane];
#pragma unroll
    for (int n = 1; n < kW; n++) {
        const Link<kC> link = part[kBack ? kW - 1 - n : n][lane];
#pragma unroll
        for (int j = 0; j < kC; j++) {
            mine.e[j] = link.p[j] * mine.e[j] + link.e[j];
            mine.p[j] *= link.p[j];
        }
    }
    float* const to = r.links + ((long long)b * r.nseg + turn + 1) * 2 * r.d;
    ch.store_params(to, mine.p);
    ch.store_params(to + r.d, mine.e);
    if (turn == 0) {
        ch.load_params(mine.e, r.enter ? r.enter + (long long)b * r.d : nullptr);
#pragma unroll
        for (int j = 0; j < kC; j++) mine.p[j] = 0.0f;
        ch.store_params(to - 2 * r.d, mine.p);
        ch.store_params(to - r.d, mine.e);
    }
}

namespace {

constexpr int kMaxWidth = 65536;

int check_recurrence(const bimamba_recurrence_desc* d)
{
    if (!d) return BIMAMBA_ERR_NULL_POINTER;
    if (d->struct_size != sizeof(bimamba_recurrence_desc) || d->d_inner < 1 || (d->reverse != 0 && d->reverse != 1)) return BIMAMBA_ERR_BAD_SHAPE;
    if (const int rc = check_rows(d->batch, d->seqlen)) return rc;
    if (!known_dtype(d->io_dtype) || (d->gate != BIMAMBA_GATE_LOG && d->gate != BIMAMBA_GATE_SIGMOID)) return BIMAMBA_ERR_UNSUPPORTED;
    if (d->batch > 65535 || d->d_inner > kMaxWidth) return BIMAMBA_ERR_UNSUPPORTED;
    return BIMAMBA_OK;
}

constexpr int kTokens = 16, kWaves = 4;   // of a wave in a step; of a workgroup

struct RecurPlan {
    int channels, nseg, seg_len;   // channels a lane
    unsigned tiles;
};
RecurPlan plan_recurrence(const bimamba_recurrence_desc* d)
{
    RecurPlan p{};
    p.channels = d->io_dtype == BIMAMBA_BF16 && d->d_inner > 1 ? 2 : 1;
    p.tiles = (d->d_inner + 64 * p.channels - 1) / (64 * p.channels);
    const int step = kTokens * kWaves;
    const long long have = (long long)p.tiles * d->batch, want = 4 * cu_count();
    const int steps = (d->seqlen + step - 1) / step;
    p.nseg = (int)(have >= want || steps < 8 ? 1 : (want + have - 1) / have);
    if (p.nseg > steps / 4) p.nseg = steps / 4 > 0 ? steps / 4 : 1;
    const int per = (steps + p.nseg - 1) / p.nseg;
    p.seg_len = per * step;
    p.nseg = (steps + per - 1) / per;
    return p;
}

size_t links_bytes(const bimamba_recurrence_desc* d, const RecurPlan& p)
{
    return p.nseg > 1 ? (size_t)d->batch * p.nseg * 2 * d->d_inner * sizeof(float) : 0;
}

template <typename IO, int kGate, int kC>
void launch_forward(const RecurPlan& p, const RecurArgs& a, int batch, hipStream_t st)
{
    const dim3 grid(p.tiles * p.nseg, batch), wg(64 * kWaves);
    if (p.nseg > 1) hipLaunchKernelGGL((recur_ends_kernel<IO, kGate, kC, kTokens, kWaves, false>), dim3(p.tiles * (p.nseg - 1), batch), wg, 0, st, a);
    hipLaunchKernelGGL((recur_kernel<IO, kGate, kC, kTokens, kWaves, 1>), grid, wg, 0, st, a);
}
template <typename IO, int kGate, int kC>
void launch_backward(const RecurPlan& p, const RecurArgs& a, int batch, hipStream_t st)
{
    const dim3 grid(p.tiles * p.nseg, batch), wg(64 * kWaves);
    if (p.nseg > 1) hipLaunchKernelGGL((recur_ends_kernel<IO, kGate, kC, kTokens, kWaves, true>), dim3(p.tiles * (p.nseg - 1), batch), wg, 0, st, a);
    hipLaunchKernelGGL((recur_bwd_kernel<IO, kGate, kC, kTokens, kWaves, 1>), grid, wg, 0, st, a);
}
template <typename IO, int kC>
void launch_gate(const bimamba_recurrence_desc* d, const RecurPlan& p, const RecurArgs& a, bool back, hipStream_t st)
{
    const bool sigmoid = d->gate == BIMAMBA_GATE_SIGMOID;
    if (back) sigmoid ? launch_backward<IO, kSigmoid, kC>(p, a, d->batch, st) : launch_backward<IO, kLog, kC>(p, a, d->batch, st);
    else sigmoid ? launch_forward<IO, kSigmoid, kC>(p, a, d->batch, st) : launch_forward<IO, kLog, kC>(p, a, d->batch, st);
}
void launch(const bimamba_recurrence_desc* d, const RecurPlan& p, const RecurArgs& a, bool back, hipStream_t st)
{
    if (d->io_dtype == BIMAMBA_F32) launch_gate<IoF32, 1>(d, p, a, back, st);
    else if (p.channels == 2) launch_gate<IoBF16, 2>(d, p, a, back, st);
    else launch_gate<IoBF16, 1>(d, p, a, back, st);
}

// An fp32 or int64 array, none if p is null.
int check_array(const void* p, long long count, size_t elem, Bytes* r)
{
    if (!aligned_to(p, elem)) return BIMAMBA_ERR_MISALIGNED;
    *r = bytes_of(p, count, elem);
    return BIMAMBA_OK;
}

}  // namespace
}  // namespace bm

using namespace bm;

extern "C" {

size_t bimamba_recurrence_workspace_bytes(const bimamba_recurrence_desc* d)
{
    if (check_recurrence(d) || d->batch == 0 || d->seqlen == 0) return 0;
    return links_bytes(d, plan_recurrence(d));
}

int bimamba_recurrence(const bimamba_recurrence_desc* d, const bimamba_tensor* x, const bimamba_tensor* g, const float* bias,
                       const bimamba_tensor* add, const int64_t* lengths, const float* h_in, const bimamba_tensor* y, float* h_out,
                       float* states, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    int rc = check_recurrence(d);
    if (rc) return rc;
    if (!x || !g || !y) return BIMAMBA_ERR_NULL_POINTER;
    if (bias && d->gate != BIMAMBA_GATE_SIGMOID) return BIMAMBA_ERR_UNSUPPORTED;
    if (d->batch == 0) return BIMAMBA_OK;
    const int Bt = d->batch, L = d->seqlen, D = d->d_inner, io = d->io_dtype;
    const size_t elem = dtype_bytes(io);
    const RecurPlan p = L ? plan_recurrence(d) : RecurPlan{};
    const size_t need = bimamba_recurrence_workspace_bytes(d);
    Bytes bx{}, bg{}, badd{}, by{}, bbias, blen, bin, bout, bkept;
    if (L) {
        if ((rc = check_view(x, Bt, L, D, io, false, &bx)) || (rc = check_view(g, Bt, L, D, io, false, &bg)) || (rc = check_view(y, Bt, L, D, io, true, &by)))
            return rc;
        if (add && (rc = check_view(add, Bt, L, D, io, false, &badd))) return rc;
    }
    if ((rc = check_array(bias, D, 4, &bbias)) || (rc = check_array(lengths, Bt, 8, &blen)) || (rc = check_array(h_in, (long long)Bt * D, 4, &bin)) ||
        (rc = check_array(h_out, (long long)Bt * D, 4, &bout)) || (rc = check_array(states, (long long)Bt * ((L + kKeep - 1) / kKeep) * D, 4, &bkept)))
        return rc;
    if ((rc = check_workspace(workspace, workspace_bytes, need))) return rc;
    const Bytes ws = bytes_of(need ? workspace : nullptr, need, 1);
    if (L) {
        if (views_meet(y, D, by, x, D, bx, Bt, elem, elem) || views_meet(y, D, by, g, D, bg, Bt, elem, elem)) return BIMAMBA_ERR_ALIAS;
        const bool same = add && add->ptr == y->ptr && add->stride_batch == y->stride_batch && add->stride_token == y->stride_token;
        if (add && !same && views_meet(y, D, by, add, D, badd, Bt, elem, elem)) return BIMAMBA_ERR_ALIAS;
    }
    const Bytes written[] = {by, bout, bkept, ws}, read[] = {bbias, blen, bin, bx, bg, badd};
    for (int i = 0; i < 4; i++) {
        for (int j = 0; j < (i == 0 ? 3 : 6); j++)
            if (meet(written[i], read[j]) && !(i == 1 && j == 2 && h_in == h_out)) return BIMAMBA_ERR_ALIAS;
        for (int j = 0; j < i; j++)
            if (meet(written[i], written[j])) return BIMAMBA_ERR_ALIAS;
    }
    RecurArgs a{};
    a.x = row_view(x), a.g = row_view(g), a.y = row_view(y);
    if (add) a.add = row_view(add);
    a.bias = bias, a.lengths = lengths, a.enter = h_in, a.leave = h_out, a.states = states, a.links = static_cast<float*>(workspace);
    a.L = L, a.d = D, a.nseg = p.nseg, a.seg_len = p.seg_len, a.reverse = d->reverse;
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    if (L) {
        launch(d, p, a, false, st);
    } else if (h_out && h_out != h_in) {
        // (no token: the state goes through; a sum of one slot, or of none)
        launch_slot_sum(SlotSumArgs{{h_in, nullptr}, {h_out, nullptr}, h_in ? 1 : 0, D, D}, Bt, st);
    }
    return launches.status();
}

size_t bimamba_recurrence_bwd_workspace_bytes(const bimamba_recurrence_desc* d)
{
    if (check_recurrence(d) || d->batch == 0 || d->seqlen == 0) return 0;
    const RecurPlan p = plan_recurrence(d);
    const long long slots = (long long)d->batch * p.nseg;
    const size_t sums = d->gate == BIMAMBA_GATE_SIGMOID && slots > 1 ? (size_t)slots * d->d_inner * sizeof(float) : 0;
    return links_bytes(d, p) + sums;
}

int bimamba_recurrence_bwd(const bimamba_recurrence_desc* d, const bimamba_tensor* x, const bimamba_tensor* g, const float* bias,
                           const int64_t* lengths, const float* states, const bimamba_tensor* dy, const float* dh_out,
                           const bimamba_tensor* dx, const bimamba_tensor* dg, float* dbias, float* dh_in,
                           void* workspace, size_t workspace_bytes, void* hip_stream)
{
    int rc = check_recurrence(d);
    if (rc) return rc;
    if (!x || !g || !dy || !dx || !dg) return BIMAMBA_ERR_NULL_POINTER;
    if ((bias || dbias) && d->gate != BIMAMBA_GATE_SIGMOID) return BIMAMBA_ERR_UNSUPPORTED;
    const int Bt = d->batch, L = d->seqlen, D = d->d_inner, io = d->io_dtype;
    const bool rows = Bt && L;
    const size_t elem = dtype_bytes(io);
    const RecurPlan p = rows ? plan_recurrence(d) : RecurPlan{};
    const size_t need = bimamba_recurrence_bwd_workspace_bytes(d);
    Bytes bx{}, bg{}, by{}, bdx{}, bdg{}, bbias, blen, bkept, bout, bdb, bin;
    if (rows) {
        if (!states) return BIMAMBA_ERR_NULL_POINTER;
        if ((rc = check_view(x, Bt, L, D, io, false, &bx)) || (rc = check_view(g, Bt, L, D, io, false, &bg)) ||
            (rc = check_view(dy, Bt, L, D, io, false, &by)) || (rc = check_view(dx, Bt, L, D, io, true, &bdx)) ||
            (rc = check_view(dg, Bt, L, D, io, true, &bdg)))
            return rc;
    }
    if ((rc = check_array(bias, D, 4, &bbias)) || (rc = check_array(lengths, Bt, 8, &blen)) ||
        (rc = check_array(states, (long long)Bt * ((L + kKeep - 1) / kKeep) * D, 4, &bkept)) || (rc = check_array(dh_out, (long long)Bt * D, 4, &bout)) ||
        (rc = check_array(dbias, D, 4, &bdb)) || (rc = check_array(dh_in, (long long)Bt * D, 4, &bin)))
        return rc;
    if ((rc = check_workspace(workspace, workspace_bytes, need))) return rc;
    const Bytes ws = bytes_of(need ? workspace : nullptr, need, 1);
    if (rows) {
        const bimamba_tensor *const in[] = {x, g, dy}, *const out[] = {dx, dg};
        const Bytes bin3[] = {bx, bg, by}, bout2[] = {bdx, bdg};
        for (int i = 0; i < 2; i++)
            for (int j = 0; j < 3; j++)
                if (views_meet(out[i], D, bout2[i], in[j], D, bin3[j], Bt, elem, elem)) return BIMAMBA_ERR_ALIAS;
        if (views_meet(dx, D, bdx, dg, D, bdg, Bt, elem, elem)) return BIMAMBA_ERR_ALIAS;
    }
    const Bytes written[] = {bdx, bdg, bdb, bin, ws}, read[] = {bbias, blen, bkept, bout, bx, bg, by};
    for (int i = 0; i < 5; i++) {
        for (int j = 0; j < (i < 2 ? 4 : 7); j++)
            if (meet(written[i], read[j]) && !(i == 3 && j == 3 && dh_in == dh_out)) return BIMAMBA_ERR_ALIAS;
        for (int j = 0; j < i; j++)
            if (meet(written[i], written[j]) && !(i == 1 && j == 0)) return BIMAMBA_ERR_ALIAS;
    }
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    const long long slots = rows ? (long long)Bt * p.nseg : 0;
    if (rows) {
        RecurArgs a{};
        a.x = row_view(x), a.g = row_view(g), a.dy = row_view(dy), a.dx = row_view(dx), a.dg = row_view(dg);
        a.bias = bias, a.lengths = lengths, a.enter = dh_out, a.leave = dh_in, a.states = const_cast<float*>(states);
        a.links = static_cast<float*>(workspace);
        float* const sums = static_cast<float*>(workspace) + links_bytes(d, p) / sizeof(float);
        a.dbias = dbias ? slots > 1 ? sums : dbias : nullptr;
        a.L = L, a.d = D, a.nseg = p.nseg, a.seg_len = p.seg_len, a.reverse = d->reverse;
        launch(d, p, a, true, st);
        if (dbias && slots > 1) launch_slot_sum(SlotSumArgs{{sums, nullptr}, {dbias, nullptr}, slots, D, D}, 1, st);
    } else {
        if (Bt && dh_in && dh_in != dh_out) launch_slot_sum(SlotSumArgs{{dh_out, nullptr}, {dh_in, nullptr}, dh_out ? 1 : 0, D, D}, Bt, st);
        if (dbias) launch_slot_sum(SlotSumArgs{{nullptr, nullptr}, {dbias, nullptr}, 0, D, D}, 1, st);
    }
    return launches.status();
}

}  // extern "C"
