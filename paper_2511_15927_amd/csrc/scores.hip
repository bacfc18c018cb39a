// Log probabilities of given tokens, entropies and the most probable tokens of rows of logits, and their gradient.
#include "model_ops.h"

#include <cfloat>
#include <cstddef>

namespace bm {

constexpr int kMaxTop = 8, kMaxSplits = 64;
constexpr float kFarBelow = -1e4f;   // a difference of logits whose exponential is 0: stands for all that lie lower, -inf among them

// One pass over a row.  A lane keeps of the logits x it has seen the largest (m), S = sum exp(x - m) and, for the entropy,
// T = sum exp(x - m) (x - m); then lse = m + log S and H = log S - T / S, no value of which is large where the row is confident.  To a
// larger maximum m' both move by r = exp(m - m'): S' = r S, T' = r (T + S (m - m')).  m starts at the lowest finite value, so a row of
// nothing but -inf keeps S = 0, and a NaN or +inf makes S a NaN.  What bounds it is the read: 8192 rows of 50304 bf16 127 us (6.5 TB/s);
// 12 vector slots a logit, of which the exponential is four, would allow twice that.  32 rows with the entropy and eight alternatives:
// 9.7 us, of which the alternatives are 3, the rest two rounds of loads and the joining of a workgroup's sums.
struct Stats {
    float m, s, t;
};
template <bool kEntropy>
__device__ __forceinline__ void move_to(Stats& a, float m)
{
    const float d = a.m - m, r = fast_exp2(d * kLog2e);
    if constexpr (kEntropy) a.t = r * (a.t + a.s * fmaxf(d, kFarBelow));
    a.s *= r;
    a.m = m;
}

// The order of the alternatives as whole numbers: a larger logit first, of equal ones (-0 and 0 among them) the lower id.  0: none.
typedef unsigned long long Key;
__device__ __forceinline__ Key key_of(float v, unsigned id)
{
    const unsigned u = __float_as_uint(v + 0.0f), ordered = u & 0x80000000u ? ~u : u | 0x80000000u;
    return (Key)ordered << 32 | ~id;
}
__device__ __forceinline__ float value_of(Key k)
{
    const unsigned o = (unsigned)(k >> 32);
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ unsigned id_of(Key k) { return ~(unsigned)k; }
// The largest key of a row of sixteen lanes or of all 64, in all of them: the largest upper half, and the largest lower half beside that.
template <int kLanes>
__device__ __forceinline__ unsigned lanes_max(unsigned v)
{
#define BM_DPP(ctrl) (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, true)
    v = max(v, BM_DPP(0xB1));    // quad_perm 1 0 3 2
    v = max(v, BM_DPP(0x4E));    // quad_perm 2 3 0 1
    v = max(v, BM_DPP(0x141));   // row_half_mirror
    v = max(v, BM_DPP(0x140));   // row_mirror
#undef BM_DPP
    if constexpr (kLanes == 64) {
        auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = max(r[0], r[1]);
        r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = max(r[0], r[1]);
    }
    return v;
}
template <int kLanes>
__device__ __forceinline__ Key lanes_max_key(Key k)
{
    const unsigned hi = lanes_max<kLanes>((unsigned)(k >> 32)), lo = lanes_max<kLanes>((unsigned)(k >> 32) == hi ? (unsigned)k : 0u);
    return (Key)hi << 32 | lo;
}

struct ScoresArgs {
    RowView logits;
    const int64_t* ids;   // or null
    long long ids_sb, ids_st;
    float *logp, *lse, *lse_rest, *entropy, *top_logp;
    int64_t* top_token;
    Stats* part;          // [rows][splits], and the parts' own alternatives [rows][splits][top_k], where a row is split
    Key* part_top;
    unsigned rows, L;
    int vocab, top_k, splits, per_split, targets_only;
};

__device__ __forceinline__ long long target_of(const ScoresArgs& a, unsigned b, unsigned t)
{
    if (!a.ids) return -1;
    const long long id = a.ids[b * a.ids_sb + t * a.ids_st];
    return id >= 0 && id < a.vocab ? id : -1;
}
// A row that is not asked for.
__device__ __forceinline__ void store_nothing(const ScoresArgs& a, unsigned row)
{
    if (a.logp) a.logp[row] = 0.0f;
    if (a.lse) a.lse[row] = 0.0f;
    if (a.lse_rest) a.lse_rest[row] = 0.0f;
    if (a.entropy) a.entropy[row] = 0.0f;
    for (int k = 0; k < a.top_k; k++) {
        if (a.top_logp) a.top_logp[(long long)row * a.top_k + k] = 0.0f;
        if (a.top_token) a.top_token[(long long)row * a.top_k + k] = -1;
    }
}
__device__ __forceinline__ void store_stats(const ScoresArgs& a, unsigned row, const Stats& s, long long target, float x)
{
    const float log_s = logf(s.s);   // (-inf for a row of nothing but -inf)
    if (a.logp) a.logp[row] = target < 0 ? 0.0f : s.s == 0.0f ? -INFINITY : (x - s.m) - log_s;
    const float lse = s.m + log_s;
    if (a.lse) a.lse[row] = lse;
    if (a.lse_rest) {   // (what the addition rounded away, exactly; all of log S beside a maximum that is large enough)
        const float added = lse - s.m;
        a.lse_rest[row] = isfinite(lse) ? (s.m - (lse - added)) + (log_s - added) : 0.0f;
    }
    if (a.entropy) a.entropy[row] = s.s == 0.0f ? 0.0f : log_s - s.t / s.s;
}
__device__ __forceinline__ void store_top(const ScoresArgs& a, unsigned row, int k, const Stats& s, Key key)
{
    const bool none = !(s.s == s.s);
    if (a.top_logp)
        a.top_logp[(long long)row * a.top_k + k] = none ? s.s : s.s == 0.0f ? -INFINITY : (value_of(key) - s.m) - logf(s.s);
    if (a.top_token) a.top_token[(long long)row * a.top_k + k] = none ? -1 : (int64_t)id_of(key);
}

// A workgroup takes a row, or one of its `splits` parts.  With kTop a lane also keeps which of its pieces first had the largest logit.
// Of sixteen groups of lanes each has a best piece; the k-th best of these sixteen bounds what the k best logits of the row can be, and
// holds back all but a few: only lanes whose own best piece reaches it have any, a dozen as a rule.  Their pieces are read again (from the
// caches), spread over all lanes, and the logits that reach the bound go on a list, where each counts how many are better.  A row
// that has more of them than the list holds (equal ones, or many large ones that one lane read) looks for the best logit below the one
// before, k times.
constexpr int kScoresAhead = 4, kMaxListed = 256;
constexpr int kManyRowsThreads = 256, kFewRowsThreads = 1024;
template <typename IO, bool kEntropy, bool kTop, int kPiece, int kScoresThreads, bool kPast>
__device__ __forceinline__ void scores_row(const ScoresArgs& a)
{
    constexpr int kScoresWaves = kScoresThreads / 64, kGroups = 16, kGroupLanes = kScoresThreads / kGroups;   // (kMaxTop groups or more)
    const unsigned row = blockIdx.x / a.splits, split = blockIdx.x - row * a.splits;
    const unsigned b = row / a.L, t = row - b * a.L;
    const long long target = target_of(a, b, t);
    if (a.targets_only && target < 0) {
        if (split == 0 && threadIdx.x == 0) store_nothing(a, row);
        return;
    }
    typedef typename IO::T T;
    const int from = split * a.per_split, n = min(a.per_split, a.vocab - from), pieces = (n + kPiece - 1) / kPiece;
    const T* const x = static_cast<const T*>(a.logits.p) + row_offset(a.logits, b, t) + from;
    const T lowest = io_value<IO>(-INFINITY);
    Stats s{-FLT_MAX, 0.0f, 0.0f};
    float best = -INFINITY;
    unsigned best_piece = ~0u;
    for (int first = threadIdx.x; first < pieces; first += kScoresThreads * kScoresAhead) {
        Piece<IO, kPiece> p[kScoresAhead];
#pragma unroll
        for (int j = 0; j < kScoresAhead; j++) p[j] = load_clamped<IO, kPiece, kPast>(x, (first + j * kScoresThreads) * kPiece, n);
#pragma unroll
        for (int j = 0; j < kScoresAhead; j++) {
            const int piece = first + j * kScoresThreads;
            if (piece < pieces) {
                settle(p[j], piece * kPiece, n, lowest);
                float m = p[j][0];
#pragma unroll
                for (int i = 1; i < kPiece; i++) m = fmaxf(m, p[j][i]);
                if constexpr (kTop) {
                    if (m > best || best_piece == ~0u) {
                        best = m;
                        best_piece = piece;
                    }
                }
                move_to<kEntropy>(s, fmaxf(s.m, m));
#pragma unroll
                for (int i = 0; i < kPiece; i++) {
                    const float d = p[j][i] - s.m, e = fast_exp2(d * kLog2e);
                    s.s += e;
                    if constexpr (kEntropy) s.t += e * fmaxf(d, kFarBelow);
                }
            }
        }
    }
    // over the workgroup
    __shared__ Stats part[kScoresWaves];
    __shared__ Key group_key[kGroups], best_key[kScoresWaves], listed[kMaxListed];
    __shared__ int chosen[kScoresThreads], n_chosen, n_listed;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    move_to<kEntropy>(s, wave_max(s.m));
    s.s = wave_sum(s.s);
    if constexpr (kEntropy) s.t = wave_sum(s.t);
    if (lane == 0) part[wave] = s;
    Key mine = 0;
    if constexpr (kTop) {
        mine = best_piece == ~0u ? 0 : key_of(best, best_piece * kPiece);
        const Key top = lanes_max_key<kGroupLanes>(mine);
        if (threadIdx.x % kGroupLanes == 0) group_key[threadIdx.x / kGroupLanes] = top;
        if (threadIdx.x == 0) n_chosen = n_listed = 0;
    }
    __syncthreads();
    s.m = part[0].m;
#pragma unroll
    for (int w = 1; w < kScoresWaves; w++) s.m = fmaxf(s.m, part[w].m);
    s.s = s.t = 0.0f;
#pragma unroll
    for (int w = 0; w < kScoresWaves; w++) {
        Stats q = part[w];
        move_to<kEntropy>(q, s.m);
        s.s += q.s;
        if constexpr (kEntropy) s.t += q.t;
    }
    const bool whole = a.splits == 1;
    if (threadIdx.x == 0) {
        if (whole) store_stats(a, row, s, target, target < 0 ? 0.0f : IO::cvt(x[target]));
        else a.part[blockIdx.x] = s;
    }
    if constexpr (kTop) {
        const auto store = [&](int k, Key key) {
            if (whole) store_top(a, row, k, s, key);
            else a.part_top[(long long)blockIdx.x * a.top_k + k] = key;
        };
        // the k-th best of the groups' best pieces (or none, of fewer pieces)
        Key threshold = 0;
        {
            const Key own = group_key[lane % kGroups];
            int better = 0;
#pragma unroll
            for (int g = 0; g < kGroups; g++) better += group_key[g] > own;
            const unsigned long long at = __ballot(better == a.top_k - 1);
            if (at) threshold = __shfl(own, __builtin_ctzll(at));
        }
        if (mine != 0 && mine >= threshold) chosen[atomicAdd(&n_chosen, 1)] = threadIdx.x;
        __syncthreads();
        const int rounds = (pieces + kScoresThreads - 1) / kScoresThreads, items = n_chosen * rounds;
        // (the logits of the threshold's piece come first among its equals; any of the piece may be the one)
        const Key bound = threshold == 0 ? 1 : threshold - (kPiece - 1);
        const auto for_items = [&](auto use) {
            for (int item = threadIdx.x; item < items; item += kScoresThreads) {
                const int which = item / rounds, piece = (item - which * rounds) * kScoresThreads + chosen[which];
                if (piece < pieces) {
                    const Piece<IO, kPiece> p = load_piece_of<IO, kPiece>(x, piece * kPiece, n, lowest);
#pragma unroll
                    for (int i = 0; i < kPiece; i++) use(piece * kPiece + i < n ? key_of(p[i], piece * kPiece + i) : 0);
                }
            }
        };
        for_items([&](Key key) {
            if (key >= bound) {
                const int at = atomicAdd(&n_listed, 1);
                if (at < kMaxListed) listed[at] = key;
            }
        });
        __syncthreads();
        const int count = n_listed;
        if (count <= kMaxListed) {
            for (int c = threadIdx.x; c < max(count, a.top_k); c += kScoresThreads) {
                const Key key = c < count ? listed[c] : 0;
                int better = c < count ? 0 : c;   // (fewer logits than alternatives, in a part of a row: none)
                if (c < count) {
#pragma unroll 4
                    for (int j = 0; j < count; j++) better += listed[j] > key;
                }
                if (better < a.top_k) store(better, key == 0 ? 0 : key - from);   // (ids count down: those of the row)
            }
        } else {
            Key below = ~0ull;
            for (int k = 0; k < a.top_k; k++) {
                Key top = 0;
                for_items([&](Key key) {
                    if (key < below && key > top) top = key;
                });
                top = lanes_max_key<64>(top);
                __syncthreads();
                if (lane == 0) best_key[wave] = top;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < kScoresWaves; w++) top = best_key[w] > top ? best_key[w] : top;
                below = top;
                if (threadIdx.x == 0) store(k, top == 0 ? 0 : top - from);
            }
        }
    }
}
template <typename IO, bool kEntropy, bool kTop, int kThreads, bool kPast>
__global__ __launch_bounds__(kThreads) void scores_kernel(const ScoresArgs a)
{
    if constexpr (kThreads == kManyRowsThreads && !kPast) {   // (rows shorter than a piece, a logit a lane: 2^24 of them are less than the caches hold)
        if (a.vocab < kPieceOf<IO>) return scores_row<IO, kEntropy, kTop, 1, kThreads, kPast>(a);
    }
    scores_row<IO, kEntropy, kTop, kPieceOf<IO>, kThreads, kPast>(a);
}

// A wave joins the parts of a row, a part a lane; the lanes' alternatives are in descending order already.
template <typename IO, bool kEntropy, bool kTop>
__global__ __launch_bounds__(64) void scores_join_kernel(const ScoresArgs a)
{
    const unsigned row = blockIdx.x, b = row / a.L, t = row - b * a.L;
    const long long target = target_of(a, b, t);
    if (a.targets_only && target < 0) return;
    const int lane = threadIdx.x;
    Stats s{-FLT_MAX, 0.0f, 0.0f};
    Key top[kMaxTop] = {};
    if (lane < a.splits) {
        const long long at = (long long)row * a.splits + lane;
        s = a.part[at];
        if constexpr (kTop) {
#pragma unroll
            for (int k = 0; k < kMaxTop; k++)
                if (k < a.top_k) top[k] = a.part_top[at * a.top_k + k];
        }
    }
    move_to<kEntropy>(s, wave_max(s.m));
    s.s = wave_sum(s.s);
    if constexpr (kEntropy) s.t = wave_sum(s.t);
    if (lane == 0) {
        float x = 0.0f;
        if (target >= 0) x = IO::cvt((static_cast<const typename IO::T*>(a.logits.p) + row_offset(a.logits, b, t))[target]);
        store_stats(a, row, s, target, x);
    }
    if constexpr (kTop) {
        for (int k = 0; k < a.top_k; k++) {
            const Key best = lanes_max_key<64>(top[0]);
            if (top[0] == best)
#pragma unroll
                for (int i = 0; i < kMaxTop; i++) top[i] = i + 1 < kMaxTop ? top[i + 1] : 0;
            if (lane == 0) store_top(a, row, k, s, best);
        }
    }
}

// ---- gradient ----
//
// Elementwise, given lse and the entropy: log p = x - lse, dx = dlogp (1[target] - p) - dentropy p (log p + H).  lse comes in two parts, the
// fp32 value and what rounding left of it: 2^-24 |lse|, by which every p of the row would be off, relatively (by e^0.001 at logits near
// 30000; a row of equal logits from 2^28 on, the type's lowest value among them, would have p = 1 throughout).  A logit is read and its
// gradient written by the same lane, so the gradient may take the logits' place.  16384 rows of 50304 bf16, half of them without a target
// and so only written: 402 to 425 us (2.47 GB, 6.1 to 5.8 TB/s), bound by the bytes.
constexpr int kGradThreads = 256, kGradPart = kGradThreads * 32;
struct ScoresBwdArgs {
    RowView logits, dlogits;
    const int64_t* ids;
    long long ids_sb, ids_st;
    const float *lse, *lse_rest, *entropy, *dlogp, *dentropy;   // lse_rest: or null
    unsigned L, parts, all;   // parts of a row, and of all rows
    int vocab, targets_only;
};
template <typename IO, bool kEntropy, bool kPast, int kPiece>
__device__ __forceinline__ void scores_bwd_part(const ScoresBwdArgs& a, unsigned row, unsigned part)
{
    typedef typename IO::T T;
    constexpr int kPieces = kGradPart / (kGradThreads * kPieceOf<IO>);
    const unsigned b = row / a.L, t = row - b * a.L;
    int target = -1;
    if (a.ids) {
        const long long id = a.ids[b * a.ids_sb + t * a.ids_st];
        if (id >= 0 && id < a.vocab) target = (int)id;
    }
    const float dl = target >= 0 && a.dlogp ? a.dlogp[row] : 0.0f;
    const float de = kEntropy && (target >= 0 || !a.targets_only) ? a.dentropy[row] : 0.0f;   // (a row that was not asked for: its scores are constants)
    const float lse = a.lse[row], rest = a.lse_rest ? a.lse_rest[row] : 0.0f, h = kEntropy ? a.entropy[row] : 0.0f;
    const T* const x = static_cast<const T*>(a.logits.p) + row_offset(a.logits, b, t);
    T* const dx = static_cast<T*>(a.dlogits.p) + row_offset(a.dlogits, b, t);
    const int first = part * kGradPart + threadIdx.x * kPiece;
    const auto at = [&](int k) { return first + k * kGradThreads * kPiece; };
    if ((dl == 0.0f && de == 0.0f) || lse == -INFINITY) {
        const float zero[kPiece] = {};
#pragma unroll
        for (int k = 0; k < kPieces; k++)
            if (at(k) < a.vocab) store_piece_of<IO, kPast>(dx, at(k), a.vocab, zero);
        return;
    }
    Piece<IO, kPiece> p[kPieces];
#pragma unroll
    for (int k = 0; k < kPieces; k++) p[k] = load_clamped<IO, kPiece>(x, at(k), a.vocab);
    // (in place a lane's later pieces, clamped to the row's end, may have been overwritten by then: those are not stored)
#pragma unroll
    for (int k = 0; k < kPieces; k++) {
        if (at(k) >= a.vocab) continue;
        settle(p[k], at(k), a.vocab, T(0));
        float f[kPiece];
#pragma unroll
        for (int i = 0; i < kPiece; i++) {
            const float d = (p[k][i] - lse) - rest, e = fast_exp2(d * kLog2e);
            if constexpr (kEntropy) f[i] = -e * (dl + de * (fmaxf(d, kFarBelow) + h));
            else f[i] = -e * dl;
        }
        if ((unsigned)(target - at(k)) < (unsigned)kPiece)   // (no target: far outside)
#pragma unroll
            for (int i = 0; i < kPiece; i++) f[i] += at(k) + i == target ? dl : 0.0f;
        store_piece_of<IO, kPast>(dx, at(k), a.vocab, f);
    }
}
template <typename IO, bool kEntropy, bool kPast>
__global__ __launch_bounds__(kGradThreads) void scores_bwd_kernel(const ScoresBwdArgs a)
{
    for (unsigned w = blockIdx.x; w < a.all; w += gridDim.x) {
        const unsigned row = w / a.parts, part = w - row * a.parts;
        if (a.vocab >= kPieceOf<IO>) scores_bwd_part<IO, kEntropy, kPast, kPieceOf<IO>>(a, row, part);
        else scores_bwd_part<IO, kEntropy, kPast, 1>(a, row, part);
    }
}

namespace {

constexpr size_t kFirstLogitsDesc = offsetof(bimamba_logits_desc, reserved);   // (a descriptor without what lse_rest brought)
float* lse_rest_of(const bimamba_logits_desc* d) { return d->struct_size == kFirstLogitsDesc ? nullptr : d->lse_rest; }
int check_logits(const bimamba_logits_desc* d)
{
    if (!d) return BIMAMBA_ERR_NULL_POINTER;
    if (d->struct_size != kFirstLogitsDesc && d->struct_size != sizeof(bimamba_logits_desc)) return BIMAMBA_ERR_BAD_SHAPE;
    if (d->struct_size == sizeof(bimamba_logits_desc) && d->reserved != 0) return BIMAMBA_ERR_BAD_SHAPE;
    if (d->vocab < 1 || (d->targets_only | 1) != 1) return BIMAMBA_ERR_BAD_SHAPE;
    if (d->top_k < 0 || d->top_k > d->vocab) return BIMAMBA_ERR_BAD_SHAPE;
    if (const int rc = check_rows(d->batch, d->seqlen)) return rc;
    if (!known_dtype(d->io_dtype) || d->top_k > kMaxTop || d->vocab > 1 << 30) return BIMAMBA_ERR_UNSUPPORTED;
    return BIMAMBA_OK;
}

// Up to a row a CU, of up to 65536 logits: a workgroup of sixteen waves each, in one launch (32 x 50304 bf16 with entropy and eight
// alternatives 10.1 us; of four waves each, in 25 parts, 7.2 and 4.4 for the second launch; 256 x 50304 11.2 against 11.9 and 4.0).  Longer rows go
// in parts until four workgroups a CU exist, none of them under 2048 logits (4 x 130001: 5.8 and 3.9 against 11.9 and 4.0 in two
// parts of sixteen waves; 300 rows 24 and 4.5).  More rows: a workgroup of four waves each (600 x 50304 20.6 us; in two parts 18.4 and 4.8;
// 900 rows with sixteen waves 37.6 against 25.5).
struct ScoresPlan {
    unsigned rows;
    int threads, splits, per_split;
    size_t stats, total;   // bytes of the parts' statistics, and of the workspace
};
ScoresPlan plan_scores(const bimamba_logits_desc* d)
{
    ScoresPlan p{};
    p.rows = (unsigned)((long long)d->batch * d->seqlen);
    p.splits = 1;
    p.threads = p.rows <= (unsigned)cu_count() && d->vocab > 4096 && d->vocab <= 65536 ? kFewRowsThreads : kManyRowsThreads;
    if (d->vocab > 65536 && p.rows > 0) {
        const long long want = 4ll * cu_count() / p.rows, most = (d->vocab + 2047) / 2048;
        p.splits = (int)(want < most ? want : most);
    }
    if (p.splits > kMaxSplits) p.splits = kMaxSplits;
    if (p.splits < 1) p.splits = 1;
    p.per_split = ((d->vocab + p.splits - 1) / p.splits + 7) / 8 * 8;   // (whole pieces of either type)
    for (;; p.per_split += 8) {   // (no last part shorter than a piece)
        p.splits = (d->vocab + p.per_split - 1) / p.per_split;
        if (p.splits == 1 || d->vocab - (p.splits - 1) * p.per_split >= 8) break;
    }
    if (p.splits > 1) {
        p.stats = ((size_t)p.rows * p.splits * sizeof(Stats) + 15) / 16 * 16;
        p.total = p.stats + (size_t)p.rows * p.splits * d->top_k * sizeof(Key);
    }
    return p;
}

template <typename IO, bool kEntropy, bool kTop>
void launch_scores(const ScoresArgs& a, int threads, hipStream_t st)
{
    const dim3 grid(a.rows * (unsigned)a.splits), wg(threads);
    // (up to a row a CU of 65536 logits is less than the caches hold)
    if (threads == kFewRowsThreads) hipLaunchKernelGGL((scores_kernel<IO, kEntropy, kTop, kFewRowsThreads, false>), grid, wg, 0, st, a);
    else if (past_caches((double)a.rows * a.vocab * sizeof(typename IO::T)))
        hipLaunchKernelGGL((scores_kernel<IO, kEntropy, kTop, kManyRowsThreads, true>), grid, wg, 0, st, a);
    else hipLaunchKernelGGL((scores_kernel<IO, kEntropy, kTop, kManyRowsThreads, false>), grid, wg, 0, st, a);
    if (a.splits > 1) hipLaunchKernelGGL((scores_join_kernel<IO, kEntropy, kTop>), dim3(a.rows), dim3(64), 0, st, a);
}
template <typename IO>
void launch_scores(const ScoresArgs& a, int threads, hipStream_t st)
{
    const bool top = a.top_k > 0;
    if (a.entropy && top) launch_scores<IO, true, true>(a, threads, st);
    else if (a.entropy) launch_scores<IO, true, false>(a, threads, st);
    else if (top) launch_scores<IO, false, true>(a, threads, st);
    else launch_scores<IO, false, false>(a, threads, st);
}

template <typename IO>
void launch_scores_bwd(const ScoresBwdArgs& a, unsigned grid, bool past, hipStream_t st)
{
    const dim3 wg(kGradThreads);
    if (a.dentropy && past) hipLaunchKernelGGL((scores_bwd_kernel<IO, true, true>), dim3(grid), wg, 0, st, a);
    else if (a.dentropy) hipLaunchKernelGGL((scores_bwd_kernel<IO, true, false>), dim3(grid), wg, 0, st, a);
    else if (past) hipLaunchKernelGGL((scores_bwd_kernel<IO, false, true>), dim3(grid), wg, 0, st, a);
    else hipLaunchKernelGGL((scores_bwd_kernel<IO, false, false>), dim3(grid), wg, 0, st, a);
}

}  // namespace
}  // namespace bm

using namespace bm;

extern "C" {

size_t bimamba_log_probs_workspace_bytes(const bimamba_logits_desc* d) { return check_logits(d) ? 0 : plan_scores(d).total; }

int bimamba_log_probs(const bimamba_logits_desc* d, const bimamba_tensor* logits, const bimamba_tokens* targets,
                      const bimamba_scores* out, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    int rc = check_logits(d);
    if (rc) return rc;
    if (!logits || !out) return BIMAMBA_ERR_NULL_POINTER;
    if (!targets && (out->logp || d->targets_only)) return BIMAMBA_ERR_NULL_POINTER;
    if ((d->top_k == 0) != (!out->top_logp && !out->top_token)) return BIMAMBA_ERR_BAD_SHAPE;
    float* const lse_rest = lse_rest_of(d);
    if (!aligned_to(out->logp, 4) || !aligned_to(out->lse, 4) || !aligned_to(lse_rest, 4) || !aligned_to(out->entropy, 4) ||
        !aligned_to(out->top_logp, 4) || !aligned_to(out->top_token, 8))
        return BIMAMBA_ERR_MISALIGNED;
    if (d->batch == 0 || d->seqlen == 0) return BIMAMBA_OK;
    if (!out->logp && !out->lse && !out->entropy && d->top_k == 0) return BIMAMBA_ERR_NULL_POINTER;
    const ScoresPlan p = plan_scores(d);
    if ((unsigned long long)p.rows * p.splits >= 1u << 24) return BIMAMBA_ERR_UNSUPPORTED;   // (a grid holds 2^32 threads)
    Bytes from, ids{0, 0};
    if ((rc = check_view(logits, d->batch, d->seqlen, d->vocab, d->io_dtype, false, &from))) return rc;
    if (targets && (rc = check_tokens(targets, d->batch, d->seqlen, &ids))) return rc;
    if ((rc = check_workspace(workspace, workspace_bytes, p.total))) return rc;
    const Bytes written[] = {bytes_of(out->logp, p.rows, 4), bytes_of(out->lse, p.rows, 4), bytes_of(out->entropy, p.rows, 4),
                             bytes_of(out->top_logp, (long long)p.rows * d->top_k, 4), bytes_of(out->top_token, (long long)p.rows * d->top_k, 8),
                             bytes_of(p.total ? workspace : nullptr, p.total, 1), bytes_of(lse_rest, p.rows, 4)};
    for (int i = 0; i < 7; i++) {
        if (meet(written[i], from) || meet(written[i], ids)) return BIMAMBA_ERR_ALIAS;
        for (int j = 0; j < i; j++)
            if (meet(written[i], written[j])) return BIMAMBA_ERR_ALIAS;
    }
    ScoresArgs a{};
    a.logits = row_view(logits);
    if (targets) a.ids = targets->ptr, a.ids_sb = targets->stride_batch, a.ids_st = targets->stride_token;
    a.logp = out->logp, a.lse = out->lse, a.lse_rest = lse_rest, a.entropy = out->entropy, a.top_logp = out->top_logp, a.top_token = out->top_token;
    a.part = static_cast<Stats*>(workspace);
    a.part_top = reinterpret_cast<Key*>(static_cast<char*>(workspace) + p.stats);
    a.rows = p.rows, a.L = d->seqlen, a.vocab = d->vocab, a.top_k = d->top_k;
    a.splits = p.splits, a.per_split = p.per_split, a.targets_only = d->targets_only;
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    if (d->io_dtype == BIMAMBA_BF16) launch_scores<IoBF16>(a, p.threads, st);
    else launch_scores<IoF32>(a, p.threads, st);
    return launches.status();
}

int bimamba_log_probs_bwd(const bimamba_logits_desc* d, const bimamba_tensor* logits, const bimamba_tokens* targets,
                          const float* lse, const float* entropy, const float* dlogp, const float* dentropy,
                          const bimamba_tensor* dlogits, void* hip_stream)
{
    int rc = check_logits(d);
    if (rc) return rc;
    if (!logits || !dlogits) return BIMAMBA_ERR_NULL_POINTER;
    if (d->batch == 0 || d->seqlen == 0) return BIMAMBA_OK;
    if (!lse || ((dlogp || d->targets_only) && !targets) || (dentropy && !entropy)) return BIMAMBA_ERR_NULL_POINTER;
    const long long rows = (long long)d->batch * d->seqlen;
    const size_t elem = dtype_bytes(d->io_dtype);
    Bytes from, to, ids{0, 0};
    if ((rc = check_view(logits, d->batch, d->seqlen, d->vocab, d->io_dtype, false, &from))) return rc;
    if ((rc = check_view(dlogits, d->batch, d->seqlen, d->vocab, d->io_dtype, true, &to))) return rc;
    if (targets && (rc = check_tokens(targets, d->batch, d->seqlen, &ids))) return rc;
    const float* const lse_rest = lse_rest_of(d);
    for (const float* r : {lse, lse_rest, entropy, dlogp, dentropy})
        if (!aligned_to(r, 4)) return BIMAMBA_ERR_MISALIGNED;
    const bool same = logits->ptr == dlogits->ptr && (d->seqlen == 1 || logits->stride_token == dlogits->stride_token) &&
                      (d->batch == 1 || logits->stride_batch == dlogits->stride_batch);
    if (!same && views_meet(dlogits, d->vocab, to, logits, d->vocab, from, d->batch, elem, elem)) return BIMAMBA_ERR_ALIAS;
    if (meet(to, ids)) return BIMAMBA_ERR_ALIAS;
    for (const float* r : {lse, lse_rest, entropy, dlogp, dentropy})
        if (meet(to, bytes_of(r, rows, 4))) return BIMAMBA_ERR_ALIAS;
    ScoresBwdArgs a{};
    a.logits = row_view(logits), a.dlogits = row_view(dlogits);
    if (targets) a.ids = targets->ptr, a.ids_sb = targets->stride_batch, a.ids_st = targets->stride_token;
    a.lse = lse, a.lse_rest = lse_rest, a.entropy = entropy, a.dlogp = dlogp, a.dentropy = dentropy;
    a.L = d->seqlen, a.vocab = d->vocab, a.targets_only = d->targets_only;
    a.parts = (unsigned)((d->vocab + (long long)kGradPart - 1) / kGradPart);
    const unsigned long long all = (unsigned long long)rows * a.parts;
    if (all >= 1ull << 31) return BIMAMBA_ERR_UNSUPPORTED;
    a.all = (unsigned)all;
    const unsigned grid = all < 1u << 22 ? (unsigned)all : 1u << 22;
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    const bool past = past_caches(2.0 * rows * d->vocab * elem);
    if (d->io_dtype == BIMAMBA_BF16) launch_scores_bwd<IoBF16>(a, grid, past, st);
    else launch_scores_bwd<IoF32>(a, grid, past, st);
    return launches.status();
}

}  // extern "C"
