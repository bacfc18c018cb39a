// Layer norm with a weight and a bias that rows share or that each batch element has of its own, and its gradients.
#include "model_ops.h"

namespace bm {

// A row stays in registers: `waves` waves hold it, 8, 16 or 32 elements a lane in pieces of 16 bytes, lanes side by side.  The statistics are
// taken in two steps over the registers (the mean, then the squares of what is left), so that a large mean costs no precision; where
// four waves share a row each takes both of its own part, and one exchange joins them (the squares around the common mean are the
// parts' own plus what their means are off by).  A wave takes many rows one after the other, the next one on its way, with weight and
// bias in registers: read again for each row they would be twice the row's own bytes.  What bounds it are the bytes: 65536 rows of
// 2048 bf16 95 us (5.6 TB/s).  Few rows, one to four waves each: 512 rows 4.2 us, the launch and one load's time.
struct NormRows {
    unsigned L, rows;      // tokens of a batch element; rows that share a vector: all, or (per_batch) those of a batch element
    unsigned per_group;    // rows that a group of waves takes, one after the other
    int per_batch;
};
struct NormRow {
    unsigned b, t;
    long long at;   // its place among all rows
};
// Row r of those that share the vector `v`.
__device__ __forceinline__ NormRow norm_row(const NormRows& n, unsigned v, unsigned r)
{
    if (n.per_batch) return NormRow{v, r, (long long)v * n.L + r};
    const unsigned b = r / n.L;
    return NormRow{b, r - b * n.L, r};
}
struct NormArgs {
    RowView x, y;
    const float *weight, *bias;
    long long weight_stride;
    float *mean, *rstd;
    NormRows n;
    int d;
    float eps;
};

template <int kWaves>
struct Exchange {
    float2 part[2][kWaves];
};
// The sums of a pair over the waves of a row; each wave gives its own, the same in all of its lanes.  `turn` alternates between calls,
// so that one barrier a call is enough.
template <int kWaves>
__device__ __forceinline__ float2 row_sum(float2 v, Exchange<kWaves>& ex, int wave, int turn)
{
    if constexpr (kWaves > 1) {
        ex.part[turn][wave] = v;   // (all lanes the same value)
        __syncthreads();
        v = ex.part[turn][0];
#pragma unroll
        for (int k = 1; k < kWaves; k++) {
            v.x += ex.part[turn][k].x;
            v.y += ex.part[turn][k].y;
        }
    }
    return v;
}

// kWaves 1: each of the workgroup's four waves takes rows of its own.
template <typename IO, int kWaves, int kPieces, int kPiece, bool kPast>
__device__ __forceinline__ void norm_rows(const NormArgs& a)
{
    __shared__ Exchange<kWaves> ex;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const unsigned group = kWaves == 1 ? blockIdx.x * 4 + wave : blockIdx.x, vector = blockIdx.y;
    const unsigned r0 = group * a.n.per_group, r1 = min(r0 + a.n.per_group, a.n.rows);
    if (r0 >= r1) return;   // (with four waves to a row: the whole workgroup)
    const int first = (kWaves == 1 ? 0 : wave * 64 * kPieces) * kPiece + lane * kPiece;
    const auto at = [&](int k) { return first + k * 64 * kPiece; };
    float w[kPieces][kPiece], c[kPieces][kPiece];
#pragma unroll
    for (int k = 0; k < kPieces; k++) {
        if (a.weight) load_floats(w[k], a.weight + vector * a.weight_stride, at(k), a.d, 0.0f);
        if (a.bias) load_floats(c[k], a.bias + vector * a.weight_stride, at(k), a.d, 0.0f);
#pragma unroll
        for (int i = 0; i < kPiece; i++) {
            if (!a.weight) w[k][i] = 1.0f;
            if (!a.bias) c[k][i] = 0.0f;
        }
    }
    const float inv = 1.0f / a.d;
    Piece<IO, kPiece> next[kPieces];
    const auto request = [&](unsigned r) {
        const NormRow row = norm_row(a.n, vector, r);
        const typename IO::T* const x = static_cast<const typename IO::T*>(a.x.p) + row_offset(a.x, row.b, row.t);
#pragma unroll
        for (int k = 0; k < kPieces; k++) next[k] = load_clamped<IO, kPiece>(x, at(k), a.d);
    };
    request(r0);
    for (unsigned r = r0; r < r1; r++) {
        float x[kPieces][kPiece], sum = 0.0f;
#pragma unroll
        for (int k = 0; k < kPieces; k++) {
            settle(next[k], at(k), a.d, typename IO::T(0));
#pragma unroll
            for (int i = 0; i < kPiece; i++) {
                x[k][i] = next[k][i];
                sum += x[k][i];
            }
        }
        if (r + 1 < r1) request(r + 1);
        sum = wave_sum(sum);
        // the part's own mean and squares around it
        const int mine = kWaves == 1 ? a.d : max(0, min(a.d - wave * 64 * kPieces * kPiece, 64 * kPieces * kPiece));
        const float part_mean = mine > 0 ? sum / mine : 0.0f;
        float sq = 0.0f;
#pragma unroll
        for (int k = 0; k < kPieces; k++)
#pragma unroll
            for (int i = 0; i < kPiece; i++) {
                const float e = at(k) + i < a.d ? x[k][i] - part_mean : 0.0f;
                sq += e * e;
            }
        sq = wave_sum(sq);
        float mean = part_mean, var;
        if constexpr (kWaves > 1) {
            const int turn = (r - r0) & 1;
            ex.part[turn][wave] = make_float2(sum, sq);
            __syncthreads();
            float all = 0.0f;
#pragma unroll
            for (int k = 0; k < kWaves; k++) all += ex.part[turn][k].x;
            mean = all * inv;
            var = 0.0f;
#pragma unroll
            for (int k = 0; k < kWaves; k++) {
                const int n = max(0, min(a.d - k * 64 * kPieces * kPiece, 64 * kPieces * kPiece));
                const float off = n > 0 ? ex.part[turn][k].x / n - mean : 0.0f;
                var += ex.part[turn][k].y + n * (off * off);
            }
            var *= inv;
        } else {
            var = sq * inv;
        }
        const float rstd = 1.0f / sqrtf(var + a.eps);
        const NormRow row = norm_row(a.n, vector, r);
        typename IO::T* const y = static_cast<typename IO::T*>(a.y.p) + row_offset(a.y, row.b, row.t);
#pragma unroll
        for (int k = 0; k < kPieces; k++) {
            float f[kPiece];
#pragma unroll
            for (int i = 0; i < kPiece; i++) f[i] = (x[k][i] - mean) * rstd * w[k][i] + c[k][i];
            store_piece_of<IO, kPast>(y, at(k), a.d, f);
        }
        if (lane == 0 && (kWaves == 1 || wave == 0)) {
            if (a.mean) a.mean[row.at] = mean;
            if (a.rstd) a.rstd[row.at] = rstd;
        }
    }
}

template <typename IO, int kWaves, int kElems, bool kPast>
__global__ __launch_bounds__(256) void norm_kernel(const NormArgs a)
{
    if constexpr (kWaves == 1 && kElems == 8) {   // (rows shorter than a piece: an element a lane)
        if (a.d < kPieceOf<IO>) return norm_rows<IO, 1, 1, 1, kPast>(a);
    }
    norm_rows<IO, kWaves, kElems / kPieceOf<IO>, kPieceOf<IO>, kPast>(a);
}

// Rows longer than the registers of four waves: one workgroup of sixteen waves to a row, which it reads three times (from the caches
// the second and third time).
constexpr int kLongThreads = 1024;
__device__ __forceinline__ float workgroup_sum(float v, float* part)
{
    v = wave_sum(v);
    __syncthreads();
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    float all = 0.0f;
#pragma unroll
    for (int k = 0; k < kLongThreads / 64; k++) all += part[k];
    return all;
}
template <typename IO>
__global__ __launch_bounds__(kLongThreads) void norm_long_kernel(const NormArgs a)
{
    constexpr int kPiece = kPieceOf<IO>;
    __shared__ float part[kLongThreads / 64];
    const unsigned vector = blockIdx.y;
    const int first = threadIdx.x * kPiece, step = kLongThreads * kPiece;
    const float inv = 1.0f / a.d;
    for (unsigned r = blockIdx.x; r < a.n.rows; r += gridDim.x) {
        const NormRow row = norm_row(a.n, vector, r);
        const typename IO::T* const x = static_cast<const typename IO::T*>(a.x.p) + row_offset(a.x, row.b, row.t);
        float s = 0.0f;
        for (int at = first; at < a.d; at += step) {
            const Piece<IO> p = load_piece_of<IO>(x, at, a.d, typename IO::T(0));
#pragma unroll
            for (int i = 0; i < kPiece; i++) s += p[i];
        }
        const float mean = workgroup_sum(s, part) * inv;
        s = 0.0f;
        for (int at = first; at < a.d; at += step) {
            const Piece<IO> p = load_piece_of<IO>(x, at, a.d, typename IO::T(0));
#pragma unroll
            for (int i = 0; i < kPiece; i++) {
                const float e = at + i < a.d ? p[i] - mean : 0.0f;
                s += e * e;
            }
        }
        const float rstd = 1.0f / sqrtf(workgroup_sum(s, part) * inv + a.eps);
        typename IO::T* const y = static_cast<typename IO::T*>(a.y.p) + row_offset(a.y, row.b, row.t);
        for (int at = first; at < a.d; at += step) {
            const Piece<IO> p = load_piece_of<IO>(x, at, a.d, typename IO::T(0));
            float f[kPiece], w[kPiece], c[kPiece];
            if (a.weight) load_floats(w, a.weight + vector * a.weight_stride, at, a.d, 0.0f);
            if (a.bias) load_floats(c, a.bias + vector * a.weight_stride, at, a.d, 0.0f);
#pragma unroll
            for (int i = 0; i < kPiece; i++) f[i] = (p[i] - mean) * rstd * (a.weight ? w[i] : 1.0f) + (a.bias ? c[i] : 0.0f);
            store_piece_of<IO>(y, at, a.d, f);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row.at] = mean;
            if (a.rstd) a.rstd[row.at] = rstd;
        }
    }
}

// ---- gradients ----
//
// A row is held as in the forward call.  A group of waves takes `per_group` rows of one batch element after the other and keeps the
// sums of dy * xh and dy over them in registers; it leaves them in a slot of its own, and a second launch adds the slots of a vector in
// a fixed order.  Where one workgroup takes all rows of a vector its sums are the gradients, and there is neither slot nor second launch.  What bounds it are the bytes: 65536 rows of 2048 bf16 156 to 162 us (5.2 to 5.0 TB/s with the slots), the second launch 6 of them;
// 3711 rows of 740 fp32 12.8 us, two launches and two rows a wave one after the other.
struct NormBwdArgs {
    RowView x, dy, dx;
    const float *weight, *mean, *rstd;
    long long weight_stride;
    float *dw, *db;   // sums of a workgroup, null: not wanted; in slots [vectors][workgroups][2][d], or the vectors' gradients themselves
    long long slot;   // from one workgroup's to the next one's
    NormRows n;
    int d;
};
template <typename IO, int kWaves, int kPieces, int kPiece, bool kPast>
__device__ __forceinline__ void norm_bwd_rows(const NormBwdArgs& a)
{
    __shared__ Exchange<kWaves> ex;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const unsigned group = kWaves == 1 ? blockIdx.x * 4 + wave : blockIdx.x, vector = blockIdx.y;
    const unsigned r0 = group * a.n.per_group, r1 = min(r0 + a.n.per_group, a.n.rows);   // (r0 >= r1: a wave without rows, which leaves zeros)
    const int first = (kWaves == 1 ? 0 : wave * 64 * kPieces) * kPiece + lane * kPiece;
    const auto at = [&](int k) { return first + k * 64 * kPiece; };
    float w[kPieces][kPiece], dw[kPieces][kPiece], db[kPieces][kPiece];
#pragma unroll
    for (int k = 0; k < kPieces; k++) {
        if (a.weight) load_floats(w[k], a.weight + vector * a.weight_stride, at(k), a.d, 0.0f);
#pragma unroll
        for (int i = 0; i < kPiece; i++) {
            if (!a.weight) w[k][i] = 1.0f;
            dw[k][i] = db[k][i] = 0.0f;
        }
    }
    const float inv = 1.0f / a.d;
    // (the next row's elements asked for while a row is computed: 8000 rows of 1500 19.5 -> 22 us, 512 rows of 2048 6.6 -> 7.4)
    for (unsigned r = r0; r < r1; r++) {
        const NormRow row = norm_row(a.n, vector, r);
        const typename IO::T* const x = static_cast<const typename IO::T*>(a.x.p) + row_offset(a.x, row.b, row.t);
        const typename IO::T* const dy = static_cast<const typename IO::T*>(a.dy.p) + row_offset(a.dy, row.b, row.t);
        Piece<IO, kPiece> px[kPieces], pd[kPieces];
#pragma unroll
        for (int k = 0; k < kPieces; k++) px[k] = load_clamped<IO, kPiece, kPast>(x, at(k), a.d);
#pragma unroll
        for (int k = 0; k < kPieces; k++) pd[k] = load_clamped<IO, kPiece, kPast>(dy, at(k), a.d);
        const float mean = a.mean[row.at], rstd = a.rstd[row.at];
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < kPieces; k++) {
            settle(px[k], at(k), a.d, typename IO::T(0));
            settle(pd[k], at(k), a.d, typename IO::T(0));   // (beyond the row: g = 0)
#pragma unroll
            for (int i = 0; i < kPiece; i++) {
                const float xh = (px[k][i] - mean) * rstd, d = pd[k][i], g = d * w[k][i];
                dw[k][i] += d * xh;
                db[k][i] += d;
                s.x += g;
                s.y += g * xh;
            }
        }
        s.x = wave_sum(s.x);
        s.y = wave_sum(s.y);
        s = row_sum<kWaves>(s, ex, wave, (r - r0) & 1);
        const float c0 = s.x * inv, c1 = s.y * inv;
        typename IO::T* const dx = static_cast<typename IO::T*>(a.dx.p) + row_offset(a.dx, row.b, row.t);
#pragma unroll
        for (int k = 0; k < kPieces; k++) {
            float f[kPiece];
#pragma unroll
            for (int i = 0; i < kPiece; i++) f[i] = rstd * (pd[k][i] * w[k][i] - c0 - (px[k][i] - mean) * rstd * c1);
            store_piece_of<IO, kPast>(dx, at(k), a.d, f);
        }
    }
    const long long slot = ((long long)vector * gridDim.x + blockIdx.x) * a.slot;
    if constexpr (kWaves > 1) {
#pragma unroll
        for (int k = 0; k < kPieces; k++) {
            if (a.dw) store_piece_of<IoF32>(a.dw + slot, at(k), a.d, dw[k]);
            if (a.db) store_piece_of<IoF32>(a.db + slot, at(k), a.d, db[k]);
        }
    } else {   // four waves' sums of the same channels: one of the two at a time through shared memory
        __shared__ float sum[4][64 * kPieces * kPiece];
#pragma unroll
        for (int which = 0; which < 2; which++) {
            float* const to = which ? a.db : a.dw;
            if (!to) continue;   // (all threads)
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kPieces; k++)
#pragma unroll
                for (int i = 0; i < kPiece; i++) sum[wave][(k * 64 + lane) * kPiece + i] = which ? db[k][i] : dw[k][i];
            __syncthreads();
            for (int c = threadIdx.x; c < a.d; c += 256) to[slot + c] = (sum[0][c] + sum[1][c]) + (sum[2][c] + sum[3][c]);
        }
    }
}

template <typename IO, int kWaves, int kElems, bool kPast>
__global__ __launch_bounds__(256) void norm_bwd_kernel(const NormBwdArgs a)
{
    if constexpr (kWaves == 1 && kElems == 8) {   // (rows shorter than a piece: an element a lane)
        if (a.d < kPieceOf<IO>) return norm_bwd_rows<IO, 1, 1, 1, kPast>(a);
    }
    norm_bwd_rows<IO, kWaves, kElems / kPieceOf<IO>, kPieceOf<IO>, kPast>(a);
}

// Long rows: two reads of a row; the sums over rows are taken by norm_long_cols_kernel from x and dy again.
template <typename IO>
__global__ __launch_bounds__(kLongThreads) void norm_bwd_long_kernel(const NormBwdArgs a)
{
    constexpr int kPiece = kPieceOf<IO>;
    __shared__ float part[kLongThreads / 64];
    const unsigned vector = blockIdx.y;
    const int first = threadIdx.x * kPiece, step = kLongThreads * kPiece;
    const float inv = 1.0f / a.d;
    const auto weights = [&](float (&w)[kPiece], int at) {
        if (a.weight) load_floats(w, a.weight + vector * a.weight_stride, at, a.d, 0.0f);
        else
            for (int i = 0; i < kPiece; i++) w[i] = 1.0f;
    };
    for (unsigned r = blockIdx.x; r < a.n.rows; r += gridDim.x) {
        const NormRow row = norm_row(a.n, vector, r);
        const typename IO::T* const x = static_cast<const typename IO::T*>(a.x.p) + row_offset(a.x, row.b, row.t);
        const typename IO::T* const dy = static_cast<const typename IO::T*>(a.dy.p) + row_offset(a.dy, row.b, row.t);
        typename IO::T* const dx = static_cast<typename IO::T*>(a.dx.p) + row_offset(a.dx, row.b, row.t);
        const float mean = a.mean[row.at], rstd = a.rstd[row.at];
        float s0 = 0.0f, s1 = 0.0f, w[kPiece];
        for (int at = first; at < a.d; at += step) {
            const Piece<IO> px = load_piece_of<IO>(x, at, a.d, typename IO::T(0)), pd = load_piece_of<IO>(dy, at, a.d, typename IO::T(0));
            weights(w, at);
#pragma unroll
            for (int i = 0; i < kPiece; i++) {
                const float g = pd[i] * w[i];
                s0 += g;
                s1 += g * ((px[i] - mean) * rstd);
            }
        }
        const float c0 = workgroup_sum(s0, part) * inv, c1 = workgroup_sum(s1, part) * inv;
        for (int at = first; at < a.d; at += step) {
            const Piece<IO> px = load_piece_of<IO>(x, at, a.d, typename IO::T(0)), pd = load_piece_of<IO>(dy, at, a.d, typename IO::T(0));
            weights(w, at);
            float f[kPiece];
#pragma unroll
            for (int i = 0; i < kPiece; i++) f[i] = rstd * (pd[i] * w[i] - c0 - (px[i] - mean) * rstd * c1);
            store_piece_of<IO>(dx, at, a.d, f);
        }
    }
}
// grid (groups of rows, vectors, columns of 256 threads): a thread sums the channels of a piece over the group's rows.
template <typename IO>
__global__ __launch_bounds__(256) void norm_long_cols_kernel(const NormBwdArgs a)
{
    constexpr int kPiece = kPieceOf<IO>;
    const unsigned vector = blockIdx.y, r0 = blockIdx.x * a.n.per_group, r1 = min(r0 + a.n.per_group, a.n.rows);
    const int at = (blockIdx.z * 256 + threadIdx.x) * kPiece;
    if (at >= a.d) return;
    float dw[kPiece] = {}, db[kPiece] = {};
    for (unsigned r = r0; r < r1; r++) {
        const NormRow row = norm_row(a.n, vector, r);
        const Piece<IO> px = load_piece_of<IO>(static_cast<const typename IO::T*>(a.x.p) + row_offset(a.x, row.b, row.t), at, a.d, typename IO::T(0));
        const Piece<IO> pd = load_piece_of<IO>(static_cast<const typename IO::T*>(a.dy.p) + row_offset(a.dy, row.b, row.t), at, a.d, typename IO::T(0));
        const float mean = a.mean[row.at], rstd = a.rstd[row.at];
#pragma unroll
        for (int i = 0; i < kPiece; i++) {
            dw[i] += pd[i] * ((px[i] - mean) * rstd);
            db[i] += pd[i];
        }
    }
    const long long slot = ((long long)vector * gridDim.x + blockIdx.x) * a.slot;
    if (a.dw) store_piece_of<IoF32>(a.dw + slot, at, a.d, dw);
    if (a.db) store_piece_of<IoF32>(a.db + slot, at, a.d, db);
}

// dweight and dbias: the slots of a vector, added up 32 channels to a workgroup, each of its rows of threads a share of the slots.
constexpr int kSumChannels = 32, kFewSums = 8, kManySums = 32;   // (rows of threads, by the number of slots)
struct NormSumArgs {
    const float* slots;
    float *dweight, *dbias;
    long long count;   // slots of one vector
    int d;
};
template <int kRows>
__global__ __launch_bounds__(kRows * kSumChannels) void norm_sum_kernel(const NormSumArgs a)
{
    float* const out = blockIdx.z ? a.dbias : a.dweight;
    if (!out) return;
    const int c = threadIdx.x % kSumChannels, r = threadIdx.x / kSumChannels, col = blockIdx.x * kSumChannels + c;
    __shared__ float sum[kRows][kSumChannels];
    float s = 0.0f;
    const float* const from = a.slots + ((long long)blockIdx.y * a.count * 2 + blockIdx.z) * a.d + col;
    if (col < a.d)
#pragma unroll 8
        for (long long i = r; i < a.count; i += kRows) s += from[i * 2 * a.d];
    sum[r][c] = s;
    __syncthreads();
    if (r == 0 && col < a.d) {
#pragma unroll
        for (int k = 1; k < kRows; k++) s += sum[k][c];
        out[(long long)blockIdx.y * a.d + col] = s;
    }
}

namespace {

constexpr int kMaxNormWidth = 65536;

int check_norm(const bimamba_norm_desc* d)
{
    if (!d) return BIMAMBA_ERR_NULL_POINTER;
    if (d->struct_size != sizeof(bimamba_norm_desc) || d->d_model < 1) return BIMAMBA_ERR_BAD_SHAPE;
    if (!(d->eps > 0.0f) || !std::isfinite(d->eps)) return BIMAMBA_ERR_BAD_SHAPE;
    if (const int rc = check_rows(d->batch, d->seqlen)) return rc;
    if (!known_dtype(d->io_dtype) || d->batch > 65535 || d->d_model > kMaxNormWidth) return BIMAMBA_ERR_UNSUPPORTED;
    return BIMAMBA_OK;
}

// Which waves hold a row, and how many rows a group of them takes.
struct NormPlan {
    int waves, elems;   // elements a lane; 0: a long row
    unsigned vectors, groups;   // vectors that rows share; workgroups of each
    NormRows n;
};
NormPlan plan_norm(const bimamba_norm_desc* d, bool per_batch, bool bwd)
{
    NormPlan p{};
    const unsigned rows = (unsigned)((long long)d->batch * d->seqlen);
    const int one = 64 * 8;
    const bool spread = rows < 4u * cu_count() || bwd;
    p.waves = d->d_model <= (bwd ? 2 : 1) * one || (!spread && d->d_model <= 4 * one) ? 1 : 4;
    const int need = (d->d_model + p.waves * one - 1) / (p.waves * one);
    p.elems = need <= 1 ? 8 : need <= 2 ? 16 : need <= 4 ? 32 : 0;
    p.vectors = per_batch ? d->batch : 1;
    p.n.L = d->seqlen;
    p.n.rows = per_batch ? d->seqlen : rows;
    p.n.per_batch = per_batch;
    const unsigned together = p.elems && p.waves == 1 ? 4 : 1;   // rows that a workgroup has in hand at once
    // Workgroups in all.  Forward: 16 a CU.  Gradients: as many as the registers hold at once (four a CU, two with 16 elements a lane or
    // more), but at least eight rows to each while every CU has one, since each leaves a slot as long as two rows (3711 rows of 740
    // fp32: 464 workgroups 9.2 + 4.7 us, 928 of them 11.0 + 5.7; 16384 rows of 4096: 512 of them 82 + 5, 1024 91 + 7).
    unsigned want = 16u * cu_count();
    if (bwd) {
        const unsigned most = (p.waves == 4 && p.elems != 8 ? 2u : 4u) * cu_count(), least = cu_count();
        want = rows / 8 < least ? least : rows / 8 > most ? most : rows / 8;
    }
    const unsigned groups = p.vectors ? (want + p.vectors - 1) / p.vectors : 1;
    const unsigned per_workgroup = (p.n.rows + groups - 1) / groups;
    p.n.per_group = (per_workgroup + together - 1) / together;
    if (p.n.per_group < 1) p.n.per_group = 1;
    const unsigned long long step = (unsigned long long)p.n.per_group * together;
    p.groups = (unsigned)((p.n.rows + step - 1) / step);
    return p;
}
unsigned long_groups(const NormRows& n) { return n.rows < 1u << 16 ? n.rows : 1u << 16; }

template <typename IO, bool kPast>
void launch_norm(const NormPlan& p, const NormArgs& a, hipStream_t st)
{
    const dim3 grid(p.groups, p.vectors), wg(256);
    switch (p.elems * 8 + p.waves) {
        case 8 * 8 + 1: hipLaunchKernelGGL((norm_kernel<IO, 1, 8, kPast>), grid, wg, 0, st, a); break;
        case 16 * 8 + 1: hipLaunchKernelGGL((norm_kernel<IO, 1, 16, kPast>), grid, wg, 0, st, a); break;
        case 32 * 8 + 1: hipLaunchKernelGGL((norm_kernel<IO, 1, 32, kPast>), grid, wg, 0, st, a); break;
        case 8 * 8 + 4: hipLaunchKernelGGL((norm_kernel<IO, 4, 8, false>), grid, wg, 0, st, a); break;   // (few rows, of 2048 at most: 16 MB)
        case 16 * 8 + 4: hipLaunchKernelGGL((norm_kernel<IO, 4, 16, kPast>), grid, wg, 0, st, a); break;
        case 32 * 8 + 4: hipLaunchKernelGGL((norm_kernel<IO, 4, 32, kPast>), grid, wg, 0, st, a); break;
        default: hipLaunchKernelGGL(norm_long_kernel<IO>, dim3(long_groups(a.n), p.vectors), dim3(kLongThreads), 0, st, a);
    }
}
template <typename IO, bool kPast>
void launch_norm_bwd(const NormPlan& p, const NormBwdArgs& a, hipStream_t st)
{
    const dim3 grid(p.groups, p.vectors), wg(256);
    switch (p.elems * 8 + p.waves) {
        case 8 * 8 + 1: hipLaunchKernelGGL((norm_bwd_kernel<IO, 1, 8, kPast>), grid, wg, 0, st, a); break;
        case 16 * 8 + 1: hipLaunchKernelGGL((norm_bwd_kernel<IO, 1, 16, kPast>), grid, wg, 0, st, a); break;
        case 8 * 8 + 4: hipLaunchKernelGGL((norm_bwd_kernel<IO, 4, 8, kPast>), grid, wg, 0, st, a); break;
        case 16 * 8 + 4: hipLaunchKernelGGL((norm_bwd_kernel<IO, 4, 16, kPast>), grid, wg, 0, st, a); break;
        case 32 * 8 + 4: hipLaunchKernelGGL((norm_bwd_kernel<IO, 4, 32, kPast>), grid, wg, 0, st, a); break;
        default:
            hipLaunchKernelGGL(norm_bwd_long_kernel<IO>, dim3(long_groups(a.n), p.vectors), dim3(kLongThreads), 0, st, a);
            if (a.dw || a.db)
                hipLaunchKernelGGL(norm_long_cols_kernel<IO>, dim3(p.groups, p.vectors, (a.d + 256 * kPieceOf<IO> - 1) / (256 * kPieceOf<IO>)), wg, 0, st, a);
    }
}

// A parameter vector for all rows, or one for each batch element.
int check_vector(const float* p, long long stride, const bimamba_norm_desc* d, Bytes* r)
{
    if (!p) {
        *r = Bytes{0, 0};
        return BIMAMBA_OK;
    }
    if (!aligned_to(p, 4)) return BIMAMBA_ERR_MISALIGNED;
    return bytes_of(p, stride, 0, d->batch, 1, d->d_model, 4, r) ? BIMAMBA_OK : BIMAMBA_ERR_BAD_SHAPE;
}

}  // namespace
}  // namespace bm

using namespace bm;

extern "C" {

int bimamba_layer_norm(const bimamba_norm_desc* d, const bimamba_tensor* x, const float* weight, const float* bias,
                       int64_t weight_stride, const bimamba_tensor* y, float* mean, float* rstd, void* hip_stream)
{
    int rc = check_norm(d);
    if (rc) return rc;
    if (!x || !y) return BIMAMBA_ERR_NULL_POINTER;
    if (weight_stride != 0 && weight_stride < d->d_model) return BIMAMBA_ERR_BAD_SHAPE;
    if (d->batch == 0 || d->seqlen == 0) return BIMAMBA_OK;
    const long long rows = (long long)d->batch * d->seqlen;
    const size_t elem = dtype_bytes(d->io_dtype);
    Bytes from, to, w, c;
    if ((rc = check_view(x, d->batch, d->seqlen, d->d_model, d->io_dtype, false, &from))) return rc;
    if ((rc = check_view(y, d->batch, d->seqlen, d->d_model, d->io_dtype, true, &to))) return rc;
    if ((rc = check_vector(weight, weight_stride, d, &w)) || (rc = check_vector(bias, weight_stride, d, &c))) return rc;
    if (!aligned_to(mean, 4) || !aligned_to(rstd, 4)) return BIMAMBA_ERR_MISALIGNED;
    const Bytes m = bytes_of(mean, rows, 4), r = bytes_of(rstd, rows, 4);
    if (views_meet(y, d->d_model, to, x, d->d_model, from, d->batch, elem, elem) || meet(to, w) || meet(to, c)) return BIMAMBA_ERR_ALIAS;
    for (const Bytes& s : {m, r})
        if (meet(s, to) || meet(s, from) || meet(s, w) || meet(s, c)) return BIMAMBA_ERR_ALIAS;
    if (meet(m, r)) return BIMAMBA_ERR_ALIAS;
    const NormPlan p = plan_norm(d, weight_stride != 0, false);
    const NormArgs a{row_view(x), row_view(y), weight, bias, weight_stride, mean, rstd, p.n, d->d_model, d->eps};
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    const bool past = past_caches(2.0 * rows * d->d_model * elem), bf16 = d->io_dtype == BIMAMBA_BF16;
    if (bf16 && past) launch_norm<IoBF16, true>(p, a, st);
    else if (bf16) launch_norm<IoBF16, false>(p, a, st);
    else if (past) launch_norm<IoF32, true>(p, a, st);
    else launch_norm<IoF32, false>(p, a, st);
    return launches.status();
}

size_t bimamba_layer_norm_bwd_workspace_bytes(const bimamba_norm_desc* d, int per_batch)
{
    if (check_norm(d) || d->batch == 0 || d->seqlen == 0) return 0;
    const NormPlan p = plan_norm(d, per_batch != 0, true);
    return p.groups > 1 ? (size_t)p.groups * p.vectors * 2 * d->d_model * sizeof(float) : 0;
}

int bimamba_layer_norm_bwd(const bimamba_norm_desc* d, const bimamba_tensor* x, const float* weight, int64_t weight_stride,
                           const float* mean, const float* rstd, const bimamba_tensor* dy, const bimamba_tensor* dx,
                           float* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    int rc = check_norm(d);
    if (rc) return rc;
    if (!x || !dy || !dx) return BIMAMBA_ERR_NULL_POINTER;
    if (weight_stride != 0 && weight_stride < d->d_model) return BIMAMBA_ERR_BAD_SHAPE;
    if (!aligned_to(dweight, 4) || !aligned_to(dbias, 4)) return BIMAMBA_ERR_MISALIGNED;
    const long long rows = (long long)d->batch * d->seqlen;
    const int vectors = weight_stride ? d->batch : 1;
    const bool sums = dweight || dbias;
    const NormPlan p = plan_norm(d, weight_stride != 0, true);
    const size_t need = rows && sums ? bimamba_layer_norm_bwd_workspace_bytes(d, weight_stride != 0) : 0;
    if (rows) {
        if (!mean || !rstd) return BIMAMBA_ERR_NULL_POINTER;
        const size_t elem = dtype_bytes(d->io_dtype);
        Bytes bx, by, to, w;
        if ((rc = check_view(x, d->batch, d->seqlen, d->d_model, d->io_dtype, false, &bx))) return rc;
        if ((rc = check_view(dy, d->batch, d->seqlen, d->d_model, d->io_dtype, false, &by))) return rc;
        if ((rc = check_view(dx, d->batch, d->seqlen, d->d_model, d->io_dtype, true, &to))) return rc;
        if ((rc = check_vector(weight, weight_stride, d, &w))) return rc;
        if (!aligned_to(mean, 4) || !aligned_to(rstd, 4)) return BIMAMBA_ERR_MISALIGNED;
        if ((rc = check_workspace(workspace, workspace_bytes, need))) return rc;
        const Bytes m = bytes_of(mean, rows, 4), r = bytes_of(rstd, rows, 4), ws = bytes_of(need ? workspace : nullptr, need, 1);
        const Bytes dw = bytes_of(dweight, (long long)vectors * d->d_model, 4), db = bytes_of(dbias, (long long)vectors * d->d_model, 4);
        if (views_meet(dx, d->d_model, to, x, d->d_model, bx, d->batch, elem, elem) ||
            views_meet(dx, d->d_model, to, dy, d->d_model, by, d->batch, elem, elem))
            return BIMAMBA_ERR_ALIAS;
        const Bytes written[] = {to, ws, dw, db}, read[] = {w, m, r, bx, by};
        for (int i = 0; i < 4; i++) {
            for (int j = 0; j < (i == 0 ? 3 : 5); j++)
                if (meet(written[i], read[j])) return BIMAMBA_ERR_ALIAS;
            for (int j = 0; j < i; j++)
                if (meet(written[i], written[j])) return BIMAMBA_ERR_ALIAS;
        }
    }
    if (vectors == 0 || (!rows && !sums)) return BIMAMBA_OK;
    const bool direct = rows && p.groups == 1;   // (one workgroup a vector)
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    if (rows) {
        float* const slots = sums ? static_cast<float*>(workspace) : nullptr;
        const NormBwdArgs a{row_view(x), row_view(dy), row_view(dx), weight, mean, rstd, weight_stride,
                            direct ? dweight : slots, direct ? dbias : slots ? slots + d->d_model : nullptr,
                            (direct ? 1ll : 2ll) * d->d_model, p.n, d->d_model};
        const bool past = past_caches(3.0 * rows * d->d_model * dtype_bytes(d->io_dtype)), bf16 = d->io_dtype == BIMAMBA_BF16;
        if (bf16 && past) launch_norm_bwd<IoBF16, true>(p, a, st);
        else if (bf16) launch_norm_bwd<IoBF16, false>(p, a, st);
        else if (past) launch_norm_bwd<IoF32, true>(p, a, st);
        else launch_norm_bwd<IoF32, false>(p, a, st);
    }
    if (sums && !direct) {   // (no rows: sums of nothing)
        const long long count = rows ? p.groups : 0;
        const NormSumArgs a{static_cast<const float*>(workspace), dweight, dbias, count, d->d_model};
        const dim3 grid((d->d_model + kSumChannels - 1) / kSumChannels, vectors, 2);
        if (count <= 8 * kFewSums) hipLaunchKernelGGL(norm_sum_kernel<kFewSums>, grid, dim3(kFewSums * kSumChannels), 0, st, a);
        else hipLaunchKernelGGL(norm_sum_kernel<kManySums>, grid, dim3(kManySums * kSumChannels), 0, st, a);
    }
    return launches.status();
}

}  // extern "C"
