// The norm of many gradient tensors, and the tensors scaled so that it is at most a given one.
#include "model_ops.h"

namespace bm {

// All tensors are cut into pieces of 8192 elements, numbered through, which the workgroups take in turn; a piece's tensor is found by
// search.  Two launches: the squares' sums, 64 bits each, one a workgroup; then every workgroup adds up all of these in the same
// order, which gives it the norm, and scales its pieces.  What bounds it are the bytes: two reads, one write.  The second launch
// goes from the last piece to the first, so that it starts with what the first has left in the caches; where the gradients are larger
// than these, the first reads all but the last 192 MB past them, and the second goes past them altogether.  609 M values, 1.2 GB: 609 us
// (each workgroup a run of pieces of its own, walked backwards, everything through the caches: 761; the pieces in turn 692; stores past
// the caches 640; nothing kept for the second launch 629).  40 tensors, 94208 values: 7.7 us, two launches and their chains of loads.
constexpr int kClipThreads = 256, kClipPiece = 8192;
constexpr int kClipSums = 8;               // sums that a thread adds up: of 2048 workgroups, eight a CU
constexpr long long kKept = 192ll << 20;   // bytes that the first launch leaves in the caches for the second
struct ClipArgs {
    const bimamba_grad* table;
    long long pieces, past;   // past: so many pieces are read past the caches at first
    int n;
    float max_norm;
    float* norm;
    double* sums;
};

// The last tensor that starts at or before a piece that there is (empty ones start where the next does).  64 tensors are looked at
// together, in the last round with all that is to be known of them.
__device__ __forceinline__ bimamba_grad tensor_of(const ClipArgs& a, long long piece)
{
    const int lane = threadIdx.x % 64;
    int lo = 0, range = a.n, step;
    while ((step = (range + 63) / 64) > 1) {
        const bool there = lane * step < range;
        const int count = __popcll(__ballot(there && a.table[there ? lo + lane * step : lo].first <= piece));   // (the first lanes)
        range = min(step, range - (count - 1) * step);
        lo += (count - 1) * step;
    }
    const bool there = lane < range;
    const bimamba_grad g = a.table[there ? lo + lane : lo];
    const int at = __popcll(__ballot(there && g.first <= piece)) - 1;
    const auto of_lane = [&](long long v) {
        return (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), at) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v, at));
    };
    bimamba_grad r{};
    r.from = reinterpret_cast<const void*>(of_lane(reinterpret_cast<long long>(g.from)));
    r.to = reinterpret_cast<void*>(of_lane(reinterpret_cast<long long>(g.to)));
    r.count = of_lane(g.count);
    r.first = of_lane(g.first);
    r.dtype = __builtin_amdgcn_readlane(g.dtype, at);
    return r;
}

// What a lane does with its elements of a piece, four loads in flight at a time: use(elements, where they start).  A piece of fewer elements
// than one load takes goes an element a lane.
constexpr int kClipAhead = 4;
template <typename IO, int N, bool kPast, typename Use>
__device__ __forceinline__ void for_piece(const typename IO::T* from, int n, Use use)
{
    for (int first = threadIdx.x * N; first < n; first += kClipThreads * N * kClipAhead) {
        Piece<IO, N> p[kClipAhead];
#pragma unroll
        for (int k = 0; k < kClipAhead; k++) p[k] = load_clamped<IO, N, kPast>(from, first + k * kClipThreads * N, n);
#pragma unroll
        for (int k = 0; k < kClipAhead; k++) {
            const int at = first + k * kClipThreads * N;
            settle(p[k], at, n, typename IO::T(0));
            use(p[k], at);
        }
    }
}
template <typename IO, bool kPast, typename Use>
__device__ __forceinline__ void for_piece(const typename IO::T* from, int n, Use use)
{
    if (n >= kPieceOf<IO>) for_piece<IO, kPieceOf<IO>, kPast>(from, n, use);
    else for_piece<IO, 1, kPast>(from, n, use);
}
template <typename IO, bool kPast>
__device__ __forceinline__ double piece_squares(const typename IO::T* from, int n)
{
    double s = 0.0;
    for_piece<IO, kPast>(from, n, [&](const auto& p, int) {
#pragma unroll
        for (auto e : p.v) {
            const double v = IO::cvt(e);
            s += v * v;
        }
    });
    return s;
}
template <typename IO, bool kPast>
__device__ __forceinline__ void piece_scaled(const typename IO::T* from, typename IO::T* to, int n, float scale)
{
    for_piece<IO, kPast>(from, n, [&](const auto& p, int at) {
        constexpr int N = sizeof p.v / sizeof p.v[0];
        float f[N];
#pragma unroll
        for (int i = 0; i < N; i++) f[i] = scale == 1.0f ? p[i] : p[i] * scale;
        store_piece_of<IO, kPast>(to, at, n, f);
    });
}

// The sum over a workgroup, the same in all lanes.
__device__ __forceinline__ double workgroup_sum(double v)
{
    __shared__ double part[kClipThreads / 64];
#pragma unroll
    for (int step = 32; step > 0; step /= 2) v += __shfl_xor(v, step);
    __syncthreads();
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ __launch_bounds__(kClipThreads) void clip_squares_kernel(const ClipArgs a)
{
    double s = 0.0;
    for (long long p = blockIdx.x; p < a.pieces; p += gridDim.x) {
        const bimamba_grad g = tensor_of(a, p);
        const long long at = (p - g.first) * kClipPiece;
        const int n = (int)min((long long)kClipPiece, (long long)g.count - at);
        const bool past = p < a.past;
        if (g.dtype == BIMAMBA_BF16) {
            const unsigned short* const from = static_cast<const unsigned short*>(g.from) + at;
            s += past ? piece_squares<IoBF16, true>(from, n) : piece_squares<IoBF16, false>(from, n);
        } else {
            const float* const from = static_cast<const float*>(g.from) + at;
            s += past ? piece_squares<IoF32, true>(from, n) : piece_squares<IoF32, false>(from, n);
        }
    }
    s = workgroup_sum(s);
    if (threadIdx.x == 0) a.sums[blockIdx.x] = s;
}

template <bool kPast>
__global__ __launch_bounds__(kClipThreads) void clip_scale_kernel(const ClipArgs a)
{
    // (the sums and the tensor of the first piece are asked for together)
    double part[kClipSums];
#pragma unroll
    for (int k = 0; k < kClipSums; k++) part[k] = k * kClipThreads + threadIdx.x < gridDim.x ? a.sums[k * kClipThreads + threadIdx.x] : 0.0;
    bimamba_grad g{};
    if (blockIdx.x < a.pieces) g = tensor_of(a, a.pieces - 1 - blockIdx.x);   // (no pieces: no table either)
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < kClipSums; k++) s += part[k];
    for (unsigned k = kClipSums * kClipThreads + threadIdx.x; k < gridDim.x; k += kClipThreads) s += a.sums[k];
    s = workgroup_sum(s);
    const double norm = sqrt(s);
    if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
    // (a norm that is not finite in 32 bits compares false or is taken out here)
    const float scale = isfinite((float)norm) && norm > (double)a.max_norm ? (float)((double)a.max_norm / norm) : 1.0f;
    for (long long k = blockIdx.x; k < a.pieces; k += gridDim.x) {
        const long long p = a.pieces - 1 - k;
        if (k != blockIdx.x) g = tensor_of(a, p);
        if (scale == 1.0f && g.from == g.to) continue;
        const long long at = (p - g.first) * kClipPiece;
        const int n = (int)min((long long)kClipPiece, (long long)g.count - at);
        if (g.dtype == BIMAMBA_BF16)
            piece_scaled<IoBF16, kPast>(static_cast<const unsigned short*>(g.from) + at, static_cast<unsigned short*>(g.to) + at, n, scale);
        else piece_scaled<IoF32, kPast>(static_cast<const float*>(g.from) + at, static_cast<float*>(g.to) + at, n, scale);
    }
}

namespace {

// Pieces of a table, or an error; `first` is checked against where the tensors before end, or filled.
int clip_pieces(const bimamba_grad* table, bimamba_grad* fill, int n, long long* pieces, long long* bytes = nullptr)
{
    if (n < 0) return BIMAMBA_ERR_BAD_SHAPE;
    if (n > 0 && !table) return BIMAMBA_ERR_NULL_POINTER;
    long long p = 0, b = 0;
    for (int i = 0; i < n; i++) {
        const bimamba_grad& g = table[i];
        if (g.count < 0 || g.reserved != 0) return BIMAMBA_ERR_BAD_SHAPE;
        if (!known_dtype(g.dtype) || g.count > 1ll << 40) return BIMAMBA_ERR_UNSUPPORTED;
        const size_t elem = dtype_bytes(g.dtype);
        if (g.count > 0) {
            if (!g.from || !g.to) return BIMAMBA_ERR_NULL_POINTER;
            if (!aligned_to(g.from, elem) || !aligned_to(g.to, elem)) return BIMAMBA_ERR_MISALIGNED;
            if (g.from != g.to && meet(bytes_of(g.from, g.count, elem), bytes_of(g.to, g.count, elem))) return BIMAMBA_ERR_ALIAS;
        }
        if (fill) fill[i].first = p;
        else if (g.first != p) return BIMAMBA_ERR_BAD_SHAPE;
        p += (g.count + kClipPiece - 1) / kClipPiece;
        b += g.count * (long long)elem;
    }
    *pieces = p;
    if (bytes) *bytes = b;
    return BIMAMBA_OK;
}

Bytes read_of(const bimamba_grad& g) { return bytes_of(g.from, g.count, dtype_bytes(g.dtype)); }
Bytes written_of(const bimamba_grad& g) { return bytes_of(g.to, g.count, dtype_bytes(g.dtype)); }

// Whether what each entry writes is apart from what all others read or write, entries being fine by themselves.  The numbers of those
// that are not empty are sorted by where they write, in the table's own `first` (which is filled afterwards): no memory is asked for.
bool clip_apart(bimamba_grad* table, int n)
{
    long long m = 0;
    for (int i = 0; i < n; i++)
        if (table[i].count > 0) table[m++].first = i;
    const auto entry = [&](long long k) -> const bimamba_grad& { return table[table[k].first]; };
    const auto before = [&](long long k, long long l) { return written_of(entry(k)).lo < written_of(entry(l)).lo; };
    const auto swap = [&](long long k, long long l) {
        const int64_t i = table[k].first;
        table[k].first = table[l].first;
        table[l].first = i;
    };
    const auto sift = [&](long long k, long long size) {   // of a heap whose root writes last
        for (long long c; (c = 2 * k + 1) < size; k = c) {
            if (c + 1 < size && before(c, c + 1)) c++;
            if (!before(k, c)) return;
            swap(k, c);
        }
    };
    for (long long k = m / 2 - 1; k >= 0; k--) sift(k, m);
    for (long long size = m - 1; size > 0; size--) {
        swap(0, size);
        sift(0, size);
    }
    for (long long k = 0; k + 1 < m; k++)
        if (written_of(entry(k)).hi > written_of(entry(k + 1)).lo) return false;
    // (what is written is apart now, so the last of it that starts before the end of what an entry reads reaches farthest)
    for (long long k = 0; k < m; k++) {
        const Bytes from = read_of(entry(k));
        long long lo = 0, hi = m;
        while (lo < hi) {
            const long long mid = (lo + hi) / 2;
            if (written_of(entry(mid)).lo < from.hi) lo = mid + 1;
            else hi = mid;
        }
        if (lo > 0 && table[lo - 1].first != table[k].first && written_of(entry(lo - 1)).hi > from.lo) return false;
    }
    return true;
}

unsigned clip_groups(long long pieces)
{
    const long long most = 8ll * cu_count();   // what the chip holds at once
    return (unsigned)(pieces < 1 ? 1 : pieces < most ? pieces : most);
}

}  // namespace
}  // namespace bm

using namespace bm;

extern "C" {

int bimamba_clip_layout(bimamba_grad* table, int n)
{
    long long pieces;
    const int rc = clip_pieces(table, table, n, &pieces);
    if (rc) return rc;
    return clip_apart(table, n) ? clip_pieces(table, table, n, &pieces) : BIMAMBA_ERR_ALIAS;
}

size_t bimamba_clip_grads_workspace_bytes(const bimamba_grad* table, int n)
{
    long long pieces;
    return clip_pieces(table, nullptr, n, &pieces) ? 0 : clip_groups(pieces) * sizeof(double);
}

int bimamba_clip_grads(const bimamba_grad* table, int n, const void* table_dev, float max_norm, float* norm, void* workspace,
                       size_t workspace_bytes, void* hip_stream)
{
    long long pieces, bytes;
    int rc = clip_pieces(table, nullptr, n, &pieces, &bytes);
    if (rc) return rc;
    if (!(max_norm >= 0.0f)) return BIMAMBA_ERR_BAD_SHAPE;
    if (n > 0 && !table_dev) return BIMAMBA_ERR_NULL_POINTER;
    if (!aligned_to(table_dev, 8) || !aligned_to(norm, 4)) return BIMAMBA_ERR_MISALIGNED;
    const unsigned groups = clip_groups(pieces);
    if ((rc = check_workspace(workspace, workspace_bytes, groups * sizeof(double)))) return rc;
    const Bytes value = bytes_of(norm, 1, 4), ws = bytes_of(workspace, groups, sizeof(double)), dev = bytes_of(table_dev, n, sizeof(bimamba_grad));
    if (meet(value, ws) || meet(value, dev) || meet(ws, dev)) return BIMAMBA_ERR_ALIAS;
    for (int i = 0; i < n; i++) {
        if (table[i].count == 0) continue;
        const Bytes from = read_of(table[i]), to = written_of(table[i]);
        if (meet(value, from) || meet(value, to) || meet(ws, from) || meet(ws, to) || meet(dev, to)) return BIMAMBA_ERR_ALIAS;
    }
    const long long past = past_caches(2.0 * bytes) && bytes > kKept ? (long long)((double)pieces * (bytes - kKept) / bytes) : 0;
    const ClipArgs a{static_cast<const bimamba_grad*>(table_dev), pieces, past, n, max_norm, norm, static_cast<double*>(workspace)};
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    hipLaunchKernelGGL(clip_squares_kernel, dim3(groups), dim3(kClipThreads), 0, st, a);
    if (past_caches(2.0 * bytes)) hipLaunchKernelGGL(clip_scale_kernel<true>, dim3(groups), dim3(kClipThreads), 0, st, a);
    else hipLaunchKernelGGL(clip_scale_kernel<false>, dim3(groups), dim3(kClipThreads), 0, st, a);
    return launches.status();
}

}  // extern "C"
