// What the operators around the mixers share: rows moved in pieces of 16 bytes, sums over a wave, and the host's checks.
#pragma once
#include "bimamba.h"
#include "kernels.h"
#include "launch.h"

#include <hip/hip_runtime.h>

#include <cmath>

namespace bm {

// Elements that a lane moves at once: 16 bytes, so that a wave's access is one run.  (fp32 rows in pieces of eight, two accesses that each
// leave every other 16 bytes to the other, were written at 4.1 TB/s, in these pieces at 7.4.)
template <typename IO>
constexpr int kPieceOf = 16 / (int)sizeof(typename IO::T);

// Neighbouring elements of a row, at any alignment that the element type allows (the memory unit takes the bytes as they lie).
template <typename IO, int N = kPieceOf<IO>>
struct Piece {
    typename IO::T v[N];
    __device__ __forceinline__ float operator[](int i) const { return IO::cvt(v[i]); }
};
// kPast: past the caches.  For calls that move more than these hold (past_caches below): what such a call leaves there is of no use, and the
// lines it has to push out cost it time.  Stores, 65536 rows of 2048: layer norm 101 -> 97 us; gradient of 16384 rows of 50304 logits
// 492 -> 407.  Loads help where little or nothing is written beside them: log probabilities of those logits 146 -> 127 us, layer norm's
// gradients 169 -> 162; in those two 97 -> 115 and 402 -> 426, which therefore load through the caches.  (A flag at run time would not
// do: the compiler joins the two accesses and drops the difference.)
template <int kBytes>
struct PastCaches {
    typedef unsigned Bits __attribute__((ext_vector_type(kBytes / 4)));
    typedef Bits Place __attribute__((aligned(2)));   // (of either element type)
};
template <typename IO, int N = kPieceOf<IO>, bool kPast = false>
__device__ __forceinline__ Piece<IO, N> load_piece(const typename IO::T* p)
{
    Piece<IO, N> r;
    if constexpr (kPast && sizeof r >= 8) {
        typedef PastCaches<sizeof r> Past;
        const typename Past::Bits bits = __builtin_nontemporal_load(reinterpret_cast<const typename Past::Place*>(p));
        __builtin_memcpy(&r, &bits, sizeof r);
    } else {
        __builtin_memcpy(&r, p, sizeof r);
    }
    return r;
}
template <typename IO, bool kPast = false, int N>
__device__ __forceinline__ void store_piece(typename IO::T* p, const float (&f)[N])
{
    Piece<IO, N> r;
#pragma unroll
    for (int i = 0; i < N; i++) r.v[i] = io_value<IO>(f[i]);
    if constexpr (kPast && sizeof r >= 8) {
        typedef PastCaches<sizeof r> Past;
        __builtin_nontemporal_store(__builtin_bit_cast(typename Past::Bits, r), reinterpret_cast<typename Past::Place*>(p));
    } else {
        __builtin_memcpy(p, &r, sizeof r);
    }
}
// The piece of a row that starts at element `at`, which may reach beyond the row's n >= N elements, in two steps.  The load takes the last N
// elements where the piece would reach beyond, so there is no branch around it and all loads of a lane are in flight together (with
// the row's end told apart by a branch the compiler waited for each load where the two ways join: the sum of a table's
// gradient ran at 1.5 TB/s).  settle() then puts what is left of the piece in its place, and `fill` beyond the row.
template <typename IO, int N = kPieceOf<IO>, bool kPast = false>
__device__ __forceinline__ Piece<IO, N> load_clamped(const typename IO::T* row, int at, int n)
{
    return load_piece<IO, N, kPast>(row + min(at, n - N));
}
template <typename IO, int N>
__device__ __forceinline__ void settle(Piece<IO, N>& p, int at, int n, typename IO::T fill)
{
    if (at + N <= n) return;
    const int off = at - (n - N);   // places to move by; N or more: beyond the row
#pragma unroll
    for (int step = N / 2; step > 0; step /= 2) {
#pragma unroll
        for (int i = 0; i < N; i++) p.v[i] = off & step ? (i + step < N ? p.v[i + step < N ? i + step : i] : fill) : p.v[i];
    }
    if (off >= N)
#pragma unroll
        for (int i = 0; i < N; i++) p.v[i] = fill;
}
template <typename IO, int N = kPieceOf<IO>>
__device__ __forceinline__ Piece<IO, N> load_piece_of(const typename IO::T* row, int at, int n, typename IO::T fill)
{
    Piece<IO, N> r = load_clamped<IO, N>(row, at, n);
    settle(r, at, n, fill);
    return r;
}
template <typename IO, bool kPast = false, int N>
__device__ __forceinline__ void store_piece_of(typename IO::T* row, int at, int n, const float (&f)[N])
{
    if (at + N <= n) {
        store_piece<IO, kPast>(row + at, f);
    } else {
#pragma unroll
        for (int i = 0; i < N; i++)
            if (at + i < n) row[at + i] = io_value<IO>(f[i]);
    }
}
// fp32 parameters beside them, in elements [at, at + N) of n >= N.
template <int N>
__device__ __forceinline__ void load_floats(float (&f)[N], const float* row, int at, int n, float fill)
{
    const Piece<IoF32, N> p = load_piece_of<IoF32, N>(row, at, n, fill);
#pragma unroll
    for (int i = 0; i < N; i++) f[i] = p[i];
}

// A value combined over the 64 lanes, the same in all of them: lane permutes within a row of sixteen, then the swaps between rows.
template <typename Op>
__device__ __forceinline__ float wave_combine(float v, Op op)
{
#define BM_DPP(ctrl) __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, 0xf, 0xf, true))
    v = op(v, BM_DPP(0xB1));    // quad_perm 1 0 3 2
    v = op(v, BM_DPP(0x4E));    // quad_perm 2 3 0 1
    v = op(v, BM_DPP(0x141));   // row_half_mirror
    v = op(v, BM_DPP(0x140));   // row_mirror
#undef BM_DPP
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float wave_sum(float v)
{
    return wave_combine(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v)
{
    return wave_combine(v, [](float a, float b) { return fmaxf(a, b); });
}

// Rows of a view, in elements.
struct RowView {
    void* p;
    long long sb, st;
};
__device__ __forceinline__ long long row_offset(const RowView& v, int b, int t) { return b * v.sb + t * v.st; }

// ---- host ----

constexpr long long kMaxRows = (1ll << 31) - 1;
// Whether a call moves more bytes than the last cache before the memory holds.
inline bool past_caches(double bytes) { return bytes > (double)(256ll << 20); }

inline RowView row_view(const bimamba_tensor* t) { return RowView{t->ptr, t->stride_batch, t->stride_token}; }
inline bool known_dtype(int d) { return d == BIMAMBA_F32 || d == BIMAMBA_BF16; }
inline size_t dtype_bytes(int d) { return d == BIMAMBA_BF16 ? 2 : 4; }
inline bool aligned_to(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// Bytes [lo, hi) that rows of `width` elements span.  False: strides are negative or the span does not fit an address.
struct Bytes {
    uintptr_t lo, hi;
};
inline bool bytes_of(const void* p, long long sb, long long st, int batch, int seqlen, long long width, size_t elem, Bytes* r)
{
    if (sb < 0 || st < 0) return false;
    const __int128 last = (__int128)(batch - 1) * sb + (__int128)(seqlen - 1) * st + width;
    const __int128 hi = (__int128)reinterpret_cast<uintptr_t>(p) + last * (__int128)elem;
    if (hi > (__int128)1 << 62) return false;
    *r = Bytes{reinterpret_cast<uintptr_t>(p), (uintptr_t)hi};
    return true;
}
inline Bytes bytes_of(const void* p, long long count, size_t elem)
{
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    return Bytes{lo, p ? lo + (uintptr_t)count * elem : lo};
}
inline bool meet(const Bytes& a, const Bytes& b) { return a.lo < b.hi && b.lo < a.hi; }

// Whether rows that are written keep apart from each other: the inner of the two strides holds a row, the outer all of the inner's.
inline bool rows_apart(const bimamba_tensor* t, int batch, int seqlen, long long width)
{
    long long inner = t->stride_token, outer = t->stride_batch, n_inner = seqlen, n_outer = batch;
    if (n_outer > 1 && n_inner > 1 && outer < inner) {
        const long long s = inner, n = n_inner;
        inner = outer, n_inner = n_outer;
        outer = s, n_outer = n;
    }
    if (n_inner > 1 && inner < width) return false;
    return n_outer <= 1 || (__int128)outer >= (__int128)(n_inner - 1) * (n_inner > 1 ? inner : 0) + width;
}

// Whether writing rows of `a` could touch rows of `b`: byte ranges apart never do; nor do column ranges apart of one buffer whose
// rows both views step through alike.
inline bool views_meet(const bimamba_tensor* a, long long wa, const Bytes& ba, const bimamba_tensor* b, long long wb, const Bytes& bb,
                       int batch, size_t elem_a, size_t elem_b)
{
    if (!meet(ba, bb)) return false;
    const long long pitch = a->stride_token;
    if (elem_a == elem_b && pitch == b->stride_token && pitch > 0 && (batch <= 1 || (a->stride_batch == b->stride_batch && a->stride_batch % pitch == 0))) {
        const long long delta = ((long long)ba.lo - (long long)bb.lo) / (long long)elem_a;
        const long long r = ((delta % pitch) + pitch) % pitch;   // a's first column, counted from b's first column
        if (r >= wb && r + wa <= pitch) return false;
    }
    return true;
}

// A view of [batch, seqlen, width] elements of a type, none of them empty.
inline int check_view(const bimamba_tensor* t, int batch, int seqlen, long long width, int dtype, bool written, Bytes* r)
{
    if (!t->ptr) return BIMAMBA_ERR_NULL_POINTER;
    if (!bytes_of(t->ptr, t->stride_batch, t->stride_token, batch, seqlen, width, dtype_bytes(dtype), r)) return BIMAMBA_ERR_BAD_SHAPE;
    if (!aligned_to(t->ptr, dtype_bytes(dtype))) return BIMAMBA_ERR_MISALIGNED;
    if (written && !rows_apart(t, batch, seqlen, width)) return BIMAMBA_ERR_BAD_SHAPE;
    return BIMAMBA_OK;
}
inline int check_tokens(const bimamba_tokens* t, int batch, int seqlen, Bytes* r)
{
    if (!t->ptr) return BIMAMBA_ERR_NULL_POINTER;
    if (!bytes_of(t->ptr, t->stride_batch, t->stride_token, batch, seqlen, 1, 8, r)) return BIMAMBA_ERR_BAD_SHAPE;
    return aligned_to(t->ptr, 8) ? BIMAMBA_OK : BIMAMBA_ERR_MISALIGNED;
}
inline int check_rows(int batch, int seqlen)
{
    if (batch < 0 || seqlen < 0) return BIMAMBA_ERR_BAD_SHAPE;
    return (long long)batch * seqlen > kMaxRows ? BIMAMBA_ERR_UNSUPPORTED : BIMAMBA_OK;
}
inline int check_workspace(const void* p, size_t have, size_t need)
{
    if (need == 0) return BIMAMBA_OK;
    if (!p) return BIMAMBA_ERR_NULL_POINTER;
    if (!aligned_to(p, 16)) return BIMAMBA_ERR_MISALIGNED;
    return have < need ? BIMAMBA_ERR_WORKSPACE_TOO_SMALL : BIMAMBA_OK;
}

// The status of the launches made since: an error that some earlier, unrelated call left behind is not theirs.
class Launches {
public:
    int status() const
    {
        const hipError_t now = hipPeekAtLastError();
        return now == hipSuccess || now == pending_ ? BIMAMBA_OK : BIMAMBA_ERR_HIP;
    }

private:
    hipError_t pending_ = hipPeekAtLastError();
};

}  // namespace bm
