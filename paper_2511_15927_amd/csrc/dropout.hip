// Dropout into the residual stream: residual + gate * dropout(x), its mask made from a counter wherever it is needed, and its gradients.
#include "slot_sums.h"

namespace bm {

// Philox4x32 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, 2011), ten rounds: four words from a counter.  One
// counter serves eight neighbouring channels, 16 bits each.
struct Words {
    unsigned w[4];
};
__device__ __forceinline__ Words philox(unsigned c0, unsigned c1, unsigned c2, unsigned c3, unsigned k0, unsigned k1)
{
#pragma unroll
    for (int i = 0; i < 10; i++) {
        const unsigned long long p0 = (unsigned long long)c0 * 0xD2511F53u, p1 = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (unsigned)(p1 >> 32) ^ c1 ^ k0;
        c1 = (unsigned)p1;
        c2 = (unsigned)(p0 >> 32) ^ c3 ^ k1;
        c3 = (unsigned)p0;
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
    return Words{{c0, c1, c2, c3}};
}

constexpr int kTeam = 4;   // waves of a workgroup

struct DropArgs {
    RowView x, residual, out;   // residual.p null: none; gradients: x (null: no dgate), dout, dx
    const int64_t* key;
    const float* gate;          // null: 1
    long long gate_stride;
    float* dgate;               // sums of a row group, null: not wanted
    long long slot;
    unsigned L, rows, per_wave; // rows that share a vector; steps that a wave takes
    int per_batch, d, lanes;    // lanes that hold a row, or 64 of a longer one
    unsigned site, threshold;   // site * 2^17
    float scale;
};
__device__ __forceinline__ unsigned half_of(const Words& r, int i) { return (r.w[i >> 1] >> (i & 1 ? 16 : 0)) & 0xffffu; }

// A lane has one piece of 16 bytes of a row in hand; with short rows a wave takes several at once.  What bounds it are the bytes, with the
// generator close behind them: where all lanes hold a piece the vector pipe is busy 88 % of the time, 82 % in the gradients (65536 rows of 2048 bf16
// with a residual and a gate: 126 to 131 us, 6.3 TB/s, at p = 0.1 and, without the generator, 124 at p = 0; a large copy reaches 6.1).  Lanes that
// hold nothing run the generator all the same, so at widths that are not 2^k pieces, or a little more than 64 of them, it is what
// bounds it: 262144 rows of 512 122 us (6.6 TB/s), of 520 206 (4.0), of 640 208 (4.8), of 768 226 (5.3), of 384 116 (5.2), of 320 110 (4.6).
// A wave takes two rows and goes, eight for the gate's gradient, so that all waves in hand
// work on neighbouring rows: 1 row 156 us, 8 rows 140, 32 rows 165; gradients with 8 rows 134 us, 2 rows 145, 32 rows 172.
template <typename IO, int kPiece>
struct DropPlace {
    int at, run;              // the lane's first channel; its row among those that the wave takes at once
    unsigned vector, r0, step, steps;
    bool real;
    __device__ __forceinline__ DropPlace(const DropArgs& a)
    {
        const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        run = lane / a.lanes;
        at = (blockIdx.x * a.lanes + lane % a.lanes) * kPiece;
        vector = blockIdx.z;
        step = 64 / a.lanes;
        r0 = (blockIdx.y * kTeam + wave) * a.per_wave * step;
        steps = r0 < a.rows ? min((unsigned)a.per_wave, (a.rows - r0 + step - 1) / step) : 0;
        real = at < a.d;
    }
};
struct DropRow {
    unsigned b, t, all;
    bool real;
};
__device__ __forceinline__ DropRow drop_row(const DropArgs& a, unsigned vector, unsigned r)
{
    const bool real = r < a.rows;
    r = min(r, a.rows - 1);
    if (a.per_batch) return DropRow{vector, r, vector * a.L + r, real};
    const unsigned b = r / a.L;
    return DropRow{b, r - b * a.L, r, real};
}
template <int kPiece>
__device__ __forceinline__ void kept_of(float (&keep)[kPiece], const DropArgs& a, unsigned row, int at, unsigned k0, unsigned k1, unsigned o0, unsigned o1)
{
    if (a.threshold == 0) {
#pragma unroll
        for (int i = 0; i < kPiece; i++) keep[i] = 1.0f;
        return;
    }
    const Words r = philox(row, (unsigned)(at >> 3) + a.site, o0, o1, k0, k1);
#pragma unroll
    for (int i = 0; i < kPiece; i++) {
        unsigned half;
        if constexpr (kPiece == 8) half = half_of(r, i);
        else if constexpr (kPiece == 4) half = (at & 4) ? half_of(r, 4 + i) : half_of(r, i);
        else {
            const int c = at & 7;
            const unsigned lo = c & 2 ? r.w[1] : r.w[0], hi = c & 2 ? r.w[3] : r.w[2], w = c & 4 ? hi : lo;
            half = c & 1 ? w >> 16 : w & 0xffffu;
        }
        keep[i] = half >= a.threshold ? a.scale : 0.0f;
    }
}

template <typename IO, int kPiece, bool kBack, bool kPast>
__device__ __forceinline__ void drop_rows(const DropArgs& a)
{
    const DropPlace<IO, kPiece> place(a);
    const unsigned long long seed = (unsigned long long)a.key[0], offset = (unsigned long long)a.key[1];
    const unsigned k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32), o0 = (unsigned)offset, o1 = (unsigned)(offset >> 32);
    const int at = min(place.at, a.d - kPiece);   // (the row's last piece is taken whole and moved into place)
    float gate[kPiece], sum[kPiece];
    const bool whole = a.d % kPiece == 0;
#pragma unroll
    for (int i = 0; i < kPiece; i++) gate[i] = 1.0f, sum[i] = 0.0f;
    if (a.gate) load_floats(gate, a.gate + place.vector * a.gate_stride, place.at, a.d, 0.0f);
    const bool wants_x = !kBack || a.x.p, wants_r = kBack || a.residual.p;
    for (unsigned s = 0; s < place.steps; s++) {
        const DropRow row = drop_row(a, place.vector, place.r0 + s * place.step + place.run);
        Piece<IO, kPiece> px{}, pr{};
        if (wants_x) px = load_piece<IO, kPiece, kPast>(static_cast<const typename IO::T*>(a.x.p) + row_offset(a.x, row.b, row.t) + at);
        if (wants_r) pr = load_piece<IO, kPiece, kPast>(static_cast<const typename IO::T*>(a.residual.p) + row_offset(a.residual, row.b, row.t) + at);
        float keep[kPiece], f[kPiece];
        kept_of(keep, a, row.all, place.at, k0, k1, o0, o1);
        if (!whole) {
            settle(px, place.at, a.d, typename IO::T(0));
            settle(pr, place.at, a.d, typename IO::T(0));
        }
#pragma unroll
        for (int i = 0; i < kPiece; i++) {
            if constexpr (kBack) {
                const float d = keep[i] > 0.0f ? pr[i] * keep[i] : 0.0f;
                f[i] = d * gate[i];
                if (row.real) sum[i] += keep[i] > 0.0f ? d * px[i] : 0.0f;
            } else {
                f[i] = (keep[i] > 0.0f ? px[i] * (keep[i] * gate[i]) : 0.0f) + pr[i];
            }
        }
        if (row.real && place.real) {
            typename IO::T* const to = static_cast<typename IO::T*>(a.out.p) + row_offset(a.out, row.b, row.t);
            if (whole) store_piece<IO, kPast>(to + place.at, f);
            else store_piece_of<IO, kPast>(to, place.at, a.d, f);
        }
    }
    if constexpr (kBack) {
        if (!a.dgate) return;   // (all threads)
        // the rows that a wave took at once, then the four waves
        __shared__ float all[kTeam][kPiece][64];
#pragma unroll
        for (int i = 0; i < kPiece; i++) all[threadIdx.x / 64][i][threadIdx.x % 64] = sum[i];
        __syncthreads();
        if ((int)threadIdx.x >= a.lanes || !place.real) return;
#pragma unroll
        for (int i = 0; i < kPiece; i++) sum[i] = 0.0f;
        for (int w = 0; w < kTeam; w++)
            for (int l = threadIdx.x; l < 64; l += a.lanes)
#pragma unroll
                for (int i = 0; i < kPiece; i++) sum[i] += all[w][i][l];
        store_piece_of<IoF32>(a.dgate + ((long long)place.vector * gridDim.y + blockIdx.y) * a.slot, place.at, a.d, sum);
    }
}
template <typename IO, bool kBack, bool kPast>
__global__ __launch_bounds__(64 * kTeam) void drop_kernel(const DropArgs a)
{
    if (a.d < kPieceOf<IO>) return drop_rows<IO, 1, kBack, kPast>(a);
    drop_rows<IO, kPieceOf<IO>, kBack, kPast>(a);
}

namespace {

int check_dropout(const bimamba_dropout_desc* d)
{
    if (!d) return BIMAMBA_ERR_NULL_POINTER;
    if (d->struct_size != sizeof(bimamba_dropout_desc) || d->d_model < 1) return BIMAMBA_ERR_BAD_SHAPE;
    if (!(d->p >= 0.0f && d->p <= 1.0f)) return BIMAMBA_ERR_BAD_SHAPE;
    if (const int rc = check_rows(d->batch, d->seqlen)) return rc;
    if (!known_dtype(d->io_dtype) || d->batch > 65535 || d->d_model > 1 << 20 || d->site < 0 || d->site >= 1 << 15) return BIMAMBA_ERR_UNSUPPORTED;
    return BIMAMBA_OK;
}

struct DropPlan {
    int lanes;
    unsigned tiles, vectors, row_groups, per_wave, rows;
};
DropPlan plan_dropout(const bimamba_dropout_desc* d, bool per_batch, bool sums)
{
    DropPlan p{};
    const int piece = d->io_dtype == BIMAMBA_BF16 ? 8 : 4, pieces = d->d_model < piece ? d->d_model : (d->d_model + piece - 1) / piece;
    p.lanes = 1;
    while (p.lanes < 64 && p.lanes < pieces) p.lanes *= 2;
    p.tiles = (pieces + p.lanes - 1) / p.lanes;
    p.vectors = per_batch ? d->batch : 1;
    p.rows = per_batch ? d->seqlen : (unsigned)((long long)d->batch * d->seqlen);
    // Rows: as many as are in hand at once go to one wave each, a few more where there are more of them.  (Sums: divided by 6 and by 16, gradients of 4096
    // rows of 2048 14.1 and 16.6 us, of 16384 of 512 16.8, 19.9; of 8192 of 2048 23.4, 22.6, of 16384 37.5, 36.3; from 65536 on and up to 2048 rows the same.)
    const unsigned together = kTeam * (64 / p.lanes), most = sums ? 8 : 2;
    const unsigned long long fair = (unsigned long long)p.rows * p.tiles * p.vectors / (together * (sums ? 6u : 16u) * cu_count());
    p.per_wave = (unsigned)(fair < 1 ? 1 : fair > most ? most : fair);
    // (a grid's second axis ends at 65535)
    const unsigned long long least = (p.rows + 65535ull * together - 1) / (65535ull * together);
    if (p.per_wave < least) p.per_wave = (unsigned)least;
    const unsigned long long step = (unsigned long long)p.per_wave * together;
    p.row_groups = (unsigned)((p.rows + step - 1) / step);
    return p;
}

template <typename IO, bool kPast>
void launch_io(const DropPlan& p, const DropArgs& a, bool back, hipStream_t st)
{
    const dim3 grid(p.tiles, p.row_groups, p.vectors), wg(64 * kTeam);
    if (back) hipLaunchKernelGGL((drop_kernel<IO, true, kPast>), grid, wg, 0, st, a);
    else hipLaunchKernelGGL((drop_kernel<IO, false, kPast>), grid, wg, 0, st, a);
}
void launch(const bimamba_dropout_desc* d, const DropPlan& p, DropArgs& a, bool per_batch, bool back, hipStream_t st)
{
    const int threshold = (int)std::floor((double)d->p * 65536.0 + 0.5);
    a.L = d->seqlen, a.rows = p.rows, a.per_wave = p.per_wave, a.per_batch = per_batch, a.d = d->d_model, a.lanes = p.lanes;
    a.site = (unsigned)d->site << 17, a.threshold = threshold, a.scale = threshold < 65536 ? 65536.0f / (65536 - threshold) : 0.0f;
    const bool past = past_caches(2.0 * d->batch * d->seqlen * d->d_model * dtype_bytes(d->io_dtype));
    if (d->io_dtype == BIMAMBA_BF16) past ? launch_io<IoBF16, true>(p, a, back, st) : launch_io<IoBF16, false>(p, a, back, st);
    else past ? launch_io<IoF32, true>(p, a, back, st) : launch_io<IoF32, false>(p, a, back, st);
}

int check_gate(const bimamba_dropout_desc* d, const float* gate, long long stride, Bytes* r)
{
    *r = Bytes{0, 0};
    if (stride != 0 && stride < d->d_model) return BIMAMBA_ERR_BAD_SHAPE;
    if (!gate || !d->batch) return BIMAMBA_OK;
    if (!aligned_to(gate, 4)) return BIMAMBA_ERR_MISALIGNED;
    return bytes_of(gate, stride, 0, d->batch, 1, d->d_model, 4, r) ? BIMAMBA_OK : BIMAMBA_ERR_BAD_SHAPE;
}
int check_key(const int64_t* key, Bytes* r)
{
    if (!key) return BIMAMBA_ERR_NULL_POINTER;
    *r = bytes_of(key, 2, 8);
    return aligned_to(key, 8) ? BIMAMBA_OK : BIMAMBA_ERR_MISALIGNED;
}
bool same_view(const bimamba_tensor* a, const bimamba_tensor* b)
{
    return a->ptr == b->ptr && a->stride_batch == b->stride_batch && a->stride_token == b->stride_token;
}

}  // namespace
}  // namespace bm

using namespace bm;

extern "C" {

int bimamba_dropout_add(const bimamba_dropout_desc* d, const int64_t* key, const bimamba_tensor* x, const float* gate,
                        int64_t gate_stride, const bimamba_tensor* residual, const bimamba_tensor* out, void* hip_stream)
{
    int rc = check_dropout(d);
    if (rc) return rc;
    if (!x || !out) return BIMAMBA_ERR_NULL_POINTER;
    Bytes bg, bk, bx, br{}, bo;
    if ((rc = check_gate(d, gate, gate_stride, &bg))) return rc;
    if (d->batch == 0 || d->seqlen == 0) return BIMAMBA_OK;
    const int Bt = d->batch, L = d->seqlen, D = d->d_model, io = d->io_dtype;
    const size_t elem = dtype_bytes(io);
    if ((rc = check_key(key, &bk)) || (rc = check_view(x, Bt, L, D, io, false, &bx)) || (residual && (rc = check_view(residual, Bt, L, D, io, false, &br))) ||
        (rc = check_view(out, Bt, L, D, io, true, &bo)))
        return rc;
    if (views_meet(out, D, bo, x, D, bx, Bt, elem, elem) || meet(bo, bg) || meet(bo, bk)) return BIMAMBA_ERR_ALIAS;
    if (residual && !same_view(residual, out) && views_meet(out, D, bo, residual, D, br, Bt, elem, elem)) return BIMAMBA_ERR_ALIAS;
    const DropPlan p = plan_dropout(d, gate && gate_stride, false);
    DropArgs a{};
    a.x = row_view(x), a.out = row_view(out);
    if (residual) a.residual = row_view(residual);
    a.key = key, a.gate = gate, a.gate_stride = gate_stride;
    const Launches launches;
    launch(d, p, a, gate && gate_stride, false, reinterpret_cast<hipStream_t>(hip_stream));
    return launches.status();
}

size_t bimamba_dropout_add_bwd_workspace_bytes(const bimamba_dropout_desc* d, int per_batch)
{
    if (check_dropout(d) || d->batch == 0 || d->seqlen == 0) return 0;
    const DropPlan p = plan_dropout(d, per_batch != 0, true);
    return p.row_groups > 1 ? (size_t)p.row_groups * p.vectors * d->d_model * sizeof(float) : 0;
}

int bimamba_dropout_add_bwd(const bimamba_dropout_desc* d, const int64_t* key, const bimamba_tensor* x, const float* gate,
                            int64_t gate_stride, const bimamba_tensor* dout, const bimamba_tensor* dx, float* dgate, void* workspace,
                            size_t workspace_bytes, void* hip_stream)
{
    int rc = check_dropout(d);
    if (rc) return rc;
    if (!dout || !dx || (dgate && !x)) return BIMAMBA_ERR_NULL_POINTER;
    Bytes bg, bk{}, bx{}, by{}, bdx{};
    if ((rc = check_gate(d, gate, gate_stride, &bg))) return rc;
    if (!aligned_to(dgate, 4)) return BIMAMBA_ERR_MISALIGNED;
    const bool rows = d->batch && d->seqlen, per_batch = gate_stride != 0;
    const int Bt = d->batch, L = d->seqlen, D = d->d_model, io = d->io_dtype;
    const size_t elem = dtype_bytes(io), need = rows && dgate ? bimamba_dropout_add_bwd_workspace_bytes(d, per_batch) : 0;
    const int vectors = per_batch ? Bt : 1;
    if (rows) {
        if ((rc = check_key(key, &bk)) || (dgate && (rc = check_view(x, Bt, L, D, io, false, &bx))) ||
            (rc = check_view(dout, Bt, L, D, io, false, &by)) || (rc = check_view(dx, Bt, L, D, io, true, &bdx)) ||
            (rc = check_workspace(workspace, workspace_bytes, need)))
            return rc;
        if (!same_view(dx, dout) && views_meet(dx, D, bdx, dout, D, by, Bt, elem, elem)) return BIMAMBA_ERR_ALIAS;
        if (dgate && views_meet(dx, D, bdx, x, D, bx, Bt, elem, elem)) return BIMAMBA_ERR_ALIAS;
    }
    const Bytes ws = bytes_of(need ? workspace : nullptr, need, 1), bdg = bytes_of(dgate, (long long)vectors * D, 4);
    const Bytes written[] = {bdx, ws, bdg}, read[] = {bg, bk, bx, by};
    for (int i = 0; i < 3; i++) {
        for (int j = 0; j < (i == 0 ? 2 : 4); j++)
            if (meet(written[i], read[j])) return BIMAMBA_ERR_ALIAS;
        for (int j = 0; j < i; j++)
            if (meet(written[i], written[j])) return BIMAMBA_ERR_ALIAS;
    }
    if (vectors == 0 || (!rows && !dgate)) return BIMAMBA_OK;
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    const DropPlan p = rows ? plan_dropout(d, per_batch, dgate != nullptr) : DropPlan{};
    const bool direct = rows && p.row_groups == 1;
    float* const slots = static_cast<float*>(workspace);
    if (rows) {
        DropArgs a{};
        if (dgate) a.x = row_view(x);
        a.residual = row_view(dout), a.out = row_view(dx);
        a.key = key, a.gate = gate, a.gate_stride = gate_stride;
        a.dgate = dgate ? direct ? dgate : slots : nullptr;
        a.slot = D;
        launch(d, p, a, per_batch, true, st);
    }
    if (dgate && !direct) launch_slot_sum(SlotSumArgs{{slots, nullptr}, {dgate, nullptr}, p.row_groups, D, D}, vectors, st);
    return launches.status();
}

}  // extern "C"
