// The norm of groups of channels with an activation or a gate, and its gradients: checks, plan and entry points.
#include "group_norm.h"
#include "slot_sums.h"

namespace bm {
template <> void launch_group_norm<BIMAMBA_ACT_NONE>(const GroupPlan&, const GroupNormArgs&, bool, bool, bool, hipStream_t);
template <> void launch_group_norm<BIMAMBA_ACT_SILU>(const GroupPlan&, const GroupNormArgs&, bool, bool, bool, hipStream_t);
template <> void launch_group_norm<BIMAMBA_ACT_GATE_BEFORE>(const GroupPlan&, const GroupNormArgs&, bool, bool, bool, hipStream_t);
template <> void launch_group_norm<BIMAMBA_ACT_GATE_AFTER>(const GroupPlan&, const GroupNormArgs&, bool, bool, bool, hipStream_t);
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

GroupPlan plan_group_norm(const bimamba_group_norm_desc* d, bool bwd)
{
    GroupPlan p{};
    const int n = d->d_inner / d->groups, piece = d->io_dtype == BIMAMBA_BF16 ? 8 : 4;
    const int pieces = n < piece ? n : (n + piece - 1) / piece;   // (of one element in small groups)
    // 16 elements a lane at most: 32 of them and the gradients' sums take the registers of half the waves (32768 x 2 groups of 2048, gated: four
    // waves to a group 127 us, one 138; gradients 241, 262; groups of 8192: eight waves 286, four 293; gradients 501, 502; of 4096: 256,
    // 263; 478, 507)
    p.waves = n <= 1024 ? 1 : n <= 2048 ? 4 : 8;
    p.lanes = 1;
    while (p.lanes < 64 && p.lanes < pieces) p.lanes *= 2;
    p.pieces = 1;
    while (p.pieces * p.lanes * p.waves < pieces) p.pieces *= 2;
    int runs = 64 / p.lanes;   // groups of a row that a wave holds; where there are not that many it holds those of several rows
    p.at_once = 1;
    while (p.waves == 1 && runs > 1 && runs / 2 >= d->groups) runs /= 2, p.at_once *= 2;
    p.tiles = (d->groups + runs - 1) / runs;
    p.team = p.waves > 1 ? p.waves : bwd && p.pieces == 1 && p.at_once == 1 ? 8 : 4;
    // Rows: as many as are in hand at once go to one wave each, up to four where there are more (four to each wave for the gradients of shared
    // groups, which otherwise leave a slot as long as two rows for every few of them: 65536 groups of 4096 32 rows 492 us, 16 512, 8 527).
    // (Gradients divided by 3 and by 8: 2048 rows of 64 groups of 64 20.7 and 24.2 us, 16384 of 4 of 128 16.4, 21.8; 512, 8192 and 65536 rows the same.)
    const unsigned rows = (unsigned)((long long)d->batch * d->seqlen), together = (p.waves == 1 ? p.team : 1) * p.at_once;
    const unsigned long long fair = (unsigned long long)rows * p.tiles / (together * (bwd ? 3u : 16u) * cu_count()), most = bwd && p.waves > 1 ? 4 * p.waves : 4;
    p.per_wave = (unsigned)(fair < 1 ? 1 : fair > most ? most : fair);
    // (a grid's second axis ends at 65535)
    const unsigned long long least = (rows + 65535ull * together - 1) / (65535ull * together);
    if (p.per_wave < least) p.per_wave = (unsigned)least;
    const unsigned long long step = (unsigned long long)p.per_wave * together;
    p.row_groups = (unsigned)((rows + step - 1) / step);
    return p;
}

void launch(const bimamba_group_norm_desc* d, const GroupPlan& p, GroupNormArgs& a, bool bwd, hipStream_t st)
{
    a.L = d->seqlen, a.rows = (unsigned)((long long)d->batch * d->seqlen), a.per_wave = p.per_wave;
    a.G = d->groups, a.n = d->d_inner / d->groups, a.d = d->d_inner, a.lanes = p.lanes, a.at_once = p.at_once, a.centred = d->centred, a.eps = d->eps;
    const bool bf16 = d->io_dtype == BIMAMBA_BF16, past = past_caches((bwd ? 3.0 : 2.0) * a.rows * a.d * dtype_bytes(d->io_dtype));
    switch (d->act) {
        case BIMAMBA_ACT_NONE: launch_group_norm<BIMAMBA_ACT_NONE>(p, a, bf16, past, bwd, st); break;
        case BIMAMBA_ACT_SILU: launch_group_norm<BIMAMBA_ACT_SILU>(p, a, bf16, past, bwd, st); break;
        case BIMAMBA_ACT_GATE_BEFORE: launch_group_norm<BIMAMBA_ACT_GATE_BEFORE>(p, a, bf16, past, bwd, st); break;
        default: launch_group_norm<BIMAMBA_ACT_GATE_AFTER>(p, a, bf16, past, bwd, st);
    }
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
