"""The calls around the mixers where they take other forms: more than 256 MB moved (loads and stores past the caches), many rows or pieces
to a workgroup.  Odd widths, column slices that start anywhere, both types; against 64-bit implementations on the GPU and against the
same rows in calls below the border.  Bounds as in test_gpu_model_ops."""
import math

import pytest
import torch

from test_gpu_model_ops import TYPES, U32, UBF, assert_scores, norm_bwd_ref, norm_ref, scores, scores_bwd_ref, scores_ref, workspace

pytestmark = pytest.mark.gpu

CACHES = 256 << 20


@pytest.fixture(scope="module")
def bd():
    from paper_2511_15927_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return binding


@pytest.fixture(autouse=True)
def empty_afterwards():
    yield
    torch.cuda.empty_cache()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, scale=1.0, io="f32"):
    return (scale * torch.randn(*shape, generator=g, device="cuda")).to(TYPES[io])


def sliced(batch, seqlen, width, io, lead=1, extra=3):
    """(a buffer of NaN, a column slice of it)"""
    buf = torch.full((batch, seqlen, width + extra), math.nan, dtype=TYPES[io], device="cuda")
    return buf, buf[..., lead:lead + width]


def as_slice(t, io, lead=1, extra=3):
    v = sliced(*t.shape, io, lead, extra)[1]
    v.copy_(t)
    return v


def untouched(buf, width, lead=1):
    assert bool(torch.isnan(buf[..., :lead]).all()) and bool(torch.isnan(buf[..., lead + width:]).all())


def within(got, ref, bound, io="f32"):
    got = got.double()
    bound = bound + (UBF * ref.abs() if io == "bf16" else 0.0) + 1e-38
    bad = ~((got - ref).abs() <= bound)
    assert got.shape == ref.shape and not bool(bad.any()), "%d of %d beyond the bound, worst %.3g times it" % (
        int(bad.sum()), bad.numel(), float(((got - ref).abs() / bound)[bad].nan_to_num(nan=math.inf).max()))


def rows_beyond(bytes_a_row, batch=3):
    """Tokens of a sequence, so that `batch` of them move a little more than the caches hold."""
    return CACHES // bytes_a_row // batch + 5


SIZE = {"f32": 4, "bf16": 2}


@pytest.mark.parametrize("table", ["f32", "bf16"])
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("d", [3, 1237, 70001])
def test_embed_rows(bd, d, io, table):
    L, V, g = rows_beyond(d * (SIZE[io] + SIZE[table])), 211, gen(d)
    tab = normal(g, V, d, io=table)
    tok = torch.randint(-2, V + 2, (3, L), generator=g, device="cuda")
    buf, out = sliced(3, L, d, io)
    bd.bimamba_embed(bd.make_embed_desc(3, L, d, V, table=table, io=io, scale=1.7), tok, tab, out)
    known = (tok >= 0) & (tok < V)
    scaled = torch.cat([tab.float() * torch.tensor(1.7).cuda(), torch.zeros(1, d, device="cuda")]).to(TYPES[io])
    assert torch.equal(out, scaled[torch.where(known, tok, V)])
    untouched(buf, d)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("seqlen,d,vocab", [(7301, 741, 80001), (1201, 2051, 40003), (23000001, 3, 1000003), (62003, 700, 3001)])
def test_embed_gradient(bd, seqlen, d, vocab, io):
    batch = 3 if seqlen < 1 << 20 else 2 if io == "bf16" else 1
    assert 4 * vocab * d + batch * seqlen * d * SIZE[io] > CACHES
    g = gen(d)
    tok = torch.randint(-1, vocab + 1, (batch, seqlen), generator=g, device="cuda")
    tok[torch.rand(batch, seqlen, generator=g, device="cuda") < 0.5] = vocab - 1
    dout = as_slice(normal(g, batch, seqlen, d, io=io), io)
    desc = bd.make_embed_desc(batch, seqlen, d, vocab, io=io, scale=0.75)
    buf = torch.full((vocab + 2, d), math.nan, device="cuda")
    ws = workspace(bd.bimamba_embed_bwd_workspace_bytes(desc))
    bd.bimamba_embed_bwd(desc, tok, dout, buf[1:-1], ws)
    assert bool(torch.isnan(buf[0]).all()) and bool(torch.isnan(buf[-1]).all())
    first = buf[1:-1].clone()
    bd.bimamba_embed_bwd(desc, tok, dout, buf[1:-1], ws)
    assert torch.equal(buf[1:-1], first)
    at, rows = torch.where((tok >= 0) & (tok < vocab), tok, vocab).reshape(-1), dout.double().reshape(-1, d)
    # (the mask's rows are added up by themselves: 64-bit atomics on one row would take long)
    masked = at == vocab - 1
    sums = torch.zeros(2, vocab + 1, d, dtype=torch.float64, device="cuda")
    for k, r in enumerate((rows, rows.abs())):
        sums[k].index_add_(0, at[~masked], r[~masked])
        sums[k, vocab - 1] = r[masked].sum(0)
    count = torch.bincount(at, minlength=vocab + 1)[:vocab].double()
    chain = count.clamp(max=64.0) + count / 8 + 12
    within(first, 0.75 * sums[0, :vocab], chain[:, None] * U32 * 0.75 * sums[1, :vocab])


NORM_WIDTHS = [("f32", 3), ("f32", 509), ("f32", 1021), ("f32", 2045), ("f32", 4093), ("f32", 8189), ("f32", 9001),
               ("bf16", 7), ("bf16", 509), ("bf16", 1023), ("bf16", 2041), ("bf16", 4095), ("bf16", 8191), ("bf16", 9001)]


@pytest.mark.parametrize("per_batch", [False, True])
@pytest.mark.parametrize("io,d", NORM_WIDTHS)
def test_layer_norm(bd, io, d, per_batch):
    L, g, eps = rows_beyond(2 * d * SIZE[io]), gen(d), 1e-5
    x = as_slice(2 * normal(g, 3, L, d) + 1, io, lead=2)
    rows = (3,) if per_batch else ()
    w, b = 1 + normal(g, *rows, d, scale=0.3), normal(g, *rows, d, scale=0.3)
    buf, y = sliced(3, L, d, io)
    mean, rstd = torch.full((2, 3, L), math.nan, device="cuda")
    desc = bd.make_norm_desc(3, L, d, io=io, eps=eps)
    bd.bimamba_layer_norm(desc, x, w, b, y, mean, rstd)
    untouched(buf, d)
    ry, rmean, rrstd, hat, rw, _ = norm_ref(x, w, b, eps)
    chain = 48 + d / 1024
    size = x.double().abs().mean(-1, keepdim=True)
    off_mean = chain * U32 * size
    off_hat = off_mean * rrstd + U32 * (4 + chain) * hat.abs() + U32 * x.double().abs() * rrstd
    off_rstd = (chain + 6) * U32 * rrstd + (off_mean * rrstd) ** 2 * rrstd + U32 * size * rrstd * rrstd
    within(mean, rmean[..., 0], off_mean[..., 0] + U32 * rmean[..., 0].abs())
    within(rstd, rrstd[..., 0], off_rstd[..., 0])
    within(y, ry, (off_hat + off_rstd / rrstd * hat.abs()) * rw.abs() + 3 * U32 * (ry.abs() + (hat * rw).abs()), io)
    # rows at the beginning, in the middle and at the end, 1100 at a time (as many as take the same form, one to a group of waves)
    n = min(1100, L)
    few = bd.make_norm_desc(1, n, d, io=io, eps=eps)
    for e, t in ((0, 0), (1, (L - n) // 2), (2, L - n)):
        part = torch.empty(1, n, d, dtype=TYPES[io], device="cuda")
        stats = torch.empty(2, 1, n, device="cuda")
        bd.bimamba_layer_norm(few, x[e:e + 1, t:t + n], w[e] if per_batch else w, b[e] if per_batch else b, part, stats[0], stats[1])
        assert torch.equal(part[0], y[e, t:t + n]) and torch.equal(stats[0, 0], mean[e, t:t + n]) and torch.equal(stats[1, 0], rstd[e, t:t + n])


@pytest.mark.parametrize("per_batch", [False, True])
@pytest.mark.parametrize("io,d", NORM_WIDTHS)
def test_layer_norm_gradient(bd, io, d, per_batch):
    L, g = rows_beyond(3 * d * SIZE[io]), gen(d + 1)
    x, dy = as_slice(2 * normal(g, 3, L, d) + 1, io, lead=2), as_slice(normal(g, 3, L, d), io, lead=3)
    w = 1 + normal(g, *((3,) if per_batch else ()), d, scale=0.3)
    _, mean, rstd, _, _, _ = norm_ref(x, w, None, 1e-5)
    mean, rstd = mean[..., 0].float(), rstd[..., 0].float()
    buf, dx = sliced(3, L, d, io)
    dw, db = torch.full((2, *w.shape), math.nan, device="cuda")
    desc = bd.make_norm_desc(3, L, d, io=io)
    bd.bimamba_layer_norm_bwd(desc, x, w, mean, rstd, dy, dx, dw, db, workspace(bd.bimamba_layer_norm_bwd_workspace_bytes(desc, per_batch)))
    untouched(buf, d)
    rdx, size, tw, tb = norm_bwd_ref(x, w, mean, rstd, dy)
    within(dx, rdx, (64 + d / 1024) * U32 * size, io)
    over = 1 if per_batch else (0, 1)
    # a workgroup's rows one after the other, of 512 workgroups or more; then their slots, 32 or more side by side
    chain = L * 3 / 512 + 200
    within(dw, tw.sum(over), chain * U32 * tw.abs().sum(over))
    within(db, tb.sum(over), chain * U32 * tb.abs().sum(over))
    n = min(1100, L)
    few = bd.make_norm_desc(1, n, d, io=io)
    for e, t in ((0, 0), (1, (L - n) // 2), (2, L - n)):
        part = torch.empty(1, n, d, dtype=TYPES[io], device="cuda")
        cut = [v[e:e + 1, t:t + n] for v in (x, mean, rstd, dy)]
        bd.bimamba_layer_norm_bwd(few, cut[0], w[e] if per_batch else w, cut[1], cut[2], cut[3], part, None, None, None)
        assert torch.equal(part[0], dx[e, t:t + n])


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("form", ["loss", "entropy", "alternatives", "both"])
@pytest.mark.parametrize("V", [9, 1237, 50257, 300001])
def test_scores(bd, V, form, io):
    L, g, k = rows_beyond(V * SIZE[io]), gen(V), 5 if form in ("alternatives", "both") else 0
    x = as_slice(normal(g, 3, L, V, scale=3.0), io, lead=2)
    x[1, ::3, V // 2:] = -math.inf
    x[2, L - 1] = -math.inf
    x[0, 1, V - 1] = math.nan
    targets = torch.randint(0, V, (3, L), generator=g, device="cuda")
    targets[torch.rand(3, L, generator=g, device="cuda") < 0.3] = -1
    want = ("logp", "lse", "entropy") if form in ("entropy", "both") else ("logp", "lse")
    got = scores(bd, x, targets, k, want=want)
    ref, spread = scores_ref(x, targets, max(k, 1))
    ref, spread = {n: t.cpu() for n, t in ref.items()}, torch.nan_to_num(spread.cpu())
    assert_scores(got, ref, spread, V)
    some = scores(bd, x, targets, k, targets_only=1, want=want)
    has = targets >= 0
    for n, t in got.items():
        assert torch.equal(some[n][has].nan_to_num(nan=7.0) if t.is_floating_point() else some[n][has], t[has].nan_to_num(nan=7.0) if t.is_floating_point() else t[has]), n
        assert bool((some[n][~has] == (-1 if n == "top_token" else 0)).all()), n


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("with_entropy", [False, True])
@pytest.mark.parametrize("V", [3, 7, 1237, 8193, 50257])
def test_scores_gradient(bd, V, with_entropy, io):
    L, g = rows_beyond(2 * V * SIZE[io]), gen(V + 1)
    x = as_slice(normal(g, 3, L, V, scale=3.0), io, lead=2)
    x[1, ::3, V // 2:] = -math.inf
    x[2, L - 1] = -math.inf
    targets = torch.randint(0, V, (3, L), generator=g, device="cuda")
    targets[torch.rand(3, L, generator=g, device="cuda") < 0.3] = -1
    ref, _ = scores_ref(x, targets, 1)
    lse, entropy = ref["lse"].float(), ref["entropy"].float()
    dlogp, dentropy = normal(g, 3, L), normal(g, 3, L) if with_entropy else None
    buf, out = sliced(3, L, V, io)
    args = bd.make_logits_desc(3, L, V, io=io), x, targets, lse, entropy if with_entropy else None, dlogp, dentropy
    bd.bimamba_log_probs_bwd(*args, out)
    untouched(buf, V)
    want, size = scores_bwd_ref(x, targets, lse, entropy, dlogp, dentropy)
    within(out, want, 8 * U32 * size, io)
    bd.bimamba_log_probs_bwd(*args, x)   # in place of the logits
    assert torch.equal(x, out)


@pytest.mark.parametrize("place", ["apart", "in place"])
@pytest.mark.parametrize("max_norm", [1.0, 1e9])
@pytest.mark.parametrize("counts", [(13,) * 5000, (70001, 3, 0, 8192, 8193) * 250, (190001,) * 250, (300001, 5) * 250, (90_000_001,)])
def test_clip(bd, counts, max_norm, place):
    """Many tensors; more pieces than workgroups; below the border, above it, and so far above that part of the first read goes past the
    caches as well.  Tensors one element off their alignment, of both types, side by side."""
    g = gen(len(counts))
    kinds = ["bf16" if i % 3 == 2 else "f32" for i in range(len(counts))]
    total = sum(n * SIZE[k] for n, k in zip(counts, kinds))
    assert total * 2 > CACHES or len(counts) != 250
    flat = {k: normal(g, 1 + sum(n for n, q in zip(counts, kinds) if q == k), io=k) for k in SIZE}
    grads, at = [], dict.fromkeys(SIZE, 1)
    for n, k in zip(counts, kinds):
        grads.append(flat[k][at[k]:at[k] + n])
        at[k] += n
    kept = {k: t.clone() for k, t in flat.items()}
    to_flat = flat if place == "in place" else {k: torch.full_like(t, math.nan) for k, t in flat.items()}
    to, at = [], dict.fromkeys(SIZE, 1)
    for n, k in zip(counts, kinds):
        to.append(to_flat[k][at[k]:at[k] + n])
        at[k] += n
    table = bd.GradTable(grads, to)
    norm = torch.full((1,), math.nan, device="cuda")
    bd.bimamba_clip_grads(table, max_norm, norm, workspace(bd.bimamba_clip_grads_workspace_bytes(table)))
    ref = math.sqrt(sum(float(t[1:].double().square().sum()) for t in kept.values()))
    assert abs(float(norm) - ref) <= 2 * U32 * ref
    factor = min(1.0, max_norm / ref)
    for k, t in to_flat.items():
        if place == "apart":
            assert bool(torch.isnan(t[:1]).all())
        else:
            assert torch.equal(t[:1], kept[k][:1])
        if factor == 1.0:
            assert torch.equal(t[1:], kept[k][1:])
        else:
            within(t[1:], kept[k][1:].double() * factor, 4 * U32 * kept[k][1:].double().abs() * factor, k)
