"""What stands around the mixers (token table, layer norm, log probabilities, clipped gradients) through the C ABI, against plain
64-bit implementations on the CPU.

Bounds are elementwise: u is the unit roundoff (2^-24 for fp32, 2^-8 for bf16), a sum of terms along a chain of n additions is off by at
most n u times the sum of their absolute values, and an output rounded to bf16 by u of itself more."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U32, UBF = 2.0 ** -24, 2.0 ** -8
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def bd():
    from paper_2511_15927_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return binding


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, scale=1.0, io="f32"):
    return (scale * torch.randn(*shape, generator=g)).to(TYPES[io])


def wide(t, extra, lead=0):
    """t on the GPU as a column slice of a buffer that is wider by `extra`, `lead` columns in; what is around it is NaN."""
    buf = torch.full(t.shape[:-1] + (t.shape[-1] + extra,), float("nan"), dtype=t.dtype, device="cuda")
    v = buf[..., lead:lead + t.shape[-1]]
    v.copy_(t)
    return v


def nans(*shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def within(got, ref, bound, io="f32"):
    got, ref = got.detach().double().cpu(), ref.double()
    assert got.shape == ref.shape
    bound = bound + (UBF * ref.abs() if io == "bf16" else 0.0) + 1e-38
    off = (got - ref).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), "%d of %d beyond the bound, worst %.3g times it" % (
        int(bad.sum()), bad.numel(), float((off / bound)[bad].nan_to_num(nan=float("inf")).max()))


def workspace(n):
    return torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")   # (NaNs, and ids of no token)


# ---- token table ----

@pytest.mark.parametrize("table", ["f32", "bf16"])
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("batch,seqlen,d,vocab,extra", [
    (1, 1, 1, 1, 0), (2, 3, 7, 5, 3), (1, 40, 8, 100, 0), (3, 5, 64, 11, 8), (2, 17, 740, 1000, 5), (1, 300, 2048, 50, 0), (2, 2, 5003, 9, 1)])
def test_embed_rows(bd, batch, seqlen, d, vocab, extra, io, table):
    g = gen(batch + 10 * d)
    tab = normal(g, vocab, d, io=table)
    tok = torch.randint(-2, vocab + 2, (batch, seqlen), generator=g)   # some outside the table
    desc = bd.make_embed_desc(batch, seqlen, d, vocab, table=table, io=io, scale=1.7)
    out = wide(torch.full((batch, seqlen, d), float("nan"), dtype=TYPES[io]), extra, extra // 2)
    bd.bimamba_embed(desc, tok.cuda(), tab.cuda(), out)
    known = (tok >= 0) & (tok < vocab)
    ref = torch.where(known[..., None], tab.float()[tok.clamp(0, vocab - 1)] * torch.tensor(1.7), torch.zeros(())).to(TYPES[io])
    assert torch.equal(out.cpu(), ref)


def test_embed_of_unknown_ids_takes_nothing_from_the_table(bd):
    table = torch.full((3, 100), float("nan"))
    out = nans(1, 4, 100)
    bd.bimamba_embed(bd.make_embed_desc(1, 4, 100, 3, io="f32"), torch.tensor([[-1, 3, 2 ** 62, -2 ** 63]], device="cuda"), table.cuda(), out)
    assert torch.equal(out, torch.zeros(1, 4, 100, device="cuda"))


def embed_bwd_ref(tok, dout, vocab, scale):
    """Gradient, sums of absolute values and counts, in 64 bits."""
    d = dout.shape[-1]
    ids, rows = tok.reshape(-1), dout.double().reshape(-1, d)
    known = (ids >= 0) & (ids < vocab)
    ids, rows = ids[known], rows[known]
    zero = torch.zeros(vocab, d, dtype=torch.float64)
    count = torch.bincount(ids, minlength=vocab).double()
    return scale * zero.index_add(0, ids, rows), abs(scale) * zero.index_add(0, ids, rows.abs()), count


def embed_bwd(bd, tok, dout, vocab, scale, io):
    batch, seqlen, d = dout.shape
    desc = bd.make_embed_desc(batch, seqlen, d, vocab, io=io, scale=scale)
    dtable = nans(vocab, d)
    bd.bimamba_embed_bwd(desc, tok, dout, dtable, workspace(bd.bimamba_embed_bwd_workspace_bytes(desc)))
    return dtable


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["spread", "half", "one", "outside"])
@pytest.mark.parametrize("batch,seqlen,d,vocab", [
    (1, 1, 1, 1), (1, 1, 513, 3), (2, 3, 7, 5), (1, 63, 8, 4), (1, 64, 8, 4), (1, 65, 520, 40), (4, 512, 64, 300), (1, 2049, 72, 1000),
    (3, 1237, 740, 3201), (2, 20000, 32, 50000), (1, 70000, 8, 70), (1, 300000, 8, 5000), (1, 5000, 3, 1 << 20)])
def test_embed_gradient(bd, batch, seqlen, d, vocab, kind, io):
    g = gen(seqlen + d)
    tok = torch.randint(0, vocab, (batch, seqlen), generator=g)
    if kind == "half":
        tok[torch.rand(batch, seqlen, generator=g) < 0.5] = vocab - 1
    elif kind == "one":
        tok[:] = vocab // 2
    elif kind == "outside":
        tok = torch.randint(-vocab, 2 * vocab, (batch, seqlen), generator=g)
        tok[0, 0] = 2 ** 40
    dout = normal(g, batch, seqlen, d, io=io)
    got = embed_bwd(bd, tok.cuda(), wide(dout, 5, 2), vocab, 0.75, io)
    ref, absolute, count = embed_bwd_ref(tok, dout, vocab, 0.75)
    chain = torch.minimum(count, torch.tensor(64.0)) + count / 8 + 12   # a slice, a wave's slices of at least eight, the waves, the scale
    within(got, ref, chain[:, None] * U32 * absolute)
    again = embed_bwd(bd, tok.cuda(), dout.cuda(), vocab, 0.75, io)
    assert torch.equal(got, again)


def test_embed_gradient_of_nothing(bd):
    assert torch.equal(embed_bwd(bd, torch.zeros(2, 0, dtype=torch.int64, device="cuda"), torch.zeros(2, 0, 9, device="cuda"), 100, 1.0, "f32"),
                       torch.zeros(100, 9, device="cuda"))


def test_embed_gradient_of_a_broadcast_input(bd):
    """A gradient that is one row for all tokens (strides of 0), and tokens that are one id for a sequence."""
    g = gen(3)
    row, tok = normal(g, 1, 1, 100), torch.randint(0, 9, (4, 1), generator=g)
    got = embed_bwd(bd, tok.cuda().expand(4, 33), row.cuda().expand(4, 33, 100), 9, 1.0, "f32")
    ref, absolute, count = embed_bwd_ref(tok.expand(4, 33), row.expand(4, 33, 100), 9, 1.0)
    within(got, ref, (count[:, None] + 12) * U32 * absolute)


# ---- layer norm ----

NORM_SHAPES = [(1, 1, 1), (2, 3, 2), (1, 5, 7), (3, 2, 8), (2, 9, 511), (1, 4, 512), (2, 7, 513), (3, 41, 740), (1, 1100, 740), (2, 700, 1000),
               (2, 6, 1024), (2, 600, 2048), (1, 3, 2049), (2, 2, 4096), (1, 3, 4100), (1, 2, 8192), (2, 3, 8193), (1, 5, 20001)]


def norm_ref(x, weight, bias, eps):
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    rstd = 1 / ((x - mean).square().mean(-1, keepdim=True) + eps).sqrt()
    hat = (x - mean) * rstd
    w = 1.0 if weight is None else weight.double() if weight.dim() == 1 else weight.double()[:, None]
    b = 0.0 if bias is None else bias.double() if bias.dim() == 1 else bias.double()[:, None]
    return hat * w + b, mean, rstd, hat, w, b


def norm_inputs(g, batch, seqlen, d, vectors, io, offset):
    x = (offset + 2 * torch.randn(batch, seqlen, d, generator=g)).to(TYPES[io])
    if vectors == "none":
        return x, None, None
    rows = (batch,) if vectors == "batch" else ()
    return x, 1 + 0.3 * torch.randn(*rows, d, generator=g), 0.3 * torch.randn(*rows, d, generator=g)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("vectors", ["shared", "batch", "none"])
@pytest.mark.parametrize("batch,seqlen,d", NORM_SHAPES)
def test_layer_norm(bd, batch, seqlen, d, vectors, io):
    g = gen(7 * d + seqlen)
    x, w, b = norm_inputs(g, batch, seqlen, d, vectors, io, 5.0)
    eps = 1e-5
    y, mean, rstd = wide(torch.zeros_like(x), 3, 1), nans(batch, seqlen), nans(batch, seqlen)
    y.fill_(float("nan"))
    side = lambda v: None if v is None else wide(v, 4, 4) if vectors == "batch" else v.cuda()  # noqa: E731
    bd.bimamba_layer_norm(bd.make_norm_desc(batch, seqlen, d, io=io, eps=eps), wide(x, 9, 5), side(w), side(b), y, mean, rstd)
    ry, rmean, rrstd, hat, rw, rb = norm_ref(x, w, b, eps)
    # a mean and a mean of squares are sums along chains of 32 values a lane (long rows: d / 1024), the lanes and the waves
    chain = 48 + d / 1024
    size = x.double().abs().mean(-1, keepdim=True)
    off_mean = chain * U32 * size                              # of the mean
    off_hat = off_mean * rrstd + U32 * (4 + chain) * hat.abs() + U32 * x.double().abs() * rrstd   # and of rstd, relative
    off_rstd = (chain + 6) * U32 * rrstd + (off_mean * rrstd) ** 2 * rrstd + U32 * size * rrstd * rrstd
    within(mean, rmean[..., 0], off_mean[..., 0] + U32 * rmean[..., 0].abs())
    within(rstd, rrstd[..., 0], off_rstd[..., 0])
    relative = off_rstd / rrstd
    within(y, ry, (off_hat + relative * hat.abs()) * (rw.abs() if w is not None else 1.0) + 3 * U32 * (ry.abs() + (hat * rw).abs()), io)


def test_layer_norm_of_a_large_mean_and_of_constants(bd):
    """The statistics are taken around the mean: 4096 + noise keeps its digits; a constant row has rstd 1 / sqrt(eps) and gives the bias."""
    g = gen(5)
    for d in (300, 2048, 9000):
        x = 4096 + torch.randn(1, 4, d, generator=g)
        x[0, 3] = 7.0
        bias = torch.randn(d, generator=g)
        y, rstd = nans(1, 4, d), nans(1, 4)
        bd.bimamba_layer_norm(bd.make_norm_desc(1, 4, d, io="f32", eps=1e-5), x.cuda(), None, bias.cuda(), y, None, rstd)
        ry, _, rrstd, hat, _, _ = norm_ref(x, None, bias, 1e-5)
        # the mean is off by a few units of 4096 u at worst, and all differences with it
        within(y[:, :3], ry[:, :3], 16 * 4096 * U32 + 64 * U32 * (hat[:, :3].abs() + ry[:, :3].abs()))
        within(rstd[:, :3], rrstd[:, :3, 0], (64 * U32 + (16 * 4096 * U32) ** 2 + 4096 * U32 * 0.1) * rrstd[:, :3, 0])
        within(rstd[:, 3], torch.full((1,), 1e-5, dtype=torch.float64).rsqrt(), torch.tensor(1e-4 * 316))
        within(y[0, 3], bias, 7 * U32 * 317 * 2 * torch.ones(d, dtype=torch.float64))


def norm_bwd_ref(x, weight, mean, rstd, dy):
    """The formula's gradients in 64 bits, and the sums of absolute values of what they add up."""
    x, dy, mean, rstd = x.double(), dy.double(), mean.double()[..., None], rstd.double()[..., None]
    hat = (x - mean) * rstd
    w = torch.ones(x.shape[-1], dtype=torch.float64) if weight is None else weight.double() if weight.dim() == 1 else weight.double()[:, None]
    gr = dy * w
    dx = rstd * (gr - gr.mean(-1, keepdim=True) - hat * (gr * hat).mean(-1, keepdim=True))
    size = rstd * (gr.abs() + gr.abs().mean(-1, keepdim=True) + hat.abs() * (gr * hat).abs().mean(-1, keepdim=True))
    return dx, size, dy * hat, dy


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("vectors", ["shared", "batch", "none"])
@pytest.mark.parametrize("batch,seqlen,d", NORM_SHAPES)
def test_layer_norm_gradient(bd, batch, seqlen, d, vectors, io):
    g = gen(11 * d + seqlen)
    x, w, _ = norm_inputs(g, batch, seqlen, d, vectors, io, 1.0)
    dy = normal(g, batch, seqlen, d, io=io)
    _, mean, rstd, _, _, _ = norm_ref(x, w, None, 1e-5)
    mean, rstd = mean[..., 0].float(), rstd[..., 0].float()
    per_batch = vectors == "batch"
    desc = bd.make_norm_desc(batch, seqlen, d, io=io)
    shape = (batch, d) if per_batch else (d,)

    def call(want=(True, True)):
        dx = wide(torch.zeros_like(x), 5, 2)
        dx.fill_(float("nan"))
        dw, db = (nans(*shape) if want[0] else None), (nans(*shape) if want[1] else None)
        ws = workspace(bd.bimamba_layer_norm_bwd_workspace_bytes(desc, per_batch)) if any(want) else None
        side = None if w is None else wide(w, 4, 4) if per_batch else w.cuda()
        bd.bimamba_layer_norm_bwd(desc, wide(x, 1), side, mean.cuda(), rstd.cuda(), wide(dy, 3, 3), dx, dw, db, ws)
        return dx, dw, db

    dx, dw, db = call()
    rdx, size, tw, tb = norm_bwd_ref(x, w, mean, rstd, dy)
    within(dx, rdx, (64 + d / 1024) * U32 * size, io)
    over = 1 if per_batch else (0, 1)
    rows = seqlen if per_batch else batch * seqlen
    chain = rows + 8   # (at worst one row after the other)
    within(dw, tw.sum(over), chain * U32 * tw.abs().sum(over) + 4 * U32 * tw.abs().sum(over))
    within(db, tb.sum(over), chain * U32 * tb.abs().sum(over))
    again = call()
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again))
    if vectors == "shared":
        only = [call((True, False)), call((False, True)), call((False, False))]
        assert all(torch.equal(o[0], dx) for o in only) and torch.equal(only[0][1], dw) and torch.equal(only[1][2], db)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("batch,seqlen,d", [(1, 1, 9000), (1100, 1, 5), (1100, 2, 72), (340, 7, 600), (1030, 9, 1000), (600, 3, 2050), (520, 2, 5000), (260, 3, 8200)])
def test_layer_norm_gradient_of_a_workgroup_a_vector(bd, batch, seqlen, d, io):
    """As many vectors as workgroups: their gradients need no workspace, and those that are not wanted are not written."""
    g = gen(13 * d + batch)
    x, w, _ = norm_inputs(g, batch, seqlen, d, "batch", io, 1.0)
    dy = normal(g, batch, seqlen, d, io=io)
    _, mean, rstd, _, _, _ = norm_ref(x, w, None, 1e-5)
    mean, rstd = mean[..., 0].float(), rstd[..., 0].float()
    desc = bd.make_norm_desc(batch, seqlen, d, io=io)
    assert bd.bimamba_layer_norm_bwd_workspace_bytes(desc, True) == 0
    args = x.cuda(), w.cuda(), mean.cuda(), rstd.cuda(), dy.cuda()

    def call(want):
        dx, around = torch.empty_like(args[0]), nans(2, 2 + batch, d)   # (with a row before and after that stays as it is)
        dw, db = (around[k, 1:-1] if want[k] else None for k in range(2))
        bd.bimamba_layer_norm_bwd(desc, *args, dx, dw, db, None)
        assert all(bool(torch.isnan(a[::batch + 1] if k else a).all()) for a, k in zip(around, want))
        return dx, dw, db

    dx, dw, db = call((True, True))
    rdx, size, tw, tb = norm_bwd_ref(x, w, mean, rstd, dy)
    within(dx, rdx, (64 + d / 1024) * U32 * size, io)
    within(dw, tw.sum(1), (seqlen + 12) * U32 * tw.abs().sum(1))
    within(db, tb.sum(1), (seqlen + 8) * U32 * tb.abs().sum(1))
    for want in ((True, False), (False, True), (False, False)):
        assert all(a is None or torch.equal(a, b) for a, b in zip(call(want), (dx, dw, db)))


@pytest.mark.parametrize("d", [5, 700, 2048, 9000])
def test_layer_norm_keeps_what_is_not_a_number_in_its_row(bd, d):
    """A row with a NaN or an infinity is NaN; the others, and the gradients of theirs, are what they are without it."""
    g = gen(d)
    x = normal(g, 2, 9, d)
    desc = bd.make_norm_desc(2, 9, d, io="f32")

    def call(x):
        y, mean, rstd, dx = nans(2, 9, d), nans(2, 9), nans(2, 9), nans(2, 9, d)
        bd.bimamba_layer_norm(desc, x.cuda(), None, None, y, mean, rstd)
        bd.bimamba_layer_norm_bwd(desc, x.cuda(), None, mean, rstd, torch.ones(1, 1, d, device="cuda").expand(2, 9, d), dx, None, None, None)
        return y, mean, dx

    clean, bad = call(x), x.clone()
    bad[0, 3, d // 2], bad[1, 8, d - 1] = math.nan, math.inf
    got = call(bad)
    hit = torch.zeros(2, 9, dtype=torch.bool, device="cuda")
    hit[0, 3] = hit[1, 8] = True
    assert bool(torch.isnan(got[0][hit]).all()) and bool(torch.isnan(got[2][hit]).all())
    assert all(torch.equal(a[~hit], b[~hit]) for a, b in zip(got, clean))


def test_layer_norm_gradient_against_differences(bd):
    g = gen(23)
    x, w, b = norm_inputs(g, 2, 3, 12, "batch", "f32", 0.5)
    dy = normal(g, 2, 3, 12)
    eps, h = 1e-3, 1e-5
    loss = lambda x, w, b: float((norm_ref(x, w, b, eps)[0] * dy.double()).sum())  # noqa: E731
    _, mean, rstd, _, _, _ = norm_ref(x, w, b, eps)
    desc = bd.make_norm_desc(2, 3, 12, io="f32", eps=eps)
    dx, dw, db = nans(2, 3, 12), nans(2, 12), nans(2, 12)
    bd.bimamba_layer_norm_bwd(desc, x.cuda(), w.cuda(), mean[..., 0].float().cuda(), rstd[..., 0].float().cuda(), dy.cuda(), dx, dw, db,
                              workspace(bd.bimamba_layer_norm_bwd_workspace_bytes(desc, True)))
    args = [t.double() for t in (x, w, b)]
    for k, got in enumerate((dx, dw, db)):
        for i in range(args[k].numel()):
            up, down = [a.clone() for a in args], [a.clone() for a in args]
            up[k].view(-1)[i] += h
            down[k].view(-1)[i] -= h
            slope = (loss(*up) - loss(*down)) / (2 * h)
            # h^2 of third derivatives and 64-bit noise over h lie near 1e-9; fp32 values of at most a few tens, 64 roundings
            assert abs(float(got.view(-1)[i]) - slope) < 64 * U32 * 30, (k, i)


def test_layer_norm_of_nothing(bd):
    desc = bd.make_norm_desc(2, 0, 9, io="f32")
    none = torch.zeros(2, 0, 9, device="cuda")
    stat = torch.zeros(2, 0, device="cuda")
    bd.bimamba_layer_norm(desc, none, None, None, none.clone(), stat, stat.clone())
    dw, db = nans(9), nans(9)
    bd.bimamba_layer_norm_bwd(desc, none, None, stat, stat, none, none.clone(), dw, db, workspace(0))
    assert torch.equal(dw, torch.zeros(9, device="cuda")) and torch.equal(db, torch.zeros(9, device="cuda"))


# ---- log probabilities ----

def scores_ref(x, targets, k):
    """In 64 bits, rows of nothing but -inf and rows with NaN or +inf as the header states them."""
    x = x.double()
    V = x.shape[-1]
    top = x.amax(-1, keepdim=True)
    empty, bad = top[..., 0] == -math.inf, (torch.isnan(x) | (x == math.inf)).any(-1)
    shift = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    d = x - shift
    e = torch.exp(d)
    log_s = torch.log(e.sum(-1))
    lse = torch.where(bad, math.nan, shift[..., 0] + log_s)
    has = (targets >= 0) & (targets < V)
    logp = x.gather(-1, targets.clamp(0, V - 1)[..., None])[..., 0] - lse
    logp = torch.where(empty, -math.inf, logp)
    logp = torch.where(has, torch.where(bad, math.nan, logp), 0.0)
    spread = torch.where(e > 0, e * d, 0.0).sum(-1)
    entropy = torch.where(empty, 0.0, torch.where(bad, math.nan, log_s - spread / e.sum(-1)))
    order = torch.sort(x, dim=-1, descending=True, stable=True)
    value = torch.where(empty[..., None], -math.inf, order.values[..., :k] - lse[..., None])
    token = torch.where(bad[..., None], -1, order.indices[..., :k])
    return dict(logp=logp, lse=lse, entropy=entropy, top_logp=torch.where(bad[..., None], math.nan, value), top_token=token), (e * d.abs().clamp(max=1e4)).sum(-1) / e.sum(-1)


def scores(bd, x, targets, k=0, targets_only=0, want=("logp", "lse", "entropy")):
    batch, seqlen, V = x.shape
    desc = bd.make_logits_desc(batch, seqlen, V, io="bf16" if x.dtype is torch.bfloat16 else "f32", top_k=k, targets_only=targets_only)
    out = {n: nans(batch, seqlen) for n in want}
    if k:
        out["top_logp"], out["top_token"] = nans(batch, seqlen, k), torch.full((batch, seqlen, k), -7, device="cuda")
    bd.bimamba_log_probs(desc, x, targets, out, workspace(bd.bimamba_log_probs_workspace_bytes(desc)))
    return out


def assert_scores(got, ref, spread, V):
    """lse = m + log S: S is a sum along a chain of V / 256 additions a lane, the lanes, waves and parts, of exponentials whose argument is
    rounded in the order of itself; the entropy takes the same sums once more, times what they are spread over."""
    unit = U32 * (48 + V / 256 + 4 * spread)
    big = lambda t: torch.nan_to_num(t, nan=0.0, posinf=0.0, neginf=0.0).abs()  # noqa: E731
    bound = dict(lse=unit + 2 * U32 * big(ref["lse"]), logp=unit + 3 * U32 * (big(ref["logp"]) + big(ref["lse"])),
                 entropy=unit * (2 + 2 * spread))
    bound["top_logp"] = (unit + 3 * U32 * big(ref["lse"]))[..., None] + 3 * U32 * big(ref["top_logp"])
    for n, t in got.items():
        if n == "top_token":
            assert torch.equal(t.cpu(), ref[n])
            continue
        t, r = t.double().cpu(), ref[n]
        assert torch.equal(torch.isnan(t), torch.isnan(r)), n
        assert torch.equal(torch.isinf(t), torch.isinf(r)) and torch.equal(t[torch.isinf(t)], r[torch.isinf(r)]), n
        fine = torch.isfinite(r)
        within(t[fine], r[fine], torch.nan_to_num(bound[n], nan=0.0, posinf=0.0).expand(r.shape)[fine])


def logits_of(g, kind, batch, seqlen, V, io):
    x = 3 * torch.randn(batch, seqlen, V, generator=g)
    if kind == "masked":
        x[torch.rand(batch, seqlen, V, generator=g) < 0.7] = -math.inf
        x[0, 0] = -math.inf                                     # nothing left
        x[-1, -1] = -math.inf
        x[-1, -1, V // 3] = 2.5                                 # one left
    elif kind == "lowest":
        low = torch.finfo(TYPES[io]).min
        x[torch.rand(batch, seqlen, V, generator=g) < 0.5] = low
        x[0, 0] = low
    elif kind == "ties":
        x = torch.randint(-2, 3, (batch, seqlen, V), generator=g).float() * (1 - 2 * torch.randint(0, 2, (batch, seqlen, V), generator=g))
        x[0, 0] = 1.0
        x[-1, -1] = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)
    elif kind == "rising":
        x = torch.arange(V).float().expand(batch, seqlen, V) * (20.0 / V)
    elif kind == "few lanes":                                   # large values only where one lane in 256 reads them
        x = torch.where((torch.arange(V) // 8) % 256 == 5, 8.0, 0.0) + 0.1 * x
    elif kind == "large":
        x = x * 1e4
    return x.to(TYPES[io])


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "masked", "lowest", "ties", "rising", "few lanes", "large"])
@pytest.mark.parametrize("batch,seqlen,V,k", [
    (1, 1, 1, 1), (1, 2, 2, 2), (2, 3, 7, 4), (1, 2, 8, 8), (3, 1, 9, 8), (1, 4, 255, 3), (2, 2, 2048, 8), (1, 3, 2049, 1), (1, 5, 4097, 8),
    (2, 2, 50257, 8), (1, 2, 131072, 5), (300, 4, 4099, 8), (700, 3, 300, 2)])
def test_scores(bd, batch, seqlen, V, k, kind, io):
    g = gen(V + 3 * k)
    x = logits_of(g, kind, batch, seqlen, V, io)
    targets = torch.randint(-1, V + 1, (batch, seqlen), generator=g)
    dx, dt = wide(x, 3, 1), targets.cuda()
    ref, spread = scores_ref(x, targets, k)
    got = scores(bd, dx, dt, k)
    assert_scores(got, ref, spread, V)
    again = scores(bd, x.cuda(), dt, k)
    assert all(torch.equal(got[n], again[n]) or bool(torch.isnan(got[n]).any()) for n in got)
    # what is wanted does not change what it is
    only = scores(bd, dx, dt, 0, want=("lse",))
    assert torch.equal(only["lse"], scores(bd, dx, dt, 0, want=("lse", "logp"))["lse"])
    assert_scores(only, ref, spread, V)
    assert_scores(scores(bd, dx, None, k, want=()), ref, spread, V)
    some = scores(bd, dx, dt, k, targets_only=1)
    has = (targets >= 0) & (targets < V)
    for n in got:
        assert torch.equal(torch.nan_to_num(some[n].cpu()[has].double(), nan=1.5), torch.nan_to_num(got[n].cpu()[has].double(), nan=1.5)), n
        assert bool((some[n].cpu()[~has] == (-1 if n == "top_token" else 0)).all()), n


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 3000, 20000])
def test_scores_of_rows_that_are_not_numbers(bd, V, io):
    g = gen(V)
    x = torch.randn(1, 6, V, generator=g)
    x[0, 0, V // 2] = math.nan
    x[0, 1, 0] = math.inf
    x[0, 2, V - 1] = math.inf
    x[0, 3] = -math.inf
    x[0, 3, 1] = math.nan
    x[0, 4, 2] = -math.nan
    x = x.to(TYPES[io])
    targets = torch.tensor([[0, 0, 1, 1, 2, 3]])
    ref, spread = scores_ref(x, targets, 4)
    assert bool(torch.isnan(ref["lse"][0, :5]).all())
    assert_scores(scores(bd, x.cuda(), targets.cuda(), 4), ref, torch.nan_to_num(spread), V)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "masked", "lowest", "large"])
@pytest.mark.parametrize("batch,seqlen,V", [(1, 1, 1), (2, 3, 7), (2, 4, 4099), (1, 2, 50257), (1, 2, 131072), (300, 4, 300)])
def test_scores_in_two_parts(bd, batch, seqlen, V, kind, io):
    """lse and lse_rest together are log sum exp beyond fp32's digits: off by what log S is (a sum along a chain of V / 256 additions a
    lane, the lanes, waves and parts), however large lse itself.  Neither lse nor anything else changes with it."""
    g = gen(V + 17)
    x = logits_of(g, kind, batch, seqlen, V, io)
    targets = torch.randint(-1, V + 1, (batch, seqlen), generator=g)
    ref, spread = scores_ref(x, targets, 1)
    names = ("logp", "lse", "entropy")
    got = scores(bd, x.cuda(), targets.cuda(), want=names + ("lse_rest",))
    assert all(torch.equal(got[n], t) for n, t in scores(bd, x.cuda(), targets.cuda(), want=names).items())
    fine = torch.isfinite(ref["lse"])
    top = x.double().amax(-1)
    # (the reference itself takes the maximum apart: far below it, 64 bits hold what is left)
    log_s = torch.log(torch.exp(x.double() - torch.where(fine, top, 0.0)[..., None]).sum(-1))
    off = (got["lse"].double().cpu() - top + got["lse_rest"].double().cpu() - log_s)[fine].abs()
    assert bool((off <= (U32 * (48 + V / 256 + 4 * spread + 4 * log_s))[fine]).all())
    assert bool((got["lse_rest"].cpu()[~fine] == 0).all())
    some = scores(bd, x.cuda(), targets.cuda(), targets_only=1, want=("lse", "lse_rest"))
    has = (targets >= 0) & (targets < V)
    assert torch.equal(some["lse_rest"].cpu()[has], got["lse_rest"].cpu()[has]) and bool((some["lse_rest"].cpu()[~has] == 0).all())


def scores_bwd_ref(x, targets, lse, entropy, dlogp, dentropy):
    """The formula in 64 bits, and the size of its terms."""
    x = x.double()
    V = x.shape[-1]
    has = (targets >= 0) & (targets < V)
    lse = lse.double()[..., None]
    empty = torch.isneginf(lse)
    logp = torch.where(empty, -math.inf, x - lse)
    p = torch.exp(logp)
    dl = torch.where(has, dlogp.double(), 0.0)[..., None] if dlogp is not None else torch.zeros_like(lse)
    d = torch.zeros_like(p).scatter(-1, targets.clamp(0, V - 1)[..., None], dl) - dl * p
    size = d.abs() + 2 * (dl * p).abs() * (1 + logp.abs().clamp(max=1e3))
    if dentropy is not None:
        inner = torch.where(p > 0, logp + entropy.double()[..., None], 0.0)
        d = d - dentropy.double()[..., None] * p * inner
        size = size + (dentropy.double()[..., None] * p).abs() * (inner.abs() + 1 + entropy.double()[..., None].abs()) * (1 + logp.abs().clamp(max=1e3))
    return torch.where(empty, 0.0, d), torch.where(empty, 0.0, size)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "masked", "lowest", "large"])
@pytest.mark.parametrize("given", ["logp", "entropy", "both"])
@pytest.mark.parametrize("batch,seqlen,V", [(1, 1, 1), (2, 3, 7), (1, 4, 2049), (3, 5, 8200), (1, 2, 50257)])
def test_scores_gradient(bd, batch, seqlen, V, given, kind, io):
    g = gen(V + 1)
    x = logits_of(g, kind, batch, seqlen, V, io)
    targets = torch.randint(-1, V + 1, (batch, seqlen), generator=g)
    ref, _ = scores_ref(x, targets, 1)
    lse, entropy = ref["lse"].float(), ref["entropy"].float()
    dlogp = normal(g, batch, seqlen) if given != "entropy" else None
    dentropy = normal(g, batch, seqlen) if given != "logp" else None
    if batch * seqlen > 2:
        for t in (dlogp, dentropy):
            if t is not None:
                t.view(-1)[1] = 0.0
    want, size = scores_bwd_ref(x, targets, lse, entropy, dlogp, dentropy)
    desc = bd.make_logits_desc(batch, seqlen, V, io=io)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    args = (targets.cuda(), lse.cuda(), dev(entropy) if dentropy is not None else None, dev(dlogp), dev(dentropy))
    out = wide(torch.zeros_like(x), 5, 4)
    out.fill_(float("nan"))
    logits = wide(x, 3, 2)
    bd.bimamba_log_probs_bwd(desc, logits, *args, out)
    within(out, want, 8 * U32 * size, io)
    bd.bimamba_log_probs_bwd(desc, logits, *args, logits)      # in place of the logits
    assert torch.equal(logits, out)


def test_scores_gradient_reads_no_row_without_one(bd):
    """Rows whose gradients are 0 get zeros whatever their logits, rows of nothing but -inf whatever their gradients."""
    x = torch.full((1, 4, 3001), float("nan"))
    x[0, 2:] = -math.inf
    x[0, 3, 5] = 0.0
    zero = torch.zeros(1, 4)
    dlogp = torch.tensor([[3.0, 0.0, 2.0, 1.0]])
    targets = torch.tensor([[-1, 7, 7, 5]])
    lse = torch.tensor([[math.nan, math.nan, -math.inf, 0.0]])
    for dentropy in (None, zero.cuda()):
        out = nans(1, 4, 3001)
        bd.bimamba_log_probs_bwd(bd.make_logits_desc(1, 4, 3001, io="f32"), x.cuda(), targets.cuda(), lse.cuda(), zero.cuda(), dlogp.cuda(), dentropy, out)
        assert torch.equal(out, torch.zeros(1, 4, 3001, device="cuda"))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 7, 3001, 8200])
def test_scores_gradient_of_rows_that_were_not_asked_for(bd, V, io):
    """With targets_only the scores of a row without a target are constants: its gradient is 0 whatever dentropy is, its logits are not
    read; the other rows get what they get without the flag."""
    g = gen(V)
    x = normal(g, 2, 9, V, scale=3.0, io=io)
    targets = torch.randint(0, V, (2, 9), generator=g)
    targets[0, ::2], targets[1, 4], targets[1, 7] = -1, V, 2 ** 40
    has = (targets >= 0) & (targets < V)
    x[~has] = 40.0
    dlogp, dentropy = normal(g, 2, 9).cuda(), normal(g, 2, 9).cuda()
    some, every = (bd.make_logits_desc(2, 9, V, io=io, targets_only=k) for k in (1, 0))
    out = scores(bd, x.cuda(), targets.cuda(), targets_only=1)
    want, got = nans(2, 9, V, dtype=TYPES[io]), nans(2, 9, V, dtype=TYPES[io])
    bd.bimamba_log_probs_bwd(every, x.cuda(), targets.cuda(), out["lse"], out["entropy"], dlogp, dentropy, want)
    x[~has] = math.nan
    bd.bimamba_log_probs_bwd(some, x.cuda(), targets.cuda(), out["lse"], out["entropy"], dlogp, dentropy, got)
    assert torch.equal(got.cpu()[~has], torch.zeros(int((~has).sum()), V, dtype=TYPES[io]))
    assert torch.equal(got.cpu()[has], want.cpu()[has])


def test_scores_gradient_against_differences(bd):
    g = gen(31)
    x, targets = torch.randn(2, 2, 9, generator=g), torch.tensor([[0, 8], [3, -1]])
    dlogp, dentropy = normal(g, 2, 2), normal(g, 2, 2)

    def loss(x):
        r, _ = scores_ref(x, targets, 1)
        return float((r["logp"] * dlogp.double() + r["entropy"] * dentropy.double()).sum())

    r, _ = scores_ref(x, targets, 1)
    dx = nans(2, 2, 9)
    bd.bimamba_log_probs_bwd(bd.make_logits_desc(2, 2, 9, io="f32"), x.cuda(), targets.cuda(), r["lse"].float().cuda(), r["entropy"].float().cuda(),
                             dlogp.cuda(), dentropy.cuda(), dx)
    h = 1e-5
    for i in range(x.numel()):
        up, down = x.double().clone(), x.double().clone()
        up.view(-1)[i] += h
        down.view(-1)[i] -= h
        assert abs(float(dx.view(-1)[i]) - (loss(up) - loss(down)) / (2 * h)) < 64 * U32 * 8, i


# ---- clipped gradients ----

def clip(bd, grads, max_norm, to=None):
    table = bd.GradTable(grads, to)
    norm = nans(1)
    bd.bimamba_clip_grads(table, max_norm, norm, workspace(bd.bimamba_clip_grads_workspace_bytes(table)))
    return norm


@pytest.mark.parametrize("counts", [(1,), (0,), (5, 0, 8191, 8192, 8193), (3, 0, 0, 70000), (4096,) * 300, (9_000_001, 17)])
@pytest.mark.parametrize("max_norm", [1.0, 0.0, 1e9, math.inf])
@pytest.mark.parametrize("place", ["apart", "in place", "odd"])
def test_clip(bd, counts, max_norm, place):
    g = gen(len(counts) + counts[0])
    src = [normal(g, n, io="bf16" if i % 3 == 2 else "f32") for i, n in enumerate(counts)]
    if place == "odd":   # one element off, so that no tensor lies on 16 bytes
        grads = [torch.cat([t[:1], t]).cuda()[1:] if t.numel() else t.cuda() for t in src]
    else:
        grads = [t.cuda() for t in src]
    to = grads if place == "in place" else [torch.full_like(t, float("nan")) for t in grads]
    norm = clip(bd, grads, max_norm, to)
    ref = math.sqrt(sum(float(t.double().square().sum()) for t in src))
    assert abs(float(norm) - ref) <= 2 * U32 * ref
    factor = min(1.0, max_norm / ref) if ref else 1.0
    for t, s in zip(to, src):
        if factor == 1.0:
            assert torch.equal(t.cpu(), s)
        else:
            within(t, s.double() * factor, 4 * U32 * s.double().abs() * factor, "bf16" if s.dtype is torch.bfloat16 else "f32")


def test_clip_of_nothing(bd):
    assert float(clip(bd, [], 1.0)) == 0.0


def test_clip_neither_overflows_nor_vanishes(bd):
    for size in (1e30, 1e-30):
        src = size * torch.ones(10000)
        to = [torch.empty(10000, device="cuda")]
        norm = clip(bd, [src.cuda()], size, to)
        assert abs(float(norm) / (100 * size) - 1) < 4 * U32
        within(to[0], src.double() / 100, 4 * U32 * src.double() / 100)


@pytest.mark.parametrize("value", [math.inf, math.nan, 3e38])
def test_clip_leaves_gradients_of_a_norm_that_is_not_finite(bd, value):
    src = torch.full((9000,), value)
    src[:4500] = 1.0
    to = [torch.zeros(9000, device="cuda")]
    norm = clip(bd, [src.cuda()], 1.0, to)
    assert not math.isfinite(float(norm))
    assert torch.equal(torch.nan_to_num(to[0].cpu(), nan=7.0), torch.nan_to_num(src, nan=7.0))


# ---- all of them ----

def test_rows_far_apart(bd):
    """Rows more than 2^31 elements apart: offsets pass 32 bits."""
    pitch = 2 ** 31 + 8
    big = torch.empty(2 * pitch + 4096, dtype=torch.bfloat16, device="cuda")
    far = lambda n: big.as_strided((1, 3, n), (3 * pitch, pitch, 1))  # noqa: E731
    g = gen(41)
    x = normal(g, 1, 3, 4000, io="bf16")
    far(4000).copy_(x)
    targets = torch.tensor([[5, -1, 3999]])
    ref, spread = scores_ref(x, targets, 8)
    assert_scores(scores(bd, far(4000), targets.cuda(), 8), ref, spread, 4000)
    desc = bd.make_norm_desc(1, 3, 4000)
    y = torch.empty(1, 3, 4000, dtype=torch.bfloat16, device="cuda")
    bd.bimamba_layer_norm(desc, far(4000), None, None, y)
    y0 = torch.empty_like(y)
    bd.bimamba_layer_norm(desc, x.cuda(), None, None, y0)
    assert torch.equal(y, y0)
    tok = torch.tensor([[2, 0, 2]])
    assert torch.equal(embed_bwd(bd, tok.cuda(), far(4000), 3, 1.0, "bf16"), embed_bwd(bd, tok.cuda(), x.cuda(), 3, 1.0, "bf16"))
    table = normal(g, 3, 4000, io="bf16").cuda()
    bd.bimamba_embed(bd.make_embed_desc(1, 3, 4000, 3, table="bf16"), tok.cuda(), table, far(4000))
    assert torch.equal(far(4000), table[tok.cuda()])
    want = torch.empty_like(y)
    lse = torch.zeros(1, 3, device="cuda")
    one = torch.ones(1, 3, device="cuda")
    ld = bd.make_logits_desc(1, 3, 4000)
    bd.bimamba_log_probs_bwd(ld, far(4000), tok.cuda(), lse, None, one, None, want)
    bd.bimamba_log_probs_bwd(ld, far(4000), tok.cuda(), lse, None, one, None, far(4000))
    assert torch.equal(want, far(4000))


def pass_through_all(bd, g_seed=51):
    """One call of each on fixed buffers: (what enqueues them, what they write)."""
    g = gen(g_seed)
    B, L, D, V = 2, 300, 520, 3000
    tok = torch.randint(0, V, (B, L), generator=g).cuda()
    table, w, b = normal(g, V, D).cuda(), normal(g, B, D).cuda(), normal(g, B, D).cuda()
    x, y, dx, logits, dlogits = (torch.zeros(B, L, n, dtype=torch.bfloat16, device="cuda") for n in (D, D, D, V, V))
    logits.copy_(normal(g, B, L, V, scale=2.0))
    dy = normal(g, B, L, D, io="bf16").cuda()
    mean, rstd, dlogp = (torch.zeros(B, L, device="cuda") for _ in range(3))
    dlogp.fill_(-1.0 / (B * L))
    out = dict(logp=torch.zeros(B, L, device="cuda"), lse=torch.zeros(B, L, device="cuda"), entropy=torch.zeros(B, L, device="cuda"),
               top_logp=torch.zeros(B, L, 3, device="cuda"), top_token=torch.zeros(B, L, 3, dtype=torch.int64, device="cuda"))
    dw, db, dtable = torch.zeros(B, D, device="cuda"), torch.zeros(B, D, device="cuda"), torch.zeros(V, D, device="cuda")
    ed, nd, ld = bd.make_embed_desc(B, L, D, V), bd.make_norm_desc(B, L, D), bd.make_logits_desc(B, L, V, top_k=3)
    ws = [torch.empty(max(n, 16), dtype=torch.uint8, device="cuda") for n in (
        bd.bimamba_embed_bwd_workspace_bytes(ed), bd.bimamba_layer_norm_bwd_workspace_bytes(nd, True), bd.bimamba_log_probs_workspace_bytes(ld))]
    norm = torch.zeros(1, device="cuda")
    grads = bd.GradTable([dtable, dw, db])
    cw = torch.empty(bd.bimamba_clip_grads_workspace_bytes(grads), dtype=torch.uint8, device="cuda")

    def enqueue(stream=None):
        bd.bimamba_embed(ed, tok, table, x, stream=stream)
        bd.bimamba_layer_norm(nd, x, w, b, y, mean, rstd, stream=stream)
        bd.bimamba_log_probs(ld, logits, tok, out, ws[2], stream=stream)
        bd.bimamba_log_probs_bwd(ld, logits, tok, out["lse"], None, dlogp, None, dlogits, stream=stream)
        bd.bimamba_layer_norm_bwd(nd, x, w, mean, rstd, dy, dx, dw, db, ws[1], stream=stream)
        bd.bimamba_embed_bwd(ed, tok, dx, dtable, ws[0], stream=stream)
        bd.bimamba_clip_grads(grads, 0.5, norm, cw, stream=stream)

    return enqueue, [x, y, mean, rstd, *out.values(), dlogits, dx, dw, db, dtable, norm], tok


def test_on_a_stream_and_in_a_graph(bd):
    """The calls on a side stream and replayed from a graph give what they give on the current stream, replay after replay."""
    enqueue, outs, tok = pass_through_all(bd)
    enqueue()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    assert 0.0 < float(want[-1])
    side = torch.cuda.Stream()
    for t in outs:
        t.fill_(0)
    torch.cuda.synchronize()
    enqueue(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        enqueue()
    for k in range(4):
        for t in outs:
            t.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), k
        (torch.randn(1000, 1000, device="cuda") @ torch.randn(1000, 1000, device="cuda")).sum().item()
    tok.copy_(tok.flip(1))
    graph.replay()
    torch.cuda.synchronize()
    replayed = [t.clone() for t in outs]
    enqueue()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, replayed)) and not torch.equal(outs[0], want[0])
