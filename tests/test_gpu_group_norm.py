"""The norm of groups of channels with an activation or a gate, and its gradients, through the C ABI, against the formulas in 64 bits on the
CPU with a running error bound."""
import pytest
import torch

from running_error import TYPES, U32, Run, blank, cuda, gen, nans, normal, wide, within, workspace

pytestmark = pytest.mark.gpu

EPS = 1e-5
CHAIN = 48   # additions that a value of a group goes through: 32 of a lane, 6 over the lanes, 4 over the waves


@pytest.fixture(scope="module")
def bd():
    from paper_2511_15927_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return binding


def inputs(B, L, G, n, io, act, seed, shift=0.3):
    g = gen(seed)
    D = G * n
    return dict(x=(shift + 2 * torch.randn(B, L, D, generator=g)).to(TYPES[io]), z=normal(g, B, L, D, scale=2.0, io=io) if act.startswith("gate") else None,
                w=1 + normal(g, D, scale=0.2), b=normal(g, D, scale=0.2), dy=normal(g, B, L, D, io=io))


def normed(i, G, act, centred):
    """u, and what is left of it without the mean."""
    B, L, D = i["x"].shape
    u = Run(i["x"])
    gate = None if i["z"] is None else Run(i["z"]).silu()
    if act == "gate_before":
        u = u * gate
    u = u.view(B, L, G, D // G)
    mean = u.mean(CHAIN) if centred else Run(torch.zeros(B, L, G, 1))
    return u, mean, gate


def forward_ref(i, G, act, centred):
    B, L, D = i["x"].shape
    u, mean, gate = normed(i, G, act, centred)
    c = u - mean if centred else u
    rstd = ((c * c).mean(CHAIN) + EPS).rsqrt()
    w, b = (Run(i[k]).view(G, D // G) if i[k] is not None else Run(float(k == "w")) for k in "wb")
    v = (c * rstd * w + b).view(B, L, D)
    y = v.silu() if act == "silu" else v * gate if act == "gate_after" else v
    return y, mean[..., 0], rstd[..., 0]


def run_forward(bd, i, G, io, act, centred, extra=0, lead=0):
    B, L, D = i["x"].shape
    desc = bd.make_group_norm_desc(B, L, D, G, io=io, act=act, centred=centred, eps=EPS)
    y, mean, rstd = blank((B, L, D), io, extra, lead), nans(B, L, G) if centred else None, nans(B, L, G)
    z = None if i["z"] is None else wide(i["z"], extra, extra - lead)
    bd.bimamba_group_norm(desc, wide(i["x"], extra, lead), z, cuda(i["w"]), cuda(i["b"]), y, mean, rstd)
    return y, mean, rstd


# groups of one channel, of less than a piece of 16 bytes, of odd sizes, of exactly what lanes and pieces hold and one more, of four waves
SHAPES = [(1, 1, 1, 1), (2, 3, 5, 1), (1, 5, 3, 3), (2, 2, 9, 7), (1, 4, 70, 8), (2, 5, 6, 16), (3, 7, 4, 37), (2, 9, 12, 64), (1, 3, 5, 100), (2, 2, 3, 500),
          (1, 5, 2, 512), (1, 3, 3, 513), (1, 2, 2, 1500), (2, 1, 1, 2048), (1, 2, 2, 2050), (1, 3, 1, 5000), (1, 2, 1, 8192), (1, 700, 2, 64), (41, 9, 1, 24)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "silu", "gate_before", "gate_after"])
@pytest.mark.parametrize("centred", [0, 1])
@pytest.mark.parametrize("B,L,G,n", SHAPES)
def test_groups(bd, B, L, G, n, centred, act, io):
    k = SHAPES.index((B, L, G, n)) + centred
    i = inputs(B, L, G, n, io, act, 7 * k + n)
    if k % 5 == 0:
        i["w" if k % 2 else "b"] = None
    extra = (0, 3, 8)[k % 3]
    y, mean, rstd = run_forward(bd, i, G, io, act, centred, extra, extra // 2)
    ry, rm, rr = forward_ref(i, G, act, centred)
    within(y, ry, io)
    within(rstd, rr)
    if centred:
        within(mean, rm)


def gradient_ref(i, G, act, centred, mean, rstd):
    B, L, D = i["x"].shape
    shape = (B, L, G, D // G)
    u, _, gate = normed(i, G, act, False)
    w, b = (Run(i[k]).view(G, D // G) if i[k] is not None else Run(float(k == "w")) for k in "wb")
    rstd = Run(rstd.double()[..., None])
    xh = (u - mean.double()[..., None] if centred else u) * rstd
    dv, dz = Run(i["dy"]).view(*shape), None
    if act in ("silu", "gate_after"):
        v = xh * w + b
        if act == "silu":
            dv = dv * v.silu_slope()
        else:
            dz = (dv * v).view(B, L, D) * Run(i["z"]).silu_slope()
            dv = dv * gate.view(*shape)
    rows = B * L
    dw, db = (t.view(rows, D).sum(0, rows) for t in (dv * xh, dv))
    g = dv * w
    du = g - xh * (g * xh).mean(CHAIN)
    if centred:
        du = du - g.mean(CHAIN)
    du = (du * rstd).view(B, L, D)
    if act == "gate_before":
        dz = du * Run(i["x"]) * Run(i["z"]).silu_slope()
        du = du * gate
    return du, dz, dw, db


def run_backward(bd, i, G, io, act, centred, mean, rstd, extra=0, lead=0):
    B, L, D = i["x"].shape
    desc = bd.make_group_norm_desc(B, L, D, G, io=io, act=act, centred=centred, eps=EPS)
    dx, dz = blank((B, L, D), io, extra, lead), blank((B, L, D), io, extra, lead) if i["z"] is not None else None
    dw, db = nans(D), nans(D)
    z = None if i["z"] is None else wide(i["z"], extra, extra - lead)
    bd.bimamba_group_norm_bwd(desc, wide(i["x"], extra, lead), z, cuda(i["w"]), cuda(i["b"]), mean, rstd, wide(i["dy"], extra, lead), dx, dz, dw, db,
                              workspace(bd.bimamba_group_norm_bwd_workspace_bytes(desc)))
    return dx, dz, dw, db


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "silu", "gate_before", "gate_after"])
@pytest.mark.parametrize("centred", [0, 1])
@pytest.mark.parametrize("B,L,G,n", SHAPES)
def test_gradients_of_groups(bd, B, L, G, n, centred, act, io):
    k = SHAPES.index((B, L, G, n)) + centred
    i = inputs(B, L, G, n, io, act, 11 * k + n)
    if k % 5 == 0:
        i["w" if k % 2 else "b"] = None
    extra = (0, 3, 8)[k % 3]
    _, mean, rstd = run_forward(bd, i, G, io, act, centred)
    got = run_backward(bd, i, G, io, act, centred, mean, rstd, extra, extra // 2)
    ref = gradient_ref(i, G, act, centred, mean.cpu() if centred else None, rstd.cpu())
    for name, a, r in zip(("dx", "dz", "dweight", "dbias"), got, ref):
        if r is not None:
            within(a, r, io if name in ("dx", "dz") else "f32")
    again = run_backward(bd, i, G, io, act, centred, mean, rstd, extra, extra // 2)
    assert all(a is None or torch.equal(a, b) for a, b in zip(got, again))
