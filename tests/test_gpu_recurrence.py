"""The gated linear recurrence and its gradients through the C ABI, against a walk in 64 bits on the CPU with a running error bound."""
import pytest
import torch

from running_error import TYPES, U32, Run, blank, cuda, gen, nans, normal, scan, wide, within, workspace

pytestmark = pytest.mark.gpu

KEEP = 64


@pytest.fixture(scope="module")
def bd():
    from paper_2511_15927_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return binding


def inputs(B, L, D, io, gate, seed, lengths=False):
    g = gen(seed)
    memory = torch.exp(torch.rand(D, generator=g) * 6)
    raw = normal(g, B, L, D, scale=0.7)
    return dict(x=normal(g, B, L, D, io=io), g=(raw if gate == "sigmoid" else 0.02 - torch.exp(raw) / memory).to(TYPES[io]),
                bias=torch.log(memory) if gate == "sigmoid" else None, h_in=normal(g, B, D), add=normal(g, B, L, D, io=io),
                dy=normal(g, B, L, D, io=io), dh_out=normal(g, B, D),
                lengths=torch.randint(-1, L + 2, (B,), generator=g) if lengths else None)


def walk(i, gate, reverse):
    """The gate's values and x in the order of the walk, with their errors; where each step's token lies; which steps count."""
    B, L, D = i["x"].shape
    length = torch.full((B,), L) if i["lengths"] is None else i["lengths"].clamp(0, L)
    s = torch.arange(L).expand(B, L)
    inside = s < length[:, None]
    place = torch.where(inside, length[:, None] - 1 - s, s) if reverse else s
    at = place[..., None].expand(B, L, D)
    take = lambda t: t.double().gather(1, at)  # noqa: E731
    x, g = take(i["x"]), take(i["g"])
    if gate == "sigmoid":
        v = Run(g) + (i["bias"].double() if i["bias"] is not None else torch.zeros(D))
        low = torch.sigmoid(-v.v.abs())
        low_off = low * (1.1 * v.e + U32 * (3 * v.v.abs() + 8))
        up = v.v > 0
        a, q = torch.where(up, 1 - low, low), torch.where(up, low, 1 - low)
        a_off, q_off = low_off + U32 * torch.where(up, a, 0), low_off + U32 * torch.where(up, 0, q)
        if i["x"].dtype == torch.bfloat16:
            # e = exp(-v), a = 1 / (1 + e), q = e a.  e is off by r = 1.1 v.e + U32 (3 |v| + 4) of itself (the product with log2 e, exp2's unit in the last
            # place), which moves 1 + e by q r of itself and e / (1 + e) by a r; the sum adds U32, the reciprocal one unit in the last place,
            # 2 U32, the last product U32.  (Below v = -87 a stays at 2^-126.)
            r = 1.1 * v.e + U32 * (3 * v.v.abs() + 4)
            a, q = torch.sigmoid(v.v), torch.sigmoid(-v.v)
            a_off, q_off = a * (q * r + 3 * U32) + 1.2e-38, q * (a * r + 4 * U32)
        u, u_off = q * x, q_off * x.abs() + U32 * (q * x).abs()
    else:
        cut = g.clamp(max=0.0)
        a = torch.exp(cut)
        a_off, u, u_off = a * U32 * (3 * cut.abs() + 3) + 1e-38, x, torch.zeros_like(x)
        q, q_off = torch.where(g > 0, 0.0, a), torch.where(g > 0, 0.0, a_off)
    m = inside[..., None]
    z = lambda t: torch.where(m, t, 0.0)  # noqa: E731
    return dict(a=torch.where(m, a, 1.0), a_off=z(a_off), q=Run(z(q), z(q_off)), u=z(u), u_off=z(u_off), x=z(x), m=m, at=at, take=take)


def back_in_place(r, w):
    """Values of the steps at their tokens, zeros behind the ends."""
    z = torch.zeros_like(r.v)
    return Run(z.scatter(1, w["at"], torch.where(w["m"], r.v, 0.0)), z.scatter(1, w["at"], torch.where(w["m"], r.e, 0.0)))


def forward_ref(i, gate, reverse, h_in, add):
    w = walk(i, gate, reverse)
    B, L, D = i["x"].shape
    before, _, last = scan(w["a"], w["a_off"], w["u"], w["u_off"], i["h_in"] if h_in else torch.zeros(B, D))
    h = Run(torch.cat([before.v[:, 1:], last.v[:, None]], 1), torch.cat([before.e[:, 1:], last.e[:, None]], 1))
    if add:
        h = h + w["take"](i["add"])
    return back_in_place(h, w), last, before[:, ::KEEP]


def run_forward(bd, i, io, gate, reverse, h_in=True, add=True, states=True, extra=0, lead=0, y=None):
    B, L, D = i["x"].shape
    desc = bd.make_recurrence_desc(B, L, D, io=io, gate=gate, reverse=reverse)
    out = dict(y=blank((B, L, D), io, extra, lead) if y is None else y, h_out=nans(B, D), states=nans(B, (L + KEEP - 1) // KEEP, D) if states else None)
    bd.bimamba_recurrence(desc, wide(i["x"], extra, lead), wide(i["g"], extra, extra - lead), cuda(i["bias"]), out["y"],
                          add=wide(i["add"], extra, lead) if add else None, lengths=cuda(i["lengths"]), h_in=cuda(i["h_in"]) if h_in else None,
                          h_out=out["h_out"], states=out["states"], workspace=workspace(bd.bimamba_recurrence_workspace_bytes(desc)))
    return out


SHAPES = [(1, 1, 1), (3, 1, 130), (2, 2, 3), (3, 5, 7), (1, 16, 64), (1, 17, 2), (2, 31, 96), (1, 64, 128), (2, 65, 129), (2, 128, 66),
          (1, 200, 257), (5, 129, 33), (1, 1237, 74), (2, 1030, 64), (70, 3, 40), (1, 2500, 5)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["log", "sigmoid"])
@pytest.mark.parametrize("reverse", [0, 1])
@pytest.mark.parametrize("B,L,D", SHAPES)
def test_states_of_a_walk(bd, B, L, D, reverse, gate, io):
    n = SHAPES.index((B, L, D)) + reverse
    lengths, h_in, add, extra = n % 3 == 0, n % 2 == 0, n % 4 < 2, (0, 3, 8)[n % 3]
    i = inputs(B, L, D, io, gate, 100 * n + L, lengths)
    if gate == "sigmoid" and n % 5 == 0:
        i["bias"] = None
    out = run_forward(bd, i, io, gate, reverse, h_in, add, True, extra, extra // 2)
    y, last, kept = forward_ref(i, gate, reverse, h_in, add)
    within(out["y"], y, io)
    within(out["h_out"], last)
    within(out["states"], kept)


def gradient_ref(i, gate, reverse, states):
    w = walk(i, gate, reverse)
    B, L, D = i["x"].shape
    before, size, _ = scan(w["a"], w["a_off"], w["u"], w["u_off"], states[:, 0])
    dy = torch.where(w["m"], w["take"](i["dy"]), 0.0)
    # q of a step = a (dy + q of the step after it): a walk from the other end whose input is a dy
    flip = lambda t: t.flip(1)  # noqa: E731
    into = (w["a"] * dy, w["a_off"] * dy.abs() + U32 * (w["a"] * dy).abs())
    q, q_size, dh_in = scan(flip(w["a"]), flip(w["a_off"]), flip(into[0]), flip(into[1]), i["dh_out"])
    after, after_size = Run(flip(q.v), flip(q.e)), flip(q_size)
    dh = Run(dy + after.v, after.e + 2 * U32 * (dy.abs() + after_size))
    before = Run(before.v, before.e + U32 * size)
    if gate == "sigmoid":
        dx = dh * w["q"]
        dg = dx * (before - w["x"]) * Run(w["a"], w["a_off"])
    else:
        dx, dg = dh, dh * before * w["q"]
    m = w["m"]
    dg = Run(torch.where(m, dg.v, 0.0), torch.where(m, dg.e, 0.0))
    return back_in_place(dx, w), back_in_place(dg, w), dg.view(B * L, D).sum(0, B * L), dh_in


def run_backward(bd, i, io, gate, reverse, states, extra=0, lead=0, stateful=True):
    B, L, D = i["x"].shape
    desc = bd.make_recurrence_desc(B, L, D, io=io, gate=gate, reverse=reverse)
    out = dict(dx=blank((B, L, D), io, extra, lead), dg=blank((B, L, D), io, extra, lead), dbias=nans(D) if gate == "sigmoid" else None,
               dh_in=nans(B, D) if stateful else None)
    bd.bimamba_recurrence_bwd(desc, wide(i["x"], extra, lead), wide(i["g"], extra, lead), cuda(i["bias"]), states, wide(i["dy"], extra, lead), out["dx"],
                              out["dg"], dbias=out["dbias"], lengths=cuda(i["lengths"]), dh_out=cuda(i["dh_out"]) if stateful else None,
                              dh_in=out["dh_in"], workspace=workspace(bd.bimamba_recurrence_bwd_workspace_bytes(desc)))
    return out


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["log", "sigmoid"])
@pytest.mark.parametrize("reverse", [0, 1])
@pytest.mark.parametrize("B,L,D", SHAPES)
def test_gradients_of_a_walk(bd, B, L, D, reverse, gate, io):
    """The kept states come from the call itself; the reference takes the state before the first step from them and is exact from there."""
    n = SHAPES.index((B, L, D)) + reverse
    extra = (0, 3, 8)[n % 3]
    i = inputs(B, L, D, io, gate, 300 * n + L, n % 3 == 1)
    states = run_forward(bd, i, io, gate, reverse)["states"]
    out = run_backward(bd, i, io, gate, reverse, states, extra, extra // 2)
    dx, dg, dbias, dh_in = gradient_ref(i, gate, reverse, states.cpu())
    within(out["dx"], dx, io)
    within(out["dg"], dg, io)
    within(out["dh_in"], dh_in)
    if gate == "sigmoid":
        within(out["dbias"], dbias)
    again = run_backward(bd, i, io, gate, reverse, states, extra, extra // 2)
    for k in out:
        assert out[k] is None or torch.equal(out[k], again[k]), k
