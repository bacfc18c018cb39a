"""Calls of the gated recurrence, the group norm and dropout as programs make them: in blocks and single tokens, in place, on views of all
kinds, padded, on other streams, captured and replayed."""
import math

import pytest
import torch

from running_error import TYPES, Run, blank, cuda, gen, nans, normal, wide, within, workspace
from test_gpu_recurrence import KEEP, bd, forward_ref, gradient_ref, inputs, run_backward, run_forward  # noqa: F401

pytestmark = pytest.mark.gpu


def equal(a, b):
    return torch.equal(a.view(torch.int16 if a.dtype == torch.bfloat16 else torch.int32), b.view(torch.int16 if b.dtype == torch.bfloat16 else torch.int32))


# ---- the recurrence ----

@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["log", "sigmoid"])
def test_blocks_and_single_tokens_go_on_where_the_last_call_stopped(bd, gate, io):
    cuts = [32, 1, 1, 3, 64, 200, 129, 5]
    B, L, D = 3, sum(cuts), 150
    i = inputs(B, L, D, io, gate, 5)
    y, last, _ = forward_ref(i, gate, 0, True, False)
    h, at = i["h_in"].cuda(), 0
    x, g, out = i["x"].cuda(), i["g"].cuda(), torch.empty(B, L, D, dtype=TYPES[io], device="cuda")
    for n in cuts:
        desc = bd.make_recurrence_desc(B, n, D, io=io, gate=gate)
        bd.bimamba_recurrence(desc, x[:, at:at + n], g[:, at:at + n], cuda(i["bias"]), out[:, at:at + n], h_in=h, h_out=h,
                              workspace=workspace(bd.bimamba_recurrence_workspace_bytes(desc)))
        at += n
    within(out, y, io)
    within(h, last)


@pytest.mark.parametrize("L", [20, 50, 300, 2000])
def test_two_directions_added_in_place(bd, L):
    i, j = (inputs(2, L, 131, "f32", "sigmoid", s) for s in (7, 8))
    forward = run_forward(bd, i, "f32", "sigmoid", 0, add=False)["y"]
    desc = bd.make_recurrence_desc(2, L, 131, io="f32", reverse=1)
    both = forward.clone()
    ws = workspace(bd.bimamba_recurrence_workspace_bytes(desc))
    bd.bimamba_recurrence(desc, j["x"].cuda(), j["g"].cuda(), cuda(j["bias"]), both, add=both, h_in=j["h_in"].cuda(), workspace=ws)
    apart = torch.empty_like(both)
    bd.bimamba_recurrence(desc, j["x"].cuda(), j["g"].cuda(), cuda(j["bias"]), apart, add=forward, h_in=j["h_in"].cuda(), workspace=ws)
    assert equal(both, apart)
    a, b = forward_ref(i, "sigmoid", 0, True, False)[0], forward_ref(j, "sigmoid", 1, True, False)[0]
    within(both, a + b)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("reverse", [0, 1])
@pytest.mark.parametrize("L,D", [(5, 9), (40, 130), (700, 66)])
def test_what_lies_behind_a_sequences_end_is_not_looked_at(bd, L, D, reverse, io):
    i = inputs(4, L, D, io, "sigmoid", L)
    i["lengths"] = torch.tensor([0, 1, L - 1, L // 2])
    behind = torch.arange(L)[None, :] >= i["lengths"][:, None]
    j = dict(i)
    for k in ("x", "g", "dy", "add"):
        i[k], j[k] = i[k].clone(), i[k].clone()
        i[k][behind] = 0.0
        j[k][behind] = math.nan if k != "g" else math.inf
    runs = [run_forward(bd, k, io, "sigmoid", reverse, extra=6, lead=4) for k in (i, j)]
    assert all(equal(runs[0][k], runs[1][k]) for k in runs[0])
    assert not bool(runs[1]["y"][behind.cuda()].any()) and equal(runs[1]["h_out"][0], i["h_in"][0].cuda())
    grads = [run_backward(bd, k, io, "sigmoid", reverse, runs[0]["states"]) for k in (i, j)]
    assert all(equal(grads[0][k], grads[1][k]) for k in grads[0])
    assert not bool(grads[1]["dx"][behind.cuda()].any()) and not bool(grads[1]["dg"][behind.cuda()].any())
    assert equal(grads[1]["dh_in"][0], i["dh_out"][0].cuda())


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("L,D", [(1, 3), (3, 64), (30, 65), (130, 131), (600, 7)])
def test_nothing_is_written_beside_the_rows(bd, L, D, io):
    i = inputs(2, L, D, io, "sigmoid", L + D)
    buf = torch.full((2, L + 2, D + 6), 7.0, dtype=TYPES[io], device="cuda")
    y = buf[:, 1:L + 1, 3:D + 3]
    out = run_forward(bd, i, io, "sigmoid", 1, y=y)
    assert equal(y.contiguous(), run_forward(bd, i, io, "sigmoid", 1)["y"])
    y.fill_(7.0)
    assert bool((buf == 7.0).all())
    grads = [torch.full((2, L + 2, D + 6), 7.0, dtype=TYPES[io], device="cuda") for _ in range(2)]
    views = [b[:, 1:L + 1, 3:D + 3] for b in grads]
    desc = bd.make_recurrence_desc(2, L, D, io=io, reverse=1)
    bd.bimamba_recurrence_bwd(desc, i["x"].cuda(), i["g"].cuda(), cuda(i["bias"]), out["states"], i["dy"].cuda(), *views,
                              workspace=workspace(bd.bimamba_recurrence_bwd_workspace_bytes(desc)))
    for v, b in zip(views, grads):
        assert not bool((v == 7.0).all())
        v.fill_(7.0)
        assert bool((b == 7.0).all())


@pytest.mark.parametrize("L", [3, 31, 300])
def test_gates_at_their_ends(bd, L):
    """A factor of exactly 0 forgets, one of exactly 1 keeps; a log gate above 0 is one of 0 and has no gradient."""
    D = 70
    x = normal(gen(L), 1, L, D)
    h0 = normal(gen(9), 1, D)
    run = lambda g, gate, **kw: run_forward(bd, dict(x=x, g=g.expand(1, L, D), bias=None, h_in=h0, lengths=None, add=None), "f32", gate, 0, add=False, **kw)  # noqa: E731
    assert equal(run(torch.tensor(-math.inf), "log")["y"], x.cuda())
    for g in (0.0, -0.0, 5.0, math.inf):
        out = run(torch.tensor(g), "log")["y"]
        walk = [h0[:, :]]
        for t in range(L):
            walk.append(walk[-1].double() + x[:, t].double())
        within(out, Run(torch.stack(walk[1:], 1), 2 * L * 2.0 ** -24 * (h0.abs().double()[:, None] + x.abs().double().cumsum(1))))
    assert equal(run(torch.tensor(-math.inf), "sigmoid")["y"], x.cuda())
    assert equal(run(torch.tensor(math.inf), "sigmoid")["y"], h0[:, None].expand(1, L, D).contiguous().cuda())
    i = dict(inputs(1, L, D, "f32", "log", 3))
    i["g"] = torch.where(torch.arange(D) % 2 == 0, 3.0, i["g"])
    states = run_forward(bd, i, "f32", "log", 0)["states"]
    assert not bool(run_backward(bd, i, "f32", "log", 0, states)["dg"][..., ::2].any())


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("L,at", [(40, 17), (900, 500)])
def test_a_value_that_is_not_finite_stays_in_its_channel_and_after_its_token(bd, L, at, value):
    i = inputs(2, L, 70, "f32", "sigmoid", L)
    clean = run_forward(bd, i, "f32", "sigmoid", 0)
    i["x"][1, at, 33] = value
    out = run_forward(bd, i, "f32", "sigmoid", 0)
    assert not bool(torch.isfinite(out["y"][1, at:, 33]).any()) and not bool(torch.isfinite(out["h_out"][1, 33]))
    for o in (clean, out):
        o["y"][1, at:, 33] = 0.0
        o["h_out"][1, 33] = 0.0
        o["states"][1, at // KEEP + 1:, 33] = 0.0
    assert all(equal(clean[k], out[k]) for k in clean)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_views_in_any_order(bd, io):
    """Tokens before batch elements, one row for all batch elements, columns of one buffer: the same bits as contiguous ones."""
    B, L, D = 3, 210, 72
    i = inputs(B, L, D, io, "sigmoid", 4)
    i["add"] = i["add"][:1].expand(B, L, D).contiguous()
    want = run_forward(bd, i, io, "sigmoid", 0)
    desc = bd.make_recurrence_desc(B, L, D, io=io)
    x = i["x"].transpose(0, 1).contiguous().cuda().transpose(0, 1)
    both = torch.empty(B, L, 2 * D + 5, dtype=TYPES[io], device="cuda")   # g | y
    both[..., :D] = i["g"].cuda()
    y = both[..., D + 2:2 * D + 2]
    bd.bimamba_recurrence(desc, x, both[..., :D], cuda(i["bias"]), y, add=i["add"][:1].cuda().expand(B, L, D), h_in=cuda(i["h_in"]),
                          workspace=workspace(bd.bimamba_recurrence_workspace_bytes(desc)))
    assert equal(y.contiguous(), want["y"]) and equal(both[..., :D].contiguous(), i["g"].cuda())


def test_no_tokens(bd):
    h, z = normal(gen(1), 2, 9).cuda(), torch.empty(2, 0, 9, device="cuda")
    desc = bd.make_recurrence_desc(2, 0, 9, io="f32")
    out = nans(2, 9)
    bd.bimamba_recurrence(desc, z, z, None, z, h_in=h, h_out=out)
    assert equal(out, h)
    bd.bimamba_recurrence(desc, z, z, None, z, h_out=out)
    assert equal(out, torch.zeros(2, 9, device="cuda"))
    dbias, dh = nans(9), nans(2, 9)
    bd.bimamba_recurrence_bwd(desc, z, z, None, torch.empty(2, 0, 9, device="cuda"), z, z, z, dbias=dbias, dh_out=h, dh_in=dh)
    assert equal(dh, h) and not bool(dbias.any())


def test_rows_further_apart_than_32_bits_reach(bd):
    """Batch elements 2^32 + 8 elements apart (17 GB of bf16, of which only the rows are touched), and what they are made of in a tight buffer."""
    B, L, D, far = 2, 150, 140, (1 << 32) + 8
    i = inputs(B, L, D, "bf16", "sigmoid", 6)
    want = run_forward(bd, i, "bf16", "sigmoid", 1)
    spread = [torch.empty(far + L * D, dtype=torch.bfloat16, device="cuda").as_strided((B, L, D), (far, D, 1)) for _ in range(2)]
    spread[0].copy_(i["x"])
    desc = bd.make_recurrence_desc(B, L, D, reverse=1)
    bd.bimamba_recurrence(desc, spread[0], i["g"].cuda(), cuda(i["bias"]), spread[1], add=i["add"].cuda(), h_in=i["h_in"].cuda(),
                          workspace=workspace(bd.bimamba_recurrence_workspace_bytes(desc)))
    assert equal(spread[1].contiguous(), want["y"])
    ndesc = bd.make_group_norm_desc(B, L, D, 5, act="gate_after")
    tight = torch.empty(B, L, D, dtype=torch.bfloat16, device="cuda")
    bd.bimamba_group_norm(ndesc, i["x"].cuda(), i["g"].cuda(), None, None, tight)
    bd.bimamba_group_norm(ndesc, spread[0], i["g"].cuda(), None, None, spread[1])
    assert equal(spread[1].contiguous(), tight)
    ddesc, key = bd.make_dropout_desc(B, L, D), torch.tensor([1, 2], device="cuda")
    bd.bimamba_dropout_add(ddesc, key, i["x"].cuda(), None, None, tight)
    bd.bimamba_dropout_add(ddesc, key, spread[0], None, None, spread[1])
    assert equal(spread[1].contiguous(), tight)


@pytest.mark.parametrize("B,L,D,io", [(1, 20000, 70, "bf16"), (3, 3000, 200, "f32"), (40, 700, 300, "bf16"), (2, 4000, 1100, "bf16")])
def test_the_same_bits_whenever_the_pieces_come(bd, B, L, D, io):
    """Many calls, beside other work on another stream: what a piece finds of those before it differs from call to call, the result must not."""
    i = inputs(B, L, D, io, "sigmoid", L)
    first = run_forward(bd, i, io, "sigmoid", 0, extra=3, lead=1)
    grads = run_backward(bd, i, io, "sigmoid", 0, first["states"])
    side, noise = torch.cuda.Stream(), torch.randn(2048, 2048, device="cuda")
    for n in range(6):
        with torch.cuda.stream(side):
            for _ in range(n):
                noise = noise @ noise * 0.01
        out = run_forward(bd, i, io, "sigmoid", 0, extra=3, lead=1)
        back = run_backward(bd, i, io, "sigmoid", 0, out["states"])
        assert all(equal(first[k], out[k]) for k in first) and all(equal(grads[k], back[k]) for k in grads)
    torch.cuda.synchronize()


def step_calls(bd, B, L, D, G, io, ws=None):
    """A block's forward and backward calls on buffers of their own, as one function; what it fills."""
    t = TYPES[io]
    e = lambda *s, dtype=t: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    f = torch.float32
    b = dict(x=e(B, L, D), g=e(B, L, D), z=e(B, L, D), bias=e(D, dtype=f), w=e(D, dtype=f), dout=e(B, L, D), key=e(2, dtype=torch.int64), residual=e(B, L, D),
             gate=e(B, D, dtype=f))
    o = dict(h=e(B, L, D), both=e(B, L, D), sf=e(B, (L + KEEP - 1) // KEEP, D, dtype=f), sb=e(B, (L + KEEP - 1) // KEEP, D, dtype=f), n=e(B, L, D),
             rstd=e(B, L, G, dtype=f), out=e(B, L, D), dn=e(B, L, D), dgate=e(B, D, dtype=f), dh=e(B, L, D), dz=e(B, L, D), dw=e(D, dtype=f), db=e(D, dtype=f),
             dxf=e(B, L, D), dgf=e(B, L, D), dxb=e(B, L, D), dgb=e(B, L, D), dbias=e(D, dtype=f))
    df, dr = (bd.make_recurrence_desc(B, L, D, io=io, reverse=k) for k in (0, 1))
    dn, dd = bd.make_group_norm_desc(B, L, D, G, io=io, act="gate_before"), bd.make_dropout_desc(B, L, D, io=io, p=0.2, site=4)
    need = max(bd.bimamba_recurrence_workspace_bytes(df), bd.bimamba_recurrence_bwd_workspace_bytes(df), bd.bimamba_group_norm_bwd_workspace_bytes(dn),
               bd.bimamba_dropout_add_bwd_workspace_bytes(dd, True))
    ws = workspace(need) if ws is None else ws

    def step():
        bd.bimamba_recurrence(df, b["x"], b["g"], b["bias"], o["h"], states=o["sf"], workspace=ws)
        bd.bimamba_recurrence(dr, b["x"], b["g"], b["bias"], o["both"], add=o["h"], states=o["sb"], workspace=ws)
        bd.bimamba_group_norm(dn, o["both"], b["z"], b["w"], None, o["n"], None, o["rstd"])
        bd.bimamba_dropout_add(dd, b["key"], o["n"], b["gate"], b["residual"], o["out"])
        bd.bimamba_dropout_add_bwd(dd, b["key"], o["n"], b["gate"], b["dout"], o["dn"], o["dgate"], ws)
        bd.bimamba_group_norm_bwd(dn, o["both"], b["z"], b["w"], None, None, o["rstd"], o["dn"], o["dh"], o["dz"], o["dw"], o["db"], ws)
        bd.bimamba_recurrence_bwd(df, b["x"], b["g"], b["bias"], o["sf"], o["dh"], o["dxf"], o["dgf"], dbias=o["dbias"], workspace=ws)
        bd.bimamba_recurrence_bwd(dr, b["x"], b["g"], b["bias"], o["sb"], o["dh"], o["dxb"], o["dgb"], workspace=ws)
    return step, b, o, ws


def fill(b, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    for k, t in b.items():
        t.copy_(torch.randint(-1 << 40, 1 << 40, t.shape, device="cuda", generator=g) if k == "key" else torch.randn(t.shape, device="cuda", generator=g))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,D,G", [(2, 40, 96, 3), (1, 700, 260, 4), (3, 300, 128, 2)])
def test_a_captured_step_replayed_and_two_graphs_that_share_a_workspace(bd, B, L, D, G, io):
    step, b, o, ws = step_calls(bd, B, L, D, G, io)
    other, b2, o2, _ = step_calls(bd, B, L // 2 + 1, D, G, io, ws=ws)
    graphs = []
    for s, buf in ((step, b), (other, b2)):
        fill(buf, 1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            s()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s()
        graphs.append(graph)
    for seed in (2, 3, 4):
        for s, buf, out, graph in ((step, b, o, graphs[0]), (other, b2, o2, graphs[1])):
            fill(buf, seed)
            s()
            want = {k: v.clone() for k, v in out.items()}
            for v in out.values():
                v.zero_()
            torch.cuda.synchronize()
            graph.replay()
            assert all(equal(out[k], want[k]) for k in out), seed
            graph.replay()
            graphs[0].replay()
            torch.cuda.synchronize()
            assert all(equal(out[k], want[k]) for k in out), seed


def test_on_other_streams(bd):
    """Two steps at once, each on a stream and a workspace of its own."""
    pairs = [step_calls(bd, 2, 900, 300, 4, "bf16") for _ in range(2)]
    wants = []
    for n, (step, b, o, _) in enumerate(pairs):
        fill(b, n)
        step()
        wants.append({k: v.clone() for k, v in o.items()})
        for v in o.values():
            v.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pairs]
    for _ in range(3):
        for s, (step, _, _, _) in zip(streams, pairs):
            with torch.cuda.stream(s):
                step()
    torch.cuda.synchronize()
    for want, (_, _, o, _) in zip(wants, pairs):
        assert all(equal(o[k], want[k]) for k in o)
    # (a stream that is handed over, not the current one)
    step, b, o, _ = pairs[0]
    key, out = b["key"], torch.empty_like(o["n"])
    desc = bd.make_dropout_desc(2, 900, 300, p=0.2, site=4)
    bd.bimamba_dropout_add(desc, key, o["n"], b["gate"], b["residual"], out, stream=streams[1])
    torch.cuda.synchronize()
    assert equal(out, o["out"])


# ---- the group norm ----

@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("G,n", [(3, 5), (2, 37), (7, 64), (1, 1500), (1, 5000)])
def test_norms_leave_what_is_beside_the_rows(bd, G, n, io):
    B, L, D = 2, 7, G * n
    g = gen(n)
    x, z, dy = (normal(g, B, L, D, io=io) for _ in range(3))
    desc = bd.make_group_norm_desc(B, L, D, G, io=io, act="gate_before", centred=1)
    bufs = [torch.full((B, L + 2, D + 6), 7.0, dtype=TYPES[io], device="cuda") for _ in range(3)]
    y, dx, dz = (b[:, 1:L + 1, 3:D + 3] for b in bufs)
    mean, rstd, dw, db = nans(B, L, G), nans(B, L, G), nans(D), nans(D)
    bd.bimamba_group_norm(desc, x.cuda(), z.cuda(), None, None, y, mean, rstd)
    bd.bimamba_group_norm_bwd(desc, x.cuda(), z.cuda(), None, None, mean, rstd, dy.cuda(), dx, dz, dw, db,
                              workspace(bd.bimamba_group_norm_bwd_workspace_bytes(desc)))
    for v, b in zip((y, dx, dz), bufs):
        assert not bool((v == 7.0).all())
        v.fill_(7.0)
        assert bool((b == 7.0).all())
    assert all(bool(torch.isfinite(t).all()) for t in (mean, rstd, dw, db))


def test_norm_of_a_large_mean_and_of_nothing(bd):
    """A mean 4000 times the deviation costs the squares no digits; a group of zeros has rstd 1 / sqrt(eps) and gives the bias."""
    x = (4000.0 + torch.randn(1, 6, 256, generator=gen(2))).cuda()
    desc = bd.make_group_norm_desc(1, 6, 256, 2, io="f32", centred=1)
    y, mean, rstd = torch.empty_like(x), nans(1, 6, 2), nans(1, 6, 2)
    bd.bimamba_group_norm(desc, x, None, None, None, y, mean, rstd)
    d = x.cpu().double().view(1, 6, 2, 128)
    want = d.var(-1, correction=0).add(1e-5) ** -0.5
    # (the mean is off by some 2^-24 * 4000 * 12, which the squares around it see squared; the rest as for any group)
    assert float((rstd.cpu().double() / want - 1).abs().max()) < 1e-5
    zero, bias = torch.zeros(1, 6, 256, device="cuda"), normal(gen(3), 256).cuda()
    for act in ("none", "gate_before"):
        desc = bd.make_group_norm_desc(1, 6, 256, 2, io="f32", act=act)
        bd.bimamba_group_norm(desc, zero, zero if act != "none" else None, None, bias, y, None, rstd)
        assert equal(y, bias.expand(1, 6, 256).contiguous()) and float((rstd * math.sqrt(1e-5) - 1).abs().max()) < 1e-6


def test_a_row_that_is_not_finite_stays_by_itself(bd):
    g = gen(4)
    x, z, dy = (normal(g, 2, 40, 96).cuda() for _ in range(3))
    desc = bd.make_group_norm_desc(2, 40, 96, 3, io="f32", act="gate_after")

    def run(x):
        y, rstd, dx, dz = torch.empty_like(x), nans(2, 40, 3), torch.empty_like(x), torch.empty_like(x)
        bd.bimamba_group_norm(desc, x, z, None, None, y, None, rstd)
        bd.bimamba_group_norm_bwd(desc, x, z, None, None, None, rstd, dy, dx, dz, None, None, None)
        return y, dx, dz
    clean = run(x)
    bad = x.clone()
    bad[1, 17, 40] = math.nan
    for a, b in zip(clean, run(bad)):
        assert not bool(torch.isfinite(b[1, 17, 32:64]).any())
        b[1, 17, 32:64] = a[1, 17, 32:64]
        assert equal(a, b)


# ---- dropout ----

@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("D", [5, 64, 130, 700])
def test_dropout_in_place_and_beside(bd, D, io):
    g = gen(D)
    x, residual, dout = (normal(g, 3, 33, D, io=io).cuda() for _ in range(3))
    gate, key, desc = normal(g, 3, D).cuda(), torch.tensor([3, 4], device="cuda"), bd.make_dropout_desc(3, 33, D, io=io, p=0.3, site=1)
    apart = torch.empty_like(x)
    bd.bimamba_dropout_add(desc, key, x, gate, residual, apart)
    buf = torch.full((3, 35, D + 6), 7.0, dtype=TYPES[io], device="cuda")
    v = buf[:, 1:34, 3:D + 3]
    v.copy_(residual)
    bd.bimamba_dropout_add(desc, key, x, gate, v, v)
    assert equal(v.contiguous(), apart)
    dx, dgate, dgate2, ws = torch.empty_like(x), nans(3, D), nans(3, D), workspace(bd.bimamba_dropout_add_bwd_workspace_bytes(desc, True))
    bd.bimamba_dropout_add_bwd(desc, key, x, gate, dout, dx, dgate, ws)
    v.copy_(dout)
    bd.bimamba_dropout_add_bwd(desc, key, x, gate, v, v, dgate2, ws)
    assert equal(v.contiguous(), dx) and equal(dgate, dgate2)
    v.fill_(7.0)
    assert bool((buf == 7.0).all())


def test_what_is_dropped_is_not_read_into_the_result(bd):
    key, desc = torch.tensor([8, 1], device="cuda"), bd.make_dropout_desc(2, 50, 72, io="f32", p=0.5)
    ones, residual = torch.ones(2, 50, 72, device="cuda"), normal(gen(6), 2, 50, 72).cuda()
    mask = torch.empty_like(ones)
    bd.bimamba_dropout_add(desc, key, ones, None, None, mask)
    x = torch.where(mask > 0, ones, math.nan)
    out, dx, dgate = torch.empty_like(x), torch.empty_like(x), nans(72)
    bd.bimamba_dropout_add(desc, key, x, None, residual, out)
    assert equal(out, torch.where(mask > 0, residual + 2.0, residual))
    bd.bimamba_dropout_add_bwd(desc, key, x, torch.ones(72, device="cuda"), x, dx, dgate, workspace(bd.bimamba_dropout_add_bwd_workspace_bytes(desc, False)))
    assert equal(dx, torch.where(mask > 0, 2.0, 0.0)) and equal(dgate, (mask > 0).float().sum((0, 1)) * 2)


def test_masks_go_by_key_and_site_and_not_by_layout(bd):
    ones = torch.ones(4, 30, 40, device="cuda")
    made = lambda key, site, B=4, L=30: bd.bimamba_dropout_add(  # noqa: E731
        bd.make_dropout_desc(B, L, 40, io="f32", p=0.5, site=site), torch.tensor(key, device="cuda"), ones.view(B, L, 40), None, None, out.view(B, L, 40))
    out = torch.empty_like(ones)
    seen = []
    for key, site in (([1, 2], 0), ([1, 3], 0), ([2, 2], 0), ([1, 2], 1), ([1, 2 + (1 << 32)], 0), ([1 + (1 << 32), 2], 0)):
        made(key, site)
        assert all(not torch.equal(out, s) for s in seen)
        seen.append(out.clone())
    made([1, 2], 0, 2, 60)   # (rows are counted through the batch)
    assert torch.equal(out, seen[0])


@pytest.mark.parametrize("D", [3, 130])
def test_sums_over_thousands_of_workgroups(bd, D):
    """More than 2048 slots, whose sums are made in two steps: dbias, dweight and dgate are the sums of what the calls give for each token.  No value
    passes 300 additions on its way, each off by 2^-24 of the magnitudes; a slot left out would be off by 1 / 2400."""
    def near(got, terms):
        terms = terms.double().flatten(0, 1)
        assert bool(((got.double() - terms.sum(0)).abs() <= 300 * 2.0 ** -24 * terms.abs().sum(0)).all())

    def r(*s, seed=3):
        return torch.randn(*s, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    room = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")  # noqa: E731
    B, L = 2100, 3
    desc = bd.make_recurrence_desc(B, L, D, io="f32")
    x, g, dy, bias = r(B, L, D), r(B, L, D, seed=4), r(B, L, D, seed=5), r(D)
    y, dx, dg, states, dbias = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty(B, 1, D, device="cuda"), torch.empty(D, device="cuda")
    bd.bimamba_recurrence(desc, x, g, bias, y, states=states, workspace=room(bd.bimamba_recurrence_workspace_bytes(desc)))
    bd.bimamba_recurrence_bwd(desc, x, g, bias, states, dy, dx, dg, dbias=dbias, workspace=room(bd.bimamba_recurrence_bwd_workspace_bytes(desc)))
    near(dbias, dg)

    B, L = 2, 300000 if D == 3 else 36000
    desc = bd.make_group_norm_desc(B, L, D, 1, io="f32", act="none")
    need = bd.bimamba_group_norm_bwd_workspace_bytes(desc)
    assert need >= 2048 * 2 * D * 4
    x, dy, w = r(B, L, D), r(B, L, D, seed=4), r(D)
    y, dx, rstd, dweight, dbias = torch.empty_like(x), torch.empty_like(x), torch.empty(B, L, 1, device="cuda"), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    bd.bimamba_group_norm(desc, x, None, w, None, y, None, rstd)
    bd.bimamba_group_norm_bwd(desc, x, None, w, None, None, rstd, dy, dx, None, dweight, dbias, room(need))
    near(dbias, dy)
    near(dweight, dy.double() * x.double() * rstd.double())

    B, L = 1, 1100000 if D == 3 else 70000
    desc = bd.make_dropout_desc(B, L, D, io="f32", p=0.25)
    need = bd.bimamba_dropout_add_bwd_workspace_bytes(desc, False)
    assert need >= 2048 * D * 4
    key, gate = torch.tensor([5, 6], device="cuda"), torch.ones(D, device="cuda")
    x, dout = r(B, L, D), r(B, L, D, seed=4)
    kept, dx, dgate = torch.empty_like(x), torch.empty_like(x), torch.empty(D, device="cuda")
    bd.bimamba_dropout_add(desc, key, x, None, None, kept)
    bd.bimamba_dropout_add_bwd(desc, key, x, gate, dout, dx, dgate, room(need))
    near(dgate, kept.double() * dout.double())


# ---- more work than the chip holds at once, in the other sizes of pieces ----

MUCH = [(1100, 70, 66), (200, 200, 66), (300, 140, 33), (400, 150, 66), (70, 300, 66), (350, 300, 66), (300, 500, 66)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,D", MUCH)
def test_walks_of_much_work(bd, B, L, D, io):
    n = MUCH.index((B, L, D)) + (io == "bf16")
    gate, reverse = ("sigmoid", "log")[n // 2 % 2], n % 2
    i = inputs(B, L, D, io, gate, 500 + n, n % 3 == 0)
    out = run_forward(bd, i, io, gate, reverse, add=n % 4 != 1)
    y, last, kept = forward_ref(i, gate, reverse, True, n % 4 != 1)
    within(out["y"], y, io)
    within(out["h_out"], last)
    within(out["states"], kept)
    back = run_backward(bd, i, io, gate, reverse, out["states"])
    dx, dg, dbias, dh_in = gradient_ref(i, gate, reverse, out["states"].cpu())
    within(back["dx"], dx, io)
    within(back["dg"], dg, io)
    within(back["dh_in"], dh_in)
    if gate == "sigmoid":
        within(back["dbias"], dbias)
    again = run_forward(bd, i, io, gate, reverse, add=n % 4 != 1), run_backward(bd, i, io, gate, reverse, out["states"])
    for one, two in ((out, again[0]), (back, again[1])):
        assert all(v is None or torch.equal(v, two[k]) for k, v in one.items())
