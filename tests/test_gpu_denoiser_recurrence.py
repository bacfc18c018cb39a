"""The denoiser with the gated recurrence: its functions against plain torch, its gradients against differences of its loss, steps with
dropout, filling."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dn():
    from paper_2511_15927_amd import denoiser
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return denoiser


def batch(dn, model, seed, rows=4, seqlen=37):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tokens = dn.synthetic_tokens(rows, seqlen, model.vocab, gen)
    return tokens, model.noised(tokens, gen)


@pytest.mark.parametrize("mixer", ["recurrence", "mamba"])
def test_gradients_against_differences_along_directions(dn, mixer):
    """fp32, with dropout (its masks stay while the key does): the loss's slope along a random direction of each parameter.  The loss (order 4) is
    known to about 1e-6, so a step that moves it by 5e-3 shows the slope to 1e-3.  Central differences of the whole and of half the
    step, extrapolated, leave a fifth-order error."""
    model = dn.Denoiser(33, 32, 2, io="f32", seed=3, mixer=mixer, dropout=0.2)
    _, noised = batch(dn, model, 5)
    names, params = list(model.params), list(model.params.values())
    grads = torch.autograd.grad(model.loss(*noised), params)
    for k, (name, p, g) in enumerate(zip(names, params, grads)):
        gen = torch.Generator().manual_seed(k)
        d = torch.randn(p.shape, generator=gen).cuda() + 2 * g / g.abs().mean()
        slope = float((g.double() * d.double()).sum())
        h = 5e-3 / abs(slope)
        with torch.no_grad():
            keep = p.clone()
            differences = []
            for step in (h, h / 2):
                side = []
                for s in (step, -step):
                    p.copy_(keep + s * d)
                    side.append(float(model.loss(*noised)))
                differences.append((side[0] - side[1]) / (2 * step))
            p.copy_(keep)
        assert abs((4 * differences[1] - differences[0]) / 3 / slope - 1) < 1e-2, (name, differences, slope)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("L", [11, 200])
def test_a_block_against_plain_torch(dn, L, io):
    """recurrence in both directions, group_norm and dropout_add chained, against the same chain in 64 bits on the CPU, whose mask is that of
    dropout_add on ones."""
    gen = torch.Generator().manual_seed(7)
    t, B, D, G = dn.TYPE[io], 3, 24, 4
    x, gf, gb, z, res = (torch.randn(B, L, D, generator=gen).to(t) for _ in range(5))
    bf, bb, w, b = (torch.randn(D, generator=gen) for _ in range(4))
    gate, h0 = torch.randn(B, D, generator=gen), torch.randn(B, D, generator=gen)
    weight = torch.randn(B, L, D, generator=gen)
    key = torch.tensor([11, 5], device="cuda")
    ones = torch.empty(B, L, D, device="cuda")
    dn.bd.bimamba_dropout_add(dn.bd.make_dropout_desc(B, L, D, io="f32", p=0.25, site=2), key, torch.ones(B, L, D, device="cuda"), None, None, ones)
    leaves = [v.cuda().requires_grad_() for v in (x, gf, gb, z, res, bf, bb, w, b, gate, h0)]

    def chain(x, gf, gb, z, res, bf, bb, w, b, gate, h0):
        h, last = dn.recurrence(x, gf, bf, h_in=h0, want_state=True)
        h = dn.recurrence(x, gb, bb, add=h, reverse=True)
        return dn.dropout_add(dn.group_norm(h, z, w, b, G, centred=True), gate, res, key, 0.25, site=2), last

    def plain(x, gf, gb, z, res, bf, bb, w, b, gate, h0):
        def walk(x, a, h):
            hs = []
            for s in range(x.shape[1]):
                h = a[:, s] * h + (1 - a[:, s]) * x[:, s]
                hs.append(h)
            return torch.stack(hs, 1), h
        h, last = walk(x, torch.sigmoid(gf + bf), h0)
        h = h + walk(x.flip(1), torch.sigmoid(gb + bb).flip(1), torch.zeros_like(h0))[0].flip(1)
        u = (h * torch.nn.functional.silu(z)).view(B, L, G, -1)
        u = u - u.mean(-1, keepdim=True)
        n = (u / torch.sqrt((u * u).mean(-1, keepdim=True) + 1e-5)).view(B, L, D) * w + b
        return res + gate[:, None] * n * ones.cpu().double(), last

    out, last = chain(*leaves)
    got = torch.autograd.grad((out.float() * weight.cuda()).sum() + last.sum(), leaves)
    ref = [v.detach().cpu().double().requires_grad_() for v in leaves]
    rout, rlast = plain(*ref)
    want = torch.autograd.grad((rout * weight.double()).sum() + rlast.sum(), ref)
    out, rout = out.detach(), rout.detach()
    # fp32: some hundred roundings of 2^-24, more where the norm of a nearly flat group enlarges them; bf16: five activations and their gradients
    # are rounded to 2^-8 on the way
    tol = 2e-5 if io == "f32" else 6 * 2.0 ** -8
    assert float((out.cpu().double() - rout).norm() / rout.norm()) < tol
    for k, (g, r) in enumerate(zip(got, want)):
        assert g.shape == r.shape and float((g.cpu().double() - r).norm() / r.norm()) < tol, k


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("L", [9, 150])
def test_padded_sequences_with_log_gates_and_what_they_add_to(dn, L, reverse):
    """recurrence with lengths (0 and 1 among them): NaN behind them reaches neither the outputs nor a gradient."""
    gen = torch.Generator().manual_seed(13)
    B, D = 4, 12
    lengths = torch.tensor([L, 0, 1, L - 3])
    behind = torch.arange(L)[None, :, None] >= lengths[:, None, None]
    x, add, weight = (torch.randn(B, L, D, generator=gen) for _ in range(3))
    g, h0 = -torch.rand(B, L, D, generator=gen), torch.randn(B, D, generator=gen)
    leaves = [v.cuda().requires_grad_() for v in [torch.where(behind, math.nan, t) if t.dim() == 3 else t for t in (x, g, add, h0)]]
    y, last = dn.recurrence(leaves[0], leaves[1], None, leaves[2], leaves[3], lengths.cuda(), gate="log", reverse=reverse, want_state=True)
    got = torch.autograd.grad((y * weight.cuda()).sum() + (last * weight[:, 0].cuda()).sum(), leaves)

    rx, rg, radd, rh = ref = [v.double().requires_grad_() for v in (x, g, add, h0)]
    ys, ends = [], []
    for b, n in enumerate(lengths.tolist()):
        h, rows = rh[b], [torch.zeros(D, dtype=torch.float64)] * L
        for s in (reversed(range(n)) if reverse else range(n)):
            h = torch.exp(rg[b, s]) * h + rx[b, s]
            rows[s] = h + radd[b, s]
        ys.append(torch.stack(rows))
        ends.append(h)
    ry, rlast = torch.stack(ys), torch.stack(ends)
    want = torch.autograd.grad((ry * weight.double()).sum() + (rlast * weight[:, 0].double()).sum(), ref)
    for a, r in zip((y, last) + got, (ry.detach(), rlast.detach()) + want):   # fp32: some hundred roundings of 2^-24
        assert float((a.detach().cpu().double() - r).norm() / r.norm()) < 2e-5


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("mixer", ["recurrence", "mamba"])
def test_steps_with_dropout_and_filling(dn, mixer, io):
    model = dn.Denoiser(17, 64, 2, io=io, seed=1, mixer=mixer, dropout=0.1)
    gen = torch.Generator(device="cuda").manual_seed(2)
    for k in range(5):
        before = {n: p.detach().clone() for n, p in model.params.items()}
        loss, norm = model.train_step(dn.synthetic_tokens(16, 32, 17, gen), gen, lr=0.1)
        assert math.isfinite(float(loss)) and float(norm) > 0 and int(model.key[1]) == k + 1
        assert all(not torch.equal(p.detach(), before[n]) for n, p in model.params.items())
    tokens = dn.synthetic_tokens(3, 32, 17, gen)
    noised = tokens.clone()
    noised[0, ::2] = model.mask
    noised[1] = model.mask
    filled = model.fill(noised, per_step=5)
    kept = noised != model.mask
    assert not bool((filled == model.mask).any()) and torch.equal(filled[kept], tokens[kept])
    assert torch.equal(model.fill(noised, per_step=5), filled)


def test_dropout_changes_with_the_key_only_and_only_in_training(dn):
    model = dn.Denoiser(17, 32, 2, io="f32", seed=1, mixer="recurrence", dropout=0.3)
    tokens, level = torch.arange(34, device="cuda").view(2, 17) % 16, torch.tensor([0.3, 0.8], device="cuda")
    with torch.no_grad():
        a, b, still = model.logits(tokens, level, train=True), model.logits(tokens, level, train=True), model.logits(tokens, level)
        model.key[1] += 1
        assert torch.equal(a, b) and not torch.equal(a, model.logits(tokens, level, train=True)) and torch.equal(still, model.logits(tokens, level))


def test_a_key_that_moves_between_forward_and_backward_is_an_error(dn):
    x, key = torch.randn(2, 5, 8, device="cuda", requires_grad=True), torch.tensor([1, 2], device="cuda")
    out = dn.dropout_add(x, None, None, key, 0.5)
    key[1] += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_second_derivatives_are_refused(dn):
    gen = torch.Generator().manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=gen).cuda().requires_grad_()  # noqa: E731
    key = torch.tensor([1, 2], device="cuda")
    for leaves, call in (([r(2, 5, 12), r(2, 5, 12), r(12), r(2, 5, 12), r(2, 12)], dn.recurrence),
                         ([r(2, 5, 12), r(2, 5, 12), r(12), r(12)], lambda *a: dn.group_norm(*a, 3)),
                         ([r(2, 5, 12), r(2, 12), r(2, 5, 12)], lambda *a: dn.dropout_add(*a, key, 0.5))):
        got = torch.autograd.grad(call(*leaves).square().sum() + sum((t ** 3).sum() for t in leaves), leaves, create_graph=True)
        want = torch.autograd.grad(call(*leaves).square().sum() + sum((t ** 3).sum() for t in leaves), leaves)
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        for g, leaf in zip(got, leaves):
            with pytest.raises(RuntimeError, match="second derivative"):
                torch.autograd.grad(g.sum(), leaf, retain_graph=True)


def test_a_captured_step(dn):
    """Forward and backward of the recurrence model in a graph, the key moved inside it: each replay is the eager step of its key."""
    model = dn.Denoiser(33, 32, 2, io="f32", seed=3, mixer="recurrence", dropout=0.2)
    _, (noised, targets, level) = batch(dn, model, 5)
    params = list(model.params.values())

    def grads():
        model.key[1] += 1
        return torch.autograd.grad(model.loss(noised, targets, level), params)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        grads()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = grads()
    for offset in (7, 8, 40):
        model.key[1] = offset
        want = grads()
        model.key[1] = offset
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        # (the products are torch's, whose order of sums need not be the same twice)
        for a, b in zip(held, want):
            assert float((a - b).norm()) <= 1e-5 * float(b.norm()) + 1e-12
        assert int(model.key[1]) == offset + 1


@pytest.mark.parametrize("B,L", [(0, 5), (2, 0), (0, 0)])
def test_no_tokens(dn, B, L):
    """Outputs without elements, and gradients of zero for what is shared."""
    r = lambda *s: torch.randn(*s, device="cuda").requires_grad_()  # noqa: E731
    D, key = 12, torch.tensor([1, 2], device="cuda")
    x, g, bias, h_in, w, gate = r(B, L, D), r(B, L, D), r(D), r(B, D), r(D), r(D)
    h, last = dn.recurrence(x, g, bias, h_in=h_in, want_state=True)
    y = dn.dropout_add(dn.group_norm(h, g, w, None, 3), gate, x, key, 0.5)
    assert y.shape == (B, L, D) and torch.equal(last, h_in)
    grads = torch.autograd.grad(y.sum() + last.sum(), (x, g, bias, h_in, w, gate))
    assert torch.equal(grads[3], torch.ones_like(h_in)) and all(not bool(t.any()) for t in (grads[2], grads[4], grads[5]))
    assert grads[0].shape == grads[1].shape == (B, L, D)


def test_broadcast_and_expanded_gradients(dn):
    """The gradient of a sum is one number seen through strides of zero."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, g, w = (torch.randn(2, 70, 24, device="cuda", generator=gen).requires_grad_() for _ in range(3))
    key = torch.tensor([1, 2], device="cuda")
    for call in (lambda: dn.recurrence(x, g, add=w), lambda: dn.group_norm(x, g, None, None, 2), lambda: dn.dropout_add(x, None, w, key, 0.5)):
        leaves = [t for t in (x, g, w) if torch.autograd.grad(call().sum(), t, allow_unused=True)[0] is not None]
        one, two = torch.autograd.grad(call().sum(), leaves), torch.autograd.grad(call(), leaves, torch.ones(2, 70, 24, device="cuda"))
        assert all(torch.equal(a, b) for a, b in zip(one, two))
