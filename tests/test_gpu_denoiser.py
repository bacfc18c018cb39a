"""The denoiser that runs the library's calls together: its gradients against differences of its loss, a step that clips, training that
learns, filling that ends."""
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


def test_gradients_against_differences_along_directions(dn):
    """fp32: the loss's slope along a random direction of each parameter.  The loss (order 4) is known to about 1e-6, so a step that moves
    it by 5e-3 shows the slope to 1e-3.  Central differences of the whole and of half the step, extrapolated, leave a fifth-order error."""
    model = dn.Denoiser(33, 32, 2, io="f32", seed=3)
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
def test_functions_against_plain_torch(dn, io):
    """embed, layer_norm and log_probs chained, against the same chain in 64 bits on the CPU."""
    gen = torch.Generator().manual_seed(7)
    t, V, D = dn.TYPE[io], 50, 24
    table, w, b = torch.randn(V, D, generator=gen), 1 + 0.2 * torch.randn(3, D, generator=gen), 0.2 * torch.randn(3, D, generator=gen)
    head = (torch.randn(V, D, generator=gen) * 0.3).to(t)
    tokens, targets = torch.randint(0, V, (3, 11), generator=gen), torch.randint(-1, V, (3, 11), generator=gen)
    leaves = [x.cuda().requires_grad_() for x in (table, w, b)]
    x = dn.layer_norm(dn.embed(leaves[0], tokens.cuda(), 2.0, t), leaves[1], leaves[2])
    logits = (x.reshape(-1, D) @ head.cuda().t()).view(3, 11, V)
    logp, entropy = dn.log_probs(logits, targets.cuda(), want_entropy=True)
    loss = (logp * torch.linspace(0.5, 1.5, 11).cuda()).sum() + 0.3 * entropy.mean()
    got = torch.autograd.grad(loss, leaves)
    ref = [x.double().requires_grad_() for x in (table, w, b)]
    y = torch.nn.functional.layer_norm(ref[0][tokens] * 2.0, (D,), eps=1e-5) * ref[1][:, None] + ref[2][:, None]
    z = torch.log_softmax((y.reshape(-1, D) @ head.double().t()).view(3, 11, V), -1)
    rl = torch.where(targets >= 0, z.gather(-1, targets.clamp(min=0)[..., None])[..., 0], 0.0)
    rloss = (rl * torch.linspace(0.5, 1.5, 11).double()).sum() + 0.3 * -(z.exp() * z).sum(-1).mean()
    want = torch.autograd.grad(rloss, ref)
    # fp32: some hundred roundings of 2^-24; bf16: activations and their gradients are rounded to 2^-8 four times on the way
    tol = 1e-5 if io == "f32" else 4 * 2.0 ** -8
    for g, r in zip(got, want):
        assert float((g.cpu().double() - r).norm() / r.norm()) < tol
    assert abs(float(loss.detach()) - float(rloss.detach())) < tol * abs(float(rloss.detach()))


def test_a_step_clips_and_descends(dn):
    model = dn.Denoiser(33, 32, 2, io="f32", seed=3)
    tokens, _ = batch(dn, model, 5)
    gen = torch.Generator(device="cuda").manual_seed(9)
    before = {k: p.detach().clone() for k, p in model.params.items()}
    loss, norm = model.train_step(tokens, gen, lr=0.5, max_norm=0.01)
    assert math.isfinite(float(loss)) and float(norm) > 0.01
    moved = math.sqrt(sum(float((p.detach() - before[k]).double().square().sum()) for k, p in model.params.items()))
    assert abs(moved - 0.5 * 0.01) < 1e-3 * 0.5 * 0.01 + 1e-6   # the clipped norm times the step (parameters of order 1 round by 6e-8 each)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_training_learns_and_filling_ends(dn, io):
    model = dn.Denoiser(17, 64, 2, io=io, seed=1)
    gen = torch.Generator(device="cuda").manual_seed(2)
    losses = [model.train_step(dn.synthetic_tokens(16, 32, 17, gen), gen, lr=0.1)[0] for _ in range(60)]
    losses = [float(x) for x in losses]
    assert all(math.isfinite(x) for x in losses)
    assert sum(losses[-10:]) < 0.8 * sum(losses[:10]), (losses[:3], losses[-3:])
    tokens = dn.synthetic_tokens(3, 32, 17, gen)
    noised = tokens.clone()
    noised[0, ::2] = model.mask
    noised[1] = model.mask
    filled = model.fill(noised, per_step=5)
    assert not bool((filled == model.mask).any())
    kept = noised != model.mask
    assert torch.equal(filled[kept], tokens[kept])
    assert torch.equal(model.fill(noised, per_step=5), filled)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["ordinary", "equal", "far up", "far down", "ties far up", "lowest", "half lowest", "nothing"])
@pytest.mark.parametrize("V", [1, 9, 3001, 32001])
def test_gradient_of_log_probs_at_large_logits(dn, V, kind, io):
    """The gradient against the softmax of the logits in 64 bits: what is rounded away of a large log-sum-exp is not missing from the
    probabilities, and a row of nothing but the type's lowest value is uniform.  p is off, relatively, by what log S (a sum along a chain
    of V / 256 additions a lane, the lanes, waves and parts) and the differences of logits are rounded by; the entropy by the same twice,
    times what it is spread over."""
    gen, t, u = torch.Generator().manual_seed(V), dn.TYPE[io], 2.0 ** -24
    x = 3 * torch.randn(2, 3, V, generator=gen)
    low = torch.finfo(t).min
    if kind == "equal":
        x = torch.tensor([30000.0, -30000.0, 1e30, 70000.0, -1e6, 300.0]).view(2, 3, 1).expand(2, 3, V)
    elif kind == "far up":
        x = x + 30000.0
    elif kind == "far down":
        x = x - 1e6
    elif kind == "ties far up":
        x = torch.where(torch.arange(V) % 5 == 0, 65536.0, x)
    elif kind == "lowest":
        x = torch.full_like(x, low)
    elif kind == "half lowest":
        x = torch.where(torch.rand(2, 3, V, generator=gen) < 0.5, low, x)
    elif kind == "nothing":
        x = torch.full_like(x, -math.inf)
    x = x.to(t)
    targets = torch.randint(0, V, (2, 3), generator=gen)
    targets[0, 1] = -1
    dlogp, dentropy = torch.randn(2, 3, generator=gen), torch.randn(2, 3, generator=gen)
    leaf = x.cuda().requires_grad_()
    logp, entropy = dn.log_probs(leaf, targets.cuda(), want_entropy=True)
    got, = torch.autograd.grad((logp * dlogp.cuda()).sum() + (entropy * dentropy.cuda()).sum(), leaf)
    alone, = torch.autograd.grad((dn.log_probs(leaf, targets.cuda())[0] * dlogp.cuda()).sum(), leaf)
    if kind == "nothing":
        assert torch.equal(got, torch.zeros_like(got)) and torch.equal(alone, torch.zeros_like(alone))
        return
    d = x.double() - x.double().amax(-1, keepdim=True)
    log_s = torch.log(torch.exp(d).sum(-1, keepdim=True))
    lp = d - log_s
    p = torch.exp(lp)
    plp = torch.where(p > 0, p * lp, 0.0)
    H = -plp.sum(-1, keepdim=True)
    dl, de = torch.where(targets >= 0, dlogp, 0.0).double()[..., None], dentropy.double()[..., None]
    hit = torch.zeros_like(p).scatter(-1, targets.clamp(min=0)[..., None], 1.0)
    spread = (torch.exp(d) * d.abs().clamp(max=1e4)).sum(-1, keepdim=True) / torch.exp(log_s)
    unit = u * (48 + V / 256 + 4 * spread + 4 * log_s)
    rel = unit + u * (8 + 4 * lp.abs().clamp(max=1e3))
    first = dl * (hit - p)
    first_off = dl.abs() * p * rel + 2 * u * dl.abs() * (hit + p)
    inner = torch.where(p > 0, lp + H, 0.0)
    both = first - de * p * inner
    both_off = first_off + de.abs() * p * (inner.abs() * (rel + 4 * u) + rel + unit * (2 + 2 * spread) + 4 * u * (lp.abs().clamp(max=1e3) + H)) + 2 * u * both.abs()
    for g, r, off in ((got, both, both_off), (alone, first, first_off)):
        off = off + 1e-37 + (2.0 ** -8 * r.abs() if io == "bf16" else 0.0)
        g = g.double().cpu()
        assert bool(((g - r).abs() <= off).all()), float(((g - r).abs() / off).max())


@pytest.mark.parametrize("how", ["none", "others"])
def test_a_step_after_the_gradients_were_freed_or_replaced(dn, how):
    """What zero_grad() of an optimizer does between steps, or a gradient put in place by the program, changes nothing of a step."""
    model, same = (dn.Denoiser(33, 32, 2, io="f32", seed=3) for _ in range(2))
    tokens, _ = batch(dn, model, 5)
    norms = []
    for k in range(3):
        for m in (model, same):
            if m is model and k > 0:
                for p in m.params.values():
                    p.grad = None if how == "none" else torch.full_like(p, 7.0)
            before = {n: p.detach().clone() for n, p in m.params.items()}
            norms.append(float(m.train_step(tokens, torch.Generator(device="cuda").manual_seed(9 + k), lr=0.5, max_norm=0.01)[1]))
            moved = math.sqrt(sum(float((p.detach() - before[n]).double().square().sum()) for n, p in m.params.items()))
            assert norms[-1] > 0.01 and abs(moved - 0.5 * 0.01) < 1e-3 * 0.5 * 0.01 + 1e-6, (k, norms, moved)
    # (the products are torch's, whose order of sums need not be the same twice: three steps of a loss that is smooth)
    assert all(abs(a - b) <= 1e-4 * b for a, b in zip(norms[::2], norms[1::2])), norms
    # gradients that a hook takes away within the step are an error, not a step of nothing
    model.params["head"].register_post_accumulate_grad_hook(lambda p: setattr(p, "grad", None))
    with pytest.raises(RuntimeError, match="head"):
        model.train_step(tokens, torch.Generator(device="cuda").manual_seed(1))


def test_second_derivatives_are_refused(dn):
    """A gradient taken with create_graph is what it is without, and says so when it is itself differentiated: its terms through these
    functions are not there.  What does not go through them has its second derivatives."""
    gen = torch.Generator().manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=gen).cuda().requires_grad_()  # noqa: E731
    tokens = torch.randint(0, 7, (2, 5), generator=gen).cuda()
    cfg = dict(batch=2, seqlen=5, d_inner=8, d_state=16, n_heads=8, n_groups=1, d_conv=4, io="f32", a_kind=dn.bd.A_PER_HEAD_STATE,
               d_kind=dn.bd.D_PER_CHANNEL, dt_softplus=1, conv_bc=0, combine=dn.bd.COMBINE_ADD)
    side = lambda: dict(conv_w=r(8, 4), conv_b=r(8), A=(-torch.rand(8, 16, generator=gen)).cuda().requires_grad_(), D=r(8), dt_bias=r(8))  # noqa: E731
    sides = side(), side()
    mixed = [r(2, 5, 8) for _ in range(3)] + [r(2, 5, 16) for _ in range(2)]
    logits = r(2, 5, 7)
    for n, (leaves, call) in enumerate((([r(7, 12)], lambda t: dn.embed(t, tokens, 2.0, torch.float32)), ([r(2, 5, 12), r(2, 12), r(2, 12)], dn.layer_norm),
                         (mixed + [p for s in sides for p in s.values()],
                          lambda *a: dn.mixer(cfg, *a[:5], *(dict(zip(dn.PARAMS, a[5 + 5 * k:10 + 5 * k])) for k in (0, 1)))),
                         ([logits], lambda x: dn.log_probs(x, tokens)[0]), ([logits], lambda x: sum(dn.log_probs(x, tokens, True))))):
        other, linear = r(3), {0: 0, 1: 2}.get(n)   # (the place of what no first derivative depends on: a table, a bias)
        # (the first is linear in what comes out, so that the gradient that comes in is a constant; the leaves' cubes have second derivatives)
        losses = (lambda: call(*leaves).sum(), lambda: call(*leaves).square().sum())
        for loss in losses:
            total = lambda: loss() + sum((t ** 3).sum() for t in leaves) + (other ** 3).sum()  # noqa: E731
            want = torch.autograd.grad(total(), leaves)
            got = torch.autograd.grad(total(), leaves + [other], create_graph=True)
            assert all(torch.equal(a, b) for a, b in zip(want, got))
            second, = torch.autograd.grad(got[-1].sum(), other, retain_graph=True)
            assert torch.allclose(second, 6 * other)
            for k, leaf in enumerate(leaves):
                if k == linear and loss is losses[0]:   # (nothing is missing: there is none)
                    assert torch.allclose(torch.autograd.grad(got[k].sum(), leaf, retain_graph=True)[0], 6 * leaf)
                    continue
                with pytest.raises(RuntimeError, match="second derivative"):
                    torch.autograd.grad(got[k].sum(), leaf, retain_graph=True)


@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_a_step_whose_norm_is_not_finite_leaves_the_parameters(dn, value):
    model = dn.Denoiser(33, 32, 2, io="f32", seed=3)
    tokens, _ = batch(dn, model, 5)
    step = lambda seed: model.train_step(tokens, torch.Generator(device="cuda").manual_seed(seed), lr=0.5, max_norm=0.01)  # noqa: E731
    step(1)
    weight = model.params["0.in"]
    with torch.no_grad():
        kept = float(weight[3, 5])
        weight[3, 5] = value
    before = {k: p.detach().clone() for k, p in model.params.items()}
    assert not math.isfinite(float(step(2)[1]))
    assert all(torch.equal(p.detach().view(torch.int32), before[k].view(torch.int32)) for k, p in model.params.items())
    with torch.no_grad():
        weight[3, 5] = kept
    assert math.isfinite(float(step(3)[1])) and not torch.equal(weight, before["0.in"])
    assert all(bool(torch.isfinite(p).all()) for p in model.params.values())
