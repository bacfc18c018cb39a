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
