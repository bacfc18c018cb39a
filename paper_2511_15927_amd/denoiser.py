"""A small masked-diffusion denoiser around the library: a training step and block-wise denoising of a sequence.

    logits = head(norm(B_N(... B_1(E(tokens), tau) ..., tau))),   B(x, tau) = x + out_proj(Mixer(in_proj(AdaLN(x; tau))))

(the paper's eqs. 7-10 without the MLP).  The token table, the norms, the mixers, the log probabilities and the clipping are calls of
the library, forward and backward; the projections are plain matrix products of torch.  embed(), layer_norm(), mixer() and
log_probs() take part in autograd and can be used on their own; they have first derivatives only, and a gradient through them that is
itself differentiated is an error.

    python -m paper_2511_15927_amd.denoiser [--steps 200] [--width 256] [--layers 4] [--io bf16]

trains on synthetic sequences (runs of consecutive ids), then fills a masked sequence, the most confident places first.
"""
import argparse
import math

import torch

from . import binding as bd

NAME = {torch.float32: "f32", torch.bfloat16: "bf16"}
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _bytes(n, like):
    return torch.empty(max(n, 16), dtype=torch.uint8, device=like.device)


def _rows(t):
    """A gradient with unit stride along its channels, as the library reads them (any strides else)."""
    return t if t.stride(-1) == 1 else t.contiguous()


class _FirstOrder(torch.autograd.Function):
    """Gradients as they are, tied to what they depend on: differentiating them is an error, for the library has no second derivatives."""
    @staticmethod
    def forward(ctx, n, *tensors):
        return tuple(t.view_as(t) for t in tensors[:n])

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("embed, layer_norm, mixer and log_probs have no second derivatives")


def _first_order(grads, *sources):
    """The gradients that a backward pass returns, given all that they were computed from."""
    if not torch.is_grad_enabled():   # (it is with create_graph only)
        return grads
    at = [k for k, g in enumerate(grads) if g is not None]
    tied = _FirstOrder.apply(len(at), *(grads[k] for k in at), *(t for t in sources if t is not None))
    return tuple(tied[at.index(k)] if k in at else None for k in range(len(grads)))


class _Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, tokens, scale, io):
        (Bt, L), (V, D) = tokens.shape, table.shape
        ctx.desc = bd.make_embed_desc(Bt, L, D, V, table=NAME[table.dtype], io=NAME[io], scale=scale)
        ctx.save_for_backward(tokens)
        out = torch.empty(Bt, L, D, dtype=io, device=table.device)
        bd.bimamba_embed(ctx.desc, tokens, table, out)
        return out

    @staticmethod
    def backward(ctx, dout):
        tokens, = ctx.saved_tensors
        dtable = torch.empty(ctx.desc.vocab, ctx.desc.d_model, device=dout.device)
        bd.bimamba_embed_bwd(ctx.desc, tokens, _rows(dout), dtable, _bytes(bd.bimamba_embed_bwd_workspace_bytes(ctx.desc), dout))
        return _first_order((dtable, None, None, None), dout)


def embed(table, tokens, scale=1.0, io=torch.bfloat16):
    """scale * table[tokens] in the type io; table float32 [vocab, d], contiguous."""
    return _Embed.apply(table, tokens, scale, io)


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        Bt, L, D = x.shape
        ctx.desc = bd.make_norm_desc(Bt, L, D, io=NAME[x.dtype], eps=eps)
        y, mean, rstd = torch.empty(Bt, L, D, dtype=x.dtype, device=x.device), *torch.empty(2, Bt, L, device=x.device)
        bd.bimamba_layer_norm(ctx.desc, x, weight, bias, y, mean, rstd)
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dweight, dbias = torch.empty_like(x, memory_format=torch.contiguous_format), *torch.empty(2, *weight.shape, device=x.device)
        ws = _bytes(bd.bimamba_layer_norm_bwd_workspace_bytes(ctx.desc, weight.dim() == 2), x)
        bd.bimamba_layer_norm_bwd(ctx.desc, x, weight, mean, rstd, _rows(dy), dx, dweight, dbias, ws)
        return _first_order((dx, dweight, dbias, None), x, weight, dy)


def layer_norm(x, weight, bias, eps=1e-5):
    """x [batch, L, d]; weight and bias float32, [d] or a vector for each batch element [batch, d]."""
    return _LayerNorm.apply(x, weight, bias, eps)


PARAMS = ("conv_w", "conv_b", "A", "D", "dt_bias")


class _Mixer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, cfg, x, z, dt, B, C, *params):
        desc = bd.make_desc(cfg)
        pf, pb = (bd.make_params(dict(zip(PARAMS, p))) for p in (params[:5], params[5:]))
        out = bd.alloc_out(cfg, device=x.device)
        bd.bimamba_fwd(desc, pf, pb, bd.make_inputs(dict(x=x, z=z, dt=dt, B=B, C=C)), None, bd.make_tensor(out), bd.alloc_workspace(desc, device=x.device))
        ctx.cfg = cfg
        ctx.save_for_backward(x, z, dt, B, C, *params)
        return out

    @staticmethod
    def backward(ctx, dout):
        x, z, dt, B, C, *params = ctx.saved_tensors
        cfg, desc = ctx.cfg, bd.make_desc(ctx.cfg)
        pf, pb = (bd.make_params(dict(zip(PARAMS, p))) for p in (params[:5], params[5:]))
        grads = dict(dx=torch.empty_like(x, memory_format=torch.contiguous_format), dz=torch.empty_like(z, memory_format=torch.contiguous_format),
                     ddt=torch.empty_like(dt, memory_format=torch.contiguous_format))
        for k in ("dB", "dC"):
            grads[k] = torch.empty(cfg["batch"], cfg["seqlen"], cfg["n_groups"], cfg["d_state"], device=x.device)
        dpar = [{"d" + k: torch.empty_like(p) for k, p in zip(PARAMS, ps)} for ps in (params[:5], params[5:])]
        bd.bimamba_bwd(desc, pf, pb, bd.make_inputs(dict(x=x, z=z, dt=dt, B=B, C=C)), None, bd.make_tensor(_rows(dout)), bd.make_input_grads(grads),
                       None, bd.make_param_grads(dpar[0]), bd.make_param_grads(dpar[1]), _bytes(bd.bimamba_bwd_workspace_bytes(desc), x))
        dB, dC = (grads[k].view(B.shape).to(B.dtype) for k in ("dB", "dC"))
        return _first_order((None, grads["dx"], grads["dz"], grads["ddt"], dB, dC, *(d["d" + k] for d in dpar for k in PARAMS)), x, z, dt, B, C, *params, dout)


def mixer(cfg, x, z, dt, B, C, pf, pb):
    """The mixer of a config dict (selective-scan layout, as synth.mixer_cfg makes it, dt_softplus 1); pf, pb: dicts of PARAMS."""
    return _Mixer.apply(cfg, x, z, dt, B, C, *(p[k] for p in (pf, pb) for k in PARAMS))


class _LogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, want_entropy):
        Bt, L, V = logits.shape
        ctx.desc = bd.make_logits_desc(Bt, L, V, io=NAME[logits.dtype], targets_only=int(not want_entropy))
        out = {k: torch.empty(Bt, L, device=logits.device) for k in ("logp", "lse", "lse_rest") + (("entropy",) if want_entropy else ())}
        bd.bimamba_log_probs(ctx.desc, logits, targets, out, _bytes(bd.bimamba_log_probs_workspace_bytes(ctx.desc), logits))
        ctx.save_for_backward(logits, targets, out["lse"], out["lse_rest"], out.get("entropy"))
        return out["logp"], out.get("entropy")

    @staticmethod
    def backward(ctx, dlogp, dentropy):
        logits, targets, lse, lse_rest, entropy = ctx.saved_tensors
        dlogits = torch.empty_like(logits, memory_format=torch.contiguous_format)
        bd.bimamba_log_probs_bwd(ctx.desc, logits, targets, lse, entropy, dlogp.contiguous(), None if entropy is None else dentropy.contiguous(), dlogits,
                                 lse_rest=lse_rest)
        return _first_order((dlogits, None, None), logits, dlogp, dentropy)


def log_probs(logits, targets, want_entropy=False):
    """(log probability of each target, entropy of each row or None); 0 where a target lies outside the vocabulary, and such rows are not
    read unless the entropy is wanted."""
    return _LogProbs.apply(logits, targets, want_entropy)


class Denoiser:
    """Parameters are float32 tensors in a dict; activations are of the type `io`.  The last id of the vocabulary is the mask."""
    FEATURES = 64   # of the noise level

    def __init__(self, vocab, width, layers, d_state=16, io="bf16", seed=0, device="cuda"):
        self.vocab, self.width, self.layers, self.d_state, self.io, self.mask = vocab, width, layers, d_state, TYPE[io], vocab - 1
        gen = torch.Generator().manual_seed(seed)
        D, Dn, N = width, 2 * width, d_state
        normal = lambda *s, scale: scale * torch.randn(*s, generator=gen)  # noqa: E731
        p = dict(table=normal(vocab, D, scale=D ** -0.5), norm_w=torch.ones(D), norm_b=torch.zeros(D), head=normal(vocab, D, scale=D ** -0.5))
        for l in range(layers):
            p["%d.cond" % l] = normal(2 * D, self.FEATURES, scale=0.02)
            p["%d.in" % l] = normal(2 * Dn, D, scale=D ** -0.5)               # x | z
            p["%d.ssm" % l] = normal(Dn + 2 * N, D, scale=D ** -0.5)          # dt | B | C
            p["%d.out" % l] = normal(D, Dn, scale=0.5 * Dn ** -0.5)
            for s in "fb":
                dt = torch.exp(torch.empty(Dn).uniform_(math.log(1e-3), math.log(1e-1), generator=gen))
                p.update({"%d.%s.conv_w" % (l, s): normal(Dn, 4, scale=0.5), "%d.%s.conv_b" % (l, s): torch.zeros(Dn),
                          "%d.%s.A_log" % (l, s): torch.log(torch.arange(1, N + 1).float()).repeat(Dn, 1), "%d.%s.D" % (l, s): torch.ones(Dn),
                          "%d.%s.dt_bias" % (l, s): torch.log(torch.expm1(dt))})
        self.params = {k: t.to(device).requires_grad_() for k, t in p.items()}
        self._clip = None   # made with the first step: the table of the gradients, which stay where they are, their norm, the workspace

    def _linear(self, x, name):
        """x [batch, L, n] times a weight's transpose, as one plain matrix product."""
        w = self.params[name].to(self.io)
        return (x.reshape(-1, x.shape[-1]) @ w.t()).view(*x.shape[:-1], w.shape[0])

    def logits(self, tokens, level):
        """Logits [batch, L, vocab] of tokens [batch, L] (the mask's is -inf) at noise levels [batch] in (0, 1]."""
        p, D, Dn, N = self.params, self.width, 2 * self.width, self.d_state
        Bt, L = tokens.shape
        cfg = dict(batch=Bt, seqlen=L, d_inner=Dn, d_state=N, n_heads=Dn, n_groups=1, d_conv=4, io=NAME[self.io], a_kind=bd.A_PER_HEAD_STATE,
                   d_kind=bd.D_PER_CHANNEL, dt_softplus=1, conv_bc=0, combine=bd.COMBINE_ADD)
        angle = level[:, None] * torch.exp(torch.linspace(0.0, 5.0, self.FEATURES // 2, device=level.device))
        feature = torch.cat([torch.cos(angle), torch.sin(angle)], 1)
        x = embed(p["table"], tokens, math.sqrt(D), self.io)
        for l in range(self.layers):
            cond = feature @ p["%d.cond" % l].t()
            gain, shift = (cond + torch.cat([torch.ones(D), torch.zeros(D)]).to(cond)).split(D, 1)   # column slices of one projection
            y = layer_norm(x, gain, shift)
            xs, z = self._linear(y, "%d.in" % l).split(Dn, 2)
            dt, B, C = self._linear(y, "%d.ssm" % l).split([Dn, N, N], 2)
            side = [dict(conv_w=p["%d.%s.conv_w" % (l, s)], conv_b=p["%d.%s.conv_b" % (l, s)], A=-torch.exp(p["%d.%s.A_log" % (l, s)]),
                         D=p["%d.%s.D" % (l, s)], dt_bias=p["%d.%s.dt_bias" % (l, s)]) for s in "fb"]
            x = x + self._linear(mixer(cfg, xs, z, dt, B, C, *side), "%d.out" % l)
        logits = self._linear(layer_norm(x, p["norm_w"], p["norm_b"]), "head")
        never = torch.zeros(self.vocab, dtype=self.io, device=logits.device)
        never[self.mask] = -math.inf
        return logits + never

    def noised(self, tokens, gen):
        """(noised tokens, targets, levels): each sequence's tokens are masked with a probability of its own; -1 where none is."""
        level = 0.05 + 0.95 * torch.rand(tokens.shape[0], device=tokens.device, generator=gen)
        hidden = torch.rand(tokens.shape, device=tokens.device, generator=gen) < level[:, None]
        return torch.where(hidden, self.mask, tokens), torch.where(hidden, tokens, -1), level

    def loss(self, noised, targets, level):
        """The masked-diffusion bound per token: -log p of the masked tokens, each weighted by 1 / level."""
        logp, _ = log_probs(self.logits(noised, level), targets)
        return -(logp / level[:, None]).sum() / noised.numel()

    def train_step(self, tokens, gen, lr=0.05, max_norm=1.0):
        """One step of gradient descent with clipping on clean tokens [batch, L].  Returns the loss and the gradients' norm (on the device).
        Where the norm is not finite the parameters stay as they are.  Each parameter's .grad is the model's own tensor, the same in every step, and afterwards holds the clipped gradient."""
        params = list(self.params.values())
        if self._clip is None:
            for p in params:
                p.grad = torch.zeros_like(p)
            table = bd.GradTable([p.grad for p in params])
            self._clip = table, torch.empty(1, device=tokens.device), _bytes(bd.bimamba_clip_grads_workspace_bytes(table), tokens)
        table, norm, ws = self._clip
        for p, g in zip(params, table.grads):
            p.grad = g   # (what the program has made of it since: freed it, put another in its place)
        torch._foreach_zero_(table.grads)
        loss = self.loss(*self.noised(tokens, gen))
        loss.backward()
        for (name, p), g in zip(self.params.items(), table.grads):
            if p.grad is not g:
                raise RuntimeError("the gradient of %s was replaced within the step" % name)
        bd.bimamba_clip_grads(table, max_norm, norm, ws)
        with torch.no_grad():   # (a norm that is not finite: nothing moves; told on the device, so that nothing is waited for)
            torch._fused_sgd_(params, table.grads, [], weight_decay=0.0, momentum=0.0, lr=lr, dampening=0.0, nesterov=False, maximize=False,
                              is_first_step=False, found_inf=(~torch.isfinite(norm)).float())
        return loss.detach(), norm

    @torch.no_grad()
    def fill(self, tokens, per_step=8):
        """Masked places of tokens [batch, L] are filled, in every step the `per_step` of each sequence whose most probable token has the
        largest log probability, less a millionth of the entropy: of equal ones the least uncertain come first."""
        tokens = tokens.clone()
        Bt, L = tokens.shape
        desc = bd.make_logits_desc(Bt, L, self.vocab, io=NAME[self.io], top_k=1)
        ws = _bytes(bd.bimamba_log_probs_workspace_bytes(desc), tokens)
        out = dict(entropy=torch.empty(Bt, L, device=tokens.device), top_logp=torch.empty(Bt, L, 1, device=tokens.device),
                   top_token=torch.empty(Bt, L, 1, dtype=torch.int64, device=tokens.device))
        for left in range(int((tokens == self.mask).sum(1).max()), 0, -per_step):
            hidden = tokens == self.mask
            bd.bimamba_log_probs(desc, self.logits(tokens, hidden.float().mean(1)), None, out, ws)
            rank = torch.where(hidden, out["top_logp"][..., 0] - 1e-6 * out["entropy"], -math.inf)
            best = rank.topk(min(per_step, left), 1).indices
            chosen = torch.zeros_like(hidden).scatter(1, best, True) & hidden
            tokens = torch.where(chosen, out["top_token"][..., 0], tokens)
        return tokens


def synthetic_tokens(batch, seqlen, vocab, gen, device="cuda"):
    """Sequences that count upwards from a random id (modulo the ids that are not the mask)."""
    start = torch.randint(0, vocab - 1, (batch, 1), device=device, generator=gen)
    return (start + torch.arange(seqlen, device=device)) % (vocab - 1)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--seqlen", type=int, default=64)
    ap.add_argument("--vocab", type=int, default=65)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--io", choices=("f32", "bf16"), default="bf16")
    a = ap.parse_args(argv)
    model = Denoiser(a.vocab, a.width, a.layers, io=a.io)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for step in range(a.steps):
        loss, norm = model.train_step(synthetic_tokens(a.batch, a.seqlen, a.vocab, gen), gen)
        if step % 20 == 0 or step == a.steps - 1:
            print("step %4d  loss %.4f  gradient norm %.3f" % (step, float(loss), float(norm)), flush=True)
    clean = synthetic_tokens(4, a.seqlen, a.vocab, gen)
    noised = clean.clone()
    noised[:, 1::2] = model.mask
    filled = model.fill(noised)
    print("filled %d of %d masked tokens as they were" % (int((filled == clean)[:, 1::2].sum()), clean[:, 1::2].numel()))


if __name__ == "__main__":
    main()
