"""What the operators around the mixer are timed on: the two ends of a masked-diffusion denoiser, its normalisation and the
clipping of its gradients, at the sizes that training and block decoding give them.

Kinds of case, each one pass through one entry point:
  embed        bimamba_embed: rows of the token table, scaled
  embed_bwd    bimamba_embed_bwd: the table's gradient (of a noised sequence a share `masked` is one and the same id)
  norm         bimamba_layer_norm: layer norm with a weight and a bias, each batch element's own (`modulated`) or shared
  norm_bwd     bimamba_layer_norm_bwd: its gradients
  scores       bimamba_log_probs: log probabilities of given tokens, entropy and the `top` most probable tokens
  scores_bwd   bimamba_log_probs_bwd: the gradient of log probabilities (and, with `entropy`, of the entropies) for the logits
  clip         bimamba_clip_grads: the norm of a model's gradients, and the gradients scaled to at most `max_norm`
Fields: `io` is the type of activations, logits and gradients, `table` that of the token table; `packed`: an activation is a
column slice of a wider buffer; `masked`: the share of tokens that are the mask token, which alone carry a target.
"""
import math

import torch

own = False

_BASE = dict(kind="embed", batch=1, seqlen=32, width=2048, vocab=50304, io="bf16", table="f32", packed=0, modulated=0, masked=0.5,
             top=0, entropy=0, layers=1)
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MAX_NORM = 1.0
EPS = 1e-5


def _case(name=None, **kw):
    c = dict(_BASE, **kw)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # a denoising step of block decoding: 16 blocks of 32 tokens enter the stack
        _case("embed_block", batch=16, seqlen=32),
        # training: the table's gradient of 32768 tokens, half of them masked
        _case("embed_grad", kind="embed_bwd", batch=8, seqlen=4096),
        # training a small fp32 model on ragged sequences
        _case("embed_grad_ragged", kind="embed_bwd", batch=3, seqlen=1237, width=740, vocab=32001, io="f32", masked=0.3),
        # one of a block's normalisations in a decoding step
        _case("norm_block", kind="norm", batch=16, seqlen=32, modulated=1),
        # the same in training at the length of the benchmark's headline
        _case("norm_train", kind="norm", batch=8, seqlen=8192, modulated=1),
        # its gradients, the conditioning's among them
        _case("norm_grad", kind="norm_bwd", batch=8, seqlen=8192, modulated=1),
        # gradients in a small fp32 model whose rows are slices of a wider buffer
        _case("norm_grad_ragged", kind="norm_bwd", batch=3, seqlen=1237, width=740, io="f32", packed=1),
        # decoding one sequence: confidence, entropy and eight candidates for each of a block's 32 tokens
        _case("scores_block", kind="scores", batch=1, seqlen=32, top=8, entropy=1),
        # training: the log probabilities that the loss sums, of the masked half of 16384 tokens
        _case("scores_train", kind="scores", batch=8, seqlen=2048),
        # the loss's gradient for the logits of the same step, the largest amount of data here
        _case("scores_grad", kind="scores_bwd", batch=8, seqlen=2048),
        # clipping the gradients of a toy model's mixers (both directions: conv, A, D and their biases)
        _case("clip_toy", kind="clip", width=256, layers=4),
        # clipping those of 24 layers with their projections
        _case("clip_model", kind="clip", width=2048, layers=24, io="bf16"),
    ]


_MOST_VALUES = 8 * 2048 * 50304   # logits of the largest listed call


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed_bwd", "norm", "norm_bwd", "scores", "scores", "scores_bwd", "clip"])
    c = dict(kind=kind, io=rng.choice(["bf16", "bf16", "f32"]), width=_log_int(rng, 128, 4096))
    if rng.random() < 0.6:
        c["width"] = max(8, c["width"] // 8 * 8)
    if kind == "clip":
        c.update(layers=rng.randint(1, 24), width=min(c["width"], 2048))
        return _case(**c)
    c.update(batch=_log_int(rng, 1, 32), seqlen=_log_int(rng, 1, 8192), packed=rng.randint(0, 1), masked=round(rng.uniform(0.05, 1.0), 3))
    if kind in ("norm", "norm_bwd"):
        c["modulated"] = rng.randint(0, 1)
    else:
        c["vocab"] = _log_int(rng, 500, 130000)
    if kind in ("embed", "embed_bwd"):
        c["table"] = rng.choice(["f32", "bf16"]) if kind == "embed" else "f32"
    if kind in ("scores", "scores_bwd"):
        c["entropy"] = rng.randint(0, 1)
        c["top"] = rng.choice([0, 1, 4, 8]) if kind == "scores" else 0
    # (a pass in its plain form that sorts whole rows for the alternatives takes far longer than one that does not)
    room = _MOST_VALUES // (4 if c["io"] == "f32" else 2) // (16 if c.get("top") else 1)
    wide = c["vocab"] if kind in ("scores", "scores_bwd") else c["width"] * 4
    c["seqlen"] = max(1, min(c["seqlen"], room // (c["batch"] * wide)))
    return _case(**c)


def _clip_shapes(c):
    """Gradients of `layers` mixer layers of two directions: the library's fp32 parameter gradients and, from a width of 512,
    those of the projections in the model's type."""
    d = 2 * c["width"]
    small = [(d, 4), (d,), (d, 16), (d,), (d,)] * (2 * c["layers"])
    large = [(c["width"], 2 * d), (d, c["width"])] * c["layers"] if c["width"] >= 512 else []
    return small, large


def _numels(shapes):
    return [math.prod(s) for s in shapes]


def _gradients(shapes, dtype, gen, scale):
    """Tensors of these shapes, and as many for the clipped ones, which are views of one buffer."""
    numels = _numels(shapes)
    total = sum(numels)
    flat = torch.empty(total, dtype=dtype, device="cuda")
    return ([(scale * torch.randn(s, device="cuda", generator=gen)).to(dtype) for s in shapes],
            [v.view(s) for v, s in zip(flat.split(numels), shapes)] if total else [], flat)


def _rows(c, gen, width, scale=1.0):
    io = _TYPES[c["io"]]
    pitch = width + (width // 2 // 8 * 8 if c["packed"] else 0)
    wide = torch.empty(c["batch"], c["seqlen"], pitch, dtype=io, device="cuda")
    wide.normal_(0.0, scale, generator=gen)
    return wide[..., pitch - width:]


def _tokens(c, gen):
    """Ids as a noised sequence has them: a share `masked` is the mask token (the last id), the others fall off as words do."""
    shape, V = (c["batch"], c["seqlen"]), c["vocab"]
    u = torch.rand(shape, device="cuda", generator=gen)
    clean = (torch.exp(u * math.log(V)) - 1).long().clamp_(0, V - 2)
    hidden = torch.rand(shape, device="cuda", generator=gen) < c["masked"]
    return clean, hidden


def prepare(case, seed):
    c = dict(_BASE, **case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    Bt, L, D, V, io = c["batch"], c["seqlen"], c["width"], c["vocab"], _TYPES[c["io"]]
    s = dict(c=c, kind=c["kind"])

    def normal(*shape, scale=1.0):
        return scale * torch.randn(*shape, device="cuda", generator=gen)

    if c["kind"] == "clip":
        small, large = _clip_shapes(c)
        s["small"], s["small_to"], s["small_flat"] = _gradients(small, torch.float32, gen, 0.02)
        s["large"], s["large_to"], s["large_flat"] = _gradients(large, io, gen, 0.001)
        return s
    if c["kind"] in ("embed", "embed_bwd"):
        clean, hidden = _tokens(c, gen)
        s["tokens"] = torch.where(hidden, V - 1, clean)
        s["scale"] = float(math.sqrt(D))
        if c["kind"] == "embed":
            s["table"] = normal(V, D, scale=0.02).to(_TYPES[c["table"]])
        else:
            s["dout"] = _rows(c, gen, D, 1e-3)
        return s
    if c["kind"] in ("norm", "norm_bwd"):
        s["x"] = _rows(c, gen, D, 2.0)
        s["x"] += 0.3
        rows = (Bt,) if c["modulated"] else ()
        s["weight"], s["bias"] = 1 + normal(*rows, D, scale=0.2), normal(*rows, D, scale=0.2)
        if c["kind"] == "norm_bwd":
            x = s["x"].float()
            s["mean"] = x.mean(-1)
            s["rstd"] = torch.rsqrt((x - s["mean"][..., None]).square().mean(-1) + EPS)
            s["dy"] = _rows(c, gen, D, 1e-2)
        return s
    s["logits"] = _rows(c, gen, V, 2.5)
    s["logits"][..., V - 1] = -math.inf   # the mask is never predicted
    clean, hidden = _tokens(c, gen)
    s["targets"] = torch.where(hidden, clean, -1)
    if c["kind"] == "scores_bwd":
        x = s["logits"].double() if s["logits"].numel() < 1 << 24 else s["logits"].float()
        s["lse"] = torch.logsumexp(x, -1).float()
        s["entropy"] = (s["lse"] - (torch.exp(x - s["lse"][..., None]) * x.clamp(min=-1e30)).sum(-1)).float() if c["entropy"] else None
        s["dlogp"] = -torch.rand(Bt, L, device="cuda", generator=gen) / (Bt * L)
        s["dentropy"] = normal(Bt, L, scale=0.1 / (Bt * L)) if c["entropy"] else None
    return s


def _plain(s):
    c, kind = s["c"], s["kind"]
    io = _TYPES[c["io"]]
    if kind == "embed":
        return (s["table"][s["tokens"]].float() * s["scale"]).to(io)
    if kind == "embed_bwd":
        dtable = torch.zeros(c["vocab"], c["width"], device="cuda")
        return dtable.index_add_(0, s["tokens"].reshape(-1), s["dout"].float().reshape(-1, c["width"]) * s["scale"])
    if kind in ("norm", "norm_bwd"):
        weight, bias = (s[k][:, None] if c["modulated"] else s[k] for k in ("weight", "bias"))
        x = s["x"].float()
        if kind == "norm":
            mean = x.mean(-1, keepdim=True)
            x = x - mean
            rstd = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
            return dict(y=(x * rstd * weight + bias).to(io), mean=mean[..., 0], rstd=rstd[..., 0])
        rstd, dy = s["rstd"][..., None], s["dy"].float()
        x = (x - s["mean"][..., None]) * rstd
        g = dy * weight
        dx = rstd * (g - g.mean(-1, keepdim=True) - x * (g * x).mean(-1, keepdim=True))
        over = 1 if c["modulated"] else (0, 1)
        return dict(dx=dx.to(io), dweight=(dy * x).sum(over), dbias=dy.sum(over))
    if kind == "clip":
        squares = torch.stack([g.float().square().sum() for g in s["small"] + s["large"]])
        norm = torch.sqrt(squares.sum())
        scale = torch.clamp(MAX_NORM / norm, max=1.0)
        [to.copy_(g.float() * scale) for g, to in zip(s["small"] + s["large"], s["small_to"] + s["large_to"])]
        return dict(norm=norm, small=s["small_flat"], large=s["large_flat"])
    x, has = s["logits"].float(), s["targets"] >= 0
    target = s["targets"].clamp(min=0)[..., None]
    if kind == "scores":
        if not (c["entropy"] or c["top"]):   # training: rows without a target are not asked for
            top = x.amax(-1, keepdim=True)
            lse = top + torch.log(torch.exp(x - top).sum(-1, keepdim=True))
            zero = torch.zeros((), device="cuda")
            return dict(logp=torch.where(has, (x.gather(-1, target) - lse)[..., 0], zero), lse=torch.where(has, lse[..., 0], zero))
        logits, top = x, x.amax(-1, keepdim=True)
        x = x - top
        e = torch.exp(x)
        total = e.sum(-1, keepdim=True)
        lse = torch.log(total)
        out = dict(logp=torch.where(has, (x.gather(-1, target) - lse)[..., 0], torch.zeros((), device="cuda")), lse=(lse + top)[..., 0])
        if c["entropy"]:
            out["entropy"] = (lse - torch.where(e > 0, e * x, 0.0).sum(-1, keepdim=True) / total)[..., 0]
        if c["top"]:   # in descending order, equal ones by their index
            value, token = torch.sort(logits, dim=-1, descending=True, stable=True)
            out["top_logp"], out["top_token"] = value[..., :c["top"]] - top - lse, token[..., :c["top"]].contiguous()
        return out
    logp = x - s["lse"][..., None]
    p = torch.exp(logp)
    dlogp = torch.where(has, s["dlogp"], 0.0)[..., None]
    d = -dlogp * p
    if c["entropy"]:
        d = d - s["dentropy"][..., None] * torch.where(p > 0, p * (logp + s["entropy"][..., None]), 0.0)
    return d.scatter_add_(-1, target, dlogp).to(io)


def _plan(s):
    """What a program keeps between its steps: descriptors, output buffers and workspaces, the table of its gradients."""
    from paper_2511_15927_amd import binding as bd
    c, kind = s["c"], s["kind"]
    Bt, L, D, V, io = c["batch"], c["seqlen"], c["width"], c["vocab"], _TYPES[c["io"]]
    empty = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    p = dict(bd=bd)
    if kind == "clip":
        p["table"] = bd.GradTable(s["small"] + s["large"], s["small_to"] + s["large_to"])
        p["norm"] = empty(1)
        p["out"] = dict(norm=p["norm"][0], small=s["small_flat"], large=s["large_flat"])
        p["ws"] = empty(max(16, bd.bimamba_clip_grads_workspace_bytes(p["table"])), dtype=torch.uint8)
    elif kind in ("embed", "embed_bwd"):
        p["desc"] = bd.make_embed_desc(Bt, L, D, V, table=c["table"], io=c["io"], scale=s["scale"])
        p["out"] = empty(Bt, L, D, dtype=io) if kind == "embed" else empty(V, D)
        if kind == "embed_bwd":
            p["ws"] = empty(max(16, bd.bimamba_embed_bwd_workspace_bytes(p["desc"])), dtype=torch.uint8)
    elif kind in ("norm", "norm_bwd"):
        p["desc"] = bd.make_norm_desc(Bt, L, D, io=c["io"], eps=EPS)
        if kind == "norm":
            p["out"] = dict(y=empty(Bt, L, D, dtype=io), mean=empty(Bt, L), rstd=empty(Bt, L))
        else:
            rows = (Bt,) if c["modulated"] else ()
            p["out"] = dict(dx=empty(Bt, L, D, dtype=io), dweight=empty(*rows, D), dbias=empty(*rows, D))
            p["ws"] = empty(max(16, bd.bimamba_layer_norm_bwd_workspace_bytes(p["desc"], bool(c["modulated"]))), dtype=torch.uint8)
    elif kind == "scores":
        p["desc"] = bd.make_logits_desc(Bt, L, V, io=c["io"], top_k=c["top"], targets_only=int(not (c["entropy"] or c["top"])))
        out = dict(logp=empty(Bt, L), lse=empty(Bt, L))
        if c["entropy"]:
            out["entropy"] = empty(Bt, L)
        if c["top"]:
            out["top_logp"], out["top_token"] = empty(Bt, L, c["top"]), empty(Bt, L, c["top"], dtype=torch.int64)
        p["out"] = out
        p["ws"] = empty(max(16, bd.bimamba_log_probs_workspace_bytes(p["desc"])), dtype=torch.uint8)
    else:
        p["desc"] = bd.make_logits_desc(Bt, L, V, io=c["io"])
        p["out"] = empty(Bt, L, V, dtype=io)
    s["plan"] = p
    return p


def run(state):
    s = state
    if not own:
        return _plain(s)
    p = s.get("plan") or _plan(s)
    bd, kind, out = p["bd"], s["kind"], p["out"]
    if kind == "embed":
        bd.bimamba_embed(p["desc"], s["tokens"], s["table"], out)
    elif kind == "embed_bwd":
        bd.bimamba_embed_bwd(p["desc"], s["tokens"], s["dout"], out, p["ws"])
    elif kind == "norm":
        bd.bimamba_layer_norm(p["desc"], s["x"], s["weight"], s["bias"], out["y"], out["mean"], out["rstd"])
    elif kind == "norm_bwd":
        bd.bimamba_layer_norm_bwd(p["desc"], s["x"], s["weight"], s["mean"], s["rstd"], s["dy"], out["dx"], out["dweight"], out["dbias"],
                                  p["ws"])
    elif kind == "scores":
        bd.bimamba_log_probs(p["desc"], s["logits"], s["targets"], out, p["ws"])
    elif kind == "scores_bwd":
        bd.bimamba_log_probs_bwd(p["desc"], s["logits"], s["targets"], s["lse"], s["entropy"], s["dlogp"], s["dentropy"], out)
    else:
        bd.bimamba_clip_grads(p["table"], MAX_NORM, p["norm"], p["ws"])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    c, kind = s["c"], s["kind"]
    if kind == "embed":
        return s["table"].double().index_select(0, s["tokens"].reshape(-1)).view(c["batch"], c["seqlen"], -1) * s["scale"]
    if kind == "embed_bwd":
        order = torch.argsort(s["tokens"].reshape(-1), stable=True)
        ids, rows = s["tokens"].reshape(-1)[order], s["dout"].double().reshape(-1, c["width"])[order]
        ends = torch.cumsum(torch.bincount(ids, minlength=c["vocab"]), 0)
        sums = torch.cat([torch.zeros(1, c["width"], dtype=torch.float64, device="cuda"), torch.cumsum(rows, 0)])
        return (sums[ends] - sums[torch.cat([ends.new_zeros(1), ends[:-1]])]) * s["scale"]
    if kind in ("norm", "norm_bwd"):
        x = s["x"].double()
        weight, bias = (s[k].double().view(-1, 1, c["width"]) for k in ("weight", "bias"))
        if kind == "norm":
            var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
            return dict(y=(x - mean) / (var + EPS).sqrt() * weight + bias, mean=mean.squeeze(-1), rstd=(var + EPS).pow(-0.5).squeeze(-1))
        rstd = s["rstd"].double().unsqueeze(-1)
        hat = (x - s["mean"].double().unsqueeze(-1)) * rstd
        dy = s["dy"].double()
        g, n = dy * weight, c["width"]
        dx = (g - (g.sum(-1, keepdim=True) + hat * (g * hat).sum(-1, keepdim=True)) / n) * rstd
        dw, db = (dy * hat).sum(1), dy.sum(1)
        return dict(dx=dx, dweight=dw if c["modulated"] else dw.sum(0), dbias=db if c["modulated"] else db.sum(0))
    if kind == "clip":
        norm = math.sqrt(sum(float(g.double().square().sum()) for g in s["small"] + s["large"]))
        f = min(1.0, MAX_NORM / norm)
        flat = [torch.cat([g.double().reshape(-1) for g in gs]) * f if gs else torch.empty(0, dtype=torch.float64, device="cuda")
                for gs in (s["small"], s["large"])]
        return dict(norm=torch.tensor(norm, dtype=torch.float64), small=flat[0], large=flat[1])
    logp = torch.log_softmax(s["logits"].double(), -1)
    has = s["targets"] >= 0
    at = s["targets"].clamp(min=0).unsqueeze(-1)
    if kind == "scores":
        lse = torch.logsumexp(s["logits"].double(), -1)
        own_logp = torch.where(has, logp.gather(-1, at).squeeze(-1), 0.0)
        if not (c["entropy"] or c["top"]):
            return dict(logp=own_logp, lse=torch.where(has, lse, 0.0))
        out = dict(logp=own_logp, lse=lse)
        if c["entropy"]:
            out["entropy"] = -torch.special.xlogy(logp.exp(), logp.exp()).sum(-1)
        if c["top"]:
            out["top_logp"], out["top_token"] = torch.topk(logp, c["top"], dim=-1).values, None
        return out
    p = logp.exp()
    dlogp = torch.where(has, s["dlogp"].double(), 0.0).unsqueeze(-1)
    d = torch.zeros_like(p).scatter_(-1, at, dlogp) - dlogp * p
    if c["entropy"]:
        entropy = -torch.special.xlogy(p, p).sum(-1, keepdim=True)
        d -= s["dentropy"].double().unsqueeze(-1) * (torch.special.xlogy(p, p) + p * entropy)
    return d


def work(case):
    c = dict(_BASE, **case)
    kind, n, D, V = c["kind"], c["batch"] * c["seqlen"], c["width"], c["vocab"]
    e = 2 if c["io"] == "bf16" else 4
    if kind == "clip":
        small, large = (sum(_numels(s)) for s in _clip_shapes(c))
        return dict(bytes=2 * (4 * small + e * large), flops=3 * (small + large))
    if kind == "embed":
        rows = min(V, max(1, int(n * (1 - c["masked"])) + 1))   # (a row of the table that several tokens take is read once)
        return dict(bytes=8 * n + rows * D * (4 if c["table"] == "f32" else 2) + n * D * e, flops=n * D)
    if kind == "embed_bwd":
        return dict(bytes=8 * n + n * D * e + 4 * V * D, flops=2 * n * D)
    per = 8 * D * (c["batch"] if c["modulated"] else 1)
    if kind == "norm":
        return dict(bytes=2 * n * D * e + 8 * n + per, flops=7 * n * D)
    if kind == "norm_bwd":
        return dict(bytes=3 * n * D * e + 8 * n + 12 * D * (c["batch"] if c["modulated"] else 1), flops=14 * n * D)
    if kind == "scores":
        read = n if c["entropy"] or c["top"] else int(n * c["masked"])
        return dict(bytes=read * V * e + 8 * n + n * (8 + 4 * c["entropy"] + 12 * c["top"]), flops=read * V * (4 + 2 * c["entropy"]))
    read = n if c["entropy"] else int(n * c["masked"])
    return dict(bytes=(read + n) * V * e + 8 * n + n * (8 + 8 * c["entropy"]), flops=read * V * (3 + 4 * c["entropy"]))
