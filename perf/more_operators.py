"""What the operators of a gated linear recurrence block are timed on: the recurrence, the normalisation of its gated output and the
dropout on the way back into the residual stream, at the sizes that training and block decoding give them.

Kinds of case, each one pass through one entry point:
  recur        bimamba_recurrence: h = a h + u along the sequence, forwards or (`reverse`) backwards
  recur_bwd    bimamba_recurrence_bwd: its gradients
  gnorm        bimamba_group_norm: the norm of each token's groups of channels, with an activation or a gate
  gnorm_bwd    bimamba_group_norm_bwd: its gradients
  drop         bimamba_dropout_add: residual + gate * dropout(x)
  drop_bwd     bimamba_dropout_add_bwd: its gradients
Fields: `io` is the type of activations and their gradients; `packed`: activations are column slices of a wider buffer; `gate` is the
recurrence's (log: a = exp(min(g, 0)), u = x; sigmoid: a = sigmoid(g + bias), u = (1 - a) x); `stateful`: the state enters and leaves the
call; `train`: the state before every 64th token is kept; `add`: y = h + add; `ragged`: sequences end before the buffer does, and what
lies behind an end gets zeros; `act` and `centred` are the norm's; `vector` says what multiplies the dropped-out values (none, one
vector, each batch element's own).
"""
import math

import torch

own = False

_BASE = dict(kind="recur", batch=1, seqlen=32, width=4096, io="bf16", packed=0, gate="sigmoid", reverse=0, stateful=0, train=0, add=0,
             ragged=0, groups=1, act="none", centred=0, p=0.1, vector="none", residual=1)
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
KEEP_EVERY = 64   # tokens between two kept states
SITE = 3          # of the dropout within its model


def _case(name=None, **kw):
    c = dict(_BASE, **kw)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # autoregressive decoding: one token of 64 sequences, the smallest call
        _case("recur_token", batch=64, seqlen=1, stateful=1),
        # a denoising step of block decoding: 16 blocks of 32 tokens, resumed from the cached state
        _case("recur_block", batch=16, seqlen=32, stateful=1),
        # training at the headline's length, the right-to-left half of a bidirectional mixer, added to the other half
        _case("recur_train", batch=8, seqlen=8192, reverse=1, train=1, add=1),
        # one long sequence with few channels
        _case("recur_long", batch=1, seqlen=65536, width=2048, gate="log", stateful=1),
        # the training step's gradients
        _case("recur_grad", kind="recur_bwd", batch=8, seqlen=8192),
        # gradients in a small fp32 model: padded sequences, rows that are slices of a wider buffer
        _case("recur_grad_ragged", kind="recur_bwd", batch=3, seqlen=1237, width=740, io="f32", packed=1, gate="log", reverse=1, ragged=1,
              stateful=1),
        # the gated output of heads of 64 channels in a decoding step
        _case("gnorm_block", kind="gnorm", batch=16, seqlen=32, groups=64, act="gate_before"),
        # training: wide groups, mean and gate behind the norm
        _case("gnorm_train", kind="gnorm", batch=8, seqlen=8192, groups=8, act="gate_after", centred=1),
        # training's gradients for heads of 64 channels
        _case("gnorm_grad", kind="gnorm_bwd", batch=8, seqlen=8192, groups=64, act="gate_before"),
        # a toy model's training step
        _case("drop_toy", kind="drop", batch=32, seqlen=64, width=256, io="f32"),
        # training at the headline's length, with each sequence's own conditioning
        _case("drop_train", kind="drop", batch=8, seqlen=8192, width=2048, vector="each"),
        # its gradients, the conditioning's among them
        _case("drop_grad", kind="drop_bwd", batch=8, seqlen=8192, width=2048, vector="each"),
    ]


_MOST_VALUES = 8 * 8192 * 4096   # bf16 values of the largest listed activation


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["recur", "recur", "recur_bwd", "gnorm", "gnorm_bwd", "drop", "drop_bwd"])
    c = dict(kind=kind, io=rng.choice(["bf16", "bf16", "f32"]), packed=rng.randint(0, 1), batch=_log_int(rng, 1, 64), seqlen=_log_int(rng, 1, 65536),
             width=_log_int(rng, 16, 8192))
    if rng.random() < 0.6:
        c["width"] = max(8, c["width"] // 8 * 8)
    if kind in ("recur", "recur_bwd"):
        c.update(gate=rng.choice(["log", "sigmoid"]), reverse=rng.randint(0, 1), stateful=rng.randint(0, 1), ragged=int(rng.random() < 0.3))
        if kind == "recur":
            c.update(train=rng.randint(0, 1), add=rng.randint(0, 1))
    elif kind in ("gnorm", "gnorm_bwd"):
        size = rng.choice([16, 32, 37, 64, 100, 128, 256, 500, 512, 1024, 2048, 4096])
        c["groups"] = max(1, c["width"] // size)
        c["width"] = c["groups"] * min(size, c["width"])
        c.update(act=rng.choice(["none", "silu", "gate_before", "gate_after"]), centred=rng.randint(0, 1))
    else:
        c.update(p=rng.choice([0.05, 0.1, 0.2, 0.5]), vector=rng.choice(["none", "one", "each"]), residual=rng.randint(0, 1) if kind == "drop" else 0)
    room = _MOST_VALUES // (2 if c["io"] == "f32" else 1)
    c["seqlen"] = max(1, min(c["seqlen"], room // (c["batch"] * c["width"])))
    return _case(**c)


def _rows(c, gen, width, scale=1.0, shift=0.0):
    io = _TYPES[c["io"]]
    pitch = width + (width // 2 // 8 * 8 if c["packed"] else 0)
    wide = torch.empty(c["batch"], c["seqlen"], pitch, dtype=io, device="cuda")
    wide.normal_(shift, scale, generator=gen)
    return wide[..., pitch - width:]


def prepare(case, seed):
    c = dict(_BASE, **case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    Bt, L, D = c["batch"], c["seqlen"], c["width"]
    s = dict(c=c, kind=c["kind"])

    def normal(*shape, scale=1.0):
        return scale * torch.randn(*shape, device="cuda", generator=gen)

    if c["kind"] in ("recur", "recur_bwd"):
        s["x"] = _rows(c, gen, D)
        # channels forget over 2 to 1000 tokens
        memory = torch.exp(torch.rand(D, device="cuda", generator=gen) * math.log(500.0)) * 2
        if c["gate"] == "sigmoid":
            s["g"], s["bias"] = _rows(c, gen, D, 0.5), torch.log(memory)
        else:
            s["g"], s["bias"] = _rows(c, gen, D, 0.5), None
            for g in s["g"]:
                g.copy_(-torch.exp(g.float() - torch.log(memory)))
        s["lengths"] = torch.randint(L // 2, L + 1, (Bt,), device="cuda", generator=gen) if c["ragged"] else None
        s["h_in"] = normal(Bt, D) if c["stateful"] else None
        if c["kind"] == "recur":
            s["add"] = _rows(c, gen, D) if c["add"] else None
        else:
            s["dy"] = _rows(c, gen, D, 1e-2)
            s["dh_out"] = normal(Bt, D, scale=1e-2) if c["stateful"] else None
            s["states"] = _plain(dict(s, kind="recur", add=None, c=dict(c, train=1)))["states"]
        return s
    if c["kind"] in ("gnorm", "gnorm_bwd"):
        s["x"] = _rows(c, gen, D, 2.0, 0.3)
        s["z"] = _rows(c, gen, D) if c["act"].startswith("gate") else None
        s["weight"], s["bias"] = 1 + normal(D, scale=0.2), normal(D, scale=0.2)
        if c["kind"] == "gnorm_bwd":
            s["dy"] = _rows(c, gen, D, 1e-2)
            stats = _plain(dict(s, kind="gnorm"))
            s["mean"], s["rstd"] = stats.get("mean"), stats["rstd"]
        return s
    s["key"] = torch.randint(-(1 << 62), 1 << 62, (2,), device="cuda", generator=gen)   # seed, offset
    s["x"] = _rows(c, gen, D)
    s["vector"] = None if c["vector"] == "none" else 0.3 * normal(*((D,) if c["vector"] == "one" else (Bt, D)))
    if c["kind"] == "drop":
        s["residual"] = _rows(c, gen, D, 2.0) if c["residual"] else None
    else:
        s["dout"] = _rows(c, gen, D, 1e-2)
    return s


# ---- plain forms ----

def _scan(a, u, h0):
    """States after every step of h = a h + u along the middle axis: pieces of about the root of its length side by side, then
    what each piece starts from."""
    Bt, L, D = a.shape
    T = 1 << (max(L - 1, 0).bit_length() // 2)
    n = (L + T - 1) // T
    if n * T != L:
        a = torch.cat([a, a.new_ones(Bt, n * T - L, D)], 1)
        u = torch.cat([u, u.new_zeros(Bt, n * T - L, D)], 1)
    a, u = a.view(Bt, n, T, D), u.view(Bt, n, T, D)
    h, decay = torch.empty_like(u), torch.empty_like(a)
    h[:, :, 0], decay[:, :, 0] = u[:, :, 0], a[:, :, 0]
    for t in range(1, T):
        h[:, :, t] = a[:, :, t] * h[:, :, t - 1] + u[:, :, t]
        decay[:, :, t] = a[:, :, t] * decay[:, :, t - 1]
    enter = [h0]
    for i in range(n - 1):
        enter.append(decay[:, i, -1] * enter[-1] + h[:, i, -1])
    decay *= torch.stack(enter, 1)[:, :, None]
    h += decay
    return h.view(Bt, n * T, D)[:, :L]


def _places(s):
    """For every step of the scan: the token that it takes [batch, L, 1], and whether it lies within the sequence."""
    c = s["c"]
    t = torch.arange(c["seqlen"], device="cuda").expand(c["batch"], -1)
    length = torch.full((c["batch"], 1), c["seqlen"], device="cuda") if s["lengths"] is None else s["lengths"][:, None]
    if c["reverse"]:
        t = torch.where(t < length, length - 1 - t, t)
    return t[..., None], (torch.arange(c["seqlen"], device="cuda") < length)[..., None]


def _plain_recur(s):
    c = s["c"]
    io = _TYPES[c["io"]]
    moved = c["reverse"] or c["ragged"]
    place, inside = _places(s)
    along = (lambda v: torch.where(inside, v.gather(1, place.expand_as(v)), 0.0)) if moved else (lambda v: v)
    back = (lambda v: torch.where(inside, v, 0.0).gather(1, place.expand_as(v))) if moved else (lambda v: v)
    x, g = along(s["x"].float()), along(s["g"].float())
    if c["gate"] == "sigmoid":
        v = g + s["bias"]
        a, rest = torch.sigmoid(v), torch.sigmoid(-v)
        u = rest * x
    else:
        a, u = torch.exp(g.clamp(max=0.0)), x
    if c["ragged"]:
        a, u = torch.where(inside, a, 1.0), torch.where(inside, u, 0.0)
    if s["kind"] == "recur":
        h0 = torch.zeros(c["batch"], c["width"], device="cuda") if s["h_in"] is None else s["h_in"]
        h = _scan(a, u, h0)
        out = {}
        if c["stateful"]:
            out["h_out"] = h[:, -1].clone()
        if c["train"]:
            out["states"] = torch.cat([h0[:, None], h[:, KEEP_EVERY - 1:c["seqlen"] - 1:KEEP_EVERY]], 1)
        y = back(h)
        if s["add"] is not None:
            y = y + s["add"].float()
            if c["ragged"]:   # (what lies behind the end)
                y = torch.where(inside, y, 0.0)
        return dict(out, y=y.to(io))
    dy = along(s["dy"].float())
    h0 = s["states"][:, 0]
    before = torch.cat([h0[:, None], _scan(a, u, h0)[:, :-1]], 1)
    # dh of a step = dy + (a dh of the step after it): the same recurrence backwards, with the factor of the step after
    last = torch.zeros(c["batch"], c["width"], device="cuda") if s["dh_out"] is None else s["dh_out"]
    after = torch.cat([a[:, 1:], a.new_ones(c["batch"], 1, c["width"])], 1).flip(1)
    dh = _scan(after, dy.flip(1), last).flip(1)
    if c["gate"] == "sigmoid":
        dx, dg = rest * dh, dh * (before - x) * a * rest
    else:
        dx, dg = dh, torch.where(g > 0, 0.0, dh * before * a)
    if c["ragged"]:
        dx, dg = torch.where(inside, dx, 0.0), torch.where(inside, dg, 0.0)
    out = dict(dx=back(dx).to(io), dg=back(dg).to(io))
    if c["gate"] == "sigmoid":
        out["dbias"] = dg.sum((0, 1))
    if c["stateful"]:
        out["dh_in"] = a[:, 0] * dh[:, 0]
    return out


def _plain_gnorm(s):
    c = s["c"]
    io, D = _TYPES[c["io"]], c["width"]
    grouped = (c["batch"], c["seqlen"], c["groups"], D // c["groups"])
    x = s["x"].float()
    z = None if s["z"] is None else s["z"].float()
    gate = None if z is None else z * torch.sigmoid(z)
    u = (x * gate if c["act"] == "gate_before" else x).reshape(grouped)
    w, b = s["weight"].view(grouped[2:]), s["bias"].view(grouped[2:])
    if s["kind"] == "gnorm":
        out = {}
        if c["centred"]:
            mean = u.mean(-1, keepdim=True)
            u = u - mean
            out["mean"] = mean[..., 0]
        rstd = 1 / torch.sqrt((u * u).mean(-1, keepdim=True) + EPS)
        v = (u * rstd * w + b).view(x.shape)
        y = v * torch.sigmoid(v) if c["act"] == "silu" else v * gate if c["act"] == "gate_after" else v
        return dict(out, y=y.to(io), rstd=rstd[..., 0])
    rstd = s["rstd"][..., None]
    hat = (u - s["mean"][..., None] if c["centred"] else u) * rstd
    dv = s["dy"].float().reshape(grouped)
    out = {}
    if c["act"] == "silu":
        v = hat * w + b
        sig = torch.sigmoid(v)
        dv = dv * sig * (1 + v * (1 - sig))
    elif c["act"] == "gate_after":
        sig = torch.sigmoid(z)
        out["dz"] = ((dv * (hat * w + b)).view(x.shape) * sig * (1 + z * (1 - sig))).to(io)
        dv = dv * gate.view(grouped)
    out["dweight"], out["dbias"] = (dv * hat).sum((0, 1)).view(D), dv.sum((0, 1)).view(D)
    k = dv * w
    du = k - hat * (k * hat).mean(-1, keepdim=True)
    if c["centred"]:
        du = du - k.mean(-1, keepdim=True)
    du = (du * rstd).view(x.shape)
    if c["act"] == "gate_before":
        sig = torch.sigmoid(z)
        out["dz"] = (du * x * sig * (1 + z * (1 - sig))).to(io)
        du = du * gate
    return dict(out, dx=du.to(io))


_LOW = 0xFFFFFFFF


def _halves(c, key):
    """The 16 random bits of every value, int64 [batch, L, ceil(width / 8) * 8]: Philox4x32 with ten rounds (Salmon et al., 2011)."""
    n, blocks = c["batch"] * c["seqlen"], (c["width"] + 7) // 8
    row = torch.arange(n, device="cuda")[:, None].expand(n, blocks)
    x = [row, (torch.arange(blocks, device="cuda") + (SITE << 17)).expand(n, blocks), key[1] & _LOW, (key[1] >> 32) & _LOW]
    k0, k1 = key[0] & _LOW, (key[0] >> 32) & _LOW
    for _ in range(10):
        p0, p1 = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57   # (modulo 2^64: the bits are right whatever the sign)
        x = [((p1 >> 32) & _LOW) ^ x[1] ^ k0, p1 & _LOW, ((p0 >> 32) & _LOW) ^ x[3] ^ k1, p0 & _LOW]
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    words = torch.stack([h for w in x for h in (w & 0xFFFF, w >> 16)], -1)
    return words.view(c["batch"], c["seqlen"], blocks * 8)[..., :c["width"]]


def _threshold(p):
    return int(math.floor(p * 65536 + 0.5))


def _plain_drop(s):
    c = s["c"]
    io, at = _TYPES[c["io"]], _threshold(c["p"])
    scale = 65536 / (65536 - at) if at < 65536 else 0.0
    kept = torch.where(_halves(c, s["key"]) >= at, scale, 0.0)
    vector = s["vector"][:, None] if c["vector"] == "each" else s["vector"]
    if s["kind"] == "drop":
        out = s["x"].float() * kept
        if vector is not None:
            out = out * vector
        return (out if s["residual"] is None else out + s["residual"].float()).to(io)
    d = s["dout"].float() * kept
    out = dict(dx=(d if vector is None else d * vector).to(io))
    if vector is not None:
        out["dgate"] = (d * s["x"].float()).sum(1 if c["vector"] == "each" else (0, 1))
    return out


def _plain(s):
    return {"r": _plain_recur, "g": _plain_gnorm, "d": _plain_drop}[s["kind"][0]](s)


# ---- the framework's calls ----

def _plan(s):
    """What a program keeps between its steps: descriptors, output buffers and workspaces."""
    from paper_2511_15927_amd import binding as bd
    c, kind = s["c"], s["kind"]
    Bt, L, D, io = c["batch"], c["seqlen"], c["width"], _TYPES[c["io"]]
    empty = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    p = dict(bd=bd, ws=None)
    need = 0
    if kind in ("recur", "recur_bwd"):
        p["desc"] = bd.make_recurrence_desc(Bt, L, D, io=c["io"], gate=c["gate"], reverse=c["reverse"])
        if kind == "recur":
            p["out"] = dict(y=empty(Bt, L, D, dtype=io))
            if c["stateful"]:
                p["out"]["h_out"] = empty(Bt, D)
            if c["train"]:
                p["out"]["states"] = empty(Bt, (L + KEEP_EVERY - 1) // KEEP_EVERY, D)
            need = bd.bimamba_recurrence_workspace_bytes(p["desc"])
        else:
            p["out"] = dict(dx=empty(Bt, L, D, dtype=io), dg=empty(Bt, L, D, dtype=io))
            if c["gate"] == "sigmoid":
                p["out"]["dbias"] = empty(D)
            if c["stateful"]:
                p["out"]["dh_in"] = empty(Bt, D)
            need = bd.bimamba_recurrence_bwd_workspace_bytes(p["desc"])
    elif kind in ("gnorm", "gnorm_bwd"):
        p["desc"] = bd.make_group_norm_desc(Bt, L, D, c["groups"], io=c["io"], act=c["act"], centred=c["centred"], eps=EPS)
        if kind == "gnorm":
            p["out"] = dict(y=empty(Bt, L, D, dtype=io), rstd=empty(Bt, L, c["groups"]))
            if c["centred"]:
                p["out"]["mean"] = empty(Bt, L, c["groups"])
        else:
            p["out"] = dict(dx=empty(Bt, L, D, dtype=io), dweight=empty(D), dbias=empty(D))
            if s["z"] is not None:
                p["out"]["dz"] = empty(Bt, L, D, dtype=io)
            need = bd.bimamba_group_norm_bwd_workspace_bytes(p["desc"])
    else:
        p["desc"] = bd.make_dropout_desc(Bt, L, D, io=c["io"], p=c["p"], site=SITE)
        if kind == "drop":
            p["out"] = empty(Bt, L, D, dtype=io)
        else:
            p["out"] = dict(dx=empty(Bt, L, D, dtype=io))
            if s["vector"] is not None:
                p["out"]["dgate"] = torch.empty_like(s["vector"])
                need = bd.bimamba_dropout_add_bwd_workspace_bytes(p["desc"], c["vector"] == "each")
    if need:
        p["ws"] = empty(need, dtype=torch.uint8)
    s["plan"] = p
    return p


def run(state):
    s = state
    if not own:
        return _plain(s)
    p = s.get("plan") or _plan(s)
    bd, kind, out = p["bd"], s["kind"], p["out"]
    if kind == "recur":
        bd.bimamba_recurrence(p["desc"], s["x"], s["g"], s["bias"], out["y"], add=s["add"], lengths=s["lengths"], h_in=s["h_in"],
                              h_out=out.get("h_out"), states=out.get("states"), workspace=p["ws"])
    elif kind == "recur_bwd":
        bd.bimamba_recurrence_bwd(p["desc"], s["x"], s["g"], s["bias"], s["states"], s["dy"], out["dx"], out["dg"], dbias=out.get("dbias"),
                                  lengths=s["lengths"], dh_out=s["dh_out"], dh_in=out.get("dh_in"), workspace=p["ws"])
    elif kind == "gnorm":
        bd.bimamba_group_norm(p["desc"], s["x"], s["z"], s["weight"], s["bias"], out["y"], out.get("mean"), out["rstd"])
    elif kind == "gnorm_bwd":
        bd.bimamba_group_norm_bwd(p["desc"], s["x"], s["z"], s["weight"], s["bias"], s["mean"], s["rstd"], s["dy"], out["dx"], out.get("dz"),
                                  out["dweight"], out["dbias"], p["ws"])
    elif kind == "drop":
        bd.bimamba_dropout_add(p["desc"], s["key"], s["x"], s["vector"], s["residual"], out)
    else:
        bd.bimamba_dropout_add_bwd(p["desc"], s["key"], s["x"], s["vector"], s["dout"], out["dx"], out.get("dgate"), p["ws"])
    return out


# ---- definitions in 64 bits ----

def _exact_recur(s):
    c = s["c"]
    Bt, L, D = c["batch"], c["seqlen"], c["width"]
    f64 = dict(dtype=torch.float64, device="cuda")
    ends = [L] * Bt if s["lengths"] is None else s["lengths"].tolist()
    out = dict(y=torch.zeros(Bt, L, D, **f64)) if s["kind"] == "recur" else dict(dx=torch.zeros(Bt, L, D, **f64), dg=torch.zeros(Bt, L, D, **f64))
    enter = torch.zeros(Bt, (L + KEEP_EVERY - 1) // KEEP_EVERY, D, **f64)
    edge = torch.zeros(Bt, D, **f64)   # the state that leaves, or the gradient of the one that entered
    dbias = torch.zeros(D, **f64)
    # (sequences of one length together)
    for end in sorted(set(ends)):
        who = [b for b in range(Bt) if ends[b] == end]
        order = range(end - 1, -1, -1) if c["reverse"] else range(end)
        x, g = s["x"][who, :end].double().transpose(0, 1).contiguous(), s["g"][who, :end].double().transpose(0, 1).contiguous()
        if c["gate"] == "sigmoid":
            a = 1 / (1 + torch.exp(-(g + s["bias"].double())))
            u = x / (1 + torch.exp(g + s["bias"].double()))
        else:
            a, u = torch.exp(torch.minimum(g, torch.zeros_like(g))), x
        start = s["h_in"] if s["kind"] == "recur" else s["states"][:, 0]
        h = torch.zeros(len(who), D, **f64) if start is None else start[who].double()
        hs = torch.empty(end, len(who), D, **f64)   # before each token
        for i, t in enumerate(order):
            if i % KEEP_EVERY == 0:
                enter[who, i // KEEP_EVERY] = h
            hs[t] = h
            h = torch.addcmul(u[t], a[t], h)
        if s["kind"] == "recur":
            enter[who, (end + KEEP_EVERY - 1) // KEEP_EVERY:] = h[:, None]
            edge[who] = h
            y = (a * hs + u).transpose(0, 1)
            out["y"][who, :end] = y if s["add"] is None else y + s["add"][who, :end].double()
            continue
        dy = s["dy"][who, :end].double().transpose(0, 1).contiguous()
        d = torch.zeros(len(who), D, **f64) if s["dh_out"] is None else s["dh_out"][who].double()
        dh = dy   # (in place)
        for t in reversed(order):
            dh[t] += d
            d = a[t] * dh[t]
        edge[who] = d
        if c["gate"] == "sigmoid":
            dx, dg = dh * (1 - a), dh * (hs - x) * a * (1 - a)
            dbias += dg.sum((0, 1))
        else:
            dx, dg = dh, dh * hs * a * (g <= 0)
        out["dx"][who, :end], out["dg"][who, :end] = dx.transpose(0, 1), dg.transpose(0, 1)
    if c["stateful"]:
        out["h_out" if s["kind"] == "recur" else "dh_in"] = edge
    if s["kind"] == "recur" and c["train"]:
        out["states"] = enter
    if s["kind"] == "recur_bwd" and c["gate"] == "sigmoid":
        out["dbias"] = dbias
    return out


def _exact_gnorm(s):
    c = s["c"]
    Bt, L, D, G = c["batch"], c["seqlen"], c["width"], c["groups"]
    out = {k: [] for k in (("y", "mean", "rstd") if s["kind"] == "gnorm" else ("dx", "dz"))}
    dw, db = torch.zeros(D, dtype=torch.float64, device="cuda"), torch.zeros(D, dtype=torch.float64, device="cuda")
    silu = lambda v: v / (1 + torch.exp(-v))  # noqa: E731
    slope = lambda v: (1 + torch.exp(-v) + v * torch.exp(-v)) / (1 + torch.exp(-v)) ** 2  # noqa: E731
    w, b = s["weight"].double().view(G, -1), s["bias"].double().view(G, -1)
    for i in range(Bt):   # a sequence after the other
        x = s["x"][i].double().unflatten(-1, (G, D // G))
        z = None if s["z"] is None else s["z"][i].double().unflatten(-1, (G, D // G))
        u = x * silu(z) if c["act"] == "gate_before" else x
        if s["kind"] == "gnorm":
            var, mean = torch.var_mean(u, -1, correction=0, keepdim=True)
            if not c["centred"]:
                var, mean = (u ** 2).mean(-1, keepdim=True), torch.zeros_like(mean)
            v = (u - mean) * (var + EPS) ** -0.5 * w + b
            out["y"].append((silu(v) if c["act"] == "silu" else v * silu(z) if c["act"] == "gate_after" else v).flatten(-2))
            out["mean"].append(mean[..., 0])
            out["rstd"].append((var[..., 0] + EPS) ** -0.5)
            continue
        rstd = s["rstd"][i].double().unsqueeze(-1)
        hat = (u - (s["mean"][i].double().unsqueeze(-1) if c["centred"] else 0)) * rstd
        v, dy = hat * w + b, s["dy"][i].double().unflatten(-1, (G, D // G))
        dv = dy * slope(v) if c["act"] == "silu" else dy * silu(z) if c["act"] == "gate_after" else dy
        dw += (dv * hat).sum(0).flatten()
        db += dv.sum(0).flatten()
        n = D // G
        du = rstd * w * dv - rstd / n * (hat * (dv * w * hat).sum(-1, keepdim=True) + (c["centred"] and (dv * w).sum(-1, keepdim=True)))
        out["dx"].append((du * silu(z) if c["act"] == "gate_before" else du).flatten(-2))
        if z is not None:
            out["dz"].append(((du * x if c["act"] == "gate_before" else dy * v) * slope(z)).flatten(-2))
    out = {k: torch.stack(v) for k, v in out.items() if v and (k != "mean" or c["centred"])}
    return dict(out, dweight=dw, dbias=db) if s["kind"] == "gnorm_bwd" else out


def _wide_product(a, b):
    """High and low 32 bits of products of 32-bit numbers, by their 16-bit halves."""
    al, ah, bl, bh = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
    mid = ah * bl + ((al * bl) >> 16)
    mid2 = al * bh + (mid & 0xFFFF)
    return ah * bh + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | (al * bl & 0xFFFF)


def _exact_drop(s):
    c = s["c"]
    Bt, L, D = c["batch"], c["seqlen"], c["width"]
    at = _threshold(c["p"])
    seed, offset = (v % (1 << 64) for v in s["key"].tolist())
    block = torch.arange(D, device="cuda") // 8 + SITE * (1 << 17)
    place = torch.arange(D, device="cuda") % 8
    out, dgate = [], []
    for b in range(Bt):
        row = (b * L + torch.arange(L, device="cuda"))[:, None].expand(L, (D + 7) // 8)
        ctr = [row, block[::8].expand_as(row), torch.full_like(row, offset % (1 << 32)), torch.full_like(row, offset >> 32)]
        key = [seed % (1 << 32), seed >> 32]
        for _ in range(10):
            hi0, lo0 = _wide_product(ctr[0], 0xD2511F53)
            hi1, lo1 = _wide_product(ctr[2], 0xCD9E8D57)
            ctr = [hi1 ^ ctr[1] ^ key[0], lo1, hi0 ^ ctr[3] ^ key[1], lo0]
            key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
        word = torch.stack(ctr, -1).repeat_interleave(2, -1).flatten(-2)[..., :D]
        bits = (word >> (place % 2 * 16)) & 0xFFFF
        kept = (bits >= at).double() * (65536.0 / max(65536 - at, 1))
        vector = 1.0 if s["vector"] is None else s["vector"].double() if c["vector"] == "one" else s["vector"][b].double()
        if s["kind"] == "drop":
            y = s["x"][b].double() * kept * vector
            out.append(y if s["residual"] is None else y + s["residual"][b].double())
        else:
            d = s["dout"][b].double() * kept
            out.append(d * vector)
            dgate.append((d * s["x"][b].double()).sum(0))
    if s["kind"] == "drop":
        return torch.stack(out)
    r = dict(dx=torch.stack(out))
    if s["vector"] is not None:
        r["dgate"] = torch.stack(dgate) if c["vector"] == "each" else torch.stack(dgate).sum(0)
    return r


def exact(case, seed):
    s = prepare(case, seed)
    return {"r": _exact_recur, "g": _exact_gnorm, "d": _exact_drop}[s["kind"][0]](s)


def work(case):
    c = dict(_BASE, **case)
    kind, n, D, e = c["kind"], c["batch"] * c["seqlen"], c["width"], 2 if c["io"] == "bf16" else 4
    if kind in ("recur", "recur_bwd"):
        kept = 4 * c["batch"] * ((c["seqlen"] + KEEP_EVERY - 1) // KEEP_EVERY) * D
        edge = 8 * c["batch"] * D * c["stateful"]
        if kind == "recur":
            return dict(bytes=n * D * e * (3 + c["add"]) + edge + kept * c["train"], flops=(8 if c["gate"] == "sigmoid" else 4) * n * D)
        return dict(bytes=n * D * e * 5 + edge + kept, flops=(18 if c["gate"] == "sigmoid" else 10) * n * D)
    if kind in ("gnorm", "gnorm_bwd"):
        gated, stats = c["act"].startswith("gate"), 4 * n * c["groups"] * (1 + c["centred"])
        if kind == "gnorm":
            return dict(bytes=n * D * e * (2 + gated) + stats + 8 * D, flops=(12 if c["act"] != "none" else 6) * n * D)
        return dict(bytes=n * D * e * (3 + 2 * gated) + stats + 16 * D, flops=(24 if c["act"] != "none" else 12) * n * D)
    vector = 4 * D * {"none": 0, "one": 1, "each": c["batch"]}[c["vector"]]
    if kind == "drop":
        return dict(bytes=n * D * e * (2 + c["residual"]) + vector, flops=3 * n * D)
    return dict(bytes=n * D * e * (2 + (c["vector"] != "none")) + 2 * vector, flops=4 * n * D)
