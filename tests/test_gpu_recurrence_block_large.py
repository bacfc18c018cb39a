"""The gated recurrence, the group norm and dropout, with their gradients, where a call moves more than 256 MB and goes past the caches: against
64-bit implementations, the recurrence also against the same rows through the caches."""
import numpy as np
import pytest
import torch

from running_error import TYPES, U32, Run, nans, workspace
from test_gpu_dropout import philox
from test_gpu_group_norm import forward_ref as norm_ref, gradient_ref as norm_bwd_ref, normed
from test_gpu_model_ops_large import CACHES, SIZE, bd, empty_afterwards, gen, normal  # noqa: F401
from test_gpu_recurrence import forward_ref, gradient_ref, run_backward, run_forward
from test_gpu_recurrence_forms import within

pytestmark = pytest.mark.gpu

# in forms of their own: many tokens in two and in one channel a lane, in pieces of either size, down to single tokens
WALKS = [(3, 4100, 4096, "bf16"), (150, 300, 1024, "bf16"), (250, 200, 1024, "bf16"), (800, 64, 1024, "bf16"), (1600, 30, 1024, "bf16"),
         (25000, 3, 1024, "bf16"), (30000, 1, 2048, "bf16"), (1, 90000, 512, "bf16"), (3, 4100, 2048, "f32"), (250, 200, 512, "f32"), (30000, 1, 1024, "f32")]


@pytest.mark.parametrize("B,L,D,io", WALKS)
def test_walks_past_the_caches(bd, B, L, D, io):  # noqa: F811
    """Rows that start at cache lines go past the caches, the same ones a step to the right go through them, in the same pieces: the same bits.
    And a sample of channels, those at the tiles' borders among them, against the walk in 64 bits (but for the longest, whose form is tested so at other sizes)."""
    assert 3 * B * L * D * SIZE[io] > CACHES and D * SIZE[io] % 128 == 0
    n = WALKS.index((B, L, D, io))
    gate, reverse, g = ("sigmoid", "log")[n % 2], n // 2 % 2, gen(n)
    memory = torch.exp(torch.rand(D, generator=g, device="cuda") * 6)
    raw = normal(g, B, L, D, scale=0.7)
    i = dict(x=normal(g, B, L, D, io=io), g=(raw if gate == "sigmoid" else 0.02 - torch.exp(raw) / memory).to(TYPES[io]),
             bias=torch.log(memory) if gate == "sigmoid" else None, h_in=normal(g, B, D), add=normal(g, B, L, D, io=io), dy=normal(g, B, L, D, io=io),
             dh_out=normal(g, B, D), lengths=torch.randint(L // 2, L + 1, (B,), generator=g, device="cuda") if n % 2 == 0 else None)
    del raw
    out = run_forward(bd, i, io, gate, reverse)
    other = run_forward(bd, i, io, gate, reverse, extra=3, lead=1)
    assert all(torch.equal(out[k], other[k]) for k in out)
    back = run_backward(bd, i, io, gate, reverse, out["states"])
    other = run_backward(bd, i, io, gate, reverse, out["states"], extra=3, lead=1)
    assert all(v is None or torch.equal(v, other[k]) for k, v in back.items())
    if L > 5000:
        return
    some = sorted({c for c in range(D) if c % 128 in (0, 1, 63, 64, 127) and c // 128 in (0, 1, D // 128 - 1)} | set(range(7, D, D // 32)))
    part = {k: None if t is None else t if k == "lengths" else t[..., some].contiguous() for k, t in i.items()}
    with torch.device("cuda"):
        for k, ref in zip(("y", "h_out", "states"), forward_ref(part, gate, reverse, True, True)):
            within(out[k][..., some], ref, io if k == "y" else "f32")
        for k, ref in zip(("dx", "dg", "dbias", "dh_in"), gradient_ref(part, gate, reverse, out["states"][..., some])):
            if back[k] is not None:
                within(back[k][..., some], ref, io if k in ("dx", "dg") else "f32")


# lanes that hold a part of a group, several rows at once, an element a lane, two and four pieces, four and eight waves
GROUPS = [(64, 64, "bf16"), (1, 24, "bf16"), (1, 5, "bf16"), (3, 1000, "bf16"), (2, 2048, "bf16"), (1, 4096, "bf16"), (1, 8192, "bf16"), (3, 700, "f32"),
          (16, 64, "f32"), (1, 1024, "f32"), (1, 2048, "f32"), (1, 8192, "f32"), (1, 3, "f32")]


@pytest.mark.parametrize("G,n,io", GROUPS)
def test_norms_past_the_caches(bd, G, n, io):  # noqa: F811
    """All rows against the formulas in 64 bits with their running error bound, in five parts; the sums over the rows with at most 300 additions on a
    term's way."""
    k, g, D = GROUPS.index((G, n, io)), gen(n), G * n
    act, centred = ("gate_before", "none", "gate_after", "silu")[k % 4], k % 2
    L = (CACHES // (2 * D * SIZE[io]) // 5 + 1) * 5
    assert 2 * L * D * SIZE[io] > CACHES
    x, z = normal(g, 1, L, D, scale=2.0, io=io) + 0.3, normal(g, 1, L, D, io=io) if act.startswith("gate") else None
    w, b, dy = 1 + normal(g, D, scale=0.2), normal(g, D, scale=0.2), normal(g, 1, L, D, io=io)
    desc = bd.make_group_norm_desc(1, L, D, G, io=io, act=act, centred=centred)
    y, dx, dz = torch.empty_like(x), torch.empty_like(x), None if z is None else torch.empty_like(x)
    mean, rstd, sums = nans(1, L, G) if centred else None, nans(1, L, G), nans(2, D)
    bd.bimamba_group_norm(desc, x, z, w, b, y, mean, rstd)
    bd.bimamba_group_norm_bwd(desc, x, z, w, b, mean, rstd, dy, dx, dz, *sums, workspace(bd.bimamba_group_norm_bwd_workspace_bytes(desc)))
    total, off = torch.zeros(2, 2, D, dtype=torch.float64, device="cuda")
    for at in range(0, L, L // 5):
        cut = lambda t: None if t is None else t[:, at:at + L // 5]  # noqa: E731
        i = dict(x=cut(x), z=cut(z), w=w, b=b, dy=cut(dy))
        with torch.device("cuda"):
            ry, rm, rr = norm_ref(i, G, act, centred)
            rdx, rdz = norm_bwd_ref(i, G, act, centred, cut(mean), cut(rstd))[:2]
            # the terms dv xh and dv of the sums
            u, _, gate = normed(i, G, act, False)
            xh = (u - cut(mean).double()[..., None] if centred else u) * cut(rstd).double()[..., None]
            dv = Run(i["dy"]).view(1, -1, G, n)
            if act == "silu":
                dv = dv * (xh * Run(w).view(G, n) + Run(b).view(G, n)).silu_slope()
            elif act == "gate_after":
                dv = dv * gate.view(1, -1, G, n)
        within(cut(y), ry, io)
        within(cut(rstd), rr)
        within(cut(dx), rdx, io)
        if centred:
            within(cut(mean), rm)
        if z is not None:
            within(cut(dz), rdz, io)
        for j, t in enumerate((dv * xh, dv)):
            s = t.view(-1, D).sum(0, 300)
            total[j] += s.v
            off[j] += s.e
    within(sums, Run(total, off))


DROPS = [(3, 11000, 2048, "bf16"), (2, 1500000, 24, "bf16"), (3, 11000, 2049, "bf16"), (1, 24000000, 3, "bf16"), (3, 5500, 2048, "f32"), (1, 12000000, 3, "f32")]


@pytest.mark.parametrize("B,L,D,io", DROPS)
def test_dropout_past_the_caches(bd, B, L, D, io):  # noqa: F811
    """A sample of rows against the generator in whole numbers; the gate's gradient against the sum of what dx and x give (gates of one and p = 1/2, so
    dx is dout times 2 or 0; at most 300 additions for a value, each off by 2^-24 of the magnitudes)."""
    assert 2 * B * L * D * SIZE[io] > CACHES
    g, each = gen(D), B > 1
    x, residual, dout = (normal(g, B, L, D, io=io) for _ in range(3))
    gate = normal(g, B, D) if each else normal(g, D)
    rows = torch.cat([torch.tensor([0, 1, L - 1, L % (B * L), B * L - 1], device="cuda"), torch.randint(0, B * L, (300,), generator=g, device="cuda")])

    def kept(p, key, site):
        blocks = (D + 7) // 8
        row, block = np.meshgrid(rows.cpu().numpy(), np.arange(blocks) + (site << 17), indexing="ij")
        words = philox([row, block, np.full_like(row, key[1] % (1 << 32)), np.full_like(row, key[1] >> 32)], (key[0] % (1 << 32), key[0] >> 32))
        bits = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], -1).reshape(len(row), blocks * 8)[:, :D]
        T = int(p * 65536 + 0.5)
        return torch.from_numpy(bits.astype(np.int64) >= T).cuda(), 65536 / (65536 - T)

    sample = lambda t: t.reshape(B * L, D)[rows]  # noqa: E731
    key, site = (123456789, (1 << 40) + 17), 5
    desc, out, dev_key = bd.make_dropout_desc(B, L, D, io=io, p=0.1, site=site), torch.empty_like(x), torch.tensor(key, device="cuda")
    bd.bimamba_dropout_add(desc, dev_key, x, gate, residual, out)
    mask, factor = kept(np.float32(0.1), key, site)
    with torch.device("cuda"):
        vector = Run(gate[rows // L] if each else gate)
        made = Run(sample(x)) * (Run(factor, U32 * factor) * vector)
        within(sample(out), Run(torch.where(mask, made.v, 0.0), torch.where(mask, made.e, 0.0)) + Run(sample(residual)), io)

    desc, dx, dgate = bd.make_dropout_desc(B, L, D, io=io, p=0.5, site=site), torch.empty_like(x), nans(*gate.shape)
    bd.bimamba_dropout_add_bwd(desc, dev_key, x, torch.ones_like(gate), dout, dx, dgate, workspace(bd.bimamba_dropout_add_bwd_workspace_bytes(desc, each)))
    assert torch.equal(sample(dx), torch.where(kept(0.5, key, site)[0], 2 * sample(dout), 0.0))
    for b in range(B):
        terms, got = dx[b].double() * x[b].double(), dgate[b] if each else dgate
        assert bool(((got.double() - terms.sum(0)).abs() <= 300 * U32 * terms.abs().sum(0)).all())
