"""Dropout into the residual stream and its gradients through the C ABI: masks bit by bit against the generator in whole numbers, values
in 64 bits."""
import math

import numpy as np
import pytest
import torch

from running_error import TYPES, U32, Run, blank, cuda, gen, nans, normal, wide, within, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bd():
    from paper_2511_15927_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return binding


def philox(counter, key):
    """Ten rounds of Philox4x32 on arrays of whole numbers."""
    c, k, low = [np.asarray(x, dtype=np.uint64) for x in counter], list(key), np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) % (1 << 32), (k[1] + 0xBB67AE85) % (1 << 32)]
    return c


def kept(rows, D, p, key, site):
    """Which values of [rows, D] are kept, and the factor of those."""
    seed, offset = (int(v) % (1 << 64) for v in key)
    blocks = (D + 7) // 8
    row, block = np.meshgrid(np.arange(rows), np.arange(blocks) + (site << 17), indexing="ij")
    words = philox([row, block, np.full_like(row, offset % (1 << 32)), np.full_like(row, offset >> 32)], (seed % (1 << 32), seed >> 32))
    bits = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], -1).reshape(rows, blocks * 8)[:, :D].astype(np.int64)
    T = math.floor(float(np.float32(p)) * 65536 + 0.5)
    return torch.from_numpy(bits >= T), 65536 / (65536 - T) if T < 65536 else 0.0


def test_the_generator_gives_its_published_words():
    """The known answers that its authors give for counters and keys of zeros and of ones."""
    assert [int(w) for w in philox([0, 0, 0, 0], (0, 0))] == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    ones = 0xFFFFFFFF
    assert [int(w) for w in philox([ones] * 4, (ones, ones))] == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


KEYS = [(0, 0), (-1, -1), (1 << 62, 5), (123456789, (1 << 40) + 17), (-(1 << 63), (1 << 63) - 1)]
SHAPES = [(1, 1, 1), (2, 3, 3), (1, 5, 7), (2, 4, 8), (3, 2, 12), (1, 9, 63), (2, 30, 64), (4, 17, 130), (1, 40, 512), (2, 3, 513), (2, 5, 2048), (1, 2, 5003),
          (70, 3, 24), (1, 3000, 16)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,D", SHAPES)
def test_masks_and_values(bd, B, L, D, io):
    for n, key in enumerate(KEYS):
        p, site = (0.1, 0.5, 0.0, 1.0, 0.93)[n], (0, 1, 32767, 7, 2)[n]
        g = gen(100 * n + D)
        x, residual = normal(g, B, L, D, io=io), normal(g, B, L, D, io=io) if n % 2 == 0 else None
        gate = (None, normal(g, D), normal(g, B, D))[n % 3]
        extra = (0, 3, 8)[n % 3]
        desc = bd.make_dropout_desc(B, L, D, io=io, p=p, site=site)
        k = torch.tensor(key, device="cuda")
        out = blank((B, L, D), io, extra, extra // 2)
        dev_gate = None if gate is None else wide(gate, 5, 2) if gate.dim() == 2 else gate.cuda()
        bd.bimamba_dropout_add(desc, k, wide(x, extra, extra // 2), dev_gate, None if residual is None else wide(residual, extra, 0), out)
        mask, factor = kept(B * L, D, p, key, site)
        mask = mask.view(B, L, D)
        vector = Run(1.0) if gate is None else Run(gate[:, None] if gate.dim() == 2 else gate)
        made = Run(x) * (Run(factor, U32 * factor) * vector)
        ref = Run(torch.where(mask, made.v, 0.0), torch.where(mask, made.e, 0.0))
        if residual is not None:
            ref = ref + Run(residual)
        within(out, ref, io)
        # gradients
        dout = normal(g, B, L, D, io=io)
        dx, dgate = blank((B, L, D), io, extra, extra // 2), None if gate is None else nans(*gate.shape)
        ws = workspace(bd.bimamba_dropout_add_bwd_workspace_bytes(desc, gate is not None and gate.dim() == 2))
        call = lambda dx, dgate: bd.bimamba_dropout_add_bwd(desc, k, wide(x, extra, 0) if gate is not None else None, dev_gate,  # noqa: E731
                                                            wide(dout, extra, extra // 2), dx, dgate, ws)
        call(dx, dgate)
        d = Run(dout) * Run(factor, U32 * factor)
        d = Run(torch.where(mask, d.v, 0.0), torch.where(mask, d.e, 0.0))
        within(dx, d * vector, io)
        if gate is not None:
            terms = d * Run(x)
            within(dgate, terms.sum(1, L) if gate.dim() == 2 else terms.view(B * L, D).sum(0, B * L))
            again = torch.empty_like(dgate)
            call(torch.empty_like(dx), again)
            assert torch.equal(dgate, again)


def test_share_that_is_kept(bd):
    """Of 2^22 values, to six standard deviations."""
    x = torch.ones(1, 1024, 4096, device="cuda")
    for p in (0.1, 0.5):
        out = torch.empty_like(x)
        bd.bimamba_dropout_add(bd.make_dropout_desc(1, 1024, 4096, io="f32", p=p), torch.tensor([5, 9], device="cuda"), x, None, None, out)
        T = math.floor(p * 65536 + 0.5) / 65536
        assert abs(float((out > 0).float().mean()) - (1 - T)) < 6 * math.sqrt(T * (1 - T) / out.numel())
        assert abs(float(out.double().mean()) - 1) < 6 * math.sqrt(T / (1 - T) / out.numel()) + 2.0 ** -22
