"""The gated recurrence in the forms that sizes choose: against the walk in 64 bits with its running error bound, made on the GPU."""
import math

import pytest
import torch

from running_error import HALF_STEP
from test_gpu_recurrence import bd, forward_ref, gradient_ref, inputs, run_backward, run_forward  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def empty_afterwards():
    yield
    torch.cuda.empty_cache()


def within(got, ref, io="f32"):
    """got (rounded once more where io is bf16) lies within ref's bound; both on the GPU."""
    bound = ref.e + (HALF_STEP[io] * (ref.v.abs() + ref.e) if io != "f32" else 0.0) + 1e-37
    off = (got.double() - ref.v).abs()
    bad = ~(off <= bound)
    assert got.shape == ref.v.shape and not bool(bad.any()), "%d of %d beyond the bound, worst %.3g times it" % (
        int(bad.sum()), bad.numel(), float((off / bound)[bad].nan_to_num(nan=math.inf).max()))


def both_ways(bd, B, L, D, io, gate, reverse, seed, lengths, extra=0):  # noqa: F811
    """A walk and its gradients, twice: within their bounds, and the same bits."""
    i = {k: None if t is None else t.cuda() for k, t in inputs(B, L, D, io, gate, seed, lengths).items()}
    out = run_forward(bd, i, io, gate, reverse, extra=extra)
    back = run_backward(bd, i, io, gate, reverse, out["states"], extra)
    with torch.device("cuda"):
        for k, ref in zip(("y", "h_out", "states"), forward_ref(i, gate, reverse, True, True)):
            within(out[k], ref, io if k == "y" else "f32")
        for k, ref in zip(("dx", "dg", "dbias", "dh_in"), gradient_ref(i, gate, reverse, out["states"])):
            if back[k] is not None:
                within(back[k], ref, io if k in ("dx", "dg") else "f32")
    again = run_forward(bd, i, io, gate, reverse, extra=extra), run_backward(bd, i, io, gate, reverse, out["states"], extra)
    for one, two in ((out, again[0]), (back, again[1])):
        assert all(v is None or torch.equal(v, two[k]) for k, v in one.items())


@pytest.mark.parametrize("B,L,D", [(129, 700, 129), (129, 500, 257), (170, 900, 129)])
@pytest.mark.parametrize("reverse", [0, 1])
def test_a_last_tile_of_one_channel_waits_for_its_own_pieces(bd, B, L, D, reverse):  # noqa: F811
    """Rows that share cache lines, two channels a lane, several pieces, a last tile of one channel, whose lanes read the channel before it as
    well; of the eight queues some begin between the tiles of one sequence.  (The words of that channel belong to pieces of another queue: a
    wait for them would not be in the order of the walk.  It would not show in the results.)"""
    tiles = -(-D // 128)
    assert tiles * B >= 256 and D % 128 == 1 and any(q * tiles * B // 8 % tiles for q in range(8))
    both_ways(bd, B, L, D, "bf16", ("sigmoid", "log")[reverse], reverse, B + L + D, L == 700)


# tokens of a wave, waves and channels a lane: what the rule of sizes gives them in bf16 (fp32: one channel), forward and for gradients
FORMS = [(3, 1, 200), (2, 3, 50), (2, 3, 200), (3, 30, 40), (2, 32, 256), (3, 50, 40), (2, 64, 256), (2, 128, 64), (2, 200, 100), (90, 200, 256), (3, 300, 64),
         (40, 500, 100)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,D", FORMS)
def test_every_form_is_there(bd, B, L, D, io):  # noqa: F811
    """(Outputs start as NaN: a form that is planned and not there would leave them.)"""
    n = FORMS.index((B, L, D))
    both_ways(bd, B, L, D, io, ("sigmoid", "log")[n % 2], n // 2 % 2, 900 + n, n % 3 == 0, extra=(0, 3)[n % 2])


# two channels a lane, sequences of several pieces, tiles whose lanes all own their channels, several of them and a last one that is cut; pieces of
# 16 x 8 and 32 x 8 and, for gradients, 16 x 4; one piece looked back at and several
WIDE = [(350, 300, 128), (180, 300, 256), (150, 300, 257), (130, 500, 256), (90, 700, 256), (57, 1100, 256), (34, 4000, 128)]


@pytest.mark.parametrize("gate", ["log", "sigmoid"])
@pytest.mark.parametrize("reverse", [0, 1])
@pytest.mark.parametrize("B,L,D", WIDE)
def test_two_channels_a_lane_in_whole_tiles(bd, B, L, D, reverse, gate):  # noqa: F811
    n = WIDE.index((B, L, D)) + reverse + 2 * (gate == "log")
    both_ways(bd, B, L, D, "bf16", gate, reverse, 700 + n, n % 3 == 0, extra=(0, 3)[n % 2])


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,D", [(2, 4096, 70), (1, 33, 130)])
def test_channels_that_remember_far(bd, B, L, D, io):  # noqa: F811
    """10^4 to 10^5 tokens: what the factor is off by in every step stays in the states, which leave the call in fp32 whatever the activations' type
    (the walk's bound: 3 units of 2^-24 a step for bf16, 1 for fp32, and 4 for the step's own rounding)."""
    i = {k: None if t is None else t.cuda() for k, t in inputs(B, L, D, io, "sigmoid", 40 + L).items()}
    i["bias"] = torch.linspace(math.log(1e4), math.log(1e5), D, device="cuda")
    i["g"] = (i["g"] / 8).to(i["x"].dtype)
    i["x"], i["h_in"] = torch.ones_like(i["x"]), torch.ones_like(i["h_in"])   # (the state stays at 1: what the factors are off by adds up)
    out = run_forward(bd, i, io, "sigmoid", 0, add=False)
    back = run_backward(bd, i, io, "sigmoid", 0, out["states"])
    with torch.device("cuda"):
        y, last, kept = forward_ref(i, "sigmoid", 0, True, False)
        dx, dg, dbias, dh_in = gradient_ref(i, "sigmoid", 0, out["states"])
        assert bool(((last.v - 1).abs() < 1e-12).all()) and bool((last.e <= 9 * 2.0 ** -24 * L).all())
        for got, ref in ((out["h_out"], last), (out["states"], kept), (back["dh_in"], dh_in), (back["dbias"], dbias)):
            within(got, ref)
        for got, ref in ((out["y"], y), (back["dx"], dx), (back["dg"], dg)):
            within(got, ref, io)
