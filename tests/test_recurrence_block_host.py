"""CPU-only checks of the gated recurrence, the group norm and dropout: what they refuse is refused on the host, before anything is
launched (no GPU is touched: the pointers are not memory)."""
import ctypes as C

import pytest
import torch

from paper_2511_15927_amd import binding as bd

OK, NULL, SHAPE, UNSUPPORTED, ALIGN, SMALL, ALIAS = 0, -1, -2, -3, -4, -5, -8
AT = [k << 40 for k in range(20)]   # addresses far from each other


def ref(s):
    return None if s is None else C.byref(s)


def view(p, width=64, L=10, st=None, sb=None):
    st = width if st is None else st
    return bd.Tensor(p, L * st if sb is None else sb, st)


def made(make, base, kw):
    """A descriptor of `base` with the fields that a call names changed, and what is left of the call."""
    d = make(**base)
    for k in [k for k in kw if k in dict(type(d)._fields_)]:
        setattr(d, k, kw.pop(k))
    return d, kw


def recurrence(**kw):
    d, kw = made(bd.make_recurrence_desc, dict(batch=2, seqlen=10, d_inner=64), kw)
    a = dict(x=view(AT[1]), g=view(AT[2]), bias=AT[3], add=view(AT[4]), lengths=AT[5], h_in=AT[6], y=view(AT[7]), h_out=AT[8], states=AT[9], ws=AT[10],
             ws_bytes=1 << 40, desc=d)
    a.update(kw)
    return bd.lib().bimamba_recurrence(ref(a["desc"]), ref(a["x"]), ref(a["g"]), a["bias"], ref(a["add"]), a["lengths"], a["h_in"], ref(a["y"]),
                                       a["h_out"], a["states"], a["ws"], a["ws_bytes"], None)


def common(call, width, views, most_batch=True):
    """What every call's descriptor and views are checked for."""
    assert call(desc=None) == NULL and call(struct_size=4) == SHAPE
    assert call(**{width: 0}) == SHAPE and call(batch=-1) == SHAPE and call(seqlen=-1) == SHAPE and call(io_dtype=7) == UNSUPPORTED
    assert call(batch=65535, seqlen=65535) == UNSUPPORTED
    if most_batch:
        assert call(batch=65536, seqlen=1) == UNSUPPORTED
    for name, written in views.items():
        assert call(**{name: view(None)}) == NULL, name
        at = AT[11]
        assert call(**{name: view(at + 1)}) == ALIGN and call(**{name: view(at, st=-64)}) == SHAPE and call(**{name: view(at, st=1 << 60)}) == SHAPE, name
        if written:
            assert call(**{name: view(at, st=63)}) == SHAPE and call(**{name: view(at, sb=64)}) == SHAPE, name


def test_recurrence_refusals():
    common(recurrence, "d_inner", dict(x=0, g=0, add=0, y=1))
    assert recurrence(x=None) == NULL and recurrence(g=None) == NULL and recurrence(y=None) == NULL
    assert recurrence(gate=2) == UNSUPPORTED and recurrence(reverse=2) == SHAPE and recurrence(d_inner=65537) == UNSUPPORTED
    assert recurrence(gate=0) == UNSUPPORTED                      # a log gate has no bias
    for name, odd in dict(bias=2, lengths=4, h_in=2, h_out=1, states=2).items():
        assert recurrence(**{name: AT[11] + odd}) == ALIGN, name
    for a, b in (("y", "x"), ("y", "g"), ("y", "add")):           # half a row on
        assert recurrence(**{a: view(AT[11]), b: view(AT[11] + 64)}) == ALIAS, (a, b)
    assert recurrence(y=view(AT[1])) == ALIAS
    for out in ("h_out", "states"):
        for read in (1, 2, 3, 4, 5, 6, 7):
            if (out, read) != ("h_out", 6):                       # (the state may be replaced)
                assert recurrence(**{out: AT[read]}) == ALIAS, (out, read)
    assert recurrence(h_out=AT[6] + 4) == ALIAS and recurrence(h_out=AT[9]) == ALIAS
    for read in (3, 5, 6):
        assert recurrence(y=view(AT[read])) == ALIAS
    assert recurrence(batch=0) == OK


def test_recurrence_workspace():
    long = bd.make_recurrence_desc(1, 65536, 64)
    need = bd.bimamba_recurrence_workspace_bytes(long)
    assert need > 0 and bd.bimamba_recurrence_workspace_bytes(bd.make_recurrence_desc(1, 0, 64)) == 0
    one = dict(desc=long, x=view(AT[1], L=65536), g=view(AT[2], L=65536), y=view(AT[7], L=65536), add=None)
    assert recurrence(ws_bytes=need - 1, **one) == SMALL and recurrence(ws=None, **one) == NULL and recurrence(ws=AT[10] + 8, **one) == ALIGN
    for at in (1, 2, 3, 5, 6, 7, 8, 9):
        assert recurrence(**dict(one, ws=AT[at])) == ALIAS, at


@pytest.mark.parametrize("batch, seqlen, d", [(8192, 64, 65536), (64, 8192, 65536), (1 << 15, 5, 16384), (1, 1 << 29, 64)])
def test_recurrence_of_more_pieces_than_a_grid_holds(batch, seqlen, d):
    """2^23 times 64 steps of 64 channels, and a step less."""
    for call in (recurrence, recurrence_bwd):
        assert call(batch=batch, seqlen=seqlen, d_inner=d) == UNSUPPORTED
    assert bd.bimamba_recurrence_bwd_workspace_bytes(bd.make_recurrence_desc(batch, seqlen, d)) == 0
    fewer = (batch - 1, seqlen) if batch > 1 else (batch, seqlen - 64)
    assert bd.bimamba_recurrence_bwd_workspace_bytes(bd.make_recurrence_desc(*fewer, d)) > 0
    assert bd.bimamba_recurrence_bwd_workspace_bytes(bd.make_recurrence_desc(65535, 4, 65536)) > 0


def test_recurrence_of_the_longest_sequences():
    """Lengths whose pieces do not fit 32 bits when they are rounded up."""
    for L in ((1 << 31) - 1, (1 << 31) - 63, (1 << 31) - 64):
        long = dict(batch=1, seqlen=L, d_inner=1)
        assert bd.bimamba_recurrence_workspace_bytes(bd.make_recurrence_desc(1, L, 1)) == 0
        assert recurrence(x=view(AT[1], 1, L), g=view(AT[2], 1, L), y=view(AT[7], 1, L), add=None, **long) == UNSUPPORTED
        assert recurrence_bwd(**long) == UNSUPPORTED


def recurrence_bwd(**kw):
    d, kw = made(bd.make_recurrence_desc, dict(batch=2, seqlen=10, d_inner=64), kw)
    a = dict(x=view(AT[1]), g=view(AT[2]), bias=AT[3], lengths=AT[4], states=AT[5], dy=view(AT[6]), dh_out=AT[7], dx=view(AT[8]), dg=view(AT[9]),
             dbias=AT[10], dh_in=AT[12], ws=AT[13], ws_bytes=1 << 40, desc=d)
    a.update(kw)
    return bd.lib().bimamba_recurrence_bwd(ref(a["desc"]), ref(a["x"]), ref(a["g"]), a["bias"], a["lengths"], a["states"], ref(a["dy"]), a["dh_out"],
                                           ref(a["dx"]), ref(a["dg"]), a["dbias"], a["dh_in"], a["ws"], a["ws_bytes"], None)


def test_recurrence_bwd_refusals():
    common(recurrence_bwd, "d_inner", dict(x=0, g=0, dy=0, dx=1, dg=1))
    need = bd.bimamba_recurrence_bwd_workspace_bytes(bd.make_recurrence_desc(2, 10, 64))
    assert need > 0 and recurrence_bwd(ws_bytes=need - 1) == SMALL and recurrence_bwd(ws=None) == NULL and recurrence_bwd(ws=AT[13] + 4) == ALIGN
    assert bd.bimamba_recurrence_bwd_workspace_bytes(bd.make_recurrence_desc(2, 10, 64, gate="log")) == 0
    for name in ("x", "g", "dy", "dx", "dg", "states"):
        assert recurrence_bwd(**{name: None}) == NULL, name
    assert recurrence_bwd(gate=0, bias=None) == UNSUPPORTED and recurrence_bwd(gate=0, dbias=None) == UNSUPPORTED
    for name, odd in dict(bias=2, lengths=4, states=2, dh_out=1, dbias=2, dh_in=2).items():
        assert recurrence_bwd(**{name: AT[11] + odd}) == ALIGN, name
    for out in ("dx", "dg"):
        for read in (1, 2, 3, 4, 5, 6, 7):
            assert recurrence_bwd(**{out: view(AT[read])}) == ALIAS, (out, read)
    assert recurrence_bwd(dx=view(AT[9] + 64)) == ALIAS
    for out in ("dbias", "dh_in", "ws"):
        for read in (1, 2, 3, 4, 5, 6, 7, 8, 9):
            if (out, read) != ("dh_in", 7):
                assert recurrence_bwd(**{out: AT[read]}) == ALIAS, (out, read)
    assert recurrence_bwd(dbias=AT[12]) == ALIAS and recurrence_bwd(ws=AT[10]) == ALIAS and recurrence_bwd(dh_in=AT[7] + 4) == ALIAS


def group_norm(**kw):
    d, kw = made(bd.make_group_norm_desc, dict(batch=2, seqlen=10, d_inner=64, groups=4, act="gate_before", centred=1), kw)
    a = dict(x=view(AT[1]), z=view(AT[2]), weight=AT[3], bias=AT[4], y=view(AT[5]), mean=AT[6], rstd=AT[7], desc=d)
    a.update(kw)
    return bd.lib().bimamba_group_norm(ref(a["desc"]), ref(a["x"]), ref(a["z"]), a["weight"], a["bias"], ref(a["y"]), a["mean"], a["rstd"], None)


def group_norm_bwd(**kw):
    d, kw = made(bd.make_group_norm_desc, dict(batch=2, seqlen=10, d_inner=64, groups=4, act="gate_before", centred=1), kw)
    a = dict(x=view(AT[1]), z=view(AT[2]), weight=AT[3], bias=AT[4], mean=AT[5], rstd=AT[6], dy=view(AT[7]), dx=view(AT[8]), dz=view(AT[9]),
             dweight=AT[10], dbias=AT[12], ws=AT[13], ws_bytes=1 << 40, desc=d)
    a.update(kw)
    return bd.lib().bimamba_group_norm_bwd(ref(a["desc"]), ref(a["x"]), ref(a["z"]), a["weight"], a["bias"], a["mean"], a["rstd"], ref(a["dy"]),
                                           ref(a["dx"]), ref(a["dz"]), a["dweight"], a["dbias"], a["ws"], a["ws_bytes"], None)


def test_group_norm_refusals():
    common(group_norm, "d_inner", dict(x=0, z=0, y=1), most_batch=False)
    common(group_norm_bwd, "d_inner", dict(x=0, z=0, dy=0, dx=1, dz=1), most_batch=False)
    for call in (group_norm, group_norm_bwd):
        assert call(groups=0) == SHAPE and call(groups=3) == SHAPE and call(groups=128) == SHAPE and call(centred=2) == SHAPE
        assert call(eps=0.0) == SHAPE and call(eps=float("nan")) == SHAPE and call(eps=float("inf")) == SHAPE
        assert call(act=4) == UNSUPPORTED and call(act=-1) == UNSUPPORTED and call(d_inner=65540) == UNSUPPORTED
        assert call(d_inner=8194, groups=1) == UNSUPPORTED                       # a group beyond the registers of four waves
        assert call(z=None) == NULL and call(act=1) == UNSUPPORTED               # a gate's input without a gate
        assert call(centred=0) == UNSUPPORTED                                    # a mean that nothing takes off
        for name in ("weight", "bias", "mean", "rstd"):
            assert call(**{name: AT[11] + 2}) == ALIGN, name
    for read in (1, 2, 3, 4, 6, 7):
        assert group_norm(y=view(AT[read])) == ALIAS, read
    for read in (1, 2, 3, 4, 5):
        assert group_norm(mean=AT[read]) == ALIAS and group_norm(rstd=AT[read]) == ALIAS, read
    assert group_norm(mean=AT[7]) == ALIAS and group_norm(seqlen=0) == OK and group_norm(batch=0) == OK
    assert group_norm_bwd(dz=None) == NULL and group_norm_bwd(mean=None) == NULL and group_norm_bwd(rstd=None) == NULL
    # 100 rows: workgroups of their own, so there are slots
    need = bd.bimamba_group_norm_bwd_workspace_bytes(bd.make_group_norm_desc(2, 50, 64, 4))
    v = {k: view(AT[n], L=50) for k, n in dict(x=1, z=2, dy=7, dx=8, dz=9).items()}
    assert need > 0 and bd.bimamba_group_norm_bwd_workspace_bytes(bd.make_group_norm_desc(2, 0, 64, 4)) == 0
    assert group_norm_bwd(seqlen=50, ws_bytes=need - 1, **v) == SMALL and group_norm_bwd(seqlen=50, ws=None, **v) == NULL
    assert group_norm_bwd(seqlen=50, ws=AT[13] + 8, **v) == ALIGN and group_norm_bwd(seqlen=50, **dict(v, ws=AT[1])) == ALIAS
    for out in ("dx", "dz"):
        for read in (1, 2, 3, 4, 5, 6, 7):
            assert group_norm_bwd(**{out: view(AT[read])}) == ALIAS, (out, read)
    assert group_norm_bwd(dx=view(AT[9] + 64)) == ALIAS
    for out in ("dweight", "dbias"):
        for read in (1, 2, 3, 4, 5, 6, 7, 8, 9):
            assert group_norm_bwd(**{out: AT[read]}) == ALIAS, (out, read)
    assert group_norm_bwd(dweight=AT[12]) == ALIAS and group_norm_bwd(dweight=AT[11] + 1) == ALIGN


def dropout(**kw):
    d, kw = made(bd.make_dropout_desc, dict(batch=2, seqlen=10, d_model=64), kw)
    a = dict(key=AT[1], x=view(AT[2]), gate=AT[3], stride=64, residual=view(AT[4]), out=view(AT[5]), desc=d)
    a.update(kw)
    return bd.lib().bimamba_dropout_add(ref(a["desc"]), a["key"], ref(a["x"]), a["gate"], a["stride"], ref(a["residual"]), ref(a["out"]), None)


def dropout_bwd(**kw):
    d, kw = made(bd.make_dropout_desc, dict(batch=2, seqlen=10, d_model=64), kw)
    a = dict(key=AT[1], x=view(AT[2]), gate=AT[3], stride=64, dout=view(AT[4]), dx=view(AT[5]), dgate=AT[6], ws=AT[7], ws_bytes=1 << 40, desc=d)
    a.update(kw)
    return bd.lib().bimamba_dropout_add_bwd(ref(a["desc"]), a["key"], ref(a["x"]), a["gate"], a["stride"], ref(a["dout"]), ref(a["dx"]), a["dgate"],
                                            a["ws"], a["ws_bytes"], None)


def test_dropout_refusals():
    common(dropout, "d_model", dict(x=0, residual=0, out=1))
    common(dropout_bwd, "d_model", dict(x=0, dout=0, dx=1))
    for call in (dropout, dropout_bwd):
        assert call(p=-0.1) == SHAPE and call(p=1.1) == SHAPE and call(p=float("nan")) == SHAPE
        assert call(site=-1) == UNSUPPORTED and call(site=1 << 15) == UNSUPPORTED and call(d_model=(1 << 20) + 1, stride=0) == UNSUPPORTED
        assert call(key=None) == NULL and call(key=AT[1] + 4) == ALIGN and call(gate=AT[3] + 2) == ALIGN
        assert call(stride=63) == SHAPE and call(stride=-64) == SHAPE and call(stride=1 << 61) == SHAPE
        assert call(batch=0) == OK
    for read in (1, 2, 3):
        assert dropout(out=view(AT[read])) == ALIAS and dropout_bwd(dx=view(AT[read])) == ALIAS, read
    assert dropout(out=view(AT[4] + 64)) == ALIAS and dropout_bwd(dx=view(AT[4] + 64)) == ALIAS
    assert dropout(x=None) == NULL and dropout(out=None) == NULL and dropout_bwd(dout=None) == NULL and dropout_bwd(dx=None) == NULL
    assert dropout_bwd(x=None) == NULL                                          # dgate needs it
    for read in (1, 2, 3, 4, 5):
        assert dropout_bwd(dgate=AT[read]) == ALIAS, read
    assert dropout_bwd(dgate=AT[6] + 2) == ALIGN
    need = bd.bimamba_dropout_add_bwd_workspace_bytes(bd.make_dropout_desc(2, 500, 64), True)
    v = {k: view(AT[n], L=500) for k, n in dict(x=2, dout=4, dx=5).items()}
    assert need > 0 and dropout_bwd(seqlen=500, ws_bytes=need - 1, **v) == SMALL and dropout_bwd(seqlen=500, ws=None, **v) == NULL
    assert dropout_bwd(seqlen=500, **dict(v, ws=AT[7] + 8)) == ALIGN and dropout_bwd(seqlen=500, **dict(v, ws=AT[6])) == ALIAS
    assert dropout_bwd(seqlen=500, **dict(v, dgate=None, ws=AT[5], batch=0)) == OK


def test_bindings_check_tensors():
    """On the CPU every tensor is the wrong one; what is wrong is said of the first."""
    t, f = torch.zeros(2, 10, 64), torch.zeros(64)
    key = torch.zeros(2, dtype=torch.int64)
    for call in (lambda: bd.bimamba_recurrence(bd.make_recurrence_desc(2, 10, 64, io="f32"), t, t, f, t),
                 lambda: bd.bimamba_recurrence_bwd(bd.make_recurrence_desc(2, 10, 64, io="f32"), t, t, f, t, t, t, t),
                 lambda: bd.bimamba_group_norm(bd.make_group_norm_desc(2, 10, 64, 4, io="f32"), t, None, f, f, t),
                 lambda: bd.bimamba_group_norm_bwd(bd.make_group_norm_desc(2, 10, 64, 4, io="f32"), t, None, f, f, None, t, t, t, None, f, f, None)):
        with pytest.raises(AssertionError, match="^x: .*on cpu"):
            call()
    for call in (lambda: bd.bimamba_dropout_add(bd.make_dropout_desc(2, 10, 64, io="f32"), key, t, None, None, t),
                 lambda: bd.bimamba_dropout_add_bwd(bd.make_dropout_desc(2, 10, 64, io="f32"), key, t, None, t, t)):
        with pytest.raises(AssertionError, match="^key: .*on cpu"):
            call()
    with pytest.raises(AssertionError, match="descriptor of another call"):
        bd.bimamba_recurrence(bd.make_norm_desc(2, 10, 64), t, t, f, t)
    with pytest.raises(KeyError):
        bd.make_recurrence_desc(2, 10, 64, gate="tanh")
