"""CPU-only checks of the calls around the mixers: what they refuse is refused on the host, before anything is launched (no GPU is
touched: the pointers are not memory)."""
import ctypes as C

import pytest
import torch

from paper_2511_15927_amd import binding as bd

OK, NULL, SHAPE, UNSUPPORTED, ALIGN, SMALL, ALIAS = 0, -1, -2, -3, -4, -5, -8
A, B, Z, D, E, F = (k << 40 for k in range(1, 7))   # addresses far from each other


def ref(s):
    return None if s is None else C.byref(s)


def view(p, width, L=10, st=None, sb=None):
    st = width if st is None else st
    return bd.Tensor(p, L * st if sb is None else sb, st)


TOK = bd.Tokens(A, 10, 1)


def embed(desc=None, tok=TOK, table=B, out=view(Z, 64), **kw):
    desc = bd.make_embed_desc(**dict(dict(batch=2, seqlen=10, d_model=64, vocab=100), **kw)) if desc is None else desc
    return bd.lib().bimamba_embed(ref(desc), ref(tok), table, ref(out), None)


def test_embed_refusals():
    d = bd.make_embed_desc(2, 10, 64, 100)
    d.struct_size += 4
    assert embed(d) == SHAPE
    assert bd.lib().bimamba_embed(None, ref(TOK), B, ref(view(Z, 64)), None) == NULL
    assert embed(tok=None) == NULL and embed(out=None) == NULL and embed(table=None) == NULL
    assert embed(tok=bd.Tokens(None, 10, 1)) == NULL and embed(out=view(None, 64)) == NULL
    assert embed(batch=-1) == SHAPE and embed(d_model=0) == SHAPE and embed(vocab=0) == SHAPE and embed(scale=float("nan")) == SHAPE
    assert embed(vocab=1 << 21) == UNSUPPORTED and embed(d_model=(1 << 20) + 1) == UNSUPPORTED
    assert embed(batch=65536, seqlen=32768) == UNSUPPORTED
    d = bd.make_embed_desc(2, 10, 64, 100)
    d.io_dtype = 7
    assert embed(d) == UNSUPPORTED
    assert embed(tok=bd.Tokens(A + 4, 10, 1)) == ALIGN and embed(table=B + 2) == ALIGN and embed(out=view(Z + 1, 64)) == ALIGN
    assert embed(out=view(Z, 64, st=63)) == SHAPE and embed(out=view(Z, 64, sb=64)) == SHAPE    # rows on top of each other
    assert embed(out=view(Z, 64, st=-64)) == SHAPE and embed(tok=bd.Tokens(A, -10, 1)) == SHAPE
    assert embed(out=view(Z, 64, st=1 << 60)) == SHAPE                                          # beyond any address
    assert embed(out=view(B + 4, 64)) == ALIAS and embed(out=view(A, 64)) == ALIAS
    assert embed(batch=0) == OK and embed(seqlen=0, tok=bd.Tokens(None, 0, 0), out=view(None, 64), table=None) == OK


def embed_bwd(desc=None, tok=TOK, dout=view(B, 64), dtable=Z, ws=D, ws_bytes=1 << 40, **kw):
    desc = bd.make_embed_desc(**dict(dict(batch=2, seqlen=10, d_model=64, vocab=100), **kw)) if desc is None else desc
    return bd.lib().bimamba_embed_bwd(ref(desc), ref(tok), ref(dout), dtable, ws, ws_bytes, None)


def test_embed_bwd_refusals():
    need = bd.bimamba_embed_bwd_workspace_bytes(bd.make_embed_desc(2, 10, 64, 100))
    assert need > 0 and bd.bimamba_embed_bwd_workspace_bytes(bd.make_embed_desc(2, 10, 64, 0)) == 0
    assert embed_bwd(tok=None) == NULL and embed_bwd(dout=None) == NULL and embed_bwd(dtable=None) == NULL and embed_bwd(ws=None) == NULL
    assert embed_bwd(dtable=Z + 2) == ALIGN and embed_bwd(ws=D + 8) == ALIGN and embed_bwd(dout=view(B + 1, 64)) == ALIGN
    assert embed_bwd(ws_bytes=need - 1) == SMALL
    assert embed_bwd(dtable=B) == ALIAS and embed_bwd(dtable=D) == ALIAS and embed_bwd(ws=A) == ALIAS and embed_bwd(dtable=A) == ALIAS
    assert embed_bwd(vocab=1 << 21) == UNSUPPORTED and embed_bwd(d_model=-1) == SHAPE
    assert embed_bwd(batch=1 << 15, seqlen=1 << 15, d_model=1 << 19) == UNSUPPORTED     # more waves than a grid holds


def norm(desc=None, x=view(A, 64), w=B, b=Z, stride=0, y=view(D, 64), mean=E, rstd=F, **kw):
    desc = bd.make_norm_desc(**dict(dict(batch=2, seqlen=10, d_model=64), **kw)) if desc is None else desc
    return bd.lib().bimamba_layer_norm(ref(desc), ref(x), w, b, stride, ref(y), mean, rstd, None)


def test_layer_norm_refusals():
    d = bd.make_norm_desc(2, 10, 64)
    d.struct_size = 0
    assert norm(d) == SHAPE
    assert norm(x=None) == NULL and norm(y=None) == NULL and norm(x=view(None, 64)) == NULL
    assert norm(eps=0.0) == SHAPE and norm(eps=float("inf")) == SHAPE and norm(d_model=0) == SHAPE and norm(seqlen=-1) == SHAPE
    assert norm(d_model=65537) == UNSUPPORTED and norm(batch=65536) == UNSUPPORTED
    assert norm(stride=63) == SHAPE and norm(stride=-64) == SHAPE
    assert norm(w=B + 2) == ALIGN and norm(b=Z + 1) == ALIGN and norm(mean=E + 2) == ALIGN and norm(y=view(D + 1, 64)) == ALIGN
    assert norm(y=view(D, 64, st=32)) == SHAPE
    assert norm(y=view(A, 64)) == ALIAS and norm(y=view(A + 64, 64)) == ALIAS                      # in place, and half a row on
    assert norm(y=view(B, 64)) == ALIAS and norm(mean=A) == ALIAS and norm(rstd=E) == ALIAS and norm(mean=D + 128) == ALIAS
    assert norm(seqlen=0) == OK


def norm_bwd(desc=None, x=view(A, 64), w=B, stride=0, mean=Z, rstd=D, dy=view(E, 64), dx=view(F, 64), dw=7 << 40, db=8 << 40, ws=9 << 40,
             ws_bytes=1 << 30, **kw):
    desc = bd.make_norm_desc(**dict(dict(batch=2, seqlen=10, d_model=64), **kw)) if desc is None else desc
    return bd.lib().bimamba_layer_norm_bwd(ref(desc), ref(x), w, stride, mean, rstd, ref(dy), ref(dx), dw, db, ws, ws_bytes, None)


def test_layer_norm_bwd_refusals():
    d = bd.make_norm_desc(2, 10, 64)
    for per_batch in (False, True):
        need = bd.bimamba_layer_norm_bwd_workspace_bytes(d, per_batch)
        assert need > 0
        assert norm_bwd(stride=64 if per_batch else 0, ws_bytes=need - 1) == SMALL
    assert bd.bimamba_layer_norm_bwd_workspace_bytes(bd.make_norm_desc(2, 10, 0), False) == 0
    assert norm_bwd(x=None) == NULL and norm_bwd(dy=None) == NULL and norm_bwd(dx=None) == NULL and norm_bwd(mean=None) == NULL
    assert norm_bwd(rstd=None) == NULL and norm_bwd(ws=None) == NULL
    assert norm_bwd(ws=(9 << 40) + 4) == ALIGN and norm_bwd(dw=(7 << 40) + 1) == ALIGN and norm_bwd(dx=view(F + 1, 64)) == ALIGN
    assert norm_bwd(dx=view(A, 64)) == ALIAS and norm_bwd(dx=view(E, 64)) == ALIAS and norm_bwd(dw=8 << 40) == ALIAS
    assert norm_bwd(db=E) == ALIAS and norm_bwd(ws=A) == ALIAS and norm_bwd(dw=B) == ALIAS and norm_bwd(dx=view(B, 64)) == ALIAS
    assert norm_bwd(stride=10) == SHAPE


def scores(desc=None, logits=view(A, 100), targets=bd.Tokens(B, 10, 1), out=None, ws=Z, ws_bytes=1 << 30, **kw):
    desc = bd.make_logits_desc(**dict(dict(batch=2, seqlen=10, vocab=100), **kw)) if desc is None else desc
    out = bd.Scores(D, E, F, None, None) if out is None else out
    return bd.lib().bimamba_log_probs(ref(desc), ref(logits), ref(targets), ref(out), ws, ws_bytes, None)


def test_log_probs_refusals():
    assert scores(logits=None) == NULL and scores(logits=view(None, 100)) == NULL
    assert scores(targets=None) == NULL and scores(targets=None, out=bd.Scores(None, E, None, None, None), targets_only=1) == NULL
    assert scores(out=bd.Scores(None, None, None, None, None)) == NULL                             # nothing wanted
    assert scores(vocab=0) == SHAPE and scores(top_k=-1) == SHAPE and scores(targets_only=2) == SHAPE
    assert scores(top_k=9) == UNSUPPORTED and scores(vocab=5, top_k=6, logits=view(A, 5)) == SHAPE
    assert scores(top_k=3) == SHAPE                                                                # nowhere to put them
    assert scores(out=bd.Scores(D, None, None, 7 << 40, None)) == SHAPE                            # none of them wanted
    assert scores(out=bd.Scores(D + 2, None, None, None, None)) == ALIGN
    assert scores(out=bd.Scores(None, None, None, None, (7 << 40) + 4), top_k=1) == ALIGN
    assert scores(out=bd.Scores(D, D, None, None, None)) == ALIAS and scores(out=bd.Scores(A, None, None, None, None)) == ALIAS
    assert scores(out=bd.Scores(B, None, None, None, None)) == ALIAS
    big = bd.make_logits_desc(1, 1, 100000, top_k=8)
    need = bd.bimamba_log_probs_workspace_bytes(big)
    assert need > 0 and bd.bimamba_log_probs_workspace_bytes(bd.make_logits_desc(1, 1, 10)) == 0
    out = bd.Scores(D, None, None, None, 7 << 40)
    one = dict(logits=view(A, 100000, L=1), out=out)
    assert scores(big, ws_bytes=need - 1, **one) == SMALL and scores(big, ws=None, **one) == NULL and scores(big, ws=Z + 8, **one) == ALIGN
    assert scores(batch=1 << 12, seqlen=1 << 12, logits=view(A, 100, L=1 << 12), targets=bd.Tokens(B, 1 << 12, 1)) == UNSUPPORTED
    assert scores(batch=0) == OK


def scores_bwd(logits=view(A, 100), targets=bd.Tokens(B, 10, 1), lse=Z, entropy=D, dlogp=E, dentropy=F, dlogits=view(7 << 40, 100), **kw):
    desc = bd.make_logits_desc(**dict(dict(batch=2, seqlen=10, vocab=100), **kw))
    return bd.lib().bimamba_log_probs_bwd(ref(desc), ref(logits), ref(targets), lse, entropy, dlogp, dentropy, ref(dlogits), None)


def test_log_probs_bwd_refusals():
    assert scores_bwd(logits=None) == NULL and scores_bwd(dlogits=None) == NULL and scores_bwd(lse=None) == NULL
    assert scores_bwd(targets=None) == NULL and scores_bwd(entropy=None) == NULL
    assert scores_bwd(lse=Z + 2) == ALIGN and scores_bwd(dlogits=view((7 << 40) + 1, 100)) == ALIGN
    assert scores_bwd(dlogits=view(7 << 40, 100, st=99)) == SHAPE
    assert scores_bwd(dlogits=view(A + 2, 100)) == ALIAS and scores_bwd(dlogits=view(A, 100, st=101)) == ALIAS
    assert scores_bwd(dlogits=view(E, 100)) == ALIAS and scores_bwd(dlogits=view(B, 100)) == ALIAS
    assert scores_bwd(seqlen=0) == OK


def test_log_probs_bwd_of_targets_only_wants_targets():
    assert scores_bwd(targets=None, dlogp=None, targets_only=1, dlogits=view(A + 2, 100)) == NULL
    assert scores_bwd(targets=None, dlogp=None, dlogits=view(A + 2, 100)) == ALIAS      # (without the flag it is the next check that refuses)


def test_log_probs_with_the_rest_of_a_log_sum():
    """A descriptor that ends before `reserved` is one without it; with it the array is checked like the others."""
    d = bd.make_logits_desc(2, 10, 100)
    assert d.struct_size == 40
    for d.struct_size in (24, 27, 29, 32, 36, 44):
        assert scores(d) == SHAPE
    d.struct_size, d.reserved = 40, 1
    assert scores(d) == SHAPE
    d.reserved = 0
    for at, rc in ((1 << 50 | 2, ALIGN), (A, ALIAS), (B + 4, ALIAS), (E, ALIAS)):
        d.lse_rest = at
        assert scores(d) == rc, at
    d.struct_size, d.reserved, d.lse_rest = 28, 1, 2        # (not read)
    assert scores(d, out=bd.Scores(D, D, None, None, None)) == ALIAS
    call = lambda: bd.lib().bimamba_log_probs_bwd(ref(d), ref(view(A, 100)), ref(bd.Tokens(B, 10, 1)), Z, D, E, F, ref(view(7 << 40, 100)), None)  # noqa: E731
    d.struct_size, d.reserved = 40, 0
    for at, rc in ((1 << 50 | 2, ALIGN), (7 << 40, ALIAS)):
        d.lse_rest = at
        assert call() == rc, at


def test_sizes_up_to_the_limits_that_the_header_states():
    """Below a limit the next check refuses, at it the size does."""
    for rows, rc in (((1 << 24) - 1, ALIGN), (1 << 24, UNSUPPORTED)):
        assert scores(batch=1, seqlen=rows, logits=view(A + 1, 100), targets=bd.Tokens(1 << 50, 0, 1)) == rc
    for seqlen, d, rc in (((1 << 31) - 64, 512, SMALL), ((1 << 31) - 63, 512, UNSUPPORTED), ((1 << 30) - 64, 513, SMALL), ((1 << 30) - 63, 513, UNSUPPORTED),
                          ((1 << 20) - 64, 1 << 20, SMALL), ((1 << 20) - 63, 1 << 20, UNSUPPORTED)):
        assert embed_bwd(batch=1, seqlen=seqlen, d_model=d, tok=bd.Tokens(1 << 50, 0, 1), dout=bd.Tensor(B, 0, 0), ws_bytes=16) == rc, (seqlen, d)
    assert scores_bwd(batch=1, seqlen=1 << 30, vocab=8193, logits=bd.Tensor(A, 0, 0), targets=bd.Tokens(1 << 50, 0, 1), dlogits=view(1 << 52, 8193),
                      lse=1 << 51, entropy=3 << 50, dlogp=5 << 50, dentropy=6 << 50) == UNSUPPORTED


def test_views_side_by_side_in_one_buffer_do_not_meet():
    """Column slices of one buffer whose rows both step alike are apart, others are not.  (A misaligned pointer elsewhere ends the call
    on the host in either case: the order of the checks tells which was found.)"""
    def call(y):
        return norm(x=view(A, 64, st=200), y=y, mean=A)   # (mean on x: ALIAS in any case, so nothing is launched)
    assert call(view(A + 128, 64, st=200)) == ALIAS
    assert norm(x=view(A, 64, st=200), y=view(A + 126, 64, st=200)) == ALIAS        # one column too near
    assert norm(x=view(A, 64, st=200), y=view(A + 2 * 140, 64, st=200)) == ALIAS    # into the next row
    assert norm(x=view(A, 64, st=200), y=view(A + 128, 64, st=201)) == ALIAS


def grads(*entries):
    t = (bd.Grad * len(entries))(*[bd.Grad(*e) for e in entries])
    return t, len(entries)


def test_clip_refusals():
    L = bd.lib()
    good = (A, B, 10000, 0, bd.F32, 0)
    t, n = grads(good, (Z, Z, 5, 0, bd.BF16, 0))
    assert L.bimamba_clip_grads(t, n, D, 1.0, E, F, 1 << 20, None) == SHAPE        # not laid out
    assert L.bimamba_clip_layout(t, n) == OK and [g.first for g in t] == [0, 2]
    need = L.bimamba_clip_grads_workspace_bytes(t, n)
    assert need > 0
    assert L.bimamba_clip_grads(t, n, None, 1.0, E, F, 1 << 20, None) == NULL
    assert L.bimamba_clip_grads(t, n, D, 1.0, E, None, 1 << 20, None) == NULL
    assert L.bimamba_clip_grads(t, n, D, 1.0, E, F, need - 1, None) == SMALL
    assert L.bimamba_clip_grads(t, n, D + 4, 1.0, E, F, 1 << 20, None) == ALIGN
    assert L.bimamba_clip_grads(t, n, D, 1.0, E + 1, F, 1 << 20, None) == ALIGN
    for bad in (-1.0, float("nan")):
        assert L.bimamba_clip_grads(t, n, D, bad, E, F, 1 << 20, None) == SHAPE
    assert L.bimamba_clip_layout(None, 1) == NULL and L.bimamba_clip_layout(t, -1) == SHAPE
    for entry, rc in (((A, B, -1, 0, 0, 0), SHAPE), ((A, B, 5, 0, 3, 0), UNSUPPORTED), ((None, B, 5, 0, 0, 0), NULL), ((A, None, 5, 0, 0, 0), NULL),
                      ((A + 2, B, 5, 0, 0, 0), ALIGN), ((A, A + 4, 5, 0, 0, 0), ALIAS), ((A, B, 5, 0, 0, 1), SHAPE), ((A, B, 1 << 41, 0, 0, 0), UNSUPPORTED)):
        t, n = grads(good, entry)
        assert L.bimamba_clip_layout(t, n) == rc, entry
        assert L.bimamba_clip_grads_workspace_bytes(t, n) == 0
    t, n = grads((None, None, 0, 0, 0, 0))
    assert L.bimamba_clip_layout(t, n) == OK


def test_clip_refuses_tensors_that_meet():
    """What one entry writes must be apart from what every other entry reads or writes: two workgroups would race on it."""
    L = bd.lib()
    KB = 1 << 10

    def layout(*entries):
        return L.bimamba_clip_layout(*grads(*[(f, t, n, 0, k, 0) for f, t, n, k in entries]))
    f32, bf16 = bd.F32, bd.BF16
    apart = [(A + k * KB, A + k * KB, 256, f32) for k in (3, 0, 2, 1)]                      # in place, side by side, in any order
    assert layout(*apart) == OK and layout(*apart, (Z, A + 4 * KB, 100, bf16)) == OK
    assert layout((A, A, 5, f32), (A, A, 5, f32)) == ALIAS                                  # a tensor twice
    assert layout((A, A, 5, f32), (Z, Z, 5, f32), (A + 16, A + 16, 5, f32)) == ALIAS        # its last value once more
    assert layout((A, A, 5, f32), (Z, Z, 5, f32), (A + 20, A + 20, 5, f32)) == OK
    assert layout((A, B, 5, f32), (Z, B, 5, f32)) == ALIAS and layout((A, B, 5, f32), (Z, B + 18, 1, bf16)) == ALIAS   # one place for two
    assert layout((A, B, 5, f32), (B, Z, 5, f32)) == ALIAS and layout((B, Z, 5, f32), (A, B, 5, f32)) == ALIAS         # crosswise
    assert layout((A, B, 5, f32), (B, A, 5, f32)) == ALIAS and layout((A, B, 5, f32), (B + 16, D, 1 << 20, f32)) == ALIAS
    assert layout((B - KB, Z, KB, f32), *[(D, B + k * KB, 5, f32) for k in range(9)]) == ALIAS                         # the first of many
    assert layout((B + KB // 2, Z, KB, f32), *[(D, B + k * KB, 5, f32) for k in range(9)]) == ALIAS                    # in the midst of them
    assert layout((B + 20, Z, 251, f32), *[(D, B + k * KB, 5, f32) for k in range(9)]) == OK                           # between two
    assert layout((A, B, 5, f32), (A, Z, 5, f32)) == OK                                     # read twice, scaled to two places
    assert layout((A, A, 5, f32), (A, A, 0, f32), (A + 4, None, 0, f32), (None, A + 8, 0, bf16)) == OK                 # (empty ones are nowhere)
    many = [(A + k * KB, A + k * KB, 256, f32) for k in range(1000)]
    t, n = grads(*[(f, to, c, 0, k, 0) for f, to, c, k in many])
    assert L.bimamba_clip_layout(t, n) == OK and [g.first for g in t] == list(range(n))
    for at in (0, 500, 999):
        assert layout(*many[:at], (A + 700 * KB + 4, Z, 1, f32), *many[at:]) == ALIAS
        assert layout(*many[:at], (Z, A + 700 * KB + 1020, 1, f32), *many[at:]) == ALIAS


def test_clip_refuses_what_it_writes_on_its_tensors():
    L = bd.lib()
    t, n = grads((A, B, 10000, 0, bd.F32, 0), (Z, Z, 5, 0, bd.BF16, 0), (None, None, 0, 0, 0, 0))
    assert L.bimamba_clip_layout(t, n) == OK
    call = lambda dev=D, norm=E, ws=F: L.bimamba_clip_grads(t, n, dev, 1.0, norm, ws, 1 << 20, None)  # noqa: E731
    for on in (A, A + 39996, B, B + 39996, Z + 8):
        assert call(norm=on) == ALIAS, on
    for on in (A, B + 39984, Z, B - 16):
        assert call(ws=on) == ALIAS, on
    for on in (B, B + 39992, Z):
        assert call(dev=on) == ALIAS, on
    assert call(norm=F) == ALIAS and call(norm=D + 100) == ALIAS and call(ws=D) == ALIAS and call(ws=D - 16) == ALIAS


def test_the_binding_checks_tensors_against_the_descriptor():
    """Host tensors, other shapes and types, descriptors of another call and what is no tensor never reach the library."""
    x = torch.zeros(2, 10, 64, dtype=torch.bfloat16)
    d, e = bd.make_norm_desc(2, 10, 64), bd.make_embed_desc(2, 10, 64, 100)
    with pytest.raises(AssertionError, match=r"x: BFloat16 \(2, 10, 64\) with strides \(640, 64, 1\) on cpu, wanted BFloat16 \(2, 10, 64\) on the GPU"):
        bd.bimamba_layer_norm(d, x, None, None, x.clone())
    with pytest.raises(AssertionError, match="x: Float"):
        bd.bimamba_layer_norm(d, x.float(), None, None, x.clone())
    with pytest.raises(AssertionError, match=r"tokens: Int .*wanted Long \(2, 10\)"):
        bd.bimamba_embed(e, torch.zeros(2, 10, dtype=torch.int32), torch.zeros(100, 64), x)
    with pytest.raises(AssertionError, match="a descriptor of another call"):
        bd.bimamba_embed(d, torch.zeros(2, 10, dtype=torch.int64), torch.zeros(100, 64), x)
    with pytest.raises(AssertionError, match="x: not a tensor"):
        bd.bimamba_layer_norm(d, [1.0], None, None, x)
    with pytest.raises(AssertionError, match="logits: BFloat16"):
        bd.bimamba_log_probs(bd.make_logits_desc(2, 10, 65), x, None, {})
    with pytest.raises(AssertionError, match="logits: BFloat16"):
        bd.bimamba_log_probs_bwd(bd.make_logits_desc(2, 10, 65), x, None, None, None, None, None, x)
    with pytest.raises(AssertionError):
        bd.bimamba_embed_bwd(e, torch.zeros(2, 10, dtype=torch.int64), x, torch.zeros(100, 64), None)
    with pytest.raises(AssertionError):
        bd.bimamba_layer_norm_bwd(d, x, None, None, None, x, x.clone(), None, None, None)
    with pytest.raises(AssertionError):
        bd.GradTable([torch.zeros(4)])
    with pytest.raises(AttributeError):
        bd.bimamba_clip_grads(None, 1.0, None, None)
    with pytest.raises(KeyError):
        bd.make_logits_desc(1, 1, 10, io="f16")


def test_workspaces_stay_small():
    """A few bytes a row and slots for as many workgroups as the chip holds, whatever the call."""
    assert bd.bimamba_embed_bwd_workspace_bytes(bd.make_embed_desc(8, 8192, 2048, 50304)) < 64 << 20
    assert bd.bimamba_layer_norm_bwd_workspace_bytes(bd.make_norm_desc(8, 8192, 2048), True) < 64 << 20
    assert bd.bimamba_layer_norm_bwd_workspace_bytes(bd.make_norm_desc(65535, 1, 2048), False) < 64 << 20
    assert bd.bimamba_log_probs_workspace_bytes(bd.make_logits_desc(8, 8192, 50304, top_k=8)) == 0


def test_workspaces_stay_small_with_vectors_of_their_own():
    """Slots for as many workgroups as the chip holds, however many batch elements have vectors of their own."""
    need = lambda b, L, d: bd.bimamba_layer_norm_bwd_workspace_bytes(bd.make_norm_desc(b, L, d), True)  # noqa: E731
    assert need(65535, 1, 2048) == 0 and need(65535, 3, 64) == 0 and need(2000, 40, 1000) == 0
    assert need(1000, 100, 2048) < 64 << 20 and need(300, 7, 2048) < 64 << 20
    # what goes without one is still refused where the results are wrong
    one = dict(batch=2000, seqlen=1, x=view(A, 64, L=1), dy=view(E, 64, L=1), dx=view(F, 64, L=1), stride=64, ws=None)
    assert norm_bwd(**dict(one, dw=8 << 40)) == ALIAS and norm_bwd(**dict(one, db=E)) == ALIAS and norm_bwd(**dict(one, dw=B + 64)) == ALIAS
