"""nmt_verify_drafts (csrc/verify.hip) against the 64-bit verification of
draft_cases: kept drafts and next words equal, log p within fp32's rounding."""
import numpy as np
import pytest

import draft_cases as dc
from paper_1605_04809_amd.workloads import param_shapes

pytestmark = pytest.mark.gpu

NAN = float("nan")


def _torch():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _model(nb, V):
    return nb.Model({n: np.zeros(s, np.float32) for n, s in param_shapes(4, V, 4, 4, 4).items()}, 4, V, 4, 4, 4)


def _dev(torch, a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _wide(torch, a, dtype, pad, shift=0):
    flat = torch.full((a.shape[0] * (a.shape[1] + pad) + shift,), NAN, dtype=dtype, device="cuda")
    w = flat[shift:].view(a.shape[0], a.shape[1] + pad)
    w[:, :a.shape[1]] = _dev(torch, a, dtype)
    return w[:, :a.shape[1]]


def _run(torch, nb, model, off, draft, target, proposal, u, tt="float32", pt="float32", pad=0, shift=0, **kw):
    S, n = len(off) - 1, len(draft)
    out = (torch.full((S,), -7, dtype=torch.int32, device="cuda"), torch.full((S,), -7, dtype=torch.int32, device="cuda"),
           torch.full((n,), 7.0, device="cuda"), torch.full((S,), 7.0, device="cuda"))
    nb.nmt_verify_drafts(model, _dev(torch, np.asarray(off, np.int32)), _dev(torch, np.asarray(draft, np.int32)),
                         _wide(torch, target, getattr(torch, tt), pad, shift),
                         None if proposal is None else _wide(torch, proposal, getattr(torch, pt), pad, shift),
                         _dev(torch, np.asarray(u, np.float32)), *out[:2], draft_logp=out[2], next_logp=out[3], **kw)
    torch.cuda.synchronize()
    return [o.cpu().numpy() for o in out]


def _same(got, want, target):
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])
    for g, w in zip(got[2:], want[2:]):
        # a log p below fp32's lowest value, -3.4028e38, is -infinity in fp32 (two logits of 3e38 and -3e38: -6e38)
        w = np.where(w < -3.4028236e38, -np.inf, w)
        # the value is rounded once; what it is made of is in 64 bits
        fin = np.isfinite(w)
        np.testing.assert_array_equal(g[~fin], w[~fin])
        assert np.all(np.abs(g[fin] - w[fin]) <= 2.0 ** -24 * np.abs(w[fin]) + 1e-12)


def _inputs(rng, V, S, k, bf16_t=False, bf16_p=False, certain=False, mask=0.0, spread=2.5, near=0.7):
    n = rng.integers(0, k + 1, size=S)
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    nd = int(off[-1])
    target = (spread * rng.standard_normal((nd + S, V))).astype(np.float32)
    seq = np.repeat(np.arange(S), n)
    prop = None
    if certain:
        draft = np.where(rng.random(nd) < 0.5, target[np.arange(nd) + seq].argmax(1) if nd else 0,
                         rng.integers(0, V, size=nd)).astype(np.int32)
    else:
        prop = (target[np.arange(nd) + seq] + near * rng.standard_normal((nd, V))).astype(np.float32)
        if mask:   # words that the proposer never draws
            prop[rng.random(prop.shape) < mask] = -np.inf
            prop[:, 0] = 0.0
        if bf16_p:
            prop = dc.round_bf16(prop)
        draft = np.array([rng.choice(V, p=np.exp(dc.log_softmax(r))) for r in prop], np.int32).reshape(nd)
    if mask:       # words that the target forbids, all but one in some rows
        target[rng.random(target.shape) < mask] = -np.inf
        target[:: 5] = -np.inf
        target[:, rng.integers(0, V)] = 1.0
    if bf16_t:
        target = dc.round_bf16(target)
    return off, draft, target, prop, rng.random(nd + S, dtype=np.float32)


@pytest.mark.parametrize("V,S,k", [(1, 3, 2), (2, 40, 3), (3, 1, 1), (63, 9, 4), (64, 9, 4), (255, 5, 3), (257, 5, 3),
                                   (1000, 1, 4), (1000, 200, 2), (4097, 6, 5), (20011, 7, 8), (100000, 3, 4),
                                   (50000, 1, 0), (777, 300, 0), (333, 2, 40)])
@pytest.mark.parametrize("certain", [False, True])
def test_sizes(V, S, k, certain):
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    model = _model(nb, V)
    rng = np.random.default_rng(V + S + k)
    ins = _inputs(rng, V, S, k, certain=certain)
    got = _run(torch, nb, model, *ins)
    want = dc.verify(*ins)
    _same(got, want, ins[2])
    assert nb.nmt_stream_status(model) == nb.NMT_OK
    print(f"V={V} S={S} k={k}: {int(want[0].sum())} of {len(ins[1])} drafts kept", flush=True)
    model.close()


@pytest.mark.parametrize("tt,pt", [("float32", "bfloat16"), ("bfloat16", "float32"), ("bfloat16", "bfloat16")])
@pytest.mark.parametrize("pad,shift,V", [(0, 0, 3000), (8, 0, 3000), (5, 3, 3000), (1, 1, 3001), (0, 1, 97)])
def test_types_strides_and_alignment(tt, pt, pad, shift, V):
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    model = _model(nb, V)
    ins = _inputs(np.random.default_rng(pad + V), V, 12, 4, tt == "bfloat16", pt == "bfloat16")
    got = _run(torch, nb, model, *ins, tt=tt, pt=pt, pad=pad, shift=shift)
    _same(got, dc.verify(*ins), ins[2])
    model.close()


@pytest.mark.parametrize("V", [50, 5000])
@pytest.mark.parametrize("mask", [0.3, 0.97])
def test_masked_words(V, mask):
    """Logits of -infinity on either side: never drawn, never kept; rows with
    one word left; drafts that the proposer could not have drawn."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    model = _model(nb, V)
    rng = np.random.default_rng(V)
    off, draft, target, prop, u = _inputs(rng, V, 30, 4, mask=mask)
    low = target.copy()
    low[np.isneginf(low)] = np.finfo(np.float32).min     # the type's lowest value instead
    other = draft.copy()
    other[::3] = rng.integers(0, V, size=len(other[::3]))
    for d, t in ((draft, target), (other, target), (draft, low)):
        ins = (off, d, t, prop, u)
        got = _run(torch, nb, model, *ins)
        _same(got, dc.verify(*ins), t)
    assert nb.nmt_stream_status(model) == nb.NMT_OK
    model.close()


@pytest.mark.parametrize("spread", [0.0, 1e-3, 30.0, 3e4, 1e38])
def test_flat_and_steep_rows(spread):
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    V = 1500
    model = _model(nb, V)
    rng = np.random.default_rng(3)
    off, draft, target, prop, u = _inputs(rng, V, 20, 3, spread=1.0)
    target, prop = np.float32(spread) * np.clip(target, -3, 3), np.float32(spread) * np.clip(prop, -3, 3)
    ins = (off, draft, target.astype(np.float32), prop.astype(np.float32), u)
    _same(_run(torch, nb, model, *ins), dc.verify(*ins), ins[2])
    model.close()


def test_random_numbers_at_their_ends_and_ties():
    """u = 0 keeps every draft of positive probability and draws the first word
    that has one; the largest u draws the last; u q = p exactly is no keep."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    V = 4
    model = _model(nb, V)
    top = np.float32(1.0 - 2.0 ** -24)
    z = np.zeros((2, V), np.float32)
    z[:, 0] = -np.inf                       # words 1, 2, 3: a third each
    half = np.full((2, V), -np.inf, np.float32)
    half[:, 1:3] = 0.0                      # words 1, 2: a half each
    for target, prop, d, u, want in [
            (z, None, 0, (0.0, 0.0), (0, 1)), (z, None, 2, (0.0, 0.0), (1, 1)), (z, None, 2, (0.0, top), (1, 3)),
            (z, None, 3, (top, top), (0, 2)), (z, None, 1, (top, 0.0), (0, 2)),
            (half, None, 1, (0.5, 0.0), (0, 2)),            # 0.5 < 0.5 does not hold
            (half, None, 1, (np.float32(0.5) - np.float32(2.0 ** -25), 0.5), (1, 2)),
            (half, half[:1], 1, (top, 0.25), (1, 1)),       # the same distribution: kept whatever the number
            (half, half[:1], 3, (0.0, 0.75), (0, 2)),       # a draft that neither gives: p itself
    ]:
        ins = ([0, 1], [d], target, prop, np.array(u, np.float32))
        got = _run(torch, nb, model, *ins)
        assert (got[0][0], got[1][0]) == want, (d, u)
        _same(got, dc.verify(*ins), target)
    model.close()


def test_bad_rows_and_ids_are_flagged_and_stay_alone():
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    V, S = 600, 9
    model = _model(nb, V)
    rng = np.random.default_rng(4)
    off = (3 * np.arange(S + 1)).astype(np.int32)
    nd = int(off[-1])
    target = rng.standard_normal((nd + S, V)).astype(np.float32)
    prop = rng.standard_normal((nd, V)).astype(np.float32)
    draft = rng.integers(0, V, size=nd).astype(np.int32)
    u = np.zeros(nd + S, np.float32)        # everything is kept ...
    u[off[1:] + np.arange(S)] = 0.5
    clean = dc.verify(off, draft, target, prop, u)
    bad = target.copy()
    bad[off[1] + 1 + 1, 7] = np.nan         # sequence 1, position 1
    bad[off[2] + 2 + 2, V - 1] = np.inf     # sequence 2, position 2
    bad[off[3] + 3 + 3] = -np.inf           # sequence 3, the row behind its drafts
    d2 = draft.copy()
    d2[off[4]] = V                          # sequence 4, position 0
    d2[off[5] + 2] = -1                     # sequence 5, position 2
    p2 = prop.copy()
    p2[off[6] + 1] = np.nan                 # sequence 6, position 1
    u2 = u.copy()
    u2[off[7] + 7] = np.float32(1.0 - 2.0 ** -24)   # sequence 7 loses draft 0 (p is far below q's share)
    prop2 = p2
    prop2[off[7], draft[off[7]]] = 20.0
    bad[off[7] + 7 + 1, 0] = np.nan         # and never reaches this row
    got = _run(torch, nb, model, off, d2, bad, prop2, u2)
    assert nb.nmt_stream_status(model) == nb.NMT_ERANGE
    assert nb.nmt_stream_status(model) == nb.NMT_OK
    for s, kept in ((1, 1), (2, 2), (3, 3), (4, 0), (5, 2), (6, 1)):
        assert (got[0][s], got[1][s]) == (kept, -1), s
        assert np.isnan(got[3][s])
    fixed = np.where(np.isfinite(bad), bad, 0.0).astype(np.float32)
    ref = dc.verify(off, np.clip(d2, 0, V - 1), fixed, np.nan_to_num(prop2), u2)
    assert (got[0][7], got[1][7]) == (ref[0][7], ref[1][7]) and got[0][7] == 0 and got[1][7] >= 0
    for s in (0, 8):
        assert (got[0][s], got[1][s]) == (clean[0][s], clean[1][s])
    assert np.isnan(got[2][off[4]]) and np.isnan(got[2][off[1] + 1]) and np.isfinite(got[2][off[1]])
    for off_bad in ([0, 2, 1, 3], [0, -1, 2, 3], [0, 1, 2, 9], [-2, 1, 2, 3]):
        t3, p3 = target[:6], prop[:3]
        out = _run(torch, nb, model, off_bad, draft[:3], t3, p3, u[:6])
        assert nb.nmt_stream_status(model) == nb.NMT_ERANGE
        for s in range(3):
            if not 0 <= off_bad[s] <= off_bad[s + 1] <= 3:
                assert (out[0][s], out[1][s]) == (0, -1)
    model.close()


def test_refusals():
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    lib = nb.load_library()
    V, S, n = 100, 2, 3
    model = _model(nb, V)
    i32 = dict(dtype=torch.int32, device="cuda")
    off, draft = torch.tensor([0, 1, 3], **i32), torch.zeros(n, **i32)
    z, q, u = torch.zeros((n + S, V), device="cuda"), torch.zeros((n, V), device="cuda"), torch.zeros(n + S, device="cuda")
    acc, nxt = torch.full((S,), -7, **i32), torch.full((S,), -7, **i32)
    need = nb.nmt_verify_workspace_bytes(model, S, n)
    ws = torch.zeros(need + 256, dtype=torch.uint8, device="cuda")
    ok = [model.handle, S, n, off.data_ptr(), draft.data_ptr(), z.data_ptr(), 0, V, q.data_ptr(), 0, V, u.data_ptr(),
          acc.data_ptr(), nxt.data_ptr(), None, None, ws.data_ptr(), need, None]
    for at, value, rc in [(1, -1, -1), (2, -1, -1), (3, None, -1), (4, None, -1), (5, None, -1), (6, 2, -1), (7, V - 1, -1),
                          (9, 7, -1), (10, V - 1, -1), (11, None, -1), (12, None, -1), (13, None, -1), (16, None, -1),
                          (16, ws.data_ptr() + 16, -1), (17, need - 1, -5), (5, z.data_ptr() + 2, -1),
                          (8, q.data_ptr() + 1, -1)]:
        args = list(ok)
        args[at] = value
        assert lib.nmt_verify_drafts(*args) == rc, (at, value)
        assert nb.last_error()
    args = list(ok)
    args[1] = 0
    assert lib.nmt_verify_drafts(*args) == nb.NMT_OK
    torch.cuda.synchronize()
    assert bool((acc == -7).all()) and bool((nxt == -7).all())
    assert nb.nmt_verify_workspace_bytes(model, 0, 3) == 0 and nb.nmt_verify_workspace_bytes(model, 3, -1) == 0
    # a workspace for more serves fewer
    sizes = [nb.nmt_verify_workspace_bytes(model, s, d) for s, d in ((1, 0), (2, 3), (2, 4), (3, 4), (64, 100), (65, 100))]
    assert sizes == sorted(sizes)
    with pytest.raises(ValueError):
        nb.nmt_verify_drafts(model, off, draft, z[:4], q, u, acc, nxt)
    with pytest.raises(ValueError):
        nb.nmt_verify_drafts(model, off.long(), draft, z, q, u, acc, nxt)
    model.close()


@pytest.mark.parametrize("V,S,k", [(1000, 2, 3), (30000, 20, 3)])
def test_streams_graphs_and_a_used_workspace(V, S, k):
    """Twice on one workspace full of other values, on another stream, and
    captured: always the eager values; optional outputs left out."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    model = _model(nb, V)
    off, draft, target, prop, u = _inputs(np.random.default_rng(6), V, S, k)
    want = dc.verify(off, draft, target, prop, u)
    n = len(draft)
    d = [_dev(torch, a) for a in (off, draft, target, prop, u)]
    i32 = dict(dtype=torch.int32, device="cuda")
    acc, nxt = torch.zeros(S, **i32), torch.zeros(S, **i32)
    ws = torch.full((nb.nmt_verify_workspace_bytes(model, S, n),), 255, dtype=torch.uint8, device="cuda")
    call = lambda: nb.nmt_verify_drafts(model, *d, acc, nxt, workspace=ws)

    def check():
        torch.cuda.synchronize()
        np.testing.assert_array_equal(acc.cpu().numpy(), want[0])
        np.testing.assert_array_equal(nxt.cpu().numpy(), want[1])
        acc.fill_(-7)
        nxt.fill_(-7)
        torch.cuda.synchronize()
    call()
    check()
    call()
    check()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call()
    check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(4):
        g.replay()
        check()
        ws.fill_(255)
        call()
        check()
    assert nb.nmt_stream_status(model) == nb.NMT_OK
    model.close()


# ---- vocabularies of more than 8,192 words: two launches, a row in parts, a
# residual in units of 512 words

@pytest.mark.parametrize("V", [8191, 8192, 8193, 8199, 8200, 10240, 16385, 131072, 131073, 300001])
@pytest.mark.parametrize("tt,pt", [("float32", "float32"), ("bfloat16", "bfloat16")])
def test_borders_of_parts_and_units(V, tt, pt):
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    model = _model(nb, V)
    off, draft, target, prop, u = _inputs(np.random.default_rng(V), V, 5, 3, tt == "bfloat16", pt == "bfloat16")
    # the row's last words carry some of the sums, and the largest u draws one of them
    target[:, -9:] += 4.0
    target = dc.round_bf16(target) if tt == "bfloat16" else target
    u[off[1:] + np.arange(5)] = np.float32([0.0, 0.25, 0.999, 1.0 - 2.0 ** -24, 0.5])
    ins = (off, draft, target, prop, u)
    _same(_run(torch, nb, model, *ins, tt=tt, pt=pt), dc.verify(*ins), target)
    assert nb.nmt_stream_status(model) == nb.NMT_OK
    model.close()


@pytest.mark.parametrize("S,k,certain", [(2, 40, False), (2, 40, True), (1500, 1, False), (1100, 0, True)])
def test_long_drafts_and_many_sequences(S, k, certain):
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    V = 8300
    model = _model(nb, V)
    ins = _inputs(np.random.default_rng(S + k), V, S, k, certain=certain, spread=4.0, near=0.3)
    want = dc.verify(*ins)
    _same(_run(torch, nb, model, *ins), want, ins[2])
    d = [_dev(torch, a) if a is not None else None for a in ins]
    acc, nxt = (torch.zeros(S, dtype=torch.int32, device="cuda") for _ in range(2))
    nb.nmt_verify_drafts(model, *d, acc, nxt)     # without log p: no position behind the end is looked at
    np.testing.assert_array_equal(acc.cpu().numpy(), want[0])
    np.testing.assert_array_equal(nxt.cpu().numpy(), want[1])
    model.close()


@pytest.mark.parametrize("tt,pt", [("float32", "bfloat16"), ("bfloat16", "float32")])
@pytest.mark.parametrize("pad,shift,V", [(8, 0, 9000), (5, 3, 9000), (1, 1, 9001), (0, 7, 12289)])
def test_types_strides_and_alignment_of_long_rows(tt, pt, pad, shift, V):
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    model = _model(nb, V)
    ins = _inputs(np.random.default_rng(pad + V), V, 6, 4, tt == "bfloat16", pt == "bfloat16")
    got = _run(torch, nb, model, *ins, tt=tt, pt=pt, pad=pad, shift=shift)
    _same(got, dc.verify(*ins), ins[2])
    model.close()


@pytest.mark.parametrize("mask", [0.3, 0.9995])
def test_masked_words_of_long_rows(mask):
    """Whole parts and units of nothing but -infinity; the type's lowest value."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    V = 20000
    model = _model(nb, V)
    rng = np.random.default_rng(V)
    off, draft, target, prop, u = _inputs(rng, V, 12, 4, mask=mask)
    low = target.copy()
    low[np.isneginf(low)] = np.finfo(np.float32).min
    other = draft.copy()
    other[::3] = rng.integers(0, V, size=len(other[::3]))
    for d, t in ((draft, target), (other, target), (draft, low)):
        ins = (off, d, t, prop, u)
        _same(_run(torch, nb, model, *ins), dc.verify(*ins), t)
    assert nb.nmt_stream_status(model) == nb.NMT_OK
    model.close()


@pytest.mark.parametrize("V", [1500, 20000])
@pytest.mark.parametrize("spread,shift", [(0.0, 0.0), (0.0, 5e4), (1.0, 199.0), (1.0, 201.0), (1.0, -199.0), (1.0, -201.0),
                                          (1.0, -690.0), (300.0, 0.0), (3e4, 0.0), (1e38, 0.0)])
def test_rows_of_any_size(V, spread, shift):
    """Logits far from 0, whose largest is taken off before the exponential,
    beside parts of ordinary ones."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    model = _model(nb, V)
    rng = np.random.default_rng(3)
    off, draft, target, prop, u = _inputs(rng, V, 8, 3, spread=1.0)
    target = (np.float32(spread) * np.clip(target, -3, 3) + np.float32(shift)).astype(np.float32)
    prop = (np.float32(spread) * np.clip(prop, -3, 3) + np.float32(shift)).astype(np.float32)
    target[::2, : V // 2] = np.clip(target[::2, : V // 2], -50, 50)
    ins = (off, draft, target, prop, u)
    _same(_run(torch, nb, model, *ins), dc.verify(*ins), target)
    assert nb.nmt_stream_status(model) == nb.NMT_OK
    model.close()


@pytest.mark.parametrize("V", [900, 9000, 140000])
def test_nothing_left_of_a_long_row(V):
    """Target and proposal alike, and a draft that neither gives: p itself; a
    target of one word, certain drafts: p without the draft is nothing."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    model = _model(nb, V)
    rng = np.random.default_rng(7)
    z = rng.standard_normal((2, V)).astype(np.float32)
    z[0, [3, V - 1]] = -np.inf
    for d, u in ((3, 0.3), (V - 1, 0.0), (V - 1, 1.0 - 2.0 ** -24), (3, 0.999)):
        ins = ([0, 1], [d], z, z[:1], np.array([0.0, u], np.float32))
        got = _run(torch, nb, model, *ins)
        assert got[0][0] == 0 and got[1][0] not in (-1, 3, V - 1)
        _same(got, dc.verify(*ins), z)
    one = np.full((2, V), -np.inf, np.float32)
    one[:, V - 2] = 3.0
    for d, u0 in ((V - 2, 0.5), (5, 0.5)):
        ins = ([0, 1], [d], one, None, np.array([u0, 0.7], np.float32))
        got = _run(torch, nb, model, *ins)
        assert (got[0][0], got[1][0]) == ((1, V - 2) if d == V - 2 else (0, V - 2))
        _same(got, dc.verify(*ins), one)
    assert nb.nmt_stream_status(model) == nb.NMT_OK
    model.close()


def test_bad_long_rows_are_flagged_and_stay_alone():
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    V, S = 9001, 6
    model = _model(nb, V)
    rng = np.random.default_rng(4)
    off = (2 * np.arange(S + 1)).astype(np.int32)
    nd = int(off[-1])
    target = rng.standard_normal((nd + S, V)).astype(np.float32)
    prop = rng.standard_normal((nd, V)).astype(np.float32)
    draft = rng.integers(0, V, size=nd).astype(np.int32)
    u = np.zeros(nd + S, np.float32)
    u[off[1:] + np.arange(S)] = 0.5
    clean = dc.verify(off, draft, target, prop, u)
    bad, d2, p2 = target.copy(), draft.copy(), prop.copy()
    bad[off[1] + 1 + 1, V - 1] = np.nan     # sequence 1, position 1
    bad[off[2] + 2 + 2] = -np.inf           # sequence 2, the row behind its drafts
    d2[off[3]] = V                          # sequence 3, position 0
    p2[off[4] + 1, 8500] = np.inf           # sequence 4, position 1
    got = _run(torch, nb, model, off, d2, bad, p2, u)
    assert nb.nmt_stream_status(model) == nb.NMT_ERANGE
    for s, kept in ((1, 1), (2, 2), (3, 0), (4, 1)):
        assert (got[0][s], got[1][s]) == (kept, -1) and np.isnan(got[3][s]), s
    for s in (0, 5):
        assert (got[0][s], got[1][s]) == (clean[0][s], clean[1][s])
    for off_bad in ([0, 2, 1, 3], [0, -1, 2, 3], [0, 1, 2, 9], [-2, 1, 2, 3]):
        out = _run(torch, nb, model, off_bad, draft[:3], target[:6], prop[:3], u[:6])
        assert nb.nmt_stream_status(model) == nb.NMT_ERANGE
        for s in range(3):
            if not 0 <= off_bad[s] <= off_bad[s + 1] <= 3:
                assert (out[0][s], out[1][s]) == (0, -1)
    model.close()


def test_two_calls_at_once():
    """On two streams, a workspace each, many times over."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    V, S = 20000, 30
    model = _model(nb, V)
    jobs = []
    for seed in (1, 2):
        ins = _inputs(np.random.default_rng(seed), V, S, 3)
        acc, nxt = (torch.zeros(S, dtype=torch.int32, device="cuda") for _ in range(2))
        jobs.append((dc.verify(*ins), [_dev(torch, a) for a in ins], acc, nxt, torch.cuda.Stream(),
                     torch.empty(nb.nmt_verify_workspace_bytes(model, S, len(ins[1])), dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(20):
        for _, d, acc, nxt, stream, ws in jobs:
            with torch.cuda.stream(stream):
                nb.nmt_verify_drafts(model, *d, acc, nxt, workspace=ws)
    torch.cuda.synchronize()
    for want, _, acc, nxt, _, _ in jobs:
        np.testing.assert_array_equal(acc.cpu().numpy(), want[0])
        np.testing.assert_array_equal(nxt.cpu().numpy(), want[1])
    model.close()


@pytest.mark.parametrize("V,S,n", [(4, 1 << 22, 0), (100, 1 << 22, 0), (9000, 1 << 22, 0), (100, 1, 1 << 23), (9000, 1, 1 << 23),
                                   (9000, 1, 2 ** 31 - 1), (300001, 1, 300000)])
def test_more_rows_than_a_launch_takes(V, S, n):
    """Refused before anything is read (a workspace of no bytes would be, too, with another status)."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    lib = nb.load_library()
    model = _model(nb, V)
    a = torch.zeros(64, device="cuda").data_ptr()
    assert lib.nmt_verify_drafts(model.handle, S, n, a, a, a, 0, V, a, 0, V, a, a, a, None, None, a, 0, None) == nb.NMT_EINVAL
    assert "too many" in nb.last_error()
    model.close()


@pytest.mark.parametrize("V", [1, 2, 5, 7, 8, 9, 15])
@pytest.mark.parametrize("tt,pt", [("bfloat16", "bfloat16"), ("float32", "bfloat16"), ("bfloat16", "float32")])
@pytest.mark.parametrize("S,pad,shift", [(6, 0, 0), (6, 3, 1), (300, 1, 1)])
def test_rows_of_few_words(V, tt, pt, S, pad, shift):
    """Rows shorter than the eight words that a lane reads at once, and of one or two such."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    model = _model(nb, V)
    ins = _inputs(np.random.default_rng(V + S), V, S, 3, tt == "bfloat16", pt == "bfloat16", near=1.5)
    _same(_run(torch, nb, model, *ins, tt=tt, pt=pt, pad=pad, shift=shift), dc.verify(*ins), ins[2])
    assert nb.nmt_stream_status(model) == nb.NMT_OK
    model.close()


@pytest.mark.parametrize("V,S", [(9000, 40), (140001, 12), (300001, 3)])
def test_nothing_left_of_many_rows(V, S):
    """Every sequence's residual is nothing, so that the sums of one pass are
    replaced by another's while waves of the block may still read them: p
    itself, call after call on one workspace."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    model = _model(nb, V)
    rng = np.random.default_rng(V)
    off = np.arange(S + 1).astype(np.int32)
    draft = rng.integers(0, V, size=S).astype(np.int32)
    target = rng.standard_normal((2 * S, V)).astype(np.float32)
    target[2 * np.arange(S), draft] = -np.inf
    prop = target[0::2].copy()
    u = rng.random(2 * S, dtype=np.float32)
    want = dc.verify(off, draft, target, prop, u)
    assert not want[0].any()
    d = [_dev(torch, a) for a in (off, draft, target, prop, u)]
    acc, nxt = (torch.zeros(S, dtype=torch.int32, device="cuda") for _ in range(2))
    ws = torch.empty(nb.nmt_verify_workspace_bytes(model, S, S), dtype=torch.uint8, device="cuda")
    for i in range(30):
        acc.fill_(-7)
        nxt.fill_(-7)
        nb.nmt_verify_drafts(model, *d, acc, nxt, workspace=ws)
        np.testing.assert_array_equal(acc.cpu().numpy(), want[0], err_msg=f"call {i}")
        np.testing.assert_array_equal(nxt.cpu().numpy(), want[1], err_msg=f"call {i}")
    assert nb.nmt_stream_status(model) == nb.NMT_OK
    model.close()
