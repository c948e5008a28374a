"""Drafted words: what the entry points refuse before they touch a device, and
the 64-bit verification that the GPU tests compare with against what it is
meant to do: the words that a round emits are distributed as the target's."""
import ctypes
from types import SimpleNamespace

import numpy as np
import pytest

import draft_cases as dc
from paper_1605_04809_amd import binding as nb


def _create(K=40, N=7, group=32, stype=0, codes=True, scales=None, zeros=None, out=True):
    lib = nb.load_library()
    G = -(-K // group) if group > 0 and K > 0 else 1
    c = np.zeros((max(K, 1), (max(N, 1) + 1) // 2), np.uint8)
    s = np.ones((G, max(N, 1)), np.float32) if scales is None else scales
    h = ctypes.c_void_p()
    d = nb.W4Dims(K, N, group, stype)
    rc = lib.nmt_w4_create(ctypes.byref(d), c.ctypes.data if codes else None, s.ctypes.data,
                           None if zeros is None else zeros.ctypes.data, None, ctypes.byref(h) if out else None)
    assert not h.value
    return rc


@pytest.mark.parametrize("kw,says", [
    (dict(K=0), "positive"), (dict(N=0), "positive"), (dict(K=-3), "positive"), (dict(group=0), "group"),
    (dict(group=48), "group"), (dict(group=-32), "group"), (dict(stype=2), "type"), (dict(codes=False), "NULL"),
    (dict(out=False), "NULL")])
def test_w4_create_refuses(kw, says):
    assert _create(**kw) == nb.NMT_EINVAL
    assert says in nb.last_error()


@pytest.mark.parametrize("value,stype", [(np.inf, 0), (-np.inf, 0), (np.nan, 0), (3.4e38, 1), (-3.4e38, 1)])
def test_w4_create_refuses_scales_that_are_not_finite(value, stype):
    s = np.ones((2, 7), np.float32)
    s[1, 6] = value
    assert _create(scales=s, stype=stype) == nb.NMT_EINVAL
    assert "scale" in nb.last_error()


def test_w4_create_refuses_zero_points_above_15():
    z = np.full((2, 7), 15, np.uint8)
    z[1, 6] = 16
    assert _create(zeros=z) == nb.NMT_ERANGE


def test_null_handles():
    lib = nb.load_library()
    out = ctypes.c_void_p()
    assert lib.nmt_w4_product(None, 1, None, 0, 1, None, 0, 1, None) == nb.NMT_EINVAL
    assert lib.nmt_w4_from_output(None, 32, 0, None, ctypes.byref(out)) == nb.NMT_EINVAL
    assert lib.nmt_w4_info(None, None, None, None) == nb.NMT_EINVAL
    assert lib.nmt_step_readouts(None, None, 1, None, 1, *([None] * 6), 0, None) == nb.NMT_EINVAL
    assert lib.nmt_logits(None, 1, None, None, 1, None, None, 0, None) == nb.NMT_EINVAL
    assert lib.nmt_verify_drafts(None, 1, 0, None, None, None, 0, 1, None, 0, 0, *([None] * 6), 0, None) == nb.NMT_EINVAL
    assert lib.nmt_verify_workspace_bytes(None, 1, 1) == 0
    lib.nmt_w4_destroy(None)


def test_binding_checks_shapes_and_types():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="device"):
        nb._rows(torch.zeros(2, 3), 3, 2)
    with pytest.raises(ValueError, match="codes"):
        nb.W4(np.zeros((4, 3), np.uint8), np.ones((1, 4), np.float32), 4, 4, 32)
    with pytest.raises(ValueError, match="scales"):
        nb.W4(np.zeros((4, 2), np.uint8), np.ones((2, 4), np.float32), 4, 4, 32)
    with pytest.raises(ValueError, match="type"):
        nb.W4(np.zeros((4, 2), np.uint8), np.ones((1, 4), np.float32), 4, 4, 32, stype="f16")


@pytest.mark.parametrize("certain", [False, True])
def test_what_a_round_emits_is_distributed_as_the_target(certain):
    """Over a fine grid of random numbers the first word that comes out (the
    draft where it is kept, the word after it where not) has the target's
    probabilities: each axis of the grid is off by at most half its spacing at
    every border, and there are at most V borders."""
    rng = np.random.default_rng(5)
    V, n = 5, 400
    z, zq = 1.5 * rng.standard_normal((2, V)), 1.5 * rng.standard_normal((1, V))
    p, q = np.exp(dc.log_softmax(z[0])), np.exp(dc.log_softmax(zq[0]))
    u = (np.arange(n) + 0.5) / n
    got = np.zeros(V)
    for d in range(V):
        weight = (1.0 / V) if certain else q[d]   # certain drafts: any word, here each as often
        kept = u * (1.0 if certain else q[d]) < p[d]
        first = np.zeros(V)
        first[d] += kept.mean()
        for k in np.nonzero(~kept)[0][:1]:        # what follows a rejection does not depend on its random number
            for w in u:
                a, nxt, _, _ = dc.verify(np.array([0, 1]), np.array([d]), z, None if certain else zq,
                                         np.array([u[k], w]))
                assert a[0] == 0
                first[nxt[0]] += (~kept).mean() / n
        got += weight * first
    assert np.abs(got - p).max() <= 2.0 * V / n


@pytest.mark.parametrize("value", [2.0 ** 116 * (1 + 2.0 ** -23), -1e35, 3e38])
@pytest.mark.parametrize("stype", [0, 1])
def test_w4_create_refuses_scales_that_products_do_not_take(value, stype):
    s = np.ones((2, 7), np.float32)
    s[0, 3] = value
    assert _create(scales=s, stype=stype) == nb.NMT_EINVAL
    assert "scale" in nb.last_error()


@pytest.mark.parametrize("shape,dtype", [((4, 63), "float32"), ((4, 64), "float64"), ((4, 64), "bfloat16"),
                                         ((256,), "float32")])
def test_readouts_refuse_a_pool_of_other_states(shape, dtype):
    """Before anything else: such a pool's rows would be read beyond its end."""
    torch = pytest.importorskip("torch")
    pool, y = torch.zeros(shape, dtype=getattr(torch, dtype)), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="state_pool"):
        nb.nmt_step_readouts(SimpleNamespace(H=64, E=32), None, pool, y, y, None, None)


@pytest.mark.parametrize("what,value", [("codes", 256 + 3), ("codes", -1), ("codes", 2.5), ("zeros", 256 + 8),
                                        ("zeros", 7.5)])
def test_codes_and_zero_points_that_are_no_bytes(what, value):
    """Refused, not taken modulo 256 or cut off."""
    a = {"codes": np.zeros((4, 2), np.float64), "zeros": np.full((1, 4), 8.0)}
    a[what][0, 1] = value
    if value == int(value):
        a = {k: v.astype(np.int64) for k, v in a.items()}
    with pytest.raises(ValueError, match=what):
        nb.W4(a["codes"], np.ones((1, 4), np.float32), 4, 4, 32, zeros=a["zeros"])


def test_codes_of_a_wider_type_that_are_bytes():
    """The same as bytes: what is refused here is a zero point above 15, by the library."""
    z = np.full((1, 4), 16, np.int64)
    with pytest.raises(nb.NmtError) as ei:
        nb.W4(np.full((4, 2), 255, np.int32), np.ones((1, 4)), 4, 4, 32, zeros=z)
    assert ei.value.status == nb.NMT_ERANGE
