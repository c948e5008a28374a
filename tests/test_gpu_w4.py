"""4-bit products (csrc/w4.hip) against 64-bit sums: odd sizes, groups, zero
points, types, strides, alignments, magnitudes, infinities, graphs."""
import numpy as np
import pytest

import draft_cases as dc
from paper_1605_04809_amd.workloads import CONFIGS, make_workload

pytestmark = pytest.mark.gpu


def _torch():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _handle(nb, c, K, N, group, stype="f32"):
    return nb.W4(dc.pack_codes(c["codes"]), c["scales"], K, N, group, zeros=c["zeros"], bias=c["bias"], stype=stype)


def _rows(torch, x, dtype, pad=0, shift=0):
    """x as rows of a wider device array that starts `shift` elements into its memory."""
    flat = torch.full((x.shape[0] * (x.shape[1] + pad) + shift,), 7.0, dtype=dtype, device="cuda")
    out = flat[shift:].view(x.shape[0], x.shape[1] + pad)
    out[:, :x.shape[1]] = torch.from_numpy(np.ascontiguousarray(x)).cuda().to(dtype)
    return out[:, :x.shape[1]], out


TYPES = {"f32": "float32", "bf16": "bfloat16"}


def _check(torch, nb, K, N, M, group, zeros, bias, xt, yt, st, pad=0, shift=0, seed=0, x=None):
    rng = np.random.default_rng(seed)
    c = dc.make_w4(rng, K, N, group, zeros, bias, st)
    w = _handle(nb, c, K, N, group, st)
    if x is None:
        x = rng.standard_normal((M, K)).astype(np.float32)
    if xt == "bf16":
        x = dc.round_bf16(x)
    xd, _ = _rows(torch, x, getattr(torch, TYPES[xt]), pad, shift)
    yd, wide = _rows(torch, np.zeros((M, N), np.float32), getattr(torch, TYPES[yt]), pad, shift)
    nb.nmt_w4_product(w, xd, yd)
    torch.cuda.synchronize()
    want = x.astype(np.float64) @ c["w"] + (0 if c["bias"] is None else c["bias"].astype(np.float64))
    got = yd.float().cpu().numpy().astype(np.float64)
    bound = dc.w4_bound(x, c, K, group, yt, want)
    worst = np.max(np.abs(got - want) / bound)
    print(f"K={K} N={N} M={M} group={group} {xt}->{yt}: error {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0
    assert pad == 0 or bool((wide[:, N:] == 7.0).all())   # between the rows: untouched
    w.close()
    return got


@pytest.mark.parametrize("K,N,M", [(1, 1, 1), (7, 3, 2), (32, 16, 1), (33, 17, 5), (127, 100, 15), (128, 64, 16),
                                   (129, 65, 17), (500, 1000, 1), (500, 1003, 31), (500, 2049, 33), (1001, 777, 64),
                                   (1001, 777, 65), (2500, 300, 12), (4096, 160, 4), (6000, 33, 3), (64, 70000, 2),
                                   (500, 500, 300), (96, 40, 1100)])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True), (256, False)])
def test_sizes_and_groups(K, N, M, group, zeros):
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    _check(torch, nb, K, N, M, group, zeros, True, "f32", "f32", "f32", seed=K + N + M)


@pytest.mark.parametrize("xt", ["f32", "bf16"])
@pytest.mark.parametrize("yt", ["f32", "bf16"])
@pytest.mark.parametrize("st", ["f32", "bf16"])
@pytest.mark.parametrize("M,bias", [(1, False), (6, True), (40, False)])
def test_types(xt, yt, st, M, bias):
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    _check(torch, nb, 500, 1002, M, 64, True, bias, xt, yt, st, seed=3)


@pytest.mark.parametrize("xt,yt", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (4, 0), (8, 8), (5, 3)])
@pytest.mark.parametrize("K,N", [(500, 96), (333, 97)])
def test_strides_and_alignment(xt, yt, pad, shift, K, N):
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    _check(torch, nb, K, N, 9, 32, False, True, xt, yt, "f32", pad=pad, shift=shift, seed=pad + shift)


@pytest.mark.parametrize("xt", ["f32", "bf16"])
def test_magnitudes(xt):
    """Rows from 2^-140 to 2^120, rows that mix them, rows of zeros: each within
    its own bound (fp32 holds 2^-149 steps: a bound cannot be below one)."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    rng = np.random.default_rng(8)
    K = 500
    x = rng.standard_normal((20, K))
    for i, e in enumerate([-140, -126, -100, -60, -30, -10, 0, 10, 15, 17, 30, 60, 100, 117]):
        x[i] *= 2.0 ** e
    x[14] = 0.0
    x[15, 1:] = 0.0                                   # one value
    x[16] *= np.where(rng.random(K) < 0.5, 1.0, 2.0 ** -20)
    x[17] *= 2.0 ** rng.integers(-40, 40, size=K)
    x[18, :128] *= 2.0 ** 60
    x[19, 128:] *= 2.0 ** 60
    _check(torch, nb, K, 200, 20, 64, True, False, xt, "f32", "f32", seed=4, x=x.astype(np.float32))


@pytest.mark.parametrize("xt", ["f32", "bf16"])
def test_infinities_and_nan_stay_in_their_rows(xt):
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    rng = np.random.default_rng(9)
    K, N, M = 300, 90, 7
    c = dc.make_w4(rng, K, N, 32, True, True)
    w = _handle(nb, c, K, N, 32)
    x = dc.round_bf16(rng.standard_normal((M, K)).astype(np.float32))
    x[1, 5] = np.inf
    x[2, 299] = -np.inf
    x[3, 17] = np.nan
    x[4, 3], x[4, 200] = np.inf, -np.inf
    x[5] = 0.0
    x[5, 40] = np.inf
    dt = getattr(torch, TYPES[xt])
    y = torch.zeros((M, N), device="cuda")
    nb.nmt_w4_product(w, _rows(torch, x, dt)[0], y)
    got = y.cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = np.stack([(x[m].astype(np.float64)[:, None] * c["w"]).sum(0) for m in range(M)]) + c["bias"]
    for m in (0, 6):
        assert np.isfinite(got[m]).all()
    for m in range(1, 6):
        np.testing.assert_array_equal(np.isnan(got[m]), np.isnan(want[m]), err_msg=f"row {m}")
        inf = np.isinf(want[m])
        np.testing.assert_array_equal(got[m][inf], want[m][inf], err_msg=f"row {m}")
    # the other rows' values are those they have beside finite rows
    clean = np.where(np.isfinite(x), x, np.float32(1.0))
    y2 = torch.zeros((M, N), device="cuda")
    nb.nmt_w4_product(w, _rows(torch, clean, dt)[0], y2)
    np.testing.assert_array_equal(y2.cpu().numpy()[[0, 6]], got[[0, 6]])
    w.close()


def test_bias_of_minus_infinity_masks_its_column():
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    c = dc.make_w4(np.random.default_rng(1), 64, 50, 32, False, True)
    c["bias"][[0, 49]] = -np.inf
    w = _handle(nb, c, 64, 50, 32)
    y = torch.zeros((3, 50), device="cuda")
    nb.nmt_w4_product(w, torch.ones((3, 64), device="cuda"), y)
    got = y.cpu().numpy()
    assert np.isneginf(got[:, [0, 49]]).all() and np.isfinite(got[:, 1:49]).all()
    w.close()


@pytest.mark.parametrize("wtype", ["f32", "bf16"])
@pytest.mark.parametrize("E,V,group,stype", [(32, 1000, 32, "f32"), (52, 301, 32, "bf16"), (100, 77, 64, "f32"),
                                             (100, 77, 128, "bf16")])
def test_a_models_output_layer(wtype, E, V, group, stype):
    """The 4-bit copy holds what its rule says: rows of the identity read the weights back."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    wl = make_workload(CONFIGS["tiny"].replace(E=E, V=V, seed=12, wtype=wtype))
    W, b = wl.params["out_W"].copy(), wl.params["out_b"]
    W[:, 3] = 0.0
    W[: group, 5] = 0.0
    wl.params["out_W"] = W
    model = nb.Model.from_workload(wl)
    q = nb.W4.from_output(model, group, stype)
    assert q.info() == {"K": E, "N": V, "group": group, "stype": stype, "zeros": False, "bias": True}
    if wtype == "bf16":
        W = dc.round_bf16(W)
    want = np.zeros((E, V), np.float64)
    for g in range(-(-E // group)):
        k = slice(g * group, (g + 1) * group)
        s = np.abs(W[k]).max(0) / np.float32(7.0)
        s = dc.round_bf16(s) if stype == "bf16" else s
        with np.errstate(invalid="ignore", divide="ignore"):
            codes = np.where(s == 0, 0.0, np.clip(np.rint(W[k] / s), -7, 7))
        want[k] = codes.astype(np.float64) * s
    x = np.eye(E, dtype=np.float32)
    y = torch.zeros((E, V), device="cuda")
    nb.nmt_w4_product(q, torch.from_numpy(x).cuda(), y)
    got = y.cpu().numpy().astype(np.float64)
    # one product, then the bias added: half a step of each
    assert np.all(np.abs(got - (want + b)) <= 2.0 ** -24 * (2 * np.abs(want) + np.abs(want + b)) + 1e-44)
    model.close()
    y.zero_()   # the copy is the program's own
    nb.nmt_w4_product(q, torch.from_numpy(x).cuda(), y)
    np.testing.assert_array_equal(y.cpu().numpy(), got.astype(np.float32))
    q.close()


def test_refusals():
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    lib = nb.load_library()
    c = dc.make_w4(np.random.default_rng(1), 40, 10, 32, False, False)
    w = _handle(nb, c, 40, 10, 32)
    x, y = torch.zeros((4, 40), device="cuda"), torch.full((4, 10), 7.0, device="cuda")
    ok = [w.handle, 4, x.data_ptr(), 0, 40, y.data_ptr(), 0, 10, None]
    for at, value in [(1, -1), (2, None), (3, 2), (3, -1), (4, 39), (5, None), (6, 2), (7, 9), (2, x.data_ptr() + 2),
                      (5, y.data_ptr() + 1)]:
        args = list(ok)
        args[at] = value
        assert lib.nmt_w4_product(*args) == nb.NMT_EINVAL, (at, value)
        assert nb.last_error()
    args = list(ok)
    args[1] = 0
    assert lib.nmt_w4_product(*args) == nb.NMT_OK
    torch.cuda.synchronize()
    assert bool((y == 7.0).all())
    for bad in (torch.zeros((4, 41), device="cuda"), torch.zeros((4, 80), device="cuda")[:, ::2],
                torch.zeros((4, 40), device="cuda", dtype=torch.float16)):
        with pytest.raises(ValueError):
            nb.nmt_w4_product(w, bad, y)
    wl = make_workload(CONFIGS["tiny"].replace(seed=12))
    wl.params["out_W"][1, 2] = np.inf
    model = nb.Model.from_workload(wl)
    base = nb.debug_alloc_hook(-1)
    with pytest.raises(nb.NmtError, match="finite") as ei:
        nb.W4.from_output(model)
    assert ei.value.status == nb.NMT_EINVAL
    with pytest.raises(nb.NmtError, match="group"):
        nb.W4.from_output(model, 20)
    assert nb.debug_alloc_hook(-1) == base
    model.close()
    w.close()


def test_allocation_failures_leave_nothing():
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    c = dc.make_w4(np.random.default_rng(1), 40, 10, 32, True, True)
    model = nb.Model.from_workload(make_workload(CONFIGS["tiny"].replace(seed=12)))
    base = nb.debug_alloc_hook(-1)
    try:
        for make in (lambda: _handle(nb, c, 40, 10, 32), lambda: nb.W4.from_output(model)):
            for n in range(10):
                nb.debug_alloc_hook(n)
                try:
                    w = make()
                except nb.NmtError as e:
                    assert e.status == nb.NMT_ENOMEM and nb.debug_alloc_hook(-1) == base
                    continue
                nb.debug_alloc_hook(-1)
                w.close()
                break
            assert n == 2 and nb.debug_alloc_hook(-1) == base
    finally:
        nb.debug_alloc_hook(-1)
    model.close()


@pytest.mark.parametrize("K,N,M", [(500, 3000, 3), (2000, 100, 20)])
def test_streams_and_graphs(K, N, M):
    """On a stream of its own, and captured: every replay gives the eager values."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    rng = np.random.default_rng(2)
    c = dc.make_w4(rng, K, N, 64, True, True)
    w = _handle(nb, c, K, N, 64)
    x = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).cuda()
    want, y = torch.zeros((M, N), device="cuda"), torch.zeros((M, N), device="cuda")
    nb.nmt_w4_product(w, x, want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        nb.nmt_w4_product(w, x, y)
    s.synchronize()
    assert torch.equal(y, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nb.nmt_w4_product(w, x, y)
    other = torch.zeros((M, N), device="cuda")
    for _ in range(4):
        y.fill_(float("nan"))
        g.replay()
        nb.nmt_w4_product(w, x.flip(0).contiguous(), other)
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(other, want.flip(0))
    w.close()


def test_a_row_does_not_depend_on_the_others():
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    rng = np.random.default_rng(3)
    c = dc.make_w4(rng, 500, 400, 32, True, True)
    w = _handle(nb, c, 500, 400, 32)
    x = rng.standard_normal((70, 500)).astype(np.float32)
    out = []
    for k in (0.0, 1e6):
        z = x * k
        z[[0, 33, 69]] = x[[0, 33, 69]]
        y = torch.zeros((70, 400), device="cuda")
        nb.nmt_w4_product(w, torch.from_numpy(z).cuda(), y)
        out.append(y.cpu().numpy()[[0, 33, 69]])
    np.testing.assert_array_equal(out[0], out[1])
    w.close()


@pytest.mark.parametrize("K,N,M,group", [(500, 200, 3, 96), (500, 200, 40, 160), (1001, 100, 20, 192), (700, 50, 1, 320),
                                         (96, 48, 2, 96), (4096, 64, 5, 4096), (500, 33, 17, 992)])
def test_groups_that_do_not_divide_a_block(K, N, M, group):
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    _check(torch, nb, K, N, M, group, True, True, "f32", "f32", "bf16", seed=group)


@pytest.mark.parametrize("K,N,M,xt", [(6001, 500, 5, "f32"), (6001, 500, 16, "f32"), (6001, 500, 17, "f32"),
                                      (6001, 500, 48, "f32"), (6001, 9000, 12, "f32"), (6001, 9000, 40, "bf16"),
                                      (3500, 34000, 33, "f32"), (3500, 17000, 64, "f32"), (12000, 20, 1, "bf16"),
                                      (1500, 66000, 20, "f32")])
@pytest.mark.parametrize("group", [32, 128])
def test_long_columns(K, N, M, xt, group):
    """K in chunks, split between waves, over several rounds of columns."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    _check(torch, nb, K, N, M, group, True, True, xt, "f32", "f32", seed=K + M)


@pytest.mark.parametrize("M", [2, 4, 5, 8, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 80, 81, 97])
@pytest.mark.parametrize("N", [2000, 40000])
def test_rows(M, N):
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    _check(torch, nb, 260, N, M, 64, True, True, "f32", "bf16", "bf16", seed=M)


def test_two_products_at_once():
    """One matrix on two streams: a product holds nothing between calls."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    rng = np.random.default_rng(5)
    c = dc.make_w4(rng, 500, 5000, 64, True, True)
    w = _handle(nb, c, 500, 5000, 64)
    xs = [torch.from_numpy(rng.standard_normal((M, 500)).astype(np.float32)).cuda() for M in (3, 40)]
    want = [torch.zeros((len(x), 5000), device="cuda") for x in xs]
    for x, y in zip(xs, want):
        nb.nmt_w4_product(w, x, y)
    torch.cuda.synchronize()
    got, streams = [torch.zeros_like(y) for y in want], [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for x, y, s in zip(xs, got, streams):
            with torch.cuda.stream(s):
                nb.nmt_w4_product(w, x, y)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    w.close()


def test_more_rows_than_a_launch_takes():
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    K, N, M = 32, 5, (1 << 21) + 3
    c = dc.make_w4(np.random.default_rng(6), K, N, 32, True, True)
    w = _handle(nb, c, K, N, 32)
    x = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    at = [0, 1, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, (1 << 21) - 1, 1 << 21, M - 1]
    few = torch.randn((len(at), K), device="cuda").bfloat16()
    x[at] = few
    y, want = torch.full((M, N), float("nan"), device="cuda"), torch.zeros((len(at), N), device="cuda")
    nb.nmt_w4_product(w, x, y)
    nb.nmt_w4_product(w, few, want)
    assert torch.equal(y[at], want) and bool(torch.isfinite(y).all())
    w.close()


@pytest.mark.parametrize("xt", ["f32", "bf16"])
@pytest.mark.parametrize("K,M,group", [(40, 3, 32), (300, 20, 32), (300, 40, 128), (7000, 3, 64)])
def test_scales_of_any_size(xt, K, M, group):
    """Columns with scales from 2^-100 to nearly 2^116 under rows whose products are ordinary: finite wherever
    fp32 holds the sum, each within the bound of its own size."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    rng = np.random.default_rng(12)
    N = 70
    c = dc.make_w4(rng, K, N, group, True, False)
    e = rng.integers(-100, 116, size=N)
    e[:6] = [115, 115, 110, 106, 102, -100]
    unit = np.exp2(np.floor(np.log2(np.abs(c["scales"]).max(0))))
    c["scales"] = (c["scales"] / unit * np.exp2(e)).astype(np.float32)   # the largest of a column in [2^e, 2^(e + 1))
    zero = c["zeros"].astype(np.float64)[np.arange(K) // group]
    c["w"] = c["scales"].astype(np.float64)[np.arange(K) // group] * (c["codes"].astype(np.float64) - zero)
    w = _handle(nb, c, K, N, group)
    x = rng.standard_normal((M, K)) * np.exp2(rng.integers(-100, 12, size=M))[:, None]
    x[0] *= np.exp2(-20 - np.log2(np.abs(x[0]).max()))      # tiny beside the largest scales
    x[1] *= np.exp2(1 - np.log2(np.abs(x[1]).max()))        # ordinary ones
    x = x.astype(np.float32)
    x = dc.round_bf16(x) if xt == "bf16" else x
    y = torch.zeros((M, N), device="cuda")
    nb.nmt_w4_product(w, _rows(torch, x, getattr(torch, TYPES[xt]))[0], y)
    got = y.cpu().numpy().astype(np.float64)
    a, aw = np.abs(x.astype(np.float64)), np.abs(c["w"])
    # a term of sum |x||w| below half of fp32's largest value cannot make any partial sum infinite
    holds = a @ aw < 2.0 ** 127
    assert holds[0].all() and holds[1, 5:].any() and np.isfinite(got[holds]).all()
    bound = dc.w4_bound(x, c, K, group, "f32", None)
    worst = np.max((np.abs(got - x.astype(np.float64) @ c["w"]) / bound)[holds])
    print(f"K={K} M={M} group={group} {xt}: error {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0
    w.close()



def test_output_layers_too_large_for_scales():
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    wl = make_workload(CONFIGS["tiny"].replace(seed=12))
    for value, ok in ((-7.0 * 2.0 ** 116, True), (7.5 * 2.0 ** 116, False)):
        wl.params["out_W"][1, 2] = value
        model = nb.Model.from_workload(wl)
        for stype in ("f32", "bf16"):
            if ok:
                nb.W4.from_output(model, 32, stype).close()
                continue
            with pytest.raises(nb.NmtError, match="above") as ei:
                nb.W4.from_output(model, 32, stype)
            assert ei.value.status == nb.NMT_EINVAL
        model.close()


@pytest.mark.parametrize("K,M", [(40, 3), (300, 20), (300, 40), (7000, 3)])
def test_the_smallest_inputs(K, M):
    """Rows of fp32's smallest values (steps of 2^-149), under scales that bring their products back to ordinary
    size: every bit of them counts."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    rng = np.random.default_rng(13)
    N, group = 50, 64
    c = dc.make_w4(rng, K, N, group, True, False)
    for k in ("scales", "w"):
        c[k] = (c[k] * 2.0 ** 100).astype(c[k].dtype)
    w = _handle(nb, c, K, N, group)
    step = np.exp2(rng.integers(0, 22, size=M))[:, None]
    step[:2] = [[1.0], [2.0]]
    x = (np.rint(rng.standard_normal((M, K)) * step) * 2.0 ** -149).astype(np.float32)
    x[0, 0], x[1, K - 1] = 2.0 ** -149, -(2.0 ** -148)
    y = torch.zeros((M, N), device="cuda")
    nb.nmt_w4_product(w, torch.from_numpy(x).cuda(), y)
    got, want = y.cpu().numpy().astype(np.float64), x.astype(np.float64) @ c["w"]
    assert np.all(np.abs(got - want) <= dc.w4_bound(x, c, K, group, "f32", want))
    w.close()
