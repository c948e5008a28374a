"""nmt_step_readouts and nmt_logits against the step that scores requested
words and the fp64 oracle, and a drafted round from end to end: a 4-bit output
layer drafts, the full model verifies."""
import numpy as np
import pytest

import draft_cases as dc
from gpu_cases import GpuRun, OracleRun, cuda, max_abs
from paper_1605_04809_amd.workloads import CONFIGS, make_workload, param_shapes

pytestmark = pytest.mark.gpu


def _torch():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _layer(nb, rng, E, V, wtype, gain=2.0, bias=0.3, spoil=False):
    p = {n: np.zeros(s, np.float32) for n, s in param_shapes(4, V, E, 8, 8).items()}
    p["out_W"] = (gain / np.sqrt(E) * rng.standard_normal((E, V))).astype(np.float32)
    p["out_b"] = (bias * rng.standard_normal(V)).astype(np.float32)
    if spoil:   # columns of magnitudes that two fp16 halves do not hold
        p["out_W"][:, ::7] *= np.float32(2.0 ** -20)
    if wtype == "bf16":
        p["out_W"] = dc.round_bf16(p["out_W"])
    return nb.Model(p, 4, V, E, 8, 8, wtype), p["out_W"].astype(np.float64), p["out_b"].astype(np.float64)


def _logits(torch, nb, model, t, pad=0, logZ=True):
    M = t.shape[0]
    wide = torch.full((M, model.V + pad), 7.0, device="cuda")
    lz = torch.full((M,), 7.0, device="cuda") if logZ else None
    nb.nmt_logits(model, cuda(t), wide[:, :model.V], logZ=lz)
    torch.cuda.synchronize()
    assert bool((wide[:, model.V:] == 7.0).all())
    return wide[:, :model.V].cpu().numpy().astype(np.float64), None if lz is None else lz.cpu().numpy().astype(np.float64)


def _check_logits(z, lz, t, W, b):
    """Each of the sum's terms and partial sums is rounded to fp32 once, and an fp32 input enters with half a
    step of 22 bits at worst (three products of halves: 4 more): E + 16 roundings of sum |t||W| + |b|."""
    t64 = t.astype(np.float64)
    want = t64 @ W + b
    bound = (W.shape[0] + 16) * 2.0 ** -24 * (np.abs(t64) @ np.abs(W) + np.abs(b)) + 1e-44
    worst = np.max(np.abs(z - want) / bound)
    assert worst <= 1.0, worst
    if lz is not None:
        m = want.max(1)
        wlz = m + np.log(np.exp(want - m[:, None]).sum(1))
        # log of a sum of V positive terms: a logit's error, V / 256 + 256 roundings of the sum, and the result's own
        tol = bound.max(1) + (W.shape[1] / 256 + 256) * 2.0 ** -24 + 2.0 ** -23 * np.abs(wlz)
        assert np.all(np.abs(lz - wlz) <= tol)
    return worst


@pytest.mark.parametrize("wtype,spoil", [("f32", False), ("f32", True), ("bf16", False)])
@pytest.mark.parametrize("E,V", [(4, 1), (32, 1000), (52, 3001), (72, 100), (96, 33), (300, 5003), (500, 4096), (560, 777)])
@pytest.mark.parametrize("M", [1, 33, 130])
def test_logits(wtype, spoil, E, V, M):
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    rng = np.random.default_rng(E + V + M)
    model, W, b = _layer(nb, rng, E, V, wtype, spoil=spoil)
    t = np.tanh(rng.standard_normal((M, E))).astype(np.float32)
    if wtype == "bf16":
        t = dc.round_bf16(t)
    z, lz = _logits(torch, nb, model, t, pad=M % 4)
    worst = _check_logits(z, lz, t, W, b)
    print(f"{wtype} E={E} V={V} M={M}: error {worst:.3f} of the bound", flush=True)
    z2, _ = _logits(torch, nb, model, t, pad=0, logZ=False)
    np.testing.assert_array_equal(z, z2)
    model.close()


@pytest.mark.parametrize("wtype", ["f32", "bf16"])
def test_logits_of_any_magnitude(wtype):
    """Readouts far from a tanh's: rows from 2^-60 to 2^60, rows that hold a NaN
    or an infinity (none of their logits finite), zeros."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    rng = np.random.default_rng(7)
    E, V = 100, 515
    model, W, b = _layer(nb, rng, E, V, wtype)
    t = rng.standard_normal((12, E))
    for i, e in enumerate([-60, -36, -20, -13, 0, 3, 5, 20, 60]):
        t[i] *= 2.0 ** e
    t[9] = 0.0
    t = dc.round_bf16(t.astype(np.float32))
    t[10, 3], t[11, 99] = np.nan, np.inf
    z, lz = _logits(torch, nb, model, t)
    _check_logits(z[:10], lz[:10], t[:10], W, b)
    assert not np.isfinite(z[10:]).any()
    model.close()
    # without a bias the small rows' own digits count
    model, W, b = _layer(nb, rng, E, V, wtype, bias=0.0)
    z, _ = _logits(torch, nb, model, t[:10])
    want = t[:10].astype(np.float64) @ W
    size = np.abs(t[:10].astype(np.float64)) @ np.abs(W)
    # a row is scaled up by at most 2^24 beyond a readout's 2^14, so below 2^-24 its values err by 2^-24 times 2^-25
    tol = (E + 16) * 2.0 ** -24 * (size + 2.0 ** -39 * np.abs(W).sum(0)) + 1e-44
    assert np.all(np.abs(z - want) <= tol)
    model.close()


def test_logits_refusals():
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    lib = nb.load_library()
    model, _, _ = _layer(nb, np.random.default_rng(0), 32, 50, "f32")
    t, z = torch.zeros((3, 32), device="cuda"), torch.full((3, 50), 7.0, device="cuda")
    need = nb.nmt_score_workspace_bytes(model, 3)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    ok = [model.handle, 3, t.data_ptr(), z.data_ptr(), 50, None, ws.data_ptr(), need, None]
    for at, value, rc in [(1, -1, -1), (2, None, -1), (2, t.data_ptr() + 4, -1), (3, None, -1), (3, z.data_ptr() + 2, -1),
                          (4, 49, -1), (6, None, -1), (6, ws.data_ptr() + 8, -1), (7, 16, -5)]:
        args = list(ok)
        args[at] = value
        assert lib.nmt_logits(*args) == rc, (at, value)
    args = list(ok)
    args[1] = 0
    assert lib.nmt_logits(*args) == nb.NMT_OK
    torch.cuda.synchronize()
    assert bool((z == 7.0).all())
    model.close()


CASES = [("tiny", {}), ("tiny", dict(wtype="bf16", E=52, V=701, H=100, A=76, B=37, S=3, len_lo=1, len_hi=9, Tpad=9)),
         ("tiny", dict(E=52, V=701, H=100, A=76, B=133, S=3, len_lo=1, len_hi=9, Tpad=9)),
         ("tiny", dict(E=100, V=501, H=256, A=128, B=70, S=2, len_lo=3, len_hi=12, Tpad=12))]


@pytest.mark.parametrize("name,kw", CASES)
def test_readouts_are_the_scoring_steps(name, kw):
    """Bit for bit the step's states and readouts; with its logits the step's log p."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    wl = make_workload(CONFIGS[name].replace(seed=41, sigma_w=0.2, **kw))
    c = wl.cfg
    run = GpuRun(wl)
    step = run.step(wl.s_prev, wl.y_prev, wl.sent_id, wl.req)
    s_new, t = torch.full((c.B, c.H), 7.0, device="cuda"), torch.full((c.B, c.E), 7.0, device="cuda")
    y, sent, sp = cuda(wl.y_prev), cuda(wl.sent_id), cuda(wl.s_prev)
    nb.nmt_step_readouts(run.model, run.src, sp, y, sent, s_new, t)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(s_new.cpu().numpy(), step["s_new"])
    np.testing.assert_array_equal(t.cpu().numpy(), step["t"])
    # from a pool, by index, and in place
    perm = np.random.default_rng(1).permutation(c.B).astype(np.int32)
    pool = torch.zeros((c.B + 5, c.H), device="cuda")
    pool[torch.from_numpy(perm).cuda().long()] = sp
    s2, t2 = torch.empty_like(s_new), torch.empty_like(t)
    nb.nmt_step_readouts(run.model, run.src, pool, y, sent, s2, t2, state_row=cuda(perm))
    nb.nmt_step_readouts(run.model, run.src, sp, y, sent, sp, t)
    torch.cuda.synchronize()
    for a, b in ((s2, s_new), (t2, t), (sp, s_new)):
        assert torch.equal(a, b)
    z, lz = torch.empty((c.B, c.V), device="cuda"), torch.empty(c.B, device="cuda")
    nb.nmt_logits(run.model, t, z, logZ=lz)
    lp = torch.gather(z, 1, cuda(wl.req).long()[:, None])[:, 0] - lz
    assert max_abs(lp.cpu().numpy(), step["logp"]) <= 4e-6 * max(1.0, np.abs(step["logp"]).max())
    ora = OracleRun(wl).step(wl.s_prev, wl.y_prev, wl.sent_id, wl.req)
    assert max_abs(lp.cpu().numpy(), ora["logp"]) <= (2e-2 if c.wtype == "bf16" else 1e-4)
    assert nb.nmt_stream_status(run.model) == nb.NMT_OK
    # ids out of range: that row alone, and the flag
    bad_y, bad_s = y.clone(), sent.clone()
    bad_y[0], bad_s[c.B - 1] = c.V, -1
    nb.nmt_step_readouts(run.model, run.src, cuda(wl.s_prev), bad_y, bad_s, s2, t2)
    assert nb.nmt_stream_status(run.model) == nb.NMT_ERANGE
    got = t2.cpu().numpy()
    assert np.isnan(got[[0, c.B - 1]]).all()
    np.testing.assert_array_equal(got[1:-1], step["t"][1:-1])
    lib = nb.load_library()
    ws = torch.zeros(nb.nmt_score_workspace_bytes(run.model, c.B), dtype=torch.uint8, device="cuda")
    ok = [run.model.handle, run.src.handle, c.B, pool.data_ptr(), c.B, None, y.data_ptr(), sent.data_ptr(),
          s2.data_ptr(), t2.data_ptr(), ws.data_ptr(), ws.numel(), None]
    for at, value, rc in [(2, -1, -1), (3, None, -1), (4, c.B - 1, -1), (6, None, -1), (7, None, -1), (8, None, -1),
                          (9, None, -1), (9, t2.data_ptr() + 4, -1), (10, None, -1), (11, 16, -5)]:
        args = list(ok)
        args[at] = value
        assert lib.nmt_step_readouts(*args) == rc, (at, value)
    run.close()


def _round(torch, nb, model, src, w4, states, last, sent, k, u_draft, u):
    """One round: k words drafted by the 4-bit output layer, verified by the full one.  Returns the drafts,
    proposals, target logits, what the verification gave, and every position's states."""
    S, H, E, V = states.shape[0], model.H, model.E, model.V
    i32 = dict(dtype=torch.int32, device="cuda")
    one = torch.arange(S + 1, **i32) * 0
    pos_states, ts, drafts, props = [], [], [], []
    st, y = states, last
    for j in range(k + 1):
        s_new, t = torch.empty((S, H), device="cuda"), torch.empty((S, E), device="cuda")
        nb.nmt_step_readouts(model, src, st, y, sent, s_new, t)
        pos_states.append(s_new)
        ts.append(t)
        if j == k:
            break
        zq = torch.empty((S, V), device="cuda")
        nb.nmt_w4_product(w4, t, zq)
        acc, word = torch.empty(S, **i32), torch.empty(S, **i32)
        nb.nmt_verify_drafts(model, one, torch.empty(0, **i32), zq, None, u_draft[j], acc, word)   # a sample of each row
        drafts.append(word)
        props.append(zq)
        st, y = s_new, word
    off = torch.arange(S + 1, **i32) * k
    draft = torch.stack(drafts, 1).reshape(-1).contiguous()
    prop = torch.stack(props, 1).reshape(S * k, V).contiguous()
    t_all = torch.stack(ts, 1).reshape(S * (k + 1), E).contiguous()
    z = torch.empty((S * (k + 1), V), device="cuda")
    nb.nmt_logits(model, t_all, z)
    acc, nxt = torch.empty(S, **i32), torch.empty(S, **i32)
    nb.nmt_verify_drafts(model, off, draft, z, prop, u, acc, nxt)
    return off, draft, prop, z, t_all, acc, nxt, torch.stack(pos_states, 1)


@pytest.mark.parametrize("wtype", ["f32", "bf16"])
def test_a_drafted_round(wtype):
    """Three rounds in a row, each from the states that the last one's kept drafts left, against the 64-bit
    verification of the same logits; the logits against the oracle's readouts."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    wl = make_workload(CONFIGS["tiny"].replace(V=701, E=52, H=100, A=76, S=6, B=6, len_lo=2, len_hi=11, Tpad=11,
                                               sigma_w=0.25, sigma_emb=0.5, seed=31, wtype=wtype))
    c = wl.cfg
    k, S = 3, c.S
    run, ora = GpuRun(wl), OracleRun(wl)
    w4 = nb.W4.from_output(run.model, 32)
    sent = torch.arange(S, dtype=torch.int32, device="cuda")
    states, last = run.s0.clone(), torch.full((S,), -1, dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(2)
    W, b = wl.params["out_W"].astype(np.float64), wl.params["out_b"].astype(np.float64)
    words = [[] for _ in range(S)]
    kept_all = 0
    for _ in range(3):
        ud = [cuda(rng.random(S, dtype=np.float32)) for _ in range(k)]
        u = cuda(rng.random(S * (k + 1), dtype=np.float32))
        s_in, y_in = states.cpu().numpy(), last.cpu().numpy()
        off, draft, prop, z, t_all, acc, nxt, pos = _round(torch, nb, run.model, run.src, w4, states, last, sent, k, ud, u)
        torch.cuda.synchronize()
        assert nb.nmt_stream_status(run.model) == nb.NMT_OK
        ins = [a.cpu().numpy() for a in (off, draft, z, prop, u)]
        want = dc.verify(*ins)
        a, n = acc.cpu().numpy(), nxt.cpu().numpy()
        np.testing.assert_array_equal(a, want[0])
        np.testing.assert_array_equal(n, want[1])
        for j in range(k):   # the drafts: each the sample of its proposal row
            got = dc.verify(np.zeros(S + 1, np.int32), np.zeros(0, np.int32), ins[3].reshape(S, k, -1)[:, j], None,
                            ud[j].cpu().numpy())
            np.testing.assert_array_equal(ins[1].reshape(S, k)[:, j], got[1])
        # the target's logits: the oracle's along the same words
        st, y = s_in.astype(np.float64), y_in
        for j in range(k + 1):
            o = ora.step(st, y, np.arange(S, dtype=np.int32), np.zeros(S, np.int32))
            tol = 5e-2 if wtype == "bf16" else 1e-4
            assert max_abs(ins[2].reshape(S, k + 1, -1)[:, j], o["t"] @ W + b) <= tol
            st = o["s_new"]
            if j < k:
                y = ins[1].reshape(S, k)[:, j]
        # the next round starts behind the kept drafts
        states = pos[torch.arange(S, device="cuda"), acc.long()].contiguous()
        last = nxt.clone()
        for s in range(S):
            words[s] += ins[1].reshape(S, k)[s, :a[s]].tolist() + [int(n[s])]
        kept_all += int(a.sum())
    print(f"{wtype}: {kept_all} of {9 * S} drafts kept, {sum(map(len, words))} words", flush=True)
    assert all(0 <= w < c.V for ws in words for w in ws) and 0 < kept_all
    w4.close()
    run.close()


def test_a_round_captured():
    """A whole round in one graph, replayed with eager work between."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    wl = make_workload(CONFIGS["tiny"].replace(S=4, B=4, sigma_w=0.2, sigma_emb=0.4, seed=33))
    run = GpuRun(wl)
    w4 = nb.W4.from_output(run.model, 32, "bf16")
    S, k = 4, 2
    rng = np.random.default_rng(3)
    sent = torch.arange(S, dtype=torch.int32, device="cuda")
    last = torch.full((S,), -1, dtype=torch.int32, device="cuda")
    ud = [cuda(rng.random(S, dtype=np.float32)) for _ in range(k)]
    u = cuda(rng.random(S * (k + 1), dtype=np.float32))
    args = (torch, nb, run.model, run.src, w4, run.s0, last, sent, k, ud, u)
    want = [x.clone() for x in _round(*args)[1:]]
    torch.cuda.synchronize()
    cap = torch.cuda.Stream()
    with torch.cuda.stream(cap):
        _round(*args)
    cap.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = _round(*args)[1:]
    for _ in range(4):
        for x in out:
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
        other = _round(*args)[1:]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(other, want))
    assert nb.nmt_stream_status(run.model) == nb.NMT_OK
    w4.close()
    run.close()


@pytest.mark.parametrize("wtype,spoil", [("f32", False), ("f32", True), ("bf16", False)])
@pytest.mark.parametrize("V,M", [(33, 3), (515, 12), (9000, 70)])
def test_log_sum_of_logits_that_are_not_finite(wtype, spoil, V, M):
    """log Z is what its row's logits give: NaN beside a NaN, infinity beside
    an infinity, and the other rows' as they are without such rows."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    rng = np.random.default_rng(V)
    E = 100
    model, W, b = _layer(nb, rng, E, V, wtype, spoil=spoil)
    t = dc.round_bf16(np.tanh(rng.standard_normal((M, E))).astype(np.float32))
    _, clean = _logits(torch, nb, model, t)
    t[0] = np.nan                    # what nmt_step_readouts gives for an id out of range
    t[1, 7] = np.inf
    t[M - 1, 99] = -np.inf
    z, lz = _logits(torch, nb, model, t)
    want = torch.logsumexp(torch.from_numpy(z), 1).numpy()
    assert np.isnan(lz[0]) and not np.isfinite(lz[[1, M - 1]]).any()
    for r in (0, 1, M - 1):
        np.testing.assert_equal(lz[r], want[r])
    np.testing.assert_array_equal(lz[2:M - 1], clean[2:M - 1])
    model.close()


@pytest.mark.parametrize("wtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [70, 9000])
def test_log_sum_beside_single_logits_that_are_not_finite(wtype, V):
    """A bias of NaN or, with fp32 weights, of infinities in single columns (V = 9,000: of one slice alone)."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    rng = np.random.default_rng(V)
    E = 32
    p = {n: np.zeros(s, np.float32) for n, s in param_shapes(4, V, E, 8, 8).items()}
    p["out_W"] = dc.round_bf16(rng.standard_normal((E, V)).astype(np.float32))
    t = np.tanh(rng.standard_normal((5, E))).astype(np.float32)
    infinite = ((np.inf, 40), (-np.inf, 3), (-np.inf, slice(0, 64)), (-np.inf, slice(None)))
    for value, at in ((np.nan, 3), (np.nan, V - 1)) + (infinite if wtype == "f32" else ()):
        p["out_b"] = np.zeros(V, np.float32)
        p["out_b"][at] = value
        model = nb.Model(p, 4, V, E, 8, 8, wtype)
        z, lz = _logits(torch, nb, model, t)
        want = torch.logsumexp(torch.from_numpy(z), 1).numpy()
        assert np.isfinite(want).all() == (value == -np.inf and at != slice(None))
        # (V / 256 + 256 roundings of the sum, and the result's own)
        tol = np.where(np.isfinite(want), (V / 256 + 256) * 2.0 ** -24 + 2.0 ** -23 * np.abs(want), 0.0)
        np.testing.assert_array_equal(np.isnan(lz), np.isnan(want))
        with np.errstate(invalid="ignore"):
            near = (lz == want) | np.isnan(want) | (np.abs(lz - want) <= tol)
        assert np.all(near), (value, at)
        model.close()


@pytest.mark.parametrize("call", ["score", "forest_step", "ensemble", "readouts", "logits", "verify"])
def test_scratch_of_a_call_on_another_stream(call):
    """A call on a stream that is not the current one, with no workspace given: memory that the current stream
    gets while the call waits its turn there is not the call's scratch."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    wl = make_workload(CONFIGS["tiny"].replace(S=4, B=4, V=3000, seed=35))
    run, c = GpuRun(wl), wl.cfg
    i32, B = dict(dtype=torch.int32, device="cuda"), wl.cfg.B
    sp, y, sent, req = cuda(wl.s_prev), cuda(wl.y_prev), cuda(wl.sent_id), cuda(wl.req)
    logp, s_new, t = torch.empty(B, device="cuda"), torch.empty((B, c.H), device="cuda"), torch.zeros((B, c.E), device="cuda")
    z, logZ = torch.zeros((B, c.V), device="cuda"), torch.empty(B, device="cuda")
    rows, off, at0 = torch.arange(B, **i32), torch.arange(B + 1, **i32), torch.zeros(B + 1, **i32)
    u, acc, nxt = torch.full((B,), 0.5, device="cuda"), torch.empty(B, **i32), torch.empty(B, **i32)
    need = nb.nmt_score_workspace_bytes(run.model, B)
    need, go = {
        "score": (need, lambda s: nb.nmt_score_batch(run.model, run.src, sp, y, sent, req, logp, s_new, stream=s)),
        "forest_step": (need, lambda s: nb.nmt_score_forest_step(run.model, run.src, sp, rows, y, sent, off, req, logp,
                                                                 s_new, stream=s)),
        "ensemble": (nb.nmt_ensemble_workspace_bytes([run.model], B),
                     lambda s: nb.nmt_score_ensemble([run.model], [run.src], [sp], y, sent, req, logp[None], [s_new],
                                                     stream=s)),
        "readouts": (need, lambda s: nb.nmt_step_readouts(run.model, run.src, sp, y, sent, s_new, t, stream=s)),
        "logits": (need, lambda s: nb.nmt_logits(run.model, t, z, logZ=logZ, stream=s)),
        "verify": (nb.nmt_verify_workspace_bytes(run.model, B, 0),
                   lambda s: nb.nmt_verify_drafts(run.model, at0, at0[:0], z, None, u, acc, nxt, stream=s)),
    }[call]
    a = torch.zeros((4096, 4096), device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(200):     # over 0.1 s, far longer than what follows takes on the host
            a = a @ a
    go(s)
    theirs = [torch.full((max(need, 256),), 7, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.current_stream().synchronize()
    assert not s.query()         # the call still waits
    s.synchronize()
    assert all(bool((x == 7).all()) for x in theirs)
    assert nb.nmt_stream_status(run.model) == nb.NMT_OK
    run.close()


@pytest.mark.parametrize("wtype,spoil", [("f32", False), ("f32", True), ("bf16", False)])
def test_logits_of_small_rows(wtype, spoil):
    """Without a bias a row of any size keeps its own digits: relative to sum |t||W|, and where it is
    fp32's smallest values that count, 2^-150 for each rounding."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    rng = np.random.default_rng(11)
    E, V = 100, 515
    model, W, b = _layer(nb, rng, E, V, wtype, bias=0.0, spoil=spoil)
    exps = [-24, -25, -40, -64, -80, -100] + ([-124, -135, -140] if wtype == "f32" and not spoil else [])
    t = np.stack([rng.standard_normal(E) * 2.0 ** e for e in exps]).astype(np.float32)
    t = dc.round_bf16(t) if wtype == "bf16" else t
    z, _ = _logits(torch, nb, model, t)
    t64 = t.astype(np.float64)
    bound = (E + 16) * 2.0 ** -24 * (np.abs(t64) @ np.abs(W)) + (E + 16) * 2.0 ** -150
    worst = np.max(np.abs(z - t64 @ W) / bound, axis=1)
    print(wtype, spoil, worst, flush=True)
    assert np.all(worst <= 1.0)
    model.close()


@pytest.mark.parametrize("wtype", ["f32", "bf16"])
def test_words_that_the_bias_masks(wtype):
    """Biases of -infinity or fp32's lowest value forbid their words, in the logits, in the step's log p and in a
    4-bit copy of the layer; the other words' are as they are without such words."""
    torch = _torch()
    from paper_1605_04809_amd import binding as nb
    wl = make_workload(CONFIGS["tiny"].replace(seed=36, sigma_w=0.2, wtype=wtype))
    c, low = wl.cfg, np.finfo(np.float32).min
    masked = {3: -np.inf, c.V - 1: -np.inf, 70: low, 500: low}
    for v, b in masked.items():
        wl.params["out_b"][v] = b
    run = GpuRun(wl)
    req = wl.req.copy()
    req[:4] = list(masked)
    step = run.step(wl.s_prev, wl.y_prev, wl.sent_id, req)
    W, b = wl.params["out_W"], wl.params["out_b"].astype(np.float64)
    W = (dc.round_bf16(W) if wtype == "bf16" else W).astype(np.float64)
    t = step["t"]
    want = t.astype(np.float64) @ W + b
    z, lz = _logits(torch, nb, run.model, t)
    rest = np.setdiff1d(np.arange(c.V), list(masked))
    assert np.isneginf(z[:, [3, c.V - 1]]).all() and (z[:, [70, 500]] < -3.4e38).all()
    _check_logits(z[:, rest], None, t, W[:, rest], b[rest])
    wlz = np.log(np.exp(want[:, rest]).sum(1))
    tol = 2.0 ** -24 * ((c.E + 16) * (np.abs(t) @ np.abs(W[:, rest]) + np.abs(b[rest])).max(1) + c.V / 256 + 256)
    for got in (lz, step["logZ"]):
        assert np.all(np.abs(got - wlz) <= tol + 2.0 ** -23 * np.abs(wlz))
    assert np.isneginf(step["logp"][:2]).all() and (step["logp"][2:4] < -3.4e38).all()
    assert np.isfinite(step["logp"][4:]).all()
    w4 = nb.W4.from_output(run.model, 32)
    y = torch.zeros((c.B, c.V), device="cuda")
    nb.nmt_w4_product(w4, cuda(t), y)
    y = y.cpu().numpy()
    assert np.isneginf(y[:, [3, c.V - 1]]).all() and (y[:, [70, 500]] < -3.4e38).all() and np.isfinite(y[:, rest]).all()
    w4.close()
    run.close()
