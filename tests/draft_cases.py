"""Shared by the tests of drafted words: 4-bit matrices and a 64-bit
verification, in numpy."""
import numpy as np

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}   # half a step of a value near 1, relative


def make_w4(rng, K, N, group, zeros, bias, stype="f32"):
    """Codes [K, N], scales, zero points and bias, with the weights they stand for in 64 bits."""
    G = -(-K // group)
    codes = rng.integers(0, 16, size=(K, N)).astype(np.uint8)
    scales = (np.exp(0.3 * rng.standard_normal((G, N))) / (4.6 * np.sqrt(K))).astype(np.float32)
    scales *= np.where(rng.random((G, N)) < 0.1, -1.0, 1.0).astype(np.float32)
    if stype == "bf16":
        scales = round_bf16(scales)
    z = rng.integers(0, 16, size=(G, N)).astype(np.uint8) if zeros else None
    b = rng.standard_normal(N).astype(np.float32) if bias else None
    g = np.arange(K) // group
    w = scales.astype(np.float64)[g] * (codes.astype(np.float64) - (z[g].astype(np.float64) if zeros else 8.0))
    return {"codes": codes, "scales": scales, "zeros": z, "bias": b, "w": w}


def pack_codes(codes):
    K, N = codes.shape
    c = np.zeros((K, N + N % 2), np.uint8)
    c[:, :N] = codes
    return c[:, 0::2] | (c[:, 1::2] << 4)


def round_bf16(x):
    """Nearest bf16 values (ties to even), kept as fp32."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000
    return u.astype(np.uint32).view(np.float32)


def w4_bound(x, case, K, group, y_type, want):
    """Most that a product may be off by.  Every fp32 sum in it rounds each partial sum once, at most
    2^-24 of sum |x||w|: a group's terms, the groups, the bias, and a fp32 input's and scale's own
    roundings (8 with a margin); an input is off by at most 2^-39 of the largest beside it; a bf16
    result by half a step more.  Below fp32's normal range a rounding is 2^-150 whatever the value
    (scales are below 1)."""
    a = np.abs(np.asarray(x, np.float64))
    aw = np.abs(case["w"])
    size = a @ aw + (0 if case["bias"] is None else np.abs(case["bias"].astype(np.float64)))
    n = min(K, group) + -(-K // group) + 8
    err = n * 2.0 ** -24 * size + 2.0 ** -39 * a.max(axis=1, initial=0.0, keepdims=True) * aw.sum(axis=0)
    return err + (HALF["bf16"] * (np.abs(want) + err) if y_type == "bf16" else 0.0) + (K + 64) * 2.0 ** -150


def log_softmax(z):
    z = np.asarray(z, np.float64)
    m = z.max()
    return (z - m) - np.log(np.exp(z - m).sum())


def verify(off, draft, target, proposal, u):
    """nmt_verify_drafts in 64 bits, one sequence after another."""
    S = len(off) - 1
    acc, nxt = np.zeros(S, np.int32), np.zeros(S, np.int32)
    dlp, nlp = np.zeros(len(draft)), np.zeros(S)
    for s in range(S):
        n, rest = off[s + 1] - off[s], None
        for j in range(n):
            lp, d = log_softmax(target[off[s] + s + j]), draft[off[s] + j]
            dlp[off[s] + j] = lp[d]
            if rest is not None:
                continue
            q = np.zeros(len(lp))
            if proposal is None:
                q[d] = 1.0
            else:
                q = np.exp(log_softmax(proposal[off[s] + j]))
            p = np.exp(lp)
            if float(u[off[s] + s + j]) * q[d] < p[d]:
                acc[s] += 1
            else:
                rest, judge = np.maximum(p - q, 0.0), lp
                if rest.sum() == 0.0:
                    rest = p
        if rest is None:
            judge = log_softmax(target[off[s] + s + n])
            rest = np.exp(judge)
        c = np.cumsum(rest)
        v = int(np.searchsorted(c, float(u[off[s] + s + n]) * c[-1], side="right"))
        nxt[s] = min(v, int(np.nonzero(rest)[0][-1]))
        nlp[s] = judge[nxt[s]]
    return acc, nxt, dlp, nlp
