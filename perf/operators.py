"""Drafting and verifying words: the operators, their plain forms and their cases.

  w4       nmt_w4_product: products of a few rows with 4-bit weights and group scales
  verify   nmt_verify_drafts: which drafted words the target's distribution keeps, and the word after them
  logits   nmt_logits: the logits of all next words and their log-sum-exp

A case is a dict of plain values.  With `own` false, run() computes the plain form in torch operations; with
`own` true it calls the library.  Inputs come from the case's seed; the output weights of a `logits` case are
drawn once per model shape, as a program loads its model once.
"""
import math
from collections import OrderedDict

import numpy as np
import torch

own = False


def listed():
    return [
        # a drafting model's output layer at the smallest sizes: one row, latency
        {"name": "w4_tiny", "kind": "w4", "K": 32, "N": 1000, "M": 1, "group": 32, "x": "f32", "y": "f32",
         "scales": "f32", "zeros": False, "bias": True, "pad": 0},
        # one sentence drafting its next word over the whole vocabulary
        {"name": "w4_v100k_m1", "kind": "w4", "K": 500, "N": 100000, "M": 1, "group": 64, "x": "f32", "y": "f32",
         "scales": "f32", "zeros": False, "bias": True, "pad": 0},
        # a beam of 12 drafting, the smallest groups, zero points, 16-bit scales
        {"name": "w4_v50k_beam12", "kind": "w4", "K": 500, "N": 50000, "M": 12, "group": 32, "x": "f32", "y": "f32",
         "scales": "bf16", "zeros": True, "bias": True, "pad": 0},
        # a square hidden layer for a few rows in 16 bits, rows of a wider array
        {"name": "w4_square_bf16", "kind": "w4", "K": 4096, "N": 4096, "M": 4, "group": 128, "x": "bf16",
         "y": "bf16", "scales": "bf16", "zeros": True, "bias": False, "pad": 24},
        # odd sizes throughout, rows that are not 16-byte aligned
        {"name": "w4_odd_m33", "kind": "w4", "K": 1001, "N": 7777, "M": 33, "group": 64, "x": "f32", "y": "bf16",
         "scales": "f32", "zeros": True, "bias": True, "pad": 3},
        # all positions of 16 sequences with 4 drafts each: many rows
        {"name": "w4_v100k_m80", "kind": "w4", "K": 500, "N": 100000, "M": 80, "group": 64, "x": "f32", "y": "f32",
         "scales": "bf16", "zeros": False, "bias": True, "pad": 0},
        # one sequence over a toy vocabulary: launches and latency
        {"name": "verify_tiny", "kind": "verify", "V": 1000, "S": 1, "k": 4, "target": "f32", "proposal": "f32"},
        # a beam of 12 sequences with up to 4 drafts
        {"name": "verify_beam12", "kind": "verify", "V": 50000, "S": 12, "k": 4, "target": "f32", "proposal": "f32"},
        # a server's batch with long drafts, logits held in 16 bits
        {"name": "verify_s64_bf16", "kind": "verify", "V": 50000, "S": 64, "k": 8, "target": "bf16",
         "proposal": "bf16"},
        # phrases of a phrase table (certain drafts) under the full model
        {"name": "verify_phrases", "kind": "verify", "V": 100000, "S": 256, "k": 4, "target": "f32",
         "proposal": "none"},
        # a sequence's 5 positions under the full output layer: weights read for few rows
        {"name": "logits_m5", "kind": "logits", "E": 500, "V": 100000, "wtype": "f32", "M": 5},
        # 64 sequences of 5 positions, bf16 weights
        {"name": "logits_bf16_m320", "kind": "logits", "E": 500, "V": 100000, "wtype": "bf16", "M": 320},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["w4", "w4", "verify", "verify", "logits"])
    if kind == "w4":
        K = _log_int(rng, 16, 6000)
        N = min(_log_int(rng, 100, 100000), 50000000 // K)
        return {"kind": "w4", "K": K, "N": N, "M": min(_log_int(rng, 1, 200), 8000000 // N),
                "group": rng.choice([32, 64, 128]), "x": rng.choice(["f32", "bf16"]),
                "y": rng.choice(["f32", "bf16"]), "scales": rng.choice(["f32", "bf16"]),
                "zeros": rng.random() < 0.5, "bias": rng.random() < 0.7, "pad": rng.choice([0, 0, 8, rng.randint(1, 40)])}
    if kind == "verify":
        V = _log_int(rng, 100, 100000)
        k = rng.randint(1, 8)
        return {"kind": "verify", "V": V, "S": min(_log_int(rng, 1, 256), max(1, 50000000 // (V * (2 * k + 1)))),
                "k": k, "target": rng.choice(["f32", "bf16"]), "proposal": rng.choice(["f32", "f32", "bf16", "none"])}
    V = _log_int(rng, 500, 60000)
    return {"kind": "logits", "E": 4 * _log_int(rng, 8, 140), "V": V, "wtype": rng.choice(["f32", "bf16"]),
            "M": min(_log_int(rng, 1, 2000), 30000000 // V)}


# ------------------------------------------------------------------ inputs

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(values, dtype, pad):
    """The values as rows of a wider array (row stride: columns + pad)."""
    wide = torch.zeros((values.shape[0], values.shape[1] + pad), dtype=dtype, device="cuda")
    out = wide[:, :values.shape[1]]
    out.copy_(values)
    return out


def _w4_inputs(case, seed):
    g = _gen(seed)
    K, N, M, G = case["K"], case["N"], case["M"], -(-case["K"] // case["group"])
    d = dict(generator=g, device="cuda")
    codes = (torch.randn((K, N), **d) * 2.7 + 8).round_().clamp_(0, 15).to(torch.uint8)
    inp = {"codes": codes, "scales": torch.exp(0.3 * torch.randn((G, N), **d)) / (2.7 * math.sqrt(K))}
    if case["scales"] == "bf16":
        inp["scales"] = inp["scales"].bfloat16().float()
    inp["zeros"] = torch.randint(5, 12, (G, N), dtype=torch.uint8, **d) if case["zeros"] else None
    inp["bias"] = 0.1 * torch.randn(N, **d) if case["bias"] else None
    # readouts for the narrow layers; hidden activations, with a few large columns, for the wide ones
    x = torch.randn((M, K), **d)
    x = torch.tanh(x) if K <= 600 else x * torch.where(torch.rand(K, **d) < 0.01, 20.0, 1.0)
    inp["x"] = _rows(x, _TYPES[case["x"]], case["pad"])
    return inp


def _packed(codes):
    """Two codes a byte: byte i of a row holds columns 2i (low half) and 2i + 1."""
    K, N = codes.shape
    c = torch.zeros((K, N + N % 2), dtype=torch.uint8, device=codes.device)
    c[:, :N] = codes
    return (c[:, 0::2] | (c[:, 1::2] << 4)).contiguous()


def _verify_inputs(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    S, k, V = case["S"], case["k"], case["V"]
    # lengths from the case alone, as output shapes: 0..k drafts, at least one in the longest
    n = np.random.default_rng(S * 100 + k).integers(0, k + 1, size=S)
    n[S // 2] = k
    off = np.zeros(S + 1, np.int32)
    off[1:] = np.cumsum(n)
    nd = int(off[-1])
    seq = np.repeat(np.arange(S), n)
    row = torch.from_numpy(np.arange(nd) + seq).cuda()   # the target row that judges each draft
    d = dict(generator=g, device="cuda")
    z = torch.randn((nd + S, V), **d) * 2.5
    inp = {"off": torch.from_numpy(off).cuda(), "proposal": None}
    if case["proposal"] == "none":   # a phrase table proposes likely words, now and then any word
        noise = z[row] - torch.log(-torch.log(torch.rand((nd, V), **d).clamp_(1e-30, 1 - 1e-7)))
        draft = noise.argmax(1)
        odd = torch.from_numpy(rng.random(nd) < 0.2).cuda()
        draft = torch.where(odd, torch.randint(0, V, (nd,), **d), draft)
    else:                            # a smaller model: the same distribution, blurred, and its own sample
        zq = (z[row] + 0.7 * torch.randn((nd, V), **d)).to(_TYPES[case["proposal"]])
        gum = -torch.log(-torch.log(torch.rand((nd, V), **d).clamp_(1e-30, 1 - 1e-7)))
        draft = (zq.float() + gum).argmax(1)
        inp["proposal"] = zq
    inp["target"] = z.to(_TYPES[case["target"]])
    inp["draft"] = draft.to(torch.int32)
    inp["u"] = torch.from_numpy(rng.random(nd + S, dtype=np.float32)).cuda()
    return inp


_weights = OrderedDict()   # a program's loaded output layers, the last few shapes
_models = OrderedDict()


def _layer(case):
    """Output weights [E x V] and bias of a model shape, fp32 (bf16 models: at bf16 values)."""
    key = (case["E"], case["V"], case["wtype"])
    if key not in _weights:
        while len(_weights) >= 3:
            _weights.popitem(last=False)
        g = _gen(20160811)
        w = torch.randn(key[:2], generator=g, device="cuda") / math.sqrt(case["E"]) * 2.0
        b = 0.1 * torch.randn(case["V"], generator=g, device="cuda")
        _weights[key] = (w.bfloat16().float() if case["wtype"] == "bf16" else w, b)
    _weights.move_to_end(key)
    return _weights[key]


def _model(E, V, wtype="f32", layer=None):
    """A library model with a target vocabulary V (and this output layer); its other widths are small."""
    from paper_1605_04809_amd import binding as nb
    from paper_1605_04809_amd import workloads as wl
    key = (E, V, wtype, layer is None)
    if key not in _models:
        while len(_models) >= 4:
            _models.popitem(last=False)
        H = 64 if layer is not None else 4
        p = {n: np.zeros(s, np.float32) for n, s in wl.param_shapes(4, V, E, H, H).items()}
        if layer is not None:
            p["out_W"], p["out_b"] = layer[0].cpu().numpy(), layer[1].cpu().numpy()
        _models[key] = nb.Model(p, 4, V, E, H, H, wtype)
    _models.move_to_end(key)
    return _models[key]


def _t(case, seed):
    """Readouts [M x E]; those of a bf16 model are at bf16 values, as its step gives them."""
    t = torch.tanh(torch.randn((case["M"], case["E"]), generator=_gen(seed), device="cuda"))
    return t.bfloat16().float() if case["wtype"] == "bf16" else t


def prepare(case, seed):
    st = {"case": case}
    f32, kind = dict(dtype=torch.float32, device="cuda"), case["kind"]
    if kind == "w4":
        inp = _w4_inputs(case, seed)
        st["x"] = inp["x"]
        st["y"] = torch.empty((case["M"], case["N"]), dtype=_TYPES[case["y"]], device="cuda")
        packed = _packed(inp["codes"])
        if own:
            from paper_1605_04809_amd import binding as nb
            host = lambda a: None if a is None else a.cpu().numpy()
            st["w"] = nb.W4(host(packed), host(inp["scales"]), case["K"], case["N"], case["group"],
                            zeros=host(inp["zeros"]), bias=host(inp["bias"]), stype=case["scales"])
        else:
            st.update(codes=packed, scales=inp["scales"], zeros=inp["zeros"], bias=inp["bias"])
    elif kind == "verify":
        st.update(_verify_inputs(case, seed))
        nd, S, i32 = st["draft"].shape[0], case["S"], dict(dtype=torch.int32, device="cuda")
        st["out"] = {"accepted": torch.empty(S, **i32), "next": torch.empty(S, **i32),
                     "draft_logp": torch.empty(nd, **f32), "next_logp": torch.empty(S, **f32)}
        if own:
            from paper_1605_04809_amd import binding as nb
            st["model"] = _model(4, case["V"])
            n = nb.nmt_verify_workspace_bytes(st["model"], S, nd)
            st["ws"] = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    else:
        st["t"] = _t(case, seed)
        if own:
            from paper_1605_04809_amd import binding as nb
            st["model"] = _model(case["E"], case["V"], case["wtype"], _layer(case))
            st["z"], st["logZ"] = torch.empty((case["M"], case["V"]), **f32), torch.empty(case["M"], **f32)
            n = nb.nmt_score_workspace_bytes(st["model"], case["M"])
            st["ws"] = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
        else:
            st["W"], st["b"] = _layer(case)
    torch.cuda.synchronize()
    return st


# ------------------------------------------------------------------ one pass

def _unpack(packed, N):
    K = packed.shape[0]
    return torch.stack([packed & 15, packed >> 4], 2).reshape(K, -1)[:, :N]


def _w4_plain(st):
    case = st["case"]
    K, N = case["K"], case["N"]
    grp = torch.arange(K, device="cuda") // case["group"]
    zero = st["zeros"].float()[grp] if st["zeros"] is not None else 8.0
    w = (_unpack(st["codes"], N).float() - zero) * st["scales"][grp]
    y = st["x"].float() @ w
    if st["bias"] is not None:
        y += st["bias"]
    return y.to(_TYPES[case["y"]])


def _probs(z):
    e = torch.exp(z.double() - z.double().max(1, keepdim=True).values)
    return e / e.sum(1, keepdim=True)


def _verify_plain(st):
    off, draft, u = st["off"].long(), st["draft"].long(), st["u"].double()
    S, nd = off.shape[0] - 1, draft.shape[0]
    p = _probs(st["target"])
    n = off[1:] - off[:-1]
    s = torch.arange(S, device="cuda")
    j = torch.arange(nd, device="cuda")
    seq = torch.searchsorted(off, j, right=True) - 1
    pd = p[j + seq, draft]
    q = None if st["proposal"] is None else _probs(st["proposal"])
    qd = torch.ones_like(pd) if q is None else q[j, draft]
    lost = torch.full((S + 1,), nd + 1, dtype=torch.long, device="cuda")
    bad = torch.where(u[j + seq] * qd < pd, nd + 1, j - off[seq])
    lost = lost.scatter_reduce(0, seq, bad, "amin")[:S]
    a = torch.minimum(lost, n)
    r = p[off[:-1] + s + a]
    cut = (a < n).nonzero()[:, 0]
    at = (off[:-1] + a)[cut]
    if q is None:
        r[cut, draft[at]] = 0.0
    else:
        r[cut] = (r[cut] - q[at]).clamp_(min=0.0)
    c = r.cumsum(1)
    word = (c <= (u[off[1:] + s] * c[:, -1])[:, None]).sum(1)
    last = r.shape[1] - 1 - (r.flip(1) > 0).to(torch.uint8).argmax(1)
    word = torch.minimum(word, last)
    return {"accepted": a.int(), "next": word.int(), "draft_logp": torch.log(pd).float(),
            "next_logp": torch.log(p[off[:-1] + s + a, word]).float()}


def _logits_plain(st):
    z = st["t"] @ st["W"] + st["b"]
    m = z.max(1, keepdim=True).values
    return {"z": z, "logZ": m[:, 0] + torch.log(torch.exp(z - m).sum(1))}


def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"w4": _w4_plain, "verify": _verify_plain, "logits": _logits_plain}[kind](st)
    from paper_1605_04809_amd import binding as nb
    if kind == "w4":
        nb.nmt_w4_product(st["w"], st["x"], st["y"])
        return st["y"]
    if kind == "verify":
        o = st["out"]
        nb.nmt_verify_drafts(st["model"], st["off"], st["draft"], st["target"], st["proposal"], st["u"], o["accepted"],
                             o["next"], draft_logp=o["draft_logp"], next_logp=o["next_logp"], workspace=st["ws"])
        return o
    nb.nmt_logits(st["model"], st["t"], st["z"], logZ=st["logZ"], workspace=st["ws"])
    return {"z": st["z"], "logZ": st["logZ"]}


# -------------------------------------------------------- work and 64 bits

_BYTES = {"f32": 4, "bf16": 2}


def _drafts(case):
    n = np.random.default_rng(case["S"] * 100 + case["k"]).integers(0, case["k"] + 1, size=case["S"])
    n[case["S"] // 2] = case["k"]
    return int(n.sum())


def work(case):
    if case["kind"] == "w4":
        K, N, M, G = case["K"], case["N"], case["M"], -(-case["K"] // case["group"])
        b = (K * N / 2 + G * N * (_BYTES[case["scales"]] + (1 if case["zeros"] else 0)) + (4 * N if case["bias"] else 0)
             + M * K * _BYTES[case["x"]] + M * N * _BYTES[case["y"]])
        return {"bytes": b, "flops": 2.0 * M * K * N}
    if case["kind"] == "verify":
        nd, S, V = _drafts(case), case["S"], case["V"]
        p = (nd + S) * V
        q = 0 if case["proposal"] == "none" else nd * V
        b = p * _BYTES[case["target"]] + q * _BYTES.get(case["proposal"], 0) + 12.0 * nd + 20.0 * S
        return {"bytes": b, "flops": 3.0 * (p + q)}
    E, V, M = case["E"], case["V"], case["M"]
    return {"bytes": _BYTES[case["wtype"]] * E * V + 4.0 * (V + M * E + M * V + M), "flops": 2.0 * M * E * V}


def exact(case, seed):
    if case["kind"] == "w4":
        inp = _w4_inputs(case, seed)
        y = torch.zeros((case["M"], case["N"]), dtype=torch.float64, device="cuda")
        x = inp["x"].double()
        for g in range(inp["scales"].shape[0]):   # group by group: whole numbers first, then the scale
            k = slice(g * case["group"], (g + 1) * case["group"])
            c = inp["codes"][k].double()
            c -= inp["zeros"][g].double() if case["zeros"] else 8.0
            y += (x[:, k] @ c) * inp["scales"][g].double()
        if case["bias"]:
            y += inp["bias"].double()
        return y.cpu().numpy()
    if case["kind"] == "logits":
        w, b = _layer(case)
        z = _t(case, seed).double() @ w.double() + b.double()
        return {"z": z.cpu().numpy(), "logZ": torch.logsumexp(z, 1).cpu().numpy()}
    inp = {k: None if v is None else (v.float() if v.is_floating_point() else v).cpu().numpy()
           for k, v in _verify_inputs(case, seed).items()}
    off, draft, u = inp["off"], inp["draft"], inp["u"].astype(np.float64)
    S, nd = case["S"], len(draft)
    out = {"accepted": np.zeros(S, np.int32), "next": np.zeros(S, np.int32), "draft_logp": np.zeros(nd),
           "next_logp": np.zeros(S)}

    def log_softmax(z):
        z = z.astype(np.float64)
        z = z - z.max()
        return z - np.log(np.exp(z).sum())

    for s in range(S):
        n, rest = off[s + 1] - off[s], None
        for j in range(n):
            lp, d = log_softmax(inp["target"][off[s] + s + j]), draft[off[s] + j]
            out["draft_logp"][off[s] + j] = lp[d]
            if rest is not None:
                continue
            q = np.zeros(case["V"])
            if inp["proposal"] is None:
                q[d] = 1.0
            else:
                q = np.exp(log_softmax(inp["proposal"][off[s] + j]))
            if u[off[s] + s + j] * q[d] < np.exp(lp[d]):
                out["accepted"][s] += 1
            else:
                rest, judge = np.maximum(np.exp(lp) - q, 0.0), lp
        if rest is None:
            judge = log_softmax(inp["target"][off[s] + s + n])
            rest = np.exp(judge)
        c = np.cumsum(rest)
        v = int(np.searchsorted(c, u[off[s] + s + n] * c[-1], side="right"))
        out["next"][s] = min(v, int(np.nonzero(rest)[0][-1]))
        out["next_logp"][s] = judge[out["next"][s]]
    return out
