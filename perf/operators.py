"""Performance cases of the operators that an end-to-end calibration of a decoder has around its linears.

  norm   layer norm and RMS norm over the features of a token, with the residual sum in front of it;
         its backward pass with the reduction of the gradients of gain and shift
  attn   attention over whole prompts: packed sequences of different lengths, shared key-value heads,
         causal or not, queries that are the end of longer keys; its backward pass
  logp   log probabilities of given tokens, entropy and the largest alternatives of a row of logits;
         its backward pass to the logits

`prepare` makes the inputs from the seed alone; `run` is one pass, in plain torch where `own` is false
and through `paper_2608_01847_amd.focus` where it is true; `exact` is the same from the definitions in
64 bits.

Definitions. H is the input of a norm: X, or X + R rounded to X's type. A causal query attends to the keys
up to its own place, the last query standing at the last key. Targets below zero are left out: their
log probability is 0 and so is the gradient that it passes on. Equal logits are ranked by their index.
"""
import math

import torch

own = False
DEV = "cuda"
IGNORED = -1


def listed():
    return [
        # one token of a model of hidden size 8,192: the residual sum and the norm in front of a linear
        {"name": "norm_token_8192", "kind": "norm", "train": False, "norm": "rms", "dtype": "bf16", "T": 1, "C": 8192,
         "residual": True, "bias": False},
        # a small fp32 layer with ragged tokens and features, gain and shift trained
        {"name": "norm_train_ragged", "kind": "norm", "train": True, "norm": "layer", "dtype": "f32", "T": 2037, "C": 1001,
         "residual": False, "bias": True},
        # a calibration batch of 32 sequences of 2,048 tokens at hidden size 2,560, forward and backward
        {"name": "norm_train_64k", "kind": "norm", "train": True, "norm": "rms", "dtype": "bf16", "T": 65536, "C": 2560,
         "residual": True, "bias": False},
        # one new token scored against a prompt of 8,192 (32 query heads on 8 key-value heads)
        {"name": "attn_last_token", "kind": "attn", "train": False, "dtype": "bf16", "Hq": 32, "Hkv": 8, "D": 128,
         "causal": True, "q": "1", "k": "8192"},
        # samples of different lengths packed without padding, scored
        {"name": "attn_packed", "kind": "attn", "train": False, "dtype": "bf16", "Hq": 32, "Hkv": 8, "D": 128, "causal": True,
         "q": "2048,1,1531,64,700,2048,333,17,1024,1999,128,905,250,1100,2047,65,481,3,1280,599", "k": ""},
        # one long document
        {"name": "attn_long_16k", "kind": "attn", "train": False, "dtype": "bf16", "Hq": 32, "Hkv": 8, "D": 128,
         "causal": True, "q": "16384", "k": ""},
        # a small fp32 encoder-like layer, no mask, ragged, forward and backward
        {"name": "attn_train_f32", "kind": "attn", "train": True, "dtype": "f32", "Hq": 8, "Hkv": 8, "D": 64, "causal": False,
         "q": "300,129,1,77,256,31", "k": ""},
        # four sequences of 2,048 with the heads of the hidden-8,192 block, forward and backward
        {"name": "attn_train_8k", "kind": "attn", "train": True, "dtype": "bf16", "Hq": 64, "Hkv": 8, "D": 128, "causal": True,
         "q": ",".join(["2048"] * 4), "k": ""},
        # a calibration batch of 32 sequences of 2,048 with the heads of the hidden-2,560 block, forward and backward
        {"name": "attn_train_64k", "kind": "attn", "train": True, "dtype": "bf16", "Hq": 32, "Hkv": 8, "D": 128,
         "causal": True, "q": ",".join(["2048"] * 32), "k": ""},
        # the logits of one token over a vocabulary of 151,936, with 20 alternatives
        {"name": "logp_token", "kind": "logp", "train": False, "dtype": "bf16", "T": 1, "V": 151936, "top": 20},
        # four scored sequences of 2,048
        {"name": "logp_score_8k", "kind": "logp", "train": False, "dtype": "bf16", "T": 8192, "V": 151936, "top": 5},
        # the cross entropy of the end-to-end stack's head at its own sizes, with an entropy term, forward and backward
        {"name": "logp_train_32k", "kind": "logp", "train": True, "dtype": "bf16", "T": 4096, "V": 32000, "top": 0},
    ]


NORM_ELEMENTS = 65536 * 2560
LOGP_ELEMENTS = 8192 * 151936


def _log(rng, lo, hi, multiple=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(multiple, int(round(v / multiple)) * multiple)


def draw(rng):
    kind = rng.choice(["norm", "attn", "attn", "logp"])
    if kind == "norm":
        while True:
            T, C = _log(rng, 1, 65536), _log(rng, 64, 8192, rng.choice([1, 8, 64]))
            dtype = rng.choice(["bf16", "bf16", "f32"])
            if T * C * (2 if dtype == "f32" else 1) <= NORM_ELEMENTS:
                break
        norm = rng.choice(["layer", "rms"])
        return {"kind": kind, "train": rng.random() < 0.6, "norm": norm, "dtype": dtype, "T": T, "C": C,
                "residual": rng.random() < 0.5, "bias": norm == "layer" and rng.random() < 0.7}
    if kind == "logp":
        while True:
            T, V = _log(rng, 1, 16384), _log(rng, 1000, 151936, rng.choice([1, 1, 8, 16]))
            dtype, train = rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.5
            if T * V * (2 if dtype == "f32" else 1) * (2 if train else 1) <= LOGP_ELEMENTS:
                break
        return {"kind": kind, "train": train, "dtype": dtype, "T": T, "V": V, "top": rng.choice([0, 1, 5, 20, 50])}
    while True:
        dtype, train = rng.choice(["bf16", "bf16", "bf16", "bf16", "f32"]), rng.random() < 0.6
        f32 = dtype == "f32"
        Hkv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8])
        n, longest = _log(rng, 1, 8 if f32 else 48), _log(rng, 64, 1024 if f32 else 16384)
        shortest = rng.choice([1, max(1, longest // 3)])
        q = [_log(rng, shortest, longest) for _ in range(n)]
        k = []
        if rng.random() < 0.3:  # queries that are the end of longer keys
            k = [a + _log(rng, 1, longest) for a in q]
            if rng.random() < 0.3:
                q = [1] * n
        case = {"kind": kind, "train": train, "dtype": dtype, "Hq": Hkv * group, "Hkv": Hkv,
                "D": rng.choice([64, 128, 128, 128, 96, 80, 40]), "causal": bool(k) or rng.random() < 0.8,
                "q": ",".join(map(str, q)), "k": ",".join(map(str, k))}
        if work(case)["flops"] <= (2e10 if f32 else 2e12) and max(sum(q), sum(k)) <= 65536 and Hkv * group <= 64:
            return case


# ---- inputs -----------------------------------------------------------------------------------------
def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + tag)
    return g


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _randn(g, dtype, *shape, scale=1.0):
    out = torch.empty(*shape, dtype=dtype, device=DEV)
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 27):
        n = min(1 << 27, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=g, device=DEV) * scale
    return out


def _lengths(case):
    q = [int(x) for x in case["q"].split(",")]
    return q, [int(x) for x in case["k"].split(",")] if case["k"] else q


def _ends(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _inputs(case, seed):
    dt, kind = _dtype(case), case["kind"]
    g = _gen(seed, {"norm": 1, "attn": 2, "logp": 3}[kind])
    if kind == "norm":
        T, C = case["T"], case["C"]
        # a residual stream: some channels carry most of it
        ch = 1.0 + 19.0 * (torch.rand(C, generator=g, device=DEV) < 0.01)
        x = {"X": _randn(g, dt, T, C).mul_(ch.to(dt)) if T * C else torch.empty(T, C, dtype=dt, device=DEV)}
        x["R"] = _randn(g, dt, T, C, scale=0.5) if case["residual"] else None
        x["w"] = (1.0 + 0.2 * torch.randn(C, generator=g, device=DEV)).to(dt)
        x["b"] = (0.1 * torch.randn(C, generator=g, device=DEV)).to(dt) if case["bias"] else None
        if case["train"]:
            x["dY"] = _randn(g, dt, T, C)
            x["dR"] = _randn(g, dt, T, C, scale=0.5) if case["residual"] else None
        return x
    if kind == "attn":
        lq, lk = _lengths(case)
        tq, tk, Hq, Hkv, D = sum(lq), sum(lk), case["Hq"], case["Hkv"], case["D"]
        x = {"q": _randn(g, dt, tq, Hq, D, scale=1.5), "k": _randn(g, dt, tk, Hkv, D, scale=1.2),
             "v": _randn(g, dt, tk, Hkv, D)}
        if case["train"]:
            x["dO"] = _randn(g, dt, tq, Hq, D)
        return x
    T, V = case["T"], case["V"]
    x = {"Z": _randn(g, dt, T, V, scale=2.5)}
    x["target"] = torch.randint(0, V, (T,), generator=g, device=DEV)
    x["target"][torch.rand(T, generator=g, device=DEV) < 0.05] = IGNORED
    if case["train"]:
        x["d_logp"] = torch.full((T,), -1.0 / T, device=DEV)
        x["d_entropy"] = (0.1 / T) * torch.rand(T, generator=g, device=DEV)
    return x


def prepare(case, seed):
    st = {"case": case, **_inputs(case, seed)}
    kind = case["kind"]
    if kind == "attn":
        lq, lk = _lengths(case)
        st["cu_q"] = torch.tensor(_ends(lq), dtype=torch.int32, device=DEV)
        st["cu_k"] = torch.tensor(_ends(lk), dtype=torch.int32, device=DEV) if case["k"] else st["cu_q"]
        st["ends"] = (_ends(lq), _ends(lk))
    if own:
        from paper_2608_01847_amd import focus as F
        st["F"] = F
        if kind == "norm":
            st["ws"] = F.workspace(F.norm_workspace_size(case["T"], case["C"]))
        elif kind == "attn":
            st["ws"] = F.workspace(F.attention_workspace_size(st["q"], st["k"], len(lq)))
        else:
            st["ws"] = F.workspace(F.token_logprobs_workspace_size(case["T"], case["V"], case["top"]))
    return st


# ---- one pass ---------------------------------------------------------------------------------------
def run(st):
    return (_own if own else _plain)[st["case"]["kind"]](st, st["case"])


def _own_norm(st, case):
    F, ws = st["F"], st["ws"]
    kind, eps = F.NORM_LAYER if case["norm"] == "layer" else F.NORM_RMS, 1e-6
    Y, H, mean, rstd = F.norm_fwd(st["X"], st["w"], st["b"], st["R"], kind, eps, ws=ws)
    out = {"Y": Y}
    if case["residual"]:
        out["H"] = H
    if case["train"]:
        dX, dw, db = F.norm_bwd(st["dY"], H if case["residual"] else st["X"], st["w"], mean, rstd, st["dR"], kind,
                                want_bias=case["bias"], ws=ws)
        out["dX"], out["dw"] = dX, dw
        if case["bias"]:
            out["db"] = db
    return out


def _own_attn(st, case):
    F, ws = st["F"], st["ws"]
    args = (st["cu_q"], st["cu_k"], case["causal"])
    O, lse = F.attention_fwd(st["q"], st["k"], st["v"], *args, ws=ws)
    out = {"O": O, "lse": lse}
    if case["train"]:
        out["dq"], out["dk"], out["dv"] = F.attention_bwd(st["dO"], st["q"], st["k"], st["v"], O, lse, *args, ws=ws)
    return out


def _own_logp(st, case):
    F, ws = st["F"], st["ws"]
    logp, entropy, lse, top_logp, top_index = F.token_logprobs(st["Z"], st["target"], case["top"], ws=ws)
    out = {"logp": logp, "entropy": entropy, "lse": lse}
    if case["top"]:
        out["top_logp"], out["top_index"] = top_logp, top_index
    if case["train"]:
        out["dZ"] = F.token_logprobs_bwd(st["Z"], st["target"], lse, entropy, st["d_logp"], st["d_entropy"], ws=ws)
    return out


_own = {"norm": _own_norm, "attn": _own_attn, "logp": _own_logp}


def _plain_norm(st, case):
    dt, eps = _dtype(case), 1e-6
    H = (st["X"].float() + st["R"].float()).to(dt) if case["residual"] else st["X"]
    h, w = H.float(), st["w"].float()
    if case["norm"] == "layer":
        d = h - h.mean(1, keepdim=True)
    else:
        d = h
    rstd = 1.0 / ((d * d).mean(1, keepdim=True) + eps).sqrt()
    xh = d * rstd
    y = xh * w
    if case["bias"]:
        y = y + st["b"].float()
    out = {"Y": y.to(dt)}
    if case["residual"]:
        out["H"] = H
    if case["train"]:
        dy = st["dY"].float()
        gy = dy * w
        dx = gy - xh * (gy * xh).mean(1, keepdim=True)
        if case["norm"] == "layer":
            dx = dx - gy.mean(1, keepdim=True)
        dx = dx * rstd
        if case["residual"]:
            dx = dx + st["dR"].float()
        out["dX"], out["dw"] = dx.to(dt), (dy * xh).sum(0)
        if case["bias"]:
            out["db"] = dy.sum(0)
    return out


def _head_step(lq, lk, group):
    """Key-value heads taken together, so that one matrix of scores stays near 2^28 elements."""
    return max(1, (1 << 28) // max(1, lq * lk * group))


def _plain_attn(st, case):
    dt, Hq, Hkv, D = _dtype(case), case["Hq"], case["Hkv"], case["D"]
    G, scale = Hq // Hkv, 1.0 / math.sqrt(D)
    q, k, v = st["q"], st["k"], st["v"]
    O, lse = torch.empty_like(q), torch.empty(Hq, q.shape[0], dtype=torch.float32, device=DEV)
    train = case["train"]
    if train:
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    eq, ek = st["ends"]
    for s in range(len(eq) - 1):
        a, b, c, d = eq[s], eq[s + 1], ek[s], ek[s + 1]
        lq, lk = b - a, d - c
        hide = None
        if case["causal"]:
            hide = torch.arange(lk, device=DEV)[None, :] > torch.arange(lq, device=DEV)[:, None] + (lk - lq)
        step = _head_step(lq, lk, G)
        for h in range(0, Hkv, step):
            n = min(step, Hkv - h)
            hs = slice(h * G, (h + n) * G)
            # [n][G lq][D] against [n][lk][D]
            qs = q[a:b, hs].float().view(lq, n, G, D).permute(1, 2, 0, 3).reshape(n, G * lq, D)
            ks = k[c:d, h:h + n].float().permute(1, 0, 2).contiguous()
            vs = v[c:d, h:h + n].float().permute(1, 0, 2).contiguous()
            S = torch.bmm(qs, ks.transpose(1, 2).contiguous()).view(n, G, lq, lk) * scale
            if hide is not None:
                S.masked_fill_(hide, -math.inf)
            m = S.amax(3, keepdim=True)
            P = (S - m).exp()
            l = P.sum(3, keepdim=True)
            P = P / l
            o = torch.bmm(P.view(n, G * lq, lk), vs)
            O[a:b, hs] = o.view(n, G, lq, D).permute(2, 0, 1, 3).reshape(lq, n * G, D).to(dt)
            lse[hs, a:b] = (m + l.log()).view(n * G, lq)
            if train:
                do = st["dO"][a:b, hs].float().view(lq, n, G, D).permute(1, 2, 0, 3).reshape(n, G * lq, D)
                dP = torch.bmm(do, vs.transpose(1, 2).contiguous()).view(n, G, lq, lk)
                delta = (do * o).sum(2).view(n, G, lq, 1)
                dS = (P * (dP - delta) * scale).view(n, G * lq, lk)
                dq[a:b, hs] = torch.bmm(dS, ks).view(n, G, lq, D).permute(2, 0, 1, 3).reshape(lq, n * G, D).to(dt)
                dk[c:d, h:h + n] = torch.bmm(dS.transpose(1, 2).contiguous(), qs).permute(1, 0, 2).to(dt)
                dv[c:d, h:h + n] = torch.bmm(P.view(n, G * lq, lk).transpose(1, 2).contiguous(), do).permute(1, 0, 2).to(dt)
    out = {"O": O, "lse": lse}
    if train:
        out.update(dq=dq, dk=dk, dv=dv)
    return out


def _plain_logp(st, case):
    T, V, top, Z, target = case["T"], case["V"], case["top"], st["Z"], st["target"]
    f32 = dict(dtype=torch.float32, device=DEV)
    out = {"logp": torch.empty(T, **f32), "entropy": torch.empty(T, **f32), "lse": torch.empty(T, **f32)}
    if top:
        out["top_logp"] = torch.empty(T, top, **f32)
        out["top_index"] = torch.empty(T, top, dtype=torch.int32, device=DEV)
    if case["train"]:
        out["dZ"] = torch.empty_like(Z)
    index = torch.arange(V, device=DEV)
    for r in range(0, T, 2048):
        e = slice(r, min(T, r + 2048))
        z = Z[e].float()
        m = z.amax(1, keepdim=True)
        lse = m + (z - m).exp().sum(1, keepdim=True).log()
        lp = z - lse
        p = lp.exp()
        entropy = -(p * lp).sum(1, keepdim=True)
        used = (target[e] >= 0)[:, None]
        at = target[e].clamp(min=0)[:, None]
        out["lse"][e], out["entropy"][e] = lse[:, 0], entropy[:, 0]
        out["logp"][e] = torch.where(used, lp.gather(1, at), torch.zeros_like(lse))[:, 0]
        if top:
            # whole numbers in the order of the logits, lower indexes above higher ones where logits are equal
            bits = (z + 0.0).view(torch.int32).long()
            key = (torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) << 32) + (V - 1 - index)
            for j in range(top):
                best = key.amax(1, keepdim=True)
                i = V - 1 - (best & 0xFFFFFFFF)
                out["top_index"][e, j] = i[:, 0].int()
                out["top_logp"][e, j] = lp.gather(1, i)[:, 0]
                key.scatter_(1, i, torch.iinfo(torch.int64).min)
        if case["train"]:
            gl = torch.where(used, st["d_logp"][e][:, None], torch.zeros_like(lse))
            dz = -p * (gl + st["d_entropy"][e][:, None] * (lp + entropy))
            dz.scatter_add_(1, at, gl)
            out["dZ"][e] = dz.to(Z.dtype)
    return out


_plain = {"norm": _plain_norm, "attn": _plain_attn, "logp": _plain_logp}


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    e = 4.0 if case["dtype"] == "f32" else 2.0
    if case["kind"] == "norm":
        T, C = case["T"], case["C"]
        tensors = 4 if case["residual"] else 2  # X, R read, H, Y written
        if case["train"]:
            tensors += 3 if case["residual"] else 2  # dY, dR read, dX written
        return {"bytes": e * T * C * tensors + 4.0 * C, "flops": 0.0}
    if case["kind"] == "logp":
        T, V = case["T"], case["V"]
        return {"bytes": e * T * V * (2 if case["train"] else 1) + 20.0 * T + 8.0 * T * case["top"], "flops": 0.0}
    lq, lk = _lengths(case)
    pairs = 0
    for a, b in zip(lq, lk):
        pairs += a * (b - a) + a * (a + 1) // 2 if case["causal"] else a * b
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    size = e * D * (2 * sum(lq) * Hq + 2 * sum(lk) * Hkv)
    flops = 4.0 * pairs * Hq * D
    if case["train"]:  # dO read, dq, dk, dv written; five products more
        size += e * D * (2 * sum(lq) * Hq + 2 * sum(lk) * Hkv)
        flops += 10.0 * pairs * Hq * D
    return {"bytes": size + 4.0 * Hq * sum(lq), "flops": flops}


# ---- the same in 64 bits ----------------------------------------------------------------------------
def _exact_norm(case, x):
    T, C, dt = case["T"], case["C"], _dtype(case)
    big = T * C > 1 << 27
    wide = torch.float32 if big else torch.float64  # what whole tensors are returned in, where they are large
    out = {"Y": torch.empty(T, C, dtype=wide, device=DEV)}
    if case["residual"]:
        out["H"] = torch.empty(T, C, dtype=wide, device=DEV)
    w = x["w"].double().requires_grad_(case["train"])
    b = x["b"].double().requires_grad_(case["train"]) if case["bias"] else None
    if case["train"]:
        out["dX"] = torch.empty(T, C, dtype=wide, device=DEV)
        dw = torch.zeros(C, dtype=torch.float64, device=DEV)
        db = torch.zeros(C, dtype=torch.float64, device=DEV)
    for r in range(0, T, 8192):
        e = slice(r, min(T, r + 8192))
        h = x["X"][e].double()
        if case["residual"]:
            h = (h + x["R"][e].double()).to(dt).double()
            out["H"][e] = h
        h.requires_grad_(case["train"])
        c = h - h.mean(1, keepdim=True) if case["norm"] == "layer" else h
        y = c / torch.sqrt(c.square().mean(1, keepdim=True) + 1e-6) * w
        y = y + b if b is not None else y
        out["Y"][e] = y.detach()
        if case["train"]:
            wrt = [h, w] + ([b] if b is not None else [])
            grads = torch.autograd.grad(y, wrt, x["dY"][e].double())
            out["dX"][e] = grads[0] + x["dR"][e].double() if case["residual"] else grads[0]
            dw += grads[1]
            if b is not None:
                db += grads[2]
    if case["train"]:
        out["dw"] = dw
        if b is not None:
            out["db"] = db
    return out


def _exact_attn(case, x):
    Hq, Hkv, D, train = case["Hq"], case["Hkv"], case["D"], case["train"]
    G = Hq // Hkv
    lq, lk = _lengths(case)
    eq, ek = _ends(lq), _ends(lk)
    f64 = dict(dtype=torch.float64, device=DEV)
    out = {"O": torch.zeros(eq[-1], Hq, D, **f64), "lse": torch.zeros(Hq, eq[-1], **f64)}
    if train:
        out.update(dq=torch.zeros(eq[-1], Hq, D, **f64), dk=torch.zeros(ek[-1], Hkv, D, **f64),
                   dv=torch.zeros(ek[-1], Hkv, D, **f64))
    for s in range(len(lq)):
        rq, rk = slice(eq[s], eq[s + 1]), slice(ek[s], ek[s + 1])
        seen = None
        if case["causal"]:
            seen = torch.ones(lq[s], lk[s], dtype=torch.bool, device=DEV).tril(lk[s] - lq[s])
        for h in range(Hq):
            q = x["q"][rq, h].double().requires_grad_(train)
            k = x["k"][rk, h // G].double().requires_grad_(train)
            v = x["v"][rk, h // G].double().requires_grad_(train)
            S = torch.mm(q, k.t()) / math.sqrt(D)
            if seen is not None:
                S = S.masked_fill(~seen, -math.inf)
            o = torch.mm(torch.softmax(S, 1), v)
            out["O"][rq, h] = o.detach()
            out["lse"][h, rq] = torch.logsumexp(S.detach(), 1)
            if train:
                dq, dk, dv = torch.autograd.grad(o, [q, k, v], x["dO"][rq, h].double())
                out["dq"][rq, h] = dq
                out["dk"][rk, h // G] += dk
                out["dv"][rk, h // G] += dv
    return out


def _exact_logp(case, x):
    T, V, top = case["T"], case["V"], case["top"]
    f64 = dict(dtype=torch.float64, device=DEV)
    out = {"logp": torch.zeros(T, **f64), "entropy": torch.zeros(T, **f64), "lse": torch.zeros(T, **f64)}
    if top:
        out["top_logp"] = torch.zeros(T, top, **f64)
        out["top_index"] = torch.zeros(T, top, dtype=torch.int32, device=DEV)
    if case["train"]:
        out["dZ"] = torch.empty(T, V, dtype=torch.float64 if T * V < 1 << 28 else torch.float32, device=DEV)
    for r in range(0, T, 512):
        e = slice(r, min(T, r + 512))
        z = x["Z"][e].double().requires_grad_(case["train"])
        lp = torch.log_softmax(z, 1)
        H = torch.special.entr(lp.exp()).sum(1)
        used = x["target"][e] >= 0
        logp = torch.where(used, lp.gather(1, x["target"][e].clamp(min=0)[:, None])[:, 0], torch.zeros_like(H))
        out["logp"][e], out["entropy"][e] = logp.detach(), H.detach()
        out["lse"][e] = torch.logsumexp(z.detach(), 1)
        if case["train"]:
            out["dZ"][e] = torch.autograd.grad((logp * x["d_logp"][e].double()).sum() +
                                               (H * x["d_entropy"][e].double()).sum(), z)[0]
        if top:
            order = torch.sort(x["Z"][e].float() + 0.0, dim=1, descending=True, stable=True)[1][:, :top]
            out["top_index"][e] = order.int()
            out["top_logp"][e] = lp.detach().gather(1, order)
    return out


def exact(case, seed):
    x = _inputs(case, seed)
    return {"norm": _exact_norm, "attn": _exact_attn, "logp": _exact_logp}[case["kind"]](case, x)
