"""Performance cases of the operators that a training step has around a decoder's blocks.

  ce     softmax cross entropy of an output layer over its vocabulary: log probabilities of given tokens from hidden states
         and weights, and the gradients of both, without the logits
  clip   the norm over all gradients of a step, and the gradients scaled so that it stays within a bound
  snorm  the norm of a block's output, its gate, the scaled residual stream and the norm in front of the next block in one
         pass; its backward pass with the reduction of the parameters' gradients

`prepare` makes the inputs from the seed alone; `run` is one pass, in plain torch where `own` is false and through
`paper_2608_01847_amd.focus` where it is true; `exact` is the same from the definitions in 64 bits.

Definitions. Targets below zero are left out: their log probability is 0 and so is the gradient that it passes on. Clipping
multiplies by max_norm / norm where the norm is larger than max_norm and by 1 elsewhere. The second norm is that of the
residual stream Y before Y is rounded to its type.
"""
import math

import torch

own = False
DEV = "cuda"
IGNORED = -1
EPS = 1e-6


def listed():
    return [
        # one token scored over a vocabulary of 151,936: the weights' way from memory
        {"name": "ce_token", "kind": "ce", "train": False, "dtype": "bf16", "T": 1, "V": 151936, "K": 2560},
        # the label loss of a small fp32 model with a ragged batch and a vocabulary of no round size
        {"name": "ce_train_ragged_f32", "kind": "ce", "train": True, "dtype": "f32", "T": 301, "V": 5003, "K": 1008},
        # the label loss at the sizes of the end-to-end stack's head, with the gradients of hidden states and weights
        {"name": "ce_train_4k", "kind": "ce", "train": True, "dtype": "bf16", "T": 4096, "V": 32000, "K": 2560},
        # samples of odd lengths scored by an odd vocabulary
        {"name": "ce_score_odd", "kind": "ce", "train": False, "dtype": "bf16", "T": 1371, "V": 50257, "K": 4096},
        # four sequences of 2,048 over the large vocabulary, forward and backward: the largest call
        {"name": "ce_train_152k", "kind": "ce", "train": True, "dtype": "bf16", "T": 8192, "V": 151936, "K": 2560},
        # scales and coefficients of one small layer: launches and latency
        {"name": "clip_layer", "kind": "clip", "dtype": "f32", "tensors": 2, "n": 4096, "spread": 4.0, "max_norm": 1.0},
        # the gradients of a small decoder, matrices and vectors in bf16 beside fp32 ones
        {"name": "clip_many", "kind": "clip", "dtype": "mixed", "tensors": 252, "n": 2000003, "spread": 3000.0, "max_norm": 1.0},
        # scales and coefficients of the seven linears of the hidden-8192 block
        {"name": "clip_block8192", "kind": "clip", "dtype": "f32", "tensors": 14, "n": 29360128, "spread": 32.0, "max_norm": 1.0},
        # one token through a block's norms at hidden size 8,192
        {"name": "snorm_token_8192", "kind": "snorm", "train": False, "norm": "rms", "dtype": "bf16", "T": 1, "C": 8192,
         "gate": "feature", "bias": False},
        # a small fp32 layer with ragged tokens and features, a gate of its own for every token, shifts trained
        {"name": "snorm_train_ragged", "kind": "snorm", "train": True, "norm": "layer", "dtype": "f32", "T": 2037, "C": 1001,
         "gate": "token", "bias": True},
        # four sequences of 2,048 at hidden size 8,192 with gates for every token, forward and backward
        {"name": "snorm_train_8k", "kind": "snorm", "train": True, "norm": "rms", "dtype": "bf16", "T": 8192, "C": 8192,
         "gate": "token", "bias": False},
        # a calibration batch of 32 sequences of 2,048 tokens at hidden size 2,560, a learned gate, forward and backward
        {"name": "snorm_train_64k", "kind": "snorm", "train": True, "norm": "rms", "dtype": "bf16", "T": 65536, "C": 2560,
         "gate": "feature", "bias": False},
    ]


CE_FLOPS = 6.0 * 8192 * 151936 * 2560
CLIP_ELEMENTS = 115000000
SNORM_ELEMENTS = 65536 * 2560


def _log(rng, lo, hi, multiple=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(multiple, int(round(v / multiple)) * multiple)


def draw(rng):
    kind = rng.choice(["ce", "ce", "clip", "snorm"])
    if kind == "ce":
        while True:
            dtype, train = rng.choice(["bf16", "bf16", "bf16", "f32"]), rng.random() < 0.6
            f32 = dtype == "f32"
            case = {"kind": kind, "train": train, "dtype": dtype, "T": _log(rng, 1, 1024 if f32 else 8192),
                    "V": _log(rng, 1000, 32000 if f32 else 151936, rng.choice([1, 1, 8, 16])),
                    "K": _log(rng, 64, 2048 if f32 else 8192, rng.choice([16, 64]))}
            if work(case)["flops"] * (16 if f32 else 1) <= CE_FLOPS:
                return case
    if kind == "clip":
        while True:
            case = {"kind": kind, "dtype": rng.choice(["f32", "bf16", "mixed"]), "tensors": _log(rng, 1, 600),
                    "n": _log(rng, 64, 30000000), "spread": float(_log(rng, 1, 3000)), "max_norm": rng.choice([0.1, 1.0, 1e6])}
            if sum(n for n, _ in _clip_sizes(case)) <= CLIP_ELEMENTS:
                return case
    while True:
        T, C = _log(rng, 1, 65536), _log(rng, 64, 8192, rng.choice([1, 8, 64]))
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if T * C * (2 if dtype == "f32" else 1) <= SNORM_ELEMENTS:
            break
    norm = rng.choice(["layer", "rms", "rms"])
    return {"kind": kind, "train": rng.random() < 0.6, "norm": norm, "dtype": dtype, "T": T, "C": C,
            "gate": rng.choice(["none", "feature", "token"]), "bias": norm == "layer" and rng.random() < 0.7}


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


def _clip_sizes(case):
    """[(elements, dtype)]: the tensors' sizes lie between n / spread and n, evenly in their logarithm; the first is n."""
    k, n, spread = case["tensors"], case["n"], case["spread"]
    kinds = {"f32": [torch.float32], "bf16": [torch.bfloat16], "mixed": [torch.bfloat16, torch.bfloat16, torch.float32]}
    sizes = [max(1, int(n * spread ** (-i / max(1, k - 1)))) for i in range(k)]
    d = kinds[case["dtype"]]
    return [(m, d[i % len(d)]) for i, m in enumerate(sizes)]


def _inputs(case, seed):
    kind = case["kind"]
    g = _gen(seed, {"ce": 11, "clip": 12, "snorm": 13}[kind])
    if kind == "ce":
        dt, T, V, K = _dtype(case), case["T"], case["V"], case["K"]
        W = _randn(g, dt, V, K, scale=0.02)
        target = torch.randint(0, V, (T,), generator=g, device=DEV)
        # hidden states that know their token more or less: its logit is raised by 0 to 14 over the others' spread
        raised = 14.0 * torch.rand(T, 1, generator=g, device=DEV) / (0.0004 * K)
        X = torch.empty(T, K, dtype=dt, device=DEV)
        for r in range(0, T, 4096):
            e = slice(r, min(T, r + 4096))
            X[e] = torch.randn(e.stop - r, K, generator=g, device=DEV) + raised[e] * W[target[e]].float()
        target[torch.rand(T, generator=g, device=DEV) < 0.05] = IGNORED
        x = {"X": X, "W": W, "target": target}
        if case["train"]:
            x["d_logp"] = torch.full((T,), -1.0 / T, device=DEV)
        return x
    if kind == "clip":
        sizes = _clip_sizes(case)
        # gradients of tensors differ by orders of magnitude
        mag = 10.0 ** (-1.0 - 4.0 * torch.rand(len(sizes), generator=g, device=DEV)).cpu()
        return {"grads": [_randn(g, dt, n, scale=float(m)) for (n, dt), m in zip(sizes, mag)]}
    dt, T, C = _dtype(case), case["T"], case["C"]
    ch = 1.0 + 19.0 * (torch.rand(C, generator=g, device=DEV) < 0.01)
    gain = lambda: (1.0 + 0.2 * torch.randn(C, generator=g, device=DEV)).to(dt)  # noqa: E731
    shift = lambda: (0.1 * torch.randn(C, generator=g, device=DEV)).to(dt) if case["bias"] else None  # noqa: E731
    x = {"X": _randn(g, dt, T, C).mul_(ch.to(dt)), "B": _randn(g, dt, T, C, scale=0.3), "w_post": gain(), "w_pre": gain(),
         "b_post": shift(), "b_pre": shift()}
    x["gate"] = None
    if case["gate"] == "feature":
        x["gate"] = (0.5 + 0.2 * torch.randn(C, generator=g, device=DEV)).to(dt)
    elif case["gate"] == "token":
        x["gate"] = _randn(g, dt, T, C).sigmoid_()
    if case["train"]:
        x["dN"], x["dY"] = _randn(g, dt, T, C), _randn(g, dt, T, C, scale=0.5)
    return x


SCALE = 0.8  # of the residual stream


def prepare(case, seed):
    st = {"case": case, **_inputs(case, seed)}
    if case["kind"] == "clip":
        # a buffer per type, the tensors behind one another at 16-byte places
        flat, st["out"] = {}, []
        for dt in sorted({d for _, d in _clip_sizes(case)}, key=str):
            flat[dt] = torch.zeros(sum((n + 7) // 8 * 8 for n, d in _clip_sizes(case) if d == dt), dtype=dt, device=DEV)
        at = {dt: 0 for dt in flat}
        for n, dt in _clip_sizes(case):
            st["out"].append(flat[dt][at[dt]:at[dt] + n])
            at[dt] += (n + 7) // 8 * 8
        st["flat"] = [flat[dt] for dt in sorted(flat, key=str)]
    if own:
        from paper_2608_01847_amd import focus as F
        st["F"] = F
        if case["kind"] == "ce":
            st["ws"] = F.workspace(F.linear_ce_workspace_size(case["T"], case["V"], case["K"], backward=case["train"]))
        elif case["kind"] == "clip":
            st["plan"] = F.GradTensors(st["grads"], st["out"])
            st["ws"] = F.workspace(F.clip_grad_norm_workspace_size(len(st["grads"])))
        else:
            st["ws"] = F.workspace(F.sandwich_norm_workspace_size(case["T"], case["C"]))
    return st


# ---- one pass ---------------------------------------------------------------------------------------
def run(st):
    return (_own if own else _plain)[st["case"]["kind"]](st, st["case"])


def _own_ce(st, case):
    F, ws = st["F"], st["ws"]
    logp, lse = F.linear_ce_fwd(st["X"], st["W"], st["target"], ws=ws)
    out = {"logp": logp, "lse": lse}
    if case["train"]:
        out["dX"], out["dW"] = F.linear_ce_bwd(st["X"], st["W"], st["target"], lse, st["d_logp"], ws=ws)
    return out


def _own_clip(st, case):
    norm = st["F"].clip_grad_norm(st["plan"], case["max_norm"], ws=st["ws"])
    return {"norm": norm, "grads": st["flat"]}


def _own_snorm(st, case):
    F, ws = st["F"], st["ws"]
    kind = F.NORM_LAYER if case["norm"] == "layer" else F.NORM_RMS
    args = dict(b_post=st["b_post"], b_pre=st["b_pre"], gate=st["gate"], residual_scale=SCALE, kind=kind, ws=ws)
    Y, N, stats = F.sandwich_norm_fwd(st["X"], st["B"], st["w_post"], st["w_pre"], eps=EPS, **args)
    out = {"Y": Y, "N": N}
    if case["train"]:
        dX, dB, grads = F.sandwich_norm_bwd(st["dN"], st["dY"], st["X"], st["B"], st["w_post"], st["w_pre"], stats, **args)
        out.update(dX=dX, dB=dB, **{"d" + name: g for name, g in grads.items() if g is not None})
    return out


_own = {"ce": _own_ce, "clip": _own_clip, "snorm": _own_snorm}


def _plain_ce(st, case):
    X, W, target = st["X"].float(), st["W"].float(), st["target"]
    Z = X @ W.t()
    m = Z.amax(1, keepdim=True)
    lse = m + (Z - m).exp().sum(1, keepdim=True).log()
    used, at = (target >= 0)[:, None], target.clamp(min=0)[:, None]
    zero = torch.zeros_like(lse)
    out = {"logp": torch.where(used, Z.gather(1, at) - lse, zero)[:, 0], "lse": lse[:, 0]}
    if case["train"]:
        g = torch.where(used, st["d_logp"][:, None], zero)
        D = Z.sub_(lse).exp_().mul_(-g)
        D.scatter_add_(1, at, g)
        out["dX"], out["dW"] = (D @ W).to(st["X"].dtype), (D.t() @ X).to(st["W"].dtype)
    return out


def _plain_clip(st, case):
    norm = torch.stack([g.double().square().sum() for g in st["grads"]]).sum().sqrt()
    scale = (case["max_norm"] / norm).clamp(max=1.0).float()
    [o.copy_(g.float() * scale) for g, o in zip(st["grads"], st["out"])]
    return {"norm": norm[None], "grads": st["flat"]}


def _normed(H, layer):
    """(H - mean) rstd over the features and rstd, in H's own precision."""
    c = H - H.mean(1, keepdim=True) if layer else H
    rstd = 1.0 / ((c * c).mean(1, keepdim=True) + EPS).sqrt()
    return c * rstd, rstd


def _norm_grad(g, xh, rstd, layer):
    d = g - xh * (g * xh).mean(1, keepdim=True)
    return rstd * (d - g.mean(1, keepdim=True) if layer else d)


def _plain_snorm(st, case):
    dt, layer = _dtype(case), case["norm"] == "layer"
    f = {k: None if st[k] is None else st[k].float() for k in ("w_post", "w_pre", "b_post", "b_pre", "gate")}
    xh1, rstd1 = _normed(st["B"].float(), layer)
    U = xh1 * f["w_post"]
    if case["bias"]:
        U = U + f["b_post"]
    gate = 1.0 if f["gate"] is None else f["gate"]
    Y = SCALE * st["X"].float() + gate * U
    xh2, rstd2 = _normed(Y, layer)
    N = xh2 * f["w_pre"]
    if case["bias"]:
        N = N + f["b_pre"]
    out = {"Y": Y.to(dt), "N": N.to(dt)}
    if case["train"]:
        dN = st["dN"].float()
        dY = st["dY"].float() + _norm_grad(dN * f["w_pre"], xh2, rstd2, layer)
        dU = dY * gate
        out["dX"] = (SCALE * dY).to(dt)
        out["dB"] = _norm_grad(dU * f["w_post"], xh1, rstd1, layer).to(dt)
        out["dw_post"], out["dw_pre"] = (dU * xh1).sum(0), (dN * xh2).sum(0)
        if case["bias"]:
            out["db_post"], out["db_pre"] = dU.sum(0), dN.sum(0)
        if case["gate"] == "feature":
            out["dgate"] = (dY * U).sum(0)
        elif case["gate"] == "token":
            out["dgate"] = (dY * U).to(dt)
    return out


_plain = {"ce": _plain_ce, "clip": _plain_clip, "snorm": _plain_snorm}


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    if case["kind"] == "ce":
        T, V, K = case["T"], case["V"], case["K"]
        e, train = 4.0 if case["dtype"] == "f32" else 2.0, case["train"]
        # X and W read, their gradients written; the logits' product, and one for each gradient
        return {"bytes": e * (T + V) * K * (2 if train else 1) + 16.0 * T, "flops": (6.0 if train else 2.0) * T * V * K}
    if case["kind"] == "clip":
        # read for the norm, read and written to be scaled
        return {"bytes": 3.0 * sum(n * (4 if d == torch.float32 else 2) for n, d in _clip_sizes(case)), "flops": 0.0}
    e, T, C = 4.0 if case["dtype"] == "f32" else 2.0, case["T"], case["C"]
    rows = 4 + (case["gate"] == "token")  # X, B read, Y, N written
    if case["train"]:
        rows += 4 + (case["gate"] == "token")  # dN, dY read, dX, dB written
    return {"bytes": e * T * C * rows + 20.0 * C, "flops": 0.0}


# ---- the same in 64 bits ----------------------------------------------------------------------------
def _exact_ce(case, x):
    T, V, K = case["T"], case["V"], case["K"]
    f64 = dict(dtype=torch.float64, device=DEV)
    W = x["W"].double()
    out = {"logp": torch.zeros(T, **f64), "lse": torch.zeros(T, **f64)}
    if case["train"]:
        out.update(dX=torch.zeros(T, K, **f64), dW=torch.zeros(V, K, **f64))
    for r in range(0, T, 2048):
        e = slice(r, min(T, r + 2048))
        X = x["X"][e].double()
        z = torch.mm(X, W.t())
        lse = torch.logsumexp(z, 1)
        t = x["target"][e]
        kept = torch.nonzero(t >= 0)[:, 0]
        out["lse"][e] = lse
        out["logp"][r + kept] = z[kept, t[kept]] - lse[kept]
        if case["train"]:
            g = torch.zeros(e.stop - r, **f64)
            g[kept] = x["d_logp"][e].double()[kept]
            D = torch.softmax(z, 1).mul_(-g[:, None])
            D[kept, t[kept]] += g[kept]
            out["dX"][e] = torch.mm(D, W)
            out["dW"].addmm_(D.t(), X)
    return out


def _exact_clip(case, x):
    total = sum(float(g.double().square().sum()) for g in x["grads"])
    norm = math.sqrt(total)
    scale = case["max_norm"] / norm if norm > case["max_norm"] else 1.0
    flat = []
    for dt in sorted({g.dtype for g in x["grads"]}, key=str):
        parts = []
        for g in x["grads"]:
            if g.dtype == dt:
                parts += [g.double() * scale, torch.zeros(-g.numel() % 8, dtype=torch.float64, device=DEV)]
        flat.append(torch.cat(parts))
    return {"norm": torch.tensor([norm], dtype=torch.float64, device=DEV), "grads": flat}


def _exact_snorm(case, x):
    T, C, dt, train = case["T"], case["C"], _dtype(case), case["train"]
    wide = torch.float32 if T * C > 1 << 26 else torch.float64  # what whole tensors are returned in, where they are large
    names = ["w_post", "w_pre"] + (["b_post", "b_pre"] if case["bias"] else []) + (["gate"] if case["gate"] == "feature" else [])
    p = {n: x[n].double().requires_grad_(train) for n in names}
    out = {n: torch.empty(T, C, dtype=wide, device=DEV) for n in ("Y", "N") + (("dX", "dB") if train else ())}
    if train and case["gate"] == "token":
        out["dgate"] = torch.empty(T, C, dtype=wide, device=DEV)
    sums = {n: torch.zeros(C, dtype=torch.float64, device=DEV) for n in names}

    def norm(h):
        c = h - h.mean(1, keepdim=True) if case["norm"] == "layer" else h
        return c / torch.sqrt(c.square().mean(1, keepdim=True) + EPS)

    for r in range(0, T, 8192):
        e = slice(r, min(T, r + 8192))
        leaf = {n: x[n][e].double().requires_grad_(train) for n in ("X", "B")}
        if case["gate"] == "token":
            leaf["gate"] = x["gate"][e].double().requires_grad_(train)
        u = norm(leaf["B"]) * p["w_post"]
        u = u + p["b_post"] if case["bias"] else u
        gate = leaf.get("gate", p.get("gate"))
        y = SCALE * leaf["X"] + (u if gate is None else gate * u)
        n = norm(y) * p["w_pre"]
        n = n + p["b_pre"] if case["bias"] else n
        out["Y"][e], out["N"][e] = y.detach(), n.detach()
        if train:
            wrt = list(leaf.values()) + list(p.values())
            grads = torch.autograd.grad([n, y], wrt, [x["dN"][e].double(), x["dY"][e].double()])
            for k, v in zip(leaf, grads):
                out["d" + k][e] = v
            for k, v in zip(p, grads[len(leaf):]):
                sums[k] += v
    if train:
        out.update({"d" + k: v for k, v in sums.items()})
    return out


def exact(case, seed):
    x = _inputs(case, seed)
    return {"ce": _exact_ce, "clip": _exact_clip, "snorm": _exact_snorm}[case["kind"]](case, x)
