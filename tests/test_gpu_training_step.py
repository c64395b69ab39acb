"""GPU tests of a training step made of norms around a block, the output layer's cross entropy, clipping and AdamW, as they are used
together: in the decoder stack, and captured into HIP graphs.

The gradient that reaches the fused q-k-v product has passed, in bf16, the output layer's backward, an input-gradient product, the
straight-through activation backwards, the norms' backward and the attention's. The reference is autograd over the same chain in
fp32, each quantisation replaced by its value with a straight-through derivative. Some ten roundings to bf16 (2^-8 at most each, 2^-9
in the mean) lie between, three of them (D, P, dS) inside sums: 5e-2 of the norm.
"""
import pytest
import torch

from gpu_common import announce, require_gpu
from test_gpu_decoder_stack import attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    return require_gpu()


@pytest.mark.parametrize("fmt", [0, 1], ids=["mx", "nv"])
@pytest.mark.parametrize("post_norm", [True, False])
def test_gradient_through_the_chain(F, fmt, post_norm):
    from paper_2608_01847_amd import calib, synth
    st = calib.DecoderStack(fmt, "crs_dgs", hidden=256, heads=(4, 2), head_dim=64, vocab=1024, lengths=(100, 1, 64, 155), k=50,
                            loss="ce", post_norm=post_norm)
    announce(f"labelled decoder stack fmt={fmt} post_norm={post_norm}")
    X = synth.activation_batch(st.w, "x", 0, st.T, device="cuda")
    target = torch.randint(0, 1024, (st.T,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    s = st.student(X, logits=False)
    assert s["Z"] is None
    loss, labels = st.label_loss(s, target)
    grads = st.backward(s, labels=labels)
    assert F.check_flags(st.ws) == F.OK

    def ste(x, x_hat, real):
        # Elements that the quantiser saturates pass no gradient. Under NVFP4 every block's largest element lies at that border
        # (|u| = 6 up to the scale's rounding), so which do is asked at the quantiser's real input: an input formed again in fp32
        # rounds to another bf16 number here and there and would turn whole elements on or off.
        m = F.fakequant_act_bwd(real, torch.ones_like(real), fmt, ws=st.ws).float()
        return x * m + (x_hat.float() - x * m).detach()

    rms = lambda h, w: h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-5) * w.float()
    qkv = s["qkv"].float().requires_grad_(True)
    Wh = s["Wh_hat"].float().requires_grad_(True)
    O = attention(*st._slices(qkv), st.cu.tolist()).flatten(1)
    Y = ste(O, s["O_hat"], s["O"].flatten(1)) @ s["Wo_hat"].float().t()
    H = X.float() + (st.gate.float() * rms(Y, st.gain["post"]) if post_norm else Y)
    Z = ste(rms(H, st.gain["out"]), s["B_hat"], s["B"]) @ Wh.t()
    ref_loss = -torch.log_softmax(Z, 1).gather(1, target[:, None]).mean()
    ref, ref_G = torch.autograd.grad(ref_loss, [qkv, Wh])
    assert abs(loss.item() - ref_loss.item()) <= 1e-2 * ref_loss.item()
    err = (grads["dqkv"].float() - ref).norm() / ref.norm()
    assert err <= 5e-2, float(err)
    # the output layer's scales and coefficients: sums over 8 to 32 elements of G, which is off by 3.9e-3 of its norm
    L = st.layers["head"]
    want = F.fakequant_bwd(ref_G, L.W, fmt, st.sb, L.s, L.c, L.alpha)
    for got, ref in zip(grads["head"], want):
        assert float((got - ref).norm() / ref.norm()) <= 2e-2


@pytest.mark.parametrize("kw", [dict(loss="ce", post_norm=True, max_grad_norm=1e-3), dict(loss="kl_top", post_norm=True),
                                dict(loss="ce")], ids=["ce-post-clip", "kl-post", "ce"])
def test_an_epoch_runs(F, kw):
    from paper_2608_01847_amd import calib
    announce(f"decoder epoch {kw}")
    vocab = 1000 if kw["loss"] == "ce" else 1024  # the input gradient from logits takes whole sixteens of them
    r = calib.decoder_epoch(0, "crs_dgs", 3, hidden=256, heads=(4, 2), head_dim=64, vocab=vocab, lengths=(100, 1, 64, 155), k=50, **kw)
    assert len(r["train_curve"]) == 3 and all(0 < x < 20 for x in r["train_curve"])
    assert set(r["eval_after"]) == {"kl_top", "nll", "entropy", "agreement"}


def test_clipping_bounds_what_the_update_reads(F):
    from paper_2608_01847_amd import calib, synth
    announce("clipped decoder step")
    make = lambda m: calib.DecoderStack(0, "crs_dgs", hidden=256, heads=(4, 2), head_dim=64, vocab=1000, lengths=(64, 65), k=50,
                                        loss="ce", max_grad_norm=m)
    free, tight = make(None), make(1e-4)
    X = synth.activation_batch(free.w, "x", 0, free.T, device="cuda")
    target = torch.randint(0, 1000, (free.T,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    norms, grads = [], []
    for st in (free, tight):
        s = st.student(X, logits=False)
        g = st.backward(s, labels=st.label_loss(s, target)[1])
        st.update(g)
        grads.append([x for n in st.layers for x in g[n]])
        norms.append(sum(float(x.double().square().sum()) for x in grads[-1]) ** 0.5)
    assert norms[0] > 1e-3 and abs(norms[1] - 1e-4) <= 1e-10
    for a, b in zip(*grads):
        assert torch.allclose(a * (1e-4 / norms[0]), b, rtol=2.0 ** -22, atol=0)


class Step:
    """Norms around a block, the output layer's loss, both backwards, clipping and AdamW on tensors that stay where they are."""

    def __init__(self, F, T, C, V, ws, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        bf = torch.bfloat16
        self.F, self.ws = F, ws
        self.X, self.B, self.W = rnd(T, C).to(bf), rnd(T, C).to(bf), (0.05 * rnd(V, C)).to(bf)
        self.w1, self.w2, self.gate = (1 + 0.1 * rnd(C)).to(bf), (1 + 0.1 * rnd(C)).to(bf), torch.sigmoid(rnd(T, C)).to(bf)
        self.target = torch.randint(0, V, (T,), generator=g, device="cuda")
        self.target[:3] = -1
        self.d = torch.full((T,), -1.0 / (T - 3), device="cuda")
        self.param, self.m, self.v = rnd(V, C), torch.zeros(V, C, device="cuda"), torch.zeros(V, C, device="cuda")
        self.dX, self.dW = torch.empty(T, C, dtype=bf, device="cuda"), torch.empty(V, C, device="cuda")
        self.norm = torch.empty(1, dtype=torch.float64, device="cuda")
        self.plan = None

    def __call__(self):
        F, ws = self.F, self.ws
        args = dict(gate=self.gate, residual_scale=0.9, kind=F.NORM_RMS, ws=ws)
        Y, N, stats = F.sandwich_norm_fwd(self.X, self.B, self.w1, self.w2, **args)
        logp, lse = F.linear_ce_fwd(N, self.W, self.target, ws=ws)
        F.linear_ce_bwd(N, self.W, self.target, lse, self.d, ws=ws, out=self.dX, dw_out=self.dW, dw_dtype=torch.float32)
        dX, dB, grads = F.sandwich_norm_bwd(self.dX, None, self.X, self.B, self.w1, self.w2, stats, **args)
        F.clip_grad_norm([self.dW, grads["w_post"], grads["w_pre"]], 1e-2, ws=ws, norm=self.norm)
        F.adamw_step(self.param, self.dW, self.m, self.v, 1, 1e-3, ws=ws)
        return [Y, N, stats, logp, lse, self.dX, self.dW, dX, dB, grads["w_post"], grads["w_pre"], grads["gate"], self.norm, self.param]

    def reset(self, param):
        self.param.copy_(param)
        self.m.zero_(), self.v.zero_()


def test_captured_steps_that_share_a_workspace(F):
    announce("captured training steps")
    shapes = [(301, 512, 1003), (40, 2560, 5000)]
    ws = F.workspace(max(max(F.linear_ce_workspace_size(T, V, C), F.sandwich_norm_workspace_size(T, C)) for T, C, V in shapes))
    steps = [Step(F, *s, ws, i) for i, s in enumerate(shapes)]
    start = [s.param.clone() for s in steps]
    graphs, outs = [], []
    for s, p in zip(steps, start):
        s()
        torch.cuda.synchronize()
        s.reset(p)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = s()
        graphs.append(graph), outs.append(out)
    for k in range(3):
        for s, p, graph, out in zip(steps, start, graphs, outs):
            with torch.no_grad():
                s.X.mul_(1.01)  # the program's own eager work between replays
            s.reset(p)
            graph.replay()
            got = [x.clone() for x in out]
            torch.cuda.synchronize()
            s.reset(p)
            want = s()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), k
    assert F.check_flags(ws) == F.OK
