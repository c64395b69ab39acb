"""GPU test of the decoder stack: norms, attention, KL-Top and log probabilities chained through quantised linears.

The gradient that reaches the fused q-k-v product has passed, in bf16, KL-Top, two input-gradient products, the straight-through
activation backwards, a norm's backward and the attention's. The reference is autograd over the same chain in fp32, each
quantisation replaced by its value with a straight-through derivative. Some ten roundings to bf16 (2^-9 each) lie
between, two of them (P, dS) inside sums: 5e-2 of the norm.
"""
import pytest
import torch

from gpu_common import announce, require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    return require_gpu()


def attention(q, k, v, cu):
    out = []
    for a, b in zip(cu[:-1], cu[1:]):
        g = q.shape[1] // k.shape[1]
        Q = q[a:b].transpose(0, 1)
        K, V = (x[a:b].transpose(0, 1).repeat_interleave(g, 0) for x in (k, v))
        S = (Q @ K.transpose(1, 2).contiguous()) * q.shape[2] ** -0.5
        S = S.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool, device=q.device).triu(1), float("-inf"))
        out.append((torch.softmax(S, 2) @ V.contiguous()).transpose(0, 1))
    return torch.cat(out)


@pytest.mark.parametrize("fmt", [0, 1])
def test_gradient_through_the_chain(F, fmt):
    from paper_2608_01847_amd import calib, synth
    st = calib.DecoderStack(fmt, "crs_dgs", hidden=256, heads=(4, 2), head_dim=64, vocab=1024, lengths=(100, 1, 64, 155), k=50)
    announce(f"decoder stack fmt={fmt}")
    X = synth.activation_batch(st.w, "x", 0, st.T, device="cuda")
    Zt = st.teacher(X)
    s = st.student(X)
    dZ, loss = F.kl_top(s["Z"], Zt, st.k, ws=st.ws)
    got = st.backward(s, dZ)["dqkv"]
    assert F.check_flags(st.ws) == F.OK

    def ste(x, x_hat):  # elements that the quantiser saturates pass no gradient (NVFP4's rounded scales)
        bf = x.detach().to(torch.bfloat16)
        m = F.fakequant_act_bwd(bf, torch.ones_like(bf), fmt, ws=st.ws).float()
        return x * m + (x_hat.float() - x * m).detach()

    cu = st.cu.tolist()
    qkv = s["qkv"].float().requires_grad_(True)
    O = attention(*st._slices(qkv), cu).flatten(1)
    Y = ste(O, s["O_hat"]) @ s["Wo_hat"].float().t()
    H = X.float() + Y
    B = H * torch.rsqrt(H.square().mean(1, keepdim=True) + 1e-5) * st.gain["out"].float()
    Z = ste(B, s["B_hat"]) @ s["Wh_hat"].float().t()
    idx = torch.sort(Zt.float(), dim=1, descending=True, stable=True)[1][:, :st.k]
    lt, ls = (torch.log_softmax(z.gather(1, idx), 1) for z in (Zt.float(), Z))
    ref_loss = (lt.exp() * (lt - ls)).sum() / st.T
    ref, = torch.autograd.grad(ref_loss, qkv)
    assert abs(loss.item() - ref_loss.item()) <= 2e-2 * ref_loss.item()
    err = (got.float() - ref).norm() / ref.norm()
    assert err <= 5e-2, float(err)


@pytest.mark.parametrize("fmt", [0, 1], ids=["mx", "nv"])
def test_an_epoch_lowers_the_loss(F, fmt):
    # hidden 2,560, 32/8 heads of 128, vocabulary 32,000, four packed sequences: held-out scores before and after
    from paper_2608_01847_amd import calib
    announce(f"decoder stack epoch fmt={fmt}")
    r = calib.decoder_epoch(fmt, "crs_dgs")
    before, after = r["eval_before"], r["eval_after"]
    assert after["kl_top"] < 0.95 * before["kl_top"], (before, after)
    assert after["nll"] < before["nll"] and after["agreement"] > before["agreement"], (before, after)
    assert 0 < after["entropy"] < 10.4  # ln 32,000 = 10.37
