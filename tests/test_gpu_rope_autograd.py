"""qk_norm_rope on tensors that require gradients: they get those of qk_norm_rope_backward, bit for bit (which test_gpu_rope
holds against the definition and against differences), or the call says that it cannot give any."""

import pytest
import torch

import paper_2605_14037_amd as spkv

pytestmark = pytest.mark.gpu


def _inputs(t, hq, hk, d, dtype):
    g = torch.Generator(device="cuda").manual_seed(t)
    rows = torch.randn(t, hq + 2 * hk, d, generator=g, device="cuda").to(dtype)
    w = 1.0 + 0.3 * torch.randn(2, d, generator=g, device="cuda")
    dy = [torch.randn(t, h, d, generator=g, device="cuda").to(dtype) for h in (hq, hk, hk)]
    pos = torch.randint(0, 1 << 20, (t,), generator=g, device="cuda", dtype=torch.int32)
    return rows, w[0].clone(), w[1].clone(), dy, pos, spkv.Rope(d, theta=1e6)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("t,hq,hk,d", [(0, 4, 2, 64), (1, 32, 8, 128), (67, 3, 3, 64), (1003, 5, 1, 128)])
@pytest.mark.parametrize("eps", [1e-6, None], ids=["norm", "plain"])
def test_gradients_reach_the_inputs(t, hq, hk, d, dtype, eps):
    rows, qw, kw, dy, pos, rope = _inputs(t, hq, hk, d, dtype)
    leaf, w = rows.clone().requires_grad_(), [x.clone().requires_grad_() for x in (qw, kw)]
    norm = dict(q_weight=w[0], k_weight=w[1], eps=eps) if eps is not None else {}
    q, k, v = leaf.split([hq, hk, hk], 1)
    out = spkv.qk_norm_rope(q, k, pos, rope, v=v, **norm)
    with torch.no_grad():
        plain = spkv.qk_norm_rope(q, k, pos, rope, v=v, **norm)
    assert all(a.requires_grad and not b.requires_grad and torch.equal(a, b) for a, b in zip(out, plain))
    torch.autograd.backward(out, dy)
    want = torch.empty_like(rows)
    q, k, v = rows.split([hq, hk, hk], 1)
    norm = dict(q=q, k=k, q_weight=qw, k_weight=kw, eps=eps) if eps is not None else {}
    want[:, hq + hk:] = dy[2]                                # (the values' gradient passes beside the call)
    dw = spkv.qk_norm_rope_backward(dy[0], dy[1], pos, rope, out=want.split([hq, hk, hk], 1), **norm)
    assert torch.equal(leaf.grad, want)
    assert all(torch.equal(a.grad, b) for a, b in zip(w, dw)) and len(dw) == (0 if eps is None else 2)


@pytest.mark.parametrize("wanted", ["q", "k", "v", "q_weight", "k_weight"])
def test_only_what_is_asked_for(wanted):
    rows, qw, kw, dy, pos, rope = _inputs(37, 4, 2, 64, torch.float32)
    q, k, v = (x.clone() for x in rows.split([4, 2, 2], 1))
    x = {"q": q, "k": k, "v": v, "q_weight": qw, "k_weight": kw}
    x[wanted].requires_grad_()
    out = spkv.qk_norm_rope(q, k, pos, rope, v=v, q_weight=qw, k_weight=kw, eps=1e-6)
    torch.autograd.backward(out, dy)
    dq, dk, dqw, dkw = spkv.qk_norm_rope_backward(dy[0], dy[1], pos, rope, q=q.detach(), k=k.detach(),
                                                  q_weight=qw.detach(), k_weight=kw.detach(), eps=1e-6)
    want = {"q": dq, "k": dk, "v": dy[2], "q_weight": dqw, "k_weight": dkw}
    assert torch.equal(x.pop(wanted).grad, want[wanted]) and all(y.grad is None for y in x.values())


def test_without_values_and_with_gradients_of_other_layouts():
    """Only the queries used; gradients that come with strides of zero, transposed, from an odd address."""
    rows, qw, kw, _, pos, rope = _inputs(9, 4, 4, 64, torch.bfloat16)
    odd = torch.randn(9 * 4 * 64 + 1, device="cuda").bfloat16()[1:].view(9, 4, 64)
    some = torch.randn(64, 9, 4, device="cuda").bfloat16().permute(1, 2, 0)
    for dy in (torch.ones((), device="cuda").bfloat16().expand(9, 4, 64), some, odd):
        q, k = (x.clone().requires_grad_() for x in rows[:, :8].split([4, 4], 1))
        out = spkv.qk_norm_rope(q, k, pos, rope, q_weight=qw, k_weight=kw, eps=1e-6)
        assert len(out) == 2
        out[0].backward(dy)
        want = spkv.qk_norm_rope_backward(dy.contiguous().clone(), torch.zeros_like(k), pos, rope, q=q.detach(), k=k.detach(), q_weight=qw,
                                          k_weight=kw, eps=1e-6, want_weights=False)
        assert torch.equal(q.grad, want[0]) and not k.grad.any()


def test_what_it_cannot_do_is_refused():
    rows, qw, kw, dy, pos, rope = _inputs(5, 4, 2, 64, torch.float32)
    q, k = rows[:, :4].clone(), rows[:, 4:6].clone()
    into = (torch.empty_like(q), torch.empty_like(k))
    with pytest.raises(ValueError, match="out"):
        spkv.qk_norm_rope(q.requires_grad_(), k, pos, rope, out=into)
    with pytest.raises(ValueError, match="out"):
        spkv.qk_norm_rope(q.detach(), k, pos, rope, q_weight=qw.requires_grad_(), eps=1e-6, out=into)
    with torch.no_grad():                                    # nothing is asked for
        spkv.qk_norm_rope(q, k, pos, rope, out=into)
    out = spkv.qk_norm_rope(q, k, pos, rope)
    again = torch.autograd.grad(out, [q], [dy[0].requires_grad_(), dy[1]], create_graph=True)
    with pytest.raises(RuntimeError):                        # the gradient's own gradient
        torch.autograd.grad(again[0].sum(), [dy[0]])
