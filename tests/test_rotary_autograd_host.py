"""The differentiable rotary calls on the CPU, with plain implementations in the place of the library's calls: what the functions save and pass on."""
import pytest
import torch

from tests import rotary_reference as R


@pytest.fixture
def A(monkeypatch):
    """autograd with mala.rotary, rotary_bwd and their packed forms in 64 bits, rounded to bf16."""
    from paper_2609_32712_b200 import autograd as a, mala

    def args(rot, norm, which, pos):
        w = None if norm is None else (norm.q_weight, norm.k_weight)[which]
        return pos, rot.inv_freq, rot.interleaved, rot.magnitude, None if norm is None else norm.eps, w

    def positions(cu, n):
        return torch.tensor([t - max(int(c) for c in cu if int(c) <= t) for t in range(n)])[None]

    def rotary(q, k, rot, positions=None, norm=None):
        pos = torch.arange(q.shape[1])[None] if positions is None else positions
        return tuple(None if t is None else R.forward(t.detach(), *args(rot, norm, x, pos)).to(torch.bfloat16) for x, t in enumerate((q, k)))

    def rotary_bwd(dq, dk, rot, positions=None, norm=None, q=None, k=None, weights=True):
        pos = torch.arange(dq.shape[1])[None] if positions is None else positions
        out = [(None, None) if t is None else R.backward(t, x, *args(rot, norm, i, pos))[:2] for i, (t, x) in enumerate(((dq, q), (dk, k)))]
        grads = [None if g is None else g.to(torch.bfloat16) for g, _ in out]
        return (*grads, *[w.float() if weights and w is not None and norm is not None and v is not None else None
                          for (_, w), v in zip(out, (norm.q_weight, norm.k_weight) if norm else (None, None))])
    monkeypatch.setattr(mala, "rotary", rotary)
    monkeypatch.setattr(mala, "rotary_bwd", rotary_bwd)
    monkeypatch.setattr(mala, "rotary_varlen", lambda q, k, cu_q, cu_k, rot, norm=None: rotary(q, k, rot, positions(cu_q, q.shape[1]), norm))
    monkeypatch.setattr(mala, "rotary_varlen_bwd", lambda dq, dk, cu_q, cu_k, rot, norm=None, q=None, k=None, weights=True:
                        rotary_bwd(dq, dk, rot, positions(cu_q, dq.shape[1]), norm, q, k, weights))
    return a


def _inputs(normed):
    g = torch.Generator().manual_seed(3)
    q, dy = (torch.randn((1, 7, 2, 16), generator=g).to(torch.bfloat16) for _ in range(2))
    w = torch.rand(16, generator=g).add(0.5).requires_grad_() if normed else None
    return q.requires_grad_(), dy, w


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("normed", [False, True])
def test_without_keys(A, packed, normed):
    from paper_2609_32712_b200 import mala
    q, dy, w = _inputs(normed)
    rot, eps = mala.Rotary(0.3 ** torch.arange(6).double(), device="cpu"), 1e-5 if normed else None
    cu = torch.tensor([0, 3, 7], dtype=torch.int32)
    out, keys = A.rotary_packed(q, None, cu, cu, rot, q_weight=w, eps=eps) if packed else A.rotary(q, None, rot, q_weight=w, eps=eps)
    assert keys is None
    out.backward(dy)
    pos = torch.tensor([0, 1, 2, 0, 1, 2, 3] if packed else range(7))[None]
    dx, dw, _ = R.backward(dy, q.detach(), pos, rot.inv_freq, False, 1.0, eps, None if w is None else w.detach())
    assert torch.equal(q.grad, dx.to(torch.bfloat16)) and (w is None or torch.equal(w.grad, dw.float()))


@pytest.mark.parametrize("change", [dict(inv_freq=lambda r: r.inv_freq / 4), dict(magnitude=lambda r: 2.0), dict(interleaved=lambda r: True)])
def test_rule_of_the_forward_pass(A, change):
    """A Rotary whose frequencies are replaced behind a forward pass (a context that grows over its length): its gradients are those of that pass."""
    from paper_2609_32712_b200 import mala
    q, dy, _ = _inputs(False)
    rot = mala.Rotary(0.3 ** torch.arange(6).double(), device="cpu")
    A.rotary(q, q.detach(), rot)[0].backward(dy)
    want, q.grad = q.grad, None
    out = A.rotary(q, q.detach(), rot)[0]
    for name, value in change.items():
        setattr(rot, name, value(rot))
    out.backward(dy)
    assert torch.equal(q.grad, want)


def test_frequencies_changed_in_place_are_noticed(A):
    from paper_2609_32712_b200 import mala
    q, dy, _ = _inputs(False)
    rot = mala.Rotary(0.3 ** torch.arange(6).double(), device="cpu")
    out = A.rotary(q, None, rot)[0]
    rot.inv_freq.mul_(0.5)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.backward(dy)
