"""What a rotation in torch's autograd holds on to until its backward pass: rows of a tensor that is normed, whose gradient reads them, and of no
other."""
import pytest

from tests.test_gpu_rotate import DEV, _mods, draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm", ["none", "q", "k"])
def test_rows_that_no_gradient_reads_are_let_go(norm):
    torch, P = _mods()
    T, H, Hk, d = 4096, 8, 4, 64
    leaf = draw(torch, (T, d), torch.bfloat16, 1).requires_grad_()
    w = (1.0 + 0.3 * draw(torch, (d,), torch.float32, 3)) if norm != "none" else None
    pos, rotary = torch.arange(T, dtype=torch.int32, device=DEV), P.Rotary(d)
    how = {} if w is None else {norm + "_weight": w}
    q, k = leaf[:, None].repeat(1, H, 1), leaf[:, None].repeat(1, Hk, 1)
    rows = {"q": q.detach().clone(), "k": k.detach().clone()}
    q_out, k_out = P.rotate_heads(q, k, pos, rotary, **how)
    before, size = torch.cuda.memory_allocated(), 0
    for name, x in (("q", q), ("k", k)):
        if name != norm:
            size += x.nbytes
            x.mul_(3.0)                                  # (a tensor that is kept for the backward pass may not be changed)
    held = {"q": q, "k": k}[norm] if w is not None else None
    del q, k, x
    assert torch.cuda.memory_allocated() <= before - size
    dq, dk = draw(torch, q_out.shape, torch.bfloat16, 5), draw(torch, k_out.shape, torch.bfloat16, 6)
    (grad,) = torch.autograd.grad([q_out, k_out], [leaf], [dq, dk])
    want = P.rotate_heads_backward(dq, dk, rows["q"], rows["k"], pos, rotary, **how)
    again = leaf.detach().clone().requires_grad_()
    by_hand = torch.autograd.grad([again[:, None].repeat(1, H, 1), again[:, None].repeat(1, Hk, 1)], [again], list(want[:2]))[0]
    assert torch.equal(grad, by_hand) and (held is None or torch.equal(held, rows[norm]))


def test_a_normed_tensor_is_kept():
    """Changed in place, torch refuses the backward pass, as for any operation whose gradient reads its input."""
    torch, P = _mods()
    leaf = draw(torch, (9, 2, 64), torch.bfloat16, 1).requires_grad_()
    w, pos = torch.ones(64, device=DEV), torch.arange(9, dtype=torch.int32, device=DEV)
    q = leaf * 1.0
    out, _ = P.rotate_heads(q, None, pos, P.Rotary(64), q_weight=w)
    q.mul_(2.0)
    with pytest.raises(RuntimeError):
        out.sum().backward()
