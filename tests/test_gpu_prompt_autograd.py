"""prompt_attention on tensors that require gradients: its backward pass is adore_prompt_attention_backward, bit for bit, and torch's own
rules see to views and broadcast tensors.  Values and tolerances as in test_gpu_prompt.py."""
import pytest

from tests.test_gpu_prompt import DEV, _mods, check, draw, reference

pytestmark = pytest.mark.gpu


def starts(torch, lengths):
    return torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("lengths", [[70, 1, 0, 130], None])
def test_gradients_are_those_of_the_call(lengths, rest, dtype):
    torch, P = _mods()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    if lengths:
        shapes, at = [(sum(lengths), h, 64) for h in (6, 2, 2, 6)], dict(q_start=starts(torch, lengths), k_start=starts(torch, lengths))
    else:
        shapes, at = [(2, h, 77, 64) for h in (6, 2, 2, 6)], {}
    q, k, v, do = (draw(torch, s, dt, i) for i, s in enumerate(shapes))
    with torch.no_grad():
        want = P.prompt_attention(q, k, v, rest=rest, scale=0.2, **at)
    grads = P.prompt_attention_backward(do, q, k, v, want[0], want[1], rest=want[2] if rest else None, scale=0.2, **at)
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    got = P.prompt_attention(*leaves, rest=rest, scale=0.2, **at)
    assert len(got) == len(want) and got[0].requires_grad
    for x, y in zip(got, want):
        assert (x is None and y is None) or torch.equal(x, y)
    assert not any(x is not None and x.requires_grad for x in got[1:])
    got[0].backward(do)
    for x, y in zip(leaves, grads):
        assert torch.equal(x.grad, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_views_of_one_projection(dtype):
    torch, P = _mods()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    n, d = 150, 64
    qkv = draw(torch, (n, 8, d), dt, 1).requires_grad_()
    do = draw(torch, (n, 4, d), dt, 2)
    at = dict(q_start=starts(torch, [n]), k_start=starts(torch, [n]))
    out, lse, _ = P.prompt_attention(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], rest=True, **at)
    out.backward(do)
    x = qkv.detach()
    want = reference(torch, x[:, :4], x[:, 4:6], x[:, 6:], do, d ** -0.5)
    check(torch, dict(out=out.detach(), lse=lse, dq=qkv.grad[:, :4], dk=qkv.grad[:, 4:6], dv=qkv.grad[:, 6:]), want, dt, d)


@pytest.mark.parametrize("which", ["q", "k", "v"])
def test_one_of_them(which):
    torch, P = _mods()
    q, k, v = (draw(torch, (1, 2, 50, 64), torch.float32, s) for s in (1, 2, 3))
    do = draw(torch, q.shape, torch.float32, 4)
    x = dict(q=q, k=k, v=v)
    out, lse = P.prompt_attention(q, k, v)
    want = dict(zip("qkv", P.prompt_attention_backward(do, q, k, v, out, lse)))
    x[which].requires_grad_()
    P.prompt_attention(q, k, v)[0].backward(do)
    assert torch.equal(x[which].grad, want[which])
    assert all(y.grad is None for name, y in x.items() if name != which)


def test_shared_keys_take_the_sum():
    """K and V of one sequence, broadcast to three: sums of three fp32 gradients, three roundings at most."""
    torch, P = _mods()
    q, do = draw(torch, (3, 4, 60, 64), torch.float32, 1), draw(torch, (3, 4, 60, 64), torch.float32, 2)
    k, v = (draw(torch, (1, 2, 60, 64), torch.float32, s).requires_grad_() for s in (3, 4))
    P.prompt_attention(q, k.expand(3, -1, -1, -1), v.expand(3, -1, -1, -1))[0].backward(do)
    kk, vv = (x.detach().expand(3, -1, -1, -1).contiguous() for x in (k, v))
    out, lse = P.prompt_attention(q, kk, vv)
    _, dk, dv = P.prompt_attention_backward(do, q, kk, vv, out, lse)
    for got, each in ((k.grad, dk), (v.grad, dv)):
        assert bool(((got[0].double() - each.double().sum(0)).abs() <= 3 * 2.0 ** -24 * each.double().abs().sum(0)).all())


def test_gradients_in_any_layout():
    """Of a sum (one element, broadcast), of another order of dimensions, of rows that do not lie on 16 bytes."""
    torch, P = _mods()
    for dt in (torch.bfloat16, torch.float32):
        q, k, v = (draw(torch, (2, 3, 40, 64), dt, s).requires_grad_() for s in (1, 2, 3))

        def grads(do):
            return torch.autograd.grad(P.prompt_attention(q, k, v)[0], (q, k, v), do)

        one = torch.ones((), dtype=dt, device=DEV).expand(q.shape)
        last = draw(torch, (2, 3, 64, 40), dt, 5).transpose(2, 3)
        odd = draw(torch, (2, 3, 40, 65), dt, 6)[..., 1:]
        shifted = draw(torch, (q.numel() + 1,), dt, 7)[1:].view(q.shape)
        for do in (one, last, odd, shifted):
            for x, y in zip(grads(do), grads(do.contiguous().clone())):
                assert torch.equal(x, y)
        loss = P.prompt_attention(q, k, v)[0].sum()
        for x, y in zip(torch.autograd.grad(loss, (q, k, v)), grads(one)):
            assert torch.equal(x, y)


def test_where_there_is_no_graph():
    torch, P = _mods()
    q = draw(torch, (1, 2, 50, 64), torch.float32, 1).requires_grad_()
    with torch.no_grad():
        out, lse = P.prompt_attention(q, q, q)
    assert not out.requires_grad and not lse.requires_grad
    assert not P.prompt_attention(q.detach(), q.detach(), q.detach())[0].requires_grad
    with pytest.raises(ValueError, match="^out: "):
        P.prompt_attention(q, q, q, out=torch.empty_like(q).detach())
    with torch.no_grad():
        mine = torch.empty_like(q)
        assert P.prompt_attention(q, q, q, out=mine)[0] is mine
    d, = torch.autograd.grad(P.prompt_attention(q, q, q)[0].square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):                                    # no gradient of the gradient, and no silence about it
        d.sum().backward()
