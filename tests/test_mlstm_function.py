"""What the differentiable recurrence hands to its backward pass: a gradient of any strides and offset, as torch makes
them, becomes rows that the library takes."""
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402

SHAPE = (2, 3, 5, 64)


def gradients(o, w):
    """Losses whose gradient of o is, in turn: w itself, a view at an odd offset, of other strides, expanded."""
    one = o.new_ones(3)
    yield "itself", (o * w).sum()
    yield "offset", (torch.cat([one, o.flatten()]) * torch.cat([one, w.flatten()])).sum()
    yield "strides", (o.permute(3, 0, 1, 2).contiguous() * w.permute(3, 0, 1, 2).contiguous()).sum()
    yield "expanded", o.float().sum()


def test_any_gradient_reaches_the_backward_pass_aligned(monkeypatch):
    seen = []

    def fwd(q, k, v, ig, fg, *args):
        return (q * 2).detach(), ig.float().detach()

    def bwd(do, q, k, v, ig, fg, *args):
        assert do.data_ptr() % 16 == 0 and do.stride(-1) == 1 and all(s % 8 == 0 for s in do.stride()[:-1]) and do.shape == q.shape
        seen.append(do.clone())
        return do, do, do, ig, fg

    monkeypatch.setattr(kv, "kvpop_mlstm_fwd", fwd)
    monkeypatch.setattr(kv, "kvpop_mlstm_bwd", bwd)
    w = torch.randn(SHAPE).to(torch.bfloat16)
    names = []
    for i in range(4):
        x = torch.randn(SHAPE).to(torch.bfloat16).requires_grad_()
        g = torch.zeros(SHAPE[:3], dtype=torch.bfloat16)
        name, loss = list(gradients(kv.kvpop_mlstm(x, x.detach(), x.detach(), g, g), w))[i]
        loss.backward()
        names.append(name)
    assert names == ["itself", "offset", "strides", "expanded"]
    assert all(torch.equal(d, w) for d in seen[:3]) and (seen[3] == 1).all()


@pytest.mark.gpu
def test_gradients_at_odd_offsets():
    gen = torch.Generator().manual_seed(0)
    rand = lambda *s: torch.rand(*s, generator=gen).to(torch.bfloat16).cuda()  # noqa: E731
    q, k, v, w = (rand(*SHAPE) for _ in range(4))
    ig, fg = rand(*SHAPE[:3]), rand(*SHAPE[:3]) + 3
    o, lse = kv.kvpop_mlstm_fwd(q, k, v, ig, fg, delay=1)
    want = kv.kvpop_mlstm_bwd(w, q, k, v, ig, fg, o, lse, delay=1)
    for i in range(3):
        a = [x.detach().clone().requires_grad_() for x in (q, k, v, ig, fg)]
        name, loss = list(gradients(kv.kvpop_mlstm(*a, delay=1), w))[i]
        loss.backward()
        for x, y in zip(a, want):
            assert torch.equal(x.grad, y), name
