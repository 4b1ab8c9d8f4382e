"""Workspaces that are views: the kernels write `need` bytes from the address on, so that a view whose
elements do not lie after each other is refused, however many it names."""
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402


def test_the_check_itself():
    cpu = torch.device("cpu")
    kv._check_workspace(torch.empty(64, dtype=torch.uint8), 64, cpu)
    kv._check_workspace(torch.empty(4, 4), 64, cpu)
    for bad in (torch.empty(1, dtype=torch.uint8).expand(64), torch.empty(128, dtype=torch.uint8)[::2],
                torch.empty(4, 8)[:, :4], torch.empty(63, dtype=torch.uint8)):
        with pytest.raises(ValueError, match="workspace"):
            kv._check_workspace(bad, 64, cpu)


@pytest.mark.gpu
def test_views_are_refused_and_contiguous_ones_serve():
    i32 = dict(dtype=torch.int32, device="cuda")
    one = torch.empty(1, dtype=torch.uint8, device="cuda")
    r = torch.randn(1, 2, 500, device="cuda")
    need = kv.kvpop_running_topk_workspace_size(1, 2, 500)
    with pytest.raises(ValueError, match="workspace"):
        kv.kvpop_running_topk(r, 2, 8, 20, workspace=one.expand(need))
    got = kv.kvpop_running_topk(r, 2, 8, 20, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
    assert all(torch.equal(got[n], x) for n, x in kv.kvpop_running_topk(r, 2, 8, 20).items())
    cache = kv.kvpop_cache_empty(1, 1, 20000, 64)
    q, held = torch.randn(1, 2, 1, 64, device="cuda").to(torch.bfloat16), torch.full((1, 1), 300, **i32)
    need = kv.kvpop_cache_attn_workspace_size(cache, 2, 1)
    assert need > 0
    with pytest.raises(ValueError, match="workspace"):
        kv.kvpop_cache_attn(q, cache, held, 0.1, workspace=one.expand(need))
    o, lse = kv.kvpop_cache_attn(q, cache, held, 0.1, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
    assert all(torch.equal(x, y) for x, y in zip((o, lse), kv.kvpop_cache_attn(q, cache, held, 0.1)))
