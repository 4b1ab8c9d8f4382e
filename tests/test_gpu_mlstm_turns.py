"""A conversation: a prompt, turns and tokens on one state are the whole sequence, where a query is read `delay` tokens later. The
queries that a part leaves unread go in front of the next part's, and are read with delay 0."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from mlstm_cases import inputs, on_gpu  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("w,parts", [(5, (200, 64, 3, 1, 90)), (100, (130, 40, 30, 200)), (64, (64, 64, 64)), (0, (70, 1, 129))])
def test_turns_are_the_whole(w, parts, D):
    B, H, T = 2, 2, sum(parts) + 4
    x, _ = on_gpu(inputs(np.random.default_rng(w), B, H, T, D), tokens=True)
    q, k, v, ig, fg = (x[n] for n in ("q", "k", "v", "ig", "fg"))
    want, _ = kv.kvpop_mlstm_fwd(q, k, v, ig, fg, delay=w)
    st = kv.kvpop_mlstm_empty(B, H, D)
    got, late, at = [], q[:, :, :0], 0
    for n in parts:
        here = slice(at, at + n)
        if at == 0:
            o, _ = kv.kvpop_mlstm_fwd(q[:, :, here], k[:, :, here], v[:, :, here], ig[:, :, here], fg[:, :, here], delay=w, state=st)
            got.append(o[:, :, :max(0, n - w)])
            late = q[:, :, max(0, n - w):n]
        else:
            late = torch.cat([late, q[:, :, here]], 2)
            o, _ = kv.kvpop_mlstm_fwd(late[:, :, :n], k[:, :, here], v[:, :, here], ig[:, :, here], fg[:, :, here], state=st)
            got.append(o)
            late = late[:, :, n:]
        at += n
    for t in range(at, T):
        late = torch.cat([late, q[:, :, t:t + 1]], 2)
        got.append(kv.kvpop_mlstm_step(late[:, :, 0], k[:, :, t], v[:, :, t], ig[:, :, t], fg[:, :, t], st)[:, :, None])
        late = late[:, :, 1:]
    got = torch.cat(got, 2)
    assert got.shape[2] == T - w
    # two roundings of o apart, and of its terms, which are no larger together than the largest |v|
    assert (got.float() - want[:, :, :T - w].float()).abs().max() <= 4 * 2.0 ** -8 * v.float().abs().max()
    assert (want[:, :, T - w:] == 0).all()
