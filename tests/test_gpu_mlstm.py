"""The mLSTM scorer's recurrence (include/kvpop_mlstm.h) against the 64-bit oracle: read-outs of whole sequences
and what is held after them, single tokens, streams and graphs."""
import numpy as np
import pytest

from oracle import mlstm as om

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import i32  # noqa: E402
from mlstm_cases import b16, check, check_read, inputs, on_gpu  # noqa: E402

pytestmark = pytest.mark.gpu

INF = float("inf")


def state_of(rng, B, H, D, m=None):
    C, z = rng.standard_normal((B, H, D, D)) * 0.2, rng.random((B, H, D)) + 0.1
    m = rng.standard_normal((B, H)) if m is None else np.full((B, H), m)
    st = [torch.as_tensor(x, dtype=torch.float32).cuda() for x in (C, z, m)]
    return kv.KvpopMlstmState(*st), [x.double().cpu().numpy() for x in st]


def run(rng, B, H, T, D, delay=0, normalize=True, lens=None, state=False, tokens=False, scale=None, edit=None, **kw):
    x = inputs(rng, B, H, T, D, **kw)
    if edit:
        edit(x)
    g, ref = on_gpu(x, tokens)
    scale = D ** -0.5 if scale is None else scale
    st, before = state_of(rng, B, H, D) if state else (None, None)
    o, lse = kv.kvpop_mlstm_fwd(g["q"], g["k"], g["v"], g["ig"], g["fg"], scale, delay, normalize,
                                None if lens is None else i32(lens), st)
    check_read(ref, lens, scale, delay, normalize, o, lse, before, st)
    return o, lse, g, ref


@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 127, 130, 300, 641])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("normalize", [True, False])
def test_lengths(T, D, normalize):
    run(np.random.default_rng(T + D), 1, 2, T, D, normalize=normalize)


@pytest.mark.parametrize("T", [1, 64, 65, 200, 700])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("normalize", [True, False])
def test_from_a_served_state(T, D, normalize):
    run(np.random.default_rng(T), 2, 2, T, D, normalize=normalize, state=True, lens=[T, T // 2], tokens=True)


@pytest.mark.parametrize("delay", [1, 7, 63, 64, 100, 256, 399, 400, 2 ** 31 - 1])
def test_delays(delay):
    run(np.random.default_rng(5), 2, 1, 400, 64, delay=delay, lens=[400, 333])


@pytest.mark.parametrize("lens", [[0, 1, 500], [64, 65, -3], [500, 499, 1000]])
@pytest.mark.parametrize("state", [False, True])
def test_ragged(lens, state):
    run(np.random.default_rng(6), 3, 2, 500, 64, delay=0 if state else 20, lens=lens, state=state)


def test_many_heads_take_one_segment():
    run(np.random.default_rng(7), 2, 260, 330, 64, delay=3)


@pytest.mark.parametrize("ig,fg", [((0, 30), (0, 30)), ((80, 1), (10, 1)), ((-90, 1), (-90, 3)), ((0, 0.1), (-60, 1)), ((0, 200), (300, 1))])
@pytest.mark.parametrize("D", [64, 128])
def test_gates_of_any_size(ig, fg, D):
    """Weights that would overflow or vanish without the common factor."""
    run(np.random.default_rng(8), 1, 2, 300, D, ig=ig, fg=fg, state=True)


@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("normalize", [True, False])
def test_masked_tokens_and_resets(state, normalize):
    """ig = -inf: no token, whatever its k and v hold; fg = -inf: everything before is forgotten."""
    def edit(x):
        rng = np.random.default_rng(1)
        off = rng.random(x["ig"].shape) < 0.2
        off[0, 0, :70] = True      # nothing is held for more than a chunk
        off[1, 1, :] = True        # nothing ever
        x["ig"][off] = -INF
        for n in ("k", "v"):
            x[n][off] = np.where(rng.random(x[n][off].shape) < 0.5, np.nan, INF)
        x["fg"][0, 0, [0, 5, 64, 66, 67, 127, 130, 400]] = -INF
        x["fg"][0, 1, 200:] = INF
        x["fg"][1, 0, 90:100] = -INF
    run(np.random.default_rng(9), 2, 2, 450, 64, normalize=normalize, state=state, edit=edit)
    run(np.random.default_rng(9), 2, 2, 450, 128, delay=0 if state else 9, normalize=normalize, state=state, edit=edit)


def test_rows_behind_a_sequence_do_not_matter():
    def edit(x):
        for n in x:
            x[n][0, :, 100:] = np.nan
    run(np.random.default_rng(10), 2, 2, 200, 64, delay=10, lens=[100, 200], edit=edit)


def test_queries_that_nothing_reads_do_not_matter():
    def edit(x):
        x["q"][:, :, 150:] = np.nan
    run(np.random.default_rng(11), 2, 1, 200, 64, delay=50, edit=edit)


def test_signed_features_without_a_normaliser():
    run(np.random.default_rng(12), 1, 2, 300, 64, normalize=False, signed=True, scale=0.3)


def test_rows_whose_normaliser_is_not_positive_are_zero():
    def edit(x):
        x["q"][:, :, ::3] *= -1
        x["q"][:, :, 1::3] = 0
    o, lse, _, _ = run(np.random.default_rng(13), 1, 2, 200, 64, edit=edit)
    assert torch.isneginf(lse[:, :, ::3]).all() and torch.isneginf(lse[:, :, 1::3]).all() and (o[:, :, ::3] == 0).all()


def test_a_long_sequence_in_segments():
    """4097 tokens of one head are cut into 65 segments; with weights that reach over all of them."""
    run(np.random.default_rng(14), 1, 1, 4097, 64, delay=100, fg=(9, 0.5))


def test_empty_state_is_no_state_and_parts_are_the_whole():
    rng = np.random.default_rng(15)
    x, _ = on_gpu(inputs(rng, 2, 2, 700, 128))
    a = [x[n] for n in ("q", "k", "v", "ig", "fg")]
    o, lse = kv.kvpop_mlstm_fwd(*a)
    st = kv.kvpop_mlstm_empty(2, 2, 128)
    o2, lse2 = kv.kvpop_mlstm_fwd(*a, state=st)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    part = kv.kvpop_mlstm_empty(2, 2, 128)
    got = [kv.kvpop_mlstm_fwd(*(y[:, :, i:j] for y in a), state=part)[0] for i, j in ((0, 1), (1, 300), (300, 364), (364, 700))]
    # two roundings of o apart, and of its terms, which are no larger together than the largest |v|
    assert (torch.cat(got, 2).float() - o.float()).abs().max() <= 4 * 2.0 ** -8 * a[2].float().abs().max()
    for y, z in zip(part, st):
        assert torch.allclose(y, z, rtol=2.0 ** -12, atol=2.0 ** -12 * float(z.abs().max()))


# ---------------------------------------------------------------------------
# One token
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("B,H,D", [(1, 1, 64), (1, 8, 128), (5, 3, 64), (33, 2, 128)])
@pytest.mark.parametrize("normalize", [True, False])
def test_tokens(B, H, D, normalize):
    rng = np.random.default_rng(B + D)
    st, _ = state_of(rng, B, H, D)
    for step in range(4):
        x = {n: y[:, :, 0] for n, y in inputs(rng, B, H, 1, D).items()}
        if step == 2:
            x["ig"][0, 0], x["k"][0, 0], x["v"][0, 0] = -INF, np.nan, INF
        if step == 3:
            x["fg"][-1, -1] = -INF
        g, ref = on_gpu(x)
        active = None if step % 2 else (np.arange(B) % 3 != 2).astype(int)
        before = [y.double().cpu().numpy() for y in st]
        o = kv.kvpop_mlstm_step(g["q"], g["k"], g["v"], g["ig"], g["fg"], st, 0.3, normalize, None if active is None else i32(active))
        for b in range(B):
            for h in range(H):
                one = {n: ref[n][b, h][None] for n in ref}
                s = [y[b, h] for y in before]
                if active is not None and not active[b]:
                    assert (o[b, h] == 0).all() and all(np.array_equal(y[b, h].double().cpu().numpy(), z) for y, z in zip(st, s))
                    continue
                with np.errstate(invalid="ignore"):
                    ro, _, _, terms, dens = om.read(one["q"], one["k"], one["v"], one["ig"], one["fg"], 0.3, 0, normalize, s)
                # nothing is rounded to bf16 but o: exponents and D sums in fp32
                tiny = 2.0 ** -17
                check("o", o[b, h].double().cpu().numpy(), ro[0], 1.01 * (2.0 ** -8 * np.abs(ro[0]) + tiny * terms[0] + (dens[0] * tiny * np.abs(ro[0]) if normalize else 0)) + 1e-37)
                rs = om.held(one["k"], one["v"], one["ig"], one["fg"], s)
                ra = om.held(np.abs(one["k"]), np.abs(one["v"]), one["ig"], one["fg"], [np.abs(s[0]), np.abs(s[1]), s[2]])
                for y, want, most in zip(st[:2], rs, ra):
                    check("state", y[b, h].double().cpu().numpy(), want, tiny * np.abs(most) + 1e-37)
                assert abs(float(st.m[b, h]) - rs[2]) <= 2.0 ** -21 * (abs(rs[2]) + 1)


def test_tokens_from_nothing_held_and_strided_rows():
    rng = np.random.default_rng(3)
    st = kv.kvpop_mlstm_empty(2, 3, 64)
    qkv = torch.from_numpy(rng.random((2, 9, 64))).to(torch.bfloat16).cuda()
    gates = torch.from_numpy(rng.standard_normal((2, 6))).to(torch.bfloat16).cuda()
    q, k, v, ig, fg = qkv[:, :3], qkv[:, 3:6], qkv[:, 6:], gates[:, ::2], gates[:, 1::2]
    o = kv.kvpop_mlstm_step(q, k, v, ig, fg, st)
    # one token: its own value, whatever the gates
    assert (o.float() - v.float()).abs().max() <= 2.0 ** -8 * 1.01 * v.float().abs().max()
    assert torch.equal(st.m, ig.float()) and torch.allclose(st.z, k.float(), rtol=1e-6)


def test_a_prompt_then_tokens_is_the_whole():
    rng = np.random.default_rng(16)
    B, H, T, D, w = 2, 2, 200, 64, 5
    x, ref = on_gpu(inputs(rng, B, H, T, D))
    a = [x[n] for n in ("q", "k", "v", "ig", "fg")]
    want, _ = kv.kvpop_mlstm_fwd(*a, delay=w)
    st = kv.kvpop_mlstm_empty(B, H, D)
    kv.kvpop_mlstm_fwd(*(y[:, :, :150].contiguous() for y in a), state=st, delay=w)
    for t in range(150, T):
        o = kv.kvpop_mlstm_step(x["q"][:, :, t - w], *(y[:, :, t] for y in a[1:]), st)
        assert (o.float() - want[:, :, t - w].float()).abs().max() <= 4 * 2.0 ** -8 * x["v"].float().abs().max()


def test_captured_calls_match_eager_ones():
    """A prompt's read-outs and a token, as one graph, replayed with other inputs, eager work between."""
    rng = np.random.default_rng(17)
    B, H, T, D = 2, 3, 700, 64
    x, _ = on_gpu(inputs(rng, B, H, T, D))
    a = [x[n] for n in ("q", "k", "v", "ig", "fg")]
    st, e = kv.kvpop_mlstm_empty(B, H, D), kv.kvpop_mlstm_empty(B, H, D)
    ws = torch.empty(kv.kvpop_mlstm_fwd_workspace_size(B, H, T, D), dtype=torch.uint8, device="cuda")
    o, lse, o1 = torch.empty_like(a[0]), torch.empty(B, H, T, device="cuda"), torch.empty(B, H, D, dtype=torch.bfloat16, device="cuda")

    def calls(state):
        kv.kvpop_mlstm_fwd(*a, state=state, o=o, lse=lse, workspace=ws)
        kv.kvpop_mlstm_step(*(y[:, :, 0] for y in a), state, o=o1)

    calls(kv.kvpop_mlstm_empty(B, H, D))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(st)
    for i in range(4):
        y, _ = on_gpu(inputs(rng, B, H, T, D))
        for n, t in zip(("q", "k", "v", "ig", "fg"), a):
            t.copy_(y[n])
        graph.replay()
        torch.cuda.synchronize()
        got = [z.clone() for z in (o, lse, o1)]
        calls(e)
        torch.cuda.synchronize()
        assert all(torch.equal(p, r) for p, r in zip(got, (o, lse, o1)))
        assert all(torch.equal(p, r) for p, r in zip(st, e))


def test_on_a_side_stream_and_twice_the_same():
    rng = np.random.default_rng(18)
    x, _ = on_gpu(inputs(rng, 1, 2, 2000, 128))
    a = [x[n] for n in ("q", "k", "v", "ig", "fg")]
    want = kv.kvpop_mlstm_fwd(*a)
    side = torch.cuda.Stream()
    out = [torch.empty_like(y) for y in want]
    side.wait_stream(torch.cuda.current_stream())
    kv.kvpop_mlstm_fwd(*a, o=out[0], lse=out[1], stream=side)
    side.synchronize()
    assert all(torch.equal(p, r) for p, r in zip(out, want))
