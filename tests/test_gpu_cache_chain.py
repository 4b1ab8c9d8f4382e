"""The compact cache as a served model uses it: a prompt's tokens ranked, kept and stored,
then tokens one at a time: retain, append, attend. Checked against the oracle on the codes,
and against kvpop_sparse_attn_fwd, which attends over the same mask in 16 bits; captured in a graph;
on another stream than the current one; and with the binding's refusals on the GPU."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2607_05061_amd as kv  # noqa: E402
from cache_cases import DTYPE, HostCache, attention_check, i32  # noqa: E402
from oracle import compact_cache as cc  # noqa: E402

pytestmark = pytest.mark.gpu


class Served:
    """A batch of sequences of one layer: inputs of T tokens, the first n of them the prompt."""

    def __init__(self, fmt="int8", B=2, Hq=6, H=2, T=400, n=300, D=64, P=32, s=2, w=16, k=60, seed=0, budgets=None):
        g = torch.Generator().manual_seed(seed)
        self.B, self.Hq, self.H, self.T, self.n, self.D, self.P = B, Hq, H, T, n, D, P
        self.s, self.w, self.k, self.S = s, w, k, s + w + k
        mk = lambda h: torch.randn(B, h, T, D, generator=g).to(torch.bfloat16).cuda()  # noqa: E731
        self.q, self.kk, self.v = mk(Hq), mk(H), mk(H)
        self.r = torch.randn(B, H, T, generator=g).cuda()
        self.lg = -torch.rand(H, generator=g).cuda() * 0.02
        ang = torch.arange(T, dtype=torch.float64)[:, None] * 1e4 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))
        self.rot = (ang.cos().float().cuda(), ang.sin().float().cuda())
        self.cache = kv.kvpop_cache_empty(B, H, self.S, D, P, dtype=DTYPE[fmt])
        self.fmt = fmt

    def prompt(self, stream=None):
        n = self.n
        r = self.r[..., :n].contiguous()
        evict = kv.kvpop_running_topk(r, self.s, self.w, self.k, log_gamma=self.lg, evict=True, stream=stream)["evict"]
        self.pos, self.prio, self.held = kv.kvpop_retain_prompt(evict, r, self.S, log_gamma=self.lg, stream=stream)
        kv.kvpop_cache_append(self.cache, self.kk[:, :, :n], self.v[:, :, :n], self.held, count=self.held, src=self.pos,
                              rotary=self.rot, stream=stream)

    def token(self, t, pos, stream=None):
        """Token t of every sequence at its position (int32 [B])."""
        slot = kv.kvpop_retain_step(self.r[..., t - self.w].contiguous(), pos, self.pos, self.prio, self.held, self.s,
                                    self.w, self.k, log_gamma=self.lg, stream=stream)
        one = slice(t, t + 1)
        q = kv.kvpop_cache_append(self.cache, self.kk[:, :, one], self.v[:, :, one], self.held,
                                  count=torch.ones_like(self.held), start=slot, q=self.q[:, :, one], rotary=self.rot,
                                  pos0=pos, stream=stream)
        o, lse = kv.kvpop_cache_attn(q, self.cache, self.held, self.D ** -0.5, stream=stream)
        return slot, q, o, lse

    def run(self, stream=None):
        self.prompt(stream)
        return [self.token(t, i32([t] * self.B), stream) for t in range(self.n, self.T)]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_serving_is_the_sparse_attention_in_8_bits(fmt):
    m = Served(fmt)
    out = m.run()
    # the sparse attention of the whole sequence over bf16 keys as rotated
    c64, s64 = (x.double().cpu().numpy() for x in m.rot)
    k64, q64, v64 = (x.double().cpu().numpy() for x in (m.kk, m.q, m.v))
    kr = cc.rotate(k64, c64, s64, False)
    qr = cc.rotate(q64, c64, s64, False)
    evict = kv.kvpop_running_topk(m.r, m.s, m.w, m.k, log_gamma=m.lg, evict=True)["evict"].cpu().numpy()
    scale = m.D ** -0.5
    for i, t in enumerate(range(m.n, m.T)):
        _, q, o, lse = out[i]
        o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
        for b in range(m.B):
            for h in range(m.H):
                keep = (np.arange(t + 1) <= t) & (evict[b, h, :t + 1] > t)
                for gq in range(h * 3, h * 3 + 3):
                    ro, rl, p = cc.attend(qr[b, gq, t:t + 1], kr[b, h, :t + 1], v64[b, h, :t + 1], keep[None], scale)
                    # int8: a page's step is below 2^(e+1) / 127 of its largest value 127 2^e's bound, all roundings of
                    # a code together are at most one step 2^e (a half, and halves of ever smaller
                    # ones before); e4m3: 2^-4 of the value once, and once more for a subnormal one, of a step of 2^(e-9).
                    def err(x):
                        big = np.abs(x[b, h]).max()
                        if fmt == "int8":
                            return np.full_like(x[b, h, :t + 1], 2 * big / 127)
                        return 2.0 ** -4 * np.abs(x[b, h, :t + 1]) + 2 * big / 448 * 2.0 ** -9
                    qa = np.abs(qr[b, gq, t])
                    dl = scale * (qa @ err(kr).T) + scale * 2.0 ** -8 * (qa @ np.abs(kr[b, h, :t + 1]).T)  # q is bf16
                    dl = dl[keep].max()
                    assert abs(lse[b, gq, 0] - rl[0]) <= dl + 1e-4
                    ev = (p[0][:, None] * err(v64)).sum(0) * math.exp(2 * dl)
                    bound = ev + math.expm1(2 * dl) * (p[0] @ np.abs(v64[b, h, :t + 1])) + 2.0 ** -7 * (
                        np.abs(ro[0]) + p[0] @ np.abs(v64[b, h, :t + 1]))
                    assert (np.abs(o[b, gq, 0] - ro[0]) <= bound).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_serving_against_the_oracle_on_the_codes(fmt):
    m = Served(fmt, T=330)
    host = HostCache(np.random.default_rng(0), m.B, m.H, m.cache.page_table.shape[2], m.P, m.D, fmt, spare=0)
    host.table[:] = m.cache.page_table.cpu().numpy()
    for s in "kv":
        host.side[s][0][:], host.side[s][1][:] = 0, 0
    c64, s64 = (x.double().cpu().numpy() for x in m.rot)
    k64, v64 = m.kk.double().cpu().numpy(), m.v.double().cpu().numpy()
    m.prompt()
    pos, held = m.pos.cpu().numpy(), m.held.cpu().numpy()
    r, lg = m.r.cpu().numpy(), m.lg.cpu().numpy()
    prio = m.prio.cpu().numpy()
    state = {}
    for b in range(m.B):
        for h in range(m.H):
            t = pos[b, h, :held[b, h]]
            host.append("k", cc.rotate(k64[b, h, t], c64[t], s64[t], False), held[b, h], 0, b, h)
            host.append("v", v64[b, h, t], held[b, h], 0, b, h)
            state[b, h] = {i: [int(x), prio[b, h, i]] for i, x in enumerate(t)}
    host.check(m.cache)
    for t in range(m.n, m.T):
        slot, q, o, lse = m.token(t, i32([t] * m.B))
        for b in range(m.B):
            for h in range(m.H):
                j = cc.retain_step(state[b, h], t, r[b, h, t - m.w], lg[h], m.s, m.w, m.k)
                assert slot[b, h].item() == j
                host.append("k", cc.rotate(k64[b, h, t:t + 1], c64[t], s64[t], False), len(state[b, h]), j, b, h)
                host.append("v", v64[b, h, t:t + 1], len(state[b, h]), j, b, h)
        attention_check(q.double().cpu().numpy(), host, m.held.cpu().numpy(), float(np.float32(m.D ** -0.5)), o, lse)
    host.check(m.cache)


def test_a_captured_step_replays_as_eager_ones():
    eager = Served(P=16, T=340)
    want = eager.run()
    m = Served(P=16, T=340)
    m.prompt()
    S = m.S
    # buffers that a step reads, filled before each replay
    q, k, v = (torch.empty(m.B, h, 1, m.D, dtype=torch.bfloat16, device="cuda") for h in (m.Hq, m.H, m.H))
    r, pos = torch.empty(m.B, m.H, device="cuda"), torch.full((m.B,), -1, dtype=torch.int32, device="cuda")

    def step():
        slot = kv.kvpop_retain_step(r, pos, m.pos, m.prio, m.held, m.s, m.w, m.k, log_gamma=m.lg)
        x = kv.kvpop_cache_append(m.cache, k, v, m.held, count=one, start=slot, q=q, rotary=m.rot, pos0=pos)
        return (slot, x) + kv.kvpop_cache_attn(x, m.cache, m.held, m.D ** -0.5)

    one = torch.ones_like(m.held)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()  # warm up: idle sequences, nothing changes
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for i, t in enumerate(range(m.n, m.T)):
        q.copy_(m.q[:, :, t:t + 1]), k.copy_(m.kk[:, :, t:t + 1]), v.copy_(m.v[:, :, t:t + 1])
        r.copy_(m.r[..., t - m.w]), pos.fill_(t)
        for x in got:
            x.fill_(-7)
        if i % 7 == 0:
            torch.cuda.synchronize()
        g.replay()
        if i % 5 == 0:
            torch.cuda.synchronize()
        for a, b in zip(got, want[i]):
            assert torch.equal(a, b), t
    for a, b in zip(m.cache, eager.cache):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert S == m.pos.shape[2]


@pytest.mark.parametrize("explicit", [True, False])
def test_side_stream_matches_the_default_one(explicit):
    want = Served(T=320).run()
    m = Served(T=320)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = m.run(side if explicit else None)
    side.synchronize()
    for a, b in zip(got, want):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


def test_workspace_on_a_stream_that_is_not_current():
    """The current stream allocates and writes memory right after each call returns."""
    rng = np.random.default_rng(2)
    host = HostCache(rng, 1, 2, 300, 64, 128, "int8")
    cache, held = host.gpu(), i32([[19000, 18000]])
    q = torch.randn(1, 8, 1, 128, device="cuda").to(torch.bfloat16)
    need = kv.kvpop_cache_attn_workspace_size(cache, 8, 1)
    assert need > 0
    ref = kv.kvpop_cache_attn(q, cache, held, 0.01)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert all(torch.equal(x, y) for x, y in zip(ref, kv.kvpop_cache_attn(q, cache, held, 0.01, workspace=ws)))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(4):
        o, lse = torch.empty_like(ref[0]), torch.empty_like(ref[1])
        side.wait_stream(torch.cuda.current_stream())
        kv.kvpop_cache_attn(q, cache, held, 0.01, o=o, lse=lse, stream=side)
        noise = [torch.full((need // 4,), float("nan"), device="cuda") for _ in range(3)]
        torch.cuda.synchronize()
        assert torch.equal(o, ref[0]) and torch.equal(lse, ref[1])
        del noise


def test_two_calls_at_once_with_memory_of_their_own():
    rng = np.random.default_rng(3)
    host = HostCache(rng, 1, 2, 300, 64, 64, "e4m3")
    cache, held = host.gpu(), i32([[19000, 18000]])
    q = torch.randn(1, 8, 3, 64, device="cuda").to(torch.bfloat16)
    ref = kv.kvpop_cache_attn(q, cache, held, 1e-3)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    outs = []
    for s in streams:
        with torch.cuda.stream(s):
            outs.append(kv.kvpop_cache_attn(q, cache, held, 1e-3))
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o[0], ref[0]) and torch.equal(o[1], ref[1])


def test_binding_refusals():
    c = kv.kvpop_cache_empty(2, 2, 100, 64, 32)
    k = torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16, device="cuda")
    held = i32([[3, 3], [3, 3]])
    ok = dict(cache=c, k=k, v=k, held=held)
    f32 = torch.zeros(8, 32, device="cuda")
    for bad, err in ((dict(k=k.float()), TypeError), (dict(v=k[:, :, :2]), ValueError), (dict(k=k.transpose(2, 3)), ValueError),
                     (dict(held=held.long()), TypeError), (dict(held=held[0]), ValueError), (dict(held=held.t()), ValueError),
                     (dict(count=i32([3, 3])), ValueError), (dict(src=i32([[0], [0]])), ValueError),
                     (dict(q=k, q_out=k.float()), TypeError), (dict(q_out=k), ValueError),
                     (dict(q=k[:1]), ValueError), (dict(rotary=(f32, f32[:4])), ValueError), (dict(pos0=i32([0])), ValueError),
                     (dict(cache=c._replace(k_pages=c.k_pages.float())), TypeError),
                     (dict(cache=c._replace(v_pages=c.v_pages[:4])), ValueError),
                     (dict(cache=c._replace(k_exp=c.k_exp[:4])), ValueError),
                     (dict(cache=c._replace(page_table=c.page_table[0])), ValueError),
                     (dict(k=k.cpu()), ValueError), (dict(k=[k]), TypeError)):
        with pytest.raises(err):
            kv.kvpop_cache_append(**{**ok, **bad})
    for bad in (dict(k=torch.zeros(2, 2, 3, 65, dtype=torch.bfloat16, device="cuda")[..., 1:]),  # odd strides, not aligned
                dict(rotary=(f32[:, :12].contiguous(), f32[:, :12].contiguous())), dict(q=k, q_out=k)):
        with pytest.raises(kv.KvpopError):
            kv.kvpop_cache_append(**{**ok, **bad})
    for bad, err in ((dict(q=k.float()), TypeError), (dict(q=k[:1]), ValueError), (dict(o=k[:, :, :1]), ValueError),
                     (dict(lse=f32), ValueError), (dict(q_lens=held), ValueError), (dict(scale=0.0), kv.KvpopError),
                     (dict(q=torch.zeros(2, 3, 1, 64, dtype=torch.bfloat16, device="cuda")), kv.KvpopError),
                     (dict(o=k), kv.KvpopError), (dict(q=k[:, :, :0]), kv.KvpopError)):
        with pytest.raises(err):
            kv.kvpop_cache_attn(**{**dict(q=k, cache=c, held=held, scale=0.1), **bad})
    long = kv.kvpop_cache_empty(1, 1, 100000, 64)
    with pytest.raises(ValueError):
        kv.kvpop_cache_attn(k[:1, :1], long, i32([[5]]), 0.1, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
