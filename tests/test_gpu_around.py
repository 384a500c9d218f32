"""A layer as a serving program runs it: rotation, the prompt's attention and its
window normalisers, compression, the kept rows in a 4-bit cache, and decoding
steps whose tokens are rotated at their own positions; the same in a captured
graph, on another stream, and for a prompt that comes in chunks."""
import numpy as np
import pytest

import around_ref as A
import cache_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_14782_amd import bacon
    bacon.lib()


def _np(t):
    return t.double().cpu().numpy()


class Layer:
    """One layer's prompt, through to its cache."""

    def __init__(self, dtype, d, hq, hkv, lens, budgets, W=8, bt=16, seed=0, chunk=None):
        import torch
        from paper_2606_14782_amd import bacon
        self.rng = np.random.default_rng(seed)
        self.dtype, self.d, self.hq, self.hkv, self.W, self.lens = dtype, d, hq, hkv, W, lens
        self.tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        a, b = d // 8, d // 4
        self.rotary = bacon.Rotary(hq, hkv, d, dtype, sections=(a, d // 2 - a - b, b), base=1e6)
        self.cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        T, B = int(self.cu[-1]), len(lens)
        qkv = self.tensor(T, hq + 2 * hkv, d)
        v = qkv[:, hq + hkv:]
        pos = np.concatenate([np.stack([np.arange(n), np.arange(n) // 7, np.arange(n) % 7]) for n in lens], 1)
        pos = torch.from_numpy(pos.astype(np.int32)).cuda()
        q, k = bacon.bacon_rotate(self.rotary, pos, qkv[:, :hq], qkv[:, hq:hq + hkv])
        self.batch = bacon.BatchLayout(self.cu, budgets)
        self.ctx = bacon.Context(1, hq, hkv, d, W, B, T, dtype, bacon.default_params(pool_kernel=5))
        self.window = torch.empty(B, hq, W, device="cuda")
        self.out = bacon.bacon_prompt_attend(self.ctx.shape, self.batch, q, k, v, window_lse=self.window)[0]
        if chunk is not None:
            self.window = self.window_by_chunks(chunk, q, k, v)
        rows = np.concatenate([np.arange(self.cu[i + 1] - W, self.cu[i + 1]) for i in range(B)])
        self.q_win = q[torch.from_numpy(rows).cuda()].contiguous()
        self.q, self.k, self.v = q, k, v.contiguous()
        self.ctx.bacon_begin_prompt(self.batch)
        self.idx = self.ctx.bacon_compress_layer_lse(0, self.batch, self.q_win, self.k, self.v, self.window)[0]
        most = max(min(x, n - W) + W for x, n in zip(budgets, lens)) + 24
        self.cache = bacon.Cache(1, hq, hkv, d, W, bt, B, most, 2000, dtype, format="e2m1")
        self.cache.memory.fill_(0x7F)
        self.cache.bacon_cache_clear()
        self.cache.bacon_cache_tables(self.batch, None, 24)
        self.cache.bacon_cache_store(self.batch, [self.k], [self.v], [self.idx])
        self.rows = []
        idx, at = self.idx.cpu().numpy(), 0
        kn, vn = _np(self.k), _np(self.v)
        for b in range(B):
            self.rows.append([])
            for h in range(hkv):
                kept = [i for i in idx[at:at + budgets[b]] if i >= 0]
                at += budgets[b]
                p = self.cu[b] + np.array(kept + list(range(lens[b] - W, lens[b])))
                self.rows[b].append([A.held(kn[p, h]), A.held(vn[p, h])])

    def window_by_chunks(self, chunks, q, k, v):
        """One buffer through the prompts' chunks, each a number of every prompt's next tokens."""
        import torch
        from paper_2606_14782_amd import bacon
        window = torch.full_like(self.window, float("nan"))
        at = [0] * len(self.lens)
        for sizes in chunks:
            to = [a + m for a, m in zip(at, sizes)]
            rows = torch.cat([q[c + a:c + e] for c, a, e in zip(self.cu, at, to)])
            keys, values = (torch.cat([x[c:c + e] for c, e in zip(self.cu, to)]) for x in (k, v))
            batch = bacon.BatchLayout(np.concatenate([[0], np.cumsum(to)]), [1] * len(to))
            bacon.bacon_prompt_attend(self.ctx.shape, batch, rows, keys, values, np.concatenate([[0], np.cumsum(sizes)]),
                                      window_lse=window, window_ends=self.lens)
            at = to
        assert at == list(self.lens)
        return window

    def tensor(self, *shape):
        import torch
        return torch.from_numpy(self.rng.standard_normal(shape).astype(np.float32)).cuda().to(self.tdt)

    def token(self, i):
        """The i-th new token of every sequence, rotated: q, k, v [B, 1, .., d]."""
        import torch
        from paper_2606_14782_amd import bacon
        B = len(self.lens)
        qkv = self.tensor(B, 1, self.hq + 2 * self.hkv, self.d)
        pos = torch.tensor([[n + i] for n in self.lens], dtype=torch.int32, device="cuda").expand(3, B, 1).contiguous()
        return qkv, pos

    def step(self, qkv, pos):
        from paper_2606_14782_amd import bacon
        q, k = bacon.bacon_rotate(self.rotary, pos, qkv[:, :, :self.hq], qkv[:, :, self.hq:self.hq + self.hkv])
        out, lse = self.cache.bacon_cache_step(0, q, k, qkv[:, :, self.hq + self.hkv:], want_lse=True)
        return q, k, out, lse

    def check(self, qkv, q, k, out, lse):
        qn, kn, vn, on, ln = _np(q), _np(k), _np(qkv[:, :, self.hq + self.hkv:]), _np(out), _np(lse)
        for b in range(len(self.lens)):
            for h in range(self.hkv):
                for kv, x in ((0, kn), (1, vn)):
                    self.rows[b][h][kv] = np.concatenate([self.rows[b][h][kv], A.held(x[b, :, h])])
            for h in range(self.hq):
                kr, vr = self.rows[b][h * self.hkv // self.hq]
                o, s, tol, stol = A.attend_held(R.attend, qn[b, 0, h], kr, vr, self.dtype)
                assert np.all(np.abs(on[b, 0, h] - o) <= tol), (b, h, float((np.abs(on[b, 0, h] - o) / tol).max()))
                assert abs(ln[b, 0, h] - s) <= stol, (b, h)


CASES = [("bf16", 128, 8, 2, [300, 1000, 65], [64, 128, 300]), ("fp32", 64, 6, 3, [200, 90], [50, 20]),
         ("bf16", 64, 4, 4, [700], [100])]


@pytest.mark.parametrize("dtype,d,hq,hkv,lens,budgets", CASES)
def test_prompt_to_decoding(dtype, d, hq, hkv, lens, budgets):
    import torch
    m = Layer(dtype, d, hq, hkv, lens, budgets)
    # the normalisers are the library's own pass's, up to two sums of different order
    own = _np(m.ctx.bacon_window_lse(m.batch, m.q_win, m.k))
    got = _np(m.window)
    size = max(np.abs(_np(m.q_win)).sum(-1).max() * np.abs(_np(m.k)).max() / np.sqrt(d), 1.0)
    # (each: a logit of d products, its exponential, a sum over chains of n / 2 + 64 terms)
    bound = 2 * ((d + 8) * size + max(lens) / 2 + 64 + 64) * A.h + 8 * A.h * np.abs(own)
    assert np.all(np.abs(got - own) <= bound), float((np.abs(got - own) / bound).max())
    # and the kept sets theirs, but for what the difference moves over the border
    m.ctx.bacon_begin_prompt(m.batch)
    idx = m.ctx.bacon_compress_layer_lse(0, m.batch, m.q_win, m.k, m.v, torch.from_numpy(own).float().cuda())[0]
    at = 0
    for b, n in enumerate(budgets):
        for h in range(hkv):
            x, y = (set(t[at:at + n].tolist()) for t in (idx, m.idx))
            assert len(x ^ y) <= 2, (b, h, len(x ^ y))
            at += n
    k, v = m.cache.bacon_cache_load(max(len(r[0][0]) for r in m.rows))
    for b in range(len(lens)):
        for h in range(hkv):
            for t, x in ((k, m.rows[b][h][0]), (v, m.rows[b][h][1])):
                np.testing.assert_array_equal(_np(t)[0, b, h, :len(x)], x)
    for i in range(18):
        qkv, pos = m.token(i)
        m.check(qkv, *m.step(qkv, pos))
    assert m.cache.bacon_cache_errors() == 0


def test_captured_decoding_on_another_stream():
    """A rotation and a step in one graph, replayed between eager work, against the
    same tokens run eagerly in a second cache: bit for bit."""
    import torch
    a, b = Layer(*CASES[0], seed=5), Layer(*CASES[0], seed=5)
    qkv, pos = a.token(0)
    b.token(0)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        a.step(qkv, pos)
        a.cache.bacon_cache_advance(-1)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            _, _, out, lse = a.step(qkv, pos)
    torch.cuda.current_stream().wait_stream(stream)
    for i in range(5):
        x, p = b.token(i)
        qkv.copy_(x)
        pos.copy_(p)
        g.replay()
        _, _, want, wlse = b.step(x, p)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, wlse), i
        assert torch.equal(a.cache.lens, b.cache.lens)


def test_a_pool_beyond_32_bits_of_bytes():
    """Block ids whose codes and scales lie past 2^32 bytes."""
    import torch
    from paper_2606_14782_amd import bacon
    d, bt, blocks = 128, 64, 600_000                                    # 4.9 GB of codes
    c = bacon.Cache(1, 4, 1, d, 1, bt, 1, 1000, blocks, "bf16", format="e2m1")
    c.bacon_cache_clear()
    rng = np.random.default_rng(9)
    free = torch.arange(blocks - 1, blocks - 20, -1, dtype=torch.int32, device="cuda")
    batch = bacon.BatchLayout([0, 700], [699])
    c.bacon_cache_tables(batch, None, 64, free)
    k, v, kn, vn = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda().bfloat16() for s in
                    ((700, 1, d), (700, 1, d), (1, 2, 1, d), (1, 2, 1, d)))
    c.bacon_cache_store(batch, [k], [v])
    c.bacon_cache_append(0, kn, vn)
    want = [A.held(np.concatenate([_np(x)[:, 0], _np(y)[0, :, 0]])) for x, y in ((k, kn), (v, vn))]
    for got, w in zip(c.bacon_cache_load(702), want):
        np.testing.assert_array_equal(_np(got)[0, 0, 0], w)
    q = torch.from_numpy(rng.standard_normal((1, 1, 4, d)).astype(np.float32)).cuda().bfloat16()
    out, lse = c.bacon_cache_attend(0, q, want_lse=True)
    for h in range(4):
        o, s, tol, stol = A.attend_held(R.attend, _np(q)[0, 0, h], *want, "bf16")
        assert np.all(np.abs(_np(out)[0, 0, h] - o) <= tol) and abs(float(lse[0, 0, h]) - s) <= stol


@pytest.mark.parametrize("case,chunk", [
    (CASES[0], [[200, 997, 60], [95, 2, 0], [4, 0, 5], [1, 1, 0]]), (CASES[1], [[193, 89], [7, 1]]),
    (CASES[2], [[64], [635], [1]])])
def test_prompt_in_chunks_to_decoding(case, chunk, monkeypatch):
    """The last chunks shorter than the window, one of a single token: the window's
    normalisers, the kept sets and the decoding as of whole prompts."""
    whole = Layer
    monkeypatch.setitem(globals(), "Layer", lambda *a, **kw: whole(*a, chunk=chunk, **kw))
    test_prompt_to_decoding(*case)
