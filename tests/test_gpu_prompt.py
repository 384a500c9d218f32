"""The prompt's attention on the GPU against plain 64-bit numpy (around_ref),
with the bounds that it derives from the arithmetic."""
import numpy as np
import pytest

import around_ref as A

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_14782_amd import bacon
    bacon.lib()


def _rand(rng, *shape, dtype="bf16", scale=1.0):
    import torch
    x = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).cuda()
    return x.to(torch.bfloat16) if dtype == "bf16" else x


def _np(t):
    return t.double().cpu().numpy()


def _shape(hq, hkv, d, W, dtype, batch=64, most=1 << 30):
    from paper_2606_14782_amd import bacon
    return bacon.Shape(1, hq, hkv, d, W, batch, most, bacon.BF16 if dtype == "bf16" else bacon.FP32)


def _cu(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def _batch(lens):
    from paper_2606_14782_amd import bacon
    return bacon.BatchLayout(_cu(lens), [1] * len(lens))


MARK = 123.0


def _check(q, k, v, lens, queries, W, dtype, out, lse, window, heads=None):
    """Against the reference, all heads or some; window entries that are no query hold MARK."""
    hq, hkv = q.shape[1], k.shape[1]
    qn, kn, vn, on, ln, wn = _np(q), _np(k), _np(v), _np(out), _np(lse), _np(window)
    cu, cuq = _cu(lens), _cu(queries)
    for b, (n, m) in enumerate(zip(lens, queries)):
        ends = np.clip(n - m + 1 + np.arange(m), 0, n)
        for h in range(hq) if heads is None else heads:
            kv = h * hkv // hq
            rows, keys = slice(cuq[b], cuq[b + 1]), slice(cu[b], cu[b + 1])
            o, s, tol, stol = A.attend(qn[rows, h], kn[keys, kv], vn[keys, kv], ends, dtype)
            err = np.abs(on[rows, h] - o)
            where = (b, n, m, h)
            assert np.all(err <= tol), (where, float((err / np.maximum(tol, 1e-300)).max()), np.argwhere(err > tol)[:3])
            none = ends <= 0
            assert np.all(on[rows, h][none] == 0) and np.all(ln[rows, h][none] == -np.inf), where
            assert np.all(np.abs(ln[rows, h][~none] - s[~none]) <= stol[~none]), where
            w = np.arange(W) + m - W
            held = w >= 0
            np.testing.assert_array_equal(wn[b, h][held], ln[rows, h][w[held]])
            assert np.all(wn[b, h][~held] == MARK), where


def _run(rng, hq, hkv, d, dtype, lens, queries=None, W=8, scale=1.0, heads=None):
    import torch
    from paper_2606_14782_amd import bacon
    m = lens if queries is None else queries
    T, Tq = int(sum(lens)), int(sum(m))
    q = _rand(rng, Tq, hq, d, dtype=dtype, scale=scale)
    kv = _rand(rng, T + 3, 2 * hkv, d, dtype=dtype)
    kv[T:] = float("nan")                                       # rows behind the last sequence
    k, v = kv[:, :hkv], kv[:, hkv:]
    window = torch.full((len(lens), hq, W), MARK, device="cuda")
    out, lse, w = bacon.bacon_prompt_attend(_shape(hq, hkv, d, W, dtype), _batch(lens), q, k, v,
                                            None if queries is None else _cu(queries), want_lse=True, window_lse=window)
    assert w is window
    _check(q, k[:T], v[:T], lens, m, W, dtype, out, lse, window, heads)
    return q, k, v, out, lse


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 2), (6, 2), (7, 1), (8, 1)])
def test_lengths(dtype, d, hq, hkv):
    """One token to several tiles, around the borders of tiles and of rows."""
    rng = np.random.default_rng(hq)
    _run(rng, hq, hkv, d, dtype, [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 0, 257])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 64), (14, 2, 64), (28, 4, 128), (32, 1, 128), (96, 2, 64)])
def test_chunks(dtype, hq, hkv, d):
    """The prompts' last tokens as queries, from one on; none; more than there are keys; no keys at all."""
    rng = np.random.default_rng(hkv)
    lens = [300, 64, 65, 1, 130, 90, 40, 0, 500]
    _run(rng, hq, hkv, d, dtype, lens, [1, 64, 2, 1, 129, 0, 47, 5, 33], W=32, heads=[0, hq // 2, hq - 1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,queries", [([3000], None), ([5000, 900], [1, 900]), ([2500, 4097, 64], [70, 130, 3])])
def test_divided_keys(dtype, lens, queries):
    """Few query rows over long prompts: parts of the keys, joined."""
    from paper_2606_14782_amd import bacon
    import ctypes as C
    cuq = None if queries is None else _cu(queries)
    need = bacon.lib().bacon_prompt_work_bytes(C.byref(_shape(4, 2, 128, 16, dtype)), C.byref(_batch(lens).c),
                                               None if cuq is None else cuq.ctypes.data)
    assert need > 0
    _run(np.random.default_rng(len(lens)), 4, 2, 128, dtype, lens, queries, W=16)


@pytest.mark.parametrize("scale", [1.0, 30.0])
@pytest.mark.parametrize("hq,hkv,d,lens,queries", [
    (28, 4, 128, [1000], None), (32, 8, 64, [1500, 70, 0, 33], None), (14, 2, 64, [2077], None),
    (28, 4, 128, [1601, 40], [700, 50]), (16, 16, 128, [2050], None)])
def test_long_rows_on_an_emptier_gpu(hq, hkv, d, lens, queries, scale):
    """Where the longest rows are what a call waits for and nothing is divided: odd
    and even numbers of tiles, rows of one tile, sequences of none."""
    from paper_2606_14782_amd import bacon
    import ctypes as C
    cuq = None if queries is None else _cu(queries)
    need = bacon.lib().bacon_prompt_work_bytes(C.byref(_shape(hq, hkv, d, 16, "bf16")), C.byref(_batch(lens).c),
                                               None if cuq is None else cuq.ctypes.data)
    assert need == 0
    _run(np.random.default_rng(d), hq, hkv, d, "bf16", lens, queries, W=16, scale=scale, heads=[0, hq // 2, hq - 1])


def test_many_units():
    """More workgroups than the GPU holds at once: nothing divided."""
    _run(np.random.default_rng(3), 64, 8, 64, "bf16", [700] * 12, heads=[0, 13, 63])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [30.0, 1e-3])
def test_sharp_and_flat_logits(dtype, scale):
    """Maxima that move by hundreds from key to key, and weights that are all alike."""
    _run(np.random.default_rng(4), 4, 2, 128, dtype, [400, 129], scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_logits_of_any_finite_size(dtype):
    """Equal logits far past 2^31 keep equal weights; the largest alone counts where they differ."""
    import torch
    from paper_2606_14782_amd import bacon
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    n, d = 150, 64
    q, k = torch.zeros(n, 1, d, dtype=t, device="cuda"), torch.zeros(n, 1, d, dtype=t, device="cuda")
    v = _rand(np.random.default_rng(5), n, 1, d, dtype=dtype)
    q[..., 0], k[..., 0] = 2.0 ** 60, 2.0 ** 55
    out, lse, _ = bacon.bacon_prompt_attend(_shape(1, 1, d, 1, dtype), _batch([n]), q, k, v, want_lse=True)
    want = np.cumsum(_np(v)[:, 0], 0) / np.arange(1, n + 1)[:, None]
    mass = np.cumsum(np.abs(_np(v)[:, 0]), 0) / np.arange(1, n + 1)[:, None]
    assert np.all(np.abs(_np(out)[:, 0] - want) <= A.HALF[dtype] * np.abs(want) + 200 * A.h * mass)
    assert np.all(_np(lse) == 2.0 ** 112)
    k[40, 0, 0] = 2.0 ** 56
    out, _, _ = bacon.bacon_prompt_attend(_shape(1, 1, d, 1, dtype), _batch([n]), q, k, v)
    assert torch.equal(out[40:], v[40:41].expand(n - 40, 1, d))
    k[:] = 0
    k[..., 0] = -2.0 ** 65                                      # far below zero: 2^125 / 8
    out, lse, _ = bacon.bacon_prompt_attend(_shape(1, 1, d, 1, dtype), _batch([n]), q, k, v, want_lse=True)
    assert np.all(np.abs(_np(out)[:, 0] - want) <= A.HALF[dtype] * np.abs(want) + 200 * A.h * mass)
    assert np.all(_np(lse) == -2.0 ** 122)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,queries", [([200], None), ([900, 70], [30, 70])])
def test_keys_and_values_that_are_not_finite(dtype, d, lens, queries):
    """They reach the queries that see them, and no others (of the same tile, row
    and workgroup): earlier queries, other heads, other sequences."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(6)
    hq, hkv, W = 4, 2, 4
    T, m = sum(lens), lens if queries is None else queries
    q, k, v = (_rand(rng, n, h, d, dtype=dtype) for n, h in ((sum(m), hq), (T, hkv), (T, hkv)))
    call = lambda: bacon.bacon_prompt_attend(_shape(hq, hkv, d, W, dtype), _batch(lens), q, k, v,  # noqa: E731
                                             None if queries is None else _cu(queries), want_lse=True)[:2]
    clean, clean_lse = call()
    for name, bad, at in (("v", float("nan"), lens[0] - 20), ("v", -float("inf"), lens[0] - 9),
                          ("k", float("nan"), lens[0] - 15)):
        x = {"k": k, "v": v}[name]
        old = x[at, 1].clone()
        x[at, 1, 3] = bad
        out, lse = call()
        first = m[0] - (lens[0] - at)                           # the first query that sees it
        unseen = torch.ones(sum(m), hq, dtype=torch.bool, device="cuda")
        unseen[first:m[0], 2:] = False
        assert torch.equal(out[unseen], clean[unseen]) and torch.equal(lse[unseen], clean_lse[unseen]), (name, bad)
        hit = out[first:m[0], 2:]
        if name == "v":
            assert not torch.isfinite(hit[..., 3]).any()
            keep = [i for i in range(d) if i != 3]
            assert torch.equal(hit[..., keep], clean[first:m[0], 2:][..., keep])
        else:
            assert torch.isnan(hit).all()
        x[at, 1] = old
    # a query that is not finite is NaN alone
    for bad in (float("nan"), float("inf")):
        q[5, 2, 0] = bad
        out, _ = call()
        assert torch.isnan(out[5, 2]).all()
        rest = torch.ones(sum(m), hq, dtype=torch.bool, device="cuda")
        rest[5, 2] = False
        assert torch.equal(out[rest], clean[rest])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("at", [5, 1700, 2955, 2990])
@pytest.mark.parametrize("hq,queries", [(2, None), (2, [3000 - 2900]), (14, None)])
def test_values_that_are_not_finite_far_back(dtype, at, hq, queries):
    """Of a key in tiles that mask none, in a part of the keys, and in the last tile."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(8)
    n, d, m = 3000, 128, 3000 if queries is None else queries[0]
    q, k, v = (_rand(rng, t, h, d, dtype=dtype) for t, h in ((m, hq), (n, hq // 2), (n, hq // 2)))
    call = lambda: bacon.bacon_prompt_attend(_shape(hq, hq // 2, d, 4, dtype), _batch([n]), q, k, v,  # noqa: E731
                                             None if queries is None else _cu(queries), want_lse=True)[:2]
    clean, clean_lse = call()
    v[at, -1, 7] = float("inf")
    out, lse = call()
    first = max(m - (n - at), 0)                                # the first query that sees it
    assert torch.equal(out[:first], clean[:first]) and torch.equal(lse, clean_lse)
    assert torch.equal(out[:, :-2], clean[:, :-2])
    assert not torch.isfinite(out[first:, -2:, 7]).any()
    keep = [i for i in range(d) if i != 7]
    assert torch.equal(out[first:][..., keep], clean[first:][..., keep])


def test_views_strides_and_guards():
    """q, k, v as parts of one projection's output; outputs between guards."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(7)
    hq, hkv, d, W, lens = 6, 2, 128, 16, [70, 130]
    T = sum(lens)
    qkv = _rand(rng, T, hq + 2 * hkv, d)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    shape, batch = _shape(hq, hkv, d, W, "bf16"), _batch(lens)
    want, want_lse, want_w = bacon.bacon_prompt_attend(shape, batch, q.contiguous(), k.contiguous(), v.contiguous(),
                                                       want_lse=True, want_window_lse=True)
    buf, lbuf, wbuf = (torch.full((n + 16,), 5.0, device="cuda", dtype=t) for n, t in
                       ((T * hq * d, torch.bfloat16), (T * hq, torch.float32), (2 * hq * W, torch.float32)))
    out, lse, w = buf[8:-8].view(T, hq, d), lbuf[8:-8].view(T, hq), wbuf[8:-8].view(2, hq, W)
    bacon.bacon_prompt_attend(shape, batch, q, k, v, out=out, lse=lse, window_lse=w)
    assert torch.equal(out, want) and torch.equal(lse, want_lse) and torch.equal(w, want_w)
    for x in (buf, lbuf, wbuf):
        assert (x[:8] == 5).all() and (x[-8:] == 5).all()


def test_window_fills_chunk_by_chunk():
    """The window's normalisers from chunks that end inside it are the whole prompt's."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(8)
    hq, hkv, d, W, n = 4, 2, 64, 32, 220
    q, k, v = (_rand(rng, n, h, d) for h in (hq, hkv, hkv))
    shape = _shape(hq, hkv, d, W, "bf16")
    want = bacon.bacon_prompt_attend(shape, _batch([n]), q, k, v, want_window_lse=True)[2]
    window = torch.full((1, hq, W), MARK, device="cuda")
    outs, at = [], 0
    for m in (100, 95, 1, 24):
        end = at + m
        # the window is the whole prompt's: a chunk's own tokens before its end shift it
        w = torch.full((1, hq, W), MARK, device="cuda")
        out, _, _ = bacon.bacon_prompt_attend(shape, _batch([end]), q[at:end], k[:end], v[:end], queries=[0, m],
                                              window_lse=w)
        assert (w[..., :max(0, W - m)] == MARK).all()
        shift = n - end
        if shift < W:
            window[..., max(0, W - m - shift):W - shift] = w[..., max(shift, W - m):]
        outs.append(out)
        at = end
    whole = bacon.bacon_prompt_attend(shape, _batch([n]), q, k, v)[0]
    assert np.abs(_np(window) - _np(want)).max() <= 200 * A.h * np.abs(_np(want)).max()
    assert np.abs(_np(torch.cat(outs)) - _np(whole)).max() <= 2.0 ** -6


def test_same_bits_again_on_streams_and_in_graphs():
    """Nothing depends on the order of workgroups: calls side by side on two
    streams, and graphs that own their scratch, repeat the eager call's bits."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(9)
    hq, hkv, d, W, lens, queries = 8, 2, 128, 16, [4000, 300, 77], [40, 300, 1]
    shape, batch, cuq = _shape(hq, hkv, d, W, "bf16"), _batch(lens), _cu(queries)
    sets = [[_rand(rng, n, h, d) for n, h in ((sum(queries), hq), (sum(lens), hkv), (sum(lens), hkv))] for _ in range(3)]
    run = lambda s: bacon.bacon_prompt_attend(shape, batch, *s, queries=cuq, want_lse=True, want_window_lse=True)[:2]  # noqa: E731
    want = [run(s) for s in sets]
    for s, w in zip(sets, want):
        assert all(torch.equal(a, b) for a, b in zip(run(s), w))
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for st, s in zip(streams, sets):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            got.append([run(s) for _ in range(4)][-1])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w))
    graphs = []
    for _ in range(2):
        x = [t.clone() for t in sets[2]]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = run(x)
        graphs.append((g, x, y))
    for i in (0, 1, 2, 0):
        for j, (g, x, y) in enumerate(graphs):
            for a, b in zip(x, sets[(i + j) % 3]):
                a.copy_(b)
        for g, _, _ in graphs:
            g.replay()
        run(sets[1])
        torch.cuda.synchronize()
        for j, (g, x, y) in enumerate(graphs):
            assert all(torch.equal(a, b) for a, b in zip(y, want[(i + j) % 3]))


def test_rows_far_into_memory():
    """Row offsets past 2^31 elements."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(10)
    d, n, gap = 64, 150, 1 << 24
    big = torch.zeros(n * gap + 64, dtype=torch.bfloat16, device="cuda")
    x = _rand(rng, n, 2, d)
    q = _rand(rng, n, 1, d)
    kv = big[:n * gap].view(n, gap)[:, :2 * d].unflatten(1, (2, d))
    kv.copy_(x)
    shape = _shape(1, 1, d, 4, "bf16")
    want = bacon.bacon_prompt_attend(shape, _batch([n]), q, x[:, :1].contiguous(), x[:, 1:].contiguous())[0]
    assert torch.equal(bacon.bacon_prompt_attend(shape, _batch([n]), q, kv[:, :1], kv[:, 1:])[0], want)


def test_binding_refuses():
    import torch
    from paper_2606_14782_amd import bacon
    shape, batch = _shape(4, 2, 64, 8, "bf16"), _batch([5, 7])
    q = torch.zeros(12, 4, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(12, 2, 64, dtype=torch.bfloat16, device="cuda")
    ok = dict(shape=shape, batch=batch, q=q, k=k, v=k)
    bacon.bacon_prompt_attend(**ok)
    f = dict(device="cuda", dtype=torch.float32)
    bad = [dict(q=q.float()), dict(k=k.cpu()), dict(v=k[:11]), dict(q=q[:11]), dict(k=k[:, :1]), dict(q=q[None]),
           dict(queries=[0, 5]), dict(queries=[0, 5, 13]), dict(queries=[0, 5, 4]), dict(queries=[1, 5, 7]),
           dict(out=torch.zeros(12, 4, 64, **f)), dict(out=q[:11]), dict(lse=torch.zeros(12, 2, **f)),
           dict(window_lse=torch.zeros(2, 4, 7, **f)), dict(batch=_batch([13])),
           dict(shape=_shape(4, 2, 64, 8, "bf16", batch=1)), dict(shape=_shape(4, 2, 64, 8, "bf16", most=11)),
           dict(shape=_shape(4, 2, 96, 8, "bf16"))]
    for kw in bad:
        with pytest.raises(bacon.BaconError):
            bacon.bacon_prompt_attend(**{**ok, **kw})
    long = _batch([5000])
    q, k = (torch.zeros(n, h, 64, dtype=torch.bfloat16, device="cuda") for n, h in ((1, 4), (5000, 2)))
    with pytest.raises(bacon.BaconError):
        bacon.bacon_prompt_attend(shape, long, q, k, k, [0, 1], work=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    bacon.bacon_prompt_attend(shape, _batch([0, 0]), q[:0], k[:0], k[:0])     # nothing to do


CHUNKED = [
    ("bf16", 4, 2, 64, 32, [220], [[200], [20]]),
    ("bf16", 4, 2, 64, 32, [220], [[100], [95], [1], [24]]),
    ("fp32", 6, 2, 128, 8, [130, 9], [[129, 4], [1, 0], [0, 5]]),
    ("fp32", 4, 4, 64, 16, [40, 10], [[25, 3], [14, 6], [1, 1]]),              # a prompt shorter than the window
    ("bf16", 4, 2, 128, 16, [5003, 700], [[4990, 690], [9, 1], [1, 0], [3, 9]]),  # keys divided
    ("fp32", 4, 2, 128, 16, [5003], [[4990], [9], [1], [3]]),
    ("bf16", 28, 4, 128, 32, [1601], [[1590], [11]]),                           # two sets of waves, then divided keys
]


def _chunks(rng, dtype, hq, hkv, d, W, lens):
    """A function of a call's chunk of every prompt, and the prompts themselves."""
    import torch
    from paper_2606_14782_amd import bacon
    q, k, v = ([_rand(rng, n, h, d, dtype=dtype) for n in lens] for h in (hq, hkv, hkv))
    shape = _shape(hq, hkv, d, W, dtype)

    def call(at, sizes, window, ends):
        to = [a + m for a, m in zip(at, sizes)]
        parts = [torch.cat([x[:e] for x, e in zip(t, to)]) for t in (k, v)]
        rows = torch.cat([x[a:e] for x, a, e in zip(q, at, to)])
        return bacon.bacon_prompt_attend(shape, _batch(to), rows, *parts, _cu(sizes), window_lse=window,
                                         window_ends=ends)[0]

    return call, q, k


@pytest.mark.parametrize("dtype,hq,hkv,d,W,lens,chunks", CHUNKED)
def test_one_window_for_all_chunks(dtype, hq, hkv, d, W, lens, chunks):
    """Chunks of any sizes, the last ones shorter than the window, leave in one buffer
    what a call over the whole prompts leaves there; a call repeated changes nothing."""
    import torch
    rng = np.random.default_rng(W + d)
    call, q, k = _chunks(rng, dtype, hq, hkv, d, W, lens)
    window = torch.full((len(lens), hq, W), MARK, device="cuda")
    at = [0] * len(lens)
    for sizes in chunks:
        call(at, sizes, window, lens)
        at = [a + m for a, m in zip(at, sizes)]
        now = window.clone()
        call([a - m for a, m in zip(at, sizes)], sizes, window, np.array(lens))
        assert torch.equal(now, window)
        for b, n in enumerate(lens):                            # filled up to the tokens so far, and no further
            w = min(max(at[b] - (n - W), max(0, W - n)), W)
            assert (window[b, :, w:] == MARK).all()
    assert at == lens
    got = _np(window)
    for b, n in enumerate(lens):
        m = min(n, W)
        assert np.all(got[b, :, :W - m] == MARK)
        qn, kn = _np(q[b]), _np(k[b])
        for h in range(hq):
            key = kn[:, h * hkv // hq]
            _, s, _, tol = A.attend(qn[n - m:, h], key, key, np.arange(n - m + 1, n + 1), dtype)
            err = np.abs(got[b, h, W - m:] - s)
            assert np.all(err <= tol), (b, h, float((err / tol).max()))


def test_window_of_a_chunk_that_ends_before_it():
    """Windows that are still to come, the furthest among them, and none named."""
    import torch
    call, _, _ = _chunks(np.random.default_rng(3), "bf16", 4, 2, 64, 16, [90])
    window = torch.full((1, 4, 16), MARK, device="cuda")
    for end in (106, 200, 2 ** 31 - 1):
        out = call([0], [90], window, [end])
        assert (window == MARK).all()
    assert torch.equal(call([0], [90], window, [105]), out)
    assert (window[..., 1:] == MARK).all() and (window[..., 0] != MARK).all()
    whole = torch.full((1, 4, 16), MARK, device="cuda")
    assert torch.equal(call([0], [90], whole, None), out)
    named = torch.full((1, 4, 16), MARK, device="cuda")
    call([0], [90], named, [90])
    assert torch.equal(whole, named) and torch.equal(window[..., 0], whole[..., -1])


def test_captured_chunks_fill_one_window():
    """The chunks' calls in one graph, replayed on other inputs between eager work."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(4)
    hq, hkv, d, W, n = 4, 2, 64, 32, 220
    shape = _shape(hq, hkv, d, W, "bf16")
    inputs = [[_rand(rng, n, h, d) for h in (hq, hkv, hkv)] for _ in range(3)]
    window = torch.full((1, hq, W), MARK, device="cuda")

    def chunks(q, k, v, window):
        for a, e in ((0, 200), (200, 219), (219, 220)):
            bacon.bacon_prompt_attend(shape, _batch([e]), q[a:e], k[:e], v[:e], [0, e - a], window_lse=window, window_ends=[n])

    x = [t.clone() for t in inputs[0]]
    chunks(*x, window)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        chunks(*x, window)
    for i in (1, 2, 0, 1):
        want = torch.full((1, hq, W), MARK, device="cuda")
        chunks(*inputs[i], want)
        for t, y in zip(x, inputs[i]):
            t.copy_(y)
        window.fill_(MARK)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(window, want) and not (window == MARK).any()


def test_binding_refuses_window_ends():
    import torch
    from paper_2606_14782_amd import bacon
    q, k = (torch.zeros(12, h, 64, dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    for ends in ([5], [5, 7, 9], [4, 7], [5, 6], [[5, 7]], 12):
        with pytest.raises(bacon.BaconError):
            bacon.bacon_prompt_attend(_shape(4, 2, 64, 8, "bf16"), _batch([5, 7]), q, k, k, window_ends=ends)
    bacon.bacon_prompt_attend(_shape(4, 2, 64, 8, "bf16"), _batch([5, 7]), q, k, k, window_ends=[5, 9])
