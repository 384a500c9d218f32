"""The 8-bit cache on the GPU against plain 64-bit numpy (cache_ref).

Tables, stored and appended values are exact (scales are powers of two and
every rounding is to nearest even).  Attention is held to the bounds that
cache_ref.attend derives from the arithmetic.  Blocks that hold no row carry
NaN codes and NaN scales throughout: nothing of them may reach a result."""
import math

import numpy as np
import pytest

import cache_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_14782_amd import bacon
    bacon.lib()


def _cache(L, hq, hkv, d, W, bt, B, most, blocks, dtype):
    """A cleared cache whose pool holds NaN codes and scales."""
    from paper_2606_14782_amd import bacon
    c = bacon.Cache(L, hq, hkv, d, W, bt, B, most, blocks, dtype)
    c.memory.fill_(0x7F)
    c.scales.fill_(float("nan"))
    c.bacon_cache_clear()
    return c


def _rand(rng, *shape, dtype="bf16", scale=1.0):
    import torch
    x = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).cuda()
    return x.to(torch.bfloat16) if dtype == "bf16" else x


def _np(t):
    return t.double().cpu().numpy()


class Model:
    """A cache of one layer with given lengths of every pair, and the same
    rows in cache_ref: filled through tables and store."""

    def __init__(self, lens, hq, d, bt, dtype, reserve=40, seed=0, layers=1, shuffle=True, W=1, scale=1.0):
        import torch
        from paper_2606_14782_amd import bacon
        self.rng = np.random.default_rng(seed)
        lens = np.asarray(lens)                                    # [B, Hkv], each >= W
        B, H = lens.shape
        self.B, self.H, self.hq, self.d, self.bt, self.dtype, self.W = B, H, hq, d, bt, dtype, W
        N = np.maximum(lens.max(1), W) + 1                         # candidates enough for every head
        cu = np.concatenate([[0], np.cumsum(N)])
        need = layers * int(((lens + reserve + bt - 1) // bt).sum())
        blocks = need + 5
        self.c = _cache(layers, hq, H, d, W, bt, B, int(lens.max()) + reserve, blocks, dtype)
        free = self.rng.permutation(blocks) if shuffle else np.arange(blocks)
        self.batch = bacon.BatchLayout(cu, np.ones(B))
        bud = torch.from_numpy(np.broadcast_to(lens - W, (layers, B, H)).astype(np.int32).copy()).cuda()
        used = self.c.bacon_cache_tables(self.batch, bud, reserve, torch.from_numpy(free.astype(np.int32)).cuda())
        assert int(used) == need
        k = _rand(self.rng, layers, int(cu[-1]), H, d, dtype=dtype, scale=scale)
        v = _rand(self.rng, layers, int(cu[-1]), H, d, dtype=dtype)
        self.c.bacon_cache_store(self.batch, list(k), list(v))
        self.rows = []                                             # [layer][b][h] -> (K rows, V rows)
        kn, vn = _np(k), _np(v)
        for l in range(layers):
            self.rows.append([])
            for b in range(B):
                self.rows[l].append([])
                for h in range(H):
                    at = list(range(lens[b, h] - W)) + list(range(N[b] - W, N[b]))
                    pair = []
                    for x in (kn, vn):
                        r = R.Rows(bt, d)
                        r.store(x[l, cu[b]:cu[b + 1], h][at])
                        pair.append(r)
                    self.rows[l][b].append(pair)

    def tokens(self, n, heads, scale=1.0):
        return _rand(self.rng, self.B, n, heads, self.d, dtype=self.dtype, scale=scale)

    def append(self, k, v, counts=None, layer=0):
        kn, vn = _np(k), _np(v)
        for b in range(self.B):
            c = k.shape[1] if counts is None else int(counts[b])
            for h in range(self.H):
                self.rows[layer][b][h][0].append(kn[b, :c, h])
                self.rows[layer][b][h][1].append(vn[b, :c, h])

    def check_values(self, layer=0):
        lens = self.c.lens.cpu().numpy()[layer]
        want_len = [[len(self.rows[layer][b][h][0]) for h in range(self.H)] for b in range(self.B)]
        np.testing.assert_array_equal(lens, want_len)
        most = max(1, int(lens.max()))
        k, v = self.c.bacon_cache_load(most, first_layer=layer, num_layers=1)
        for got, kv in ((_np(k)[0], 0), (_np(v)[0], 1)):
            for b in range(self.B):
                for h in range(self.H):
                    r = self.rows[layer][b][h][kv]
                    np.testing.assert_array_equal(got[b, h, :len(r)], r.x, err_msg=f"kv {kv} b {b} h {h}")
                    assert not got[b, h, len(r):].any()

    def check_attend(self, q, out, lse, counts=None, layer=0):
        qn, on, ln = _np(q), _np(out), None if lse is None else _np(lse)
        B, n, G = self.B, q.shape[1], self.hq // self.H
        for b in range(B):
            c = n if counts is None else int(counts[b])
            for j in range(n):
                for hq in range(self.hq):
                    kr, vr = self.rows[layer][b][hq // G]
                    end = max(0, len(kr) - (c - 1 - j)) if j < c else 0
                    o, s, tol, stol = R.attend(qn[b, j, hq], kr.x[:end], vr.x[:end], self.dtype)
                    where = f"b {b} token {j} head {hq} end {end}"
                    assert np.all(np.abs(on[b, j, hq] - o) <= tol), \
                        (where, float(np.max(np.abs(on[b, j, hq] - o) / np.maximum(tol, 1e-300))))
                    if ln is not None:
                        assert ln[b, j, hq] == s if end == 0 else abs(ln[b, j, hq] - s) <= stol, where


# ---------------------------------------------------------------- tables

def _tables_ref(K, N, W, bt, reserve, free, max_blocks):
    """lens, starts, table, used and whether a pair found no blocks; K [L, B, H]."""
    L, B, H = K.shape
    lens, starts = np.zeros((L, B, H), int), np.zeros((L, B, H), int)
    table = np.full((L, B, H, max_blocks), -1)
    at, short = 0, False
    for l in range(L):
        start = 0
        for b in range(B):
            for h in range(H):
                rows = min(K[l, b, h], N[b] - W) + W
                need = -(-(rows + reserve) // bt)
                starts[l, b, h] = start
                start += K[l, b, h]
                if at + need <= len(free) and need <= max_blocks:
                    lens[l, b, h] = rows
                    table[l, b, h, :need] = free[at:at + need]
                else:
                    short = True
                at += need
    return lens, starts, table, at, short


@pytest.mark.parametrize("L,B,H,bt,reserve,kind", [
    (1, 1, 1, 16, 0, "batch"), (2, 3, 4, 32, 64, "batch"), (5, 7, 3, 16, 9, "device"),
    (33, 64, 8, 64, 300, "device"), (3, 5, 4, 16, 7, "short"), (2, 4, 2, 16, 5, "tall"), (4, 2, 8, 32, 0, "sequential"),
])
def test_tables(L, B, H, bt, reserve, kind):
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(L * 100 + B)
    W, N = 8, rng.integers(8, 900, B)
    K = rng.integers(1, 400, (L, B, H))
    budgets = rng.integers(1, 400, B)
    if kind == "batch":
        K = np.broadcast_to(budgets[None, :, None], (L, B, H))
    rows = np.minimum(K, N[None, :, None] - W) + W
    need = -(-(rows + reserve) // bt)
    most = int((rows + reserve).max()) if kind != "tall" else int(np.median(rows + reserve))
    blocks = int(need.sum()) + 4
    c = _cache(L, H, H, 64, W, bt, B, most, blocks, "bf16")
    free = rng.permutation(blocks)
    if kind == "short":
        free = free[:blocks * 2 // 3]
    elif kind == "sequential":
        free = np.arange(blocks)
    # the device's budgets may carry more sequences than the batch
    dev = np.concatenate([K, rng.integers(1, 9, (L, 2, H))], 1).astype(np.int32)
    batch = bacon.BatchLayout(np.concatenate([[0], np.cumsum(N)]), budgets)
    used = c.bacon_cache_tables(batch, None if kind == "batch" else torch.from_numpy(dev).cuda(), reserve,
                                None if kind == "sequential" else torch.from_numpy(free.astype(np.int32)).cuda())
    lens, starts, table, at, short = _tables_ref(K, N, W, bt, reserve, free, c.table.shape[-1])
    np.testing.assert_array_equal(c.lens.cpu().numpy(), lens)
    np.testing.assert_array_equal(c.starts.cpu().numpy(), starts)
    np.testing.assert_array_equal(c.table.cpu().numpy(), table)
    assert int(used) == at
    assert c.bacon_cache_errors() == (bacon.CACHE_NO_BLOCKS if short else 0)
    assert short == (kind in ("short", "tall"))
    c.bacon_cache_clear()
    assert not c.lens.any() and (c.table == -1).all() and c.bacon_cache_errors() == 0


def test_tables_of_one_sequence_leave_the_others():
    import torch
    from paper_2606_14782_amd import bacon
    c = _cache(2, 4, 2, 64, 4, 16, 5, 100, 400, "bf16")
    bud = torch.full((2, 5, 2), 20, dtype=torch.int32, device="cuda")
    c.bacon_cache_tables(bacon.BatchLayout([0, 50, 100, 150, 200, 250], [1] * 5), bud, 10)
    lens, table = c.lens.clone(), c.table.clone()
    free = torch.arange(200, 300, dtype=torch.int32, device="cuda")
    c.bacon_cache_clear(3, 1)
    c.bacon_cache_tables(bacon.BatchLayout([0, 70], [60]), None, 5, free, first_seq=3)
    keep = [0, 1, 2, 4]
    assert torch.equal(c.lens[:, keep], lens[:, keep]) and torch.equal(c.table[:, keep], table[:, keep])
    assert (c.lens[:, 3] == 64).all() and c.table[0, 3, 0, :5].tolist() == [200, 201, 202, 203, 204]
    assert c.bacon_cache_errors() == 0


def test_ids_outside_the_pool_become_absent():
    import torch
    from paper_2606_14782_amd import bacon
    c = _cache(1, 2, 1, 64, 4, 16, 1, 64, 10, "bf16")
    free = torch.tensor([3, 10, -7, 5], dtype=torch.int32, device="cuda")
    c.bacon_cache_tables(bacon.BatchLayout([0, 60], [56]), None, 0, free)
    assert c.table[0, 0, 0].tolist() == [3, -1, -1, 5]
    assert c.bacon_cache_errors() == bacon.CACHE_BAD_BLOCK


# ---------------------------------------------------------- store and load

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,bt", [(64, 16), (64, 64), (128, 16), (128, 32), (128, 64)])
def test_store_whole_rows(dtype, d, bt):
    Model([[1, 15], [16, 17], [63, 64], [65, 200]], 2, d, bt, dtype).check_values()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_store_gathers_idx(dtype):
    """Kept positions with gaps, entries of -1 past the candidates, several
    layers, one sequence short of candidates, into the middle of the cache."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(3)
    L, H, d, W, bt, N, K = 3, 3, 64, 4, 16, [90, 20, 4], [30, 25, 6]
    c = _cache(L, H, H, d, W, bt, 6, 60, 200, dtype)
    cu = np.concatenate([[0], np.cumsum(N)])
    batch = bacon.BatchLayout(cu, K)
    c.bacon_cache_tables(batch, None, 3, first_seq=2)
    k, v = (_rand(rng, L, int(cu[-1]), H, d, dtype=dtype) for _ in range(2))
    idx, kept = [], {}
    for l in range(L):
        e = []
        for b in range(3):
            for h in range(H):
                at = np.sort(rng.permutation(N[b] - W)[:K[b]])
                kept[l, b, h] = np.concatenate([at, np.arange(N[b] - W, N[b])])
                e += list(at) + [-1] * (K[b] - len(at))
        idx.append(torch.tensor(e, dtype=torch.int32, device="cuda"))
    c.bacon_cache_store(batch, list(k[1:]), list(v[1:]), idx[1:], first_seq=2, first_layer=1)
    gk, gv = c.bacon_cache_load(34, first_layer=1, first_seq=2, num_seqs=3)
    for got, src in ((_np(gk), _np(k)), (_np(gv), _np(v))):
        for l in (1, 2):
            for b in range(3):
                for h in range(H):
                    r = R.Rows(bt, d)
                    r.store(src[l, cu[b]:cu[b + 1], h][kept[l, b, h]])
                    np.testing.assert_array_equal(got[l - 1, b, h, :len(r)], r.x)
                    assert not got[l - 1, b, h, len(r):].any()
    assert c.bacon_cache_errors() == 0


def test_store_of_a_bad_index_is_a_zero_row():
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(4)
    c = _cache(1, 1, 1, 64, 2, 16, 1, 32, 4, "fp32")
    batch = bacon.BatchLayout([0, 12], [4])
    c.bacon_cache_tables(batch)
    k, v = (_rand(rng, 12, 1, 64, dtype="fp32") for _ in range(2))
    idx = torch.tensor([0, 11, -1, 1 << 30], dtype=torch.int32, device="cuda")    # 11 is a window row
    c.bacon_cache_store(batch, [k], [v], [idx])
    got = _np(c.bacon_cache_load(6)[0])[0, 0, 0]
    assert got[0].any() and not got[1:4].any() and got[4].any() and got[5].any()
    assert c.bacon_cache_errors() == bacon.CACHE_BAD_INDEX
    # entries past the end of a short idx are not read
    c.bacon_cache_clear()
    c.bacon_cache_tables(batch)
    c.bacon_cache_store(batch, [k], [v], [idx.zero_()[:2]])
    got = _np(c.bacon_cache_load(6)[0])[0, 0, 0]
    assert got[:2].any(1).all() and not got[2:4].any() and got[4:].any(1).all()
    assert c.bacon_cache_errors() == bacon.CACHE_BAD_INDEX


def test_store_of_many_layers():
    """More layers than one launch takes, from lists of separate tensors."""
    m = Model([[5, 20]], 2, 64, 16, "bf16", layers=67)
    for l in (0, 1, 63, 64, 66):
        m.check_values(l)


def test_store_over_the_range_of_magnitudes():
    """Zero blocks, the least and the largest magnitudes, ties and subnormal codes."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(5)
    bt, d, W = 16, 64, 1
    n = bt * 10
    x = rng.standard_normal((n, 1, d)).astype(np.float32)
    x[:bt] = 0
    x[bt:2 * bt] *= 2.0 ** -140
    x[2 * bt:3 * bt] = np.clip(x[2 * bt:3 * bt], -1, 1) * 2.0 ** 127
    x[3 * bt:4 * bt] = rng.integers(-448, 449, (bt, 1, d))
    x[4 * bt:5 * bt] = rng.integers(-64, 65, (bt, 1, d)) * 2.0 ** -11
    x[4 * bt, 0, 0] = 448
    x[5 * bt, 0, 0] = 448 * (1 + 2.0 ** -23)
    x[6 * bt] *= 2.0 ** 20
    x[7 * bt:8 * bt] *= 2.0 ** -60
    c = _cache(1, 1, 1, d, W, bt, 1, n, 10, "fp32")
    batch = bacon.BatchLayout([0, n], [n - W])
    c.bacon_cache_tables(batch)
    t = torch.from_numpy(x).cuda()
    c.bacon_cache_store(batch, [t], [t])
    r = R.Rows(bt, d)
    r.store(x[:, 0].astype(np.float64))
    scales = c.scales.cpu().numpy()[c.table[0, 0, 0].cpu().numpy()]
    np.testing.assert_array_equal(scales, np.exp2(np.array(r.e, np.float64))[:, None].repeat(2, 1))
    k, v = c.bacon_cache_load(n)
    np.testing.assert_array_equal(_np(k)[0, 0, 0], r.x)
    np.testing.assert_array_equal(_np(v)[0, 0, 0], r.x)


@pytest.mark.parametrize("first,count", [(0, 1), (3, 40), (-1, 1), (-20, 20), (-50, 7), (60, 10), (1000, 3)])
def test_load_ranges(first, count):
    m = Model([[5, 70]], 2, 64, 32, "bf16")
    k, _ = m.c.bacon_cache_load(count, first_token=first)
    for h in range(2):
        x = m.rows[0][0][h][0].x
        want = np.zeros((count, 64))
        for i in range(count):
            p = first + i + (len(x) if first < 0 else 0)
            if 0 <= p < len(x):
                want[i] = x[p]
        np.testing.assert_array_equal(_np(k)[0, 0, h], want)


# ---------------------------------------------------------------- append

@pytest.mark.parametrize("dtype,d,bt,n", [("bf16", 128, 16, 1), ("fp32", 64, 32, 1), ("bf16", 64, 64, 5),
                                          ("fp32", 128, 16, 37), ("bf16", 128, 32, 64)])
def test_append(dtype, d, bt, n):
    """Blocks that begin, end and grow; each call's tokens larger than the last's."""
    m = Model([[1, 15, 16], [31, 32, 33], [64, 47, 63]], 3, d, bt, dtype, reserve=3 * n)
    for i, scale in enumerate((0.3, 5.0, 100.0)):
        k, v = m.tokens(n, m.H, scale), m.tokens(n, m.H, 1.0 / scale)
        m.c.bacon_cache_append(0, k, v)
        m.append(k, v)
        m.check_values()
    assert m.c.bacon_cache_errors() == 0


def test_append_counts_and_empty_sequences():
    import torch
    m = Model([[1, 9], [16, 2], [5, 5]], 2, 64, 16, "bf16", layers=2)
    m.c.bacon_cache_advance(-1000, first_seq=0, num_seqs=1)             # sequence 0 becomes empty
    for kv in (0, 1):
        for h in range(2):
            for l in range(2):
                m.rows[l][0][h][kv].cut(0)
    counts = torch.tensor([3, 0, 9], dtype=torch.int32, device="cuda")  # 9 is held to the 4 there are
    k, v = m.tokens(4, 2), m.tokens(4, 2)
    m.c.bacon_cache_append(1, k, v, counts)
    m.append(k, v, [3, 0, 4], layer=1)
    m.check_values(1)
    m.check_values(0)
    neg = torch.tensor([-2, -2, -2], dtype=torch.int32, device="cuda")
    m.c.bacon_cache_append(0, k, v, neg)
    m.check_values(0)


def test_append_without_room_leaves_the_pair():
    from paper_2606_14782_amd import bacon
    m = Model([[16, 10]], 2, 64, 16, "bf16", reserve=0)
    k, v = m.tokens(3, 2), m.tokens(3, 2)
    m.c.bacon_cache_append(0, k, v)                                     # head 0's only block is full
    kn, vn = _np(k), _np(v)
    m.rows[0][0][1][0].append(kn[0, :, 1])
    m.rows[0][0][1][1].append(vn[0, :, 1])
    m.check_values()
    assert m.c.bacon_cache_errors() == bacon.CACHE_NO_BLOCKS


def test_append_one_by_one_equals_the_reference():
    m = Model([[3]], 1, 64, 16, "fp32")
    for i in range(36):
        k, v = m.tokens(1, 1, 1.3 ** i), m.tokens(1, 1, 1.3 ** -i)
        m.c.bacon_cache_append(0, k, v)
        m.append(k, v)
    m.check_values()


# ---------------------------------------------------------------- attend

LENS = [[1, 2], [15, 16], [17, 31], [63, 64], [65, 127], [128, 129], [255, 300], [511, 513]]


@pytest.mark.parametrize("dtype,d,bt,G,n", [
    ("bf16", 128, 64, 1, 1), ("bf16", 128, 32, 4, 1), ("bf16", 64, 16, 7, 1), ("fp32", 64, 32, 4, 1),
    ("fp32", 128, 16, 2, 3), ("bf16", 128, 64, 7, 5), ("bf16", 64, 64, 8, 8), ("fp32", 128, 64, 16, 4),
    ("bf16", 128, 16, 16, 1), ("bf16", 128, 32, 17, 1), ("bf16", 64, 32, 1, 64), ("fp32", 64, 16, 33, 1),
])
def test_attend(dtype, d, bt, G, n):
    m = Model(LENS, 2 * G, d, bt, dtype)
    q = m.tokens(n, 2 * G, 1.5)
    out, lse = m.c.bacon_cache_attend(0, q, want_lse=True)
    m.check_attend(q, out, lse)
    assert m.c.bacon_cache_errors() == 0


@pytest.mark.parametrize("dtype,d,G,n,most", [("bf16", 128, 4, 1, None), ("bf16", 128, 4, 1, 6000),
                                              ("bf16", 64, 7, 3, 100), ("fp32", 128, 2, 2, 6000),
                                              ("bf16", 128, 16, 4, None), ("fp32", 64, 16, 3, None)])
def test_attend_long_and_ragged(dtype, d, G, n, most):
    """Few long pairs (work divided along them) beside short ones, whatever length was expected."""
    m = Model([[5003, 7], [1, 2500]], 2 * G, d, 64, dtype)
    q = m.tokens(n, 2 * G, 2.0)
    out, lse = m.c.bacon_cache_attend(0, q, max_tokens=most, want_lse=True)
    m.check_attend(q, out, lse)


@pytest.mark.parametrize("dtype,d,G,n", [("bf16", 64, 7, 3), ("bf16", 128, 8, 6), ("fp32", 64, 7, 3), ("bf16", 64, 4, 1)])
def test_attend_many_pairs(dtype, d, G, n):
    """128 pairs, a few of them long: long parts, in which more query rows share a workgroup."""
    lens = np.random.default_rng(5).integers(1, 40, (4, 32))
    lens[1, 3], lens[3, 31], lens[0, 0] = 2300, 1100, 513
    m = Model(lens, 32 * G, d, 32, dtype)
    q = m.tokens(n, 32 * G, 1.5)
    m.check_attend(q, *m.c.bacon_cache_attend(0, q, want_lse=True))


def test_attend_over_the_longest():
    """More rows than the longest prompt, of which the last queries see different numbers."""
    m = Model([[131072 + 17]], 4, 64, 64, "bf16")
    q = m.tokens(2, 4, 1.5)
    m.check_attend(q, *m.c.bacon_cache_attend(0, q, want_lse=True))


def test_attend_padded_and_empty():
    """Sequences without rows, padding queries, queries whose mask leaves nothing."""
    import torch
    m = Model([[1, 3], [40, 2], [70, 70], [20, 20]], 4, 64, 16, "bf16")
    m.c.bacon_cache_advance(-5000, first_seq=3, num_seqs=1)
    for h in range(2):
        for kv in (0, 1):
            m.rows[0][3][h][kv].cut(0)
    counts = torch.tensor([4, 2, 0, 3], dtype=torch.int32, device="cuda")
    q = m.tokens(4, 4)
    out = torch.full((4, 4, 4, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    out, lse = m.c.bacon_cache_attend(0, q, counts, out=out, want_lse=True)
    m.check_attend(q, out, lse, counts.tolist())
    assert not out[2].any() and torch.isinf(lse[2]).all() and not out[1, 2:].any()
    assert not out[0, 0].any()              # 1 row, 4 tokens: the first sees none (3 rows: none either)


def test_attend_of_large_and_equal_logits():
    """Logits far apart (weights that vanish) and all equal (weights 1 / n)."""
    m = Model([[300, 90]], 2, 128, 64, "fp32", scale=20.0)
    q = m.tokens(1, 2, 8.0)
    m.check_attend(q, *m.c.bacon_cache_attend(0, q, want_lse=True))
    zero = q * 0
    out, lse = m.c.bacon_cache_attend(0, zero, want_lse=True)
    m.check_attend(zero, out, lse)
    assert abs(float(lse[0, 0, 0]) - math.log(300)) < 1e-5


def test_attend_over_absent_blocks():
    """Table entries outside the pool hide their rows and are noted."""
    from paper_2606_14782_amd import bacon
    m = Model([[100, 40]], 2, 64, 16, "bf16")
    m.c.table[0, 0, 0, 2] = -1
    m.c.table[0, 0, 0, 4] = 1 << 30
    k, v = m.c.bacon_cache_load(100)
    assert m.c.bacon_cache_errors() == bacon.CACHE_BAD_BLOCK
    for t in (k, v):
        rows = t[0, 0, 0].any(-1)
        assert not rows[32:48].any() and not rows[64:80].any() and int(rows.sum()) == 68
    q = m.tokens(1, 2)
    out, lse = m.c.bacon_cache_attend(0, q, want_lse=True)
    assert m.c.bacon_cache_errors() == bacon.CACHE_BAD_BLOCK
    for kv in (0, 1):
        x = m.rows[0][0][0][kv].x
        m.rows[0][0][0][kv].x = np.concatenate([x[:32], x[48:64], x[80:]])
    m.check_attend(q, out, lse)
    for i in range(m.c.table.shape[-1]):
        m.c.table[0, 0, 0, i] = -1
    out, lse = m.c.bacon_cache_attend(0, q, want_lse=True)
    assert not out[0, 0, 0].any() and float(lse[0, 0, 0]) == -math.inf


def test_attend_far_into_the_pool():
    """Block ids whose bytes lie beyond 32 bits."""
    import torch
    from paper_2606_14782_amd import bacon
    d, bt, blocks = 128, 64, 300_000                                    # 4.9 GB of codes
    c = bacon.Cache(1, 4, 1, d, 1, bt, 1, 1000, blocks, "bf16")
    c.bacon_cache_clear()
    rng = np.random.default_rng(9)
    batch = bacon.BatchLayout([0, 700], [699])
    free = torch.arange(blocks - 1, blocks - 20, -1, dtype=torch.int32, device="cuda")
    c.bacon_cache_tables(batch, None, 64, free)
    k, v = (_rand(rng, 700, 1, d) for _ in range(2))
    c.bacon_cache_store(batch, [k], [v])
    kn, vn = _rand(rng, 1, 2, 1, d), _rand(rng, 1, 2, 1, d)
    c.bacon_cache_append(0, kn, vn)
    m = Model([[1]], 4, d, bt, "bf16")
    m.c = c
    for kv, x, new in ((0, k, kn), (1, v, vn)):
        m.rows[0][0][0][kv].store(_np(x)[:, 0])
        m.rows[0][0][0][kv].append(_np(new)[0, :, 0])
    m.check_values()
    q = _rand(rng, 1, 1, 4, d)
    m.check_attend(q, *c.bacon_cache_attend(0, q, want_lse=True))


# ------------------------------------------------------------------ step

@pytest.mark.parametrize("dtype,d,bt,G,n", [("bf16", 128, 64, 4, 1), ("fp32", 64, 16, 1, 1), ("bf16", 64, 32, 7, 4),
                                            ("bf16", 128, 16, 1, 30), ("fp32", 128, 64, 5, 6), ("fp32", 64, 16, 2, 16),
                                            ("bf16", 128, 32, 8, 8), ("fp32", 64, 64, 1, 64)])
def test_step_is_append_then_attend(dtype, d, bt, G, n):
    import torch
    lens = [[1, 16], [15, 700], [64, 63], [200, 33]]
    a, b = Model(lens, 2 * G, d, bt, dtype, reserve=4 * n), Model(lens, 2 * G, d, bt, dtype, reserve=4 * n)
    counts = torch.tensor([n, 1, 0, n], dtype=torch.int32, device="cuda")
    for i, cnt in enumerate((None, counts, None)):
        q, k, v = a.tokens(n, 2 * G), a.tokens(n, 2, 3.0 ** i), a.tokens(n, 2, 3.0 ** i)
        out, lse = a.c.bacon_cache_step(0, q, k, v, cnt, want_lse=True)
        b.c.bacon_cache_append(0, k, v, cnt)
        out2, lse2 = b.c.bacon_cache_attend(0, q, cnt, want_lse=True)
        a.append(k, v, None if cnt is None else cnt.tolist())
        a.check_values()
        assert torch.equal(a.c.lens, b.c.lens)
        a.check_attend(q, out, lse, None if cnt is None else cnt.tolist())
        a.check_attend(q, out2, lse2, None if cnt is None else cnt.tolist())
    assert a.c.bacon_cache_errors() == 0


def test_step_without_room_attends_over_what_is_there():
    from paper_2606_14782_amd import bacon
    m = Model([[16, 10]], 2, 64, 16, "bf16", reserve=0)
    q, k, v = m.tokens(1, 2), m.tokens(1, 2), m.tokens(1, 2)
    out, lse = m.c.bacon_cache_step(0, q, k, v, want_lse=True)
    m.rows[0][0][1][0].append(_np(k)[0, :, 1])
    m.rows[0][0][1][1].append(_np(v)[0, :, 1])
    m.check_values()
    m.check_attend(q, out, lse)
    assert m.c.bacon_cache_errors() == bacon.CACHE_NO_BLOCKS


def test_rolled_back_tokens():
    """Drafted tokens taken back, others appended in their place."""
    import torch
    m = Model([[30, 47], [5, 16]], 4, 64, 16, "bf16")
    q, k, v = m.tokens(5, 4), m.tokens(5, 2), m.tokens(5, 2)
    m.c.bacon_cache_step(0, q, k, v)
    m.append(k, v)
    m.c.bacon_cache_advance(counts=torch.tensor([-3, -5], dtype=torch.int32, device="cuda"))
    for b, cut in ((0, 3), (1, 5)):
        for h in range(2):
            for kv in (0, 1):
                r = m.rows[0][b][h][kv]
                n = len(r) - cut
                # a block that began with rejected tokens starts anew
                r.cut(n)
    m.check_values()
    q, k, v = m.tokens(1, 4), m.tokens(1, 2, 7.0), m.tokens(1, 2, 7.0)
    out, lse = m.c.bacon_cache_step(0, q, k, v, want_lse=True)
    m.append(k, v)
    m.check_values()
    m.check_attend(q, out, lse)


# ------------------------------------------------- views, streams, graphs

def test_views_of_a_projection():
    import torch
    m = Model([[40, 41], [7, 90]], 6, 64, 32, "bf16")
    for n in (1, 3):
        qkv = m.tokens(n, 6 + 4)
        q, k, v = qkv[:, :, :6], qkv[:, :, 6:8], qkv[:, :, 8:]
        out, lse = m.c.bacon_cache_step(0, q, k, v, want_lse=True)
        m.append(k, v)
        m.check_values()
        m.check_attend(q, out, lse)
    # every second sequence of a larger batch
    big = _rand(m.rng, 4, 1, 6, 64)
    q = big[::2]
    m.check_attend(q, *m.c.bacon_cache_attend(0, q, want_lse=True))


def test_binding_refuses_what_the_kernels_do_not_read():
    import torch
    from paper_2606_14782_amd import bacon
    m = Model([[40, 41], [7, 90]], 6, 64, 32, "bf16")
    c, q, k = m.c, m.tokens(2, 6), m.tokens(2, 2)

    def refused(fn, *a, **kw):
        with pytest.raises(bacon.BaconError) as e:
            fn(*a, **kw)
        assert e.value.status in (bacon.ERR_INVALID, bacon.ERR_UNSUPPORTED), e.value
    refused(c.bacon_cache_attend, 0, q.float())
    refused(c.bacon_cache_attend, 0, q.cpu())
    refused(c.bacon_cache_attend, 0, q[:, :, :5])
    refused(c.bacon_cache_attend, 0, q.transpose(0, 1))
    refused(c.bacon_cache_attend, 0, q[..., ::2])
    refused(c.bacon_cache_attend, 0, q[0])
    refused(c.bacon_cache_attend, 0, q, torch.ones(2, device="cuda"))
    refused(c.bacon_cache_attend, 0, q, torch.ones(3, dtype=torch.int32, device="cuda"))
    refused(c.bacon_cache_attend, 0, q, out=torch.empty(2, 2, 6, 32, dtype=torch.bfloat16, device="cuda"))
    refused(c.bacon_cache_attend, 0, m.tokens(30, 6))
    refused(c.bacon_cache_attend, 1, q)
    refused(c.bacon_cache_append, 0, k, k[:, :1])
    refused(c.bacon_cache_append, 0, k[:0], k[:0])
    refused(c.bacon_cache_step, 0, q, k[:, :1], k[:, :1])
    refused(c.bacon_cache_load, 0)
    refused(c.bacon_cache_load, 4, num_layers=2)
    odd = torch.empty(2 * 2 * 6 * 64 + 8, dtype=torch.bfloat16, device="cuda")[1:2 * 2 * 6 * 64 + 1].view(2, 2, 6, 64)
    refused(c.bacon_cache_attend, 0, odd)
    refused(c.bacon_cache_tables, m.batch, torch.ones(1, 1, 2, dtype=torch.int32, device="cuda"))
    refused(c.bacon_cache_tables, m.batch, torch.ones(1, 2, 3, dtype=torch.int32, device="cuda"))
    refused(c.bacon_cache_store, m.batch, [q], [q])
    m.check_attend(q, *c.bacon_cache_attend(0, q, want_lse=True))


def test_two_streams_attend_beside_each_other():
    import torch
    m = Model([[3000, 1500]], 8, 128, 64, "bf16", layers=2)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    qs = [m.tokens(1, 8), m.tokens(1, 8)]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for l, s in enumerate(streams):
            with torch.cuda.stream(s):
                got.append((l, *m.c.bacon_cache_attend(l, qs[l], want_lse=True)))
    torch.cuda.synchronize()
    for l, out, lse in got:
        m.check_attend(qs[l], out, lse, layer=l)


@pytest.mark.parametrize("lens", [[[40, 33], [100, 7]], [[4000, 2100], [9, 100]]])
def test_captured_step_replays(lens):
    """A captured step appends and attends anew on every replay, with eager
    work between the replays, beside the same steps run eagerly."""
    import torch
    a, b = Model(lens, 8, 128, 32, "bf16", reserve=64), Model(lens, 8, 128, 32, "bf16", reserve=64)
    q, k, v = a.tokens(2, 8), a.tokens(2, 2), a.tokens(2, 2)
    out, lse = a.c.bacon_cache_step(0, q, k, v, want_lse=True)          # eager, on both
    b.c.bacon_cache_step(0, q, k, v)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        gout, glse = a.c.bacon_cache_step(0, q, k, v, want_lse=True)
        a.c.bacon_cache_advance(-1)
    for i in range(4):
        for t, n in ((q, 8), (k, 2), (v, 2)):
            t.copy_(a.tokens(2, n, 1.0 + i))
        g.replay()
        eager, elog = b.c.bacon_cache_step(0, q, k, v, want_lse=True)
        b.c.bacon_cache_advance(-1)
        torch.cuda.synchronize()
        assert torch.equal(gout, eager) and torch.equal(glse, elog), i
        x, y = a.c.bacon_cache_load(200), b.c.bacon_cache_load(200)
        assert torch.equal(a.c.lens, b.c.lens) and torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


def test_two_captured_graphs_replay_beside_each_other():
    """Each captured attend owns its scratch: replays on two streams do not mix."""
    import torch
    m = Model([[3000, 2900]], 8, 128, 64, "bf16", layers=2)
    qs = [m.tokens(1, 8), m.tokens(1, 8)]
    want = [m.c.bacon_cache_attend(l, qs[l], want_lse=True) for l in range(2)]
    graphs, got, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for l in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(m.c.bacon_cache_attend(l, qs[l], want_lse=True))
        graphs.append(g)
    for _ in range(5):
        torch.cuda.synchronize()
        for l in range(2):
            got[l][0].zero_()
        torch.cuda.synchronize()
        for l in range(2):
            with torch.cuda.stream(streams[l]):
                graphs[l].replay()
        torch.cuda.synchronize()
        for l in range(2):
            assert torch.equal(got[l][0], want[l][0]) and torch.equal(got[l][1], want[l][1])


def test_tables_and_store_in_a_captured_graph():
    """A prompt that joins a batch, captured: every replay gives the same cache
    as eager calls, with other work between the replays."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(21)
    d, W, bt, N, K = 64, 4, 16, [200, 90], [50, 60]
    cu = np.concatenate([[0], np.cumsum(N)])
    batch = bacon.BatchLayout(cu, K)
    c = _cache(2, 4, 2, d, W, bt, 2, 100, 60, "bf16")
    k, v = (_rand(rng, 2, int(cu[-1]), 2, d) for _ in range(2))
    bud = torch.from_numpy(rng.integers(1, 60, (2, 2, 2)).astype(np.int32)).cuda()
    used = torch.zeros(1, dtype=torch.int64, device="cuda")

    def fill():
        c.bacon_cache_clear()
        c.bacon_cache_tables(batch, bud, 5, used=used)
        c.bacon_cache_store(batch, k, v)
        return c.bacon_cache_load(64)
    fill()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        gk, gv = fill()
    for i in range(4):
        bud.copy_(torch.from_numpy(rng.integers(1, 60, (2, 2, 2)).astype(np.int32)))
        k.copy_(_rand(rng, 2, int(cu[-1]), 2, d))
        g.replay()
        torch.cuda.synchronize()
        table, lens, n = c.table.clone(), c.lens.clone(), int(used)
        a, b = gk.clone(), gv.clone()
        ek, ev = fill()
        assert torch.equal(table, c.table) and torch.equal(lens, c.lens) and n == int(used)
        assert torch.equal(a, ek) and torch.equal(b, ev), i


def test_rows_that_are_not_named_stay():
    """Guards around the outputs and every block of other pairs stay as they were."""
    import torch
    m = Model([[20, 21], [22, 23], [24, 25]], 4, 64, 16, "bf16", layers=2)
    used = m.c.table[1, 1].reshape(-1)
    before_codes, before_scales = m.c.codes.clone(), m.c.scales.view(torch.int32).clone()
    before_lens, before_table = m.c.lens.clone(), m.c.table.clone()
    big = torch.full((3, 2, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    q, k, v = (_rand(m.rng, 1, 2, h, 64) for h in (4, 2, 2))
    m.c.bacon_cache_step(1, q, k, v, first_seq=1, out=big[1:2])
    torch.cuda.synchronize()
    assert (big[0] == 3).all() and (big[2] == 3).all()
    mine = torch.zeros(m.c.codes.shape[0], dtype=torch.bool, device="cuda")
    mine[used[used >= 0].long()] = True
    assert torch.equal(m.c.codes[~mine], before_codes[~mine])
    assert torch.equal(m.c.scales.view(torch.int32)[~mine], before_scales[~mine])
    changed = m.c.lens != before_lens
    assert changed[1, 1].all() and int(changed.sum()) == 2 and torch.equal(m.c.table, before_table)


def test_outputs_and_scratch_keep_to_their_buffers():
    """Guards before and after every buffer of a call, odd sizes; and the same
    bits from a second run."""
    import torch
    from paper_2606_14782_amd import bacon
    m = Model([[1500, 3], [70, 900]], 14, 64, 32, "bf16")
    n, G = 3, 7

    def guarded(numel, dtype):
        t = torch.full((numel + 256,), 7, dtype=dtype, device="cuda")
        return t, t[128:128 + numel]

    def untouched(t, numel):
        return bool((t[:128] == 7).all()) and bool((t[128 + numel:] == 7).all())
    q = m.tokens(n, 14)
    need = bacon.lib().bacon_cache_work_bytes(m.c._h, 2, n, 1600)
    assert need > 0
    sizes = (2 * n * 14 * 64, 2 * n * 14, need)
    bufs = [guarded(x, d) for x, d in zip(sizes, (torch.bfloat16, torch.float32, torch.uint8))]
    work = torch.full((need + 1024,), 7, dtype=torch.uint8, device="cuda")
    skip = -work.data_ptr() % 256 + 256
    got = []
    for _ in range(2):
        out, lse = bufs[0][1].view(2, n, 14, 64), bufs[1][1].view(2, n, 14)
        m.c.bacon_cache_attend(0, q, max_tokens=1600, out=out, lse=lse, work=work[skip:skip + need])
        got.append((out.clone(), lse.clone()))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    m.check_attend(q, out, lse)
    assert untouched(bufs[0][0], sizes[0]) and untouched(bufs[1][0], sizes[1])
    assert bool((work[:skip] == 7).all()) and bool((work[skip + need:] == 7).all())
    for count, first in ((33, 0), (1501, 0), (17, -17), (5, -1502)):
        size = 2 * 2 * count * 64
        k, v = guarded(size, torch.bfloat16), guarded(size, torch.bfloat16)
        shape = (1, 2, 2, count, 64)
        m.c.bacon_cache_load(count, first_token=first, out=(k[1].view(shape), v[1].view(shape)))
        assert untouched(k[0], size) and untouched(v[0], size)
    # blocks that no table names are as they were
    used = torch.zeros(m.c.codes.shape[0], dtype=torch.bool, device="cuda")
    used[m.c.table[m.c.table >= 0].long()] = True
    assert bool((m.c.codes[~used] == 0x7F).all()) and bool(m.c.scales[~used].isnan().all())


def test_functions_of_the_module_are_the_methods():
    import torch
    from paper_2606_14782_amd import bacon
    m = Model([[20, 21]], 4, 64, 16, "bf16")
    q, k, v = m.tokens(1, 4), m.tokens(1, 2), m.tokens(1, 2)
    bacon.bacon_cache_append(m.c, 0, k, v)
    m.append(k, v)
    m.check_attend(q, *bacon.bacon_cache_attend(m.c, 0, q, want_lse=True))
    bacon.bacon_cache_step(m.c, 0, q, k, v)
    bacon.bacon_cache_advance(m.c, -1)
    a, b = bacon.bacon_cache_load(m.c, 22), m.c.bacon_cache_load(22)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    bacon.bacon_cache_clear(m.c)
    assert int(bacon.bacon_cache_tables(m.c, m.batch)) > 0
    x = torch.zeros(1, m.batch.total, 2, 64, dtype=torch.bfloat16, device="cuda")
    bacon.bacon_cache_store(m.c, m.batch, x, x)
    assert not bacon.bacon_cache_load(m.c, 5)[0].any()


# -------------------------------------------------------------- together

@pytest.mark.parametrize("adaptive", [False, True])
def test_prompt_then_decode(adaptive):
    """A prompt compressed by the framework, its kept rows moved into the cache
    and several tokens decoded over them, layer by layer."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(11)
    L, hq, H, d, W, bt, N, K = 3, 8, 2, 64, 8, 16, [300, 517], [24, 40]
    cu = np.concatenate([[0], np.cumsum(N)])
    T = int(cu[-1])
    params = bacon.default_params(pool_kernel=5, head_alloc=bacon.ALLOC_ADAPTIVE if adaptive else bacon.ALLOC_GIVEN)
    ctx = bacon.Context(L, hq, H, d, W, 2, T, "bf16", params)
    batch = bacon.BatchLayout(cu, K)
    qs = [_rand(rng, 2 * W, hq, d, scale=2.0) for _ in range(L)]
    ks, vs = ([_rand(rng, T, H, d) for _ in range(L)] for _ in range(2))
    budgets = None
    if adaptive:
        budgets = torch.zeros(L, 2, H, dtype=torch.int32, device="cuda")
        ctx.bacon_alloc_output(budgets)
    ctx.bacon_begin_prompt(batch)
    outs = ctx.bacon_compress_prompt(0, batch, qs, ks, vs)
    c = _cache(L, hq, H, d, W, bt, 2, max(K) * H + W + 32, 200, "bf16")
    used = c.bacon_cache_tables(batch, budgets, 32)
    c.bacon_cache_store(batch, ks, vs, [o[0] for o in outs])
    bud = np.broadcast_to(np.array(K)[None, :, None], (L, 2, H)) if budgets is None else budgets.cpu().numpy()
    assert int(used) == int(((bud + W + 32 + bt - 1) // bt).sum())
    m = Model([[1, 1], [1, 1]], hq, d, bt, "bf16", layers=L, W=1)
    m.c, m.W = c, W
    for l in range(L):
        idx, at = outs[l][0].cpu().numpy(), 0
        for b in range(2):
            for h in range(H):
                kept = idx[at:at + bud[l, b, h]]
                at += bud[l, b, h]
                pos = np.concatenate([kept, np.arange(N[b] - W, N[b])]) + cu[b]
                for kv, x in ((0, ks), (1, vs)):
                    m.rows[l][b][h][kv].store(_np(x[l])[pos, h])
        m.check_values(l)
        if not adaptive:                    # the compacted cache's own rows, rounded to the cache's numbers
            rows = _np(outs[l][1])
            r = R.Rows(bt, d)
            r.store(rows[:K[0] + W, 1])
            np.testing.assert_array_equal(r.x, m.rows[l][0][1][0].x)
    for _ in range(3):
        for l in range(L):
            q, k, v = m.tokens(1, hq), m.tokens(1, H), m.tokens(1, H)
            out, lse = c.bacon_cache_step(l, q, k, v, want_lse=True)
            m.append(k, v, layer=l)
            m.check_attend(q, out, lse, layer=l)
    for l in range(L):
        m.check_values(l)
    assert c.bacon_cache_errors() == 0


# ------------------------------------------------- ends of the numbers' range

def _equal_keys(m, sign, power, rows):
    """Keys that are 1.375 x 2^a in the first dimension (1.5 x 2^a in every third
    row) and 0 elsewhere, and queries of their own value x 2^b there, a + b =
    power: every logit is the same product in every row of its kind, so the
    softmax is the mean over the kind that `sign` makes the larger, exactly.
    Returns queries and the kinds."""
    import torch
    a = power // 2
    kind = np.arange(rows) % 3 == 2
    key = np.where(kind, 1.5, 1.375) * 2.0 ** a
    q = m.tokens(1, m.hq)
    first = (1.0 + q[..., 0].abs() % 1.0) * sign * 2.0 ** (power - a)
    q.zero_()
    q[..., 0] = first
    k = torch.zeros(rows, m.H, m.d, dtype=q.dtype, device="cuda")
    k[..., 0] = torch.from_numpy(key).cuda()[:, None].to(q.dtype)
    return q, k, kind if sign > 0 else ~kind


@pytest.mark.parametrize("dtype,d,G", [("bf16", 128, 4), ("fp32", 64, 1), ("fp32", 128, 17), ("bf16", 64, 20)])
@pytest.mark.parametrize("rows", [1, 2, 300, 5000])
def test_attend_of_logits_as_large_as_floats(dtype, d, G, rows):
    """Logits of either sign up to 2^120: finite ones never count as no row, and
    the largest has weight 1 whatever its size.  Weights are 0 and 1 exactly, so the
    bound is that of the sums (n / 16 + 64 terms a chain, as in cache_ref) and of the
    output's rounding; lse comes of at most eight roundings (of the sum over the query's
    parts two, the scale, the product, log2 l and its sum, ln 2, the product)."""
    from paper_2606_14782_amd import bacon
    for power in (40, 70, 104, 120):
        for sign in (1, -1):
            m = Model([[1]], G, d, 32, dtype)
            q, k, kind = _equal_keys(m, sign, power, rows)
            v = _rand(m.rng, rows, 1, d, dtype=dtype)
            m.c = _cache(1, G, 1, d, 1, 32, 1, rows, rows // 32 + 2, dtype)
            batch = bacon.BatchLayout([0, rows], [max(1, rows - 1)])
            m.c.bacon_cache_tables(batch)
            m.c.bacon_cache_store(batch, [k], [v])
            for kv, x in ((0, k), (1, v)):
                m.rows[0][0][0][kv].store(_np(x)[:, 0])
            m.check_values()
            out, lse = m.c.bacon_cache_attend(0, q, want_lse=True)
            held, key = m.rows[0][0][0][1].x, m.rows[0][0][0][0].x[:, 0]
            won = held[kind] if kind.any() else held
            s = _np(q)[0, 0, :, 0] * (key[kind].max() if kind.any() else key[0]) / math.sqrt(d)
            h = 2.0 ** -24
            tol = R.HALF[dtype] * np.abs(won.mean(0)) + (2 * (rows / 16 + 64) + 4) * h * np.abs(won).mean(0) * 1.01
            assert np.all(np.abs(_np(out)[0, 0] - won.mean(0)) <= tol), (power, sign)
            want = s + math.log(len(won))
            assert np.all(np.abs(_np(lse)[0, 0] - want) <= 8 * h * np.abs(want)), (power, sign)
            assert m.c.bacon_cache_errors() == 0


@pytest.mark.parametrize("dtype,d,G,n", [("bf16", 128, 4, 1), ("fp32", 64, 7, 3), ("bf16", 64, 7, 4), ("fp32", 128, 5, 5)])
@pytest.mark.parametrize("lens", [[[40, 1], [300, 65]], [[4100, 2000], [3, 1000]]])
def test_a_query_that_is_not_finite_is_nan_alone(dtype, d, G, n, lens):
    """All of its output and its lse, however the rows are divided; the other
    queries of its workgroup as without it, bit for bit."""
    import torch
    m = Model(lens, 2 * G, d, 64, dtype)
    q = m.tokens(n, 2 * G, 1.5)
    out, lse = m.c.bacon_cache_attend(0, q, want_lse=True)
    m.check_attend(q, out, lse)
    bad = torch.zeros(lse.shape, dtype=torch.bool, device="cuda")
    for i, (b, h, x) in enumerate(((0, 0, math.nan), (0, 2 * G - 1, math.inf), (1, 1, -math.inf), (1, G, math.nan))):
        q[b, n - 1 - i % n, h, 7 * i] = x
        bad[b, n - 1 - i % n, h] = True
    bad &= ~torch.isneginf(lse)                       # (a query that sees no row stays one)
    got, glse = m.c.bacon_cache_attend(0, q, want_lse=True)
    assert got[bad].isnan().all() and glse[bad].isnan().all()
    assert torch.equal(got[~bad], out[~bad]) and torch.equal(glse[~bad], lse[~bad])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64)])
@pytest.mark.parametrize("rows", [1, 128, 5000])
def test_logits_past_the_largest_float(dtype, d, rows):
    """Infinite logits: upward NaN, downward no weight, and NaN where that leaves none.
    The first half's logits are 0: their weights are equal."""
    import torch
    from paper_2606_14782_amd import bacon
    half = rows // 128 * 64
    m = Model([[1]], 4, d, 32, dtype)
    q, v = m.tokens(1, 4) * 0, _rand(m.rng, rows, 1, d, dtype=dtype)
    q[0, 0, :, 0] = torch.tensor([2.0 ** 20, -2.0 ** 20, -2.0 ** 60, 0.0])
    for low in (half, 0):                             # rows whose logits are 0
        k = torch.zeros(rows, 1, d, dtype=q.dtype, device="cuda")
        k[low:, 0, 0] = 2.0 ** 127
        c = _cache(1, 4, 1, d, 1, 32, 1, rows, rows // 32 + 2, dtype)
        batch = bacon.BatchLayout([0, rows], [max(1, rows - 1)])
        c.bacon_cache_tables(batch)
        c.bacon_cache_store(batch, [k], [v])
        m.rows[0][0][0][1].store(_np(v)[:, 0])
        held, h = m.rows[0][0][0][1].x, 2.0 ** -24
        out, lse = c.bacon_cache_attend(0, q, want_lse=True)
        on, ln = _np(out)[0, 0], _np(lse)[0, 0]
        for i, seen in enumerate((0, low, low, rows)):
            if not seen:
                assert np.isnan(on[i]).all() and np.isnan(ln[i]), (low, i)
                continue
            won = held[:seen]
            tol = R.HALF[dtype] * np.abs(won.mean(0)) + (2 * (rows / 16 + 64) + 4) * h * np.abs(won).mean(0) * 1.01
            assert np.all(np.abs(on[i] - won.mean(0)) <= tol), (low, i)
            assert abs(ln[i] - math.log(seen)) <= (rows / 16 + 64 + 8) * h * (1 + math.log(seen)), (low, i)


@pytest.mark.parametrize("lens", [[[200, 130], [70, 300]], [[2500, 130], [70, 4000]]])
def test_padding_may_hold_anything(lens):
    """Padding queries over whole tiles of rows: zeros and -infinity, whatever they hold."""
    import torch
    m = Model(lens, 6, 64, 32, "bf16")
    counts = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    q = m.tokens(4, 6)
    q[0, 1:], q[1] = math.nan, math.inf
    out, lse = m.c.bacon_cache_attend(0, q, counts, want_lse=True)
    m.check_attend(q, out, lse, [1, 0])


@pytest.mark.parametrize("device", [False, True])
def test_budgets_whose_sum_passes_32_bits(device):
    """Offsets into idx past 2^31 - 1 name no entry, also where they are small
    numbers again past 2^32: the rows are zero, no other pair's."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(31)
    H, W, N, big = 8, 2, 12, 1 << 30
    c = _cache(2, H, H, 64, W, 16, 1, 16, 40, "fp32")
    batch = bacon.BatchLayout([0, N], [big])
    bud = torch.full((2, 1, H), big, dtype=torch.int32, device="cuda")
    c.bacon_cache_tables(batch, bud if device else None)
    assert (c.lens == N).all()
    starts = c.starts[:, 0].cpu().numpy()
    assert (starts == [0, big] + [-1] * (H - 2)).all()
    k, v = (_rand(rng, 2, N, H, 64, dtype="fp32") for _ in range(2))
    idx = torch.arange(N - W, dtype=torch.int32, device="cuda").expand(2, N - W).contiguous()
    c.bacon_cache_store(batch, k, v, idx)
    got = c.bacon_cache_load(N)
    for x in got:
        assert x[:, 0, 0].any(-1).all()                           # entries 0 .. 9
        assert not x[:, 0, 1:, :N - W].any() and x[:, 0, :, N - W:].any(-1).all()
    assert c.bacon_cache_errors() == bacon.CACHE_BAD_INDEX


def test_an_empty_list_of_free_ids_gives_no_blocks():
    """A pool without a free block: no pair takes the ids that others hold."""
    import torch
    from paper_2606_14782_amd import bacon
    c = _cache(1, 2, 2, 64, 4, 16, 2, 64, 10, "bf16")
    c.bacon_cache_tables(bacon.BatchLayout([0, 40], [30]), None, 10)
    table = c.table.clone()
    for free in (torch.empty(0, dtype=torch.int32, device="cuda"), torch.arange(9, dtype=torch.int32, device="cuda")[9:]):
        c.bacon_cache_clear(1, 1)
        used = c.bacon_cache_tables(bacon.BatchLayout([0, 40], [30]), None, 10, free, first_seq=1)
        assert int(used) == 6
        assert torch.equal(c.table[:, 0], table[:, 0]) and (c.table[:, 1] == -1).all()
        assert (c.lens[:, 0] == 34).all() and not c.lens[:, 1].any()
        assert c.bacon_cache_errors() == bacon.CACHE_NO_BLOCKS


# --------------------------------------------- appends into divided pairs

@pytest.mark.parametrize("dtype,d,bt,G,n,part", [
    ("bf16", 128, 64, 4, 4, 64), ("bf16", 64, 16, 1, 16, 64), ("bf16", 128, 32, 7, 2, 64), ("bf16", 128, 16, 8, 1, 64),
    ("fp32", 64, 32, 5, 3, 64), ("fp32", 128, 16, 1, 13, 64), ("bf16", 128, 64, 5, 6, 256), ("bf16", 64, 16, 1, 32, 256),
    ("fp32", 128, 32, 8, 4, 256), ("fp32", 64, 64, 3, 9, 256)])
def test_step_over_the_borders_of_parts(dtype, d, bt, G, n, part):
    """Pairs divided along their rows, lengths just below the border of two parts:
    two workgroups put some of the new rows in place each, and the join moves the
    lengths.  Parts are 64 rows for up to 16 query rows, else 256."""
    import torch
    from paper_2606_14782_amd import bacon
    parts = 20 if part == 64 else 10
    lens = [[4 * part - 1, 2 * part - n // 2], [(parts - 1) * part - n, 5 * part - n - (n + 1) // 2]]
    most = parts * part
    m = Model(lens, 2 * G, d, bt, dtype, reserve=part + n)
    assert bacon.lib().bacon_cache_work_bytes(m.c._h, 2, n, most) >= 4 * parts * G * n * (8 + 4 * d)   # divided so
    counts = torch.tensor([n, (n + 1) // 2], dtype=torch.int32, device="cuda")
    for i, cnt in enumerate((None, counts, None)):
        q, k, v = m.tokens(n, 2 * G, 1.5), m.tokens(n, 2, 3.0 ** i), m.tokens(n, 2, 3.0 ** i)
        out, lse = m.c.bacon_cache_step(0, q, k, v, cnt, max_tokens=most, want_lse=True)
        cl = None if cnt is None else cnt.tolist()
        m.append(k, v, cl)
        m.check_values()
        m.check_attend(q, out, lse, cl)
    assert m.c.bacon_cache_errors() == 0


@pytest.mark.parametrize("dtype,G,n", [("bf16", 4, 3), ("bf16", 5, 6), ("fp32", 1, 2)])
def test_divided_step_without_room_attends_over_what_is_there(dtype, G, n):
    """Two of four pairs have no block left: they stay, the others grow."""
    from paper_2606_14782_amd import bacon
    m = Model([[1024, 1000], [777, 2048]], 2 * G, 64, 32, dtype, reserve=0)
    q, k, v = m.tokens(n, 2 * G), m.tokens(n, 2), m.tokens(n, 2)
    assert bacon.lib().bacon_cache_work_bytes(m.c._h, 2, n, 2048) > 0
    out, lse = m.c.bacon_cache_step(0, q, k, v, max_tokens=2048, want_lse=True)
    kn, vn = _np(k), _np(v)
    for b, h in ((0, 1), (1, 0)):
        m.rows[0][b][h][0].append(kn[b, :, h])
        m.rows[0][b][h][1].append(vn[b, :, h])
    m.check_values()
    m.check_attend(q, out, lse)
    assert m.c.bacon_cache_errors() == bacon.CACHE_NO_BLOCKS


@pytest.mark.parametrize("dtype,append", [("bf16", False), ("bf16", True), ("fp32", True)])
def test_magnitudes_of_the_whole_range(dtype, append):
    """Zeros, the least and the largest magnitudes, ties and subnormal codes,
    stored or appended: the values held are the nearest, exactly."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(6)
    bt, d = 16, 64
    n = bt * 9
    x = rng.standard_normal((n, 1, d))
    x[:bt] = 0
    x[bt:2 * bt] *= 2.0 ** -128
    x[2 * bt:3 * bt] = np.clip(x[2 * bt:3 * bt], -1, 1) * 2.0 ** 127
    x[3 * bt:4 * bt] = rng.integers(-448, 449, (bt, 1, d))
    x[4 * bt:5 * bt] = rng.integers(-64, 65, (bt, 1, d)) * 2.0 ** -11
    x[4 * bt, 0, 0] = 448
    x[5 * bt, 0, 0] = 450
    x[6 * bt:7 * bt] *= 2.0 ** -107                       # about the least scale
    x[7 * bt + 3] *= 2.0 ** 100                           # rows whose scale leaves nothing of the others
    t = torch.from_numpy(x).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    c = _cache(1, 1, 1, d, 1, bt, 1, n, 10, dtype)
    held = R.Rows(bt, d)
    if append:
        c.bacon_cache_tables(bacon.BatchLayout([0, 1], [1]), None, n - 1)
        c.bacon_cache_store(bacon.BatchLayout([0, 1], [1]), [t[:1]], [t[:1]])
        held.store(_np(t)[:1, 0])
        at = 1
        while at < n:
            new = t[at:at + int(rng.integers(1, 30))]
            c.bacon_cache_append(0, new[None], new[None])
            held.append(_np(new)[:, 0])
            at += len(new)
    else:
        c.bacon_cache_tables(bacon.BatchLayout([0, n], [n - 1]))
        c.bacon_cache_store(bacon.BatchLayout([0, n], [n - 1]), [t], [t])
        held.store(_np(t)[:, 0])
    scales = c.scales.cpu().numpy()[c.table[0, 0, 0, :9].cpu().numpy()]
    np.testing.assert_array_equal(scales, np.exp2(np.array(held.e, np.float64))[:, None].repeat(2, 1))
    for got in c.bacon_cache_load(n):
        np.testing.assert_array_equal(_np(got)[0, 0, 0], held.x)
    assert c.bacon_cache_errors() == 0
