"""Rotary positions on the GPU against plain 64-bit numpy (around_ref), with the
bounds that it derives."""
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


def _check(got, x, pos, f, m, layout, dtype, sections=None, weight=None, eps=0.0):
    want, tol = A.rotate(_np(x), pos, f, m, layout, dtype, sections, None if weight is None else _np(weight), eps)
    err = np.abs(_np(got) - want)
    assert np.all(err <= tol), float((err / np.maximum(tol, 1e-300)).max())


def _rotary(hq, hkv, d, dtype, r=None, layout="half", scaling="plain", **kw):
    from paper_2606_14782_amd import bacon
    kinds = {"plain": bacon.ROTARY_PLAIN, "linear": bacon.ROTARY_LINEAR, "ntk": bacon.ROTARY_NTK,
             "yarn": bacon.ROTARY_YARN, "given": bacon.ROTARY_GIVEN}
    return bacon.Rotary(hq, hkv, d, dtype, r, {"half": bacon.ROTARY_HALF, "pairs": bacon.ROTARY_PAIRS}[layout],
                        scaling=kinds[scaling], **kw)


def _positions(pos):
    import torch
    return torch.from_numpy(np.ascontiguousarray(pos, dtype=np.int32)).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("d,r", [(64, 64), (128, 128), (128, 64), (64, 16), (128, 2), (64, 22), (128, 126), (128, 34)])
def test_rotate(dtype, layout, d, r):
    """Whole heads and parts of them, of sizes that eights do and do not divide."""
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(r)
    for tokens, hq, hkv in ((1, 1, 1), (3, 7, 1), (70, 5, 3), (33, 17, 2)):
        q, k = _rand(rng, tokens, hq, d, dtype=dtype), _rand(rng, tokens, hkv, d, dtype=dtype, scale=4)
        pos = rng.integers(0, 40000, tokens)
        qo, ko = bacon.bacon_rotate(_rotary(hq, hkv, d, dtype, r, layout), _positions(pos), q, k)
        f, m = A.frequencies(r, 10000.0)
        _check(qo, q, pos, f, m, layout, dtype)
        _check(ko, k, pos, f, m, layout, dtype)


@pytest.mark.parametrize("scaling,kw", [
    ("linear", dict(factor=4.0)), ("ntk", dict(factor=8.0, base=5e5)), ("yarn", dict(factor=4.0, base=1e6)),
    ("yarn", dict(factor=1.0)), ("yarn", dict(factor=40.0, fast=16.0, slow=2.0)),
])
def test_scaled_frequencies(scaling, kw):
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(1)
    trained = 4096 if scaling == "yarn" else 0
    f, m = A.frequencies(128, kw.get("base", 10000.0), scaling, kw["factor"], trained, kw.get("fast", 32.0),
                         kw.get("slow", 1.0))
    rot = _rotary(2, 1, 128, "fp32", scaling=scaling, base=kw.get("base", 10000.0), factor=kw["factor"],
                  trained_tokens=trained, beta_fast=kw.get("fast", 32.0), beta_slow=kw.get("slow", 1.0))
    np.testing.assert_allclose(rot.frequencies, f, rtol=1e-14)
    assert rot.magnitude == m
    q, k = _rand(rng, 50, 2, 128, dtype="fp32"), _rand(rng, 50, 1, 128, dtype="fp32")
    pos = rng.integers(0, 1 << 20, 50)
    qo, ko = bacon.bacon_rotate(rot, _positions(pos), q, k)
    _check(qo, q, pos, f, m, "half", "fp32")
    _check(ko, k, pos, f, m, "half", "fp32")


def test_given_frequencies_and_magnitude():
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(2)
    f = np.concatenate([[0.0, -0.5, 1e6, 3.0], rng.uniform(0, 2, 12)])
    rot = _rotary(3, 1, 64, "fp32", 32, "pairs", "given", frequencies=f, magnitude=1.5)
    x, pos = _rand(rng, 9, 3, 64, dtype="fp32"), rng.integers(-1000, 1000, 9)
    got, none = bacon.bacon_rotate(rot, _positions(pos), x)
    assert none is None
    _check(got, x, pos, f, 1.5, "pairs", "fp32")


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_far_positions(layout):
    """The largest and the least int32: what 64 bits leave of the angle is what is lost."""
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(3)
    pos = np.array([0, 1, -1, 131071, 1 << 24, (1 << 24) + 1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 7])
    k = _rand(rng, len(pos), 2, 128, dtype="fp32")
    _, got = bacon.bacon_rotate(_rotary(1, 2, 128, "fp32", layout=layout), _positions(pos), None, k)
    f, m = A.frequencies(128, 10000.0)
    _check(got, k, pos, f, m, layout, "fp32")


def test_quarter_turns_are_exact():
    """Angles at the borders of the quarters."""
    from paper_2606_14782_amd import bacon
    import torch
    f = np.full(32, np.pi / 2)
    x = torch.zeros(8, 1, 64, device="cuda")
    x[..., 0::2] = 1.0
    got = _np(bacon.bacon_rotate(_rotary(1, 1, 64, "fp32", layout="pairs", scaling="given", frequencies=f),
                                 _positions(np.arange(8) - 3), x)[0])[:, 0]
    angle = (np.arange(8) - 3) * np.pi / 2
    assert np.abs(got[:, 0::2] - np.cos(angle)[:, None]).max() <= 8 * A.h
    assert np.abs(got[:, 1::2] - np.sin(angle)[:, None]).max() <= 8 * A.h


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sections", [(16, 24, 24), (0, 0, 64), (64, 0, 0), (1, 62, 1)])
def test_three_rows_of_positions(dtype, sections):
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(4)
    q, k = _rand(rng, 41, 6, 128, dtype=dtype), _rand(rng, 41, 2, 128, dtype=dtype)
    pos = rng.integers(0, 9000, (3, 41))
    qo, ko = bacon.bacon_rotate(_rotary(6, 2, 128, dtype, sections=sections), _positions(pos), q, k)
    f, m = A.frequencies(128, 10000.0)
    _check(qo, q, pos, f, m, "half", dtype, sections)
    _check(ko, k, pos, f, m, "half", dtype, sections)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("d,r", [(128, 128), (64, 32), (64, 20)])
def test_normalised_heads(dtype, layout, d, r):
    """Large, small and zero heads; one side normalised, or both."""
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(5)
    q, k = _rand(rng, 19, 6, d, dtype=dtype), _rand(rng, 19, 3, d, dtype=dtype)
    q[3] *= 1e4
    q[4] *= 1e-4
    k[5] = 0
    wq, wk = _rand(rng, d, dtype=dtype), _rand(rng, d, dtype=dtype)
    pos = rng.integers(0, 5000, 19)
    f, m = A.frequencies(r, 10000.0)
    rot = _rotary(6, 3, d, dtype, r, layout, norm_eps=1e-5)
    qo, ko = bacon.bacon_rotate(rot, _positions(pos), q, k, wq, wk)
    _check(qo, q, pos, f, m, layout, dtype, None, wq, 1e-5)
    _check(ko, k, pos, f, m, layout, dtype, None, wk, 1e-5)
    qo, ko = bacon.bacon_rotate(rot, _positions(pos), q, k, None, wk)
    _check(qo, q, pos, f, m, layout, dtype)
    _check(ko, k, pos, f, m, layout, dtype, None, wk, 1e-5)


def test_dimensions_past_the_turned_ones_pass_as_they_are():
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(6)
    for r, layout in ((32, "half"), (32, "pairs"), (20, "half"), (6, "pairs")):
        for dtype in ("bf16", "fp32"):
            x = _rand(rng, 5, 3, 64, dtype=dtype)
            x[..., r:] = torch.tensor([float("nan"), float("inf"), -0.0, -float("inf")], device="cuda").to(x.dtype).repeat(
                16)[:64 - r]
            got = bacon.bacon_rotate(_rotary(3, 1, 64, dtype, r, layout), _positions(np.arange(5)), x)[0]
            assert torch.isfinite(got[..., :r]).all()
            a, b = got[..., r:].float(), x[..., r:].float()
            assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(7), b.nan_to_num(7))
            assert torch.equal(a.signbit() & ~a.isnan(), b.signbit() & ~b.isnan())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("r", [128, 20])
def test_views_in_place_and_between_guards(dtype, r):
    """q and k as parts of one projection's output, turned where they lie: v and
    everything else stays; outputs that are views of other buffers."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(7)
    b, n, hq, hkv, d = 3, 5, 6, 2, 128
    qkv = _rand(rng, b, n, hq + 2 * hkv, d, dtype=dtype)
    rot, pos = _rotary(hq, hkv, d, dtype, r), _positions(rng.integers(0, 999, (b, n)))
    q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
    want_q, want_k = bacon.bacon_rotate(rot, pos, q, k)
    kept = v.clone()
    big = torch.full((b, n, hq + 4, d), 7.0, device="cuda", dtype=qkv.dtype)
    bacon.bacon_rotate(rot, pos, q, None, q_out=big[:, :, 2:2 + hq])
    assert torch.equal(big[:, :, 2:2 + hq], want_q)
    assert (big[:, :, :2] == 7).all() and (big[:, :, 2 + hq:] == 7).all()
    bacon.bacon_rotate(rot, pos, q, k, q_out=q, k_out=k)
    assert torch.equal(q, want_q) and torch.equal(k, want_k) and torch.equal(v, kept)


def test_moving_keys_by_the_difference_of_positions():
    """A key turned by p, then by n - p, is the key turned by n: each turn is off by
    10 half steps of |a| + |b|, which a turn may raise by the root of 2."""
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(8)
    rot, k = _rotary(1, 4, 128, "fp32"), _rand(rng, 30, 4, 128, dtype="fp32")
    p, n = rng.integers(0, 30000, 30), np.arange(30)
    once = _np(bacon.bacon_rotate(rot, _positions(n), None, k)[1])
    twice = _np(bacon.bacon_rotate(rot, _positions(n - p), None, bacon.bacon_rotate(rot, _positions(p), None, k)[1])[1])
    both = np.tile(np.abs(_np(k)).reshape(30, 4, 2, 64).sum(2), 2)       # |a| + |b| of each value's pair
    assert np.all(np.abs(once - twice) <= both * 4 * 12 * A.h)


def test_no_tokens_and_many():
    import torch
    from paper_2606_14782_amd import bacon
    rot = _rotary(2, 1, 64, "bf16")
    q = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.empty(0, 1, 64, dtype=torch.bfloat16, device="cuda")
    qo, ko = bacon.bacon_rotate(rot, torch.empty(0, dtype=torch.int32, device="cuda"), q, k)
    assert qo.shape == q.shape and ko.shape == k.shape
    # offsets past 2^31 elements: the last tokens of a long run, against a short call
    n, rng = 17_000_001, np.random.default_rng(9)
    big = torch.zeros(n, 2, 64, dtype=torch.bfloat16, device="cuda")
    tail = _rand(rng, 9, 2, 64)
    big[-9:] = tail
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    bacon.bacon_rotate(rot, pos, big, q_out=big)
    assert torch.equal(big[-9:], bacon.bacon_rotate(rot, pos[-9:].contiguous(), tail)[0])
    assert not big[:-9].any()


def test_streams_graphs_and_few_tokens():
    """A captured call replays on new inputs; another stream gives the same bits;
    a token's heads divided over waves the same as not."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(10)
    rot = _rotary(28, 4, 128, "bf16", sections=(16, 24, 24))
    q, k = _rand(rng, 9000, 28, 128), _rand(rng, 9000, 4, 128)
    pos = _positions(rng.integers(0, 9000, (3, 9000)))
    wq, wk = bacon.bacon_rotate(rot, pos, q, k)
    one = pos[:, 77:80].contiguous()
    a, b = bacon.bacon_rotate(rot, one, q[77:80], k[77:80])
    assert torch.equal(a, wq[77:80]) and torch.equal(b, wk[77:80])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a, b = bacon.bacon_rotate(rot, pos, q, k)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(a, wq) and torch.equal(b, wk)
    g, xq, xk, xp = torch.cuda.CUDAGraph(), q[:3].clone(), k[:3].clone(), pos[:, :3].contiguous()
    with torch.cuda.graph(g):
        gq, gk = bacon.bacon_rotate(rot, xp, xq, xk)
    for i in (5, 100, 8000):
        xq.copy_(q[i:i + 3]); xk.copy_(k[i:i + 3]); xp.copy_(pos[:, i:i + 3])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(gq, wq[i:i + 3]) and torch.equal(gk, wk[i:i + 3])


def test_binding_refuses():
    import torch
    from paper_2606_14782_amd import bacon
    rot = _rotary(4, 2, 64, "bf16")
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    p = torch.zeros(3, dtype=torch.int32, device="cuda")
    bad = [dict(q=q.float()), dict(q=q.cpu()), dict(q=q[:2]), dict(k=k[:, :1]), dict(q=None, k=None), dict(positions=p[:2]),
           dict(positions=p.long()), dict(positions=torch.zeros(3, 3, dtype=torch.int32, device="cuda")),
           dict(q_norm=torch.ones(32, dtype=torch.bfloat16, device="cuda")), dict(q_norm=torch.ones(64, device="cuda")),
           dict(q_out=torch.zeros(3, 4, 64, device="cuda")), dict(q_out=q[:, :, :32]),
           dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)), dict(k=None, k_out=k)]
    for kw in bad:
        args = dict(positions=p, q=q, k=k)
        args.update(kw)
        with pytest.raises(bacon.BaconError):
            bacon.bacon_rotate(rot, **args)


def test_one_token_of_any_view():
    """A decoded token's heads in a projection's output, with leading dimensions, in
    place, and refused where they do not lie together or the tokens differ."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(12)
    rot = _rotary(4, 2, 64, "bf16")
    both = _rand(rng, 5, 8, 64)
    p = torch.tensor([70000], dtype=torch.int32, device="cuda")
    q, k = both[3:4, :4], both[3:4, 4:6]
    wq, wk = bacon.bacon_rotate(rot, p, q.contiguous(), k.contiguous())
    a, b = bacon.bacon_rotate(rot, p, q, k)
    assert torch.equal(a, wq) and torch.equal(b, wk) and a.is_contiguous()
    a, b = bacon.bacon_rotate(rot, p[None], q[None], k[None])
    assert torch.equal(a, wq[None]) and torch.equal(b, wk[None])
    with pytest.raises(bacon.BaconError):
        bacon.bacon_rotate(rot, p, both[3:4, ::2], k)
    with pytest.raises(bacon.BaconError):
        bacon.bacon_rotate(rot, p, q, both[:2, 4:6])
    with pytest.raises(bacon.BaconError):
        bacon.bacon_rotate(rot, p, q, k, k_out=torch.empty_like(both[:2, 4:6]))
    rest = both[:, 6:].clone()
    bacon.bacon_rotate(rot, p, q, k, q_out=q, k_out=k)
    assert torch.equal(both[3:4, :4], wq) and torch.equal(both[3:4, 4:6], wk) and torch.equal(both[:, 6:], rest)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("d,r", [(128, 128), (64, 20)])
@pytest.mark.parametrize("eps", [0.0, 1e-60, 1e-30, 1e-6, 1e30])
def test_normalised_heads_of_any_magnitude(dtype, layout, d, r, eps):
    """Heads whose squares pass a float's range on either side, beside ordinary ones
    of the same token and wave, and with an eps that counts for some of them only."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(14)
    e = [0, 40, 58, 61, 64, 70, 100, 124, -30, -39, -41, -50, -63, -75, -100, -120]
    x = rng.uniform(0.5, 2, (len(e), 5, d)) * rng.choice([-1.0, 1.0], (len(e), 5, d))
    x[:, 1::2] *= 2.0 ** np.array(e)[:, None, None]             # (heads 0, 2, 4 stay as they are)
    x[3, 1, ::2] = 0
    x[6, 1, 5] *= 2.0 ** 20                                     # one value makes the sum
    t = torch.from_numpy(x.astype(np.float32)).cuda()
    t = t.bfloat16() if dtype == "bf16" else t
    w = torch.from_numpy(rng.uniform(0.5, 2, d).astype(np.float32)).cuda().to(t.dtype)
    pos = rng.integers(0, 5000, len(e))
    if eps == 1e30:                                             # outputs of the small ones are no normal floats
        t[8:, 1::2] = 0
    f, m = A.frequencies(r, 10000.0)
    got = bacon.bacon_rotate(_rotary(5, 1, d, dtype, r, layout, norm_eps=eps), _positions(pos), t, None, w)[0]
    assert torch.isfinite(got).all()
    _check(got, t, pos, f, m, layout, dtype, None, w, eps)


def test_normalised_heads_that_are_not_finite():
    """They are NaN where a value or the root is, and no head beside them changes."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(15)
    rot, pos = _rotary(4, 1, 64, "fp32", 32), _positions(np.arange(6))
    x, w = _rand(rng, 6, 4, 64, dtype="fp32"), torch.ones(64, device="cuda")
    want = bacon.bacon_rotate(rot, pos, x, None, w)[0]
    y = x.clone()
    y[1, 2, 40] = float("nan")
    y[4, 0, 41] = float("inf")
    got = bacon.bacon_rotate(rot, pos, y, None, w)[0]
    assert got[1, 2].isnan().all() and got[4, 0, 41].isnan() and (got[4, 0, 42:] == 0).all()
    same = torch.ones(6, 4, dtype=torch.bool, device="cuda")
    same[1, 2] = same[4, 0] = False
    assert torch.equal(got[same], want[same])
