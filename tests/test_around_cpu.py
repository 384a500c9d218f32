"""Host-side checks of positions, the prompt's attention and the cache's formats:
refusals before anything is enqueued, layouts and frequencies (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest

import around_ref as A
from paper_2606_14782_amd import bacon

FAKE = 0x200000
INV, UNS, WORK = bacon.ERR_INVALID, bacon.ERR_UNSUPPORTED, bacon.ERR_WORKSPACE


def _refused(status, want):
    assert status == want and bacon.lib().bacon_last_error()


# ---------------------------------------------------------------- rotary

def _rotary(**kw):
    r = bacon.RotaryParams()
    bacon.lib().bacon_default_rotary(C.byref(r))
    r.num_q_heads, r.num_kv_heads = 4, 2
    for k, v in kw.items():
        if k == "sections":
            r.sections[:] = v
        elif k == "frequencies":
            r.frequencies = v.ctypes.data_as(C.POINTER(C.c_double))
        else:
            setattr(r, k, v)
    return r


def _frequencies(r):
    f, m = np.full(64, -1.0), C.c_double()
    return bacon.lib().bacon_rotary_frequencies(C.byref(r), f.ctypes.data, C.byref(m)), f, m.value


def test_rotary_defaults():
    r = bacon.RotaryParams()
    bacon.lib().bacon_default_rotary(C.byref(r))
    assert (r.num_q_heads, r.num_kv_heads, r.head_dim, r.rotary_dim) == (1, 1, 128, 128)
    assert (r.layout, r.scaling, r.base, r.factor) == (bacon.ROTARY_HALF, bacon.ROTARY_PLAIN, 10000.0, 1.0)
    assert (r.beta_fast, r.beta_slow, r.magnitude, r.norm_eps, r.dtype) == (32.0, 1.0, 0.0, 1e-6, bacon.BF16)
    assert list(r.sections) == [0, 0, 0]


@pytest.mark.parametrize("name,kind,kw", [
    ("plain", bacon.ROTARY_PLAIN, {}), ("plain", bacon.ROTARY_PLAIN, dict(base=1e6, rotary_dim=48)),
    ("linear", bacon.ROTARY_LINEAR, dict(factor=8.0)), ("ntk", bacon.ROTARY_NTK, dict(factor=4.0, rotary_dim=64)),
    ("yarn", bacon.ROTARY_YARN, dict(factor=16.0, trained_tokens=4096, base=5e5)),
    ("yarn", bacon.ROTARY_YARN, dict(factor=1.0, trained_tokens=1)),
])
def test_frequencies_follow_their_formulas(name, kind, kw):
    r = _rotary(scaling=kind, **kw)
    st, f, m = _frequencies(r)
    want, wm = A.frequencies(r.rotary_dim, r.base, name, r.factor, r.trained_tokens)
    assert st == bacon.OK and m == wm
    np.testing.assert_allclose(f[:r.rotary_dim // 2], want, rtol=1e-14)
    assert (f[r.rotary_dim // 2:] == -1).all()


def test_yarn_keeps_fast_pairs_and_stretches_slow_ones():
    r = _rotary(scaling=bacon.ROTARY_YARN, factor=4.0, trained_tokens=8192, base=1e6)
    _, f, _ = _frequencies(r)
    w = _frequencies(_rotary(base=1e6))[1]                      # (the library's own: kept ones are kept exactly)
    turns = 8192 * w / (2 * np.pi)
    assert (f[turns >= 32] == w[turns >= 32]).all()
    np.testing.assert_allclose(f[turns <= 1], w[turns <= 1] / 4, rtol=1e-14)
    assert ((f >= w / 4 * (1 - 1e-14)) & (f <= w)).all()


def test_given_frequencies_and_magnitude():
    g = np.linspace(-1, 1, 64)
    st, f, m = _frequencies(_rotary(scaling=bacon.ROTARY_GIVEN, frequencies=g, magnitude=2.5, base=0, factor=0))
    assert st == bacon.OK and (f == g).all() and m == 2.5


BAD_ROTARY = [
    (dict(num_q_heads=0), INV), (dict(num_kv_heads=0), INV), (dict(num_q_heads=4097), UNS), (dict(dtype=3), UNS),
    (dict(head_dim=96), UNS), (dict(rotary_dim=0), INV), (dict(rotary_dim=130), INV), (dict(rotary_dim=7), INV),
    (dict(layout=2), INV), (dict(layout=-1), INV), (dict(sections=(-1, 33, 32)), INV), (dict(sections=(10, 10, 10)), INV),
    (dict(sections=(2 ** 31 - 1, 2 ** 31 - 1, 66)), INV),
    (dict(norm_eps=-1.0), INV), (dict(norm_eps=float("nan")), INV), (dict(magnitude=-1.0), INV),
    (dict(magnitude=float("inf")), INV), (dict(scaling=5), INV), (dict(scaling=-1), INV),
    (dict(scaling=bacon.ROTARY_GIVEN), INV), (dict(base=1.0), INV), (dict(base=float("inf")), INV),
    (dict(base=float("nan")), INV), (dict(factor=0.5), INV), (dict(factor=2.0), INV),
    (dict(scaling=bacon.ROTARY_LINEAR, factor=float("inf")), INV), (dict(scaling=bacon.ROTARY_NTK, rotary_dim=2), INV),
    (dict(scaling=bacon.ROTARY_YARN), INV), (dict(scaling=bacon.ROTARY_YARN, trained_tokens=9, beta_slow=0.0), INV),
    (dict(scaling=bacon.ROTARY_YARN, trained_tokens=9, beta_fast=1.0), INV),
    (dict(scaling=bacon.ROTARY_GIVEN, frequencies=np.array([np.nan] * 64)), INV),
    (dict(scaling=bacon.ROTARY_GIVEN, frequencies=np.array([0.0] * 63 + [1e7])), INV),
]


@pytest.mark.parametrize("kw,want", BAD_ROTARY)
def test_bad_rotary_refused(kw, want):
    r = _rotary(**kw)
    _refused(_frequencies(r)[0], want)
    _refused(_rotate(r), want)


def _rotate(r=None, **kw):
    a = dict(tokens=5, pos=FAKE, q=FAKE, qs=512, k=FAKE, ks=256, qn=None, kn=None, qo=FAKE, qos=512, ko=FAKE, kos=256)
    a.update(kw)
    r = r or _rotary()
    return bacon.lib().bacon_rotate(C.byref(r), a["tokens"], a["pos"], a["q"], a["qs"], a["k"], a["ks"], a["qn"], a["kn"],
                                    a["qo"], a["qos"], a["ko"], a["kos"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(tokens=-1), INV), (dict(tokens=(1 << 25) + 1), UNS), (dict(pos=None), INV), (dict(pos=FAKE + 2), INV),
    (dict(q=None), INV), (dict(k=None), INV), (dict(q=None, qo=None, k=None, ko=None), INV), (dict(qo=None), INV),
    (dict(ko=None), INV), (dict(q=FAKE + 8), INV), (dict(k=FAKE + 8), INV), (dict(qo=FAKE + 4), INV),
    (dict(ko=FAKE + 2), INV), (dict(qs=504), INV), (dict(qs=516, qo=FAKE * 2), INV), (dict(ks=248), INV),
    (dict(ks=260), INV), (dict(qos=500), INV), (dict(kos=0), INV), (dict(qs=-512), INV), (dict(qos=1024), INV),
    (dict(kos=512), INV), (dict(qn=FAKE + 8), INV), (dict(kn=FAKE + 4), INV),
])
def test_rotate_refused_before_enqueueing(kw, want):
    _refused(_rotate(**kw), want)


def test_rotate_of_nothing():
    assert _rotate(tokens=0, pos=None) == bacon.OK
    _refused(bacon.lib().bacon_rotate(None, 1, FAKE, FAKE, 512, FAKE, 256, None, None, FAKE, 512, FAKE, 256, None), INV)
    f = np.zeros(64)
    _refused(bacon.lib().bacon_rotary_frequencies(C.byref(_rotary()), None, f.ctypes.data), INV)
    _refused(bacon.lib().bacon_rotary_frequencies(C.byref(_rotary()), f.ctypes.data, None), INV)
    bacon.lib().bacon_default_rotary(None)


def test_binding_refuses_without_a_gpu():
    with pytest.raises(bacon.BaconError):
        bacon.Rotary(4, 2, 64, "fp16")
    with pytest.raises(bacon.BaconError):
        bacon.Rotary(4, 2, 64, "bf16", sections=(32,))
    with pytest.raises(bacon.BaconError):
        bacon.Rotary(4, 2, 64, "bf16", scaling=bacon.ROTARY_GIVEN, frequencies=[1.0])
    with pytest.raises(bacon.BaconError):
        bacon.Rotary(4, 2, 80, "bf16")
    r = bacon.Rotary(4, 2, 64, "fp32", 32, base=1e5)
    np.testing.assert_allclose(r.frequencies, A.frequencies(32, 1e5)[0], rtol=1e-14)
    import torch
    with pytest.raises(bacon.BaconError):
        bacon.bacon_rotate(r, torch.zeros(1, dtype=torch.int32), torch.zeros(1, 4, 64))
    with pytest.raises(bacon.BaconError):
        bacon.bacon_rotate(r, None)


@pytest.mark.parametrize("scaling", [None, bacon.ROTARY_PLAIN, bacon.ROTARY_LINEAR, bacon.ROTARY_NTK, bacon.ROTARY_YARN])
def test_frequencies_that_no_scaling_uses_refused(scaling):
    """A table is what turns the pairs, or the call ends: it is never dropped."""
    f = np.full(32, 0.5)
    kw = {} if scaling is None else dict(scaling=scaling, trained_tokens=4096)
    with pytest.raises(bacon.BaconError):
        bacon.Rotary(4, 2, 64, "bf16", frequencies=f, **kw)
    assert (bacon.Rotary(4, 2, 64, "bf16", scaling=bacon.ROTARY_GIVEN, frequencies=f).frequencies == 0.5).all()


# ---------------------------------------------------------------- prompt

def _shape(**kw):
    d = dict(num_layers=1, num_q_heads=8, num_kv_heads=2, head_dim=128, window=16, max_batch=4, max_total_tokens=100000,
             dtype=bacon.BF16)
    d.update(kw)
    return bacon.Shape(**d)


def _batch(lens):
    cu = np.concatenate([[0], np.cumsum(lens)])
    return bacon.BatchLayout(cu, [1] * len(lens))


def _prompt(shape=None, batch=None, cuq=None, work=FAKE, work_bytes=1 << 40, **kw):
    a = dict(q=FAKE, qs=1024, k=FAKE, ks=256, v=FAKE, vs=256, out=FAKE, lse=FAKE, win=FAKE)
    a.update(kw)
    shape, batch = shape or _shape(), batch or _batch([50, 60])
    q = None if cuq is None else np.ascontiguousarray(cuq, np.int32)
    return bacon.lib().bacon_prompt_attend(C.byref(shape), C.byref(batch.c), None if q is None else q.ctypes.data,
                                           a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["out"], a["lse"], a["win"],
                                           work, work_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(num_q_heads=7), INV), (dict(num_q_heads=0), INV), (dict(window=0), INV), (dict(max_batch=0), INV),
    (dict(max_total_tokens=0), INV), (dict(head_dim=96), UNS), (dict(dtype=2), UNS), (dict(max_batch=65), UNS),
    (dict(num_q_heads=4096, num_kv_heads=2), UNS), (dict(max_total_tokens=1 << 31), UNS), (dict(max_batch=1), INV),
    (dict(max_total_tokens=109), INV),
])
def test_prompt_shapes_refused(kw, want):
    _refused(_prompt(_shape(**kw)), want)
    b = _batch([50, 60])
    assert bacon.lib().bacon_prompt_work_bytes(C.byref(_shape(**kw)), C.byref(b.c), None) == 0


@pytest.mark.parametrize("kw,want", [
    (dict(cuq=[1, 2, 3]), INV), (dict(cuq=[0, 5, 4]), INV), (dict(batch=_batch([50, -1])), INV),
    (dict(q=None), INV), (dict(k=None), INV), (dict(v=None), INV), (dict(out=None), INV), (dict(q=FAKE + 8), INV),
    (dict(k=FAKE + 8), INV), (dict(v=FAKE + 2), INV), (dict(out=FAKE + 8), INV), (dict(lse=FAKE + 2), INV),
    (dict(win=FAKE + 1), INV), (dict(qs=1016), INV), (dict(ks=248), INV), (dict(vs=252), INV), (dict(qs=1028), INV),
    (dict(vs=260), INV), (dict(ks=-256), INV),
])
def test_prompt_refused_before_enqueueing(kw, want):
    _refused(_prompt(**kw), want)


def test_prompt_scratch():
    L, b, s = bacon.lib(), _batch([60000]), _shape()
    q = np.array([0, 3], np.int32)
    need = L.bacon_prompt_work_bytes(C.byref(s), C.byref(b.c), q.ctypes.data)
    assert need > 0 and need % 256 == 0
    _refused(_prompt(batch=b, cuq=q, work=None), INV)
    _refused(_prompt(batch=b, cuq=q, work=FAKE + 16), INV)
    _refused(_prompt(batch=b, cuq=q, work_bytes=need - 1), WORK)
    # a prompt that fills the GPU by itself needs none
    many = _batch([4000] * 4)
    assert L.bacon_prompt_work_bytes(C.byref(_shape(num_q_heads=64, num_kv_heads=8)), C.byref(many.c), None) == 0


def test_prompt_of_nothing():
    assert _prompt(batch=_batch([0, 0]), q=None, k=None, v=None, out=None) == bacon.OK
    assert _prompt(cuq=[0, 0, 0], q=None, out=None) == bacon.OK
    L, s = bacon.lib(), _shape()
    _refused(L.bacon_prompt_attend(None, C.byref(_batch([3]).c), None, *[FAKE, 1024] * 1, FAKE, 256, FAKE, 256, FAKE, None,
                                   None, None, 0, None), INV)
    _refused(L.bacon_prompt_attend(C.byref(s), None, None, FAKE, 1024, FAKE, 256, FAKE, 256, FAKE, None, None, None, 0,
                                   None), INV)
    empty = bacon.Batch(1, None, None, None)
    _refused(L.bacon_prompt_attend(C.byref(s), C.byref(empty), None, FAKE, 1024, FAKE, 256, FAKE, 256, FAKE, None, None,
                                   None, 0, None), INV)


def test_prompt_units_bounded():
    """More query rows than a launch's workgroups hold are refused on the host."""
    s = _shape(num_q_heads=1024, num_kv_heads=16, max_total_tokens=1 << 30, max_batch=64)
    _refused(_prompt(s, _batch([1 << 20] * 64), qs=1024 * 128, ks=16 * 128, vs=16 * 128), UNS)


# ---------------------------------------------------------------- formats of the cache

def _cache_shape(**kw):
    d = dict(num_layers=3, num_q_heads=8, num_kv_heads=2, head_dim=128, window=32, block_tokens=32, max_batch=4,
             max_blocks=10, num_blocks=200, dtype=bacon.BF16, format=bacon.CACHE_E2M1)
    d.update(kw)
    return bacon.CacheShape(**d)


@pytest.mark.parametrize("d,bt", [(64, 16), (64, 64), (128, 16), (128, 32), (128, 64)])
def test_layout_of_4_bits(d, bt):
    off = bacon.CacheOffsets()
    assert bacon.lib().bacon_cache_layout(C.byref(_cache_shape(head_dim=d, block_tokens=bt)), C.byref(off)) == bacon.OK
    pairs = 3 * 4 * 2
    sizes = {"errors": 4, "lens": 4 * pairs, "starts": 4 * pairs, "table": 4 * pairs * 10,
             "scales": 200 * 2 * bt * d // 32, "codes": 200 * bt * d}
    parts = sorted((getattr(off, n), n) for n in sizes)
    ends = [at for at, _ in parts[1:]] + [off.total]
    for (at, name), end in zip(parts, ends):
        assert at % 256 == 0 and at + sizes[name] <= end < at + sizes[name] + 256, name
    eight = bacon.CacheOffsets()
    bacon.lib().bacon_cache_layout(C.byref(_cache_shape(format=0, head_dim=d, block_tokens=bt)), C.byref(eight))
    assert eight.total - eight.codes >= 2 * (off.total - off.codes) - 256


@pytest.mark.parametrize("fmt", [-1, 2, 7])
def test_formats_that_are_none_refused(fmt):
    off, h = bacon.CacheOffsets(), C.c_void_p()
    s = _cache_shape(format=fmt)
    _refused(bacon.lib().bacon_cache_layout(C.byref(s), C.byref(off)), UNS)
    _refused(bacon.lib().bacon_cache_init(C.byref(h), C.byref(s), C.c_void_p(0x100000), 1 << 50), UNS)
    with pytest.raises(bacon.BaconError):
        bacon.Cache(1, 4, 2, 64, 8, 16, 1, 64, 8, "bf16", format="int4")


def test_a_shape_without_a_format_is_in_8_bits():
    s = bacon.CacheShape(3, 8, 2, 128, 32, 32, 4, 10, 200, bacon.BF16)
    assert s.format == bacon.CACHE_E4M3


def _chunk(ends, **kw):
    s, b, e = _shape(), _batch([50, 60]), np.asarray(ends, np.int32)
    a = dict(cuq=[0, 10, 20], q=FAKE)
    a.update(kw)
    q = np.asarray(a["cuq"], np.int32)
    return bacon.lib().bacon_prompt_attend_chunk(C.byref(s), C.byref(b.c), q.ctypes.data, e.ctypes.data, a["q"], 1024, FAKE,
                                                 256, FAKE, 256, FAKE, FAKE, FAKE, FAKE, 1 << 40, None)


def test_window_ends_before_the_keys_refused():
    for ends in ([49, 60], [50, 59], [0, 0], [-1, 60], [50, -2 ** 31]):
        _refused(_chunk(ends), INV)
        _refused(_chunk(ends, cuq=[0, 0, 0]), INV)              # (also of a sequence without queries)
    _refused(_chunk([50, 2 ** 31 - 1], q=None), INV)            # the other checks are bacon_prompt_attend's
    assert _chunk([50, 2 ** 31 - 1], cuq=[0, 0, 0]) == bacon.OK


def test_the_format_lies_in_former_padding():
    """Callers built without the field: the same size, every other field in its place."""
    before = [(n, t) for n, t in bacon.CacheShape._fields_ if n != "format"]

    class Old(C.Structure):
        _fields_ = before

    assert C.sizeof(Old) == C.sizeof(bacon.CacheShape) == 48
    for n, _ in before:
        assert getattr(Old, n).offset == getattr(bacon.CacheShape, n).offset, n
    assert bacon.CacheShape.format.offset == Old.dtype.offset + 4
    old, a, b = Old(3, 8, 2, 128, 32, 32, 4, 10, 200, bacon.BF16), bacon.CacheOffsets(), bacon.CacheOffsets()
    L = bacon.lib()
    assert L.bacon_cache_layout(C.cast(C.byref(old), C.POINTER(bacon.CacheShape)), C.byref(a)) == bacon.OK
    assert L.bacon_cache_layout(C.byref(_cache_shape(format=bacon.CACHE_E4M3)), C.byref(b)) == bacon.OK
    assert a.total == b.total and a.codes == b.codes
