"""Host-side checks of the 8-bit cache: layouts, and refusals of every call
before anything is enqueued (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest

import cache_ref as R
from paper_2606_14782_amd import bacon

FAKE = 0x200000


def _shape(**kw):
    d = dict(num_layers=3, num_q_heads=8, num_kv_heads=2, head_dim=128, window=32, block_tokens=32,
             max_batch=4, max_blocks=10, num_blocks=200, dtype=bacon.BF16)
    d.update(kw)
    return bacon.CacheShape(**d)


def _cache(**kw):
    L, shape, off, h = bacon.lib(), _shape(**kw), bacon.CacheOffsets(), C.c_void_p()
    assert L.bacon_cache_layout(C.byref(shape), C.byref(off)) == bacon.OK
    assert L.bacon_cache_init(C.byref(h), C.byref(shape), C.c_void_p(0x100000), off.total) == bacon.OK
    return h


def test_layout_holds_every_part():
    off = bacon.CacheOffsets()
    assert bacon.lib().bacon_cache_layout(C.byref(_shape()), C.byref(off)) == bacon.OK
    pairs = 3 * 4 * 2
    sizes = {"errors": 4, "lens": 4 * pairs, "starts": 4 * pairs, "table": 4 * pairs * 10, "scales": 8 * 200,
             "codes": 200 * 2 * 32 * 128}
    parts = sorted((getattr(off, n), n) for n in sizes)
    ends = [at for at, _ in parts[1:]] + [off.total]
    for (at, name), end in zip(parts, ends):
        assert at % 256 == 0 and at + sizes[name] <= end, name


def test_layout_counts_past_32_bits():
    off = bacon.CacheOffsets()
    s = _shape(num_blocks=1 << 20, block_tokens=64)
    assert bacon.lib().bacon_cache_layout(C.byref(s), C.byref(off)) == bacon.OK
    assert off.total > (1 << 34)


@pytest.mark.parametrize("kw,status", [
    (dict(num_q_heads=7), bacon.ERR_INVALID), (dict(num_layers=0), bacon.ERR_INVALID),
    (dict(window=0), bacon.ERR_INVALID), (dict(max_batch=0), bacon.ERR_INVALID),
    (dict(max_blocks=0), bacon.ERR_INVALID), (dict(num_blocks=0), bacon.ERR_INVALID),
    (dict(head_dim=96), bacon.ERR_UNSUPPORTED), (dict(block_tokens=48), bacon.ERR_UNSUPPORTED),
    (dict(block_tokens=128), bacon.ERR_UNSUPPORTED), (dict(max_batch=65), bacon.ERR_UNSUPPORTED),
    (dict(dtype=5), bacon.ERR_UNSUPPORTED), (dict(num_blocks=1 << 31), bacon.ERR_UNSUPPORTED),
    (dict(max_blocks=1 << 30), bacon.ERR_UNSUPPORTED), (dict(num_layers=1 << 25), bacon.ERR_UNSUPPORTED),
    (dict(num_q_heads=130), bacon.ERR_UNSUPPORTED),
    (dict(num_q_heads=2000, num_kv_heads=2000), bacon.ERR_UNSUPPORTED),
])
def test_bad_shapes_refused(kw, status):
    off, h = bacon.CacheOffsets(), C.c_void_p()
    s = _shape(**kw)
    assert bacon.lib().bacon_cache_layout(C.byref(s), C.byref(off)) == status
    assert bacon.lib().bacon_last_error()
    assert bacon.lib().bacon_cache_init(C.byref(h), C.byref(s), C.c_void_p(0x100000), 1 << 50) == status
    assert not h.value


def test_init_checks_its_memory():
    L, s, off, h = bacon.lib(), _shape(), bacon.CacheOffsets(), C.c_void_p()
    L.bacon_cache_layout(C.byref(s), C.byref(off))
    assert L.bacon_cache_init(C.byref(h), C.byref(s), C.c_void_p(0x100010), off.total) == bacon.ERR_WORKSPACE
    assert L.bacon_cache_init(C.byref(h), C.byref(s), C.c_void_p(0x100000), off.total - 1) == bacon.ERR_WORKSPACE
    assert L.bacon_cache_init(C.byref(h), C.byref(s), None, off.total) == bacon.ERR_INVALID
    assert L.bacon_cache_init(None, C.byref(s), C.c_void_p(0x100000), off.total) == bacon.ERR_INVALID
    assert L.bacon_cache_layout(C.byref(s), None) == bacon.ERR_INVALID
    assert L.bacon_cache_free(None) == bacon.ERR_INVALID


def test_calls_refused_before_enqueueing():
    L, h = bacon.lib(), _cache()
    INV, UNS, ORD = bacon.ERR_INVALID, bacon.ERR_UNSUPPORTED, bacon.ERR_ORDER
    f, odd = C.c_void_p(FAKE), C.c_void_p(FAKE + 2)
    b2 = bacon.BatchLayout([0, 100, 300], [16, 32])
    hb = bacon.BatchLayout([0, 100, 300], [16, 32], head_budgets=np.full((2, 2), 8))
    arr = (C.c_void_p * 3)(FAKE, FAKE, FAKE)
    bad = (C.c_void_p * 3)(FAKE, FAKE + 4, FAKE)
    # clear
    for first, n in ((-1, 1), (0, 0), (0, 5), (3, 2), (4, 1)):
        assert L.bacon_cache_clear(h, first, n, None) == INV
    assert L.bacon_cache_clear(None, 0, 1, None) == INV

    # tables(cache, batch, first, budgets, budgets_batch, reserve, free, num_free, used)
    def tables(c=h, bt=b2, first=0, bud=None, nb=0, reserve=0, free=None, nf=0, used=None):
        return L.bacon_cache_tables(c, C.byref(bt.c) if bt else None, first, bud, nb, reserve, free, nf, used, None)
    assert tables(c=None) == INV and tables(bt=None) == INV
    assert tables(first=3) == INV and tables(first=-1) == INV
    assert tables(bt=hb) == INV and b"d_budgets" in L.bacon_last_error()
    assert tables(bt=bacon.BatchLayout([0, 10], [4])) == INV          # shorter than the window
    assert tables(bt=bacon.BatchLayout([5, 100], [4])) == INV
    assert tables(bt=bacon.BatchLayout([0, 100], [0])) == INV
    assert tables(bud=odd, nb=2) == INV and tables(bud=f, nb=1) == INV
    assert tables(reserve=-1) == INV and tables(reserve=321) == INV
    assert tables(free=odd, nf=4) == INV and tables(free=f, nf=-1) == INV
    assert tables(used=C.c_void_p(FAKE + 4)) == INV
    assert tables() == ORD and tables(bud=f, nb=2, bt=hb) == ORD      # head_budgets unread with d_budgets

    def store(c=h, bt=b2, first=0, fl=0, nl=3, k=arr, v=arr, idx=arr, count=96):
        return L.bacon_cache_store(c, C.byref(bt.c) if bt else None, first, fl, nl, k, v, idx, count, None)
    assert store(c=None) == INV and store(bt=None) == INV and store(first=3) == INV
    assert store(fl=1) == INV and store(fl=-1) == INV and store(nl=0) == INV
    assert store(k=None) == INV and store(v=None) == INV and store(k=bad) == INV and store(v=bad) == INV
    assert store(idx=(C.c_void_p * 3)(FAKE, None, FAKE)) == INV
    assert store(count=-1) == INV
    assert store() == ORD and store(idx=None) == ORD

    def load(c=h, fl=0, nl=3, fs=0, ns=4, ft=0, n=8, k=f, v=f):
        return L.bacon_cache_load(c, fl, nl, fs, ns, ft, n, k, v, None)
    assert load(c=None) == INV and load(nl=4) == INV and load(ns=5) == INV and load(n=0) == INV
    assert load(k=None) == INV and load(v=C.c_void_p(FAKE + 4)) == INV and load(ft=-(1 << 31)) == INV
    assert load() == ORD

    def append(c=h, layer=0, fs=0, ns=2, n=1, counts=None, k=f, ks=256, v=f, vs=256):
        return L.bacon_cache_append(c, layer, fs, ns, n, counts, k, ks, v, vs, None)
    assert append(c=None) == INV and append(layer=3) == INV and append(layer=-1) == INV and append(ns=5) == INV
    assert append(n=0) == INV and append(n=65) == UNS and append(counts=odd) == INV
    assert append(k=None) == INV and append(v=C.c_void_p(FAKE + 8)) == INV
    assert append(ks=255) == INV and append(vs=257) == INV and append(vs=-256) == INV
    assert append() == ORD

    def attend(c=h, layer=0, fs=0, ns=2, n=1, counts=None, q=f, qs=1024, most=0, out=f, lse=None):
        return L.bacon_cache_attend(c, layer, fs, ns, n, counts, q, qs, most, out, lse, f, 1 << 40, None)
    assert attend(c=None) == INV and attend(layer=3) == INV and attend(fs=3) == INV and attend(ns=0) == INV
    assert attend(n=0) == INV and attend(n=17) == UNS and attend(most=-1) == INV        # G * n = 68
    assert attend(q=None) == INV and attend(qs=1020) == INV and attend(out=None) == INV
    assert attend(out=C.c_void_p(FAKE + 8)) == INV and attend(lse=odd) == INV
    assert attend() == ORD

    def step(n=1, k=f, q=f, ks=256):
        return L.bacon_cache_step(h, 0, 0, 2, n, None, q, 1024, k, ks, f, 256, 0, f, None, f, 1 << 40, None)
    assert step(k=None) == INV and step(q=None) == INV and step(n=17) == UNS and step(ks=8) == INV
    assert step() == ORD

    def advance(c=h, fl=0, nl=3, fs=0, ns=4, d=None):
        return L.bacon_cache_advance(c, fl, nl, fs, ns, 1, d, None)
    assert advance(c=None) == INV and advance(fl=3) == INV and advance(ns=5) == INV and advance(d=odd) == INV
    assert advance() == ORD
    assert L.bacon_cache_errors(None) == -1
    L.bacon_cache_free(h)


def test_work_is_asked_for_and_checked():
    L, h = bacon.lib(), _cache(max_blocks=4096, num_blocks=5000)
    need = L.bacon_cache_work_bytes(h, 1, 1, 131072)
    f = C.c_void_p(FAKE)

    def attend(work, nbytes, most=131072):
        return L.bacon_cache_attend(h, 0, 0, 1, 1, None, f, 1024, most, f, None, work, nbytes, None)
    if need:
        assert attend(None, need) == bacon.ERR_INVALID
        assert attend(C.c_void_p(FAKE + 16), need) == bacon.ERR_INVALID
        assert attend(f, need - 1) == bacon.ERR_WORKSPACE
    assert attend(f, need) == bacon.ERR_ORDER
    # nonsense asks for nothing
    assert L.bacon_cache_work_bytes(None, 1, 1, 0) == 0
    assert L.bacon_cache_work_bytes(h, 0, 1, 0) == 0 and L.bacon_cache_work_bytes(h, 1, 0, 0) == 0
    L.bacon_cache_free(h)


def test_binding_refuses_other_devices_and_dtypes():
    for kw, status in ((dict(device="cpu"), bacon.ERR_INVALID), (dict(dtype="fp16"), bacon.ERR_UNSUPPORTED),
                       (dict(block_tokens=0), bacon.ERR_INVALID), (dict(block_tokens=24), bacon.ERR_UNSUPPORTED),
                       (dict(max_tokens=0), bacon.ERR_INVALID)):
        a = dict(num_layers=1, num_q_heads=4, num_kv_heads=2, head_dim=64, window=8, block_tokens=16, max_batch=2,
                 max_tokens=100, num_blocks=10, dtype="bf16", device="cpu")
        a.update(kw)
        with pytest.raises(bacon.BaconError) as e:
            bacon.Cache(**a)
        assert e.value.status == status, kw


def test_reference_rounding():
    """The test's own rounding: values, ties to even, the exponents' borders."""
    assert R.E4M3[-1] == 448.0 and len(R.E4M3) == 127
    assert R.exponent(448.0) == 0 and R.exponent(448.0001) == 1 and R.exponent(1.75) == -8
    assert R.exponent(0.0) == -100 and R.exponent(2.0 ** -130) == -100 and R.exponent(2.0 ** 127) == 119
    x = np.array([17.0, 19.0, 18.0, -21.0, 2.0 ** -10, 3 * 2.0 ** -10, 447.0])
    assert R.round8(x, 0).tolist() == [16.0, 20.0, 18.0, -20.0, 0.0, 2.0 ** -8, 448.0]
    r = R.Rows(4, 2)
    r.append(np.full((6, 2), 1.0))
    r.append(np.full((1, 2), 1000.0))
    assert len(r) == 7 and r.e[0] == R.exponent(1.0) and r.e[1] == R.exponent(1000.0)
    assert np.allclose(r.x[4:6], 1.0) and np.allclose(r.x[6], 1024.0)


def test_a_load_of_more_threads_than_a_launch_holds_is_refused():
    """2^24 workgroups of 256 threads are one launch too large; one fewer goes on
    to the next check."""
    f = C.c_void_p(FAKE)
    kw = dict(num_q_heads=1024, num_kv_heads=1024, max_batch=64, max_blocks=1, num_blocks=1, block_tokens=16)
    for d, layers, count, status in ((64, 256, 1, bacon.ERR_UNSUPPORTED), (64, 255, 1, bacon.ERR_ORDER),
                                     (64, 255, 112, bacon.ERR_ORDER), (64, 255, 113, bacon.ERR_UNSUPPORTED),
                                     (128, 256, 48, bacon.ERR_UNSUPPORTED), (128, 255, 48, bacon.ERR_ORDER),
                                     (128, 255, 49, bacon.ERR_UNSUPPORTED), (128, 1, 1 << 30, bacon.ERR_UNSUPPORTED)):
        h = _cache(num_layers=layers, head_dim=d, **kw)
        assert bacon.lib().bacon_cache_load(h, 0, layers, 0, 64, 0, count, f, f, None) == status, (d, layers, count)
        bacon.lib().bacon_cache_free(h)
