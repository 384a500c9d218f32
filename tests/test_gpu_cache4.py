"""The cache in e2m1 on the GPU against plain 64-bit numpy (around_ref).

Stored, appended and loaded values are exact (scales are powers of two, every
rounding is to nearest even); attention is held to the bounds that
cache_ref.attend derives.  The tests of the 8-bit cache that say nothing of its
numbers run for this format too, on the same lengths, tables, masks and calls."""
import numpy as np
import pytest

import around_ref as A
import test_gpu_cache as T

pytestmark = pytest.mark.gpu


def _cache4(L, hq, hkv, d, W, bt, B, most, blocks, dtype):
    """A cleared cache whose pool holds bytes that no row put there: scales of NaN."""
    from paper_2606_14782_amd import bacon
    c = bacon.Cache(L, hq, hkv, d, W, bt, B, most, blocks, dtype, format="e2m1")
    c.memory.fill_(0x7F)
    c.scales.fill_(0xFF)
    c.bacon_cache_clear()
    return c


@pytest.fixture(autouse=True)
def _e2m1(monkeypatch):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    monkeypatch.setattr(T, "_cache", _cache4)
    monkeypatch.setattr(T.R, "Rows", A.Rows4)
    attend = T.R.attend
    monkeypatch.setattr(T.R, "attend", lambda q, k, v, dtype: A.attend_held(attend, q, k, v, dtype))


def test_values_over_the_range_of_magnitudes():
    """Every rounding of e2m1 with its ties, rows of zeros, the least and the
    largest magnitudes, scales on both sides of a power of two."""
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(5)
    d, W, n = 64, 1, 160
    x = rng.standard_normal((n, 1, d)).astype(np.float32)
    x[:8] = 0
    x[8:16] *= 2.0 ** -140
    x[16:24] = np.clip(x[16:24], -1, 1) * 2.0 ** 127
    x[24:90, 0] = rng.integers(-48, 49, (66, d)) / 8.0
    x[24:90, 0, ::32] = 6
    x[90, 0, ::32] = 6 * (1 + 2.0 ** -23)
    x[91, 0] = np.linspace(-6, 6, d)
    x[92:100] *= 2.0 ** 20
    x[100:108] *= 2.0 ** -60
    x[108, 0, :32] = 2.0 ** 126 * 1.5
    x[109, 0, 0] = 2.0 ** 127
    for dtype in ("fp32", "bf16"):
        t = torch.from_numpy(x).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)
        want = A.held(T._np(t)[:, 0])
        c = _cache4(1, 1, 1, d, W, 16, 1, n + 16, 11, dtype)
        batch = bacon.BatchLayout([0, n], [n - W])
        c.bacon_cache_tables(batch, None, 16)
        c.bacon_cache_store(batch, [t], [t])
        k, v = c.bacon_cache_load(n)
        np.testing.assert_array_equal(T._np(k)[0, 0, 0], want)
        np.testing.assert_array_equal(T._np(v)[0, 0, 0], want)
        # the same values appended, in runs of up to 64 tokens
        c.bacon_cache_clear()
        c.bacon_cache_tables(bacon.BatchLayout([0, 1], [1]), None, n)
        for at in range(0, n, 64):
            rows = t[at:at + 64][None]
            c.bacon_cache_append(0, rows, rows)
        k, v = c.bacon_cache_load(n, first_token=-n)
        np.testing.assert_array_equal(T._np(k)[0, 0, 0], want)
        np.testing.assert_array_equal(T._np(v)[0, 0, 0], want)


def test_layout_is_as_the_header_says():
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(6)
    d, bt, n = 128, 32, 75
    c = _cache4(1, 1, 1, d, 1, bt, 1, n, 5, "fp32")
    batch = bacon.BatchLayout([0, n], [n - 1])
    c.bacon_cache_tables(batch, None, 0, torch.tensor([3, 0, 4], dtype=torch.int32, device="cuda"))
    k, v = (T._rand(rng, n, 1, d, dtype="fp32") for _ in range(2))
    c.bacon_cache_store(batch, [k], [v])
    scales, codes = c.scales.cpu().numpy().astype(int), c.codes.cpu().numpy()
    values = np.concatenate([A.E2M1, -A.E2M1])
    for kv, x in ((0, k), (1, v)):
        want = A.held(T._np(x)[:, 0])
        for p in (0, 1, 15, 16, 31, 32, 63, 64, 74):
            blk, r = (3, 0, 4)[p // bt], p % bt
            row = codes[blk, kv]
            byte = row.reshape(bt, d // 2)[r] if kv == 0 else row.reshape(bt // 16, d // 2, 16)[r // 16, :, r % 16]
            y = np.stack([values[byte & 15], values[byte >> 4]], -1).reshape(d)
            e = scales[blk, kv, r // 16, :, r % 16] - 127
            np.testing.assert_array_equal(y * np.repeat(2.0 ** e, 32), want[p])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,bt", [(64, 16), (64, 64), (128, 16), (128, 32), (128, 64)])
def test_store_whole_rows(dtype, d, bt):
    T.test_store_whole_rows(dtype, d, bt)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_store_gathers_idx(dtype):
    T.test_store_gathers_idx(dtype)


def test_store_of_bad_indices_and_many_layers():
    T.test_store_of_a_bad_index_is_a_zero_row()
    T.test_store_of_many_layers()


@pytest.mark.parametrize("first,count", [(0, 1), (3, 40), (-1, 1), (-20, 20), (-50, 7), (60, 10), (1000, 3)])
def test_load_ranges(first, count):
    T.test_load_ranges(first, count)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,bt", [(64, 16), (128, 32), (64, 64)])
@pytest.mark.parametrize("n", [1, 3, 17, 64])
def test_append(dtype, d, bt, n):
    T.test_append(dtype, d, bt, n)


def test_append_counts_room_and_one_by_one():
    T.test_append_counts_and_empty_sequences()
    T.test_append_without_room_leaves_the_pair()
    T.test_append_one_by_one_equals_the_reference()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,bt", [(64, 16), (128, 32), (128, 64)])
@pytest.mark.parametrize("G,n", [(1, 1), (7, 1), (4, 5), (16, 4), (8, 3)])
def test_attend(dtype, d, bt, G, n):
    T.test_attend(dtype, d, bt, G, n)


@pytest.mark.parametrize("dtype,d,G,n,most", [("bf16", 128, 4, 1, 5000), ("fp32", 64, 7, 5, 3000),
                                              ("bf16", 64, 8, 8, 2000), ("bf16", 128, 7, 5, 9000)])
def test_attend_long_and_ragged(dtype, d, G, n, most):
    T.test_attend_long_and_ragged(dtype, d, G, n, most)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,G,n", [(128, 1, 1), (64, 4, 6)])
def test_attend_many_pairs(dtype, d, G, n):
    T.test_attend_many_pairs(dtype, d, G, n)


def test_attend_padded_empty_and_absent():
    T.test_attend_padded_and_empty()
    T.test_attend_of_large_and_equal_logits()
    T.test_attend_over_absent_blocks()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,bt", [(64, 16), (128, 32), (128, 64)])
@pytest.mark.parametrize("G,n", [(1, 1), (7, 4), (16, 4), (2, 17)])
def test_step_is_append_then_attend(dtype, d, bt, G, n):
    T.test_step_is_append_then_attend(dtype, d, bt, G, n)


def test_step_without_room_rolled_back_and_views():
    T.test_step_without_room_attends_over_what_is_there()
    T.test_rolled_back_tokens()
    T.test_views_of_a_projection()


def test_streams_and_graphs():
    T.test_two_streams_attend_beside_each_other()
    T.test_two_captured_graphs_replay_beside_each_other()
    T.test_tables_and_store_in_a_captured_graph()


@pytest.mark.parametrize("lens", [[[40, 33], [100, 7]], [[4000, 2100], [9, 100]]])
def test_captured_step_replays(lens):
    T.test_captured_step_replays(lens)


@pytest.mark.parametrize("dtype,d,bt,G,n,part", [
    ("bf16", 128, 64, 4, 4, 64), ("bf16", 64, 16, 1, 16, 64), ("fp32", 64, 32, 5, 3, 64), ("bf16", 128, 64, 5, 6, 256),
    ("fp32", 128, 32, 8, 4, 256)])
def test_step_over_the_borders_of_parts(dtype, d, bt, G, n, part):
    T.test_step_over_the_borders_of_parts(dtype, d, bt, G, n, part)


@pytest.mark.parametrize("dtype,d,G,n", [("bf16", 128, 4, 1), ("fp32", 64, 7, 3)])
@pytest.mark.parametrize("lens", [[[40, 1], [300, 65]], [[4100, 2000], [3, 1000]]])
def test_a_query_that_is_not_finite_is_nan_alone(dtype, d, G, n, lens):
    T.test_a_query_that_is_not_finite_is_nan_alone(dtype, d, G, n, lens)


@pytest.mark.parametrize("dtype,d,G", [("bf16", 128, 4), ("fp32", 64, 1), ("bf16", 64, 20)])
@pytest.mark.parametrize("rows", [1, 300, 5000])
def test_attend_of_logits_as_large_as_floats(dtype, d, G, rows):
    """Logits of either sign up to 2^120 of two kinds of key, 4 and 6 (exact in e2m1):
    the larger ones' weights are 1, the others' 0.  The bounds are those of the
    8-bit cache's test of the same: sums, and the output's rounding."""
    import math
    import torch
    from paper_2606_14782_amd import bacon
    rng = np.random.default_rng(rows)
    for power in (40, 104, 117):
        for sign in (1, -1):
            q = torch.zeros(1, 1, G, d, device="cuda")
            q[..., 0] = sign * 2.0 ** (power - power // 2)
            kind = rng.integers(0, 2, rows)
            key = np.where(kind == 1, 6.0, 4.0) * 2.0 ** (power // 2)
            k = torch.zeros(rows, 1, d, device="cuda")
            k[:, 0, 0] = torch.from_numpy(key.astype(np.float32)).cuda()
            v = torch.from_numpy(rng.standard_normal((rows, 1, d)).astype(np.float32)).cuda()
            q, k, v = (x.to(torch.bfloat16 if dtype == "bf16" else torch.float32) for x in (q, k, v))
            c = _cache4(1, G, 1, d, 1, 32, 1, rows, rows // 32 + 2, dtype)
            batch = bacon.BatchLayout([0, rows], [max(1, rows - 1)])
            c.bacon_cache_tables(batch)
            c.bacon_cache_store(batch, [k], [v])
            out, lse = c.bacon_cache_attend(0, q, want_lse=True)
            s = sign * 2.0 ** (power - power // 2) * key / math.sqrt(d)
            won = A.held(T._np(v)[:, 0])[s == s.max()]
            tol = A.HALF[dtype] * np.abs(won.mean(0)) + (2 * (rows / 16 + 64) + 4) * A.h * np.abs(won).mean(0) * 1.01
            assert np.all(np.abs(T._np(out)[0, 0] - won.mean(0)) <= tol), (power, sign)
            want = s.max() + math.log(len(won))
            assert np.all(np.abs(T._np(lse)[0, 0] - want) <= 8 * A.h * np.abs(want)), (power, sign)


@pytest.mark.parametrize("dtype,G,n", [("bf16", 4, 1), ("fp32", 2, 3)])
def test_divided_step_without_room_attends_over_what_is_there(dtype, G, n):
    T.test_divided_step_without_room_attends_over_what_is_there(dtype, G, n)


def test_rows_not_named_and_padding():
    T.test_rows_that_are_not_named_stay()
    T.test_padding_may_hold_anything([[40, 33], [100, 7]])


def test_attend_over_the_longest():
    T.test_attend_over_the_longest()
