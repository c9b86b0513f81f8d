"""The bounded cache's plans and refusals through the C ABI, on the CPU: work lists of
the fp8 store, the key weights and the eviction against oracle/cache_ref.py, the host
page table's truncation, pins of the oracle itself, and every host-side rejection."""
import ctypes

import numpy as np
import pytest

from oracle import cache_ref as R
from oracle import fp8_ref
from paper_2601_12784_amd import binding as B

FAKE = 0x10000   # aligned, never dereferenced
OK, INVALID, UNSUPPORTED, CAPACITY, MISMATCH = 0, 1, 2, 3, 4

LENGTHS = [
    ([37, 5, 64], [37, 5, 64]),
    ([90, 33, 17, 48], [20, 1, 17, 16]),
    ([40, 16, 1, 0], [0, 9, 1, 0]),
    ([5000, 300, 1200], [5000, 44, 1]),
    ([20000, 16000], [20000, 16000]),      # runs of four pages
    ([17, 64, 130, 300], [1, 1, 1, 1]),
    ([30000] * 20, [1] * 20),              # more than 16 pages per item
    ([], []),
]


def _desc(lens, hq=28, hkv=4, d=128, stride=None, pages=None):
    need = [-(-n // 16) for n in lens]
    return B.make_desc(len(lens), hq, hkv, d, stride or max(need, default=1) or 1, pages or max(1, sum(need)), 0.1)


def _rows(work, info, ints):
    return np.asarray(work)[: info.work_bytes // 4].reshape(-1, ints).tolist()


def test_struct_sizes():
    assert ctypes.sizeof(B.sf_store_info) == 24
    assert ctypes.sizeof(B.sf_weights_info) == 48
    assert ctypes.sizeof(B.sf_evict_info) == 56


@pytest.mark.parametrize("lens,news", LENGTHS)
def test_store_plan(lens, news):
    info, work = B.sf_kv_store_fp8_plan(_desc(lens), lens, news)
    want = R.store_plan(lens, news)
    assert info.num_rows == len(want) and info.num_q_rows == sum(news)
    assert _rows(work, info, 8) == want


@pytest.mark.parametrize("lens,news", LENGTHS)
@pytest.mark.parametrize("heads", [(28, 4), (8, 8), (16, 1)])
def test_weights_plan(lens, news, heads):
    hq, hkv = heads
    info, work = B.sf_key_weights_plan(_desc(lens, hq, hkv), lens, news)
    items, merges, waves = R.weights_plan(lens, news, hq, hkv)
    assert (info.num_items, info.num_merge, info.steps) == (len(items), len(merges), waves)
    assert _rows(work, info, 16) == items + merges
    seen = {}
    for s, h, p0, p1, t0, t1, slot, L, P, cu, held, pos, following, *rest in items:
        assert 0 <= t0 < t1 <= news[s] and 0 <= p0 < p1 <= -(-L // 16) and rest == [0] * 3
        seen.setdefault((s, h) if waves else (s, h, p0), []).append((p0, p1) if waves else (t0, t1))
    if waves:   # the segments of every (sequence, KV head) cover its pages once
        for (s, h), spans in seen.items():
            spans.sort()
            assert spans[0][0] == 0 and spans[-1][1] == -(-lens[s] // 16)
            assert all(a[1] == b[0] for a, b in zip(spans, spans[1:]))
        return
    # the parts of every block of keys cover the query rows that see it once
    for (s, h, p0), spans in seen.items():
        spans.sort()
        assert spans[0][0] == max(0, p0 * 16 - (lens[s] - news[s])) and spans[-1][1] == news[s]
        assert all(a[1] == b[0] for a, b in zip(spans, spans[1:]))


def test_weights_plan_held_and_positions():
    lens, news, held, pos = [40, 9], [3, 9], [20, 0], [100, 7]
    info, work = B.sf_key_weights_plan(_desc(lens), lens, news, held_lens=held, first_pos=pos, opts=B.make_opts(num_cus=1))
    items, merges, _ = R.weights_plan(lens, news, 28, 4, held, pos, num_cus=1)
    assert _rows(work, info, 16) == items + merges
    for bad in (dict(held_lens=[-1, 0]), dict(held_lens=[41, 0]), dict(first_pos=[-1, 0]),
                dict(held_lens=held, first_pos=[2**31 - 20, 0])):
        with pytest.raises(B.SfError) as e:
            B.sf_key_weights_plan(_desc(lens), lens, news, **bad)
        assert e.value.status == INVALID


@pytest.mark.parametrize("lens,keep", [([40, 17, 0, 16], [20, 17, 5, 0]), ([3, 40000, 7, 4097, 4096], [9, 36000, 3, 4097, 1]), ([40000, 9000], [33333, 20]), ([33], [16]), ([], [])])
def test_evict_plan(lens, keep):
    hkv = 4
    info, work = B.sf_kv_evict_plan(_desc(lens), lens, keep)
    rows, moved, hole, tail = R.evict_plan(lens, keep, hkv)
    assert _rows(work, info, 8) == rows + moved
    assert (info.num_seqs, info.num_moves, info.hole_pages) == (len(lens), len(moved), hole)
    assert info.workspace_bytes == (hole * 8 + 255) // 256 * 256 + tail * 4
    assert info.num_long == sum(n > 4096 for n in lens)
    assert bool(info.boundary) == any(min(k, n) < n and min(k, n) % 16 for n, k in zip(lens, keep))


def test_evict_plan_rejects():
    desc = _desc([40, 40])
    for kw in (dict(keep_lens=[-1, 4]), dict(keep_lens=[20, 20], sinks=-1), dict(keep_lens=[20, 20], recent=-1),
               dict(keep_lens=[20, 19], sinks=4, recent=16), dict(keep_lens=[20, 20], ends=[40, 39])):
        with pytest.raises(B.SfError) as e:
            B.sf_kv_evict_plan(desc, [40, 40], **kw)
        assert e.value.status == INVALID
    for lens in ([-1, 40], [40, 49]):     # 49 tokens do not fit 3 pages
        with pytest.raises(B.SfError):
            B.sf_kv_evict_plan(desc, lens, [0, 0])
    # all protected and short: fine
    B.sf_kv_evict_plan(desc, [10, 40], [10, 20], sinks=4, recent=16)


@pytest.mark.parametrize("plan", [B.sf_kv_store_fp8_plan, B.sf_key_weights_plan])
def test_new_token_plans_reject_bad_lengths(plan):
    for lens, news in (([40], [41]), ([40], [-1]), ([49], [1])):
        with pytest.raises(B.SfError) as e:
            plan(_desc([40], stride=3), lens, news)
        assert e.value.status == INVALID
    big = B.make_desc(1, 1, 1, 64, 1 << 27, 1 << 20, 0.1)
    with pytest.raises(B.SfError):
        plan(big, [(1 << 30) + 1], [1])
    with pytest.raises(B.SfError):
        plan(_desc([8], d=96), [8], [1])
    with pytest.raises(ValueError):
        plan(_desc([8, 8]), [8], [1])


def test_plans_too_large_for_a_launch():
    lens = [1 << 30] * 2
    desc = B.make_desc(2, 8, 8, 64, 1 << 26, 1 << 27, 0.1)
    info = B.sf_weights_info()
    h, e = np.array(lens, np.int32), np.array([40, 40], np.int32)
    assert B.lib().sf_key_weights_plan(ctypes.byref(desc), h.ctypes.data, e.ctypes.data, None, None, None, None, 0,
                                       ctypes.byref(info)) == UNSUPPORTED
    one = np.array([1, 1], np.int32)          # a decode step over them is planned: a row per segment
    assert B.lib().sf_key_weights_plan(ctypes.byref(desc), h.ctypes.data, one.ctypes.data, None, None, None, None, 0,
                                       ctypes.byref(info)) == OK and info.steps == 2048
    ev = B.sf_evict_info()
    assert B.lib().sf_kv_evict_plan(ctypes.byref(desc), h.ctypes.data, h.ctypes.data, None, 0, 0, None, 0, ctypes.byref(ev)) == UNSUPPORTED
    many = np.ones(1 << 24, np.int32)
    desc = B.make_desc(1 << 24, 1, 1, 64, 1, 1 << 24, 0.1)
    assert B.lib().sf_kv_store_fp8_plan(ctypes.byref(desc), many.ctypes.data, many.ctypes.data, None, 0,
                                        ctypes.byref(B.sf_store_info())) == UNSUPPORTED


def test_capacity_is_reported_with_the_sizes():
    desc = _desc([400])
    for plan, args, info in ((B.sf_kv_store_fp8_plan, ([400], [400]), B.sf_store_info()),
                             (B.sf_key_weights_plan, ([400], [400]), B.sf_weights_info()),
                             (B.sf_kv_evict_plan, ([400], [200]), B.sf_evict_info())):
        with pytest.raises(B.SfError) as e:
            plan(desc, *args, work_host=np.zeros(4, np.int32))
        assert e.value.status == CAPACITY


def _call(fn, *args):
    return getattr(B.lib(), fn)(*args)


def _store_args(desc, info):
    return [ctypes.byref(desc), ctypes.byref(info), None, FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, FAKE, None]


def _weights_args(desc, info):
    return [ctypes.byref(desc), ctypes.byref(info), None, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, FAKE,
            info.workspace_bytes, None]


def _evict_args(desc, info):
    return [ctypes.byref(desc), ctypes.byref(info), None, FAKE, FAKE, FAKE, None, None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE,
            info.workspace_bytes, None]


def _extend_args(desc, info):
    return [ctypes.byref(desc), ctypes.byref(info), None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 0, FAKE, None]


CALLS = [
    # function, plan, its arguments, indexes that must not be NULL, that must be 16-byte aligned, that must be 4-byte aligned
    ("sf_kv_store_fp8", B.sf_kv_store_fp8_plan, ([400], [400]), _store_args, (3, 4, 5, 7, 8, 9, 10, 11), (3, 4, 5, 7, 8), (6, 9, 10, 11)),
    ("sf_key_weights", B.sf_key_weights_plan, ([400], [400]), _weights_args, (3, 4, 5, 6, 8, 9, 10, 12), (3, 4, 6, 9, 10, 11, 12), (5, 7, 8)),
    ("sf_kv_evict", B.sf_kv_evict_plan, ([400], [200]), _evict_args, (3, 4, 5, 8, 9, 10, 11, 12, 13), (3, 4, 5, 9, 10, 11, 12, 13), (8,)),
    ("sf_extend_attn_fp8", B.sf_extend_attn_plan, ([400], [400]), _extend_args, (3, 4, 5, 6, 7, 8, 9, 10), (3, 4, 5, 6, 10), (7, 8, 9, 12)),
]


@pytest.mark.parametrize("case", CALLS, ids=[c[0] for c in CALLS])
def test_calls_reject_bad_arguments(case):
    fn, plan, lens, args_of, needed, by16, by4 = case
    desc = _desc([400])
    info, _ = plan(desc, *lens)
    for at in needed:
        args = args_of(desc, info)
        args[at] = None
        assert _call(fn, *args) == INVALID, at
    for at in by16:
        args = args_of(desc, info)
        args[at] = FAKE + 8
        assert _call(fn, *args) == INVALID, at
    for at in by4:
        args = args_of(desc, info)
        args[at] = FAKE + 2
        assert _call(fn, *args) == INVALID, at
    args = args_of(desc, info)
    args[1] = None
    assert _call(fn, *args) == INVALID
    args = args_of(desc, info)
    args[0] = None
    assert _call(fn, *args) == INVALID
    other = _desc([400], d=64)
    args = args_of(other, info)
    assert _call(fn, *args) == MISMATCH
    args = args_of(desc, info)
    info.work_bytes += 32
    assert _call(fn, *args) == MISMATCH


def test_workspace_too_small():
    desc = _desc([400])
    info, _ = B.sf_key_weights_plan(desc, [400], [400])
    assert info.workspace_bytes > 0
    args = _weights_args(desc, info)
    args[13] -= 1
    assert _call("sf_key_weights", *args) == CAPACITY
    info, _ = B.sf_kv_evict_plan(desc, [400], [200])
    args = _evict_args(desc, info)
    args[14] -= 1
    assert _call("sf_kv_evict", *args) == CAPACITY
    args = _evict_args(desc, info)
    args[6] = FAKE                          # one scale array without the other
    assert _call("sf_kv_evict", *args) == INVALID
    info, _ = B.sf_extend_attn_plan(desc, [400], [400])
    args = _extend_args(desc, info)
    args[11] = 2
    assert _call("sf_extend_attn_fp8", *args) == INVALID


def test_nothing_to_do_needs_no_pointers():
    desc = B.make_desc(2, 28, 4, 128, 3, 0, 0.1)
    info, _ = B.sf_kv_store_fp8_plan(desc, [0, 0], [0, 0])
    assert _call("sf_kv_store_fp8", ctypes.byref(desc), ctypes.byref(info), *[None] * 11) == OK
    info, _ = B.sf_key_weights_plan(desc, [0, 0], [0, 0])
    assert _call("sf_key_weights", ctypes.byref(desc), ctypes.byref(info), *[None] * 11, 0, None) == OK
    info, _ = B.sf_kv_evict_plan(desc, [0, 0], [5, 0])
    assert _call("sf_kv_evict", ctypes.byref(desc), ctypes.byref(info), *[None] * 12, 0, None) == OK


def test_runner_calls_reject_without_a_device():
    desc = _desc([400])
    L = B.lib()
    assert L.sf_runner_store_fp8(None, ctypes.byref(desc), *[FAKE] * 11) == INVALID
    assert L.sf_runner_key_weights(None, ctypes.byref(desc), *[FAKE] * 13) == INVALID
    assert L.sf_runner_evict(None, ctypes.byref(desc), FAKE, FAKE, FAKE, 0, 0, *[FAKE] * 10) == INVALID
    m, info = B.sf_runner_memory(), B.sf_extend_info()
    assert L.sf_runner_extend_fp8(None, ctypes.byref(desc), *[FAKE] * 10, ctypes.byref(m), None, ctypes.byref(info), FAKE, FAKE,
                                  0) == INVALID


def test_truncate_returns_the_pages_behind():
    bt = np.full((3, 4), -1, np.int32)
    bt[0, :3], bt[1, :1], bt[2, :4] = [4, 0, 7], [2], [9, 1, 3, 8]
    table = B.PageTable(10, bt, [40, 5, 64])
    free = table.pool.available()
    table.truncate([16, 5, 17])
    assert table.pool.available() == free + 2 + 2
    assert table.bt.tolist() == [[4, -1, -1, -1], [2, -1, -1, -1], [9, 1, -1, -1]]
    assert table.pool.alloc(4).tolist() == [8, 3, 7, 0]          # the page returned last comes first
    assert table.prev.tolist() == [16, 5, 17]
    for keep in ([17, 5, 17], [-1, 5, 17]):
        with pytest.raises(B.SfError):
            table.truncate(keep)
    assert table.bt[0].tolist() == [4, -1, -1, -1]
    table.truncate([0, 0, 0])
    assert np.all(table.bt == -1)


def test_truncate_is_all_or_nothing():
    bt = np.array([[1, 2], [1, 3]], np.int32)                      # page 1 twice: cannot be returned twice
    pool = B.PagePool(4)
    pool.claim([1, 2, 3])
    lens, keep = np.array([32, 32], np.int32), np.zeros(2, np.int32)
    st = B.lib().sf_page_table_truncate(pool._p, bt.ctypes.data, 2, 2, lens.ctypes.data, keep.ctypes.data)
    assert st == INVALID and pool.available() == 1 and bt.tolist() == [[1, 2], [1, 3]]


# ---------------------------------------------------------------------------
# the oracle itself
# ---------------------------------------------------------------------------
def test_oracle_fresh_tile_is_the_quantizers():
    rng = np.random.default_rng(3)
    bits = (rng.standard_normal((16, 64)).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    for n in (1, 7, 16):
        new = np.arange(16) < n
        codes, scale = R.requantize(np.full((16, 64), 0x7F, np.uint8), np.float32(np.nan), np.zeros(16, bool),
                                    fp8_ref.widen_bf16(bits), new)
        want, want_scale = fp8_ref.quantize_tile(bits, n, slot_axis=0)
        assert scale == want_scale and np.array_equal(codes, want)


def test_oracle_growth_by_hand():
    # one held token of value 448 * 0.5 in slot 0, a new one of 3.3 times that in slot 1: two doublings
    codes = np.zeros((16, 64), np.uint8)
    codes[0, 0] = 0x7E            # 448
    codes[0, 1] = 0x01            # 2^-9, the smallest subnormal
    held, new = np.arange(16) == 0, np.arange(16) == 1
    x = np.zeros((16, 64), np.float32)
    x[1, 0] = 739.2
    out, scale = R.requantize(codes, np.float32(0.5), held, x, new)
    assert scale == 2.0
    assert fp8_ref.values()[out[0, 0]] == 112.0 and out[0, 1] == 0        # 2^-11 rounds to even: 0
    assert fp8_ref.values()[out[1, 0]] == 384.0                            # 369.6 lies between 352 and 384
    # equal to the tile's largest value: no growth
    x[1, 0] = 224.0
    out, scale = R.requantize(codes, np.float32(0.5), held, x, new)
    assert scale == 0.5 and out[1, 0] == 0x7E and out[0, 1] == 1
    # held codes of value zero only: as a fresh tile
    out, scale = R.requantize(np.full((16, 64), 0x80, np.uint8), np.float32(1.0), held, x, new)
    assert scale == np.float32(0.5) and out[1, 0] == 0x7E


def test_oracle_keeps_by_hand():
    w = np.array([1, 5, 5, np.nan, 0, 5, -1, np.inf], np.float32)
    pos = np.arange(8)
    assert np.nonzero(R.kept_slots(w, pos, 3, 0, 0, 8))[0].tolist() == [1, 2, 7]
    assert np.nonzero(R.kept_slots(w, pos, 7, 0, 0, 8))[0].tolist() == [0, 1, 2, 4, 5, 6, 7]
    assert np.nonzero(R.kept_slots(w, pos, 4, 1, 2, 8))[0].tolist() == [0, 1, 6, 7]
    dst, src = R.moves(R.kept_slots(w, pos, 4, 1, 2, 8), 4)
    assert dst.tolist() == [2, 3] and src.tolist() == [6, 7]


def test_oracle_weights_sum_to_the_rows():
    rng = np.random.default_rng(5)
    q, k, v = rng.standard_normal((4, 3, 8)), rng.standard_normal((9, 8)), rng.standard_normal((9, 8))
    out, lse, _, _ = R.attention(q, k, v, 0.3, 5)
    u, _ = R.key_weights(q, lse, k, 0.3, 5)
    assert np.isclose(u.sum(), 12.0)
    lse[1, 2] = -np.inf
    assert np.isclose(R.key_weights(q, lse, k, 0.3, 5)[0].sum(), 11.0)
