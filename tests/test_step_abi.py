"""A group rollout's step through the C ABI, on the CPU: frequencies, plans, shared pages and every host-side refusal."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import step_ref as R
from paper_2601_12784_amd import binding as B

FAKE = 0x10000   # aligned, never dereferenced
OK, INVALID, UNSUPPORTED, CAPACITY, MISMATCH = 0, 1, 2, 3, 4
TWO_PI = 2 * Fraction(314159265358979323846264338327950288419716939937510582097494, 10 ** 59)


def test_struct_sizes():
    for t, n in ((B.sf_shared_info, 48), (B.sf_rotary_desc, 16), (B.sf_rotary_scaling, 32), (B.sf_sample_desc, 24)):
        assert ctypes.sizeof(t) == n


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("turn,base", [(16, 10000.0), (64, 10000.0), (128, 1e6), (128, 0.5)])
@pytest.mark.parametrize("scaling", [None, (4.0, 0.0, 1.0, 4.0), (8.0, 4096.0, 1.0, 32.0), (0.5, 100.0, 0.0, 2.0)])
def test_frequencies(turn, base, scaling):
    got = B.sf_rotary_frequencies(turn, base, None if scaling is None else B.sf_rotary_scaling(*scaling))
    want = R.frequencies(turn, base) if scaling is None else R.frequencies(turn, base, *scaling)
    assert np.allclose(got, want, rtol=2 ** -50, atol=0)   # pow, and three roundings


def test_turns():
    """Nearest multiple of 2^-64 of a turn, whole turns left out, off by one unit at most below 2 pi."""
    freq = np.array([1.0, 0.5, 1e-9, 0.0, -0.25, 6.283185307179586, 100.0, 2.0 ** -80])
    got = B.sf_rotary_turns(freq)
    for f, t in zip(freq.tolist(), got.tolist()):
        exact = Fraction(f) / TWO_PI
        off = (Fraction(t) - exact * 2 ** 64) % 2 ** 64
        off = min(off, 2 ** 64 - off)
        assert off <= max(1, abs(f) / 4), (f, float(off))


@pytest.mark.parametrize("call", [
    lambda L, f: L.sf_rotary_frequencies(15, 10000.0, None, f),
    lambda L, f: L.sf_rotary_frequencies(0, 10000.0, None, f),
    lambda L, f: L.sf_rotary_frequencies(16, 0.0, None, f),
    lambda L, f: L.sf_rotary_frequencies(16, math.nan, None, f),
    lambda L, f: L.sf_rotary_frequencies(16, math.inf, None, f),
    lambda L, f: L.sf_rotary_frequencies(16, 10000.0, None, None),
    lambda L, f: L.sf_rotary_frequencies(16, 1e4, ctypes.byref(B.sf_rotary_scaling(0.0, 0.0, 1.0, 4.0)), f),
    lambda L, f: L.sf_rotary_frequencies(16, 1e4, ctypes.byref(B.sf_rotary_scaling(2.0, -1.0, 1.0, 4.0)), f),
    lambda L, f: L.sf_rotary_frequencies(16, 1e4, ctypes.byref(B.sf_rotary_scaling(2.0, 100.0, 4.0, 4.0)), f),
    lambda L, f: L.sf_rotary_turns(np.array([math.inf]).ctypes.data, 1, f),
    lambda L, f: L.sf_rotary_turns(np.array([math.nan]).ctypes.data, 1, f),
    lambda L, f: L.sf_rotary_turns(None, 1, f),
    lambda L, f: L.sf_rotary_turns(f, -1, f),
])
def test_frequency_refusals(call):
    assert call(B.lib(), np.zeros(64).ctypes.data) == INVALID


def _rotary(desc=(128, 128, 0, 1.0), tokens=4, hq=4, hkv=2, **change):
    a = dict(turns=FAKE, positions=FAKE, q=FAKE, qs=hq * 128, qo=FAKE + 4096, qos=hq * 128, k=FAKE, ks=hkv * 128, ko=FAKE + 4096,
             kos=hkv * 128)
    a.update(change)
    return B.lib().sf_rotary(None if desc is None else ctypes.byref(B.sf_rotary_desc(*desc)), tokens, hq, hkv, a["turns"],
                             a["positions"], a["q"], a["qs"], a["qo"], a["qos"], a["k"], a["ks"], a["ko"], a["kos"], None)


@pytest.mark.parametrize("want,change", [
    (INVALID, dict(desc=None)), (UNSUPPORTED, dict(desc=(96, 96, 0, 1.0))), (INVALID, dict(desc=(128, 0, 0, 1.0))),
    (INVALID, dict(desc=(64, 128, 0, 1.0))), (UNSUPPORTED, dict(desc=(128, 24, 0, 1.0))), (INVALID, dict(desc=(128, 64, 2, 1.0))),
    (INVALID, dict(desc=(128, 64, 0, math.nan))), (INVALID, dict(tokens=-1)), (INVALID, dict(hq=-1)), (INVALID, dict(hkv=-1)),
    (UNSUPPORTED, dict(tokens=(1 << 27) + 1)), (INVALID, dict(turns=None)), (INVALID, dict(turns=FAKE + 4)), (INVALID, dict(positions=None)),
    (INVALID, dict(positions=FAKE + 2)), (INVALID, dict(q=FAKE + 8)), (INVALID, dict(qo=None)), (INVALID, dict(qs=511)),
    (INVALID, dict(qs=516)), (INVALID, dict(qos=100)), (INVALID, dict(ko=None)), (INVALID, dict(ks=255)), (INVALID, dict(kos=0)),
    (INVALID, dict(k=FAKE + 2)), (INVALID, dict(q=FAKE, qo=FAKE, qs=1024, qos=512)), (INVALID, dict(k=FAKE, ko=FAKE, ks=512, kos=256)),
    (OK, dict(tokens=0)), (OK, dict(q=None, k=None)), (OK, dict(hq=0, hkv=0)),
])
def test_rotary_refusals(want, change):
    assert _rotary(**change) == want


def _desc(lens, hq=28, hkv=4, d=128, stride=None, pages=None):
    need = [-(-n // 16) for n in lens]
    return B.make_desc(len(lens), hq, hkv, d, stride or max(need, default=1) or 1, max(1, sum(need)) if pages is None else pages, 0.1)


@pytest.mark.parametrize("lens,news,first", [
    ([37, 5, 64], [37, 5, 64], None), ([90, 33, 17, 0, 48], [20, 1, 0, 0, 48], [1000, 32, 0, 0, 7]),
    ([17, 0, 32, 33], None, None), ([17, 0, 32, 33], None, [5, 9, 2 ** 31 - 2, 0]), ([20000, 16000], [20000, 16000], None), ([], [], None)])
def test_store_plan(lens, news, first):
    """Each new token is in exactly one row, with its query row and position; long lists go in runs of four pages."""
    desc = _desc(lens)
    info, work = B.sf_rotary_store_plan(desc, lens, news, first)
    rows = np.asarray(work)[: info.work_bytes // 4].reshape(-1, 8).tolist()
    e = [int(n > 0) for n in lens] if news is None else news
    assert info.num_q_rows == (len(lens) if news is None else sum(news)) and info.num_rows == len(rows)
    seen, at = {}, 0
    for s, pb, np_, lo, hi, qrow, pos, zero in rows:
        assert hi == lens[s] and lo == lens[s] - e[s] and zero == 0 and 1 <= np_ <= 4
        for t in range(max(lo, pb * 16), min(hi, (pb + np_) * 16)):
            assert (s, t) not in seen
            seen[s, t] = (qrow + t - lo, pos + t - lo)
    for s, n in enumerate(lens):
        for j in range(e[s]):
            p0 = n - e[s] if first is None else first[s]
            assert seen.pop((s, n - e[s] + j)) == ((s if news is None else at) + (0 if news is None else j), p0 + j)
        at += e[s]
    assert not seen


@pytest.mark.parametrize("want,lens,news,first,kw", [
    (INVALID, [5], [6], None, {}), (INVALID, [-1], [0], None, {}), (INVALID, [5], [-1], None, {}), (INVALID, [40], [1], None, dict(stride=2)),
    (INVALID, [5], [1], None, dict(pages=0)), (INVALID, [5], [2], [-1], {}), (INVALID, [5], [2], [2 ** 31 - 2], {}),
    (INVALID, [5], None, [-5], {}), (UNSUPPORTED, [5], [2], None, dict(d=96)), (OK, [0], None, None, dict(pages=0))])
def test_store_plan_refusals(want, lens, news, first, kw):
    a = [None if x is None else np.array(x, np.int32) for x in (lens, news, first)]
    info = B.sf_store_info()
    desc = _desc([max(n, 0) for n in lens], **kw)
    st = B.lib().sf_rotary_store_plan(ctypes.byref(desc), *[None if x is None else x.ctypes.data for x in a], None, 0, ctypes.byref(info))
    assert st == want


def test_store_plan_capacity():
    desc, lens = _desc([100]), np.array([100], np.int32)
    info, work = B.sf_store_info(), np.empty(8, np.int32)
    assert B.lib().sf_rotary_store_plan(ctypes.byref(desc), lens.ctypes.data, lens.ctypes.data, None, work.ctypes.data, 32,
                                        ctypes.byref(info)) == CAPACITY
    assert info.work_bytes == 7 * 32


def _store(want, desc=None, rope=(128, 64, 0, 1.0), info=None, **change):
    lens = [20, 5]
    desc = desc or _desc(lens)
    if info is None:
        info, _ = B.sf_rotary_store_plan(desc, lens, [3, 5])
    a = dict(work=FAKE, turns=FAKE, q=FAKE, qs=28 * 128, qo=FAKE, qos=28 * 128, k=FAKE, ks=512, v=FAKE, vs=512, pages=FAKE, kp=FAKE,
             vp=FAKE, bt=FAKE)
    a.update(change)
    r = None if rope is None else ctypes.byref(B.sf_rotary_desc(*rope))
    st = B.lib().sf_rotary_store(ctypes.byref(desc), r, ctypes.byref(info), None, a["work"], a["turns"], a["q"], a["qs"], a["qo"], a["qos"],
                                 a["k"], a["ks"], a["v"], a["vs"], a["pages"], a["kp"], a["vp"], a["bt"], None)
    assert st == want


@pytest.mark.parametrize("change", [
    dict(work=None), dict(work=FAKE + 8), dict(turns=None), dict(turns=FAKE + 4), dict(kp=None), dict(vp=None), dict(kp=FAKE + 8),
    dict(bt=None), dict(bt=FAKE + 2), dict(pages=FAKE + 1), dict(k=None), dict(k=FAKE + 4), dict(ks=504), dict(ks=516), dict(v=None),
    dict(vs=511), dict(qo=None), dict(qs=100), dict(qos=28 * 128 + 8), dict(q=FAKE + 2), dict(rope=(64, 64, 0, 1.0)), dict(rope=(128, 8, 0, 1.0))])
def test_store_refusals(change):
    _store(INVALID, **change)


def test_store_takes_its_own_plan_only():
    desc, lens = _desc([20, 5]), [20, 5]
    _store(MISMATCH, desc, info=B.sf_kv_store_fp8_plan(desc, lens, [3, 5])[0])
    _store(MISMATCH, _desc([20, 21]), info=B.sf_rotary_store_plan(desc, lens, [3, 5])[0])
    info, _ = B.sf_rotary_store_plan(desc, lens, [3, 5])
    info.work_bytes += 32
    _store(MISMATCH, desc, info=info)
    assert B.lib().sf_kv_store_fp8(ctypes.byref(desc), ctypes.byref(B.sf_rotary_store_plan(desc, lens, [3, 5])[0]), None, *[FAKE] * 10) == MISMATCH


def test_rotary_class():
    r = B.Rotary(64, rotary_dim=32, base=500.0, scaling=dict(factor=4.0, original=4096.0, low=1.0, high=32.0, magnitude=1.25))
    assert np.allclose(r.freq, R.frequencies(32, 500.0, 4.0, 4096.0, 1.0, 32.0), rtol=2 ** -50)
    assert r.desc.magnitude == 1.25 and r.desc.rotary_dim == 32 and not r.desc.interleaved
    assert np.allclose(B.Rotary(64, scaling=dict(factor=2.0)).freq, R.frequencies(64, 10000.0) / 2)
    assert np.array_equal(B.Rotary(64, rotary_dim=16, freq=np.arange(8.0)).freq, np.arange(8.0))
    for bad in (dict(layout="other"), dict(rotary_dim=16, freq=np.zeros(7)), dict(scaling=dict(factor=2.0, depth=1.0)),
                dict(scaling=dict(magnitude=2.0, original=4096.0, low=1.0))):
        with pytest.raises((ValueError, KeyError)):
            B.Rotary(64, **bad)
    for bad in (dict(rotary_dim=128), dict(rotary_dim=24), dict(rotary_dim=0, freq=np.zeros(0)), dict(scaling=dict(factor=-2.0)),
                dict(scaling=dict(magnitude=math.inf))):
        with pytest.raises(B.SfError):
            B.Rotary(64, **bad)
    with pytest.raises(B.SfError):
        B.Rotary(96)


# ---------------------------------------------------------------------------
# attention over shared prompts: the plan
# ---------------------------------------------------------------------------
def _shared_rows(info, work):
    w = np.asarray(work)[: info.work_bytes // 4].tolist()
    at = 16 * info.num_workers
    table = [w[16 * i: 16 * i + 16] for i in range(info.num_workers)]
    items = [w[at + 16 * i: at + 16 * i + 16] for i in range(info.num_work)]
    at += 16 * info.num_work
    return table, items, [w[at + 8 * i: at + 8 * i + 8] for i in range(info.num_merge)]


def _groups(rng):
    lens, offsets, shared = [], [0], []
    for _ in range(rng.integers(1, 7)):
        n = int(rng.choice([0, 1, 2, 5, 16, 40]))
        common = int(rng.choice([0, 5, 16, 17, 250, 1600]))
        lens += [0 if rng.random() < 0.15 else common + int(rng.integers(0 if common else 1, 200)) for _ in range(n)]
        offsets.append(len(lens))
        shared.append(common)
    return lens, offsets, shared


@pytest.mark.parametrize("seed", range(40))
def test_shared_plan_covers_everything_once(seed):
    """Every (sequence, head row, page) is in one segment; its partial rows are its own, and the merge rows find them."""
    rng = np.random.default_rng(seed)
    lens, offsets, shared = _groups(rng)
    hq, hkv = [(28, 4), (4, 1), (16, 1), (8, 8)][seed % 4]
    g = hq // hkv
    opts = B.make_opts(num_cus=int(rng.choice([1, 3, 256])), min_chunk_pages=int(rng.choice([0, 1, 50])))
    desc = _desc(lens, hq, hkv)
    info, work = B.sf_shared_attn_plan(desc, lens, offsets, shared, opts, fp8=bool(seed % 3))
    table, items, merges = _shared_rows(info, work)
    assert [r[0] for r in table] == np.cumsum([0] + [r[1] for r in table])[:-1].tolist() and sum(r[1] for r in table) == len(items)
    for r in table:
        if r[1]:
            assert r[2:] == items[r[0]][2:]
    if info.workers_per_group == 8:     # a workgroup that walks a prompt together does the same in all waves
        for i in range(0, len(table), 8):
            walks = [[it[2:8] + [it[11]] for it in items[r[0]: r[0] + r[1]]] for r in table[i: i + 8]]
            if any(it[-1] for w in walks for it in w):
                assert all(w == walks[0] for w in walks) and all(it[-1] in (2, 4, 8) for it in walks[0])
    else:
        assert info.workers_per_group == 1 and not any(it[11] for it in items)
    source = {}
    for i in range(len(shared)):
        live = [s for s in range(offsets[i], offsets[i + 1]) if lens[s] > 0]
        if len(live) > 1 and shared[i] >= 16:
            source.update({s: (live[0], shared[i] // 16) for s in live})
    seen, parts, used = set(), {}, set()
    for _, _, seq0, src, kvh, pb, pe, end, slot, row0, rows, together, split, *_ in items:
        pages = [p for p in range(pb, pe) if not together or (p - pb) // 2 % (8 // together) == split]
        assert 0 <= pb < pe and 1 <= rows <= 32 and row0 % 16 == 0
        for r in range(rows):
            s, h = seq0 + (row0 + r) // g, (row0 + r) % g
            if slot >= 0:
                assert slot + r not in used and slot + r < info.num_rows
                used.add(slot + r)
                parts.setdefault((s, kvh, h), []).append(slot + r)
            else:
                assert src == s and (pb, pe) == (0, -(-lens[s] // 16))
            for p in pages:
                assert (s, kvh, h, p) not in seen
                seen.add((s, kvh, h, p))
            if lens[s] == 0:
                continue    # a sequence without tokens between its group's members
            common = source.get(s, (s, 0))
            assert src == (common[0] if pb < common[1] else s) and (pe <= common[1] or pb >= common[1])
            assert end == (common[1] * 16 if pb < common[1] else lens[s])
    for s, n in enumerate(lens):
        want = {(s, k, h, p) for k in range(hkv) for h in range(g) for p in range(-(-n // 16))} if n else set()
        assert n == 0 or want <= seen
    merged = {(m[0], m[1]): m for m in merges}
    assert len(merged) == len(merges)
    for s, n in enumerate(lens):
        for k in range(hkv):
            m = merged.get((s, k))
            if m is None:
                assert (s, k, 0) not in parts and n > 0
                continue
            _, _, own, own_n, pre, pre_n, stride, _ = m
            for h in range(g):
                rows = [pre + c * stride + h for c in range(pre_n)] + [own + c * g + h for c in range(own_n)]
                assert sorted(rows) == sorted(parts.get((s, k, h), [])) if n else rows == []
    assert info.workspace_bytes == (0 if not info.num_rows else -(-info.num_rows * 512 // 256) * 256 + info.num_rows * 4)


def test_shared_plan_uses_the_whole_gpu():
    """A prompt's blocks of rows and the members' own pages take all waves and hardly one too many."""
    for members, common, own in ((16, 2048, 2000), (64, 32760, 300), (256, 4000, 1000), (2, 100000, 1)):
        lens = [common + own] * members
        info, work = B.sf_shared_attn_plan(_desc(lens), lens, [0, members], [common])
        busy = sum(r[1] > 0 for r in _shared_rows(info, work)[0])
        assert 1800 <= busy <= 2048 and info.num_workers <= 2064, (members, busy, info.num_workers)


@pytest.mark.parametrize("want,lens,offsets,shared", [
    (INVALID, [20, 20], [0, 1], [16]), (INVALID, [20, 20], [1, 2], [16]), (INVALID, [20, 20], [0, 3], [16]), (INVALID, [20, 20], [0, 2], [-1]),
    (INVALID, [20, 20, 20], [0, 2, 1, 3], [16, 0, 16]), (INVALID, [20, 15], [0, 2], [16]), (INVALID, [20, -1], [0, 2], [16]),
    (OK, [20, 0], [0, 2], [16]), (OK, [0, 0], [0, 2], [100]), (OK, [20, 16], [0, 2], [16]), (OK, [], [0], [])])
def test_shared_plan_refusals(want, lens, offsets, shared):
    a = [np.array(x, np.int32) for x in (lens, offsets, shared)]
    desc, info = _desc([max(n, 0) for n in lens]), B.sf_shared_info()
    st = B.lib().sf_shared_attn_plan(ctypes.byref(desc), a[0].ctypes.data, len(shared), a[1].ctypes.data, a[2].ctypes.data, 0, None, None, 0,
                                     ctypes.byref(info))
    assert st == want


def test_shared_plan_more_refusals():
    L, info = B.lib(), B.sf_shared_info()
    lens, off, sh = (np.array(x, np.int32) for x in ([40, 40], [0, 2], [32]))
    desc = _desc([40, 40])

    def call(desc=desc, lens=lens.ctypes.data, n=1, off=off.ctypes.data, sh=sh.ctypes.data, fp8=0, opts=None, work=None, cap=0, info=info):
        return L.sf_shared_attn_plan(None if desc is None else ctypes.byref(desc), lens, n, off, sh, fp8, None if opts is None else ctypes.byref(opts),
                                     work, cap, None if info is None else ctypes.byref(info))

    assert call() == OK
    for bad in (dict(desc=None), dict(lens=None), dict(n=-1), dict(n=0), dict(off=None), dict(sh=None), dict(info=None), dict(fp8=2),
                dict(opts=B.make_opts(num_cus=-1)), dict(opts=B.make_opts(min_chunk_pages=-1)), dict(desc=_desc([40, 40], stride=2)),
                dict(desc=_desc([40, 40], pages=0))):
        assert call(**bad) == INVALID, bad
    assert call(desc=_desc([40, 40], d=96)) == UNSUPPORTED
    work = np.empty(info.work_bytes // 4, np.int32)
    assert call(work=work.ctypes.data, cap=info.work_bytes - 4) == CAPACITY
    assert call(work=work.ctypes.data, cap=info.work_bytes) == OK


def _shared(want, info=None, **change):
    desc = _desc([40, 40])
    if info is None:
        info, _ = B.sf_shared_attn_plan(desc, [40, 40], [0, 2], [32])
    a = dict(work=FAKE, q=FAKE, k=FAKE, v=FAKE, ks=None, vs=None, bt=FAKE, out=FAKE, bf16=0, lse=FAKE, ws=FAKE, n=info.workspace_bytes)
    a.update(change)
    assert B.lib().sf_shared_attn(ctypes.byref(desc), ctypes.byref(info), None, a["work"], a["q"], a["k"], a["v"], a["ks"], a["vs"], a["bt"],
                                  a["out"], a["bf16"], a["lse"], a["ws"], a["n"], None) == want


def test_shared_refusals():
    for bad in (dict(work=None), dict(work=FAKE + 4), dict(q=None), dict(q=FAKE + 8), dict(k=None), dict(v=FAKE + 2), dict(bt=None), dict(bt=FAKE + 1),
                dict(out=None), dict(out=FAKE + 8), dict(lse=FAKE + 2), dict(ks=FAKE), dict(vs=FAKE), dict(ks=FAKE + 2, vs=FAKE), dict(bf16=2),
                dict(ws=FAKE + 8)):
        _shared(INVALID, **bad)
    _shared(CAPACITY, n=0)
    _shared(CAPACITY, ws=None)
    desc = _desc([40, 40])
    _shared(MISMATCH, B.sf_shared_attn_plan(_desc([40, 400]), [40, 400], [0, 2], [32])[0], n=1 << 30)
    for name in ("num_work", "num_merge", "num_rows", "workers_per_group"):
        info, _ = B.sf_shared_attn_plan(desc, [40, 40], [0, 2], [32])
        setattr(info, name, getattr(info, name) + 1)
        _shared(MISMATCH, info, n=1 << 30)


# ---------------------------------------------------------------------------
# pages with several holders
# ---------------------------------------------------------------------------
def test_shared_pages_are_free_when_the_last_holder_is_gone():
    pool = B.PagePool(8)
    pool.claim([5, 2])
    pool.share([5, 5, 2])
    assert pool.available() == 6
    pool.release([5, 2, 5])
    assert pool.available() == 6
    for bad in ([5, 5], [2, 2], [7], [8], [-1]):
        with pytest.raises(B.SfError):
            pool.release(bad)
        assert pool.available() == 6
    pool.release([5])
    assert pool.available() == 7 and pool.alloc(1).tolist() == [5]
    for bad in ([0], [8], [-1], [2, 0]):
        with pytest.raises(B.SfError):
            pool.share(bad)
    with pytest.raises(B.SfError):
        pool.claim([5])
    pool.release([2, 5])
    assert pool.available() == 8


def _table():
    bt = np.full((4, 6), -1, np.int32)
    bt[0, :3], bt[1, :4], bt[2, :3], bt[3, :1] = [7, 1, 4], [7, 1, 9, 8], [7, 1, 6], [3]
    return bt


def test_page_table_of_groups():
    t = B.PageTable(12, _table(), [40, 50, 36, 5], ([0, 3, 4], [35, 0]))
    assert t.pool.available() == 12 - 7
    t.advance([41, 51, 0, 6])          # 6 is free, 7 and 1 are not
    assert t.pool.available() == 6
    t.advance([0, 0, 0, 7])            # both of the others leave at once
    assert t.pool.available() == 11
    t.advance([0, 0, 0, 0])
    assert t.pool.available() == 12


def test_page_table_needs_pages_that_come_free_in_the_same_step():
    bt = np.array([[0, 1], [0, 2]], np.int32)
    t = B.PageTable(3, bt, [32, 32], ([0, 2], [16]))
    with pytest.raises(B.SfError):
        t.advance([33, 33])
    assert t.pool.available() == 0
    bt = np.array([[0, 1, -1], [0, 2, -1]], np.int32)
    t = B.PageTable(3, bt, [32, 32], ([0, 2], [16]))
    assert t.advance([33, 0]).tolist() == [2, -1]     # the other's own page; the shared one stays


def test_page_table_group_refusals():
    for lens, groups in (([40, 50, 36, 5], ([0, 3], [35])), ([40, 50, 36, 5], ([0, 3, 4], [34, 16])), ([40, 50, 36, 5], ([0, 3, 4], [48, 0])),
                         ([40, 50, 36, 5], ([0, 3, 2, 4], [16, 0, 0])), ([40, 50, 36, 5], ([1, 3, 4], [16, 0])), ([40, 50, 36, 5], ([0, 4], [-1]))):
        with pytest.raises(ValueError):
            B.PageTable(12, _table(), lens, groups)
    bt = _table()
    bt[2, 1] = 11
    with pytest.raises(ValueError):
        B.PageTable(12, bt, [40, 50, 36, 5], ([0, 3, 4], [32, 0]))
    with pytest.raises(B.SfError):     # pages in two rows of a table without groups
        B.PageTable(12, _table(), [40, 50, 36, 5])


# ---------------------------------------------------------------------------
# sampling
# ---------------------------------------------------------------------------
def _sample(desc=(4, 1000, 1000, 0, 0), **change):
    d, need = B.sf_sample_desc(*desc), ctypes.c_uint64()
    st = B.lib().sf_sample_workspace(ctypes.byref(d), ctypes.byref(need))
    if st:
        return st
    a = dict(logits=FAKE, t=FAKE, k=FAKE, p=FAKE, m=FAKE, u=FAKE, token=FAKE, logprob=FAKE, kept=FAKE, ws=FAKE, n=need.value)
    a.update(change)
    return B.lib().sf_sample(ctypes.byref(d), *[a[x] for x in ("logits", "t", "k", "p", "m", "u", "token", "logprob", "kept", "ws", "n")], None)


@pytest.mark.parametrize("want,change", [
    (INVALID, dict(desc=(-1, 10, 10, 0, 0))), (INVALID, dict(desc=(1, 0, 10, 0, 0))), (INVALID, dict(desc=(1, 10, 9, 0, 0))),
    (INVALID, dict(desc=(1, 10, 10, 0, 1))), (UNSUPPORTED, dict(desc=(1, 10, 10, 3, 0))), (UNSUPPORTED, dict(desc=(1, 10, 10, -1, 0))),
    (UNSUPPORTED, dict(desc=(1, (1 << 19) + 1, 1 << 20, 0, 0))), (UNSUPPORTED, dict(desc=(1 << 22, 1, 1, 0, 0))),
    (UNSUPPORTED, dict(desc=(1 << 20, 1 << 19, 1 << 19, 1, 0))), (OK, dict(desc=(0, 10, 10, 0, 0))),
    (INVALID, dict(logits=None)), (INVALID, dict(logits=FAKE + 2)), (INVALID, dict(u=None)), (INVALID, dict(token=None)),
    (INVALID, dict(t=FAKE + 1)), (INVALID, dict(k=FAKE + 2)), (INVALID, dict(p=FAKE + 2)), (INVALID, dict(m=FAKE + 3)), (INVALID, dict(u=FAKE + 2)),
    (INVALID, dict(token=FAKE + 2)), (INVALID, dict(logprob=FAKE + 2)), (INVALID, dict(kept=FAKE + 2)), (INVALID, dict(ws=None)),
    (INVALID, dict(ws=FAKE + 8)), (CAPACITY, dict(n=0)), (INVALID, dict(desc=(4, 1000, 1000, 1, 0), logits=FAKE + 1))])
def test_sample_refusals(want, change):
    assert _sample(**change) == want


def test_sample_workspace_needs_a_place():
    assert B.lib().sf_sample_workspace(ctypes.byref(B.sf_sample_desc(1, 10, 10, 0, 0)), None) == INVALID
    assert B.lib().sf_sample_workspace(None, ctypes.byref(ctypes.c_uint64())) == INVALID


# ---------------------------------------------------------------------------
# the binding's own checks (tensors that say they are on the GPU; nothing is launched)
# ---------------------------------------------------------------------------
class OnGpu(torch.Tensor):
    is_cuda = True


def gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


@pytest.mark.parametrize("make", [
    lambda: torch.zeros(4, 2, 64, dtype=torch.bfloat16), lambda: gpu(4, 2, 64, dtype=torch.float16), lambda: gpu(3, 2, 64), lambda: gpu(4, 2, 32),
    lambda: gpu(4, 64, 2).transpose(1, 2), lambda: gpu(4, 3, 64)[:, ::2], lambda: gpu(1, 2, 64).expand(4, 2, 64), lambda: None,
    lambda: gpu(4, 2, 128)[..., ::2]])
def test_token_rows_are_checked(make):
    with pytest.raises((ValueError, TypeError)):
        B._rows(make(), "q", (4, 2, 64))


def test_token_rows_may_lie_apart():
    x = gpu(4, 8 * 64)
    assert B._rows(x[:, 64:192].view(4, 2, 64), "k", (4, 2, 64)) == 512
    assert B._rows(gpu(4, 2, 64), "k", (4, 2, 64)) == 128
    assert B._rows(gpu(9, 2, 64)[:1], "k", (1, 2, 64)) == 128


def test_outputs_that_overlap_inputs_are_refused():
    x = gpu(6, 8 * 64)
    q, k, v = x[:, :256].view(6, 4, 64), x[:, 256:384].view(6, 2, 64), x[:, 384:].view(6, 2, 64)
    B._check_turned(q, q, "q_out", [q, k, v])            # in place, beside the others
    B._check_turned(q, gpu(6, 4, 64), "q_out", [q, k, v])
    with pytest.raises(ValueError):
        B._check_turned(q, x[:, 64:320].view(6, 4, 64), "q_out", [q, k, v])
    y = gpu(7, 4, 64)
    with pytest.raises(ValueError):
        B._check_turned(y[:6], y[1:], "q_out", [y[:6]])


def test_outputs_in_place_of_what_is_read_twice_are_refused():
    """One tensor as queries and keys (or values): turned in place, one part of the call would read what another has written."""
    x, y, at = gpu(6, 4, 64), gpu(6, 4, 64), gpu(6, dtype=torch.int32)
    B._check_turned(x, y, "q_out", [x, x])
    with pytest.raises(ValueError):
        B._check_turned(x, x, "q_out", [x, x])
    rotary = B.Rotary(64)
    for kw in (dict(q_out=x), dict(q_out=y, k_out=x), dict(q_out=x, k_out=y)):
        with pytest.raises(ValueError, match="overlaps an input"):
            rotary(x, x, at, **kw)
    attn = B.DecodeAttention(4, 4, 64, num_cus=256)
    k_pool, v_pool = gpu(6, 4, 8, 16, 8), gpu(6, 4, 64, 16)
    for k_new, v_new in ((x, y), (y, x), (x, x)):
        with pytest.raises(ValueError, match="overlaps an input"):
            attn.rotate_store(None, x, k_new, v_new, k_pool, v_pool, gpu(6, 1, dtype=torch.int32), [1] * 6, q_out=x)


def test_outputs_that_overlap_each_other_are_refused():
    q, k, at, wide = gpu(6, 4, 64), gpu(6, 4, 64), gpu(6, dtype=torch.int32), gpu(6, 8 * 64)
    rotary, out = B.Rotary(64), gpu(6, 4, 64)
    for a, b in ((out, out), (wide[:, :256].view(6, 4, 64), wide[:, 192:448].view(6, 4, 64)), (out, out.view(6, 4, 64))):
        with pytest.raises(ValueError, match="k_out overlaps q_out"):
            rotary(q, k, at, q_out=a, k_out=b)
    assert not B._overlap(wide[:, :256].view(6, 4, 64), wide[:, 256:].view(6, 4, 64))


# ---------------------------------------------------------------------------
# SF_DEBUG_CHECKS: the block-table entries that a call reads
# ---------------------------------------------------------------------------
def _refused(check, *args):
    try:
        check(*args)
    except (ValueError, B.SfError):
        return True
    return False


def test_debug_check_of_shared_pages():
    lens, offsets, shared = np.array([70, 0, 50, 49, 20], np.int32), np.array([0, 4, 5], np.int32), np.array([48, 16], np.int32)
    good = np.array([[5, 6, 7, 8, 9], [-1] * 5, [5, 6, 7, 3, -1], [5, 6, 7, 2, -1], [1, 0, -1, -1, -1]], np.int32)
    desc = B.make_desc(5, 4, 1, 64, 5, 10, 0.1)
    B._check_group_pages(desc, good, lens, offsets, shared)
    kept = good.copy()
    B._check_group_pages(desc, torch.from_numpy(good), lens, offsets, shared)
    assert np.array_equal(good, kept)
    for row, col, value, bad in ((2, 1, -1, False), (2, 0, -(1 << 30), False), (3, 2, 10, False),      # not read, and no page
                                 (2, 1, 4, True), (3, 0, 6, True),                                      # another page than the group's
                                 (0, 1, -1, True), (0, 2, 10, True), (2, 3, -1, True), (3, 3, 10, True), (4, 1, -5, True), (1, 0, 99, False)):
        table = good.copy()
        table[row, col] = value
        assert _refused(B._check_group_pages, desc, table, lens, offsets, shared) == bad, (row, col, value)
    # what the call refuses by itself does not get in the way
    B._check_group_pages(desc, good, lens, np.array([0, 99, 5], np.int32)[[0, 2, 2]], np.array([-4, 16], np.int32))


def test_debug_check_of_stored_pages():
    """A store reads the entries of its new tokens' pages, less those it writes: the others may hold anything."""
    lens, news = np.array([70, 0, 33, 40], np.int32), np.array([3, 0, 1, 20], np.int32)
    table = np.full((4, 5), -(1 << 30), np.int32)
    table[0, 4], table[2, 2], table[3, 1:3] = 8, 7, (5, 6)
    desc = B.make_desc(4, 4, 1, 64, 5, 10, 0.1)
    B._check_stored_pages(desc, table, lens, news, None)
    for row, col in ((0, 4), (2, 2), (3, 1), (3, 2)):
        for value in (-1, 10):
            bad = table.copy()
            bad[row, col] = value
            assert _refused(B._check_stored_pages, desc, bad, lens, news, None)
            named = np.full(4, -1, np.int32)
            named[row] = 9
            assert _refused(B._check_stored_pages, desc, bad, lens, news, named) == (col == 1)     # its last page is named
    for value in (-2, 10):
        assert _refused(B._check_stored_pages, desc, table, lens, news, np.array([-1, -1, value, -1], np.int32))


def test_a_refused_step_of_a_group_loop_moves_nothing():
    """The page table goes on only with a step that is taken."""
    bt = np.array([[3, 1], [3, 2]], np.int32)
    pools = gpu(6, 2, 8, 16, 8), gpu(6, 2, 64, 16)
    loop = B.DecodeLoopRunner(4, 2, 64, *pools, gpu(2, 2, dtype=torch.int32), bt, [17, 17], 0.1, num_cus=256, groups=([0, 2], [16]))
    loop.steps = 1       # (the first one attends alone)
    free, before = loop.pool.available(), loop.bt_host.copy()
    for kw in (dict(attn_events=(1, 2)), dict(k_new=None), dict(lens=[15, 18])):
        a = dict(q=gpu(2, 4, 64), lens=[18, 0], k_new=gpu(2, 2, 64), v_new=gpu(2, 2, 64))
        a.update(kw)
        with pytest.raises(ValueError):
            loop.step(**a)
        assert loop.pool.available() == free and loop.table.prev.tolist() == [17, 17] and np.array_equal(loop.bt_host, before)


def test_no_new_token_goes_into_a_page_that_others_hold():
    """After a cut into the shared tokens, or where a begun page is shared, the next token would change the others' keys."""
    t = B.PageTable(12, _table(), [40, 50, 36, 5], ([0, 3, 4], [35, 0]))
    t.truncate([20, 50, 36, 5])        # the first member's cache ends inside a page of all three
    free, before = t.pool.available(), t.bt.copy()
    for lens in ([21, 51, 37, 6], [21, 51, 0, 6]):
        with pytest.raises(B.SfError):
            t.advance(lens)
        assert t.pool.available() == free and np.array_equal(t.bt, before) and t.prev.tolist() == [20, 50, 36, 5]
    assert t.advance([20, 50, 36, 5], appending=False).tolist() == [-1] * 4      # it may be read
    t.advance([21, 0, 0, 6])           # the others leave: the page is its own
    t.advance([22, 0, 0, 0])
    assert t.pool.available() == 12 - 2
    # a page of several holders that is begun
    pool, bt = B.PagePool(4), np.array([[2], [2]], np.int32)
    pool.claim([2])
    pool.share([2])
    lens, new = np.array([5, 5], np.int32), np.zeros(2, np.int32)
    step = lambda to: B.lib().sf_page_table_step(pool._p, bt.ctypes.data, 1, 2, lens.ctypes.data,  # noqa: E731
                                                 np.array(to, np.int32).ctypes.data, 1, new.ctypes.data)
    assert step([6, 6]) == INVALID and step([6, 0]) == OK and pool.available() == 3
