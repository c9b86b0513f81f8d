"""GPU parity of a group rollout's step against oracle/step_ref.py in 64 bits: rotary positions, attention over shared
prompts, sampling, each alone and all in one loop.

Tolerances, u = 2^-24 (half a step of fp32), half a step of bf16 2^-8:
  rotation: the angle less whole quarter turns enters fp32 (u of at most pi/4), the series end below 2.5e-8 < u, their
    evaluation and the magnitude cost 4 u, two products and a sum 3 u: 2^-21 (|a| + |b|) magnitude with room for all,
    then half a step of bf16.
  attention: as tests/test_gpu_cache.py: a score is off by (D + 8) u Z, Z the largest sum of |q k| scale of the row, a
    weight by twice that relatively (its own and the sum's), 2^-22 of exp2, 2^-16 as two bf16 parts; sums of n terms in
    fp32 by n u; a joined result by the log-sum-exps' 2^-22 |lse| once more. Of sum of p |v|.
  sampling: tokens are equal, or ones to whose share of the sum the draw is nearer than V 2^-43 of everything; logprob
    and kept are rounded once, with sums off by V 2^-44.
"""
import math

import numpy as np
import pytest
import torch

from oracle import cache_ref, step_ref as R
from paper_2601_12784_amd import binding as B
from tests.test_gpu_cache import Cache, bits, wide

pytestmark = pytest.mark.gpu
PAGE = 16
U = 2.0 ** -24
BF16 = torch.finfo(torch.bfloat16).eps / 2


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()
    yield
    torch.cuda.synchronize()


def randn(rng, *shape, mult=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * mult).astype(np.float32)).to(torch.bfloat16).cuda()


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
def check_turned(got, x, positions, rotary, what):
    """got, x: bf16 [T, H, D]."""
    got, x = wide(got), wide(x)
    for t, p in enumerate(np.asarray(positions).tolist()):
        want, size = R.rotate(x[t], p, rotary.freq, rotary.desc.interleaved, rotary.desc.magnitude)
        off = np.abs(got[t] - want) - (2.0 ** -21 * size + BF16 * np.abs(want))
        assert off.max(initial=-1) <= 0, f"{what}: token {t} at {p} is {off.max()} beyond"


LAYOUTS = [(64, 64, "half"), (64, 16, "interleaved"), (64, 48, "half"), (128, 128, "interleaved"), (128, 128, "half"), (128, 32, "half"),
           (128, 112, "interleaved")]


@pytest.mark.parametrize("d,turn,layout", LAYOUTS)
@pytest.mark.parametrize("t", [1, 2, 7, 33])
@pytest.mark.parametrize("packed", [False, True])
def test_rotary(d, turn, layout, t, packed):
    rng = np.random.default_rng(d + turn + t)
    hq, hkv = (7, 3) if t < 33 else (40, 8)
    rotary = B.Rotary(d, rotary_dim=turn, layout=layout, base=1e6, scaling=dict(factor=4.0, original=4096.0, low=1.0, high=32.0, magnitude=1.1386))
    positions = rng.integers(0, 1 << 31, t)
    positions[: min(t, 5)] = [0, 2 ** 31 - 1, 131071, 1, 4096][: min(t, 5)]
    x = randn(rng, t, (hq + 2 * hkv) * d)
    if packed:
        q, k = x[:, : hq * d].view(t, hq, d), x[:, hq * d: (hq + hkv) * d].view(t, hkv, d)
    else:
        q, k = randn(rng, t, hq, d), randn(rng, t, hkv, d)
    q0, k0, x0 = q.clone(), k.clone(), x.clone()
    at = torch.from_numpy(positions.astype(np.int32)).cuda()
    q1, k1 = rotary(q, k, at)
    assert torch.equal(q, q0) and torch.equal(k, k0)
    check_turned(q1, q0, positions, rotary, "q")
    check_turned(k1, k0, positions, rotary, "k")
    # in place, one of the two alone, into wider rows
    only_q = rotary(q0, None, at)[0]
    only_k = rotary(None, k0, at)[1]
    assert torch.equal(only_q, q1) and torch.equal(only_k, k1)
    wider = torch.full((t, (hq + 1) * d), 7.0, dtype=torch.bfloat16, device="cuda")
    rotary(q, None, at, q_out=wider[:, d:].view(t, hq, d))
    assert torch.equal(wider[:, d:].view(t, hq, d), q1) and (wider[:, :d] == 7).all()
    rotary(q, k, at, q_out=q, k_out=k)
    assert torch.equal(q, q1) and torch.equal(k, k1)
    if packed:
        assert torch.equal(x[:, (hq + hkv) * d:], x0[:, (hq + hkv) * d:])


@pytest.mark.parametrize("t,hq,hkv", [(5000, 4, 1), (17000, 3, 1)])
def test_rotary_tiles_of_several_tokens(t, hq, hkv):
    """Longer calls share a workgroup among tokens: the same bits as token by token."""
    rng = np.random.default_rng(t)
    rotary = B.Rotary(64, rotary_dim=32)
    q, k = randn(rng, t, hq, 64), randn(rng, t, hkv, 64)
    at = torch.from_numpy(rng.integers(0, 200000, t).astype(np.int32)).cuda()
    q1, k1 = rotary(q, k, at)
    some = np.unique(np.concatenate([[0, 1, t - 1, t - 2], rng.integers(0, t, 20)]))
    check_turned(q1[some], q[some], at.cpu().numpy()[some], rotary, "q")
    for a in range(0, t, 1000):
        q2, k2 = rotary(q[a: a + 1000], k[a: a + 1000], at[a: a + 1000])
        assert torch.equal(q2, q1[a: a + 1000]) and torch.equal(k2, k1[a: a + 1000])


def test_negative_positions_turn_back():
    """Turning by -t undoes a turn by t, which is the gradient's way: <R x, y> = <x, R^-1 y>, up to the two roundings."""
    rng = np.random.default_rng(5)
    rotary = B.Rotary(128, layout="interleaved")
    x, y = randn(rng, 20, 4, 128), randn(rng, 20, 4, 128)
    at = torch.from_numpy(rng.integers(1, 100000, 20).astype(np.int32)).cuda()
    there = rotary(x, None, at)[0]
    back = rotary(y, None, -at)[0]
    check_turned(back, y, -at.cpu().numpy(), rotary, "back")
    a, b = (wide(there) * wide(y)).sum(2), (wide(x) * wide(back)).sum(2)
    size = (np.abs(wide(there)) * np.abs(wide(y)) + np.abs(wide(x)) * np.abs(wide(back))).sum(2)
    assert (np.abs(a - b) <= size * (BF16 + 2.0 ** -20)).all()


def test_rotary_of_nothing():
    rotary = B.Rotary(64)
    q, k = rotary(torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda"), None, torch.empty(0, dtype=torch.int32, device="cuda"))
    assert q.shape == (0, 4, 64) and k is None
    assert rotary(None, None, None) == (None, None)


def test_infinities_and_nan_stay_in_their_pair():
    rotary = B.Rotary(64, rotary_dim=32)
    x = torch.ones(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    x[0, 0, 3], x[0, 0, 40] = math.nan, math.inf
    y = rotary(x, None, torch.tensor([77], dtype=torch.int32, device="cuda"))[0].float().cpu()[0, 0]
    assert torch.isnan(y[[3, 19]]).all() and y[40] == math.inf
    rest = [i for i in range(64) if i not in (3, 19, 40)]
    assert torch.isfinite(y[rest]).all()


# ---------------------------------------------------------------------------
# the storing form
# ---------------------------------------------------------------------------
STORES = [([37, 5, 64], [37, 5, 64]), ([90, 33, 17, 0, 48], [20, 1, 0, 0, 48]), ([16, 32, 1], [1, 16, 1]), ([700], [650]), ([20], [20])]


def store_ref(cache, rotary, kn, vn, lens, news, first):
    """The oracle's pools after the store; the GPU's turned keys are checked against 64 bits and their bits stored."""
    row = 0
    for s, (n, e) in enumerate(zip(lens, news)):
        for j in range(e):
            t = n - e + j
            page = cache.bt[s, t // PAGE]
            cache.k[page, :, :, t % PAGE, :] = bits(kn[row]).reshape(cache.hkv, cache.d // 8, 8)
            cache.v[page, :, :, t % PAGE] = bits(vn[row]).reshape(cache.hkv, cache.d)
            row += 1


def pools(cache):
    k = bits(cache.g_k).reshape(cache.k.shape)
    v = bits(cache.g_v).reshape(cache.v.shape)
    return k, v


@pytest.mark.parametrize("lens,news", STORES)
@pytest.mark.parametrize("hq,hkv,d,turn,layout", [(4, 1, 64, 64, "half"), (28, 4, 128, 128, "interleaved"), (7, 7, 128, 32, "half"), (32, 2, 64, 16, "interleaved")])
def test_store(lens, news, hq, hkv, d, turn, layout):
    rng = np.random.default_rng(sum(lens) + hq)
    cache = Cache(lens, hkv, d, False, seed=sum(news))
    attn, rotary = B.DecodeAttention(hq, hkv, d), B.Rotary(d, rotary_dim=turn, layout=layout)
    t = sum(news)
    x = randn(rng, t, (hq + 2 * hkv) * d)      # a projection's packed output
    q, kn, vn = (x[:, a * d: b * d].view(t, b - a, d) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    first = rng.integers(0, 100000, len(lens)).astype(np.int32)
    positions = np.concatenate([first[s] + np.arange(e) for s, e in enumerate(news)])
    want = rotary(q, kn, torch.from_numpy(positions.astype(np.int32)).cuda())
    check_turned(want[0], q, positions, rotary, "q")
    got = attn.rotate_store(rotary, q, kn, vn, cache.g_k, cache.g_v, cache.g_bt, lens, news, first_pos=first)
    assert torch.equal(got, want[0])
    store_ref(cache, rotary, want[1], vn, lens, news, first)
    k, v = pools(cache)
    assert np.array_equal(k, cache.k) and np.array_equal(v, cache.v)
    assert np.array_equal(cache.g_bt.cpu().numpy(), cache.bt)


def test_store_positions_are_the_cache_index_unless_given():
    lens, news = [40, 21], [9, 21]
    rng = np.random.default_rng(0)
    rotary = B.Rotary(64)
    kn, vn = randn(rng, 30, 2, 64), randn(rng, 30, 2, 64)
    both = []
    for first in (None, [31, 0]):
        cache = Cache(lens, 2, 64, False, seed=3)
        assert B.DecodeAttention(4, 2, 64).rotate_store(rotary, None, kn, vn, cache.g_k, cache.g_v, cache.g_bt, lens, news, first_pos=first) is None
        both.append(pools(cache))
    assert all(np.array_equal(a, b) for a, b in zip(*both))


@pytest.mark.parametrize("turned", [True, False])
def test_decode_store(turned):
    """One token per running sequence, some of which open a page; the rows of the others are left alone."""
    lens = [33, 0, 48, 1, 16, 0, 17, 100]
    rng = np.random.default_rng(1)
    cache = Cache(lens, 4, 128, False, seed=8)
    attn, rotary = B.DecodeAttention(28, 4, 128), B.Rotary(128) if turned else None
    q, kn, vn = randn(rng, 8, 28, 128), randn(rng, 8, 4, 128), randn(rng, 8, 4, 128)
    q_out = torch.full_like(q, 5.0)
    last = np.maximum(np.array(lens) - 1, 0)
    fresh = np.full(8, -1, np.int32)
    for s in (0, 3, 6):
        fresh[s] = cache.bt[s, last[s] // PAGE]
        cache.g_bt[s, last[s] // PAGE] = -1
    first = (last + 1000).astype(np.int32)
    want = (q, kn) if rotary is None else rotary(q, kn, torch.from_numpy(first).cuda())
    attn.rotate_store(rotary, q, kn, vn, cache.g_k, cache.g_v, cache.g_bt, lens, first_pos=first, new_pages=fresh, q_out=q_out)
    live = [s for s, n in enumerate(lens) if n]
    dead = [s for s, n in enumerate(lens) if not n]
    assert torch.equal(q_out[live], want[0][live]) and (q_out[dead] == 5).all()
    store_ref(cache, rotary, want[1][live], vn[live], [lens[s] for s in range(8)], [int(n > 0) for n in lens], first)
    k, v = pools(cache)
    assert np.array_equal(k, cache.k) and np.array_equal(v, cache.v) and np.array_equal(cache.g_bt.cpu().numpy(), cache.bt)


def test_store_of_many_pages_in_runs():
    lens, news = [40000, 3000], [39990, 3000]
    rng = np.random.default_rng(2)
    cache = Cache(lens, 1, 64, False, seed=4)
    rotary = B.Rotary(64, rotary_dim=32)
    kn, vn = randn(rng, sum(news), 1, 64), randn(rng, sum(news), 1, 64)
    B.DecodeAttention(4, 1, 64).rotate_store(rotary, None, kn, vn, cache.g_k, cache.g_v, cache.g_bt, lens, news)
    at = np.concatenate([np.arange(n - e, n) for n, e in zip(lens, news)]).astype(np.int32)
    turned = rotary(None, kn, torch.from_numpy(at).cuda())[1]
    some = rng.integers(0, at.size, 50)
    check_turned(turned[some], kn[some], at[some], rotary, "k")
    store_ref(cache, rotary, turned, vn, lens, news, None)
    k, v = pools(cache)
    assert np.array_equal(k, cache.k) and np.array_equal(v, cache.v)


# ---------------------------------------------------------------------------
# attention over shared prompts
# ---------------------------------------------------------------------------
class Grouped(Cache):
    """A cache whose groups' members start with the same pages. What no token holds is poisoned."""

    def __init__(self, lens, offsets, shared, hkv, d, fp8, seed, **kw):
        super().__init__(lens, hkv, d, fp8, seed, **kw)
        self.lens, self.offsets, self.shared = list(lens), list(offsets), list(shared)
        for i, common in enumerate(shared):
            live = [s for s in range(offsets[i], offsets[i + 1]) if lens[s] > 0]
            for s in live[1:]:
                self.bt[s, : common // PAGE] = self.bt[live[0], : common // PAGE]
        # the entries that a call must not read: the other members' of shared pages
        table = self.bt.copy()
        for i, common in enumerate(shared):
            live = [s for s in range(offsets[i], offsets[i + 1]) if lens[s] > 0]
            for s in live[1:]:
                table[s, : common // PAGE] = -(1 << 30)
        self.g_bt = torch.from_numpy(table).cuda()

    def check(self, q, out, lse, scale, hq, what=""):
        g = hq // self.hkv
        qw, ow = wide(q), out.double().cpu().numpy()
        lw = None if lse is None else lse.double().cpu().numpy()
        tol_out = BF16 if out.dtype is torch.bfloat16 else U
        for s, n in enumerate(self.lens):
            for h in range(self.hkv):
                rows = slice(h * g, (h + 1) * g)
                if n == 0:
                    assert (ow[s, rows] == 0).all() and (lw is None or (lw[s, rows] == -np.inf).all())
                    continue
                k, v = self.dense(s, h, n)
                want, want_lse, size, z = R.attend(qw[s, rows], k, v, scale)
                score = (self.d + 8) * U * z + 2.0 ** -22
                tol = size * (2 * score + 2.0 ** -16 + n * U + 2.0 ** -22 * np.abs(want_lse))[:, None] + tol_out * np.abs(want)
                off = np.abs(ow[s, rows] - want) - tol
                assert off.max() <= 0, f"{what}: sequence {s} head {h}: {off.max()} beyond {tol.max()}"
                if lw is not None:
                    assert (np.abs(lw[s, rows] - want_lse) <= score + n * U + 2.0 ** -21 * np.maximum(1, np.abs(want_lse))).all(), f"{what}: lse"


GROUPS = {
    "one group": ([200, 130, 161], [0, 3], [128]),
    "prompt ends in a page": ([200, 130, 161, 141], [0, 4], [130]),
    "nothing of their own": ([64, 64, 70, 64], [0, 4], [64]),
    "no prompt": ([9, 40, 17], [0, 2, 3], [7, 0]),
    "empty members": ([0, 90, 0, 70, 0, 0, 33], [0, 5, 7], [64, 20]),
    "all empty": ([0, 0, 0], [0, 2, 3], [16, 40]),
    "one token": ([1], [0, 1], [1]),
    "groups of all sizes": ([50, 50, 49, 300, 1, 33, 34, 35, 36, 37, 38, 500, 480], [0, 3, 4, 4, 5, 11, 13], [48, 300, 9, 0, 32, 470]),
    "sixty members": ([100 + (7 * i) % 90 for i in range(60)], [0, 60], [96]),
    "long prompt": ([5000, 4900, 5100, 4811], [0, 4], [4800]),
    "odd pages": ([49, 48, 60], [0, 3], [48]),
}


@pytest.mark.parametrize("name", sorted(GROUPS))
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (28, 4, 128), (16, 1, 128), (7, 7, 64)])
@pytest.mark.parametrize("fp8", [False, True])
def test_shared(name, hq, hkv, d, fp8):
    lens, offsets, shared = GROUPS[name]
    cache = Grouped(lens, offsets, shared, hkv, d, fp8, seed=len(name) + hq, spread=1.0 if fp8 else 0.0)
    q = randn(np.random.default_rng(hq), len(lens), hq, d)
    attn = B.DecodeAttention(hq, hkv, d)
    scale = 1.0 / math.sqrt(d)
    lse = torch.full((len(lens), hq), 9.0, device="cuda")
    out = attn.shared(q, cache.g_k, cache.g_v, cache.g_bt, lens, offsets, shared, scale, lse=lse, fp8=cache.g_fp8)
    cache.check(q, out, lse, scale, hq, name)
    half = torch.full((len(lens), hq, d), 9.0, dtype=torch.bfloat16, device="cuda")
    attn.shared(q, cache.g_k, cache.g_v, cache.g_bt, lens, offsets, shared, scale, out=half, fp8=cache.g_fp8)
    assert torch.equal(half, out.to(torch.bfloat16))      # one rounding of the same result


@pytest.mark.parametrize("opts", [dict(num_cus=1), dict(num_cus=3), dict(min_chunk_pages=1), dict(min_chunk_pages=1000), dict(num_cus=256, min_chunk_pages=2)])
@pytest.mark.parametrize("name", ["groups of all sizes", "sixty members", "long prompt"])
def test_shared_cut_in_any_way(name, opts):
    lens, offsets, shared = GROUPS[name]
    cache = Grouped(lens, offsets, shared, 2, 128, False, seed=6)
    q = randn(np.random.default_rng(4), len(lens), 14, 128)
    lse = torch.empty(len(lens), 14, device="cuda")
    out = B.DecodeAttention(14, 2, 128, opts=B.make_opts(**opts)).shared(q, cache.g_k, cache.g_v, cache.g_bt, lens, offsets, shared, 0.09, lse=lse)
    cache.check(q, out, lse, 0.09, 14, name)


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
@pytest.mark.parametrize("fp8", [False, True])
def test_shared_scales(scale, fp8):
    """Negative, zero, and so large that references move many times (keys rise along the sequence)."""
    lens, offsets, shared = GROUPS["long prompt"]
    cache = Grouped(lens, offsets, shared, 2, 64, fp8, seed=6, k_mult=2.0)
    q = randn(np.random.default_rng(4), 4, 8, 64)
    lse = torch.empty(4, 8, device="cuda")
    out = B.DecodeAttention(8, 2, 64).shared(q, cache.g_k, cache.g_v, cache.g_bt, lens, offsets, shared, scale, lse=lse, fp8=cache.g_fp8)
    cache.check(q, out, lse, scale, 8)


def test_shared_is_the_plain_step():
    """Within both kernels' errors: the plain step's bound is this one's."""
    lens, offsets, shared = GROUPS["groups of all sizes"]
    cache = Grouped(lens, offsets, shared, 4, 128, False, seed=9)
    q = randn(np.random.default_rng(4), len(lens), 28, 128)
    attn = B.DecodeAttention(28, 4, 128)
    lse, lse2 = torch.empty(len(lens), 28, device="cuda"), torch.empty(len(lens), 28, device="cuda")
    out = attn.shared(q, cache.g_k, cache.g_v, cache.g_bt, lens, offsets, shared, 0.1, lse=lse)
    cache.check(q, out, lse, 0.1, 28)
    plain = attn(q, cache.g_k, cache.g_v, torch.from_numpy(cache.bt).cuda(), np.array(lens, np.int32), 0.1, lse=lse2)
    cache.check(q, plain, lse2, 0.1, 28)


def test_members_queries_do_not_meet():
    """NaN or infinite queries of one member, or of one that has left, change nothing for the others."""
    lens, offsets, shared = [200, 0, 161, 170], [0, 4], [128]
    cache = Grouped(lens, offsets, shared, 2, 128, False, seed=2)
    q = randn(np.random.default_rng(4), 4, 14, 128)
    attn = B.DecodeAttention(14, 2, 128)
    out = attn.shared(q, cache.g_k, cache.g_v, cache.g_bt, lens, offsets, shared, 0.09)
    bad = q.clone()
    bad[1], bad[2] = math.nan, math.inf
    got = attn.shared(bad, cache.g_k, cache.g_v, cache.g_bt, lens, offsets, shared, 0.09)
    for s in (0, 1, 3):
        tol = 4 * BF16 * out[s].abs().max().item() + 1e-6     # references may have moved at other blocks: weights round elsewhere
        assert (got[s] - out[s]).abs().max().item() <= tol
    assert not torch.isfinite(got[2]).any()


def test_shared_far_pages():
    """Pages whose elements lie beyond 2^31 (and bytes beyond 2^32)."""
    hq, hkv, d, n = 8, 8, 128, 140000
    kp = torch.empty((n, hkv, d // 8, PAGE, 8), dtype=torch.bfloat16, device="cuda")
    vp = torch.empty((n, hkv, d, PAGE), dtype=torch.bfloat16, device="cuda")
    lens, offsets, shared = [50, 40, 37], [0, 3], [32]
    bt = np.array([[n - 1, n - 9, n - 3, n - 4], [n - 1, n - 9, n - 5, 0], [n - 1, n - 9, n - 6, 0]], np.int32)
    rng = np.random.default_rng(3)
    rotary, attn = B.Rotary(d), B.DecodeAttention(hq, hkv, d)
    k, v = randn(rng, sum(lens), hkv, d), randn(rng, sum(lens), hkv, d)
    at = np.cumsum([0] + lens)
    for s in (1, 2):     # the members' copies of the prompt are the prompt
        k[at[s]: at[s] + 32], v[at[s]: at[s] + 32] = k[:32], v[:32]
    g_bt = torch.from_numpy(bt).cuda()
    q = randn(rng, 3, hq, d)
    attn.rotate_store(rotary, None, k, v, kp, vp, g_bt, lens, lens)
    positions = np.concatenate([np.arange(x) for x in lens]).astype(np.int32)
    kt = wide(rotary(None, k, torch.from_numpy(positions).cuda())[1])
    lse = torch.empty(3, hq, device="cuda")
    out = attn.shared(q, kp, vp, g_bt, lens, offsets, shared, 0.1, lse=lse).double().cpu().numpy()
    vw, qw = wide(v), wide(q)
    for s in range(3):
        for h in range(hkv):
            rows = slice(at[s], at[s] + lens[s])
            want, want_lse, size, z = R.attend(qw[s, h: h + 1], kt[rows, h], vw[rows, h], 0.1)
            tol = size * (2 * ((d + 8) * U * z + 2.0 ** -22) + 2.0 ** -16 + lens[s] * U + 2.0 ** -22 * np.abs(want_lse))[:, None] + U * np.abs(want)
            assert (np.abs(out[s, h: h + 1] - want) <= tol).all()


def test_shared_many_calls_and_streams():
    """More calls than the ring has slots, over two streams, of other shapes in turn."""
    attn = B.DecodeAttention(8, 2, 64)
    caches = [Grouped(*GROUPS[name], 2, 64, False, seed=5) for name in ("one group", "groups of all sizes", "long prompt")]
    qs = [randn(np.random.default_rng(i), len(c.lens), 8, 64) for i, c in enumerate(caches)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = []
    for i in range(80):
        c, q = caches[i % 3], qs[i % 3]
        out = torch.empty(len(c.lens), 8, 64, device="cuda")
        torch.cuda.synchronize() if i == 0 else None
        outs.append((i % 3, attn.shared(q, c.g_k, c.g_v, c.g_bt, c.lens, c.offsets, c.shared, 0.1, out=out, stream=streams[(i // 5) % 2])))
    torch.cuda.synchronize()
    first = {}
    for i, out in outs:
        assert torch.equal(out, first.setdefault(i, out))
    for i, c in enumerate(caches):
        c.check(qs[i], first[i], None, 0.1, 8)


# ---------------------------------------------------------------------------
# sampling
# ---------------------------------------------------------------------------
def check_samples(logits, u, got, **params):
    token, logprob, kept = (x.cpu().double().numpy() for x in got)
    x = logits.double().cpu().numpy()
    b, v = x.shape
    get = lambda name, i, default: default if params.get(name) is None else params[name][i].item()  # noqa: E731
    for i in range(b):
        t = get("temperature", i, 1.0)
        want, kp = R.sample(x[i], u[i].item(), t, get("top_k", i, 0), get("top_p", i, 1.0), get("min_p", i, 0.0))
        assert int(token[i]) in want, f"row {i} ({ {k: get(k, i, None) for k in params} }): {token[i]} for {want}"
        if -1 in want:
            assert logprob[i] == -np.inf and kept[i] == 0
            continue
        lp = want[int(token[i])]
        assert abs(logprob[i] - lp) <= 2.0 ** -24 * abs(lp) + v * 2.0 ** -44, f"row {i}: logprob {logprob[i]} for {lp}"
        assert abs(kept[i] - kp) <= 2.0 ** -24 * kp + v * 2.0 ** -43, f"row {i}: kept {kept[i]} for {kp}"


def cuda(x, dtype):
    return torch.tensor(x, dtype=dtype, device="cuda")


VOCABS = [1, 2, 7, 8, 9, 63, 255, 1000, 2047, 2049, 8191, 8193, 32001, 70000]


@pytest.mark.parametrize("v", VOCABS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_sample(v, dtype):
    """All cuts alone and together, over rows that start at odd places."""
    rng = np.random.default_rng(v)
    b = 24
    whole = torch.from_numpy((rng.standard_normal((b, v + 5)) * rng.choice([0.5, 2.0, 5.0], (b, 1))).astype(np.float32)).to(dtype).cuda()
    logits = whole[:, 3: 3 + v]
    u = cuda(rng.random(b), torch.float32)
    S = B.Sampler()
    check_samples(logits, u, S(logits, u))
    params = dict(temperature=cuda(rng.choice([0.0, 0.3, 0.7, 1.0, 1.5], b), torch.float32),
                  top_k=cuda(rng.choice([0, -3, 1, 2, 5, 50, 1000, v, 10 ** 9], b), torch.int32),
                  top_p=cuda(rng.choice([0.0, 1e-6, 0.1, 0.5, 0.9, 0.99, 1.0, 2.0], b), torch.float32),
                  min_p=cuda(rng.choice([0.0, 1e-4, 0.05, 0.3, 1.0], b), torch.float32))
    for name in params:
        check_samples(logits, u, S(logits, u, **{name: params[name]}), **{name: params[name]})
    check_samples(logits, u, S(logits, u, **params), **params)


def test_sample_equal_logits():
    """Equal logits go by their index: a cut among them keeps the lowest."""
    S = B.Sampler()
    x = torch.zeros(6, 5000, device="cuda")
    x[1:3, ::7] = 1.0
    x[3, ::2] = -0.0
    x[4] = torch.randint(0, 4, (5000,), device="cuda").float()
    x[5, 100:] = -5.0
    u = cuda([0.999, 0.5, 0.01, 0.7, 0.3, 0.9], torch.float32)
    for top_k in (1, 3, 700, 715, 4999):
        p = dict(top_k=cuda([top_k] * 6, torch.int32))
        check_samples(x, u, S(x, u, **p), **p)
        assert S(x, u, **p)[0][0].item() < top_k
    for top_p in (0.0001, 0.20003, 0.5001, 0.77):
        p = dict(top_p=cuda([top_p] * 6, torch.float32))
        check_samples(x, u, S(x, u, **p), **p)
        p["top_k"] = cuda([900] * 6, torch.int32)
        check_samples(x, u, S(x, u, **p), **p)


@pytest.mark.parametrize("dtype, bits, view", [(torch.float32, 0x7F800001, torch.int32), (torch.bfloat16, 0x7F81, torch.int16),
                                               (torch.float16, 0x7C01, torch.int16)])
def test_sample_signalling_nan_is_no_entry(dtype, bits, view):
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.standard_normal((3, 9001)).astype(np.float32)).to(dtype)
    x.view(view)[0, ::2] = bits
    x.view(view)[1, 1:] = bits
    x.view(view)[2, [0, 9000]] = bits
    x, u, S = x.cuda(), cuda([0.3, 0.6, 0.9], torch.float32), B.Sampler()
    for params in (dict(), dict(top_p=cuda([0.7] * 3, torch.float32)), dict(top_k=cuda([5000] * 3, torch.int32)),
                   dict(temperature=cuda([0.0] * 3, torch.float32))):
        check_samples(x, u, S(x, u, **params), **params)


def test_sample_masked_and_broken_logits():
    rng = np.random.default_rng(0)
    inf, nan = math.inf, math.nan
    x = torch.from_numpy(rng.standard_normal((9, 3001)).astype(np.float32)).cuda()
    x[0] = -inf
    x[1] = nan
    x[2, 1:] = -inf
    x[3, ::2] = nan
    x[4, [7, 900, 3000]] = inf
    x[5, :2990] = -inf
    x[6] = -3e38
    x[6, 5] = 3e38
    x[7, 1500:] = torch.finfo(torch.float32).min
    x[8, 0] = -inf
    u = cuda([0.5, 0.5, 0.5, 0.2, 0.4, 0.77, 0.3, 0.6, 0.0], torch.float32)
    S = B.Sampler()
    for params in (dict(), dict(top_p=cuda([0.7] * 9, torch.float32)), dict(top_k=cuda([2] * 9, torch.int32)), dict(min_p=cuda([0.2] * 9, torch.float32)),
                   dict(temperature=cuda([0.0] * 9, torch.float32)), dict(top_k=cuda([2000] * 9, torch.int32), top_p=cuda([0.9] * 9, torch.float32))):
        check_samples(x, u, S(x, u, **params), **params)
    half = x.clamp(-1e4, 1e4).half()
    check_samples(half, u, S(half, u))


def test_sample_extreme_parameters():
    """u at and beyond its ends, temperatures and shares of any kind."""
    rng = np.random.default_rng(7)
    inf, nan = math.inf, math.nan
    us = [0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, nan, 2.0 ** -30, 0.5]
    x = torch.from_numpy((rng.standard_normal((8, 1111)) * 3).astype(np.float32)).cuda()
    u = cuda(us, torch.float32)
    S = B.Sampler()
    for t in (1e-30, 1e-3, 1e30, inf, nan, -1.0):
        p = dict(temperature=cuda([t] * 8, torch.float32))
        check_samples(x, u, S(x, u, **p), **p)
    for name, dtype, values in (("top_p", torch.float32, [nan, inf, -inf, -0.5, 1e-38]), ("min_p", torch.float32, [nan, inf, -1.0, 1e-38, 5.0]),
                                ("top_k", torch.int32, [-2 ** 31, 2 ** 31 - 1, 1111, 1110])):
        for value in values:
            p = {name: cuda([value] * 8, dtype)}
            check_samples(x, u, S(x, u, **p), **p)


def test_sample_large_and_small_batches():
    """Chunks of both sizes: enough rows for the long ones, the largest vocabulary for the most."""
    rng = np.random.default_rng(11)
    S = B.Sampler()
    for b, v in ((1, 1 << 19), (40, 120000), (3, 200003)):
        x = torch.from_numpy(rng.standard_normal((b, v)).astype(np.float32)).cuda().mul_(3).to(torch.bfloat16)
        u = cuda(rng.random(b), torch.float32)
        p = dict(top_p=cuda([0.9] * b, torch.float32), top_k=cuda([5000] * b, torch.int32))
        rows = [0, b // 2, b - 1]
        for params in (dict(), p):
            got = S(x, u, **params)
            check_samples(x[rows], u[rows], [t[rows] for t in got], **{k: t[rows] for k, t in params.items()})


def test_sample_follows_the_distribution():
    """Draws by evenly spread numbers: each token's count is its share of them, off by at most one at each of its ends."""
    n = 4096
    x = torch.log(cuda([0.4, 0.05, 0.25, 0.0, 0.3], torch.float32)).expand(n, 5).contiguous()
    u = (torch.arange(n, device="cuda", dtype=torch.float32) + 0.5) / n
    token, logprob, kept = B.Sampler()(x, u)
    counts = torch.bincount(token, minlength=5).cpu().numpy()
    assert (np.abs(counts - np.array([0.4, 0.05, 0.25, 0.0, 0.3]) * n) <= 1).all() and (kept == 1).all()


def test_sample_into_given_tensors_and_checks():
    x, u = torch.randn(3, 100, device="cuda"), torch.rand(3, device="cuda")
    S = B.Sampler()
    mine = [torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(3, device="cuda"), torch.empty(3, device="cuda")]
    got = S(x, u, token=mine[0], logprob=mine[1], kept=mine[2])
    assert all(a is b for a, b in zip(got, mine))
    check_samples(x, u, got)
    empty = S(x[:0], u[:0])
    assert [t.numel() for t in empty] == [0, 0, 0]
    for bad in (dict(logits=x.double()), dict(logits=x[0]), dict(logits=x.cpu()), dict(logits=x.t()), dict(uniform=u[:2]), dict(uniform=u.double()),
                dict(top_k=u), dict(top_p=u.double()), dict(min_p=u[:1]), dict(temperature=u.cpu()), dict(token=mine[1]), dict(logits=x[:1].expand(3, 100))):
        a = dict(logits=x, uniform=u)
        a.update(bad)
        with pytest.raises((ValueError, TypeError)):
            S(a.pop("logits"), a.pop("uniform"), **a)


# ---------------------------------------------------------------------------
# graphs and streams
# ---------------------------------------------------------------------------
def test_captured_step_replays():
    """Turn, store, attention and sampling of one step in one graph, by their plan forms; every replay, with other inputs
    and the program's own calls between, has the eager calls' bits."""
    hq, hkv, d, v = 28, 4, 128, 5000
    lens, offsets, shared = [200, 130, 161, 0, 300, 290], [0, 4, 6], [128, 280]
    rng = np.random.default_rng(1)
    cache = Grouped(lens, offsets, shared, hkv, d, False, seed=5)
    b, n = len(lens), cache.n
    desc = B.make_desc(b, hq, hkv, d, cache.bt.shape[1], n, 0.1)
    info_s, work_s = B.sf_rotary_store_plan(desc, lens)
    info_a, work_a = B.sf_shared_attn_plan(desc, lens, offsets, shared)
    dev = [torch.from_numpy(np.asarray(w)).cuda() for w in (work_s, work_a)]
    ws = torch.empty(info_a.workspace_bytes, dtype=torch.uint8, device="cuda")
    rotary, S = B.Rotary(d), B.Sampler()
    turns = rotary.turns_on(torch.device("cuda", 0))
    q, k, val = randn(rng, b, hq, d), randn(rng, b, hkv, d), randn(rng, b, hkv, d)
    logits, u = torch.randn(b, v, device="cuda"), torch.rand(b, device="cuda")
    top_p = torch.full((b,), 0.9, device="cuda")
    qo = torch.zeros_like(q)

    def step():
        B.sf_rotary_store(desc, rotary.desc, info_s, None, dev[0], turns, q, qo, k, val, None, cache.g_k, cache.g_v, cache.g_bt)
        out, lse = torch.empty(b, hq, d, device="cuda"), torch.empty(b, hq, device="cuda")
        B.sf_shared_attn(desc, info_a, None, dev[1], qo, cache.g_k, cache.g_v, cache.g_bt, out, lse, workspace=ws)
        return (out, lse, *S(logits, u, top_p=top_p), *rotary(q, k, cap_pos))

    cap_pos = torch.from_numpy(np.maximum(np.array(lens) - 1, 0).astype(np.int32)).cuda()
    step()
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = step()
    for i in range(4):
        for t in (q, k, val):
            t.copy_(randn(rng, *t.shape))
        logits.normal_()
        u.uniform_()
        graph.replay()
        torch.cuda.synchronize()
        mine = [t.clone() for t in got]
        want = step()
        for a, w in zip(mine, want):
            assert torch.equal(a, w), f"replay {i}"
        check_samples(logits, u, want[2:5], top_p=top_p)


def test_runner_calls_refuse_a_capture():
    cache = Grouped(*GROUPS["one group"], 2, 64, False, seed=5)
    attn = B.DecodeAttention(8, 2, 64)
    q = randn(np.random.default_rng(0), 3, 8, 64)
    out = torch.empty(3, 8, 64, device="cuda")
    attn.shared(q, cache.g_k, cache.g_v, cache.g_bt, cache.lens, cache.offsets, cache.shared, 0.1, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out.add_(0)
        with pytest.raises(B.SfError):
            attn.shared(q, cache.g_k, cache.g_v, cache.g_bt, cache.lens, cache.offsets, cache.shared, 0.1, out=out)
        with pytest.raises(RuntimeError):
            B.Rotary(64)(q, None, torch.zeros(3, dtype=torch.int32, device="cuda"), q_out=q)
    attn.shared(q, cache.g_k, cache.g_v, cache.g_bt, cache.lens, cache.offsets, cache.shared, 0.1, out=out)
    cache.check(q, out, None, 0.1, 8)


def test_calls_on_another_stream():
    """The stream argument and the current stream, with inputs still being made on it."""
    rng = np.random.default_rng(2)
    rotary, S = B.Rotary(128), B.Sampler()
    q, at = randn(rng, 300, 28, 128), torch.arange(300, dtype=torch.int32, device="cuda")
    want = rotary(q, None, at)[0]
    logits, u = torch.randn(64, 20000, device="cuda"), torch.rand(64, device="cuda")
    top_k = torch.full((64,), 40, dtype=torch.int32, device="cuda")
    tokens = S(logits, u, top_k=top_k)[0]
    torch.cuda.synchronize()
    for given in (False, True):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            q2, l2 = torch.zeros_like(q), torch.zeros_like(logits)
            for _ in range(20):
                q2.copy_(q)
                l2.copy_(logits)
            if not given:
                got, drawn = rotary(q2, None, at)[0], S(l2, u, top_k=top_k)[0]
        if given:
            got, drawn = rotary(q2, None, at, stream=stream)[0], S(l2, u, top_k=top_k, stream=stream)[0]
        stream.synchronize()
        assert torch.equal(got, want) and torch.equal(drawn, tokens)


# ---------------------------------------------------------------------------
# all of them: the loop of a group rollout
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("grouped", [True, False])
def test_group_rollout_loop(fp8, grouped):
    """Prompts with several samples each: every step turns, stores, attends and draws; some samples end. Every step's
    attention is checked against 64 bits over the cache as the store's own definition leaves it."""
    hq, hkv, d, v = 8, 2, 64, 500
    rng = np.random.default_rng(3)
    prompts, members = [70, 33, 16], [3, 1, 4]
    lens = np.repeat(prompts, members).astype(np.int64)
    offsets = np.cumsum([0] + members)
    room = [n + 24 for n in lens]     # pages for what is to come, too
    cache = Grouped(lens, offsets, prompts, hkv, d, fp8, seed=12, spare=40, stride_extra=3)
    if grouped:
        for i in range(3):     # the begun page of each prompt was copied for every member
            page, rest = prompts[i] // PAGE, prompts[i] % PAGE
            for s in range(offsets[i] + 1, offsets[i + 1]):
                if rest:
                    for pool in (cache.g_k, cache.g_v) + (cache.g_fp8 or ()):
                        pool[int(cache.bt[s, page])] = pool[int(cache.bt[offsets[i], page])]
        groups = (offsets, prompts)
    else:
        cache = Cache(lens, hkv, d, fp8, seed=12, spare=40, stride_extra=3)
        groups = None
    bt = cache.bt.copy()
    g_bt = torch.from_numpy(bt).cuda()
    rotary, S = B.Rotary(d, base=500.0), B.Sampler()
    loop = B.DecodeLoopRunner(hq, hkv, d, cache.g_k, cache.g_v, g_bt, bt, lens, 0.2, fp8=cache.g_fp8, rotary=rotary, groups=groups)
    b = lens.size
    free0 = loop.pool.available()
    del room
    for step in range(20):
        q, kn, vn = randn(rng, b, hq, d), randn(rng, b, hkv, d), randn(rng, b, hkv, d)
        if step > 0:
            lens = np.where(lens > 0, lens + 1, 0)
        if step == 5:
            lens[1] = lens[7] = 0
        if step == 9:
            lens[0] = lens[2] = 0
        lse = torch.empty(b, hq, device="cuda")
        out = loop.step(q, lens, *((kn, vn) if step else ()), lse=lse)
        logits = torch.from_numpy(rng.standard_normal((b, v)).astype(np.float32)).cuda()
        u = cuda(rng.random(b), torch.float32)
        check_samples(logits, u, S(logits, u))
        # the cache as it is now, in 64 bits
        torch.cuda.synchronize()
        assert all(np.array_equal(g_bt.cpu().numpy()[s, : -(-int(n) // PAGE)], loop.bt_host[s, : -(-int(n) // PAGE)]) for s, n in enumerate(lens))
        now = Cache.__new__(Cache)
        now.bt, now.hkv, now.d, now.fp8 = loop.bt_host, hkv, d, fp8
        if fp8:
            now.k, now.v = cache.g_k.cpu().numpy(), cache.g_v.cpu().numpy()
            now.ks, now.vs = (x.cpu().numpy() for x in cache.g_fp8)
        else:
            now.k, now.v = pools(cache)
            now.ks = now.vs = None
        at = np.maximum(lens - 1, 0)
        turned = wide(rotary(q, None, torch.from_numpy(at.astype(np.int32)).cuda())[0])
        check_turned(rotary(q, None, torch.from_numpy(at.astype(np.int32)).cuda())[0], q, at, rotary, "q")
        tk = rotary(None, kn, torch.from_numpy(at.astype(np.int32)).cuda())[1]
        for s, n in enumerate(lens.tolist()):
            if n == 0:
                assert (out[s] == 0).all()
                continue
            for h in range(hkv):
                k, val = (cache_ref.dense(p, sc, now.bt[s, : -(-n // PAGE)], h, n, d, is_v) for p, sc, is_v in ((now.k, now.ks, False), (now.v, now.vs, True)))
                if step and not fp8:     # what this step stored
                    assert np.array_equal(k[-1], wide(tk)[s, h]) and np.array_equal(val[-1], wide(vn)[s, h])
                rows = slice(h * 4, (h + 1) * 4)
                want, want_lse, size, z = R.attend(turned[s, rows], k, val, 0.2)
                score = (d + 8) * U * z + 2.0 ** -22
                tol = size * (2 * score + 2.0 ** -16 + n * U + 2.0 ** -22 * np.abs(want_lse))[:, None] + U * np.abs(want)
                assert (np.abs(out[s, rows].double().cpu().numpy() - want) <= tol).all(), (step, s, h)
    # shared pages are free once their last holder has left
    loop.step(q, np.zeros(b), kn, vn)
    held = len({int(p) for s, n in enumerate(np.repeat(prompts, members)) for p in bt[s, : -(-int(n) // PAGE)]})
    assert loop.pool.available() == free0 + held


def test_grouped_loop_refuses_what_it_cannot_do():
    cache = Grouped([40, 40], [0, 2], [32], 2, 64, False, seed=1)
    args = (8, 2, 64, cache.g_k, cache.g_v, torch.from_numpy(cache.bt).cuda(), cache.bt, [40, 40], 0.2)
    loop = B.DecodeLoopRunner(*args, groups=([0, 2], [32]))
    q, k = torch.zeros(2, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    loop.step(q, [40, 40])
    w, pos = torch.zeros(cache.n, 2, 16, device="cuda"), torch.zeros(cache.n, 2, 16, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        loop.key_weights(q, torch.zeros(2, 8, device="cuda"), w, pos)
    with pytest.raises(ValueError):
        loop.evict(16, w, pos)
    loop.step(q, [41, 0], k, k)
    with pytest.raises(ValueError):
        loop.step(q, [42, 1], k, k)
    with pytest.raises(ValueError):
        B.DecodeLoopRunner(*args, groups=([0, 2], [48]))
    attn = B.DecodeAttention(8, 2, 64)
    for bad in (dict(q=q[:1]), dict(out=torch.empty(2, 8, 64, dtype=torch.float16, device="cuda")), dict(lse=torch.empty(8, 2, device="cuda")),
                dict(v_pool=cache.g_k), dict(shared_lens=[32, 32]), dict(group_offsets=[0, 1])):
        a = dict(q=q, k_pool=cache.g_k, v_pool=cache.g_v, block_table=args[5], seq_lens=[40, 40], group_offsets=[0, 2], shared_lens=[32], scale=0.2)
        a.update(bad)
        with pytest.raises((ValueError, B.SfError)):
            attn.shared(**a)
    with pytest.raises(ValueError):
        attn.rotate_store(B.Rotary(128), None, k, k, cache.g_k, cache.g_v, args[5], [40, 40])
    with pytest.raises(ValueError):
        attn.rotate_store(None, None, k, k, cache.g_k, cache.g_v, args[5], [40, 40], q_out=q)


def test_sample_more_flat_rows_than_places():
    """More rows that a list does not hold than the workspace has places: the rest take another way to the same token."""
    rng = np.random.default_rng(3)
    row = torch.from_numpy((0.1 * rng.standard_normal(9001)).astype(np.float32))
    x = row.expand(1500, -1).contiguous().cuda()
    u, top_p = cuda([0.7] * 1500, torch.float32), cuda([0.9] * 1500, torch.float32)
    token, logprob, kept = B.Sampler()(x, u, top_p=top_p)
    check_samples(x[:2], u[:2], (token[:2], logprob[:2], kept[:2]), top_p=top_p[:2])
    assert (token == token[0]).all() and (logprob == logprob[0]).all() and (kept == kept[0]).all()


@pytest.mark.parametrize("vocab, dtype", [(9001, torch.float32), (50001, torch.bfloat16)])
def test_sample_min_p_of_a_flat_row(vocab, dtype):
    """More entries stay than a list holds, with and without a top-p among the rows."""
    rng = np.random.default_rng(vocab)
    x = torch.from_numpy((0.3 * rng.standard_normal((6, vocab))).astype(np.float32)).to(dtype)
    x[4] = x[4] * 10
    x[5] = 0.0
    x, u = x.cuda(), cuda([0.0, 0.3, 0.999, 0.5, 0.8, 0.6], torch.float32)
    for params in (dict(min_p=cuda([0.01, 0.05, 0.2, 0.3, 0.0001, 1.0], torch.float32)),
                   dict(min_p=cuda([0.3, 0.3, 0.0, 0.4, 0.2, 0.5], torch.float32),
                        top_p=cuda([1.0, 0.9, 0.9, math.nan, 0.99, 0.5], torch.float32))):
        check_samples(x, u, B.Sampler()(x, u, **params), **params)


def test_sample_after_a_refused_call():
    """A shape that is refused leaves nothing behind for the next call of the one before it."""
    S, u = B.Sampler(), cuda([0.3, 0.8], torch.float32)
    x = torch.randn(2, 1000, generator=torch.Generator().manual_seed(5)).cuda()
    want = [t.clone() for t in S(x, u)]
    with pytest.raises(B.SfError):
        S(torch.zeros(2, (1 << 19) + 1, device="cuda"), u)
    for a, b in zip(S(x, u), want):
        assert torch.equal(a, b)
