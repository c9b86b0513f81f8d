"""GPU parity of the bounded cache against oracle/cache_ref.py, through the C ABI: the
store into fp8 pages (bit for bit), appending fp8 steps, extend over an fp8 cache, key
weights, eviction (bit for bit), and the loop of all of them.

Tolerances, u = 2^-24 (half a step of fp32), Z = max_t scale sum_d |q_d k_td| of a row:
a score is off by at most (D + 8) u Z (D products in fp32, the scale, the base change),
which its weight e^z is off by relatively, and so are the weights' sum and lse (the
hardware's exp2 and log2 are good to 2^-22).
  append: weights enter P.V as two fp16 parts, off by 2^-22 (a value scale 2^-4 of the largest: 2^-20 of its row's
    size, parts below 2^-14 being subnormal), in a plain step as two bf16 ones, by 2^-16; sums of n terms by n u.
  extend: weights and values enter P.V as fp16, off by 2^-11 each; a bf16 result by 2^-8.
  key weights: n_rows terms, each off by its score's error, u |lse|, 2^-22, and the sum's n_rows u.
"""
import numpy as np
import pytest
import torch

from oracle import cache_ref as R
from oracle.extend_ref import kv_store
from paper_2601_12784_amd import binding as B

pytestmark = pytest.mark.gpu
PAGE = 16
U = 2.0 ** -24
HEADS = [(4, 1, 64), (7, 7, 128), (28, 4, 128), (32, 2, 64)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()
    yield
    torch.cuda.synchronize()


def bits(t):
    return t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def wide(t):
    """bf16 tensor as float64."""
    return t.detach().cpu().to(torch.float32).numpy().astype(np.float64)


class Cache:
    """A scattered cache on the host (numpy, the oracle's) and on the GPU. What no token holds is poisoned."""

    def __init__(self, lens, hkv, d, fp8, seed, spare=3, stride_extra=1, spread=0.0, k_mult=1.0):
        rng = np.random.default_rng(seed)
        lens = np.asarray(lens, np.int64)
        need = -(-lens // PAGE)
        self.n = int(need.sum()) + spare
        perm = rng.permutation(self.n)
        self.bt = np.full((lens.size, int(need.max(initial=0)) + stride_extra), -1, np.int32)
        at = 0
        for s, m in enumerate(need):
            self.bt[s, :m] = perm[at: at + m]
            at += m
        self.free = perm[at:].astype(np.int32)
        self.hkv, self.d, self.fp8 = hkv, d, fp8
        valid = np.zeros((self.n, PAGE), bool)
        for s, L in enumerate(lens):
            t = np.arange(L)
            valid[self.bt[s, t // PAGE], t % PAGE] = True
        if fp8:
            self.k = np.full((self.n, hkv, PAGE * d), 0x7F, np.uint8)
            self.v = np.full((self.n, hkv, PAGE * d), 0xFF, np.uint8)
            self.ks = np.full((self.n, hkv), np.nan, np.float32)
            self.vs = np.full((self.n, hkv), np.nan, np.float32)
            for p in range(self.n):
                if not valid[p].any():
                    continue
                for pool, scale, is_v, mult in ((self.k, self.ks, False, k_mult), (self.v, self.vs, True, 1.0)):
                    for h in range(hkv):
                        x = rng.standard_normal((PAGE, d)).astype(np.float32) * np.float32(2.0 ** (spread * rng.standard_normal()) * mult)
                        codes, scale[p, h] = R.requantize(np.zeros((PAGE, d), np.uint8), np.float32(1), np.zeros(PAGE, bool), x, valid[p])
                        codes[~valid[p]] = 0x7F
                        R.put_tile_codes(pool, p, h, d, is_v, codes)
        else:
            self.k = self._bf16(rng, (self.n, hkv, d // 8, PAGE, 8)) if k_mult == 1.0 else self._bf16(rng, (self.n, hkv, d // 8, PAGE, 8), k_mult)
            self.v = self._bf16(rng, (self.n, hkv, d, PAGE))
            self.k[np.broadcast_to(~valid[:, None, None, :, None], self.k.shape)] = 0x7FC0
            self.v[np.broadcast_to(~valid[:, None, None, :], self.v.shape)] = 0x7FC0
            self.ks = self.vs = None
        self.g_bt = torch.from_numpy(self.bt.copy()).cuda()
        self.g_k, self.g_v = self._up(self.k), self._up(self.v)
        self.g_fp8 = (torch.from_numpy(self.ks.copy()).cuda(), torch.from_numpy(self.vs.copy()).cuda()) if fp8 else None

    @staticmethod
    def _bf16(rng, shape, mult=1.0):
        x = (rng.standard_normal(shape) * mult).astype(np.float32)
        return bits(torch.from_numpy(x).to(torch.bfloat16)).reshape(shape).copy()

    def _up(self, a):
        if self.fp8:
            return torch.from_numpy(a.copy()).cuda()
        return torch.from_numpy(a.view(np.int16).copy()).view(torch.bfloat16).cuda()

    def dense(self, s, h, n):
        pages = self.bt[s, : -(-n // PAGE)]
        return (R.dense(self.k, self.ks, pages, h, n, self.d, False), R.dense(self.v, self.vs, pages, h, n, self.d, True))

    def same(self, what="pools", table=True):
        """The GPU's cache is the oracle's, bit for bit."""
        if self.fp8:
            for a, b, name in ((self.g_k.cpu().numpy(), self.k, "k8"), (self.g_v.cpu().numpy(), self.v, "v8"),
                               (self.g_fp8[0].cpu().numpy().view(np.uint32), self.ks.view(np.uint32), "k_scale"),
                               (self.g_fp8[1].cpu().numpy().view(np.uint32), self.vs.view(np.uint32), "v_scale")):
                assert np.array_equal(a, b), f"{what}: {name} differs at {np.argwhere(a != b)[:4].tolist()}"
        else:
            assert np.array_equal(bits(self.g_k).reshape(self.k.shape), self.k), f"{what}: k"
            assert np.array_equal(bits(self.g_v).reshape(self.v.shape), self.v), f"{what}: v"
        if table:
            assert np.array_equal(self.g_bt.cpu().numpy(), self.bt), f"{what}: block table"


def new_tokens(rows, hkv, d, seed, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((2, rows, hkv, d), generator=g)
    if kind == "growing":      # each token larger than the ones before it
        x *= torch.logspace(-3, 3, max(rows, 1))[None, :, None, None]
    elif kind == "mixed":      # tokens of very different size, zeros, tiny values and negative zeros among them
        x *= 2.0 ** torch.randint(-40, 30, (2, rows, hkv, 1), generator=g).float()
        x[:, torch.rand(rows, generator=g) < 0.2] = 0.0
        x[:, torch.rand(rows, generator=g) < 0.1] *= -0.0
        x[:, torch.rand(rows, generator=g) < 0.1] = 2.0 ** -120
    elif kind == "zero":
        x.zero_()
    return x.to(torch.bfloat16)


def check(got, ref, tol, what):
    got = np.asarray(got, np.float64)
    assert np.array_equal(np.isfinite(got), np.isfinite(ref)), f"{what}: finiteness"
    fin = np.isfinite(ref)
    err = np.abs(got - ref)[fin]
    worst = float((err / np.broadcast_to(tol, ref.shape)[fin]).max(initial=0.0))
    print(f"  {what}: max err {err.max(initial=0):.3e}, worst err/bound {worst:.3f}", flush=True)
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound"


def reference(c, q, lens, news, scale, kind, out_bf16=False):
    """out, lse and their bounds for the rows of q [T, Hq, D] (bf16 tensor)."""
    T, hq, d = q.shape
    g = hq // c.hkv
    qd = wide(q)
    out, lse, tol, tl = np.zeros((T, hq, d)), np.full((T, hq), -np.inf), np.zeros((T, hq, d)), np.ones((T, hq))
    row = 0
    for s, (L, e) in enumerate(zip(lens, news)):
        for h in range(c.hkv):
            if e == 0:
                continue
            k, v = c.dense(s, h, L)
            o, l, spread, size = R.attention(qd[row:row + e, h * g:(h + 1) * g], k, v, scale, L - e)
            rel = 2 * (c.d + 8) * U * size + 2.0 ** -21 + 2 * L * U
            part = {"fine": 2.0 ** -20, "append": 2.0 ** -16, "extend": 2.0 ** -10}[kind]
            t = (part + rel)[..., None] * spread * 1.0001 + 1e-30
            if out_bf16:
                t = t + 2.0 ** -8 * (np.abs(o) + t)
            sl = (slice(row, row + e), slice(h * g, (h + 1) * g))
            out[sl], lse[sl], tol[sl], tl[sl] = o, l, t, rel + 4 * U * np.abs(l) + 2.0 ** -21
        row += e
    return out, lse, tol, tl


# ---------------------------------------------------------------------------
# store
# ---------------------------------------------------------------------------
STORES = [
    ([0, 1, 15, 16, 17, 33], [0, 1, 1, 1, 1, 1], "normal"),
    ([0, 1, 15, 16, 17, 33, 50], [0, 1, 15, 16, 17, 33, 0], "normal"),
    ([90, 33, 17, 48, 200], [20, 1, 17, 16, 3], "mixed"),
    ([31, 31, 31], [1, 7, 15], "growing"),
    ([40, 20], [5, 20], "zero"),
    ([300], [257], "mixed"),
]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens,news,kind", STORES)
def test_store(heads, lens, news, kind):
    hq, hkv, d = heads
    held = [L - e for L, e in zip(lens, news)]
    c = Cache(held, hkv, d, True, 7 * hkv + d, spare=40, stride_extra=25)
    _give_pages(c, held, lens)
    kn, vn = new_tokens(sum(news), hkv, d, 3 + hkv, kind)
    desc = B.make_desc(len(lens), hq, hkv, d, c.bt.shape[1], c.n, 1.0)
    info, work = B.sf_kv_store_fp8_plan(desc, lens, news)
    B.sf_kv_store_fp8(desc, info, None, torch.from_numpy(work).cuda(), kn.cuda(), vn.cuda(), None, c.g_k, c.g_v, *c.g_fp8, c.g_bt)
    R.store_fp8(bits(kn).reshape(kn.shape), bits(vn).reshape(vn.shape), lens, news, c.bt, c.k, c.v, c.ks, c.vs)
    c.same("store")


def _give_pages(c, held, lens):
    """Block-table entries for the pages that lens needs beyond held, on both sides."""
    at = 0
    for s, (a, b) in enumerate(zip(held, lens)):
        for p in range(-(-a // PAGE), -(-b // PAGE)):
            c.bt[s, p] = c.free[at]
            at += 1
    c.free = c.free[at:]
    c.g_bt.copy_(torch.from_numpy(c.bt))


def test_store_in_runs_of_four_pages():
    hkv, d = 2, 64
    lens, news = [20000, 16001, 3], [19990, 16001, 0]
    c = Cache([10, 0, 3], hkv, d, True, 5, spare=2300, stride_extra=1300)
    _give_pages(c, [10, 0, 3], lens)
    kn, vn = new_tokens(sum(news), hkv, d, 9, "mixed")
    info, _ = B.sf_kv_store_fp8_plan(B.make_desc(3, 4, hkv, d, c.bt.shape[1], c.n, 1.0), lens, news)
    assert info.num_rows < 700
    B.DecodeAttention(4, hkv, d).store_fp8(kn.cuda(), vn.cuda(), c.g_k, c.g_v, c.g_fp8, c.g_bt, lens, news)
    R.store_fp8(bits(kn).reshape(kn.shape), bits(vn).reshape(vn.shape), lens, news, c.bt, c.k, c.v, c.ks, c.vs)
    c.same("store in runs")


def test_store_of_whole_pages_is_the_quantizer():
    hkv, d, n = 4, 128, 37
    g = torch.Generator(device="cuda").manual_seed(1)
    kn = torch.randn((n * PAGE, hkv, d), generator=g, device="cuda").to(torch.bfloat16)
    vn = torch.randn((n * PAGE, hkv, d), generator=g, device="cuda").to(torch.bfloat16)
    kp = kn.view(n, PAGE, hkv, d // 8, 8).permute(0, 2, 3, 1, 4).contiguous()
    vp = vn.view(n, PAGE, hkv, d).permute(0, 2, 3, 1).contiguous()
    desc = B.make_desc(1, 28, hkv, d, n, n, 1.0)
    want = [torch.zeros((n, hkv, PAGE * d), dtype=torch.uint8, device="cuda") for _ in range(2)] + [torch.zeros((n, hkv), device="cuda") for _ in range(2)]
    pages = torch.arange(n, dtype=torch.int32, device="cuda")
    B.sf_kv_quantize_fp8(desc, kp, vp, pages, torch.full_like(pages, PAGE), *want)
    got = [torch.full_like(t, 9) for t in want]
    B.DecodeAttention(28, hkv, d).store_fp8(kn, vn, got[0], got[1], (got[2], got[3]), pages.view(1, n), [n * PAGE], [n * PAGE])
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ["normal", "mixed", "growing"])
@pytest.mark.parametrize("heads", [(4, 1, 64), (28, 4, 128)])
def test_store_token_by_token(heads, kind):
    hq, hkv, d = heads
    steps, lens = 40, np.array([3, 16, 0], np.int64)
    c = Cache(lens, hkv, d, True, 11, spare=20, stride_extra=4)
    kn, vn = new_tokens(3 * steps, hkv, d, 21, kind)
    attn = B.DecodeAttention(hq, hkv, d)
    for i in range(steps):
        lens = lens + 1
        pages = np.where((lens - 1) % PAGE == 0, 0, -1).astype(np.int32)
        for s in np.nonzero(pages == 0)[0]:
            pages[s], c.free = c.free[0], c.free[1:]
        k, v = kn[3 * i:3 * i + 3], vn[3 * i:3 * i + 3]
        attn.store_fp8(k.cuda(), v.cuda(), c.g_k, c.g_v, c.g_fp8, c.g_bt, lens, [1, 1, 1], new_pages=pages)
        R.store_fp8(bits(k).reshape(k.shape), bits(v).reshape(v.shape), lens, [1, 1, 1], c.bt, c.k, c.v, c.ks, c.vs, pages)
        c.same(f"step {i}")


# ---------------------------------------------------------------------------
# appending step over an fp8 cache
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens", [[1], [17, 64, 130, 300], [0, 1, 16, 17, 2, 0, 700], [33] * 40, [9000, 3]])
def test_append_step(heads, lens):
    hq, hkv, d = heads
    held = [max(0, L - 1) for L in lens]
    c = Cache(held, hkv, d, True, 31 + d, spare=len(lens) + 2, stride_extra=1, spread=1.0)
    pages = np.full(len(lens), -1, np.int32)
    for s, L in enumerate(lens):
        if L > 0 and (L - 1) % PAGE == 0:
            pages[s], c.free = c.free[0], c.free[1:]
    kn, vn = new_tokens(len(lens), hkv, d, 8, "normal")
    q = new_tokens(len(lens), hq, d, 9)[0]
    out = torch.full((len(lens), hq, d), 7.0, device="cuda")
    lse = torch.full((len(lens), hq), 7.0, device="cuda")
    scale = 1.0 / np.sqrt(d)
    attn = B.DecodeAttention(hq, hkv, d)
    attn(q.cuda(), c.g_k, c.g_v, c.g_bt, lens, scale, out=out, lse=lse, append=(kn.cuda(), vn.cuda(), pages), fp8=c.g_fp8)
    news = [min(1, L) for L in lens]
    live = np.asarray(lens) > 0
    R.store_fp8(bits(kn).reshape(kn.shape)[live], bits(vn).reshape(vn.shape)[live], lens, news, c.bt, c.k, c.v, c.ks, c.vs, pages)
    c.same("append")
    ro, rl, to, tl = reference(c, q[torch.from_numpy(live)], lens, news, scale, "fine")
    ts = reference(c, q[torch.from_numpy(live)], lens, news, scale, "append")[2]
    o, l = out.cpu().numpy(), lse.cpu().numpy()
    check(o[live], ro, to, "out")
    check(l[live], rl, tl, "lse")
    assert np.all(o[~live] == 0) and np.all(np.isneginf(l[~live]))
    # the same without the lse: the same bits; a plain step over the stored cache rounds its weights to 16 bits
    again = attn(q.cuda(), c.g_k, c.g_v, c.g_bt, lens, scale, append=(kn.cuda(), vn.cuda(), pages), fp8=c.g_fp8)
    plain = attn(q.cuda(), c.g_k, c.g_v, c.g_bt, lens, scale, fp8=c.g_fp8)
    c.same("append again")
    assert torch.equal(again, out)
    check(plain.cpu().numpy()[live], ro, ts, "plain step")


def test_append_step_refusals():
    attn = B.DecodeAttention(4, 1, 64)
    c = Cache([5], 1, 64, True, 1)
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda")
    kn = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    before = c.g_k.clone()
    with pytest.raises(B.SfError):      # a value array that is not 16-byte aligned
        odd = torch.zeros(65, dtype=torch.bfloat16, device="cuda")[1:].view(1, 1, 64)
        attn(q, c.g_k, c.g_v, c.g_bt, [6], 0.1, append=(kn, odd, [-1]), fp8=c.g_fp8)
    with pytest.raises(ValueError):
        attn(q, c.g_k, c.g_v, c.g_bt, [6], 0.1, append=(kn, kn.half(), [-1]), fp8=c.g_fp8)
    with pytest.raises(ValueError):
        attn.store_fp8(kn, kn, c.g_k, c.g_v, c.g_fp8, c.g_bt, [6], [2])      # two new tokens, one row
    with pytest.raises(ValueError):
        attn.store_fp8(kn, kn, c.g_k, c.g_v, c.g_fp8, c.g_bt, [6, 7], [1])
    torch.cuda.synchronize()
    assert torch.equal(before, c.g_k)


# ---------------------------------------------------------------------------
# extend over an fp8 cache
# ---------------------------------------------------------------------------
EXTENDS = [
    ([1], [1]),
    ([37, 5, 64, 0, 20], [37, 5, 64, 0, 0]),
    ([90, 33, 17, 48], [20, 1, 17, 16]),
    ([700], [700]),
    ([1500, 40], [3, 2]),
    ([260, 129, 31, 33], [1, 128, 31, 2]),
]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens,news", EXTENDS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_extend(heads, lens, news, dtype):
    hq, hkv, d = heads
    held = [L - e for L, e in zip(lens, news)]
    c = Cache(held, hkv, d, True, 41 + d, spare=60, stride_extra=45, spread=2.0)
    _give_pages(c, held, lens)
    T = sum(news)
    kn, vn = new_tokens(T, hkv, d, 13)
    q = new_tokens(T, hq, d, 14)[0]
    scale = -0.13 if len(lens) == 3 else 1.0 / np.sqrt(d)
    attn = B.ExtendAttention(hq, hkv, d)
    out = torch.full((T, hq, d), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((T, hq), 7.0, device="cuda")
    attn(q.cuda(), c.g_k, c.g_v, c.g_bt, lens, news, scale, out=out, lse=lse, k_new=kn.cuda(), v_new=vn.cuda(), fp8=c.g_fp8)
    R.store_fp8(bits(kn).reshape(kn.shape), bits(vn).reshape(vn.shape), lens, news, c.bt, c.k, c.v, c.ks, c.vs)
    c.same("extend")
    ro, rl, to, tl = reference(c, q, lens, news, scale, "extend", dtype is torch.bfloat16)
    check(out.float().cpu().numpy(), ro, to, "out")
    check(lse.cpu().numpy(), rl, tl, "lse")
    # the plan of whole items, over the cache as it now stands
    desc = B.make_desc(len(lens), hq, hkv, d, c.bt.shape[1], c.n, scale)
    info, work = B.sf_extend_attn_plan(desc, lens, news)
    o2, l2 = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    B.sf_extend_attn_fp8(desc, info, None, torch.from_numpy(work).cuda(), q.cuda(), c.g_k, c.g_v, *c.g_fp8, c.g_bt, o2, l2)
    check(o2.float().cpu().numpy(), ro, to, "out, whole items")
    check(l2.cpu().numpy(), rl, tl, "lse, whole items")


@pytest.mark.parametrize("heads", [(28, 4, 128), (14, 2, 64)])
def test_extend_cut_walks_and_unlike_pages(heads):
    """A short grid: key walks cut into parts. Value scales from 2^-9 to 2^9, so the reference moves in mid-walk."""
    hq, hkv, d = heads
    lens, news = [6000], [40]
    c = Cache([5960], hkv, d, True, 43, spare=4, stride_extra=4, spread=3.0)
    _give_pages(c, [5960], lens)
    kn, vn = new_tokens(40, hkv, d, 15)
    q = new_tokens(40, hq, d, 16)[0]
    attn = B.ExtendAttention(hq, hkv, d)
    out, lse = torch.empty((40, hq, d), device="cuda"), torch.empty((40, hq), device="cuda")
    attn(q.cuda(), c.g_k, c.g_v, c.g_bt, lens, news, 0.02, out=out, lse=lse, k_new=kn.cuda(), v_new=vn.cuda(), fp8=c.g_fp8)
    R.store_fp8(bits(kn).reshape(kn.shape), bits(vn).reshape(vn.shape), lens, news, c.bt, c.k, c.v, c.ks, c.vs)
    c.same("extend")
    ro, rl, to, tl = reference(c, q, lens, news, 0.02, "extend")
    check(out.cpu().numpy(), ro, to, "out")
    check(lse.cpu().numpy(), rl, tl, "lse")


def test_extend_of_one_token_is_the_appending_step():
    hq, hkv, d = 28, 4, 128
    lens = [50, 17, 400]
    held = [L - 1 for L in lens]
    a, b = (Cache(held, hkv, d, True, 47, spare=5, stride_extra=1) for _ in range(2))
    _give_pages(a, held, lens)
    _give_pages(b, held, lens)
    kn, vn = (x.cuda() for x in new_tokens(3, hkv, d, 17))
    q = new_tokens(3, hq, d, 18)[0].cuda()
    x = B.ExtendAttention(hq, hkv, d)(q, a.g_k, a.g_v, a.g_bt, lens, [1] * 3, 0.09, k_new=kn, v_new=vn, fp8=a.g_fp8)
    y = B.DecodeAttention(hq, hkv, d)(q, b.g_k, b.g_v, b.g_bt, lens, 0.09, append=(kn, vn, [-1] * 3), fp8=b.g_fp8)
    assert torch.equal(a.g_k, b.g_k) and torch.equal(a.g_v, b.g_v)
    assert torch.allclose(x, y, rtol=2.0 ** -9, atol=2.0 ** -9 * float(y.abs().max()))


def test_extend_scale_zero_averages():
    hq, hkv, d = 4, 1, 64
    c = Cache([0], hkv, d, True, 48, spare=5, stride_extra=3)
    _give_pages(c, [0], [40])
    kn, vn = new_tokens(40, hkv, d, 19)
    q = new_tokens(40, hq, d, 20)[0].cuda()
    out = B.ExtendAttention(hq, hkv, d)(q, c.g_k, c.g_v, c.g_bt, [40], [40], 0.0, k_new=kn.cuda(), v_new=vn.cuda(), fp8=c.g_fp8)
    R.store_fp8(bits(kn).reshape(kn.shape), bits(vn).reshape(vn.shape), [40], [40], c.bt, c.k, c.v, c.ks, c.vs)
    _, v = c.dense(0, 0, 40)
    want = np.cumsum(v, 0) / np.arange(1, 41)[:, None]
    check(out.cpu().numpy(), np.repeat(want[:, None], 4, 1), 2.0 ** -9 * np.abs(v).max(), "averages")


# ---------------------------------------------------------------------------
# key weights
# ---------------------------------------------------------------------------
def run_weights(c, q, lse, lens, news, hq, scale, w0, pos0, held=None, first=None, in_place=False, runner=True, opts=None):
    w, pos = torch.from_numpy(w0.copy()).cuda(), torch.from_numpy(pos0.copy()).cuda()
    out = w if in_place else torch.full_like(w, 5.0)
    ks = c.g_fp8[0] if c.fp8 else None
    if runner:
        B.DecodeAttention(hq, c.hkv, c.d, opts=opts).key_weights(q, lse, c.g_k, c.g_bt, lens, news, scale, w, out, positions=pos,
                                                                 held_lens=held, first_pos=first, k_scale=ks)
    else:
        desc = B.make_desc(len(lens), hq, c.hkv, c.d, c.bt.shape[1], c.n, scale)
        info, work = B.sf_key_weights_plan(desc, lens, news, held, first, opts=opts)
        ws = torch.full((max(1, info.workspace_bytes // 4),), float("nan"), device="cuda")
        B.sf_key_weights(desc, info, None, torch.from_numpy(work).cuda(), q, lse, c.g_k, c.g_bt, w, out, positions=pos,
                         k_scale=ks, workspace=ws)
    return out.cpu().numpy(), pos.cpu().numpy()


WEIGHTS = [
    ([1], [1]),
    ([17, 64, 130, 300, 0, 33], [1, 1, 1, 1, 0, 1]),
    ([90, 33, 17, 48, 20], [20, 1, 17, 16, 0]),
    ([700, 65], [700, 65]),
    ([5000], [3]),
    ([9000, 4000], [1, 1]),
    ([1030, 16], [40, 9]),
]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,news", WEIGHTS)
def test_key_weights(heads, fp8, lens, news):
    hq, hkv, d = heads
    g = hq // hkv
    c = Cache(lens, hkv, d, fp8, 51 + d, k_mult=1.5)
    T = sum(news)
    rng = np.random.default_rng(4)
    q = new_tokens(T, hq, d, 22)[0]
    scale = -0.11 if len(lens) == 5 else 1.0 / np.sqrt(d)
    _, rl, _, _ = reference(c, q, lens, news, scale, "append")
    lse = rl.astype(np.float32)
    if T > 3:   # rows that add nothing
        lse[1, 0], lse[2, hq - 1] = -np.inf, np.nan
    w0 = (rng.random((c.n, hkv, PAGE)) * 9).astype(np.float32)
    w0[rng.random(w0.shape) < 0.1] = 0
    pos0 = rng.integers(0, 1000, w0.shape).astype(np.int32)
    held = [L - e for L, e in zip(lens, news)] if len(lens) % 2 else [(L - e) // 2 for L, e in zip(lens, news)]
    first = [h + 50 for h in held]
    # what stands for keys weighed first must not be read
    for s, (L, h) in enumerate(zip(lens, held)):
        for t in range(h, L):
            w0[c.bt[s, t // PAGE], :, t % PAGE] = np.nan
    args = (c, q.cuda(), torch.from_numpy(lse).cuda(), lens, news, hq, scale, w0, pos0, held, first)
    got, pos = run_weights(*args)
    want, tol, want_pos = np.full_like(w0, 5.0, dtype=np.float64), np.zeros(w0.shape), pos0.copy()
    qd, row = wide(q), 0
    for s, (L, e) in enumerate(zip(lens, news)):
        for h in range(hkv if e else 0):
            k, _ = c.dense(s, h, L)
            ls = lse[row:row + e, h * g:(h + 1) * g].astype(np.float64)
            u, size = R.key_weights(qd[row:row + e, h * g:(h + 1) * g], ls, k, scale, L - e)
            top = np.abs(ls[np.isfinite(ls)]).max(initial=0)
            rel = 2 * (d + 8) * U * size + 4 * U * top + 2.0 ** -21 + (e * g + 4) * U
            t = np.arange(L)
            pg = c.bt[s, t // PAGE]
            before = np.where(t < held[s], w0[pg, h, t % PAGE], 0).astype(np.float64)
            want[pg, h, t % PAGE] = before + u
            tol[pg, h, t % PAGE] = rel * u + 2 * U * (before + u) + 1e-37
            new = t >= held[s]
            want_pos[pg[new], h, t[new] % PAGE] = first[s] + t[new] - held[s]
        row += e
    touched = tol > 0
    assert np.all(got[~touched] == 5.0) or np.array_equal(got[~touched], np.full((~touched).sum(), 5.0, np.float32))
    check(got[touched], want[touched], tol[touched], "weights")
    assert np.array_equal(pos, want_pos)
    again, _ = run_weights(*args, runner=False, in_place=True)
    assert np.array_equal(again[touched], got[touched])           # in place, by the plan form: the same bits
    one, pos = run_weights(*args, runner=False, opts=B.make_opts(num_cus=1))   # eight waves, many blocks of keys each
    check(one[touched], want[touched], tol[touched], "weights, one compute unit")
    assert np.array_equal(pos, want_pos)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("news", [[2, 1, 0], [40, 17, 3]])   # the list of a decode step and that of items
def test_key_weights_of_rows_that_hold_no_numbers(fp8, news):
    """A row whose lse is not finite adds nothing whatever its queries hold: the same bits as with zeros there."""
    lens, (hq, hkv, d) = [90, 17, 33], (8, 2, 128)
    c = Cache(lens, hkv, d, fp8, 58, k_mult=1.5)
    q = new_tokens(sum(news), hq, d, 23)[0]
    lse = reference(c, q, lens, news, 0.1, "append")[1].astype(np.float32)
    zeros, bad = q.clone(), q.clone()
    row = 0
    for value, dead in ((float("nan"), -np.inf), (float("inf"), np.nan), (-float("inf"), np.inf)):
        for h in (0, hq - 1):
            lse[row, h], zeros[row, h], bad[row, h] = dead, 0, value
        row = (row + news[0] - 1) % sum(news)
    w0, pos0 = np.ones((c.n, hkv, PAGE), np.float32), np.zeros((c.n, hkv, PAGE), np.int32)
    held = [L - e for L, e in zip(lens, news)]
    got = [run_weights(c, x.cuda(), torch.from_numpy(lse).cuda(), lens, news, hq, 0.1, w0, pos0, held, held)[0] for x in (zeros, bad)]
    assert np.all(np.isfinite(got[0])) and np.array_equal(*got)


def test_key_weights_cut_walks_are_the_same_up_to_rounding():
    """A device of one compute unit cuts nothing, one of 4096 cuts every walk to eight tiles."""
    hq, hkv, d, L = 28, 4, 128, 900
    c = Cache([L], hkv, d, False, 61)
    q = new_tokens(L, hq, d, 23)[0].cuda()
    out = torch.empty((L, hq, d), device="cuda")
    lse = torch.empty((L, hq), device="cuda")
    B.ExtendAttention(hq, hkv, d)(q, c.g_k, c.g_v, c.g_bt, [L], [L], 0.1, out=out, lse=lse)
    w0, p0 = np.zeros((c.n, hkv, PAGE), np.float32), np.zeros((c.n, hkv, PAGE), np.int32)
    got = []
    for cus in (1, 256, 4096):
        x, _ = run_weights(c, q, lse, [L], [L], hq, 0.1, w0, p0, held=[0], opts=B.make_opts(num_cus=cus), runner=False)
        got.append(x)
    y, _ = run_weights(c, q, lse, [L], [L], hq, 0.1, w0, p0, held=[0], opts=B.make_opts(num_cus=256))
    assert np.array_equal(y, got[1], equal_nan=True)
    t = np.arange(L)
    rows = [x[c.bt[0, t // PAGE], :, t % PAGE].astype(np.float64) for x in got]
    for x in rows:
        assert np.allclose(x, rows[0], rtol=7 * L * 2 * U, atol=0)
        assert np.allclose(x.sum(0), 7 * L, rtol=1e-4)           # every row's weights sum to 1


# ---------------------------------------------------------------------------
# eviction
# ---------------------------------------------------------------------------
EVICTS = [
    # lens, keep, sinks, recent, weights
    ([40, 17, 0, 16, 5, 100], [20, 17, 5, 0, 9, 33], 0, 0, "random"),
    ([40, 17, 33], [20, 16, 32], 4, 8, "random"),
    ([130, 64], [64, 48], 2, 16, "ties"),
    ([130, 64, 31], [100, 1, 30], 0, 0, "equal"),
    ([200], [90], 0, 1, "odd"),
    ([5000, 4097], [3001, 4096], 4, 100, "random"),
]


def make_weights(kind, shape, rng):
    w = rng.random(shape).astype(np.float32)
    if kind == "ties":
        w = np.floor(w * 4).astype(np.float32) * np.float32(0.25)
    elif kind == "equal":
        w[:] = 1.0
    elif kind == "odd":
        w = ((w - 0.3) * 10).astype(np.float32)
        for value in (np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-42):
            w[rng.random(shape) < 0.1] = value
    return w


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("case", EVICTS, ids=lambda c: f"{c[4]}-{len(c[0])}-{c[0][0]}")
def test_evict(heads, fp8, case):
    lens, keep, sinks, recent, kind = case
    hq, hkv, d = heads
    c = Cache(lens, hkv, d, fp8, 71 + d, spread=1.5)
    rng = np.random.default_rng(6)
    w = make_weights(kind, (c.n, hkv, PAGE), rng)
    pos = np.zeros((c.n, hkv, PAGE), np.int32)
    ends = [L + 30 for L in lens]
    for s, L in enumerate(lens):
        for h in range(hkv):
            t = np.arange(L)
            # distinct positions below the end, not in slot order, the last ones the newest
            p = np.sort(rng.choice(ends[s], L, replace=False))
            p[: L // 2] = rng.permutation(p[: L // 2])
            pos[c.bt[s, t // PAGE], h, t % PAGE] = p
    gw, gp = torch.from_numpy(w.copy()).cuda(), torch.from_numpy(pos.copy()).cuda()
    wo, po = torch.full_like(gw, 3.0), torch.full_like(gp, -7)
    want_w, want_p = np.full_like(w, 3.0), np.full_like(pos, -7)
    kw = dict(ends=ends, sinks=sinks, recent=recent)
    attn = B.DecodeAttention(hq, hkv, d)
    attn.evict(c.g_k, c.g_v, c.g_bt, lens, keep, gw, gp, weights_out=wo, positions_out=po, fp8=c.g_fp8, **kw)
    before = (c.k.copy(), c.v.copy())
    R.evict(c.k, c.v, c.ks, c.vs, c.bt, lens, keep, w.copy(), pos.copy(), want_w, want_p, **kw)
    assert np.array_equal(wo.cpu().numpy(), want_w, equal_nan=True)
    assert np.array_equal(po.cpu().numpy(), want_p)
    assert np.array_equal(gw.cpu().numpy(), w, equal_nan=True) and np.array_equal(gp.cpu().numpy(), pos)
    c.same("evict")
    # in place, by the plan form, from the same start
    again = Cache(lens, hkv, d, fp8, 71 + d, spread=1.5)
    assert np.array_equal(before[0], again.k) and np.array_equal(before[1], again.v)
    desc = B.make_desc(len(lens), hq, hkv, d, c.bt.shape[1], c.n, 1.0)
    info, work = B.sf_kv_evict_plan(desc, lens, keep, ends, sinks, recent)
    ws = torch.full((info.workspace_bytes // 4 + 1,), 0x7F7F7F7F, dtype=torch.int32, device="cuda")
    B.sf_kv_evict(desc, info, None, torch.from_numpy(work).cuda(), again.g_k, again.g_v, again.g_bt, gw, gp, fp8=again.g_fp8,
                  workspace=ws)
    assert torch.equal(again.g_k.view(torch.uint8), c.g_k.view(torch.uint8))
    assert torch.equal(again.g_v.view(torch.uint8), c.g_v.view(torch.uint8))
    R.evict(before[0].copy(), before[1].copy(), None if c.ks is None else c.ks.copy(), None if c.vs is None else c.vs.copy(), c.bt,
            lens, keep, w, pos, w, pos, **kw)
    assert np.array_equal(gw.cpu().numpy(), w, equal_nan=True) and np.array_equal(gp.cpu().numpy(), pos)


def test_evict_many_pages():
    """More than 2048 kept pages (runs of four) and sequences of several rounds of a workgroup's pages."""
    hq, hkv, d = 2, 1, 64
    lens, keep = [40000, 9000, 100], [33333, 1234, 100]
    c = Cache(lens, hkv, d, False, 75)
    rng = np.random.default_rng(8)
    w = make_weights("ties", (c.n, hkv, PAGE), rng) + (rng.random((c.n, hkv, PAGE)) < 0.5).astype(np.float32)
    pos = np.zeros((c.n, hkv, PAGE), np.int32)
    for s, L in enumerate(lens):
        t = np.arange(L)
        pos[c.bt[s, t // PAGE], 0, t % PAGE] = t
    gw, gp = torch.from_numpy(w.copy()).cuda(), torch.from_numpy(pos.copy()).cuda()
    B.DecodeAttention(hq, hkv, d).evict(c.g_k, c.g_v, c.g_bt, lens, keep, gw, gp, sinks=4, recent=1000)
    R.evict(c.k, c.v, None, None, c.bt, lens, keep, w, pos, w, pos, sinks=4, recent=1000)
    c.same("evict")
    assert np.array_equal(gw.cpu().numpy(), w) and np.array_equal(gp.cpu().numpy(), pos)


# ---------------------------------------------------------------------------
# streams and graphs
# ---------------------------------------------------------------------------
def test_runner_calls_refuse_a_capturing_stream():
    hq, hkv, d = 4, 1, 64
    c = Cache([40], hkv, d, True, 81)
    kn, vn = (x.cuda() for x in new_tokens(1, hkv, d, 30))
    attn = B.DecodeAttention(hq, hkv, d)
    attn.store_fp8(kn, vn, c.g_k, c.g_v, c.g_fp8, c.g_bt, [40], [1])
    torch.cuda.synchronize()
    before = c.g_k.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(B.SfError) as e:
            attn.store_fp8(-kn, vn, c.g_k, c.g_v, c.g_fp8, c.g_bt, [40], [1])
        assert e.value.status == B.UNSUPPORTED
        kn.add_(0)      # something to capture
    torch.cuda.synchronize()
    assert torch.equal(c.g_k, before)


def test_captured_calls_replay():
    """Store, extend, weights and eviction captured by their plan forms; every replay against the eager result."""
    hq, hkv, d, lens, news, keep = 28, 4, 128, [300, 77], [40, 77], [150, 60]
    held = [L - e for L, e in zip(lens, news)]
    c = Cache(held, hkv, d, True, 83, spare=20, stride_extra=15)
    _give_pages(c, held, lens)
    kn, vn = (x.cuda() for x in new_tokens(117, hkv, d, 31))
    q = new_tokens(117, hq, d, 32)[0].cuda()
    start = [t.clone() for t in (c.g_k, c.g_v, *c.g_fp8)]
    out, lse = torch.zeros((117, hq, d), device="cuda"), torch.zeros((117, hq), device="cuda")
    w = torch.zeros((c.n, hkv, PAGE), device="cuda")
    pos = torch.zeros((c.n, hkv, PAGE), dtype=torch.int32, device="cuda")
    desc = B.make_desc(2, hq, hkv, d, c.bt.shape[1], c.n, 0.09)
    plans = [B.sf_kv_store_fp8_plan(desc, lens, news), B.sf_extend_attn_plan(desc, lens, news),
             B.sf_key_weights_plan(desc, lens, news, held_lens=[0, 0]), B.sf_kv_evict_plan(desc, lens, keep, sinks=2, recent=8)]
    work = [torch.from_numpy(x).cuda() for _, x in plans]
    space = [torch.zeros(max(1, getattr(i, "workspace_bytes", 0)), dtype=torch.uint8, device="cuda") for i, _ in plans]

    def reset():
        for t, s in zip((c.g_k, c.g_v, *c.g_fp8), start):
            t.copy_(s)
        w.fill_(float("nan"))

    def calls():
        B.sf_kv_store_fp8(desc, plans[0][0], None, work[0], kn, vn, None, c.g_k, c.g_v, *c.g_fp8, c.g_bt)
        B.sf_extend_attn_fp8(desc, plans[1][0], None, work[1], q, c.g_k, c.g_v, *c.g_fp8, c.g_bt, out, lse)
        B.sf_key_weights(desc, plans[2][0], None, work[2], q, lse, c.g_k, c.g_bt, w, positions=pos, k_scale=c.g_fp8[0], workspace=space[2])
        B.sf_kv_evict(desc, plans[3][0], None, work[3], c.g_k, c.g_v, c.g_bt, w, pos, fp8=c.g_fp8, workspace=space[3])

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (c.g_k, c.g_v, *c.g_fp8, out, lse, w.view(torch.int32), pos)]

    reset()
    calls()
    eager = results()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        calls()
    for _ in range(3):
        reset()
        out.zero_()
        graph.replay()
        for a, b in zip(results(), eager):
            assert torch.equal(a, b) or (a.is_floating_point() and torch.equal(torch.isnan(a), torch.isnan(b)))
        reset()
        calls()
        for a, b in zip(results(), eager):
            assert torch.equal(a, b) or (a.is_floating_point() and torch.equal(torch.isnan(a), torch.isnan(b)))


def test_captured_extend_object_over_an_fp8_cache():
    hq, hkv, d, lens, news = 28, 4, 128, [130, 20], [50, 20]
    held = [80, 0]
    c = Cache(held, hkv, d, True, 85, spare=20, stride_extra=8)
    _give_pages(c, held, lens)
    kn, vn = (x.cuda() for x in new_tokens(70, hkv, d, 33))
    q = new_tokens(70, hq, d, 34)[0].cuda()
    attn = B.ExtendAttention(hq, hkv, d)
    out, lse = torch.zeros((70, hq, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((70, hq), device="cuda")
    call = lambda: attn(q, c.g_k, c.g_v, c.g_bt, lens, news, 0.09, out=out, lse=lse, k_new=kn, v_new=vn, fp8=c.g_fp8)  # noqa: E731
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in (out, lse, c.g_k, c.g_v)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for t in (out, lse):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.g_k, want[2]) and torch.equal(c.g_v, want[3])
        assert torch.allclose(out.float(), want[0].float(), rtol=2.0 ** -7, atol=1e-3) and torch.allclose(lse, want[1], rtol=1e-5)
        call()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_side_stream_and_many_calls_of_a_ring():
    """70 stores, weights and evictions in a row (the ring has 32 slots), on a stream of their own."""
    hq, hkv, d = 28, 4, 128
    lens = np.array([50, 33], np.int32)
    c, e = (Cache(lens, hkv, d, True, 87, spare=30, stride_extra=14) for _ in range(2))
    for x in (c, e):
        _give_pages(x, lens, lens + 80)
    attn, stream = B.DecodeAttention(hq, hkv, d), torch.cuda.Stream()
    kn, vn = new_tokens(140, hkv, d, 35, "mixed")
    q = new_tokens(2, hq, d, 36)[0].cuda()
    lse = torch.full((2, hq), 3.0, device="cuda")
    w, pos = torch.zeros((c.n, hkv, PAGE), device="cuda"), torch.zeros((c.n, hkv, PAGE), dtype=torch.int32, device="cuda")
    gk, gv = kn.cuda(), vn.cuda()
    stream.wait_stream(torch.cuda.current_stream())
    total = w.clone()
    for i in range(70):
        n = lens + i + 1
        attn.store_fp8(gk[2 * i:2 * i + 2], gv[2 * i:2 * i + 2], c.g_k, c.g_v, c.g_fp8, c.g_bt, n, [1, 1], stream=stream)
        attn.key_weights(q, lse, c.g_k, c.g_bt, n, [1, 1], 0.01, w, positions=pos, held_lens=n - 1 if i else [0, 0],
                         k_scale=c.g_fp8[0], stream=stream)
    stream.synchronize()
    for i in range(70):
        R.store_fp8(bits(kn)[2 * i:2 * i + 2].reshape(2, hkv, d), bits(vn)[2 * i:2 * i + 2].reshape(2, hkv, d), lens + i + 1, [1, 1],
                    c.bt, c.k, c.v, c.ks, c.vs)
    c.same("70 steps")
    assert total.sum() == 0
    for s in range(2):
        t = np.arange(lens[s] + 70)
        p = pos.cpu().numpy()[c.bt[s, t // PAGE], :, t % PAGE]
        assert np.array_equal(p, np.repeat(t[:, None], hkv, 1))


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads", [(4, 1, 64), (28, 4, 128)])
def test_a_loop_within_a_budget(heads, fp8):
    """Prompts, their window's weights, a cut to the budget, then steps that weigh and evict: lengths, positions,
    pages and every output against the oracle on the same decisions."""
    hq, hkv, d = heads
    g = hq // hkv
    prompts, budget, steps = np.array([70, 35, 9], np.int32), 32, 24
    c = Cache([0, 0, 0], hkv, d, fp8, 91, spare=14, stride_extra=6)
    _give_pages(c, [0, 0, 0], prompts)
    scale = 1.0 / np.sqrt(d)
    T = int(prompts.sum())
    kn, vn = new_tokens(T, hkv, d, 41)
    q = new_tokens(T, hq, d, 42)[0]
    lse = torch.empty((T, hq), device="cuda")
    extend = B.ExtendAttention(hq, hkv, d)
    extend(q.cuda(), c.g_k, c.g_v, c.g_bt, prompts, prompts, scale, lse=lse, k_new=kn.cuda(), v_new=vn.cuda(), fp8=c.g_fp8)
    if fp8:
        R.store_fp8(bits(kn).reshape(kn.shape), bits(vn).reshape(vn.shape), prompts, prompts, c.bt, c.k, c.v, c.ks, c.vs)
        c.same("prompts")
    else:
        kv_store(c.k, c.v, c.bt, prompts, prompts, bits(kn).reshape(kn.shape), bits(vn).reshape(vn.shape))
        c.same("prompts")
    # the loop's first "step" is the prompts' last rows
    cu = np.cumsum(prompts)
    last = torch.from_numpy(cu - 1)
    table_lens = prompts.copy()
    loop = B.DecodeLoopRunner(hq, hkv, d, c.g_k, c.g_v, c.g_bt, c.bt, table_lens, scale, fp8=c.g_fp8)
    w = torch.full((c.n, hkv, PAGE), float("nan"), device="cuda")
    pos = torch.full((c.n, hkv, PAGE), -1, dtype=torch.int32, device="cuda")
    l1 = torch.empty((3, hq), device="cuda")
    loop.step(q[last].cuda(), prompts, lse=l1)
    with pytest.raises(ValueError):
        loop.evict(budget, w, pos)
    loop.key_weights(q[last].cuda(), l1, w, pos)
    lens = loop.evict(budget, w, pos, sinks=2, recent=4)
    assert lens.tolist() == [32, 32, 9]

    def mirror():
        """The oracle's cache from the GPU's (the decisions were checked on their own)."""
        torch.cuda.synchronize()
        if fp8:
            c.k, c.v = c.g_k.cpu().numpy(), c.g_v.cpu().numpy()
            c.ks, c.vs = c.g_fp8[0].cpu().numpy(), c.g_fp8[1].cpu().numpy()
        else:
            c.k, c.v = bits(c.g_k).reshape(c.k.shape), bits(c.g_v).reshape(c.v.shape)
        c.bt = loop.bt_host

    def decide(before_w, before_p, lens_before, ends):
        """Kept positions of every pair by the oracle's rule."""
        kept = {}
        for s, L in enumerate(lens_before):
            t = np.arange(L)
            for h in range(hkv):
                m = R.kept_slots(before_w[s][h], before_p[s][h], min(L, budget), 2, 4, ends[s])
                kept[s, h] = sorted(before_p[s][h][m].tolist())
        return kept

    seen = prompts.astype(np.int64)
    for i in range(steps):
        lens = lens + 1
        kn, vn = new_tokens(3, hkv, d, 100 + i, "normal")
        q = new_tokens(3, hq, d, 200 + i)[0]
        out, l1 = torch.empty((3, hq, d), device="cuda"), torch.empty((3, hq), device="cuda")
        loop.step(q.cuda(), lens, kn.cuda(), vn.cuda(), out=out, lse=l1)
        seen += 1
        mirror()
        ro, rl, to, tl = reference(c, q, lens.tolist(), [1, 1, 1], scale, "append")
        slack = 0 if fp8 else 2.0 ** -12     # a bf16 step's newest token joins in fp32: well within the bound of the others
        check(out.cpu().numpy(), ro, to + slack * np.abs(ro), f"step {i} out")
        check(l1.cpu().numpy(), rl, tl + slack, f"step {i} lse")
        loop.key_weights(q.cuda(), l1, w, pos)
        torch.cuda.synchronize()
        hw, hp = w.cpu().numpy(), pos.cpu().numpy()
        at = [np.arange(L) for L in lens]
        before_w = [[hw[c.bt[s, t // PAGE], h, t % PAGE] for h in range(hkv)] for s, t in enumerate(at)]
        before_p = [[hp[c.bt[s, t // PAGE], h, t % PAGE] for h in range(hkv)] for s, t in enumerate(at)]
        for s in range(3):
            for h in range(hkv):
                assert before_p[s][h][-1] == seen[s] - 1 and len(set(before_p[s][h])) == lens[s]
                assert np.all(np.isfinite(before_w[s][h]))
        if i % 5 == 4:
            want = decide(before_w, before_p, lens, seen)
            lens = loop.evict(budget, w, pos, sinks=2, recent=4)
            assert np.all(lens <= budget)
            torch.cuda.synchronize()
            hp = pos.cpu().numpy()
            for s, L in enumerate(lens):
                t = np.arange(L)
                for h in range(hkv):
                    assert sorted(hp[loop.bt_host[s, t // PAGE], h, t % PAGE].tolist()) == want[s, h]
    held = [-(-int(L) // PAGE) for L in loop.table.prev]
    assert loop.pool.available() == c.n - sum(held)


@pytest.mark.parametrize("fp8", [False, True])
def test_loop_whose_sequences_end_and_start(fp8):
    """Rows of sequences that are not running are left out of the weights, and a sequence that starts in an ended
    one's place has none of its counts."""
    hq, hkv, d, scale = 8, 2, 64, 0.125
    prompts, budget = np.array([40, 24, 9], np.int64), 16
    c = Cache([64, 64, 64], hkv, d, fp8, 95)
    loop = B.DecodeLoopRunner(hq, hkv, d, c.g_k, c.g_v, c.g_bt, c.bt, prompts, scale, fp8=c.g_fp8)
    w = torch.full((c.n, hkv, PAGE), float("nan"), device="cuda")
    pos = torch.full((c.n, hkv, PAGE), -1, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()

    def step(lens, seed, weigh=True, stream=None):
        q = new_tokens(3, hq, d, seed)[0].cuda()
        kn, vn = (x.cuda() for x in new_tokens(3, hkv, d, seed + 1))
        l1 = torch.empty((3, hq), device="cuda")
        loop.step(q, np.asarray(lens), kn if loop.steps else None, vn if loop.steps else None, lse=l1)
        if not weigh:
            return
        before = w.clone()
        torch.cuda.synchronize()
        live = np.asarray(lens) > 0
        held = np.minimum(loop.weighed, lens)
        loop.key_weights(q, l1, w, pos, stream=stream)
        torch.cuda.synchronize()
        if live.any():
            rows = torch.from_numpy(np.flatnonzero(live)).cuda()
            loop.attn.key_weights(q[rows], l1[rows], c.g_k, c.g_bt, np.asarray(lens), live.astype(np.int32), scale, before,
                                  held_lens=held, first_pos=held + loop.evicted, k_scale=c.g_fp8[0] if fp8 else None)
        assert torch.equal(torch.isnan(w), torch.isnan(before)) and torch.equal(w.nan_to_num(), before.nan_to_num())

    step(prompts, 300)
    assert loop.evict(budget, w, pos).tolist() == [16, 16, 9]
    step([17, 0, 10], 310)                 # the second ends
    step([18, 0, 11], 320, stream=side)
    step([19, 1, 12], 330)                 # another starts in its place
    torch.cuda.synchronize()
    first = loop.bt_host[1, 0]
    assert pos[first, :, 0].tolist() == [0, 0] and loop.evicted.tolist() == [24, 0, 0]
    step([0, 0, 13], 340, weigh=False)
    step([1, 0, 14], 350)                  # no call between has weighed
    assert pos[loop.bt_host[0, 0], :, 0].tolist() == [0, 0] and loop.weighed.tolist() == [1, 0, 14]
    assert loop.evict(budget, w, pos).tolist() == [1, 0, 14]
    step([0, 0, 0], 360)
    assert loop.evicted.tolist() == [0, 0, 0] and loop.weighed.tolist() == [0, 0, 0]
