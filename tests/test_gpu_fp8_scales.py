"""Attention over an fp8 cache whose pages have unlike value scales, against oracle/cache_ref.py in 64 bits.

A page of zero values has scale 1 by the store's rule, whatever the other pages hold; a channel that is large in one page sets
that page's scale. In the outputs below such a page has no part (its codes are zero there), so what the other pages'
products keep is what is tested, whatever the ratio of the scales.

Bounds, u = 2^-24, as in test_gpu_cache.py (scores, lse, sums) and
  an appending step: its weights times the page's scale enter P.V exactly but for the product's own rounding, u: 2^-23 with
    the division's; held here to 2^-20 of sum_t p_t |V_t| / sum_t p_t;
  a plain step: two bf16 parts, 2^-16 of it.
"""
import numpy as np
import pytest
import torch

from oracle import cache_ref as R
from oracle import fp8_ref
from paper_2601_12784_amd import binding as B
from test_gpu_cache import Cache, _give_pages, bits, check, new_tokens, reference, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()
    yield
    torch.cuda.synchronize()


def unlike(c, lens, kind, size):
    """Rewrites the values of the cache's held pages, on both sides: times 2^size, and by kind
    zero: every sequence's second page (or its only one) is all zeros, scale 1;
    channel: the first page has values in dim 0 alone, 2^40 times as large;
    late: the same of the last page but one."""
    for s, L in enumerate(lens):
        pages = c.bt[s, : -(-L // 16)]
        c.vs[pages] *= np.float32(2.0 ** size)
        if L < 2:
            continue
        for h in range(c.hkv):
            if kind == "zero":
                p = pages[min(1, len(pages) - 1)]
                R.put_tile_codes(c.v, p, h, c.d, True, np.zeros((16, c.d), np.uint8))
                c.vs[p, h] = 1
            else:
                p = pages[0 if kind == "channel" else max(0, len(pages) - 2)]
                codes = R.tile_codes(c.v, p, h, c.d, True)
                codes[:, 1:] = 0
                R.put_tile_codes(c.v, p, h, c.d, True, codes)
                c.vs[p, h] *= np.float32(2.0 ** 40)
    c.g_v.copy_(torch.from_numpy(c.v))
    c.g_fp8[1].copy_(torch.from_numpy(c.vs))


@pytest.mark.parametrize("heads", [(4, 1, 64), (28, 4, 128)])
@pytest.mark.parametrize("kind,size", [("zero", 0), ("zero", -4), ("zero", -10), ("zero", -30), ("zero", 30), ("channel", 0),
                                       ("channel", -40), ("late", 0), ("spread", 0)])
@pytest.mark.parametrize("lens", [[3000, 40], [70, 33, 17, 400, 2]])   # cut walks, and short ones
def test_append_step_over_unlike_scales(heads, kind, size, lens):
    hq, hkv, d = heads
    held = [L - 1 for L in lens]
    c = Cache(held, hkv, d, True, 101 + d, spare=len(lens) + 2, stride_extra=1, spread=5.0 if kind == "spread" else 0.5)
    if kind != "spread":
        unlike(c, held, kind, size)
    pages = np.full(len(lens), -1, np.int32)
    for s, L in enumerate(lens):
        if (L - 1) % 16 == 0:
            pages[s], c.free = c.free[0], c.free[1:]
    kn, vn = new_tokens(len(lens), hkv, d, 50)
    vn = (vn.float() * 2.0 ** size).to(torch.bfloat16)
    q = new_tokens(len(lens), hq, d, 51)[0]
    out, lse = torch.empty((len(lens), hq, d), device="cuda"), torch.empty((len(lens), hq), device="cuda")
    attn, scale = B.DecodeAttention(hq, hkv, d), 1.0 / np.sqrt(d)
    attn(q.cuda(), c.g_k, c.g_v, c.g_bt, lens, scale, out=out, lse=lse, append=(kn.cuda(), vn.cuda(), pages), fp8=c.g_fp8)
    news = [1] * len(lens)
    R.store_fp8(bits(kn).reshape(kn.shape), bits(vn).reshape(vn.shape), lens, news, c.bt, c.k, c.v, c.ks, c.vs, pages)
    c.same("append")
    want, wl, tol, tl = reference(c, q, lens, news, scale, "fine")
    check(out.cpu().numpy(), want, tol, "appending step")
    check(lse.cpu().numpy(), wl, tl, "lse")
    plain = attn(q.cuda(), c.g_k, c.g_v, c.g_bt, lens, scale, fp8=c.g_fp8)
    check(plain.cpu().numpy(), want, reference(c, q, lens, news, scale, "append")[2], "plain step")


@pytest.mark.parametrize("heads", [(4, 1, 64), (28, 4, 128)])
@pytest.mark.parametrize("lens,news", [([900, 60], [70, 60]), ([6000], [40])])   # whole walks, and walks cut into parts
@pytest.mark.parametrize("lift,small", [(0, 9), (13, 9), (20, 0), (-6, 5)])
def test_extend_bound_over_unlike_scales(heads, lens, news, lift, small):
    """The header's bound, with each of its terms the largest somewhere: the first page's value scale is 2^lift times the
    others' (lift > 0: for dim 0, its only one), and half of every tile's dims are 2^-small of the others. p_t = exp(z_t - max z), P its sum, S the
    largest value scale: 2^-10 sum p|V| / P + 2^-24 S + 2^-25 sum |V| / P, and fp32's part as in test_gpu_cache.py."""
    hq, hkv, d = heads
    g = hq // hkv
    held = [L - e for L, e in zip(lens, news)]
    c = Cache(held, hkv, d, True, 111 + d, spare=20, stride_extra=8, spread=0.5, k_mult=2.0)
    for s, L in enumerate(held):
        for p in c.bt[s, : -(-L // 16)]:
            for h in range(hkv):
                codes = R.tile_codes(c.v, p, h, d, True)
                value = fp8_ref.values()[codes[:, d // 2:]] * 2.0 ** -small
                codes[:, d // 2:] = fp8_ref.encode(np.where(np.isnan(value), 0, value).astype(np.float32))
                if lift > 0 and p == c.bt[s, 0]:
                    codes[:, 1:] = 0
                R.put_tile_codes(c.v, p, h, d, True, codes)
        if L:
            c.vs[c.bt[s, 0]] *= np.float32(2.0 ** lift)
    c.g_v.copy_(torch.from_numpy(c.v))
    c.g_fp8[1].copy_(torch.from_numpy(c.vs))
    _give_pages(c, held, lens)
    T, scale = sum(news), 1.0 / np.sqrt(d)
    kn, vn = new_tokens(T, hkv, d, 52)
    q = new_tokens(T, hq, d, 53)[0]
    out = torch.empty((T, hq, d), device="cuda")
    B.ExtendAttention(hq, hkv, d)(q.cuda(), c.g_k, c.g_v, c.g_bt, lens, news, scale, out=out, k_new=kn.cuda(), v_new=vn.cuda(),
                                  fp8=c.g_fp8)
    R.store_fp8(bits(kn).reshape(kn.shape), bits(vn).reshape(vn.shape), lens, news, c.bt, c.k, c.v, c.ks, c.vs)
    c.same("extend")
    want, _, tol, _ = reference(c, q, lens, news, scale, "extend")
    print("of the first term alone:", float((np.abs(out.cpu().numpy() - want) / tol).max()))
    qd, row = wide(q), 0
    for s, (L, e) in enumerate(zip(lens, news)):
        largest = float(c.vs[c.bt[s, : -(-L // 16)]].max())
        for h in range(hkv):
            k, v = c.dense(s, h, L)
            z = scale * np.einsum("egd,td->egt", qd[row:row + e, h * g:(h + 1) * g], k)
            seen = np.arange(L)[None, :] <= L - e + np.arange(e)[:, None]
            z = np.where(seen[:, None, :], z, -np.inf)
            total = np.exp(z - z.max(axis=2, keepdims=True)).sum(axis=2)
            every = np.einsum("et,td->ed", seen.astype(float), np.abs(v))
            tol[row:row + e, h * g:(h + 1) * g] += 2.0 ** -24 * largest + 2.0 ** -25 * every[:, None, :] / total[..., None]
        row += e
    check(out.cpu().numpy(), want, tol, "extend")
