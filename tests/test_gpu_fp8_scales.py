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
from paper_2601_12784_amd import binding as B
from test_gpu_cache import Cache, bits, check, new_tokens, reference

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
