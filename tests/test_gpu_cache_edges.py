"""The bounded cache at the ends of its ranges, against oracle/cache_ref.py: launches of more than 2^31 threads, more calls
in a row than a runner's ring has slots, graphs replayed bit for bit, fp8 evictions in runs of pages."""
import numpy as np
import pytest
import torch

from oracle import cache_ref as R
from oracle import fp8_ref
from paper_2601_12784_amd import binding as B
from test_gpu_cache import PAGE, U, Cache, _give_pages, bits, check, make_weights, new_tokens, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()
    yield
    torch.cuda.synchronize()


def test_store_of_more_than_two_to_the_31_threads():
    """A token of 2^23 + 4096 sequences: every scale, and the tiles of the first, the middle and the last rows."""
    n, d = (1 << 23) + 4096, 64
    desc = B.make_desc(n, 1, 1, d, 1, n, 1.0)
    one = np.ones(n, np.int32)
    info, work = B.sf_kv_store_fp8_plan(desc, one, one)
    assert info.num_rows * 256 > 2 ** 31
    gen = torch.Generator(device="cuda").manual_seed(5)
    kn = torch.randn((n, 1, d), device="cuda", generator=gen, dtype=torch.float32).to(torch.bfloat16)
    vn = (kn.flip(0) * 0.5).contiguous()
    pools = [torch.full((n, 1, PAGE * d), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((n, 1), float("nan"), device="cuda") for _ in range(2)]
    table = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda").view(n, 1).contiguous()
    B.sf_kv_store_fp8(desc, info, None, torch.from_numpy(work).cuda(), kn, vn, None, *pools, *scales, table)
    torch.cuda.synchronize()
    for x, pool, scale, is_v in ((kn, pools[0], scales[0], False), (vn, pools[1], scales[1], True)):
        top = x.abs().amax(dim=2).float().cpu().numpy()
        assert top.min() > 0
        assert np.array_equal(scale.cpu().numpy()[::-1], np.maximum(top, np.float32(2.0 ** -100)) / np.float32(448))
        for rows in (range(40), range((1 << 23) - 40, (1 << 23) + 40), range(n - 40, n)):
            at = torch.tensor(rows, device="cuda")
            got, mine = pool[n - 1 - at].cpu().numpy(), fp8_ref.widen_bf16(bits(x[at]).reshape(len(rows), d))
            for i in range(len(rows)):
                full = np.zeros((PAGE, d), np.float32)
                full[0] = mine[i]
                want, _ = R.requantize(np.zeros((PAGE, d), np.uint8), np.float32(1), np.zeros(PAGE, bool), full, np.arange(PAGE) == 0)
                assert np.array_equal(R.tile_codes(got[i:i + 1], 0, 0, d, is_v), want)


# ---------------------------------------------------------------------------
# calls in a row
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("fp8", [False, True])
def test_seventy_weighed_steps_in_a_row(fp8):
    """More calls than the ring has slots, none waited for: the sums of all of them. Bound per call as in test_gpu_cache.py
    (score, lse, exp2, sum of g rows), and one rounding of the running total."""
    hq, hkv, d, steps = 28, 4, 128, 70
    g, lens, scale = hq // hkv, np.array([50, 33], np.int32), 0.09
    c = Cache(lens + steps, hkv, d, fp8, 121)
    attn, stream = B.DecodeAttention(hq, hkv, d), torch.cuda.Stream()
    q = new_tokens(2 * steps, hq, d, 90)[0]
    lse = torch.linspace(2.0, 4.0, 2 * steps * hq).view(2 * steps, hq)
    shape = (c.n, hkv, PAGE)
    w, pos = torch.full(shape, float("nan"), device="cuda"), torch.zeros(shape, dtype=torch.int32, device="cuda")
    gq, gl = q.cuda(), lse.cuda()
    stream.wait_stream(torch.cuda.current_stream())
    for i in range(steps):
        n = lens + i + 1
        attn.key_weights(gq[2 * i:2 * i + 2], gl[2 * i:2 * i + 2], c.g_k, c.g_bt, n, [1, 1], scale, w, positions=pos,
                         held_lens=n - 1 if i else [0, 0], k_scale=c.g_fp8[0] if fp8 else None, stream=stream)
    stream.synchronize()
    qd, ld = wide(q).reshape(steps, 2, hq, d), lse.double().numpy().reshape(steps, 2, hq)
    for s in range(2):
        L = int(lens[s]) + steps
        t = np.arange(L)
        for h in range(hkv):
            k, _ = c.dense(s, h, L)
            want, tol = np.zeros(L), np.zeros(L)
            for i in range(steps):
                n = int(lens[s]) + i + 1
                u, size = R.key_weights(qd[i, s:s + 1, h * g:(h + 1) * g], ld[i, s:s + 1, h * g:(h + 1) * g], k[:n], scale, n - 1)
                want[:n] += u
                tol[:n] += (2 * (d + 8) * U * size + 4 * U * 4 + 2.0 ** -21 + (g + 4) * U) * u + 2 * U * want[:n]
            check(w.cpu().numpy()[c.bt[s, t // PAGE], h, t % PAGE], want, tol, f"sequence {s}, head {h}")
        assert np.array_equal(pos.cpu().numpy()[c.bt[s, t // PAGE], :, t % PAGE], np.repeat(t[:, None], hkv, 1))


@pytest.mark.parametrize("fp8", [False, True])
def test_forty_evictions_in_a_row(fp8):
    """Each cuts what the one before left, none waited for: pools, weights and positions bit for bit."""
    hq, hkv, d = 4, 2, 64
    lens = np.array([1500, 700, 64], np.int64)
    c = Cache(lens, hkv, d, fp8, 123, spread=1.0)
    rng = np.random.default_rng(9)
    w = make_weights("random", (c.n, hkv, PAGE), rng)
    pos = rng.permutation(w.size).reshape(w.shape).astype(np.int32)
    gw, gp = torch.from_numpy(w.copy()).cuda(), torch.from_numpy(pos.copy()).cuda()
    attn, at = B.DecodeAttention(hq, hkv, d), lens.copy()
    for i in range(40):
        keep = np.maximum(at - [31, 1 + i % 17, i % 2], 5)
        attn.evict(c.g_k, c.g_v, c.g_bt, at, keep, gw, gp, ends=[w.size] * 3, fp8=c.g_fp8)
        R.evict(c.k, c.v, c.ks, c.vs, c.bt, at, keep, w, pos, w, pos, ends=[w.size] * 3)
        at = keep
    torch.cuda.synchronize()
    for s, n in enumerate(at):
        t = np.arange(n)
        page = c.bt[s, t // PAGE]
        assert np.array_equal(gw.cpu().numpy()[page, :, t % PAGE], w[page, :, t % PAGE])
        assert np.array_equal(gp.cpu().numpy()[page, :, t % PAGE], pos[page, :, t % PAGE])
        if fp8:
            full = c.bt[s, : n // PAGE]      # whole pages: a tile's scale and all of its codes
            assert np.array_equal(c.g_k.cpu().numpy()[full], c.k[full]) and np.array_equal(c.g_v.cpu().numpy()[full], c.v[full])
            for got, ref in zip(c.g_fp8, (c.ks, c.vs)):
                assert np.array_equal(got.cpu().numpy()[c.bt[s, : -(-n // PAGE)]], ref[c.bt[s, : -(-n // PAGE)]])
        else:
            assert np.array_equal(bits(c.g_k).reshape(c.k.shape)[page, :, :, t % PAGE], c.k[page, :, :, t % PAGE])
            assert np.array_equal(bits(c.g_v).reshape(c.v.shape)[page, :, :, t % PAGE], c.v[page, :, :, t % PAGE])


# ---------------------------------------------------------------------------
# graphs
# ---------------------------------------------------------------------------
def test_captured_calls_replay_bit_for_bit():
    """Store, extend (both outputs' types), weights and eviction captured by their plan forms: every replay has the eager call's
    bits, from outputs and workspaces that hold something else."""
    hq, hkv, d, lens, news, keep = 28, 4, 128, [300, 77, 500], [40, 77, 3], [150, 60, 499]
    held = [L - e for L, e in zip(lens, news)]
    c = Cache(held, hkv, d, True, 125, spare=20, stride_extra=15)
    _give_pages(c, held, lens)
    T = sum(news)
    kn, vn = (x.cuda() for x in new_tokens(T, hkv, d, 91, "mixed"))
    q = new_tokens(T, hq, d, 92)[0].cuda()
    start = [t.clone() for t in (c.g_k, c.g_v, *c.g_fp8)]
    outs = [torch.zeros((T, hq, d), device="cuda", dtype=t) for t in (torch.float32, torch.bfloat16)]
    lse = torch.zeros((T, hq), device="cuda")
    w = torch.zeros((c.n, hkv, PAGE), device="cuda")
    pos = torch.zeros((c.n, hkv, PAGE), dtype=torch.int32, device="cuda")
    desc = B.make_desc(3, hq, hkv, d, c.bt.shape[1], c.n, 0.01)
    store, extend = B.sf_kv_store_fp8_plan(desc, lens, news), B.sf_extend_attn_plan(desc, lens, news)
    weigh = B.sf_key_weights_plan(desc, lens, news, held_lens=[0, 0, 0])
    cut = B.sf_kv_evict_plan(desc, lens, keep, sinks=2, recent=8)
    work = [torch.from_numpy(x).cuda() for _, x in (store, extend, weigh, cut)]
    space = [torch.zeros(max(1, i.workspace_bytes), dtype=torch.uint8, device="cuda") for i, _ in (weigh, cut)]
    everything = (c.g_k, c.g_v, *c.g_fp8, *outs, lse, w, pos)

    def reset(fill):
        for t, s in zip(everything, start):
            t.copy_(s)
        for t in (*outs, lse, w, pos, *space):
            t.view(torch.uint8).fill_(fill)

    def calls():
        B.sf_kv_store_fp8(desc, store[0], None, work[0], kn, vn, None, c.g_k, c.g_v, *c.g_fp8, c.g_bt)
        for out in outs:
            B.sf_extend_attn_fp8(desc, extend[0], None, work[1], q, c.g_k, c.g_v, *c.g_fp8, c.g_bt, out, lse)
        B.sf_key_weights(desc, weigh[0], None, work[2], q, lse, c.g_k, c.g_bt, w, positions=pos, k_scale=c.g_fp8[0],
                         workspace=space[0])
        B.sf_kv_evict(desc, cut[0], None, work[3], c.g_k, c.g_v, c.g_bt, w, pos, fp8=c.g_fp8, workspace=space[1])

    def results():
        torch.cuda.synchronize()
        return [t.view(torch.uint8).clone() for t in everything]

    reset(0x40)
    calls()
    eager = results()
    for out in outs:
        assert torch.isfinite(out.float()).all() and out.float().abs().sum() > 0
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        calls()
    for run in (graph.replay, graph.replay, calls, graph.replay):
        reset(0x40)
        run()
        for i, (a, b) in enumerate(zip(results(), eager)):
            assert torch.equal(a, b), i


# ---------------------------------------------------------------------------
# evictions of many pages
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("heads,count,length", [((4, 1, 64), 40, 1000), ((28, 4, 128), 34, 990)])
@pytest.mark.parametrize("fp8", [False, True])
def test_evict_in_runs_of_pages(heads, count, length, fp8):
    """More than 2048 kept pages that take few tokens each: rows of four pages, budgets inside a run and a page and on their
    borders, tiles that take none, one, two and more tokens."""
    hq, hkv, d = heads
    lens = np.array([length + 7 * (i % 9) for i in range(count)])
    keep = np.array([L - (64, 16, 33, 1, 0, 47, 17)[i % 7] for i, L in enumerate(lens)])
    keep[::5] = keep[::5] // 64 * 64
    keep[1::5] = keep[1::5] // 16 * 16
    assert sum(-(-keep // PAGE)) > 2048 and (lens - keep).sum() < 4 * sum(-(-keep // PAGE))
    c = Cache(lens, hkv, d, fp8, 127, spread=1.5)
    rng = np.random.default_rng(10)
    w = make_weights("random", (c.n, hkv, PAGE), rng)
    w[rng.random(c.n) < 0.02] *= np.float32(1e-3)      # pages that lose most of their tokens
    pos = rng.permutation(w.size).reshape(w.shape).astype(np.int32)
    gw, gp = torch.from_numpy(w.copy()).cuda(), torch.from_numpy(pos.copy()).cuda()
    kw = dict(ends=[w.size] * count, sinks=1, recent=3)
    B.DecodeAttention(hq, hkv, d).evict(c.g_k, c.g_v, c.g_bt, lens, keep, gw, gp, fp8=c.g_fp8, **kw)
    # the oracle a sequence at a time, on that sequence's pages alone
    for s, L in enumerate(lens):
        pages = c.bt[s, : -(-L // PAGE)]
        part = [None if x is None else x[pages] for x in (c.k, c.v, c.ks, c.vs)]
        pw, pp = w[pages], pos[pages]
        R.evict(*part, np.arange(len(pages))[None, :], [L], keep[s:s + 1], pw, pp, pw, pp, ends=[w.size], sinks=1, recent=3)
        for x, y in zip((c.k, c.v, c.ks, c.vs, w, pos), (*part, pw, pp)):
            if x is not None:
                x[pages] = y
    c.same("evict")
    assert np.array_equal(gw.cpu().numpy(), w) and np.array_equal(gp.cpu().numpy(), pos)
