"""GPU tests of a group rollout's step at its edges. Tolerances as in tests/test_gpu_step.py and
tests/test_gpu_cache.py."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_ref
from paper_2601_12784_amd import binding as B
from tests.test_gpu_cache import Cache, bits, check, wide
from tests.test_gpu_step import U, Grouped, check_samples, check_turned, cuda, randn

pytestmark = pytest.mark.gpu
PAGE = 16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()
    yield
    torch.cuda.synchronize()


# ---------------------------------------------------------------------------
# sampling
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,block,chunks", [(96, 8192, 16), (96, 8192, 24), (96, 2048, 16), (64, 2048, 24)])
@pytest.mark.parametrize("cut", [False, True])
def test_draws_at_the_border_of_equal_chunks(rows, block, chunks, dtype, cut):
    """Rows of one near-flat block repeated, with u on the blocks' borders: the sums of up to 2^57 units are rounded
    as they are joined, and every row has a token all the same."""
    rng = np.random.default_rng(block + chunks)
    b, v = rows, block * chunks
    x = torch.from_numpy((0.3 * rng.standard_normal((b, block))).astype(np.float32)).to(dtype).repeat(1, chunks).cuda()
    u = cuda((1 + np.arange(b) % (chunks - 1)) / chunks, torch.float32)
    token = torch.full((b,), -7, dtype=torch.int32, device="cuda")
    logprob, kept = torch.full((b,), 7.0, device="cuda"), torch.full((b,), 7.0, device="cuda")
    params = dict(top_p=torch.ones(b, device="cuda")) if cut else {}
    B.Sampler()(x, u, token=token, logprob=logprob, kept=kept, **params)
    assert (token >= 0).all() and (token < v).all(), f"rows without a token: {torch.nonzero(token < 0)[:, 0].tolist()}"
    assert (logprob < 0).all() and (kept == 1).all()
    some = list(range(0, b, 16))
    check_samples(x[some], u[some], (token[some], logprob[some], kept[some]), **{k: t[some] for k, t in params.items()})


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("vocab", [4700, 9001, 50000])
@pytest.mark.parametrize("top_k", [0, 372, 4500])
def test_a_least_weight_above_the_other_cuts(top_k, vocab, dtype):
    """min-p is the strictest of three cuts of rows that a list does not hold: no token is lighter."""
    rng = np.random.default_rng(vocab + top_k)
    b = 64
    x = torch.from_numpy(rng.standard_normal((b, vocab)).astype(np.float32)).to(dtype).cuda()
    u = cuda(rng.random(b), torch.float32)
    for top_p in (0.9, 0.99, 1.0):
        params = dict(temperature=torch.full((b,), 3.0, device="cuda"), top_p=torch.full((b,), top_p, device="cuda"),
                      min_p=cuda(rng.choice([0.2, 0.5, 0.9, 1.0], b), torch.float32))
        if top_k:
            params["top_k"] = torch.full((b,), top_k, dtype=torch.int32, device="cuda")
        token, logprob, kept = B.Sampler()(x, u, **params)
        weight = torch.exp((x.double() - x.double().amax(1, keepdim=True)) / 3.0).gather(1, token.long()[:, None])[:, 0]
        assert (weight >= params["min_p"].double() * (1 - 2.0 ** -40)).all(), torch.nonzero(weight < params["min_p"])[:, 0].tolist()
        some = list(range(0, b, 9))
        check_samples(x[some], u[some], (token[some], logprob[some], kept[some]), **{k: t[some] for k, t in params.items()})


@pytest.mark.parametrize("vocab", [700, 9001, 50000])
@pytest.mark.parametrize("cuts", ["min_p", "top_p", "top_k", "all"])
def test_entries_a_hair_below_the_least_weight(vocab, cuts):
    """Logits within the margin of the bound that the groups are searched by: their own weights decide, on every way that a
    row takes."""
    rng = np.random.default_rng(vocab)
    b = 24
    edge = math.log(0.5)
    x = rng.uniform(-0.6, 0.0, (b, vocab)).astype(np.float32)
    below, at = rng.random((b, vocab)) < 0.4, rng.random((b, vocab)) < 0.1
    x[below] = (edge - rng.choice([1e-7, 2e-7, 4e-7, 1e-5], below.sum())).astype(np.float32)
    x[at] = (edge + rng.choice([6e-8, 1e-6], at.sum())).astype(np.float32)
    x[:, 5] = 0.0
    x, u = torch.from_numpy(x).cuda(), cuda(rng.random(b), torch.float32)
    params = dict(min_p=torch.full((b,), 0.5, device="cuda"))
    if cuts in ("top_p", "all"):
        params["top_p"] = cuda(rng.choice([0.9, 0.999], b), torch.float32)
    if cuts in ("top_k", "all"):
        params["top_k"] = torch.full((b,), vocab - 50, dtype=torch.int32, device="cuda")
    got = B.Sampler()(x, u, **params)
    check_samples(x, u, got, **params)
    if cuts == "min_p" and vocab == 9001:      # more rows than places: some go by one workgroup
        many = x.repeat(50, 1), u.repeat(50)
        more = B.Sampler()(*many, min_p=params["min_p"].repeat(50))
        assert all(torch.equal(t, g.repeat(50)) for t, g in zip(more, got))


# ---------------------------------------------------------------------------
# attention over shared prompts
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("hq,hkv,d", [(14, 2, 64), (14, 2, 128)])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("members", [2, 4, 10, 20])
def test_a_members_bits_are_its_own(members, fp8, hq, hkv, d):
    """Rows of several members share a wave. Whatever the others' queries hold, large ones whose references move at
    many blocks, NaN, infinities, or a place whose sequence has left: every bit of the rest stays."""
    prefix = 805
    lens = [prefix + 1 + 7 * s for s in range(members)]
    if members > 2:
        lens[2] = 0
    cache = Grouped(lens, [0, members], [prefix], hkv, d, fp8, seed=members)
    q = randn(np.random.default_rng(d), members, hq, d)
    attn = B.DecodeAttention(hq, hkv, d)
    others = [s for s in range(members) if s % 2 == 0]
    rest = [s for s in range(members) if s % 2]

    def run(q):
        lse = torch.empty(members, hq, device="cuda")
        return attn.shared(q, cache.g_k, cache.g_v, cache.g_bt, lens, [0, members], [prefix], 1.0 / math.sqrt(d), lse=lse, fp8=cache.g_fp8), lse

    out, lse = run(q)
    cache.check(q, out, lse, 1.0 / math.sqrt(d), hq)
    for what, value in (("large", q[others] * 40), ("nan", math.nan), ("inf", math.inf)):
        changed = q.clone()
        changed[others] = value
        got, got_lse = run(changed)
        assert torch.equal(got[rest], out[rest]) and torch.equal(got_lse[rest], lse[rest]), what


# ---------------------------------------------------------------------------
# tensors that a call makes
# ---------------------------------------------------------------------------
def stream_of(t):
    """The stream whose memory a tensor lies in."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not torch's memory")


def test_results_belong_to_the_stream_that_writes_them():
    """Memory of the current stream may still be read there by what came before: a call on another stream must not
    take its result from it."""
    cache = Grouped([200, 130, 161], [0, 3], [128], 2, 64, False, seed=5)
    table = torch.from_numpy(cache.bt).cuda()
    lens = np.array(cache.lens, np.int32)
    q, kv = randn(np.random.default_rng(0), 3, 8, 64), randn(np.random.default_rng(1), 3, 2, 64)
    attn, extend, side = B.DecodeAttention(8, 2, 64), B.ExtendAttention(8, 2, 64), torch.cuda.Stream()
    torch.cuda.synchronize()
    calls = dict(
        shared=lambda s: attn.shared(q, cache.g_k, cache.g_v, cache.g_bt, lens, [0, 3], [128], 0.1, stream=s),
        step=lambda s: attn(q, cache.g_k, cache.g_v, table, lens, 0.1, stream=s),
        append=lambda s: attn(q, cache.g_k, cache.g_v, table, lens, 0.1, stream=s, append=(kv, kv, np.full(3, -1, np.int32))),
        extend=lambda s: extend(q, cache.g_k, cache.g_v, table, lens, [1, 1, 1], 0.1, stream=s),
        extend_handle=lambda s: extend(q, cache.g_k, cache.g_v, table, lens, [1, 1, 1], 0.1, stream=s and s.cuda_stream),
    )
    for name, call in calls.items():
        out = call(side)
        side.synchronize()
        assert stream_of(out) == side.cuda_stream, name
        if name == "append":
            assert stream_of(attn._lse) == side.cuda_stream
        here = call(None)
        torch.cuda.synchronize()
        assert stream_of(here) == torch.cuda.current_stream().cuda_stream and torch.equal(here, out), name


def test_an_appending_steps_own_lse_outlives_a_larger_one():
    """The buffer that a larger batch replaces may still be written by a call on another stream."""
    attn = B.DecodeAttention(8, 2, 64)
    buffers = []
    for n in (1, 100):
        cache = Cache([20] * n, 2, 64, False, seed=5)
        q, kv = randn(np.random.default_rng(0), n, 8, 64), randn(np.random.default_rng(1), n, 2, 64)
        attn(q, cache.g_k, cache.g_v, cache.g_bt, np.full(n, 20, np.int32), 0.1, append=(kv, kv, np.full(n, -1, np.int32)))
        buffers.append(attn._lse.data_ptr())
        torch.cuda.synchronize()
    taken = [torch.empty(8 * 5 // 4 + 64, device="cuda") for _ in range(64)]
    assert buffers[0] not in [t.data_ptr() for t in taken]


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
def test_a_rotary_made_for_the_current_device_can_be_captured():
    """device="cuda" uploads the frequencies ahead, where the calls look for them."""
    q, at = randn(np.random.default_rng(0), 5, 4, 64), torch.arange(5, dtype=torch.int32, device="cuda")
    rotary = B.Rotary(64, device="cuda")
    got, stream, graph = torch.empty_like(q), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        rotary(q, None, at, q_out=got)
    for _ in range(3):
        q.copy_(randn(np.random.default_rng(1), 5, 4, 64))
        graph.replay()
        torch.cuda.synchronize()
        check_turned(got, q, range(5), rotary, "replay")
        assert torch.equal(got, rotary(q, None, at)[0])
    assert rotary.turns_on(torch.device("cuda")) is rotary.turns_on(q.device)


@pytest.mark.parametrize("d,turn", [(64, 64), (64, 32), (128, 128), (128, 96)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_storing_and_plain_turns_have_the_same_bits(d, turn, layout):
    """Pairs whose turn nearly cancels show every rounding of the products: both kernels have to make the same ones."""
    hq, hkv, t = 28, 4, 3200      # so many pages that a thread takes several heads
    rng = np.random.default_rng(d + turn)
    rotary = B.Rotary(d, rotary_dim=turn, layout=layout)
    first = int(rng.integers(0, 1 << 20))
    angle = (first + np.arange(t, dtype=np.float64))[:, None, None] * rotary.freq
    size = rng.uniform(0.5, 2.0, (t, hq + hkv, turn // 2))
    sign = rng.integers(0, 2, (t, hq + hkv, 1)).astype(bool)
    # (a, b) ~ (sin, cos): a cos - b sin is near 0; (cos, -sin): b cos + a sin is
    a, b = (np.where(sign, p, r) * size for p, r in ((np.sin(angle), np.cos(angle)), (np.cos(angle), -np.sin(angle))))
    x = rng.standard_normal((t, hq + hkv, d))
    if layout == "half":
        x[..., : turn // 2], x[..., turn // 2: turn] = a, b
    else:
        x[..., 0: turn: 2], x[..., 1: turn: 2] = a, b
    x = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda()
    q, k = x[:, :hq].contiguous(), x[:, hq:].contiguous()
    at = torch.arange(first, first + t, dtype=torch.int32, device="cuda")
    want = rotary(q, k, at)
    for some in (slice(0, 60), slice(t - 60, t)):
        check_turned(want[0][some], q[some], at[some].cpu().numpy(), rotary, "q")
        check_turned(want[1][some], k[some], at[some].cpu().numpy(), rotary, "k")
    cache = Cache([t], hkv, d, False, seed=1)
    got = B.DecodeAttention(hq, hkv, d).rotate_store(rotary, q, k, k, cache.g_k, cache.g_v, cache.g_bt, [t], [t], first_pos=[first])
    assert torch.equal(got, want[0])
    pages = cache.g_bt[0, : t // PAGE].long()
    stored = cache.g_k[pages].permute(0, 3, 1, 2, 4).reshape(t, hkv, d)
    assert torch.equal(stored, want[1])
    for n in (1, 17):        # few tokens: other shapes of the launch
        assert all(torch.equal(y[:n], z) for y, z in zip(want, rotary(q[:n].contiguous(), k[:n].contiguous(), at[:n].contiguous())))


def test_rotary_of_more_tokens_than_a_launch_has_tiles_of_four():
    """Beyond 2^24 tokens a workgroup takes sixteen of them: the same bits, to the last token."""
    t = (1 << 24) + 5
    rotary, q = B.Rotary(64, rotary_dim=32), torch.randn(t, 1, 64, device="cuda", dtype=torch.bfloat16)
    at = torch.arange(t, dtype=torch.int32, device="cuda")
    out = rotary(q, None, at)[0]
    for a in (0, 1 << 23, t - 1000):
        some = slice(a, a + 1000)
        assert torch.equal(out[some], rotary(q[some], None, at[some])[0])
    check_turned(out[-20:], q[-20:], range(t - 20, t), rotary, "q")


def test_debug_checks_accept_what_the_calls_allow(monkeypatch):
    """Entries of shared pages in the other members' rows stay unfilled: stores and steps do not read them."""
    monkeypatch.setattr(B, "DEBUG_CHECKS", True)
    for fp8 in (False, True):
        lens, offsets, shared = [50, 0, 49, 60, 20], [0, 4, 5], [48, 16]
        cache = Grouped(lens, offsets, shared, 2, 64, fp8, seed=3)
        attn = B.DecodeAttention(8, 2, 64)
        q, kv = randn(np.random.default_rng(0), 5, 8, 64), randn(np.random.default_rng(1), 5, 2, 64)
        page = int(cache.g_bt[2, 3])
        cache.g_bt[2, 3] = -1       # a page that the call opens
        fresh = np.array([-1, -1, page, -1, -1], np.int32)
        if fp8:
            attn.store_fp8(kv[:4], kv[:4], cache.g_k, cache.g_v, cache.g_fp8, cache.g_bt, lens, [1, 0, 1, 1, 1], new_pages=fresh)
        else:
            attn.rotate_store(B.Rotary(64), q, kv, kv, cache.g_k, cache.g_v, cache.g_bt, lens, new_pages=fresh)
        attn.shared(q, cache.g_k, cache.g_v, cache.g_bt, lens, offsets, shared, 0.1, fp8=cache.g_fp8)
        cache.g_bt[3, 0] = page
        with pytest.raises(ValueError, match="sequence 3 does not start with"):
            attn.shared(q, cache.g_k, cache.g_v, cache.g_bt, lens, offsets, shared, 0.1, fp8=cache.g_fp8)
        torch.cuda.synchronize()


# ---------------------------------------------------------------------------
# loops
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("fp8", [False, True])
def test_weights_of_a_loop_with_rotary_positions(fp8):
    """key_weights takes the step's queries as they came and weighs with the turned ones: against 64 bits, with an
    eviction, a sequence that ends, and rows of the running ones alone."""
    hq, hkv, d, g = 8, 2, 64, 4
    rng = np.random.default_rng(6)
    lens = np.array([40, 24, 9], np.int64)
    c = Cache([64, 64, 64], hkv, d, fp8, 95)
    rotary = B.Rotary(d, base=500.0, layout="interleaved")
    loop = B.DecodeLoopRunner(hq, hkv, d, c.g_k, c.g_v, c.g_bt, c.bt, lens, 0.125, fp8=c.g_fp8, rotary=rotary)
    w = torch.full((c.n, hkv, PAGE), float("nan"), device="cuda")
    pos = torch.full((c.n, hkv, PAGE), -1, dtype=torch.int32, device="cuda")
    for i in range(8):
        q, kn, vn = randn(rng, 3, hq, d), randn(rng, 3, hkv, d), randn(rng, 3, hkv, d)
        lse = torch.empty((3, hq), device="cuda")
        if i:
            lens = np.where(lens > 0, lens + 1, 0)
        if i == 5:
            lens[1] = 0
        loop.step(q, lens, *((kn, vn) if i else ()), lse=lse)
        at = np.maximum(lens - 1 + loop.evicted, 0).astype(np.int32)
        turned = rotary(q, None, torch.from_numpy(at).cuda())[0]
        check_turned(turned, q, at, rotary, "q")
        held, before = np.minimum(loop.weighed, lens), w.double().cpu().numpy()
        rows = torch.from_numpy(np.flatnonzero(lens)).cuda()
        given = (q[rows], lse[rows]) if i == 6 else (q, lse)
        loop.key_weights(*given, w, pos)
        torch.cuda.synchronize()
        k, ks = (c.g_k.cpu().numpy(), c.g_fp8[0].cpu().numpy()) if fp8 else (bits(c.g_k).reshape(c.k.shape), None)
        got, qw, lw = w.double().cpu().numpy(), wide(turned), lse.double().cpu().numpy()
        for s in np.flatnonzero(lens):
            n = int(lens[s])
            pages = loop.bt_host[s, : -(-n // PAGE)]
            for h in range(hkv):
                heads = slice(h * g, (h + 1) * g)
                keys = cache_ref.dense(k, ks, pages, h, n, d, False)
                u, size = cache_ref.key_weights(qw[s: s + 1, heads], lw[s: s + 1, heads], keys, 0.125, n - 1)
                t = np.arange(n)
                old = np.where(t < held[s], before[pages[t // PAGE], h, t % PAGE], 0.0)
                rel = 2 * (d + 8) * U * size + 4 * U * np.abs(lw[s, heads]).max() + 2.0 ** -21 + (g + 4) * U
                check(got[pages[t // PAGE], h, t % PAGE], old + u, rel * u + 2 * U * (old + u) + 1e-37, f"step {i}")
        if i == 3:
            lens = loop.evict(16, w, pos, sinks=2, recent=4).astype(np.int64)
            assert lens.tolist() == [16, 16, 12]


@pytest.mark.parametrize("hq,hkv,d", [(14, 2, 64), (28, 4, 128)])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("members,together", [(4, 2), (10, 4), (20, 8), (40, 8)])
def test_many_steps_of_a_prompts_walk(members, together, fp8, hq, hkv, d):
    """Prompts whose rows take two, four, eight and sixteen blocks, walked far enough that the ring of registers and that
    of LDS come round several times, with an odd number of pages and some own tokens."""
    prefix = 1205
    lens = [prefix + 1 + 11 * s % 60 for s in range(members)]
    cache = Grouped(lens, [0, members], [prefix], hkv, d, fp8, seed=members, spread=0.5 if fp8 else 0.0)
    opts = B.make_opts(num_cus=2)
    desc = B.make_desc(members, hq, hkv, d, cache.bt.shape[1], cache.n, 0.1)
    info, work = B.sf_shared_attn_plan(desc, lens, [0, members], [prefix], opts=opts, fp8=fp8)
    items = np.asarray(work[16 * info.num_workers: 16 * (info.num_workers + info.num_work)]).reshape(-1, 16)
    walks = items[items[:, 11] > 0]
    assert (walks[:, 11] == together).all() and ((walks[:, 6] - walks[:, 5] + 1) // 2 // (8 // together)).max() >= 9
    q = randn(np.random.default_rng(members), members, hq, d)
    lse = torch.empty(members, hq, device="cuda")
    out = B.DecodeAttention(hq, hkv, d, opts=opts).shared(q, cache.g_k, cache.g_v, cache.g_bt, lens, [0, members], [prefix], 0.1, lse=lse, fp8=cache.g_fp8)
    cache.check(q, out, lse, 0.1, hq)


@pytest.mark.parametrize("turned,grouped", [(True, True), (True, False), (False, True)])
def test_what_a_loop_over_fp8_pages_stores(turned, grouped):
    """Every step's keys and values, turned or as they came, of the running sequences alone, against the oracle's store:
    all codes and scales, bit for bit."""
    hq, hkv, d = 8, 2, 64
    rng = np.random.default_rng(8)
    prompts, members = [70, 33, 16], [3, 1, 4]
    lens, offsets = np.repeat(prompts, members).astype(np.int64), np.cumsum([0] + members)
    c = (Grouped(lens, offsets, prompts, hkv, d, True, seed=13, spare=40, stride_extra=3) if grouped else
         Cache(lens, hkv, d, True, seed=13, spare=40, stride_extra=3))
    rotary = B.Rotary(d, base=500.0) if turned else None
    c.g_bt = torch.from_numpy(c.bt.copy()).cuda()
    loop = B.DecodeLoopRunner(hq, hkv, d, c.g_k, c.g_v, c.g_bt, c.bt, lens, 0.2, fp8=c.g_fp8, rotary=rotary,
                              groups=(offsets, prompts) if grouped else None)
    b = lens.size
    for step in range(20):
        q, kn, vn = randn(rng, b, hq, d), randn(rng, b, hkv, d, mult=2.0 ** rng.integers(-3, 3)), randn(rng, b, hkv, d)
        if step:
            lens = np.where(lens > 0, lens + 1, 0)
        for s in {5: (1, 7), 9: (0, 2)}.get(step, ()):
            lens[s] = 0
        loop.step(q, lens, *((kn, vn) if step else ()))
        if step:
            at = np.maximum(lens - 1, 0)
            keys = kn if rotary is None else rotary(None, kn, torch.from_numpy(at.astype(np.int32)).cuda())[1]
            if turned:
                check_turned(keys, kn, at, rotary, "k")
            live = np.flatnonzero(lens)
            c.bt = loop.bt_host
            cache_ref.store_fp8(bits(keys).reshape(kn.shape)[live], bits(vn).reshape(vn.shape)[live], lens, (lens > 0).astype(int),
                                c.bt, c.k, c.v, c.ks, c.vs)
        torch.cuda.synchronize()
        c.same(f"step {step}", table=False)
