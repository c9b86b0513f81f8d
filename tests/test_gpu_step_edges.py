"""GPU tests of a group rollout's step at its edges. Tolerances as in tests/test_gpu_step.py."""
import math

import numpy as np
import pytest
import torch

from paper_2601_12784_amd import binding as B
from tests.test_gpu_step import Grouped, check_samples, cuda, randn

pytestmark = pytest.mark.gpu


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
