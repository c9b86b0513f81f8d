"""GPU tests of a group rollout's step at its edges. Tolerances as in tests/test_gpu_step.py."""
import numpy as np
import pytest
import torch

from paper_2601_12784_amd import binding as B
from tests.test_gpu_step import check_samples, cuda

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
