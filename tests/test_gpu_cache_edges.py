"""The bounded cache at the ends of its ranges, against oracle/cache_ref.py: launches of more than 2^31 threads."""
import numpy as np
import pytest
import torch

from oracle import cache_ref as R
from oracle import fp8_ref
from paper_2601_12784_amd import binding as B
from test_gpu_cache import PAGE, bits

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
