"""One DecodeAttention whose calls come on several streams: they share its workspace, so each waits on the device for
the ones before it. Every stream has a cache of its own; nothing is synchronized between the calls."""
import numpy as np
import pytest
import torch

from paper_2601_12784_amd import binding as B
from test_gpu_cache import PAGE, Cache, _give_pages, new_tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()
    yield
    torch.cuda.synchronize()


class Side:
    """A cache, its inputs and one round of calls: a step that appends, its weights, a prompt's weights, an eviction."""

    def __init__(self, i, fp8, heads):
        hq, hkv, d = heads
        self.rng = np.random.default_rng(i)
        self.lens = np.array([900 + 200 * i, 70, 600], np.int32)
        self.c = Cache(self.lens - 1, hkv, d, fp8, 200 + i, spare=3, stride_extra=1)
        _give_pages(self.c, self.lens - 1, self.lens)
        self.q, self.many = (new_tokens(n, hq, d, 60 + i)[0].cuda() for n in (3, 300))
        self.kn, self.vn = (x.cuda() for x in new_tokens(3, hkv, d, 70 + i))
        self.out, self.lse = torch.empty((3, hq, d), device="cuda"), torch.empty((3, hq), device="cuda")
        self.far = torch.full((300, hq), 9.0, device="cuda")
        shape = (self.c.n, hkv, PAGE)
        self.w = torch.from_numpy(self.rng.random(shape).astype(np.float32)).cuda()
        self.heavy = torch.zeros(shape, device="cuda")
        self.pos = torch.zeros(shape, dtype=torch.int32, device="cuda")
        self.left = torch.zeros(shape, dtype=torch.int32, device="cuda")

    def calls(self, attn, stream):
        c, append = self.c, (self.kn, self.vn, [-1, -1, -1])
        attn(self.q, c.g_k, c.g_v, c.g_bt, self.lens, 0.1, out=self.out, lse=self.lse, append=append, fp8=c.g_fp8, stream=stream)
        attn.key_weights(self.q, self.lse, c.g_k, c.g_bt, self.lens, [1, 1, 1], 0.1, self.w, positions=self.pos,
                         k_scale=c.g_fp8[0] if c.fp8 else None, stream=stream)
        # walks cut into parts, in the workspace
        attn.key_weights(self.many, self.far, c.g_k, c.g_bt, self.lens, [200, 50, 50], 0.1, self.heavy, held_lens=[0, 0, 0],
                         k_scale=c.g_fp8[0] if c.fp8 else None, stream=stream)
        keep = self.lens - [100, 7, 33]
        attn.evict(c.g_k, c.g_v, c.g_bt, self.lens, keep, self.w, self.pos, weights_out=self.heavy, positions_out=self.left,
                   recent=1, fp8=c.g_fp8, stream=stream)

    def results(self):
        c = self.c
        return [t.clone() for t in (c.g_k, c.g_v, *(c.g_fp8 or ()), self.out, self.lse, self.w, self.heavy, self.pos, self.left)]


@pytest.mark.parametrize("fp8", [False, True])
def test_calls_on_alternating_streams(fp8):
    heads, rounds = (28, 4, 128), 12
    want = []
    for i in range(3):
        side, attn = Side(i, fp8, heads), B.DecodeAttention(*heads)
        for _ in range(rounds):
            side.calls(attn, None)
            torch.cuda.synchronize()
        want.append(side.results())
    sides, attn = [Side(i, fp8, heads) for i in range(3)], B.DecodeAttention(*heads)
    streams = [torch.cuda.Stream() for _ in sides]
    torch.cuda.synchronize()
    for _ in range(rounds):
        for side, stream in zip(sides, streams):
            side.calls(attn, stream)
    torch.cuda.synchronize()
    for side, expected in zip(sides, want):
        for got, ref in zip(side.results(), expected):
            assert torch.equal(got.view(torch.uint8), ref.view(torch.uint8))


def test_a_step_follows_the_last_stream_once():
    """Back and forth between the current stream and another, with more steps than the ring has slots on each."""
    hq, hkv, d = heads = (8, 2, 64)
    lens = np.array([3000, 500], np.int32)
    c = Cache(lens, hkv, d, False, 220)
    q = [new_tokens(2, hq, d, 80 + i)[0].cuda() for i in range(2)]
    want = [B.DecodeAttention(*heads)(x, c.g_k, c.g_v, c.g_bt, lens, 0.1).clone() for x in q]
    attn, side, out = B.DecodeAttention(*heads), torch.cuda.Stream(), torch.empty((200, 2, hq, d), device="cuda")
    torch.cuda.synchronize()
    for i in range(200):
        stream = side if i % 7 < 3 or 60 < i < 100 else None
        attn(q[i % 2], c.g_k, c.g_v, c.g_bt, lens, 0.1, out=out[i], stream=stream)
    torch.cuda.synchronize()
    for i in range(200):
        assert torch.equal(out[i], want[i % 2])
