"""The calls around a group rollout's decode step (rotary positions, attention over a shared prompt, sampling), with
their plain forms, work and 64-bit results.

Several trajectories are sampled from every prompt, and one step of all of them runs, per GPU:
  rotate   queries and new keys are turned by their positions (and nothing is stored);
  store    the same, with the turned keys and the values written into the pages of a bf16 cache: one new token per
           trajectory in a decode step, all tokens of prompts before it;
  shared   one query per trajectory attends over its cached tokens, where the trajectories of a group have their first
           tokens in the same pages (their block tables start with the same entries);
  sample   one token per trajectory is drawn from its logits by a given uniform number, with temperature, top-k, top-p
           and min-p, and its log-probability is kept for training.
Head layouts and length distributions are those of the workloads in paper_2601_12784_amd/workloads.py, vocabularies
are generic. Every tensor is drawn on the GPU from the seed; lengths follow from the case alone.

Rotation: pair i of a head's first `turn` dims, i < turn/2, is (x[i], x[i + turn/2]) in the half layout and
(x[2i], x[2i+1]) in the interleaved one. At position t it becomes (a cos - b sin, b cos + a sin) * magnitude of the angle
t f_i, f_i = base^(-2i/turn). Scaled by a factor F for contexts longer than n tokens: with r = n f_i / (2 pi) turns in
n tokens and s = clamp((r - low) / (high - low), 0, 1), f_i is s f_i + (1 - s) f_i / F.

Sampling: w_v = exp((l_v - max l) / T). In the order of falling logits (equal ones: of rising index) the first k stay,
of these every one before which less than top_p of their sum lies, of these the ones with w >= min_p. The token is the
first index at which the running sum of the weights that stayed, in index order, exceeds u times their sum. T = 0 takes
the largest logit. logprob = ln(w / sum of all w) (T = 0: as T = 1); kept = what stayed of the sum of all w.
"""
import math

import numpy as np
import torch

own = False
PAGE = 16
DEV = "cuda"
HEADS = {"4/1x64": (4, 1, 64), "14/2x64": (14, 2, 64), "8/8x64": (8, 8, 64), "28/4x128": (28, 4, 128),
         "32/8x128": (32, 8, 128), "40/8x128": (40, 8, 128), "16/1x128": (16, 1, 128)}
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # four samples of one short prompt on a small model: latency of a step's attention
        dict(name="shared_tiny", kind="shared", heads="4/1x64", groups=1, members=4, prefix=300, median=40, longest=64,
             fp8=False, lens_seed=1),
        # 16 prompts of 2048 tokens with 16 samples each, whose own lengths are long-tailed
        dict(name="shared_groups", kind="shared", heads="28/4x128", groups=16, members=16, prefix=2048, median=512,
             longest=4096, fp8=False, lens_seed=2),
        # 64 samples go on from one long context (a document, an agent's history)
        dict(name="shared_long", kind="shared", heads="32/8x128", groups=1, members=64, prefix=32760, median=300,
             longest=1024, fp8=False, lens_seed=3),
        # instructions that a whole batch starts with
        dict(name="shared_system", kind="shared", heads="28/4x128", groups=1, members=256, prefix=4000, median=1000,
             longest=8192, fp8=False, lens_seed=4),
        # 8 prompts with 8 samples each over an fp8 cache
        dict(name="shared_fp8", kind="shared", heads="40/8x128", groups=8, members=8, prefix=8000, median=1000,
             longest=4096, fp8=True, lens_seed=5),
        # one step's new tokens of 512 trajectories into their pages
        dict(name="store_step", kind="store", heads="28/4x128", turn=128, layout="half", base=1000000.0, factor=1.0,
             batch=512, median=4096, longest=32768, new=1, gap=0, lens_seed=6),
        # prompts written whole, turned for contexts four times as long as the model was trained on
        dict(name="store_prompts", kind="store", heads="28/4x128", turn=128, layout="half", base=10000.0, factor=4.0,
             batch=32, median=2048, longest=16384, new=0, gap=0, lens_seed=7),
        # four tokens of a small model whose heads are turned in part
        dict(name="rotate_tiny", kind="rotate", heads="8/8x64", turn=32, layout="interleaved", base=10000.0, factor=1.0,
             rows=4, far=5000, packed=True),
        # a chunk of prompts in one projection's packed output, at far positions
        dict(name="rotate_chunk", kind="rotate", heads="32/8x128", turn=128, layout="interleaved", base=500000.0,
             factor=8.0, rows=8192, far=131072, packed=True),
        # one sequence of a small vocabulary: latency
        dict(name="sample_one", kind="sample", rows=1, vocab=32000, dtype="fp32", cut="nucleus"),
        # a rollout's step: the plain distribution, as the policy gradient wants it
        dict(name="sample_rollout", kind="sample", rows=256, vocab=131072, dtype="bf16", cut="none"),
        # an evaluation's or a service's step: every request with its own temperature and cuts
        dict(name="sample_served", kind="sample", rows=192, vocab=200003, dtype="fp32", cut="mixed"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["shared", "shared", "store", "rotate", "sample", "sample"])
    c = dict(kind=kind)
    if kind == "sample":
        c.update(rows=_log_int(rng, 1, 512), vocab=_log_int(rng, 1000, 262144), dtype=rng.choice(sorted(DTYPES)),
                 cut=rng.choice(["none", "nucleus", "mixed"]))
    else:
        c["heads"] = rng.choice(sorted(HEADS) + ["28/4x128", "40/8x128"])
        c["lens_seed"] = rng.randint(0, 1 << 30)
    if kind == "shared":
        c.update(groups=_log_int(rng, 1, 32), members=_log_int(rng, 2, 64), prefix=_log_int(rng, 16, 32768),
                 median=_log_int(rng, 4, 2048), fp8=rng.random() < 0.4)
        c["longest"] = 8 * c["median"]
    if kind in ("store", "rotate"):
        d = HEADS[c["heads"]][2]
        c.update(turn=rng.choice([d, d, d // 2, d // 4]), layout=rng.choice(["half", "interleaved"]),
                 base=rng.choice([10000.0, 500000.0, 1000000.0]), factor=rng.choice([1.0, 4.0, 8.0]))
    if kind == "rotate":
        c.update(rows=_log_int(rng, 1, 16384), far=_log_int(rng, 100, 1 << 20), packed=rng.random() < 0.7)
    if kind == "store":
        c.update(batch=_log_int(rng, 1, 512), median=_log_int(rng, 16, 8192), new=rng.choice([0, 1, _log_int(rng, 1, 2048)]),
                 gap=rng.choice([0, 0, 5000]))
        c["longest"] = 8 * c["median"]
    most = {k: max((work(x) for x in listed() if x["kind"] == kind), key=lambda w: w[k])[k] for k in ("bytes", "flops")}
    while any(work(c)[k] > most[k] for k in most):
        for k in ("groups", "members", "prefix", "batch", "median", "rows"):
            if k in c:
                c[k] = max(1, c[k] * 4 // 5)
        if "longest" in c:
            c["longest"] = 8 * c["median"]
    return c


# --------------------------------------------------------------------------
# lengths, pages and inputs
# --------------------------------------------------------------------------
def _lognormal(c, n):
    rng = np.random.default_rng(c["lens_seed"])
    return np.clip(np.rint(np.exp(math.log(c["median"]) + rng.standard_normal(n))), 1, c["longest"]).astype(np.int32)


def _lengths(c):
    """Cached tokens per sequence, from the case alone: the new ones among them (store), the prompt's too (shared)."""
    if c["kind"] == "shared":
        return c["prefix"] + _lognormal(c, c["groups"] * c["members"])
    return _lognormal(c, c["batch"])


def _new_lengths(c, lens):
    return lens.copy() if c["new"] == 0 else np.minimum(lens, c["new"]).astype(np.int32)


def _normal(g, shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV, dtype=dtype)


def _codes(g, shape):
    """E4M3 codes of normal values quantized with their largest magnitude near 448."""
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16).mul_(100.0).clamp_(-448.0, 448.0)
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def prepare(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    rng = np.random.default_rng(seed)
    return {"shared": _prepare_shared, "store": _prepare_store, "rotate": _prepare_rotate, "sample": _prepare_sample}[c["kind"]](c, g, rng)


def _prepare_shared(c, g, rng):
    hq, hkv, d = HEADS[c["heads"]]
    lens = _lengths(c)
    # whole pages of a prompt are shared; its last, begun one was copied for every member
    common = c["prefix"] // PAGE
    pages = (lens.astype(np.int64) + PAGE - 1) // PAGE
    n = int((pages - common).sum()) + c["groups"] * common
    ids, at = rng.permutation(n).astype(np.int32), 0
    bt = np.full((lens.size, int(pages.max())), -1, dtype=np.int32)
    for i in range(c["groups"]):
        first = i * c["members"]
        bt[first:first + c["members"], :common] = ids[at:at + common]
        at += common
        for s in range(first, first + c["members"]):
            bt[s, common:pages[s]] = ids[at:at + pages[s] - common]
            at += int(pages[s]) - common
    s = dict(c=c, lens=lens, scale=1.0 / math.sqrt(d), bt=torch.from_numpy(bt).to(DEV))
    s["groups"] = np.arange(c["groups"] + 1, dtype=np.int32) * c["members"]
    s["prefix"] = np.full(c["groups"], c["prefix"], dtype=np.int32)
    if c["fp8"]:
        s["kp"], s["vp"] = _codes(g, (n, hkv, PAGE * d)), _codes(g, (n, hkv, PAGE * d))
        s["ks"] = torch.rand((n, hkv), generator=g, device=DEV).mul_(0.004).add_(0.005)
        s["vs"] = torch.rand((n, hkv), generator=g, device=DEV).mul_(0.004).add_(0.005)
    else:
        s["kp"], s["vp"] = _normal(g, (n, hkv, d // 8, PAGE, 8)), _normal(g, (n, hkv, d, PAGE))
        if common < -(-c["prefix"] // PAGE):   # the copies hold what they were copied from
            for i in range(c["groups"]):
                page = bt[i * c["members"]:(i + 1) * c["members"], common].astype(np.int64)
                rest = c["prefix"] % PAGE
                s["kp"][page[1:], :, :, :rest] = s["kp"][page[0], :, :, :rest]
                s["vp"][page[1:], :, :, :rest] = s["vp"][page[0], :, :, :rest]
    s["q"] = _normal(g, (lens.size, hq, d))
    # the projection behind a step's attention takes bf16
    s["out"] = torch.empty((lens.size, hq, d), dtype=torch.bfloat16, device=DEV)
    s["lse"] = torch.empty((lens.size, hq), dtype=torch.float32, device=DEV)
    return s


def _rotation(c):
    """Scaling of a case's frequencies: (factor, trained length, low, high, magnitude)."""
    return (c["factor"], 4096.0, 1.0, 32.0, 0.1 * math.log(c["factor"]) + 1.0)


def _prepare_rotate(c, g, rng):
    hq, hkv, d = HEADS[c["heads"]]
    t = c["rows"]
    s = dict(c=c, positions=torch.randint(0, c["far"], (t,), generator=g, device=DEV, dtype=torch.int32))
    x = _normal(g, (t, (hq + 2 * hkv) * d if c["packed"] else (hq + hkv) * d))
    if c["packed"]:   # views into the output of one projection to queries, keys and values
        s["q"], s["k"] = x[:, :hq * d].view(t, hq, d), x[:, hq * d:(hq + hkv) * d].view(t, hkv, d)
    else:
        s["q"], s["k"] = x[:, :hq * d].reshape(t, hq, d).contiguous(), x[:, hq * d:].reshape(t, hkv, d).contiguous()
    s["q_out"] = torch.empty((t, hq, d), dtype=torch.bfloat16, device=DEV)
    s["k_out"] = torch.empty((t, hkv, d), dtype=torch.bfloat16, device=DEV)
    return s


def _prepare_store(c, g, rng):
    hq, hkv, d = HEADS[c["heads"]]
    lens = _lengths(c)
    new = _new_lengths(c, lens)
    pages = (lens.astype(np.int64) + PAGE - 1) // PAGE
    n, t = int(pages.sum()), int(new.sum())
    bt = np.full((lens.size, int(pages.max())), -1, dtype=np.int32)
    bt[np.arange(bt.shape[1])[None, :] < pages[:, None]] = rng.permutation(n)
    # the newest token's page is new in this step where the token opens one
    opens = ((lens - 1) % PAGE == 0) & (new == 1)
    at = (lens - 1) // PAGE
    fresh = np.where(opens, bt[np.arange(lens.size), at], -1).astype(np.int32)
    bt[np.nonzero(opens)[0], at[opens]] = -1
    s = dict(c=c, lens=lens, new=new, fresh=fresh, bt=torch.from_numpy(bt).to(DEV))
    # a cache that gave up tokens goes on at its next position
    s["first"] = (lens - new + c["gap"]).astype(np.int32)
    s["q"], s["kn"], s["vn"] = _normal(g, (t, hq, d)), _normal(g, (t, hkv, d)), _normal(g, (t, hkv, d))
    s["kp"], s["vp"] = _normal(g, (n, hkv, d // 8, PAGE, 8)), _normal(g, (n, hkv, d, PAGE))
    s["q_out"] = torch.empty((t, hq, d), dtype=torch.bfloat16, device=DEV)
    return s


def _prepare_sample(c, g, rng):
    b, v = c["rows"], c["vocab"]
    x = _normal(g, (b, v), torch.float32).mul_(2.2)
    # a few tokens stand out, by more in rows whose next token is nearly certain
    peak = torch.rand((b, 1), generator=g, device=DEV).mul_(14.0)
    at = torch.randint(0, v, (b, 24), generator=g, device=DEV)
    x.scatter_add_(1, at, torch.rand((b, 24), generator=g, device=DEV) * peak)
    if c["cut"] == "mixed":   # constrained rows: a grammar forbids most tokens
        banned = torch.rand((b, v), generator=g, device=DEV) < 0.9
        banned &= torch.rand((b, 1), generator=g, device=DEV) < 0.1
        x.masked_fill_(banned, -math.inf)
    s = dict(c=c, logits=x.to(DTYPES[c["dtype"]]), u=torch.rand((b,), generator=g, device=DEV))
    if c["cut"] == "none":
        return s
    f = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)  # noqa: E731
    s["temperature"] = f(rng.uniform(0.6, 1.2, b).astype(np.float32))
    s["top_p"] = f(rng.choice([0.8, 0.9, 0.95, 0.99], b).astype(np.float32))
    if c["cut"] == "mixed":
        s["temperature"][f(rng.random(b) < 0.1)] = 0.0
        s["top_p"][f(rng.random(b) < 0.3)] = 1.0
        s["top_k"] = f(np.where(rng.random(b) < 0.5, 0, np.exp(rng.uniform(0, math.log(min(v, 2000)), b))).astype(np.int32))
        s["min_p"] = f(np.where(rng.random(b) < 0.6, 0.0, rng.choice([0.01, 0.05, 0.1], b)).astype(np.float32))
    return s


# --------------------------------------------------------------------------
# the calls
# --------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2601_12784_amd import binding as B

    c = s["c"]
    if c["kind"] == "sample":
        if "call" not in s:   # the object that a program keeps
            s["call"] = B.Sampler(DEV)
        token, logprob, kept = s["call"](s["logits"], s["u"], temperature=s.get("temperature"), top_k=s.get("top_k"),
                                         top_p=s.get("top_p"), min_p=s.get("min_p"))
        return dict(token=token, logprob=logprob, kept=kept)
    hq, hkv, d = HEADS[c["heads"]]
    if c["kind"] == "shared":
        if "call" not in s:
            s["call"] = B.DecodeAttention(hq, hkv, d)
        s["call"].shared(s["q"], s["kp"], s["vp"], s["bt"], s["lens"], s["groups"], s["prefix"], s["scale"], out=s["out"],
                         lse=s["lse"], fp8=(s["ks"], s["vs"]) if c["fp8"] else None)
        return dict(out=s["out"], lse=s["lse"])
    if "rotary" not in s:
        factor, trained, low, high, magnitude = _rotation(c)
        scaling = dict(factor=factor, original=trained, low=low, high=high, magnitude=magnitude) if factor != 1.0 else None
        s["rotary"] = B.Rotary(d, rotary_dim=c["turn"], base=c["base"], layout=c["layout"], scaling=scaling)
    if c["kind"] == "rotate":
        s["rotary"](s["q"], s["k"], s["positions"], q_out=s["q_out"], k_out=s["k_out"])
        return dict(q=s["q_out"], k=s["k_out"])
    if "call" not in s:
        s["call"] = B.DecodeAttention(hq, hkv, d)
    s["call"].rotate_store(s["rotary"], s["q"], s["kn"], s["vn"], s["kp"], s["vp"], s["bt"], s["lens"], s["new"],
                           first_pos=s["first"], new_pages=s["fresh"], q_out=s["q_out"])
    return dict(q=s["q_out"], kp=s["kp"], vp=s["vp"], bt=s["bt"])


# --------------------------------------------------------------------------
# plain forms
# --------------------------------------------------------------------------
def _plain(s):
    return {"shared": _plain_shared, "store": _plain_store, "rotate": _plain_rotate, "sample": _plain_sample}[s["c"]["kind"]](s)


def _cached(s, pages):
    """Keys and values of pages, each [Hkv, tokens, D] in fp32."""
    hq, hkv, d = HEADS[s["c"]["heads"]]
    k, v = s["kp"][pages], s["vp"][pages]
    n = k.shape[0]
    if "ks" in s:
        k = k.view(torch.float8_e4m3fn).float() * s["ks"][pages][:, :, None]
        v = v.view(torch.float8_e4m3fn).float() * s["vs"][pages][:, :, None]
        k = k.view(n, hkv, d // 64, 4, PAGE, 2, 8).permute(1, 0, 4, 2, 5, 3, 6)
        v = v.view(n, hkv, d // 64, 4, 16, 4, 4).permute(1, 0, 3, 6, 2, 5, 4)
        return k.reshape(hkv, -1, d), v.reshape(hkv, -1, d)
    k, v = k.float().permute(1, 0, 3, 2, 4), v.float().permute(1, 0, 3, 2)
    return k.reshape(hkv, -1, d), v.reshape(hkv, -1, d)


def _plain_shared(s):
    """Every sequence by itself, over its whole block-table row."""
    hq, hkv, d = HEADS[s["c"]["heads"]]
    for i, n in enumerate(s["lens"].tolist()):
        k, v = _cached(s, s["bt"][i, : -(-n // PAGE)].long())
        q = s["q"][i].float().view(hkv, hq // hkv, d)
        z = (q @ k[:, :n].transpose(1, 2).contiguous()).mul_(s["scale"])
        top = z.amax(2, keepdim=True)
        p = z.sub_(top).exp_()
        total = p.sum(2, keepdim=True)
        s["lse"][i] = (top + total.log()).view(hq)
        s["out"][i] = ((p @ v[:, :n].contiguous()) / total).view(hq, d).to(s["out"].dtype)
    return dict(out=s["out"], lse=s["lse"])


def _frequencies(c):
    f = c["base"] ** (-torch.arange(0, c["turn"], 2, dtype=torch.float64, device=DEV) / c["turn"])
    factor, trained, low, high, magnitude = _rotation(c)
    if factor == 1.0:
        return f, 1.0
    stay = ((trained * f / (2.0 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
    return stay * f + (1.0 - stay) * f / factor, magnitude


def _turned(c, x, positions):
    """x [T, H, D] bf16 turned by positions [T]; angles in 64 bits."""
    f, magnitude = _frequencies(c)
    angle = positions.double()[:, None] * f
    cos, sin = (angle.cos() * magnitude).float()[:, None], (angle.sin() * magnitude).float()[:, None]
    y = x.float()
    half = c["turn"] // 2
    if c["layout"] == "half":
        a, b = y[..., :half].clone(), y[..., half:c["turn"]].clone()
        y[..., :half], y[..., half:c["turn"]] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = y[..., 0:c["turn"]:2].clone(), y[..., 1:c["turn"]:2].clone()
        y[..., 0:c["turn"]:2], y[..., 1:c["turn"]:2] = a * cos - b * sin, b * cos + a * sin
    return y.to(torch.bfloat16)


def _plain_rotate(s):
    s["q_out"].copy_(_turned(s["c"], s["q"], s["positions"]))
    s["k_out"].copy_(_turned(s["c"], s["k"], s["positions"]))
    return dict(q=s["q_out"], k=s["k_out"])


def _new_tokens(s):
    """Sequence and cache index of every new token (host)."""
    new = s["new"].astype(np.int64)
    seq = np.repeat(np.arange(new.size), new)
    return seq, np.arange(seq.size) - np.repeat(np.cumsum(new) - new, new) + (s["lens"] - s["new"])[seq]


def _plain_store(s):
    c, on = s["c"], lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV).long()
    at = np.nonzero(s["fresh"] >= 0)[0]
    s["bt"][on(at), on((s["lens"][at] - 1) // PAGE)] = on(s["fresh"][at]).int()
    seq, index = _new_tokens(s)
    positions = on(index - (s["lens"] - s["new"])[seq] + s["first"][seq])
    page, slot = s["bt"][on(seq), on(index // PAGE)].long(), on(index % PAGE)
    s["q_out"].copy_(_turned(c, s["q"], positions))
    k = _turned(c, s["kn"], positions)
    s["kp"][page, :, :, slot] = k.view(k.shape[0], k.shape[1], -1, 8)
    s["vp"][page, :, :, slot] = s["vn"]
    return dict(q=s["q_out"], kp=s["kp"], vp=s["vp"], bt=s["bt"])


def _plain_sample(s):
    """Weights and their sums in 64 bits: the draw compares running sums with a share of the whole."""
    x, u = s["logits"], s["u"].double()[:, None]
    b, n = x.shape
    one = torch.ones((b, 1), dtype=torch.float64, device=DEV)
    t = s["temperature"].double()[:, None] if "temperature" in s else one
    greedy = t[:, 0] == 0
    t = torch.where(t == 0, one, t)
    order = x.sort(dim=1, descending=True, stable=True).indices
    w = x.double()
    top = w.amax(1, keepdim=True)
    y = w.sub_(top).div_(t)
    w = y.exp()
    total = w.sum(1, keepdim=True)
    stay = torch.ones((b, n), dtype=torch.bool, device=DEV)
    if s["c"]["cut"] != "none":
        ranked = w.gather(1, order)
        if "top_k" in s:
            k = torch.where(s["top_k"] <= 0, n, s["top_k"]).long()[:, None]
            ranked.masked_fill_(torch.arange(n, device=DEV)[None, :] >= k, 0.0)
        before = ranked.cumsum(1).sub_(ranked)
        keep = before < s["top_p"].double()[:, None].clamp(max=1.0) * ranked.sum(1, keepdim=True)
        keep |= s["top_p"][:, None] >= 1.0
        keep &= ranked > 0
        if "min_p" in s:
            keep &= ranked >= s["min_p"].double()[:, None]
        stay = torch.zeros_like(stay).scatter_(1, order, keep)
    stay = torch.where(greedy[:, None], torch.zeros_like(stay).scatter_(1, order[:, :1], True), stay)
    run_sum = torch.where(stay, w, 0.0).cumsum(1)
    kept = run_sum[:, -1:].clone()
    token = (run_sum > u * kept).to(torch.uint8).argmax(1)
    logprob = y.gather(1, token[:, None]) - total.log()
    return dict(token=token.int(), logprob=logprob[:, 0].float(), kept=(kept / total)[:, 0].float())


# --------------------------------------------------------------------------
# work and the 64-bit results
# --------------------------------------------------------------------------
def work(c):
    if c["kind"] == "sample":
        n = c["rows"] * c["vocab"]
        return {"bytes": n * (4 if c["dtype"] == "fp32" else 2) + c["rows"] * 32, "flops": 4 * n}
    hq, hkv, d = HEADS[c["heads"]]
    if c["kind"] == "rotate":
        return {"bytes": c["rows"] * ((hq + hkv) * d * 4 + 4), "flops": c["rows"] * (hq + hkv) * c["turn"] * 3}
    lens = _lengths(c).astype(np.int64)
    if c["kind"] == "store":
        t = int(_new_lengths(c, lens).sum())
        return {"bytes": t * (hq + 2 * hkv) * d * 4 + t * 4, "flops": t * (hq + hkv) * c["turn"] * 3}
    common = c["prefix"] // PAGE * PAGE
    tokens = int((lens - common).sum()) + c["groups"] * common
    element = 1 if c["fp8"] else 2
    return {"bytes": 2 * tokens * hkv * d * element + (tokens // PAGE * hkv * 8 if c["fp8"] else 0) + lens.size * hq * (4 * d + 4),
            "flops": int(lens.sum()) * hq * 4 * d}


def exact(c, seed):
    s = prepare(c, seed)
    return {"shared": _exact_shared, "store": _exact_store, "rotate": _exact_rotate, "sample": _exact_sample}[c["kind"]](s)


def _tile(s, pool, pages):
    """Pages of a pool by (page, KV head, slot, dim), in 64 bits."""
    d = HEADS[s["c"]["heads"]][2]
    x = s[pool][pages]
    if "ks" in s:
        t, j = torch.arange(PAGE, device=DEV)[:, None], torch.arange(d, device=DEV)[None, :]
        if pool == "kp":
            at = ((j // 64 * 4 + j % 32 // 8) * 16 + t) * 16 + j // 32 % 2 * 8 + j % 8
        else:
            at = ((j // 64 * 4 + t // 4) * 16 + j % 16) * 16 + j // 16 % 4 * 4 + t % 4
        return x.view(torch.float8_e4m3fn).double()[:, :, at] * s["ks" if pool == "kp" else "vs"][pages].double()[..., None, None]
    return x.double().permute(0, 1, 3, 2, 4).flatten(3) if pool == "kp" else x.double().permute(0, 1, 3, 2)


def _exact_shared(s):
    """Softmax over the prompt's keys and each member's own, joined by their sums."""
    hq, hkv, d = HEADS[s["c"]["heads"]]
    members, common = s["c"]["members"], s["c"]["prefix"] // PAGE
    out = torch.empty(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device=DEV)
    for i in range(s["c"]["groups"]):
        rows = range(i * members, (i + 1) * members)
        pages = s["bt"][rows[0], :common].long()
        q = s["q"][rows[0]:rows[-1] + 1].double().view(members, hkv, hq // hkv, d)
        k, v = _tile(s, "kp", pages), _tile(s, "vp", pages)
        for h in range(hkv):
            z = (q[:, h].reshape(-1, d) @ k[:, h].reshape(-1, d).t().contiguous()).mul_(s["scale"])
            ref = torch.logsumexp(z, 1, keepdim=True) if common else torch.full((z.shape[0], 1), -math.inf, dtype=torch.float64, device=DEV)
            o = torch.exp(z - ref) @ v[:, h].reshape(-1, d)
            for m, r in enumerate(rows):
                n = int(s["lens"][r])
                own_pages = s["bt"][r, common: -(-n // PAGE)].long()
                heads = slice(m * (hq // hkv), (m + 1) * (hq // hkv))
                to = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
                if own_pages.numel() == 0:
                    out[r, to], lse[r, to] = o[heads], ref[heads, 0]
                    continue
                ok, ov = (_tile(s, p, own_pages)[:, h].reshape(-1, d)[: n - common * PAGE] for p in ("kp", "vp"))
                y = (q[m, h] @ ok.t().contiguous()).mul_(s["scale"])
                mine = torch.logsumexp(y, 1, keepdim=True)
                both = torch.logaddexp(mine, ref[heads])
                out[r, to] = torch.exp(y - both) @ ov + torch.exp(ref[heads] - both) * o[heads]
                lse[r, to] = both[:, 0]
    return dict(out=out, lse=lse)


def _exact_turn(c, x, positions):
    """Pairs as complex numbers, times magnitude e^(i angle)."""
    i = torch.arange(c["turn"] // 2, dtype=torch.float64, device=DEV)
    f = torch.exp(-(2.0 * i / c["turn"]) * math.log(c["base"]))
    magnitude = 1.0
    if c["factor"] != 1.0:
        factor, trained, low, high, magnitude = _rotation(c)
        stay = torch.clamp((trained * f / (2.0 * math.pi) - low) / (high - low), 0.0, 1.0)
        f = f / factor + stay * (f - f / factor)
    z = x.double()
    turned = z[..., :c["turn"]]
    pair = (turned.unflatten(-1, (2, -1)).transpose(-1, -2) if c["layout"] == "half" else turned.unflatten(-1, (-1, 2))).contiguous()
    y = torch.view_as_complex(pair) * torch.polar(torch.full_like(positions, magnitude, dtype=torch.float64)[:, None].expand(-1, f.numel()).contiguous(),
                                                  positions.double()[:, None] * f)[:, None]
    y = torch.view_as_real(y)
    y = y.transpose(-1, -2).flatten(-2) if c["layout"] == "half" else y.flatten(-2)
    return torch.cat([y, z[..., c["turn"]:]], -1)


def _exact_rotate(s):
    return dict(q=_exact_turn(s["c"], s["q"], s["positions"]), k=_exact_turn(s["c"], s["k"], s["positions"]))


def _exact_store(s):
    seq, index = _new_tokens(s)
    page = s["bt"].cpu().numpy().astype(np.int64)[seq, index // PAGE]
    last = (index == s["lens"][seq] - 1) & (s["fresh"][seq] >= 0)
    page = torch.from_numpy(np.where(last, s["fresh"][seq], page)).to(DEV)
    slot = torch.from_numpy(index % PAGE).to(DEV)
    positions = torch.from_numpy(index - (s["lens"] - s["new"])[seq] + s["first"][seq]).to(DEV)
    kp, vp = s["kp"].double(), s["vp"].double()
    k = _exact_turn(s["c"], s["kn"], positions)
    kp[page, :, :, slot] = k.unflatten(-1, (-1, 8))
    vp[page, :, :, slot] = s["vn"].double()
    bt = s["bt"].clone()
    for i in np.nonzero(s["fresh"] >= 0)[0].tolist():
        bt[i, (int(s["lens"][i]) - 1) // PAGE] = int(s["fresh"][i])
    return dict(q=_exact_turn(s["c"], s["q"], positions), kp=kp, vp=vp, bt=bt)


def _exact_sample(s):
    """Row by row, with normalised probabilities."""
    b, n = s["logits"].shape
    get = lambda name, default: s[name].cpu().tolist() if name in s else [default] * b  # noqa: E731
    t, k, p, low, u = get("temperature", 1.0), get("top_k", 0), get("top_p", 1.0), get("min_p", 0.0), get("u", 0.0)
    token = torch.empty(b, dtype=torch.int32, device=DEV)
    logprob, kept = (torch.empty(b, dtype=torch.float64, device=DEV) for _ in range(2))
    for i in range(b):
        logits = s["logits"][i].double()
        prob = torch.log_softmax(logits / (t[i] if t[i] > 0 else 1.0), 0)
        if t[i] == 0:
            at = (logits == logits.max()).nonzero()[0, 0]
            token[i], logprob[i], kept[i] = at, prob[at], prob[at].exp()
            continue
        weight = prob.exp()
        # candidates: what top-k leaves, the heaviest first and equal ones by index
        place = torch.argsort(-logits, stable=True)[: k[i] if k[i] > 0 else n]
        ranked = weight[place]
        if p[i] < 1.0:
            sums = torch.cumsum(ranked, 0)
            m = int((sums < p[i] * sums[-1]).sum()) + 1
            place, ranked = place[:m], ranked[:m]
        place = place[ranked >= low[i] * ranked[0]] if low[i] > 0 else place
        place = place.sort().values
        sums = torch.cumsum(weight[place], 0)
        at = place[min(int((sums <= u[i] * sums[-1]).sum()), place.numel() - 1)]
        token[i], logprob[i], kept[i] = at, prob[at], sums[-1]
    return dict(token=token, logprob=logprob, kept=kept)
