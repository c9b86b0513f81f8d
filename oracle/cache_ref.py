"""A cache of bounded size, written plainly: the store of new tokens into an fp8
cache whose tiles' scales grow, the attention weights of cached keys, and the
eviction that goes by them.

TEST INFRASTRUCTURE ONLY. A rollout instance holds its trajectories' KV caches
within a budget (Sec. 5.2). This library keeps them in 8 bits and gives up the
tokens that the queries attend to least; the rules are this repository's own and
stated here a second time, one tile, key and token after the other.

Store: new token j of sequence s (position p = L_s - E_s + j, row cu_s + j) goes to
slot p % 16 of page block_table[s][p // 16]. A (page, KV head) tile that new tokens
land in has held tokens (slots of earlier positions) and new ones:
  m = max |new values|; s = the tile's scale; all in fp32
  no held code has a nonzero value: S = max(m, 2^-100) / 448, f = 448 / max(m, 2^-100)
                                    (m = 0: S = f = 1)
  else: k = least integer >= 0 with fp32(m / fp32(448 s)) <= 2^k, S = s 2^k,
        f = fp32(1 / S); held codes become the nearest code of value * 2^-k
  new codes: nearest code of fp32(x f); slots without a token: code 0
Weights: u[t] = sum over the new tokens j with t <= P_s + j and the group's query
heads of exp(scale q.K[t] - lse); rows with an lse that is not finite are left out.
Eviction: of L tokens n stay: protected ones (position < sinks, or >= end - recent),
then the largest weights, the lower slot among equals. The i-th kept token of the
slots n .. L-1 moves to the i-th slot below n whose token goes; in an fp8 cache its
values code * scale are stored there as new ones, all other slots below L held.
"""
from __future__ import annotations

import numpy as np

from oracle import fp8_ref

PAGE = 16
f32 = np.float32


def cu_lens(q_lens):
    return np.concatenate([[0], np.cumsum(np.asarray(q_lens, dtype=np.int64))])


# ---------------------------------------------------------------------------
# fp8 tiles
# ---------------------------------------------------------------------------
def tile_codes(pool8, page, kvh, d, is_v):
    """Codes of a tile by (slot, dim), uint8 [16, D]."""
    t, j = np.meshgrid(np.arange(PAGE), np.arange(d), indexing="ij")
    return pool8[page, kvh][(fp8_ref.v_offset if is_v else fp8_ref.k_offset)(t, j)]


def put_tile_codes(pool8, page, kvh, d, is_v, codes):
    t, j = np.meshgrid(np.arange(PAGE), np.arange(d), indexing="ij")
    pool8[page, kvh][(fp8_ref.v_offset if is_v else fp8_ref.k_offset)(t, j)] = codes


def requantize(codes, scale, held, x, new):
    """The tile rule: codes uint8 [16, D], scale fp32, held and new slot masks [16], x fp32 [16, D]."""
    value = fp8_ref.values()
    held_values = np.where(held[:, None], value[codes], 0.0)
    m = f32(np.max(np.abs(x[new]))) if new.any() else f32(0)
    shift = 0
    with np.errstate(over="ignore"):
        if not np.any(held_values != 0):
            if m == 0:
                s = f = f32(1)
            else:
                top = max(m, f32(2.0) ** f32(-100))
                s, f = f32(top) / f32(448), f32(448) / f32(top)
        else:
            ratio = f32(m) / f32(f32(448) * f32(scale))
            while float(ratio) > 2.0 ** shift:
                shift += 1
            s = f32(float(scale) * 2.0 ** shift)
            f = f32(1) / s
    out = np.zeros_like(codes)
    kept = codes if shift == 0 else fp8_ref.encode((held_values * 2.0 ** -shift).astype(np.float32))
    out[held] = kept[held]
    out[new] = fp8_ref.encode((x[new] * f).astype(np.float32))
    return out, s


def store_fp8(k_bits, v_bits, seq_lens, q_lens, block_table, k8, v8, k_scale, v_scale, new_pages=None):
    """Stores the new tokens (uint16 bf16 bits [T, Hkv, D]) in place; new_pages are recorded in block_table."""
    hkv, d = k_bits.shape[1:]
    cu = cu_lens(q_lens)
    for s, (L, e) in enumerate(zip(np.asarray(seq_lens, np.int64), np.asarray(q_lens, np.int64))):
        if e == 0:
            continue
        if new_pages is not None and new_pages[s] >= 0:
            block_table[s, (L - 1) // PAGE] = new_pages[s]
        for p in range((L - e) // PAGE, (L - 1) // PAGE + 1):
            pos = p * PAGE + np.arange(PAGE)
            new, held = (pos >= L - e) & (pos < L), pos < L - e
            page = block_table[s, p]
            for bits, pool, scales, is_v in ((k_bits, k8, k_scale, False), (v_bits, v8, v_scale, True)):
                for h in range(hkv):
                    x = np.zeros((PAGE, d), dtype=np.float32)
                    x[new] = fp8_ref.widen_bf16(bits[cu[s] + pos[new] - (L - e), h])
                    codes, scales[page, h] = requantize(tile_codes(pool, page, h, d, is_v), scales[page, h], held, x, new)
                    put_tile_codes(pool, page, h, d, is_v, codes)


# ---------------------------------------------------------------------------
# the cached values
# ---------------------------------------------------------------------------
def dense(pool, scales, pages, kvh, n, d, is_v):
    """Cached keys or values of the first n tokens of the listed pages, float64 [n, D]: uint16 bf16 pools (scales None)
    in the decode layouts, or uint8 codes."""
    rows = []
    for page in pages:
        if scales is not None:
            rows.append(fp8_ref.values()[tile_codes(pool, page, kvh, d, is_v)] * float(scales[page, kvh]))
        elif is_v:
            rows.append(fp8_ref.widen_bf16(pool[page, kvh]).astype(np.float64).T)
        else:
            rows.append(fp8_ref.widen_bf16(pool[page, kvh]).astype(np.float64).transpose(1, 0, 2).reshape(PAGE, d))
    return np.concatenate(rows)[:n] if rows else np.zeros((0, d))


def attention(q, k, v, scale, first):
    """Causal attention of rows q [E, g, D] at positions first + j over k, v [n, D]: out, lse, and for tests the sums
    sum_t p_t |v_t| / sum_t p_t [E, g, D] and max_t scale sum_d |q_d k_td| [E, g] that error bounds are made of."""
    z = scale * np.einsum("egd,td->egt", q, k)
    seen = np.arange(k.shape[0])[None, :] <= first + np.arange(q.shape[0])[:, None]
    z = np.where(seen[:, None, :], z, -np.inf)
    top = z.max(axis=2, keepdims=True)
    p = np.exp(z - top)
    total = p.sum(axis=2, keepdims=True)
    out = np.einsum("egt,td->egd", p, v) / total
    spread = np.einsum("egt,td->egd", p, np.abs(v)) / total
    size = abs(scale) * np.einsum("egd,td->egt", np.abs(q), np.abs(k))
    return out, (top + np.log(total))[..., 0], spread, np.where(seen[:, None, :], size, 0).max(axis=2)


def key_weights(q, lse, k, scale, first):
    """u [n] of one (sequence, KV head): q float64 [E, g, D], lse float64 [E, g], keys [n, D]; and the largest
    scale sum_d |q_d k_td| of each key."""
    z = scale * np.einsum("egd,td->egt", q, k)
    seen = np.arange(k.shape[0])[None, :] <= first + np.arange(q.shape[0])[:, None]
    ok = seen[:, None, :] & np.isfinite(lse)[:, :, None]
    size = np.where(ok, abs(scale) * np.einsum("egd,td->egt", np.abs(q), np.abs(k)), 0).max(axis=(0, 1), initial=0)
    with np.errstate(invalid="ignore"):
        return np.where(ok, np.exp(z - lse[:, :, None]), 0).sum(axis=(0, 1)), size


# ---------------------------------------------------------------------------
# eviction
# ---------------------------------------------------------------------------
def kept_slots(weights, positions, n, sinks, recent, end):
    """Mask of the kept ones among L tokens (weights fp32 [L], positions [L])."""
    L = weights.shape[0]

    def rank(t):
        guarded = positions[t] < sinks or (recent > 0 and positions[t] >= end - recent)
        w = float(weights[t])
        # lexicographic: protected first, then numbers by size, NaN last, the lower slot among equals
        return (0 if guarded else 1, 0 if guarded or not np.isnan(w) else 1, 0.0 if guarded or np.isnan(w) else -w, t)

    mask = np.zeros(L, dtype=bool)
    mask[sorted(range(L), key=rank)[:n]] = True
    return mask


def moves(mask, n):
    """(destination, source) slots of the tokens that move."""
    return np.nonzero(~mask[:n])[0], n + np.nonzero(mask[n:])[0]


def evict(k_pool, v_pool, k_scale, v_scale, block_table, seq_lens, keep_lens, weights, positions, weights_out,
          positions_out, sinks=0, recent=0, ends=None):
    """In place on the pools (uint16 bf16 in the decode layouts, or uint8 codes with scales). weights, positions
    [N, Hkv, 16]; the outputs may be the same arrays."""
    hkv = k_pool.shape[1]
    for s, (L, keep) in enumerate(zip(np.asarray(seq_lens, np.int64), np.asarray(keep_lens, np.int64))):
        n = min(int(keep), int(L))
        end = int(L) if ends is None else int(ends[s])
        pages = block_table[s, : (L + PAGE - 1) // PAGE]
        t = np.arange(L)
        for h in range(hkv):
            w, pos = weights[pages[t // PAGE], h, t % PAGE].copy(), positions[pages[t // PAGE], h, t % PAGE].copy()
            dst, src = moves(kept_slots(w, pos, n, sinks, recent, end), n)
            w[dst], pos[dst] = w[src], pos[src]
            front = t[:n]
            weights_out[pages[front // PAGE], h, front % PAGE] = w[:n]
            positions_out[pages[front // PAGE], h, front % PAGE] = pos[:n]
            if k_scale is None:
                k, v = k_pool[:, h].copy(), v_pool[:, h].copy()
                for a, b in zip(dst, src):
                    k_pool[pages[a // PAGE], h, :, a % PAGE] = k[pages[b // PAGE], :, b % PAGE]
                    v_pool[pages[a // PAGE], h, :, a % PAGE] = v[pages[b // PAGE], :, b % PAGE]
                continue
            for pool, scales, is_v in ((k_pool, k_scale, False), (v_pool, v_scale, True)):
                d = pool.shape[2] // PAGE
                before, scale_before = pool.copy(), scales.copy()
                for p in np.unique(dst // PAGE):
                    new = np.zeros(PAGE, dtype=bool)
                    x = np.zeros((PAGE, d), dtype=np.float32)
                    for a, b in zip(dst, src):
                        if a // PAGE == p:
                            page = pages[b // PAGE]
                            code = tile_codes(before, page, h, d, is_v)[b % PAGE]
                            x[a % PAGE] = fp8_ref.values()[code].astype(np.float32) * f32(scale_before[page, h])
                            new[a % PAGE] = True
                    held = (p * PAGE + np.arange(PAGE) < L) & ~new
                    page = pages[p]
                    codes, scales[page, h] = requantize(tile_codes(before, page, h, d, is_v), scale_before[page, h], held, x, new)
                    put_tile_codes(pool, page, h, d, is_v, codes)


# ---------------------------------------------------------------------------
# work lists
# ---------------------------------------------------------------------------
def _pages(n):
    return -(-n // PAGE)


def store_plan(seq_lens, q_lens):
    cu = cu_lens(q_lens)
    spans = [(s, (L - e) // PAGE, _pages(L)) for s, (L, e) in enumerate(zip(seq_lens, q_lens)) if e > 0]
    run = 4 if sum(b - a for _, a, b in spans) > 2048 else 1
    return [[s, p, min(run, b - p), seq_lens[s] - q_lens[s], seq_lens[s], int(cu[s]), 0, 0]
            for s, a, b in spans for p in range(a, b, run)]


def weights_plan(seq_lens, q_lens, hq, hkv, held=None, first_pos=None, num_cus=256):
    """(items, merges, waves)."""
    g = hq // hkv
    cu = cu_lens(q_lens)
    live = [s for s in range(len(seq_lens)) if q_lens[s] > 0]

    def row(s, h, p0, p1, t0, t1, slot, following=0):
        h0 = seq_lens[s] - q_lens[s] if held is None else held[s]
        return [s, h, p0, p1, t0, t1, slot, seq_lens[s], seq_lens[s] - q_lens[s], int(cu[s]), h0,
                h0 if first_pos is None else first_pos[s], following, 0, 0, 0]

    if max([q_lens[s] * g for s in live], default=0) <= 16:
        blocks = [(s, h, p) for s in live for h in range(hkv) for p in range(0, _pages(seq_lens[s]), 4)]
        waves = min(8 * num_cus, len(blocks))
        first, rest = [], []
        for w in range(waves):
            mine = blocks[len(blocks) * w // waves: len(blocks) * (w + 1) // waves]
            pairs = sorted(set((s, h) for s, h, _ in mine))
            segments = []
            for s, h in pairs:
                p = [x[2] for x in mine if x[:2] == (s, h)]
                segments.append(row(s, h, p[0], min(_pages(seq_lens[s]), p[-1] + 4), 0, q_lens[s], -1, -1))
            at = [w] + [waves + len(rest) + i for i in range(len(segments) - 1)]
            for i, r in enumerate(segments[:-1]):
                r[12] = at[i + 1]
            first.append(segments[0])
            rest += segments[1:]
        return first + rest, [], waves
    tiles = sum(-(-((q_lens[s] - max(0, p * PAGE - (seq_lens[s] - q_lens[s]))) * g) // 16)
                for s in live for p in range(0, _pages(seq_lens[s]), 16))
    tokens = max(1, max(8, tiles * hkv // (8 * num_cus)) * 16 // g)
    items, merges, slot = [], [], 0
    for s in live:
        L, e = seq_lens[s], q_lens[s]
        for p in range(0, _pages(L), 16):
            t0, end = max(0, p * PAGE - (L - e)), min(_pages(L), p + 16)
            parts = -(-(e - t0) // tokens)
            for h in range(hkv):
                if parts > 1:
                    merges.append(row(s, h, p, end, slot, parts, -1))
                for i in range(parts):
                    items.append(row(s, h, p, end, t0 + (e - t0) * i // parts, t0 + (e - t0) * (i + 1) // parts, slot if parts > 1 else -1))
                    slot += parts > 1
    items.sort(key=lambda r: -(-((r[5] - r[4]) * g) // 16), reverse=True)   # the most row tiles first
    return items, merges, 0


def evict_plan(seq_lens, keep_lens, hkv, ends=None):
    n = [min(L, k) for L, k in zip(seq_lens, keep_lens)]
    pages = sum(_pages(x) for x in n)
    run = 4 if pages > 2048 and sum(min(x, L - x) for x, L in zip(n, seq_lens)) < 4 * pages else 1
    rows, moved, hole, tail = [], [], 0, 0
    for s, L in enumerate(seq_lens):
        rows.append([L, n[s], hole, tail, L if ends is None else ends[s], s, 0, 0])
        moved += [[s, p, min(run, _pages(n[s]) - p), L, n[s], hole, tail, 0] for p in range(0, _pages(n[s]), run)]
        hole += _pages(n[s]) * hkv
        tail += min(n[s], L - n[s]) * hkv
    return sorted(rows, key=lambda r: r[0] <= 4096), moved, hole, tail
