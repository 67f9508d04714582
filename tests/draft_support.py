"""64-bit references and error bounds for the masked attention operators, and
drafted trees.

The bound of an output element, from the kernels' arithmetic (u = 2^-24, half a
step of fp32; 2^-8, half a step of bf16):
  * a score is a sum of d exact products in fp32: off by at most
    (d + 2) u scale sum|q k|; its weight by twice that in relative terms, and by
    2^-21 for the exponential and its argument;
  * the weight is rounded to bf16 for the product with V: 2^-8;
  * sums over n keys are formed at least 16 keys at a time in the matrix unit:
    (n / 16 + 64) u each, for the numerator and for the denominator, the joins of
    pieces among the 64;
  * the output is rounded to bf16: 2^-8 |o|.
All but the last multiply sum_j p_j |v_j|.
"""
import math

import torch

U = 2.0 ** -24
HALF_BF16 = 2.0 ** -8


def attend64(q, k, v, seen, scale):
    """One head: q [n, d], k and v [m, d], seen bool [n, m].  Returns float64
    (o, lse, bound of o, bound of lse); rows that see nothing give 0 and -inf, and
    unseen keys count for nothing, NaN or not."""
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    seen = seen.cpu()
    n, m = seen.shape
    d = q.shape[1]
    o = torch.zeros((n, d), dtype=torch.float64)
    bo = torch.zeros((n, d), dtype=torch.float64)
    lse = torch.full((n,), -math.inf, dtype=torch.float64)
    bl = torch.zeros(n, dtype=torch.float64)
    if m == 0:
        return o, lse, bo, bl
    kz = torch.where(torch.isfinite(k), k, torch.zeros_like(k))
    vz = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
    x = (q @ kz.t()) * scale
    x = x.masked_fill(~seen, -math.inf)
    any_key = seen.any(1)
    lse = torch.logsumexp(x, 1)
    p = torch.where(seen, torch.exp(x - lse[:, None]), torch.zeros_like(x))
    p[~any_key] = 0
    o = p @ vz
    score = (d + 2) * U * scale * (q.abs() @ kz.abs().t()).masked_fill(~seen, 0).amax(1)
    sums = (seen.sum(1) / 16 + 64) * U
    rel = HALF_BF16 * (1 + HALF_BF16) + 2 * score + 2.0 ** -21 + 2 * sums
    bo = HALF_BF16 * o.abs() + rel[:, None] * (p @ vz.abs()) * (1 + HALF_BF16) + 1e-30
    bl = score + 2.0 ** -21 + sums + 4 * U * lse.abs().nan_to_num(0, 0, 0) + 1e-30
    # a row that sees a non-finite key or value has no bound: NaN marks it
    bad = ((~torch.isfinite(k)).any(1) | (~torch.isfinite(v)).any(1))[None, :] & seen
    bo[bad.any(1)] = math.nan
    bl[bad.any(1)] = math.nan
    return o, lse, bo, bl


def within(got, want, bound, what=""):
    """Every element with a bound is finite and inside it."""
    g = got.double().cpu()
    has = ~torch.isnan(bound)
    assert torch.isfinite(g[has]).all(), f"{what}: non-finite output"
    over = (g - want).abs() - bound
    worst = over[has].max().item() if has.any() else 0.0
    assert worst <= 0, f"{what}: {worst:.3e} beyond the bound"


def tree_parents(rng, n, chain=None):
    """n nodes, parents before their children; -1: the last key before them."""
    chain = rng.randint(1, n) if chain is None else chain
    return [i - 1 if i < chain else rng.randint(-1, i - 1) for i in range(n)]


def ancestor_seen(parents):
    """bool [n, n]: node i sees itself and its ancestors."""
    n = len(parents)
    seen = torch.zeros((n, n), dtype=torch.bool)
    for i, p in enumerate(parents):
        if p >= 0:
            seen[i] = seen[p]
        seen[i, i] = True
    return seen


def mask_words(seen_list, words, fill=0):
    """Packed masks int64 [sum n, words]; bits behind a sequence's nodes are
    `fill`'s (ignored by the operator)."""
    rows = []
    for seen in seen_list:
        n = seen.shape[0]
        for i in range(n):
            bits = sum(1 << j for j in range(n) if seen[i, j])
            bits |= fill & ((1 << 64 * words) - 1) & ~((1 << n) - 1)
            w = [(bits >> 64 * k) & ((1 << 64) - 1) for k in range(words)]
            rows.append([x - (1 << 64) if x >> 63 else x for x in w])
    return torch.tensor(rows, dtype=torch.int64).reshape(-1, words)


def dense_keys(cache, table, s, n):
    """Keys 0..n-1 of sequence s, [n, hkv, d], on the CPU."""
    pages = table[s, :(n + 15) // 16].long()
    x = cache[pages].permute(0, 2, 1, 3)
    return x.reshape(-1, cache.shape[1], cache.shape[3])[:n].cpu()


def reference_tree(q, k_cache, v_cache, table, kv_lens, seen_list, scale):
    """(o, bound) [Tq, hq, d] in 64 bits of rag_attn_decode_paged_tree."""
    hq, d = q.shape[1], q.shape[2]
    hkv = k_cache.shape[1]
    o = torch.zeros(q.shape, dtype=torch.float64)
    b = torch.zeros(q.shape, dtype=torch.float64)
    at = 0
    for s, seen in enumerate(seen_list):
        n, nk = seen.shape[0], kv_lens[s]
        if n == 0:
            continue
        k, v = dense_keys(k_cache, table, s, nk), dense_keys(v_cache, table, s, nk)
        full = torch.cat([torch.ones((n, nk - n), dtype=torch.bool), seen], 1)
        for h in range(hq):
            g = h // (hq // hkv)
            o[at:at + n, h], _, b[at:at + n, h], _ = attend64(q[at:at + n, h], k[:, g], v[:, g],
                                                             full, scale)
        at += n
    return o, b


def range_seen(nq, nk, ranges):
    """bool [nq, nk] of the rows' (shared, start)."""
    j = torch.arange(nk)[None, :]
    p = (nk - nq + torch.arange(nq))[:, None]
    r = torch.as_tensor(ranges).reshape(nq, 2).long()
    return (j < r[:, :1]) | ((j >= r[:, 1:]) & (j <= p))


def reference_ranges(q, k, v, lens_q, lens_k, ranges, scale):
    """(o, lse [hq, Tq], bounds of both) in 64 bits of
    rag_attn_prefill_varlen_ranges."""
    hq, hkv = q.shape[1], k.shape[1]
    o = torch.zeros(q.shape, dtype=torch.float64)
    bo = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.zeros((hq, q.shape[0]), dtype=torch.float64)
    bl = torch.zeros_like(lse)
    a = b = 0
    for nq, nk in zip(lens_q, lens_k):
        seen = range_seen(nq, nk, ranges[a:a + nq].cpu())
        for h in range(hq):
            g = h // (hq // hkv)
            r = attend64(q[a:a + nq, h], k[b:b + nk, g], v[b:b + nk, g], seen, scale)
            o[a:a + nq, h], lse[h, a:a + nq], bo[a:a + nq, h], bl[h, a:a + nq] = r
        a, b = a + nq, b + nk
    return o, lse, bo, bl


def pages_of(n):
    return (n + 15) // 16


def reference_pages(table, stack, num_free, old, new, capacity):
    """rag_kv_pages_update on lists, one page and one token after another."""
    table, stack, width = [list(r) for r in table], list(stack), len(table[0]) if table else 0
    pile = stack[:num_free]
    for s in range(len(old)):
        pile += [table[s][p] for p in range(pages_of(new[s]), pages_of(old[s]))]
    lens, cu, slots, granted = [], [0], [], len(old)
    for s in range(len(old)):
        if new[s] > old[s] and granted == len(old):
            need = pages_of(new[s]) - pages_of(old[s])
            if need > len(pile) or pages_of(new[s]) > width or len(slots) + new[s] - old[s] > capacity:
                granted = s
        if new[s] <= old[s]:
            lens.append(new[s])
        elif granted < len(old):
            lens.append(old[s])
        else:
            for p in range(pages_of(old[s]), pages_of(new[s])):
                table[s][p] = pile.pop()
            lens.append(new[s])
            slots += [table[s][t // 16] * 16 + t % 16 for t in range(old[s], new[s])]
        cu.append(len(slots))
    stack[num_free:len(pile)] = pile[num_free:]
    return dict(table=table, stack=stack, free=len(pile), lens=lens, cu=cu,
                slots=slots + [-1] * (capacity - len(slots)), granted=granted)
