"""64-bit references and error bounds of the new tokens' norm, rotation and cache
writes, of the 4-bit cache and its attention, and of the verification of drafted
tokens; plain Python and CPU tensors.

u = 2^-24 and 2^-8 are half a step of fp32 and of bf16.
"""
import math
import random

import numpy as np
import torch

from draft_support import HALF_BF16, U, pages_of


# ---------------------------------------------------------------------------
# norm and rotation
# ---------------------------------------------------------------------------
def angles(positions, rot, base=10000.0):
    """cos_sin fp32 [positions, rot]."""
    freq = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    a = torch.arange(positions, dtype=torch.float64)[:, None] * freq
    return torch.cat([a.cos(), a.sin()], 1).float()


def reference_rope(x, weight, eps, positions, cos_sin, interleaved):
    """(rows, bound) in 64 bits of [T, H, d] bf16 rows.  The bound: a sum of d squares and
    its root are off by (d / 2 + 6) u in relative terms, the products behind them by 2 u, a
    rotated value by 3 u more of the sum of its products' sizes; rounding by 2^-8."""
    x = x.double().cpu()
    d = x.shape[2]
    if weight is not None:
        x = x * weight.double().cpu() / torch.sqrt(x.square().mean(2, keepdim=True) + eps)
    size = x.abs()
    if positions is not None:
        cs = cos_sin.double().cpu()[positions.long().cpu()][:, None]
        rot = cs.shape[2]
        cos, sin = cs[..., :rot // 2], cs[..., rot // 2:]
        out, big = x.clone(), size.clone()
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
            c, s = cos[..., i], sin[..., i]
            out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
            big[..., a] = size[..., a] * c.abs() + size[..., b] * s.abs()
            big[..., b] = size[..., b] * c.abs() + size[..., a] * s.abs()
        x, size = out, big
    return x, HALF_BF16 * x.abs() * (1 + HALF_BF16) + (d / 2 + 12) * U * size + 1e-30


# ---------------------------------------------------------------------------
# the 4-bit page
# ---------------------------------------------------------------------------
def _bf16_round(x):
    """A float as the nearest bf16, ties to even."""
    return float(torch.tensor(x, dtype=torch.float64).float().bfloat16())


def quantize(row):
    """A row's groups of 64: [(codes, z, s)], from its bf16 values."""
    out = []
    for a in range(0, len(row), 64):
        g = [float(x) for x in row[a:a + 64]]
        if not all(math.isfinite(x) for x in g):
            out.append(([0] * 64, None, math.nan))
            continue
        lo, hi = min(0.0, min(g)), max(0.0, max(g))
        s = _bf16_round((hi - lo) / 15)
        if s == 0:
            out.append(([0] * 64, 0, 0.0))
            continue
        z = min(round(-lo / s), 15)              # (Python rounds ties to even)
        out.append(([min(max(round(x / s) + z, 0), 15) for x in g], z, s))
    return out


def page_get(page, d, token, values):
    """A token's row in a page (bytes): [(codes, z, s)] of its groups."""
    out = []
    for g in range(d // 64):
        codes = []
        for c in range(64):
            if values:
                at, e = 2 * ((c // 4 * 16 + token) * (d // 64) + g), c % 4
            else:
                word = ((token * 4 + c // 16) * (d // 64) + g) * 2 + c % 16 // 8
                at, e = 4 * word, c % 8 // 2 + 4 * (c % 2)
            codes.append(page[at + e // 2] >> 4 * (e % 2) & 15)
        pair = np.frombuffer(bytes(page[8 * d + 4 * (16 * g + token):][:4]), dtype=np.uint16)
        zz, s = (np.array([int(x) << 16], dtype=np.uint32).view(np.float32)[0] for x in pair)
        out.append((codes, float(zz) - 128, float(s)))
    return out


def page_put(page, d, token, values, groups):
    """Writes a token's row into a page (bytearray)."""
    def bits(x):
        return int(np.array([x], dtype=np.float32).view(np.uint32)[0] >> 16)
    for g, (codes, z, s) in enumerate(groups):
        for c, code in enumerate(codes):
            if values:
                at, e = 2 * ((c // 4 * 16 + token) * (d // 64) + g), c % 4
            else:
                word = ((token * 4 + c // 16) * (d // 64) + g) * 2 + c % 16 // 8
                at, e = 4 * word, c % 8 // 2 + 4 * (c % 2)
            byte = at + e // 2
            page[byte] = page[byte] & ~(15 << 4 * (e % 2)) | code << 4 * (e % 2)
        at = 8 * d + 4 * (16 * g + token)
        page[at:at + 4] = int(bits(s) << 16 | bits(128 + z)).to_bytes(4, "little")


def unpack(cache, d, values):
    """cache uint8 [N, H, 9 d] -> (rows float64 [N, 16, H, d], scales [N, 16, H, d])."""
    raw = cache.cpu().numpy()
    n, h = raw.shape[:2]
    c = np.arange(64)
    rows = np.zeros((n, h, 16, d))
    steps = np.zeros((n, h, 16, d))
    for g in range(d // 64):
        for t in range(16):
            if values:
                at, e = 2 * ((c // 4 * 16 + t) * (d // 64) + g), c % 4
            else:
                at = 4 * (((t * 4 + c // 16) * (d // 64) + g) * 2 + c % 16 // 8)
                e = c % 8 // 2 + 4 * (c % 2)
            codes = raw[:, :, at + e // 2] >> 4 * (e % 2) & 15
            at = 8 * d + 4 * (16 * g + t)
            pair = np.ascontiguousarray(raw[:, :, at:at + 4]).view(np.uint16).astype(np.uint32) << 16
            pair = pair.view(np.float32).astype(np.float64)
            with np.errstate(invalid="ignore"):
                rows[:, :, t, 64 * g:64 * g + 64] = pair[..., 1:] * (codes - (pair[..., :1] - 128))
            steps[:, :, t, 64 * g:64 * g + 64] = pair[..., 1:]
    return (torch.from_numpy(x).permute(0, 2, 1, 3) for x in (rows, steps))


def random_pool(lens, hkv, d, seed, k_scale=1.0, poison=False):
    """(k_cache, v_cache, table) on the CPU: pages in random order, random codes, scales
    near those of N(0, 1) rows; with poison the scales of every slot that holds no key are
    NaN, and the table's entries behind a row's pages lie outside the pool."""
    g = torch.Generator().manual_seed(seed)
    need = sum(pages_of(n) for n in lens)
    blocks, width = need + need // 4 + 2, max([pages_of(n) for n in lens] + [1])
    perm = torch.randperm(blocks, generator=g)
    table = torch.full((len(lens), width), 1 << 30 if poison else 0, dtype=torch.int32)
    used = torch.zeros((blocks, 16), dtype=torch.bool)
    at = 0
    for s, n in enumerate(lens):
        p = pages_of(n)
        table[s, :p] = perm[at:at + p].int()
        for j in range(p):
            used[perm[at + j], :min(16, n - 16 * j)] = True
        at += p
    caches = []
    for scale in (k_scale, 1.0):
        c = torch.randint(0, 256, (blocks, hkv, 9 * d), generator=g, dtype=torch.uint8)
        s = (scale * (0.2 + 0.2 * torch.rand((blocks, hkv, d // 64, 16), generator=g))).bfloat16()
        if poison:
            s = torch.where(used[:, None, None, :], s, torch.tensor(math.nan, dtype=torch.bfloat16))
        z = (128 + torch.randint(4, 12, s.shape, generator=g)).bfloat16()
        pair = torch.stack([z, s], -1).contiguous().view(torch.uint8)
        c[..., 8 * d:] = pair.reshape(blocks, hkv, d)
        caches.append(c)
    return caches[0], caches[1], table


def attend_kv4(q, k, v, ks, vs, seen, scale):
    """One head: q [n, d]; k, v, their scales ks, vs [m, d]; seen bool [n, m].  Returns
    float64 (o, bound).  Beside the terms of draft_support's bound: the codes are multiplied as
    128 + c <= 143, so that a score's sums, of 64 products and one correction a group,
    are off by (2 64 + 8) u 143 scale sum s|q|, and the output's by twice their relative error
    times 143 sum p s."""
    q, d = q.double().cpu(), q.shape[1]
    n, m = seen.shape
    o, b = torch.zeros((n, d), dtype=torch.float64), torch.full((n, d), 1e-30, dtype=torch.float64)
    if m == 0 or n == 0:
        return o, b
    dead = ~torch.isfinite(ks).all(1)
    assert not (dead & seen.any(0)).any()
    k, v, ks, vs = (torch.where(dead[:, None], torch.zeros_like(x), x) for x in (k, v, ks, vs))
    v, vs = (torch.where(torch.isfinite(x), x, torch.zeros_like(x)) for x in (v, vs))
    x = ((q @ k.t()) * scale).masked_fill(~seen, -math.inf)
    some = seen.any(1)
    p = torch.zeros_like(x)
    p[some] = torch.softmax(x[some], 1)
    o = p @ v
    score = (2 * 64 + 8) * U * 143 * scale * (q.abs() @ ks.t()).masked_fill(~seen, 0).amax(1)
    sums = (seen.sum(1) / 16 + 64) * U
    rel = HALF_BF16 * (1 + HALF_BF16) + 2 * score + 2.0 ** -20 + 2 * sums
    b = HALF_BF16 * o.abs() + (rel[:, None] * (p @ v.abs()) + 2 * 143 * sums[:, None] * (p @ vs)) * \
        (1 + HALF_BF16) + 1e-30
    return o, b


def reference_kv4(q, k_cache, v_cache, table, kv_lens, rows, scale):
    """(o, bound) in 64 bits of rag_attn_decode_paged_kv4; rows: query rows a sequence."""
    hq, d = q.shape[1], q.shape[2]
    hkv = k_cache.shape[1]
    (k, ks), (v, vs) = unpack(k_cache, d, False), unpack(v_cache, d, True)
    o = torch.zeros(q.shape, dtype=torch.float64)
    b = torch.zeros(q.shape, dtype=torch.float64)
    at = 0
    for s, (n, m) in enumerate(zip(rows, kv_lens)):
        pages = table[s, :pages_of(m)].long().cpu()
        part = [x[pages].reshape(-1, hkv, d)[:m] for x in (k, v, ks, vs)]
        seen = torch.arange(m)[None, :] <= m - n + torch.arange(n)[:, None]
        for h in range(hq):
            g = h // (hq // hkv)
            o[at:at + n, h], b[at:at + n, h] = attend_kv4(q[at:at + n, h], *(x[:, g] for x in part),
                                                          seen, scale)
        at += n
    return o, b


# ---------------------------------------------------------------------------
# verification
# ---------------------------------------------------------------------------
def _weights(logits, heat):
    x = np.asarray(logits, dtype=np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if not math.isfinite(top):
        return np.zeros(len(x)), int(np.argmax(x))
    return (np.exp((x - top) / heat) if heat > 0 else np.zeros(len(x))), int(np.argmax(x))


def _pick(w, u):
    """First index whose running sum exceeds u times the total; the last with a weight where
    none does."""
    c = np.cumsum(w)
    above = np.nonzero(c > float(u) * c[-1])[0]
    return int(above[0]) if len(above) else int(np.nonzero(w > 0)[0][-1])


def _token(logits, heat, u):
    w, best = _weights(logits, heat)
    return _pick(w, u) if w.sum() > 0 else best


def reference_verify(logits, tokens, cu, heat, uniforms, max_kept, parents=None, draft=None):
    """(kept, num_kept, next_token) as lists, one node after another."""
    kept, count, nxt = [], [], []
    for s in range(len(cu) - 1):
        a, n, t = cu[s], cu[s + 1] - cu[s], heat[s]
        if n == 0:
            kept.append([-1] * max_kept)
            count.append(0)
            nxt.append(-1)
            continue
        path = [0]
        if draft is None:
            while True:
                token = _token(logits[a + path[-1]], t, uniforms[a + path[-1]])
                children = [j for j in range(path[-1] + 1, n) if tokens[a + j] == token and
                            (j - 1 if parents is None else parents[a + j]) == path[-1]]
                if len(path) == max_kept or not children:
                    break
                path.append(children[0])
        else:
            token = None
            while len(path) < min(n, max_kept):
                row = a + len(path)
                w, best = _weights(logits[row - 1], t)
                x = tokens[row]
                if w.sum() == 0:
                    ok = x == best
                else:
                    ok = 0 <= x < len(w) and float(uniforms[row]) * float(draft[row][x]) < w[x] / w.sum()
                if not ok:
                    rest = np.maximum(w / w.sum() - np.asarray(draft[row], dtype=np.float64), 0) \
                        if w.sum() > 0 else w
                    token = _pick(rest, uniforms[a]) if rest.sum() > 0 else None
                    break
                path.append(len(path))
            if token is None:
                token = _token(logits[a + path[-1]], t, uniforms[a])
        kept.append(path + [-1] * (max_kept - len(path)))
        count.append(len(path))
        nxt.append(token)
    return kept, count, nxt


def verify_case(seed, lens, vocab, chain, spread=3.0, near=0.3, heats=(0.0, 0.7, 1.0, 2.0)):
    """(logits fp32 [T, V], tokens, parents, cu, heat, uniforms, draft probabilities) on the
    CPU, the drafts near what the logits say."""
    r = random.Random(seed)
    g = torch.Generator().manual_seed(seed)
    total = sum(lens)
    logits = (spread * torch.randn((total, vocab), generator=g)).bfloat16().float()
    uniforms = torch.rand(total, generator=g)
    cu, parents, tokens, draft = [0], [], [], torch.zeros((total, vocab))
    for n in lens:
        a = cu[-1]
        for i in range(n):
            p = i - 1 if chain else r.randint(0, i - 1) if i else -1
            parents.append(p)
            if i == 0:
                tokens.append(r.randrange(vocab))
                continue
            y = logits[a + p] + near * torch.randn(vocab, generator=g)
            draft[a + i] = torch.softmax(y, 0)
            if chain:
                tokens.append(int(torch.multinomial(draft[a + i], 1, generator=g)))
            else:
                rank = min(parents[a:a + i].count(p), vocab - 1)
                tokens.append(int(y.topk(rank + 1).indices[-1]))
        cu.append(a + n)
    heat = [r.choice(heats) for _ in lens]
    return logits, tokens, parents, cu, heat, uniforms, draft
