"""Work of a serving iteration around the attention, through five operators: the
norm of each head of Q and K, their rotation by position and the new tokens'
way into the paged cache (`rope`), the same into a cache held in 4 bits, with
the keys read back as packed rows (`write`), the reading alone (`read`),
attention over the 4-bit cache (`attn`) and the verification of drafted tokens
against the model's logits (`verify`).

A case is a dict of plain values; its `kind` is one of the five.  Lengths and
trees are drawn from the case's own `sizes` seed and belong to the case; values
are drawn on the GPU from prepare()'s seed.

With `own` false, run() computes the operators from elementary torch
operations, in fp32 (verification in fp64: a drawn token depends on sums over
the vocabulary); with `own` true it calls this package's binding.

A 4-bit page holds 16 tokens of one kv head in 9 D bytes.  Each 64 channels of a
token have a scale s (bf16) and a zero point z of 0..15; a code c stands for
s (c - z).
  K codes   u32 [16 tokens][4][D / 64][2]: word (i, g, w) holds channels 64 g +
            16 i + 8 w + e, e = 0..7, the even e in its four low nibbles, the odd
            ones in its four high ones
  V codes   u16 [16][16 tokens][D / 64]: the unit (i, g) of a token holds
            channels 64 g + 4 i + e, e = 0..3, a nibble each
  at 8 D    u32 [D / 64][16 tokens]: the bits of s above those of bf16(128 + z)
"""
import math
import random

import torch

own = False

BLOCK = 16
TINY = dict(hq=4, hkv=2, d=64)
HEADS_7B = dict(hq=32, hkv=8, d=128)
EPS = 1e-6


def listed():
    return [
        # one call's next token on a small model: launch latency
        dict(name="rope_one", kind="rope", rows=1, new_lo=1, new_hi=1, prior_lo=300, prior_hi=300,
             rot=64, interleaved=False, norm=True, packed=False, **TINY, sizes=3001),
        # a prefill batch of ragged stuffed prompts: Q, K and V also as packed rows
        dict(name="rope_prompts", kind="rope", rows=4, new_lo=1500, new_hi=2624, prior_lo=0,
             prior_hi=0, rot=128, interleaved=False, norm=True, packed=True, **HEADS_7B, sizes=3002),
        # the next token of 64 running calls, each with some keys in its last page
        dict(name="write_decode", kind="write", rows=64, new_lo=1, new_hi=1, held_lo=0, held_hi=15,
             prior_lo=300, prior_hi=10304, rot=128, interleaved=False, norm=False, **HEADS_7B,
             sizes=3003),
        # the prompts of 16 map_reduce mappers, written in 4 bits and read back as rows
        dict(name="write_prompts", kind="write", rows=16, new_lo=300, new_hi=576, held_lo=0,
             held_hi=0, prior_lo=0, prior_hi=0, rot=128, interleaved=False, norm=True, **HEADS_7B,
             sizes=3004),
        # the keys before a short piece of one call on a small model
        dict(name="read_tiny", kind="read", rows=1, kv_lo=300, kv_hi=300, **TINY, sizes=3005),
        # the keys before chunked-prefill pieces of four long calls
        dict(name="read_pieces", kind="read", rows=4, kv_lo=2000, kv_hi=8192, **HEADS_7B, sizes=3006),
        # one stuffed query alone on the GPU
        dict(name="attn_one", kind="attn", rows=1, new_lo=1, new_hi=1, kv_lo=4782, kv_hi=4782,
             **HEADS_7B, sizes=3007),
        # a decode step of 64 stuffed queries: the cache's bytes count
        dict(name="attn_batch", kind="attn", rows=64, new_lo=1, new_hi=1, kv_lo=2624, kv_hi=10304,
             **HEADS_7B, sizes=3008),
        # chains of drafted tokens of ragged length judged in one step
        dict(name="attn_drafts", kind="attn", rows=32, new_lo=3, new_hi=9, kv_lo=700, kv_hi=10304,
             **HEADS_7B, sizes=3009),
        # a chain of four drafts of one call, the drafter's probabilities at hand
        dict(name="verify_one", kind="verify", rows=1, nodes_lo=5, nodes_hi=5, vocab=32768, wide=False,
             chain=True, padded=0, greedy=0.0, sizes=3010),
        # chains of a serving batch on a large vocabulary of odd size, logits in fp32
        dict(name="verify_chains", kind="verify", rows=48, nodes_lo=3, nodes_hi=9, vocab=128077,
             wide=True, chain=True, padded=0, greedy=0.2, sizes=3011),
        # trees of drafted tokens, chosen without chance; some calls greedy
        dict(name="verify_trees", kind="verify", rows=16, nodes_lo=24, nodes_hi=64, vocab=128000,
             wide=False, chain=False, padded=64, greedy=0.3, sizes=3012),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for: 1 to 256 calls
    with 1 to 2624 new tokens each, pieces of 1 to 36k keys, 1 to 256 decode rows
    or chains of up to 16 drafts over 1 to 36k keys, 1 to 64 chains or trees of 1 to
    64 nodes over vocabularies of 1000 to 160,000; the model shapes above and
    generic ones."""
    kind = rng.choice(["rope", "rope", "write", "write", "read", "attn", "attn", "attn", "verify",
                       "verify"])
    hq, hkv, d = rng.choice([(32, 8, 128), (32, 8, 128), (64, 8, 128), (4, 2, 64), (32, 8, 64),
                             (16, 16, 128), (20, 4, 128), (32, 2, 128), (14, 2, 64)])
    heads = dict(hq=hq, hkv=hkv, d=d)
    sizes = rng.randrange(1 << 20)
    if kind in ("rope", "write"):
        new = sorted((_log_int(rng, 1, 2624), _log_int(rng, 1, 2624)))
        most = (9000 if kind == "rope" else 7000) * 6144 // ((hq + 2 * hkv) * d)
        new = [min(x, most) for x in new]
        c = dict(kind=kind, rows=min(_log_int(rng, 1, 256), max(1, most // new[1])), new_lo=new[0],
                 new_hi=new[1], prior_lo=0, prior_hi=rng.choice([0, 0, _log_int(rng, 1, 36000)]),
                 rot=rng.choice([d, d, d // 2, 32]), interleaved=rng.random() < 0.3,
                 norm=rng.random() < 0.5, **heads, sizes=sizes)
        if kind == "rope":
            c["packed"] = rng.random() < 0.5
        else:
            c.update(held_lo=0, held_hi=rng.choice([0, 15]))
        return c
    if kind == "verify":
        nodes = sorted((_log_int(rng, 1, 64), _log_int(rng, 1, 64)))
        chain, wide = rng.random() < 0.5, rng.random() < 0.5
        if chain:
            nodes = [min(x, 16) for x in nodes]
        vocab = _log_int(rng, 1000, 160000)
        most = 35_000_000 if wide else 80_000_000
        return dict(kind=kind, rows=min(_log_int(rng, 1, 64), max(1, most // (vocab * nodes[1]))),
                    nodes_lo=nodes[0], nodes_hi=nodes[1], vocab=vocab, wide=wide, chain=chain,
                    padded=rng.choice([0, 0, 1, 64]), greedy=rng.choice([0.0, 0.3, 1.0]), sizes=sizes)
    kv = sorted((_log_int(rng, 1, 36000), _log_int(rng, 1, 36000)))
    if kind == "read":
        return dict(kind=kind, rows=min(_log_int(rng, 1, 64), max(1, 18000 * 8 * 128 // (kv[1] * hkv * d))),
                    kv_lo=kv[0], kv_hi=max(kv[0], min(kv[1], 18000 * 8 * 128 // (hkv * d))), **heads,
                    sizes=sizes)
    new = rng.choice([(1, 1), (1, 1), (1, 16), (2, 8)])
    rows = min(_log_int(rng, 1, 256), max(1, 300000 * 8 * 128 // (kv[1] * hkv * d)),
               max(1, 300000 * 32 * 4 // (kv[1] * hq * new[1])))
    return dict(kind=kind, rows=rows, new_lo=new[0], new_hi=new[1], kv_lo=kv[0], kv_hi=kv[1], **heads,
                sizes=sizes)


# ---------------------------------------------------------------------------
# sizes (host, from the case's own seed)
# ---------------------------------------------------------------------------
def _new_tokens(c):
    """Per call of `rope` and `write`: its new tokens, the position of the first and
    the keys that the pages at hand hold before it."""
    r = random.Random(c["sizes"])
    new = [r.randint(c["new_lo"], c["new_hi"]) for _ in range(c["rows"])]
    prior = [r.randint(c["prior_lo"], c["prior_hi"]) for _ in new]
    held = [r.randint(c["held_lo"], c["held_hi"]) if "held_lo" in c else 0 for _ in new]
    return new, prior, held


def _key_lens(c):
    r = random.Random(c["sizes"])
    return [_log_int(r, c["kv_lo"], c["kv_hi"]) for _ in range(c["rows"])]


def _query_lens(c):
    r = random.Random(c["sizes"] + 1)
    return [min(n, r.randint(c["new_lo"], c["new_hi"])) for n in _key_lens(c)]


def _trees(c):
    """Each call's nodes as their parents; node 0 is the last token of the text."""
    r = random.Random(c["sizes"])
    out = []
    for _ in range(c["rows"]):
        n = r.randint(c["nodes_lo"], c["nodes_hi"])
        chain = n if c["chain"] else r.randint(1, n)
        out.append([i - 1 if i < chain else r.randint(0, i - 1) for i in range(n)])
    return out


def _pages_of(n):
    return (n + BLOCK - 1) // BLOCK


def work(c):
    if c["kind"] == "verify":
        nodes = sum(map(len, _trees(c)))
        by = nodes * (c["vocab"] * (4.0 if c["wide"] else 2.0) + 12)
        if c["chain"]:                       # the drafter's row behind each last accepted node
            by += c["rows"] * c["vocab"] * 4.0
        return {"bytes": by + 8.0 * c["rows"], "flops": 0.0}
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    row4 = 2 * hkv * 9.0 * d / 16            # a key's K and V in 4 bits with their scales
    if c["kind"] in ("rope", "write"):
        new, _, held = _new_tokens(c)
        t = sum(new)
        by = t * (2.0 * d * (2 * hq + 2 * hkv) + 8)
        if c["kind"] == "rope":
            by += t * 4.0 * d * hkv * (2 if c["packed"] else 1)
        else:
            by += t * row4 + (t + sum(held)) * (row4 + 4.0 * d * hkv)
        return {"bytes": by, "flops": 0.0}
    if c["kind"] == "read":
        return {"bytes": sum(_key_lens(c)) * (row4 + 4.0 * d * hkv), "flops": 0.0}
    keys, rows = _key_lens(c), _query_lens(c)
    pairs = sum(n * k - n * (n - 1) // 2 for n, k in zip(rows, keys))
    return {"bytes": sum(keys) * (row4 + 0.25) + sum(rows) * 4.0 * d * hq,
            "flops": 4.0 * d * hq * pairs}


# ---------------------------------------------------------------------------
# the 4-bit pages, plain
# ---------------------------------------------------------------------------
def _codes(x):
    """x [..., D] bf16 -> codes and the zero points and scales of its 64s, fp32."""
    g = x.float().reshape(*x.shape[:-1], x.shape[-1] // 64, 64)
    lo, hi = g.amin(-1, keepdim=True).clamp(max=0), g.amax(-1, keepdim=True).clamp(min=0)
    s = ((0.5 * hi - 0.5 * lo) / 7.5).to(torch.bfloat16).float()
    at = torch.where(s > 0, s, torch.ones_like(s))
    z = torch.round(-lo / at).clamp(0, 15) * (s > 0)
    return (torch.round(g / at) + z).clamp(0, 15) * (s > 0), z, s


def _values(codes, z, s):
    return (s * (codes - z)).flatten(-2)


def _pack(x, values):
    """Rows [N, 16, H, D] bf16 as pages uint8 [N, H, 9 D]."""
    n, _, h, d = x.shape
    codes, z, s = _codes(x)
    codes = codes.to(torch.int32).permute(0, 2, 1, 3, 4)            # [N, H, 16, G, 64]
    if values:
        u = codes.reshape(n, h, 16, d // 64, 16, 4)
        u = sum(u[..., e] << 4 * e for e in range(4)).permute(0, 1, 4, 2, 3)
        body = u.to(torch.int16).contiguous().view(torch.uint8)
    else:
        u = codes.reshape(n, h, 16, d // 64, 4, 2, 8)
        w = sum(u[..., e].long() << (2 * e if e % 2 == 0 else 2 * e + 14) for e in range(8))
        w = torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)
        body = w.permute(0, 1, 2, 4, 3, 5).contiguous().view(torch.uint8)
    bits = torch.cat([128 + z, s], -1).to(torch.bfloat16).permute(0, 2, 3, 1, 4)
    return torch.cat([body.reshape(n, h, 8 * d), bits.contiguous().view(torch.uint8).reshape(n, h, d)], -1)


def _unpack(pages, d, values):
    """Pages uint8 [N, H, 9 D] as rows fp32 [N, 16, H, D]."""
    n, h = pages.shape[:2]
    g, body = d // 64, pages[..., :8 * d].contiguous()
    e = torch.arange(8, device=pages.device, dtype=torch.int32)
    if values:
        u = body.view(torch.int16).reshape(n, h, 16, 16, g).int()
        codes = (u[..., None] >> 4 * e[:4] & 15).permute(0, 3, 1, 4, 2, 5)   # [N, 16, H, G, 16, 4]
    else:
        w = body.view(torch.int32).reshape(n, h, 16, 4, g, 2)
        shift = torch.where(e % 2 == 0, 2 * e, 2 * e + 14)
        codes = (w[..., None] >> shift & 15).permute(0, 2, 1, 4, 3, 5, 6)    # [N, 16, H, G, 4, 2, 8]
    codes = codes.reshape(n, 16, h, g, 64).float()
    bits = pages[..., 8 * d:].contiguous().view(torch.bfloat16).reshape(n, h, g, 16, 2)
    bits = bits.permute(0, 3, 1, 2, 4).float()                              # [N, 16, H, G, 2]
    return _values(codes, bits[..., :1] - 128, bits[..., 1:])


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return _i32(cu)


class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed))

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda")

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda")

    def table(self, lens):
        """A block table for rows of these lengths over a pool a quarter larger, its
        pages in random order."""
        n = torch.tensor([_pages_of(x) for x in lens], device="cuda")
        need, width = int(n.sum()), max(1, int(n.max()))
        blocks = need + need // 4 + 1
        perm = torch.randperm(blocks, generator=self.g, device="cuda").to(torch.int32)
        table = torch.zeros((len(lens), width), dtype=torch.int32, device="cuda")
        table[torch.arange(width, device="cuda")[None, :] < n[:, None]] = perm[:need]
        return table, blocks

    def cache(self, blocks, hkv, d, values):
        """A pool of 4-bit pages: N(0, 1), keys with some channels larger than the rest."""
        out = torch.empty((blocks, hkv, 9 * d), dtype=torch.uint8, device="cuda")
        wide = 1 + 1.5 * self.uniform(hkv, d) ** 4
        for a in range(0, blocks, 2048):
            x = self.normal(min(2048, blocks - a), 16, hkv, d)
            out[a:a + 2048] = _pack((x if values else x * wide).to(torch.bfloat16), values)
        return out


def _angles(positions, rot):
    """cos and sin of every position up to `positions`, fp32 [positions, rot]."""
    freq = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.cat([a.cos(), a.sin()], 1).float()


def _prepare_tokens(c, rng):
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    new, prior, held = _new_tokens(c)
    t, total = sum(new), [a + b for a, b in zip(new, held)]
    table, blocks = rng.table(total)
    lens, first = torch.tensor(new, device="cuda"), torch.tensor(held, device="cuda")
    row = torch.repeat_interleave(torch.arange(len(new), device="cuda"), lens)
    i = torch.arange(t, device="cuda") - (lens.cumsum(0) - lens)[row]
    key = i + first[row]
    qkv = rng.normal(t, hq + 2 * hkv, d).to(torch.bfloat16)         # the projection's output
    s = dict(qkv=qkv, q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:],
             table=table, cu=_cu(total), total=total, interleaved=c["interleaved"],
             slots=(table[row, key // BLOCK] * BLOCK + key % BLOCK).int(),
             positions=(torch.tensor(prior, device="cuda")[row] + key).int(), row=row, key=key,
             angles=_angles(max(p + n for p, n in zip(prior, total)), c["rot"]),
             q_weight=None, k_weight=None, q_out=torch.empty((t, hq, d), dtype=torch.bfloat16, device="cuda"))
    if c["norm"]:
        s.update(q_weight=(1 + 0.2 * rng.normal(d)).to(torch.bfloat16),
                 k_weight=(1 + 0.2 * rng.normal(d)).to(torch.bfloat16))
    if c["kind"] == "rope":
        shape = (blocks, hkv, BLOCK, d)
        s.update(k_cache=rng.normal(*shape).to(torch.bfloat16),
                 v_cache=rng.normal(*shape).to(torch.bfloat16), k_out=None, v_out=None)
        if c["packed"]:
            s.update(k_out=torch.empty((t, hkv, d), dtype=torch.bfloat16, device="cuda"))
            s.update(v_out=torch.empty_like(s["k_out"]))
        return s
    s.update(k_cache=rng.cache(blocks, hkv, d, False), v_cache=rng.cache(blocks, hkv, d, True))
    s.update(_rows_out(total, hkv, d))
    return s


def _rows_out(lens, hkv, d):
    k = torch.empty((sum(lens), hkv, d), dtype=torch.bfloat16, device="cuda")
    return dict(k_rows=k, v_rows=torch.empty_like(k))


def _prepare_read(c, rng):
    lens = _key_lens(c)
    table, blocks = rng.table(lens)
    return dict(table=table, cu=_cu(lens), total=lens, k_cache=rng.cache(blocks, c["hkv"], c["d"], False),
                v_cache=rng.cache(blocks, c["hkv"], c["d"], True), **_rows_out(lens, c["hkv"], c["d"]))


def _prepare_attn(c, rng):
    s, lens = _prepare_read(c, rng), _query_lens(c)
    del s["k_rows"], s["v_rows"]
    s.update(kv=_i32(s["total"]), lens=lens, scale=1.0 / math.sqrt(c["d"]), max_new=max(lens),
             cu_q=None if max(lens) == 1 else _cu(lens),
             q=rng.normal(sum(lens), c["hq"], c["d"]).to(torch.bfloat16))
    s["o"] = torch.empty_like(s["q"])
    if own:                                     # what the serving program keeps for its steps
        from paper_2412_10543_amd import binding
        n = binding.rag_attn_decode_kv4_workspace_size(c["rows"], s["max_new"], c["hq"], c["hkv"],
                                                       c["d"], s["table"].shape[1])
        s["ws"] = torch.zeros(n, dtype=torch.uint8, device="cuda") if n else None
    return s


def _prepare_verify(c, rng):
    trees, vocab = _trees(c), c["vocab"]
    lens = [len(p) for p in trees]
    nodes, width = sum(lens), max(lens)
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    parents = _i32([p for ps in trees for p in ps])
    # each node's row of the parent that it was drafted behind, and its place among its siblings
    behind = torch.tensor([a + max(p, 0) for a, ps in zip(at, trees) for p in ps], device="cuda")
    place = torch.tensor([ps[:i].count(p) for ps in trees for i, p in enumerate(ps)], device="cuda")
    r = random.Random(c["sizes"] + 2)
    heat = [0.0 if r.random() < c["greedy"] else r.choice([0.6, 1.0]) for _ in trees]
    s = dict(lens=lens, width=width, cu=_cu(lens), parents=None if c["chain"] else parents,
             heat=torch.tensor(heat, dtype=torch.float32, device="cuda"), draft=None)
    # logits of a model: a few likely tokens over a wide floor; the drafter's are near them
    store = torch.empty((nodes, vocab + c["padded"]), device="cuda",
                        dtype=torch.float32 if c["wide"] else torch.bfloat16)
    s["logits"] = store[:, :vocab]
    near = torch.empty((nodes, vocab), dtype=torch.float32, device="cuda") if c["chain"] else None
    tokens = torch.empty(nodes, dtype=torch.int32, device="cuda")
    for a in range(0, nodes, 128):              # (in parts: the noise of all rows is large)
        b = min(nodes, a + 128)
        s["logits"][a:b] = rng.normal(b - a, vocab) * 1.5 + 9 * rng.uniform(b - a, vocab) ** 40
    for a in range(0, nodes, 128):
        b = min(nodes, a + 128)
        y = s["logits"][behind[a:b]].float() + 0.4 * rng.normal(b - a, vocab)
        if c["chain"]:
            near[a:b] = torch.softmax(y, 1)
            y = near[a:b].log() - rng.uniform(b - a, vocab).clamp(1e-30).log().neg().log()
            tokens[a:b] = y.argmax(1).int()     # drawn from the drafter's probabilities
        else:
            k = min(int(place[a:b].max()) + 1, vocab)
            tokens[a:b] = y.topk(k, 1).indices.gather(1, place[a:b, None] % k)[:, 0].int()
    s.update(tokens=tokens, uniforms=rng.uniform(nodes), draft=near,
             kept=torch.empty((len(lens), width), dtype=torch.int32, device="cuda"),
             num_kept=torch.empty(len(lens), dtype=torch.int32, device="cuda"),
             next_token=torch.empty(len(lens), dtype=torch.int32, device="cuda"))
    if own:
        from paper_2412_10543_amd import binding
        n = binding.rag_draft_verify_workspace_size(nodes, len(lens), vocab)
        s["ws"] = torch.zeros(n, dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    s = {"rope": _prepare_tokens, "write": _prepare_tokens, "read": _prepare_read,
         "attn": _prepare_attn, "verify": _prepare_verify}[case["kind"]](case, _Draw(seed))
    s["kind"] = case["kind"]
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _norm(x, weight):
    x = x.float()
    if weight is None:
        return x
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()


def _rotate(x, s):
    """x fp32 [T, H, D], turned by its tokens' positions."""
    rot = s["angles"].shape[1]
    a = s["angles"][s["positions"].long()][:, None, :]
    cos, sin = a[..., :rot // 2], a[..., rot // 2:]
    if s["interleaved"]:
        u, w = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([u * cos - w * sin, w * cos + u * sin], -1).flatten(-2)
    else:
        u, w = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([u * cos - w * sin, w * cos + u * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_tokens(s):
    q = _rotate(_norm(s["q"], s["q_weight"]), s).to(torch.bfloat16)
    k = _rotate(_norm(s["k"], s["k_weight"]), s).to(torch.bfloat16)
    page, at = s["slots"].long() // BLOCK, s["slots"].long() % BLOCK
    if s["kind"] == "rope":
        s["k_cache"][page, :, at] = k
        s["v_cache"][page, :, at] = s["v"]
        return [q, s["k_cache"], s["v_cache"]] + ([k, s["v"].clone()] if s["k_out"] is not None else [])
    rows = _plain_read(s)
    place = s["cu"].long()[s["row"]] + s["key"]
    for out, x in zip(rows, (k, s["v"])):
        out[place] = _values(*_codes(x)).to(torch.bfloat16)
    return [q, *rows]


def _plain_read(s):
    """Each call's keys in turn, as bf16 rows [T, Hkv, D]."""
    lens = torch.tensor(s["total"], device="cuda")
    row = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), lens)
    key = torch.arange(len(row), device="cuda") - s["cu"].long()[row]
    page = s["table"][row, key // BLOCK].long()
    out = []
    for cache, values in ((s["k_cache"], False), (s["v_cache"], True)):
        x = _unpack(cache, cache.shape[2] // 9, values)
        out.append(x[page, key % BLOCK].to(torch.bfloat16))
    return out


def _plain_attn(s):
    """A group of calls at a time, padded to the longest: scores, weights, products."""
    hkv, d = s["k_cache"].shape[1], s["k_cache"].shape[2] // 9
    q, o = s["q"].float(), torch.empty_like(s["q"])
    lens, keys = s["lens"], s["total"]
    order, at = sorted(range(len(lens)), key=lambda i: keys[i]), s["cu_q"]
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    while order:
        some = order[-max(1, 400000 // keys[order[-1]]):]
        order = order[:-len(some)]
        n, m = max(lens[i] for i in some), max(keys[i] for i in some)
        pages = s["table"][some, :_pages_of(m)].long()
        j = torch.arange(_pages_of(m) * BLOCK, device="cuda")
        left, top = (torch.tensor([x[i] for i in some], device="cuda") for x in (lens, keys))
        rows = torch.tensor([cu[i] for i in some], device="cuda")[:, None] + torch.arange(n, device="cuda")
        real = torch.arange(n, device="cuda") < left[:, None]
        last = (top - left)[:, None] + torch.arange(n, device="cuda")          # the last key seen
        x = q[rows.clamp(max=len(q) - 1)].reshape(len(some), n, hkv, -1, d)
        k = _unpack(s["k_cache"][pages.flatten()], d, False).reshape(len(some), -1, hkv, d)
        y = torch.matmul(x.permute(0, 2, 1, 3, 4).flatten(2, 3), k.permute(0, 2, 3, 1).contiguous())
        y = y.reshape(len(some), hkv, n, -1, len(j)) * s["scale"]
        y = y.masked_fill((j > last[..., None])[:, None, :, None], -math.inf)
        y = torch.exp(y - y.amax(-1, keepdim=True))
        y = (y / y.sum(-1, keepdim=True)).flatten(2, 3)
        v = _unpack(s["v_cache"][pages.flatten()], d, True).reshape(len(some), -1, hkv, d)
        v = v.masked_fill((j >= top[:, None])[..., None, None], 0).permute(0, 2, 1, 3).contiguous()
        y = torch.matmul(y, v).reshape(len(some), hkv, n, -1, d).permute(0, 2, 1, 3, 4).flatten(2, 3)
        o[rows[real]] = y[real].to(torch.bfloat16)
    return o


def _plain_verify(s):
    lens, width = torch.tensor(s["lens"], device="cuda"), s["width"]
    row = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), lens)
    first = s["cu"].long()[:-1]
    heat = s["heat"].double()[row][:, None]
    x = s["logits"].double()
    top = x.amax(1, keepdim=True)
    index = torch.arange(x.shape[1], device="cuda")
    best = torch.where(x == top, index, x.shape[1]).amin(1)
    p = torch.exp((x - top) / torch.where(heat > 0, heat, torch.ones_like(heat)))
    del x

    def pick(p, u):
        c = p.cumsum(1)
        return (c <= u.double()[:, None] * c[:, -1:]).sum(1).clamp(max=p.shape[1] - 1)

    kept = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    kept[:, 0] = 0
    at = torch.arange(width, device="cuda")
    node = (first[:, None] + at).clamp(max=len(row) - 1)              # [S, width]
    real = at < lens[:, None]
    if s["draft"] is not None:
        p = p / p.sum(1, keepdim=True)
        before = (torch.arange(len(row), device="cuda") - 1).clamp(min=0)
        token = s["tokens"].long()[:, None]
        fits = s["uniforms"].double() * s["draft"].gather(1, token)[:, 0].double() < p[before].gather(1, token)[:, 0]
        fits = torch.where(heat[:, 0] > 0, fits, best[before] == token[:, 0])
        go = (fits[node] & real)
        go[:, 0] = True
        count = go.long().cumprod(1).sum(1)
        kept = torch.where(at < count[:, None], at, -1).int()
        last = first + count - 1
        rest = (p[last] - s["draft"][(last + 1).clamp(max=len(row) - 1)].double()).clamp(min=0)
        rest = torch.where(((count < lens) & (rest.sum(1) > 0))[:, None], rest, p[last])
        token = torch.where(heat[first, 0] > 0, pick(rest, s["uniforms"][first]), best[last])
        return [kept, count.int(), token.int()]
    drawn = torch.where(heat[:, 0] > 0, pick(p, s["uniforms"]), best)
    parents = torch.where(real, s["parents"].long()[node], -2)
    tokens, here = s["tokens"].long()[node], torch.zeros_like(first)
    count, going = torch.ones_like(first), torch.ones_like(first, dtype=torch.bool)
    for _ in range(width - 1):
        child = (parents == here[:, None]) & (tokens == drawn[first + here][:, None]) & (at > here[:, None])
        child &= going[:, None]
        going = child.any(1)
        here = torch.where(going, torch.where(child, at, width).amin(1), here)
        kept = torch.where((at == count[:, None]) & going[:, None], here[:, None].int(), kept)
        count = count + going
    return [kept, count.int(), drawn[first + here].int()]


# ---------------------------------------------------------------------------
# this package's operators
# ---------------------------------------------------------------------------
def _own(s):
    from paper_2412_10543_amd import binding
    if s["kind"] == "rope":
        binding.rag_qkv_rope_write(s["q"], s["k"], s["v"], s["q_out"], s["positions"], s["angles"],
                                   s["slots"], s["k_cache"], s["v_cache"], k_out=s["k_out"],
                                   v_out=s["v_out"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                                   eps=EPS, interleaved=s["interleaved"])
        return [s["q_out"], s["k_cache"], s["v_cache"]] + \
            ([s["k_out"], s["v_out"]] if s["k_out"] is not None else [])
    if s["kind"] == "write":
        binding.rag_qkv_rope_write_kv4(s["q"], s["k"], s["v"], s["q_out"], s["positions"],
                                       s["angles"], s["slots"], s["k_cache"], s["v_cache"],
                                       q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                                       interleaved=s["interleaved"])
    if s["kind"] in ("write", "read"):
        binding.rag_kv4_read(s["k_cache"], s["v_cache"], s["table"], s["cu"], s["k_rows"], s["v_rows"])
        return ([s["q_out"]] if s["kind"] == "write" else []) + [s["k_rows"], s["v_rows"]]
    if s["kind"] == "attn":
        binding.rag_attn_decode_paged_kv4(s["q"], s["k_cache"], s["v_cache"], s["o"], s["table"],
                                          s["kv"], s["scale"], cu_seqlens_q=s["cu_q"],
                                          max_seqlen_q=s["max_new"], workspace=s["ws"])
        return s["o"]
    binding.rag_draft_verify(s["logits"], s["tokens"], s["cu"], s["heat"], s["uniforms"], s["kept"],
                             s["num_kept"], s["next_token"], parents=s["parents"],
                             draft_probs=s["draft"], workspace=s["ws"])
    return [s["kept"], s["num_kept"], s["next_token"]]


def run(state):
    if own:
        return _own(state)
    if state["kind"] in ("rope", "write"):
        return _plain_tokens(state)
    return {"read": _plain_read, "attn": _plain_attn, "verify": _plain_verify}[state["kind"]](state)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_turned(x, weight, s):
    """Norm and rotation of [T, H, D], the pairs as complex numbers."""
    x = x.double()
    if weight is not None:
        x = x / (x.pow(2).sum(2, keepdim=True) / x.shape[2] + EPS).sqrt() * weight.double()
    half = s["angles"].shape[1] // 2
    angle = s["angles"].double()[s["positions"].long()]
    turn = torch.complex(angle[:, :half].contiguous(), angle[:, half:].contiguous())[:, None]
    first = torch.arange(half, device="cuda") * (2 if s["interleaved"] else 1)
    second = first + (1 if s["interleaved"] else half)
    z = torch.complex(x[..., first], x[..., second]) * turn
    out = x.clone()
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _exact_quantized(x):
    """What [T, H, D] reads back as, 64 channels at a time."""
    out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
    for c in range(0, x.shape[2], 64):
        part = x[..., c:c + 64].to(torch.bfloat16).double()
        low = torch.minimum(part.min(2).values, torch.zeros((), device="cuda", dtype=torch.float64))
        high = torch.maximum(part.max(2).values, torch.zeros((), device="cuda", dtype=torch.float64))
        step = ((high - low) / 15).to(torch.bfloat16).double()[..., None]
        step = torch.where(step == 0, torch.ones_like(step), step)
        zero = (-low[..., None] / step).round().clamp(0, 15)
        out[..., c:c + 64] = step * (((part / step).round() + zero).clamp(0, 15) - zero)
    return out


def _exact_page(page, d, values):
    """One kv head's pages, uint8 [n, 9 D] -> [16 n, D], nibble by nibble."""
    out = torch.empty((page.shape[0], 16, d), dtype=torch.float64, device="cuda")
    for g in range(d // 64):
        at = 8 * d + 64 * g + 4 * torch.arange(16, device="cuda")
        pair = page[:, at[:, None] + torch.arange(4, device="cuda")].contiguous().view(torch.bfloat16)
        for c in range(64):
            if values:
                byte = (c // 4 * 16 + torch.arange(16, device="cuda")) * (d // 32) + 2 * g + c % 4 // 2
                nibble = c % 2
            else:
                byte = torch.arange(16, device="cuda") * (d // 2) + c // 16 * (d // 8) + 8 * g + \
                    4 * (c % 16 // 8) + (c % 8 // 2 + 4 * (c % 2)) // 2
                nibble = (c % 8 // 2) % 2
            code = page[:, byte] >> 4 * nibble & 15
            zero = pair[..., 0].double() - 128
            out[:, :, 64 * g + c] = pair[..., 1].double() * (code.double() - zero)
    return out.flatten(0, 1)


def exact(case, seed):
    if case["kind"] == "verify":
        return None                             # whole numbers
    s = prepare(case, seed)
    lens = s["total"]
    if case["kind"] in ("rope", "write"):
        q = _exact_turned(s["q"], s["q_weight"], s)
        k = _exact_turned(s["k"], s["k_weight"], s)
        if case["kind"] == "rope":
            caches = []
            for name, x in (("k_cache", k), ("v_cache", s["v"].double())):
                cache = s[name].double()
                rows = cache.permute(0, 2, 1, 3).flatten(0, 1)
                rows[s["slots"].long()] = x
                caches.append(rows.unflatten(0, (-1, BLOCK)).permute(0, 2, 1, 3))
            return [q, *caches] + ([k, s["v"].double()] if case["packed"] else [])
    if case["kind"] != "attn":
        out = [torch.empty((sum(lens), case["hkv"], case["d"]), dtype=torch.float64, device="cuda")
               for _ in range(2)]
        for i, n in enumerate(lens):
            a, pages = sum(lens[:i]), s["table"][i, :_pages_of(n)].long()
            for h in range(case["hkv"]):
                out[0][a:a + n, h] = _exact_page(s["k_cache"][pages, h], case["d"], False)[:n]
                out[1][a:a + n, h] = _exact_page(s["v_cache"][pages, h], case["d"], True)[:n]
        if case["kind"] == "read":
            return out
        new = [n - h for n, h in zip(lens, _new_tokens(case)[2])]
        a = b = 0
        for n, m in zip(lens, new):
            out[0][b + n - m:b + n] = _exact_quantized(k[a:a + m])
            out[1][b + n - m:b + n] = _exact_quantized(s["v"][a:a + m].double())
            a, b = a + m, b + n
        return [q, *out]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    group, a = case["hq"] // case["hkv"], 0
    for i, (n, m) in enumerate(zip(s["lens"], lens)):
        pages = s["table"][i, :_pages_of(m)].long()
        seen = torch.arange(m, device="cuda")[None, :] <= m - n + torch.arange(n, device="cuda")[:, None]
        for h in range(case["hkv"]):
            k = _exact_page(s["k_cache"][pages, h], case["d"], False)[:m]
            v = _exact_page(s["v_cache"][pages, h], case["d"], True)[:m]
            for g in range(h * group, (h + 1) * group):
                y = (s["q"][a:a + n, g].double() @ k.t()) * s["scale"]
                o[a:a + n, g] = torch.softmax(y.masked_fill(~seen, -math.inf), 1) @ v
        a += n
    return o
