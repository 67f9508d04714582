"""Work of a RAG answer that is served with drafted tokens, through four
operators: the stuffed prompt whose documents do not see one another
(`prompt`), the pages that requests of changing length hold in the paged cache
(`pages`), attention of a tree of drafted tokens over that cache (`tree`) and
the accepted drafts' move to the end of their sequence (`keep`).

A case is a dict of plain values; its `kind` is one of the four.  Lengths,
trees and documents are drawn from the case's own `sizes` seed and belong to
the case; values (Q, K, V ~ N(0, 1) in bf16, pages in random physical order)
are drawn on the GPU from prepare()'s seed.

With `own` false, run() computes the operators from elementary torch
operations in fp32; with `own` true it calls this package's binding.
"""
import math
import random

import torch

own = False

BLOCK = 16
TINY = dict(hq=4, hkv=2, d=64)
HEADS_7B = dict(hq=32, hkv=8, d=128)
HEADS_70B = dict(hq=64, hkv=8, d=128)


def listed():
    return [
        # a short two-document prompt on a small model: launch latency
        dict(name="docs_tiny", kind="prompt", prompts=1, shared=17, docs_lo=2, docs_hi=2, doc_lo=100,
             doc_hi=128, query=32, mask="docs", lse=True, **TINY, sizes=2001),
        # one stuffed query at low load: nine chunks behind a system prompt, the
        # query at the end seeing all of them
        dict(name="docs_one_query", kind="prompt", prompts=1, shared=96, docs_lo=9, docs_hi=9,
             doc_lo=512, doc_hi=512, query=77, mask="docs", lse=False, **HEADS_7B, sizes=2002),
        # a batch of 16 stuffed queries of 5 to 20 chunks of ragged length
        dict(name="docs_batch", kind="prompt", prompts=16, shared=64, docs_lo=5, docs_hi=20,
             doc_lo=400, doc_hi=512, query=64, mask="docs", lse=False, **HEADS_7B, sizes=2003),
        # the engine's tick: 64 running calls of a few hundred to 10k tokens,
        # each with the next drafts to place, some giving rejected ones back
        dict(name="pages_tick", kind="pages", rows=64, old_lo=300, old_hi=10304, grow_lo=1,
             grow_hi=64, shrink=0.25, admit=0.0, sizes=2004),
        # all mappers of 16 map_reduce queries admitted at once while as many
        # finished calls give their pages back
        dict(name="pages_admit", kind="pages", rows=640, old_lo=500, old_hi=900, grow_lo=576,
             grow_hi=576, shrink=0.5, admit=1.0, sizes=2005),
        # a small draft for one short call on a small model
        dict(name="tree_tiny", kind="tree", rows=1, nodes_lo=7, nodes_hi=7, kv_lo=300, kv_hi=300,
             **TINY, sizes=2006),
        # one stuffed query alone on the GPU, 25 drafted tokens a step
        dict(name="tree_one_query", kind="tree", rows=1, nodes_lo=25, nodes_hi=25, kv_lo=4782,
             kv_hi=4782, **HEADS_7B, sizes=2007),
        # a serving batch with small trees of ragged size: the cache's bytes count
        dict(name="tree_small_batch", kind="tree", rows=48, nodes_lo=5, nodes_hi=12, kv_lo=700,
             kv_hi=10304, **HEADS_7B, sizes=2008),
        # 16 stuffed queries with trees of 64 drafted tokens: both bytes and products
        dict(name="tree_batch", kind="tree", rows=16, nodes_lo=64, nodes_hi=64, kv_lo=2624,
             kv_hi=10304, **HEADS_7B, sizes=2009),
        # long contexts with the 70B model's heads and large trees
        dict(name="tree_long_70b", kind="tree", rows=4, nodes_lo=40, nodes_hi=64, kv_lo=33000,
             kv_hi=36000, **HEADS_70B, sizes=2010),
        # the accepted path of one call's draft
        dict(name="keep_one", kind="keep", rows=1, nodes_lo=25, nodes_hi=25, kv_lo=4782, kv_hi=4782,
             depth=5, **HEADS_7B, sizes=2015),
        # the accepted paths of a full batch, deep drafts among them
        dict(name="keep_batch", kind="keep", rows=256, nodes_lo=8, nodes_hi=64, kv_lo=576,
             kv_hi=704, depth=16, **HEADS_7B, sizes=2012),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for: prompts of
    one short document to 16 prompts of 20 chunks, with the three masks; 1 to
    2048 rows of pages; 1 to 64 trees of 1 to 128 nodes over 1 to 36k keys; 1 to
    512 accepted paths; the model shapes above and generic ones."""
    kind = rng.choice(["prompt", "prompt", "tree", "tree", "tree", "pages", "keep"])
    hq, hkv, d = rng.choice([(32, 8, 128), (32, 8, 128), (64, 8, 128), (4, 2, 64), (32, 8, 64),
                             (16, 16, 128), (20, 4, 128), (32, 2, 128), (14, 2, 64)])
    heads = dict(hq=hq, hkv=hkv, d=d)
    sizes = rng.randrange(1 << 20)
    if kind == "prompt":
        doc = sorted((_log_int(rng, 1, 1024), _log_int(rng, 1, 1024)))
        c = dict(kind=kind, prompts=_log_int(rng, 1, 16), shared=rng.choice([0, rng.randint(1, 300)]),
                 docs_lo=1, docs_hi=_log_int(rng, 1, 20), doc_lo=doc[0], doc_hi=doc[1],
                 query=rng.randint(0, 128), mask=rng.choice(["docs", "docs", "prefix", "window"]),
                 lse=rng.random() < 0.5, **heads, sizes=sizes)
        # no more products than the batch of 16, and scores that fit the plain form
        while work(c)["flops"] > 5e11 or max(_prompt_lens(c)) ** 2 * (hq // hkv) > 4e8 or \
                sum(_prompt_lens(c)) > 110000:
            c["prompts"] = max(1, c["prompts"] // 2)
            c["docs_hi"] = max(1, c["docs_hi"] // 2)
        return c
    if kind == "pages":
        old = sorted((rng.choice([0, _log_int(rng, 1, 36000)]), _log_int(rng, 1, 36000)))
        grow = sorted((_log_int(rng, 1, 4000), _log_int(rng, 1, 4000)))
        rows = min(_log_int(rng, 1, 2048), max(1, 200000 // grow[1]))
        return dict(kind=kind, rows=rows, old_lo=old[0], old_hi=old[1], grow_lo=grow[0],
                    grow_hi=grow[1], shrink=rng.choice([0.0, 0.25, 0.7]),
                    admit=rng.choice([0.0, 0.3, 1.0]), sizes=sizes)
    nodes = sorted((_log_int(rng, 1, 128), _log_int(rng, 1, 128)))
    kv = sorted((_log_int(rng, 1, 36000), _log_int(rng, 1, 36000)))
    if kind == "tree":
        rows = min(_log_int(rng, 1, 64), max(1, 36000 * 4 * 64 * 64 // (kv[1] * nodes[1] * hq)),
                   max(1, 300000 // kv[1]))
        return dict(kind=kind, rows=rows, nodes_lo=nodes[0], nodes_hi=nodes[1], kv_lo=kv[0],
                    kv_hi=kv[1], **heads, sizes=sizes)
    kv = [min(x, 8000) for x in kv]
    return dict(kind=kind, rows=min(_log_int(rng, 1, 512), max(1, 400000 // (kv[1] + nodes[1]))),
                nodes_lo=nodes[0], nodes_hi=nodes[1], kv_lo=kv[0], kv_hi=kv[1],
                depth=rng.randint(1, 24), **heads, sizes=sizes)


# ---------------------------------------------------------------------------
# sizes (host, from the case's own seed)
# ---------------------------------------------------------------------------
def _prompt_docs(c):
    r = random.Random(c["sizes"])
    return [[r.randint(c["doc_lo"], c["doc_hi"]) for _ in range(r.randint(c["docs_lo"], c["docs_hi"]))]
            for _ in range(c["prompts"])]


def _prompt_lens(c):
    return [c["shared"] + sum(docs) + c["query"] for docs in _prompt_docs(c)]


def _ranges(c):
    """(shared, start) of every token of the prompts: a token at position p sees
    keys j < shared and keys start <= j <= p.
      docs    the system prompt is causal; a document's token sees the system
              prompt and its own document; a query token sees everything
      prefix  every token sees the whole prompt but its query, and what comes
              before it
      window  the last doc_hi tokens, and the first `shared` ones"""
    out = []
    for docs in _prompt_docs(c):
        length = c["shared"] + sum(docs) + c["query"]
        if c["mask"] == "prefix":
            out += [(length - c["query"], 0)] * length
        elif c["mask"] == "window":
            out += [(min(c["shared"], p + 1), max(0, p - c["doc_hi"] + 1)) for p in range(length)]
        else:
            out += [(0, 0)] * c["shared"]
            at = c["shared"]
            for n in docs:
                out += [(c["shared"], at)] * n
                at += n
            out += [(0, 0)] * c["query"]
    return out


def _tree_sizes(c):
    """Per row: keys before the drafts, and each drafted node's parent (-1: the
    last key before the drafts)."""
    r = random.Random(c["sizes"])
    prior, parents = [], []
    for _ in range(c["rows"]):
        n = r.randint(c["nodes_lo"], c["nodes_hi"])
        prior.append(max(0, _log_int(r, c["kv_lo"], c["kv_hi"]) - r.choice([0, n])))
        # the likeliest chain first, then branches off any node before
        chain = r.randint(1, n)
        parents.append([i - 1 if i < chain else r.randint(-1, i - 1) for i in range(n)])
    return prior, parents


def _ancestors(parents):
    """Bit j of the i-th number: node i sees node j (itself and its ancestors)."""
    bits = []
    for i, p in enumerate(parents):
        bits.append((bits[p] if p >= 0 else 0) | 1 << i)
    return bits


def _paths(c, parents):
    """The accepted nodes of each row: a path from the root, at most `depth` long."""
    r = random.Random(c["sizes"] + 1)
    out = []
    for ps in parents:
        node, path = r.randrange(len(ps) // 2, len(ps)), []
        while node >= 0:
            path.append(node)
            node = ps[node]
        out.append(path[::-1][:r.choice([0, c["depth"], c["depth"], c["depth"]])])
    return out


def _page_sizes(c):
    """Tokens that each row holds, and is to hold."""
    r = random.Random(c["sizes"])
    old, new = [], []
    for _ in range(c["rows"]):
        n = r.randint(c["old_lo"], c["old_hi"])
        if r.random() < c["shrink"]:
            old.append(n)
            new.append(0 if r.random() < c["admit"] else max(0, n - r.randint(1, 64)))
        else:
            old.append(0 if r.random() < c["admit"] else n)
            new.append(old[-1] + r.randint(c["grow_lo"], c["grow_hi"]))
    return old, new


def _pages_of(n):
    return (n + BLOCK - 1) // BLOCK


def work(c):
    if c["kind"] == "pages":
        old, new = _page_sizes(c)
        moved = sum(abs(_pages_of(b) - _pages_of(a)) for a, b in zip(old, new))
        slots = sum(max(0, b - a) for a, b in zip(old, new))
        # lengths read, lengths and offsets written; a page's id read and written; a slot written
        return {"bytes": 16.0 * c["rows"] + 8.0 * moved + 4.0 * slots, "flops": 0.0}
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if c["kind"] == "prompt":
        pairs, total = 0, 0
        for length in _prompt_lens(c):
            for p, (shared, start) in enumerate(_ranges(c)[total:total + length]):
                both = max(0, min(shared, p + 1) - start)          # seen through either
                pairs += min(shared, length) + max(0, p + 1 - start) - both
            total += length
        by = total * (4.0 * d * (hq + hkv) + 8) + (4.0 * hq * total if c["lse"] else 0)
        return {"bytes": by, "flops": 4.0 * d * hq * pairs}
    prior, parents = _tree_sizes(c)
    if c["kind"] == "keep":
        moved = sum(sum(i != n for i, n in enumerate(p)) for p in _paths(c, parents))
        return {"bytes": 8.0 * hkv * d * moved + 8.0 * c["rows"] + 4.0 * moved, "flops": 0.0}
    pairs = sum(n * len(ps) + sum(bin(b).count("1") for b in _ancestors(ps))
                for n, ps in zip(prior, parents))
    nodes = sum(map(len, parents))
    keys = sum(prior) + nodes
    return {"bytes": 4.0 * d * (keys * hkv + nodes * hq) + keys / 4.0 + 8.0 * nodes,
            "flops": 4.0 * d * hq * pairs}


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
        return torch.randn(shape, generator=self.g, device="cuda").to(torch.bfloat16)

    def pages(self, lens, blocks, width):
        """A block table for rows of these lengths over a pool of `blocks` pages in
        random order, and the pages that no row holds."""
        n = torch.tensor([_pages_of(x) for x in lens], device="cuda")
        perm = torch.randperm(blocks, generator=self.g, device="cuda").to(torch.int32)
        table = torch.zeros((len(lens), width), dtype=torch.int32, device="cuda")
        table[torch.arange(width, device="cuda")[None, :] < n[:, None]] = perm[:int(n.sum())]
        return table, perm[int(n.sum()):]


def _prepare_pages(c, rng):
    old, new = _page_sizes(c)
    held = sum(map(_pages_of, old))
    need = sum(_pages_of(max(a, b)) for a, b in zip(old, new))
    blocks = need + need // 8 + 1
    table, free = rng.pages(old, blocks, _pages_of(max(map(max, zip(old, new)))) + 1)
    stack = torch.zeros(blocks, dtype=torch.int32, device="cuda")
    stack[:blocks - held] = free
    tokens = sum(max(0, b - a) for a, b in zip(old, new))
    s = dict(table=table, stack=stack, free=_i32([blocks - held]), old=_i32(old), new=_i32(new),
             tokens=tokens + 5)                 # a capacity that the tokens need not fill
    s.update(free_out=torch.empty_like(s["free"]), granted=torch.empty_like(s["free"]),
             lens=torch.empty_like(s["old"]), cu=_i32([0] * (len(old) + 1)),
             slots=torch.empty(s["tokens"], dtype=torch.int32, device="cuda"))
    return s


def _prepare_cache(c, rng):
    prior, parents = _tree_sizes(c)
    kv = [p + len(ps) for p, ps in zip(prior, parents)]
    need = sum(map(_pages_of, kv))
    blocks = need + need // 4 + 1
    table, _ = rng.pages(kv, blocks, _pages_of(max(kv)))
    shape = (blocks, c["hkv"], BLOCK, c["d"])
    return prior, parents, dict(table=table, kv=_i32(kv), prior=_i32(prior), k_cache=rng.normal(*shape),
                                v_cache=rng.normal(*shape), max_kv=max(kv))


def _prepare_tree(c, rng):
    _, parents, s = _prepare_cache(c, rng)
    words = (max(map(len, parents)) + 63) // 64
    rows = [[b >> 64 * w & (1 << 64) - 1 for w in range(words)] for ps in parents
            for b in _ancestors(ps)]
    rows = [[x - (1 << 64) if x >> 63 else x for x in r] for r in rows]
    s.update(mask=torch.tensor(rows, dtype=torch.int64, device="cuda"),
             cu=_cu(list(map(len, parents))), max_nodes=max(map(len, parents)),
             q=rng.normal(len(rows), c["hq"], c["d"]), scale=1.0 / math.sqrt(c["d"]))
    s["o"] = torch.empty_like(s["q"])
    if own:                                     # what the serving program keeps for its steps
        from paper_2412_10543_amd import binding
        n = binding.rag_attn_decode_tree_workspace_size(c["rows"], s["max_nodes"], c["hq"], c["hkv"],
                                                        c["d"], s["table"].shape[1])
        s["ws"] = torch.zeros(n, dtype=torch.uint8, device="cuda") if n else None
    return s


def _prepare_keep(c, rng):
    _, parents, s = _prepare_cache(c, rng)
    paths = _paths(c, parents)
    width = max(1, max(map(len, paths)))
    s.update(kept=_i32([p + [-1] * (width - len(p)) for p in paths]),
             num_kept=_i32(list(map(len, paths))))
    return s


def _prepare_prompt(c, rng):
    lens = _prompt_lens(c)
    total = sum(lens)
    s = dict(q=rng.normal(total, c["hq"], c["d"]), k=rng.normal(total, c["hkv"], c["d"]),
             v=rng.normal(total, c["hkv"], c["d"]), cu=_cu(lens), lens=lens, max_len=max(lens),
             ranges=_i32(_ranges(c)), scale=1.0 / math.sqrt(c["d"]))
    s["o"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((c["hq"], total), device="cuda") if c["lse"] else None
    return s


def prepare(c, seed):
    rng = _Draw(seed)
    s = {"pages": _prepare_pages, "tree": _prepare_tree, "keep": _prepare_keep,
         "prompt": _prepare_prompt}[c["kind"]](c, rng)
    s["kind"] = c["kind"]
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _plain_pages(s):
    old, new, table, stack = s["old"].long(), s["new"].long(), s["table"], s["stack"]
    (rows, width), blocks, n = table.shape, s["stack"].numel(), s["free"][0].long()
    held, want = (old + BLOCK - 1) // BLOCK, (new + BLOCK - 1) // BLOCK
    page = torch.arange(width, device="cuda")

    def before(x):                              # the sum of the rows above
        return (x.cumsum(0) - x)[:, None]

    # pages given back go behind the stack's, rows in order, pages in order
    back = (held - want).clamp(min=0)
    at = torch.where((page >= want[:, None]) & (page < held[:, None]),
                     n + before(back) + page - want[:, None], blocks)
    pile = torch.cat([stack, stack[:1]]).scatter(0, at.reshape(-1), table.reshape(-1))
    avail = n + back.sum()
    grow, tokens = (want - held).clamp(min=0), (new - old).clamp(min=0)
    fits = (grow.cumsum(0) <= avail) & (want <= width) & (tokens.cumsum(0) <= s["tokens"])
    # rows from the first that does not fit on get nothing
    ok = (fits | (tokens == 0)).long().cumprod(0)
    grow, tokens = grow * ok, tokens * ok
    lens = torch.where(ok.bool() | (new < old), new, old)
    nth = before(grow) + page - held[:, None]
    taken = (page >= held[:, None]) & (page < (held + grow)[:, None])
    table = torch.where(taken, pile[(avail - 1 - nth).clamp(0, blocks - 1)], table)
    left = avail - grow.sum()
    i = torch.arange(blocks, device="cuda")
    stack = torch.where((i >= n) & (i < left), pile[:blocks], stack)
    cu = torch.cat([tokens.new_zeros(1), tokens.cumsum(0)])
    i = torch.arange(s["tokens"], device="cuda")
    row = (torch.searchsorted(cu, i, right=True) - 1).clamp(max=rows - 1)
    key = i - cu[row] + old[row]
    slots = table[row, (key // BLOCK).clamp(max=width - 1)] * BLOCK + key % BLOCK
    slots = torch.where(i < cu[rows], slots, -1)
    return dict(table=table, stack=stack, free=left.int().reshape(1), lens=lens.int(), cu=cu.int(),
                slots=slots.int(), granted=ok.sum().int().reshape(1))


def _attend(q, k, v, seen, scale):
    """q [.., rows, d], k and v [.., keys, d], seen [.., rows, keys]: softmax over
    the seen keys, zero where none is, and the log of the sum."""
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()) * scale
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    return out, (top + torch.log(total)).squeeze(-1)


def _plain_tree(s):
    table, kv, q = s["table"].long(), s["kv"].long(), s["q"]
    hkv, d = s["k_cache"].shape[1], q.shape[2]
    rows, nodes, group = kv.numel(), s["max_nodes"], q.shape[1] // hkv
    cu = s["cu"].long()
    count = cu[1:] - cu[:-1]

    def dense(cache):                           # [rows, hkv, keys, d], fp32
        x = cache[table.reshape(-1)].reshape(rows, -1, hkv, BLOCK, d)
        return x.transpose(1, 2).reshape(rows, hkv, -1, d).float()

    k, v = dense(s["k_cache"]), dense(s["v_cache"])
    node, key = torch.arange(nodes, device="cuda"), torch.arange(k.shape[2], device="cuda")
    real = node < count[:, None]                                   # [rows, nodes]
    at = torch.where(real, cu[:-1, None] + node, torch.zeros_like(real, dtype=torch.long))
    prior = (kv - count)[:, None]
    j = key[None, :] - prior                                       # the key's node, or below 0
    word = (j.clamp(0, nodes - 1) // 64)[:, None, :].expand(-1, nodes, -1)
    bit = s["mask"][at].gather(2, word) >> (j.clamp(min=0) % 64)[:, None, :] & 1
    seen = (j[:, None, :] < 0) | (bit.bool() & (j < count[:, None])[:, None, :])
    seen = (seen & (key < kv[:, None])[:, None, :])[:, None]
    qx = q[at].float().reshape(rows, nodes, hkv, group, d).permute(0, 2, 3, 1, 4)
    seen = seen.expand(-1, group, -1, -1).reshape(rows, 1, group * nodes, -1)
    o, _ = _attend(qx.reshape(rows, hkv, group * nodes, d), k, v, seen, s["scale"])
    o = o.reshape(rows, hkv, group, nodes, d).permute(0, 3, 1, 2, 4)
    return o.reshape(rows, nodes, hkv * group, d)[real].to(q.dtype)


def _plain_keep(s):
    table, kept, base = s["table"].long(), s["kept"].long(), s["prior"].long()[:, None]
    i = torch.arange(kept.shape[1], device="cuda")[None, :].expand_as(kept)
    real = i < s["num_kept"][:, None]
    row = torch.arange(table.shape[0], device="cuda")[:, None].expand_as(kept)[real]
    src, dst = (base + kept)[real], (base + i)[real]
    sp, dp = table[row, src // BLOCK], table[row, dst // BLOCK]
    for cache in (s["k_cache"], s["v_cache"]):
        cache[dp, :, dst % BLOCK] = cache[sp, :, src % BLOCK]      # read whole, then written
    return [s["k_cache"], s["v_cache"]]


def _plain_prompt(s):
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    hq, hkv = q.shape[1], k.shape[1]
    group, outs, sums, at = hq // hkv, [], [], 0
    for n in s["lens"]:                         # ragged prompts: one after another
        key = torch.arange(n, device="cuda")
        shared, start = s["ranges"][at:at + n].long().unbind(1)
        seen = (key < shared[:, None]) | ((key >= start[:, None]) & (key <= key[:, None]))
        heads = [_attend(q[at:at + n, h * group:(h + 1) * group].transpose(0, 1).contiguous(),
                         k[at:at + n, h].contiguous(), v[at:at + n, h].contiguous(), seen, s["scale"])
                 for h in range(hkv)]           # the scores of all heads would not fit
        outs.append(torch.cat([o for o, _ in heads]).transpose(0, 1))
        sums.append(torch.cat([x for _, x in heads]))
        at += n
    o = torch.cat(outs).to(s["q"].dtype)
    return [o] if s["lse"] is None else [o, torch.cat(sums, 1)]


def run(s):
    if not own:
        return {"pages": _plain_pages, "tree": _plain_tree, "keep": _plain_keep,
                "prompt": _plain_prompt}[s["kind"]](s)
    from paper_2412_10543_amd import binding
    if s["kind"] == "pages":
        binding.rag_kv_pages_update(s["table"], s["stack"], s["free"], s["old"], s["new"],
                                    s["free_out"], s["lens"], s["cu"], s["slots"], s["granted"])
        return dict(table=s["table"], stack=s["stack"], free=s["free_out"], lens=s["lens"],
                    cu=s["cu"], slots=s["slots"], granted=s["granted"])
    if s["kind"] == "tree":
        binding.rag_attn_decode_paged_tree(s["q"], s["k_cache"], s["v_cache"], s["o"], s["mask"],
                                           s["table"], s["kv"], s["cu"], s["max_nodes"], s["scale"],
                                           workspace=s["ws"])
        return s["o"]
    if s["kind"] == "keep":
        binding.rag_kv_cache_keep(s["k_cache"], s["v_cache"], s["table"], s["prior"], s["kept"],
                                  s["num_kept"])
        return [s["k_cache"], s["v_cache"]]
    binding.rag_attn_prefill_varlen_ranges(s["q"], s["k"], s["v"], s["o"], s["lse"], s["cu"], s["cu"],
                                           s["ranges"], s["max_len"], s["max_len"], s["scale"])
    return [s["o"]] if s["lse"] is None else [s["o"], s["lse"]]


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def _rows_of(q, k, v, seen, scale):
    """One head: q [rows, d], k and v [keys, d], seen [rows, keys], float64.  The
    log of the sum first, the weights from it."""
    x = q @ k.t().contiguous() * scale
    x = torch.where(seen, x, torch.full_like(x, -math.inf))
    lse = torch.logsumexp(x, 1)
    p = torch.where(seen, torch.exp(x - lse[:, None]), torch.zeros_like(x))
    return p @ v, lse


def exact(c, seed):
    if c["kind"] == "pages":
        return None                             # whole numbers
    s = prepare(c, seed)
    if c["kind"] == "keep":
        prior, parents = _tree_sizes(c)
        table = s["table"].tolist()
        out = [s["k_cache"].double(), s["v_cache"].double()]
        for r, path in enumerate(_paths(c, parents)):
            for i, node in enumerate(path):     # a later node lies behind every earlier place
                a, b = prior[r] + node, prior[r] + i
                for x in out:
                    x[table[r][b // BLOCK], :, b % BLOCK] = x[table[r][a // BLOCK], :, a % BLOCK]
        return out
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    o = torch.zeros((s["q"].shape[0], hq, d), dtype=torch.float64, device="cuda")
    if c["kind"] == "tree":
        prior, parents = _tree_sizes(c)
        at = 0
        for r, (n, ps) in enumerate(zip(prior, parents)):
            m, keys = len(ps), n + len(ps)
            seen = torch.ones((m, keys), dtype=torch.bool)
            seen[:, n:] = torch.tensor([[b >> j & 1 for j in range(m)] for b in _ancestors(ps)]).bool()
            seen = seen.cuda()
            pages = s["table"][r, :_pages_of(keys)].long()
            for h in range(hkv):
                k, v = (x[pages, h].reshape(-1, d)[:keys].double() for x in (s["k_cache"], s["v_cache"]))
                for g in range(hq // hkv):
                    y = h * (hq // hkv) + g
                    o[at:at + m, y] = _rows_of(s["q"][at:at + m, y].double(), k, v, seen, s["scale"])[0]
            at += m
        return o
    lse = torch.zeros((hq, o.shape[0]), dtype=torch.float64, device="cuda")
    at = 0
    for n in s["lens"]:
        spans = s["ranges"][at:at + n].double()
        key = torch.arange(n, device="cuda", dtype=torch.float64)
        seen = (key[None] < spans[:, :1]) | ((key[None] >= spans[:, 1:]) & (key[None] <= key[:, None]))
        for y in range(hq):
            h = y // (hq // hkv)
            k, v = s["k"][at:at + n, h].double(), s["v"][at:at + n, h].double()
            o[at:at + n, y], lse[y, at:at + n] = _rows_of(s["q"][at:at + n, y].double(), k, v, seen,
                                                          s["scale"])
        at += n
    return [o] if s["lse"] is None else [o, lse]
