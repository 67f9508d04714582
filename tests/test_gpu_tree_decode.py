"""rag_attn_decode_paged_tree on the GPU against 64 bits, element by element
within the bound that the arithmetic gives (draft_support)."""
import math
import random

import pytest
import torch

import draft_support as ds
from paper_2412_10543_amd import binding
from paper_2412_10543_amd.workloads import normal_bf16, paged_pool

pytestmark = pytest.mark.gpu

i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731


class Case:
    def __init__(self, priors, seen, hq, hkv, d, seed, q_scale=1.0, words=None, fill=0, poison=True,
                 max_blocks=None):
        self.seen, self.hq, self.hkv, self.d = seen, hq, hkv, d
        self.n = [x.shape[0] for x in seen]
        self.kv = [p + n for p, n in zip(priors, self.n)]
        self.pool = paged_pool([max(x, 1) for x in self.kv], hkv, d, seed, device="cuda", poison=poison,
                               max_blocks=max_blocks)
        self.q = normal_bf16((sum(self.n), hq, d), seed + 5, "cuda", q_scale)
        self.max_nodes = max(self.n + [1])
        words = (self.max_nodes + 63) // 64 if words is None else words
        self.mask = ds.mask_words(seen, words, fill).cuda()
        self.cu = [0]
        for n in self.n:
            self.cu.append(self.cu[-1] + n)
        self.scale = 1.0 / math.sqrt(d)

    def workspace(self, splits=0):
        n = binding.rag_attn_decode_tree_workspace_size(
            len(self.n), self.max_nodes, self.hq, self.hkv, self.d, self.pool.block_tables.shape[1],
            num_splits=splits)
        return torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None   # NaN

    def run(self, splits=0, ws="own", stream=None, o=None):
        o = torch.full_like(self.q, float("nan")) if o is None else o
        binding.rag_attn_decode_paged_tree(
            self.q, self.pool.k_cache, self.pool.v_cache, o, self.mask, self.pool.block_tables,
            i32(self.kv), i32(self.cu), self.max_nodes, self.scale, num_splits=splits,
            workspace=self.workspace(splits) if isinstance(ws, str) else ws, stream=stream)
        return o

    def want(self):
        return ds.reference_tree(self.q, self.pool.k_cache, self.pool.v_cache, self.pool.block_tables,
                                 self.kv, self.seen, self.scale)

    def check(self, splits=(0,)):
        o, b = self.want()
        for s in splits:
            got = self.run(s)
            torch.cuda.synchronize()
            ds.within(got, o, b, f"splits {s}")


def trees(rng, counts):
    return [ds.ancestor_seen(ds.tree_parents(rng, n)) if n else torch.zeros((0, 0), dtype=torch.bool)
            for n in counts]


HEADS = [(4, 2, 64), (32, 8, 128), (8, 8, 128), (20, 4, 128), (14, 2, 64), (32, 2, 128), (3, 3, 64),
         (25, 1, 128)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("nodes", [1, 2, 9, 16, 17, 33])
def test_trees_of_every_shape(hq, hkv, d, nodes):
    rng = random.Random(nodes * 31 + hq)
    Case([0, 1, 47, 150], trees(rng, [nodes] * 4), hq, hkv, d, nodes + hq).check((0, 3))


@pytest.mark.parametrize("prior", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 500, 1033])
def test_every_place_of_the_nodes_in_their_pages(prior):
    rng = random.Random(prior)
    Case([prior, prior + 7], trees(rng, [20, 5]), 8, 2, 128, prior).check((0, 1, 2, 64))


@pytest.mark.parametrize("nodes", [63, 64, 65, 100, 128, 130, 300])
def test_large_trees(nodes):
    rng = random.Random(nodes)
    Case([200, 3], trees(rng, [nodes, nodes // 2]), 8, 2, 64, nodes).check((0, 1, 4))


def test_ragged_batch_with_empty_sequences():
    rng = random.Random(8)
    Case([300, 0, 33, 0, 900, 16], trees(rng, [7, 0, 64, 1, 0, 12]), 16, 4, 128, 8).check((0, 1, 5))


@pytest.mark.parametrize("seed", range(4))
def test_any_mask(seed):
    """Bits that no tree has: rows that see nothing of the nodes (and nothing at
    all, without keys before them), rows that see later nodes; bits behind the
    nodes and spare words are ignored."""
    g = torch.Generator().manual_seed(seed)
    seen = [torch.rand((n, n), generator=g) < p for n, p in ((40, 0.3), (12, 0.1), (70, 0.9), (5, 0.0))]
    seen[0][3] = False
    c = Case([0, 20, 0, 0], seen, 8, 2, 128, seed, words=3, fill=-1)
    c.check((0, 2))
    o = c.run()
    torch.cuda.synchronize()
    assert (o[3] == 0).all() and (o[-5:] == 0).all()


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("side", ["k", "v"])
@pytest.mark.parametrize("prior,hq", [(50, 8), (50, 32), (0, 8)])
def test_unseen_values_never_arrive(value, side, prior, hq):
    """A node holds `value`: the rows that see it may, no other row does."""
    rng = random.Random(6)
    parents = [-1, 0, 0, 1, 2, 3, 4, -1, 7, 8] + [rng.randint(-1, 9) for _ in range(20)]
    c = Case([prior], [ds.ancestor_seen(parents)], hq, 2, 128, 6)
    cache = c.pool.k_cache if side == "k" else c.pool.v_cache
    for node in (2, 9, 13):
        at = prior + node
        cache[c.pool.block_tables[0, at // 16].long(), :, at % 16, 5] = value
    o, b = c.want()
    assert torch.isnan(b).any() and not torch.isnan(b).all()
    for s in (0, 1, 2):
        got = c.run(s)
        torch.cuda.synchronize()
        ds.within(got, o, b)
        if math.isnan(value):
            seeing = torch.isnan(b[:, 0, 0])
            assert torch.isnan(got[seeing.cuda()].float()).any(-1).all()


def test_unseen_values_where_a_workgroup_has_several_sequences():
    """Wide tables, short and long sequences: shares end in one and begin in another,
    some of them with values that must not arrive."""
    rng = random.Random(12)
    counts = [9, 1, 30, 0, 17, 64, 3, 5]
    c = Case([50, 20, 0, 70, 7, 700, 33, 400], trees(rng, counts), 8, 8, 128, 12, max_blocks=256)
    for s, node in ((0, 4), (2, 11), (4, 2), (5, 40), (7, 1)):
        at = c.kv[s] - counts[s] + node
        for cache, value in ((c.pool.v_cache, math.nan), (c.pool.k_cache, math.inf)):
            cache[c.pool.block_tables[s, at // 16].long(), :, at % 16, 9] = value
    o, b = c.want()
    assert 0 < torch.isnan(b).double().mean() < 0.8
    for s in (0, 2):
        got = c.run(s)
        torch.cuda.synchronize()
        ds.within(got, o, b, f"splits {s}")


@pytest.mark.parametrize("q_scale", [0.0, 8.0, 40.0])
def test_flat_and_peaky_scores(q_scale):
    rng = random.Random(1)
    Case([700, 90], trees(rng, [30, 64]), 8, 2, 128, 4, q_scale=q_scale).check((0, 1, 3))


def test_one_node_is_a_decode_row():
    rng = random.Random(2)
    kv = [1, 17, 400, 1200]
    c = Case([n - 1 for n in kv], trees(rng, [1] * 4), 32, 8, 128, 12)
    c.check((0, 2))
    o = torch.empty_like(c.q)
    n = binding.rag_attn_decode_workspace_size(4, 32, 8, 128, c.pool.block_tables.shape[1])
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda") if n else None
    binding.rag_attn_decode_paged(c.q, c.pool.k_cache, c.pool.v_cache, o, c.pool.block_tables,
                                  i32(kv), c.scale, workspace=ws)
    want, b = c.want()
    torch.cuda.synchronize()
    ds.within(o, want, b)


@pytest.mark.parametrize("rows", [64, 65, 130, 256, 257])
def test_batches_of_many_sequences(rows):
    """The cuts are made from 64 lengths at a time; with more than 256 none are."""
    rng = random.Random(rows)
    counts = [rng.choice([0, 1, 2, 5, 9]) for _ in range(rows)]
    priors = [rng.choice([0, 3, rng.randint(0, 90), rng.randint(0, 400)]) for _ in range(rows)]
    priors[rows // 2], priors[rows - 1], counts[rows - 1] = 5000, 1700, 4
    Case(priors, trees(rng, counts), 2, 1, 64, rows).check((0, 2))


@pytest.mark.parametrize("rows,hkv", [(64, 8), (65, 8), (200, 4), (256, 8)])
def test_a_few_long_sequences_among_many_short_ones(rows, hkv):
    """Alone the short ones are units enough; the long ones are cut all the same, and
    their partials have the workspace to themselves."""
    rng = random.Random(rows + hkv)
    counts = [rng.choice([0, 1, 2, 4]) for _ in range(rows)]
    priors = [rng.choice([0, 5, rng.randint(0, 70)]) for _ in range(rows)]
    for s, n in ((0, 3000), (rows // 3, 1100), (rows - 1, 2100)):
        priors[s], counts[s] = n, 5
    c = Case(priors, trees(rng, counts), hkv, hkv, 64, rows)
    assert 0 < c.workspace().numel() < 1 << 25
    c.check()


@pytest.mark.parametrize("hq,hkv,d", [(25, 1, 128), (28, 4, 64)])
def test_joins_of_many_rows(hq, hkv, d):
    """More rows than waves fit on the chip: a wave joins several, the last fewer."""
    rng = random.Random(hq)
    Case([900, 40, 2000, 300], trees(rng, [101, 3, 90, 51]), hq, hkv, d, hq).check((0, 5, 64))


def test_wide_table_and_long_context():
    rng = random.Random(3)
    Case([9000, 40, 2500], trees(rng, [25, 60, 3]), 8, 2, 128, 21, max_blocks=2300).check((0, 64))


def test_same_bits_every_time_and_in_any_page_order():
    rng = random.Random(4)
    c = Case([1000, 333], trees(rng, [64, 20]), 32, 8, 128, 30, poison=False)
    a = c.run()
    b = c.run()
    assert torch.equal(a, b)
    perm = torch.randperm(c.pool.num_blocks, device="cuda")
    back = torch.argsort(perm)
    c.pool.k_cache, c.pool.v_cache = c.pool.k_cache[perm].contiguous(), c.pool.v_cache[perm].contiguous()
    c.pool.block_tables = back[c.pool.block_tables.long()].to(torch.int32).contiguous()
    assert torch.equal(a, c.run())


def test_rows_behind_the_last_sequence_stay():
    rng = random.Random(5)
    c = Case([100, 20], trees(rng, [9, 30]), 8, 2, 64, 40)
    big = torch.full((60, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    q = torch.cat([c.q, normal_bf16((21, 8, 64), 1, "cuda")])
    m = torch.cat([c.mask, torch.full((21, 1), -1, dtype=torch.int64, device="cuda")])
    c.q, c.mask = q, m
    for s in (1, 3):
        c.run(s, o=big)
        torch.cuda.synchronize()
        assert (big[39:] == 7.0).all()
        big[39:] = 7.0


def test_offsets_past_32_bits():
    """Pages whose elements lie beyond 2^32 bytes of a cache."""
    hkv, d = 8, 128
    blocks = 2 ** 32 // (hkv * 16 * d) + 40           # elements past 2^32
    c = Case([70], trees(random.Random(1), [11]), 32, hkv, d, 2)
    kc = torch.empty((blocks, hkv, 16, d), dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    ids = torch.tensor([blocks - 1, 3, blocks - 20, 2 ** 31 // (hkv * 16 * d) + 1, blocks - 7, 9],
                       device="cuda")
    old = c.pool.block_tables[0, :6].long()
    kc[ids], vc[ids] = c.pool.k_cache[old], c.pool.v_cache[old]
    want, b = c.want()
    c.pool.k_cache, c.pool.v_cache = kc, vc
    c.pool.block_tables = ids.to(torch.int32)[None].contiguous()
    for s in (1, 2):
        got = c.run(s)
        torch.cuda.synchronize()
        ds.within(got, want, b)


def test_streams_and_workspaces():
    """Two calls at once on two streams, each with its workspace; then calls of
    other sizes one after another in one of them."""
    rng = random.Random(7)
    cases = [Case([900], trees(rng, [40]), 32, 8, 128, 50), Case([500, 80], trees(rng, [9, 64]), 8, 2, 64, 51)]
    want = [c.want() for c in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        streams = [torch.cuda.Stream() for _ in cases]
        ws = [c.workspace(4) for c in cases]
        outs = [torch.empty_like(c.q) for c in cases]
        torch.cuda.synchronize()
        for c, s, w, o in zip(cases, streams, ws, outs):
            with torch.cuda.stream(s):
                c.run(4, ws=w, stream=s, o=o)
        torch.cuda.synchronize()
        for got, (o, b) in zip(outs, want):
            ds.within(got, o, b)
    shared = torch.empty(max(x.numel() for x in ws), dtype=torch.uint8, device="cuda")
    for i in (0, 1, 0, 1):
        got = cases[i].run(4, ws=shared)
        torch.cuda.synchronize()
        ds.within(got, *want[i])


def test_smaller_steps_in_the_workspace_of_the_largest():
    """One workspace for a serving program's largest step; its steps of fewer rows,
    smaller trees and narrower tables run in it."""
    rng = random.Random(13)
    n = binding.rag_attn_decode_tree_workspace_size(260, 70, 16, 8, 128, 100)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    for rows, nodes, width in ((260, 9, 33), (70, 9, 100), (63, 9, 100), (64, 8, 100), (7, 70, 100),
                               (7, 64, 100), (1, 70, 100), (1, 1, 100), (3, 16, 40), (9, 65, 31)):
        counts = [rng.randint(0, nodes) for _ in range(rows)]
        counts[-1] = nodes
        priors = [rng.choice([0, 5, rng.randint(0, min(width * 16 - nodes, 200))]) for _ in range(rows)]
        priors[0] = width * 16 - nodes
        print(f"{rows} rows of up to {nodes} nodes, {width} pages", flush=True)
        c = Case(priors, trees(rng, counts), 16, 8, 128, rows + nodes, max_blocks=width)
        want, bound = c.want()
        got = c.run(0, ws=ws)
        torch.cuda.synchronize()
        ds.within(got, want, bound, f"{rows} rows")


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (14, 2, 64)])
@pytest.mark.parametrize("splits", [0, 2, 5])
def test_nothing_is_written_behind_the_workspace(hq, hkv, d, splits):
    """Batches whose units are a chipful, and one alone, in a workspace of their size
    with other bytes behind it."""
    rng = random.Random(hq + splits)
    for priors, counts in (([2500, 30, 900, 1700], [9, 4, 16, 1]), ([3000, 2000], [70, 25]), ([1200], [3]),
                           ([700 + 40 * i for i in range(20)], [1 + i % 7 for i in range(20)])):
        c = Case(priors, trees(rng, counts), hq, hkv, d, len(priors) + hq)
        n = binding.rag_attn_decode_tree_workspace_size(len(c.n), c.max_nodes, hq, hkv, d,
                                                        c.pool.block_tables.shape[1], num_splits=splits)
        assert n > 0
        buf = torch.full((n + (1 << 20),), 90, dtype=torch.uint8, device="cuda")
        got = c.run(splits, ws=buf[:n])
        want, bound = c.want()
        torch.cuda.synchronize()
        ds.within(got, want, bound)
        assert (buf[n:] == 90).all()


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (14, 2, 64)])
@pytest.mark.parametrize("bound", [0, 20, 65, 300])
@pytest.mark.parametrize("large", [0, 128])
def test_bound_of_the_nodes_far_above_the_trees(hq, hkv, d, bound, large):
    """max_nodes of a step that is made for larger trees, and one large tree among
    small ones: row blocks that few sequences, or none, have rows in."""
    rng = random.Random(bound + large + hq)
    counts = [rng.choice([0, 1, 3, 9, 12]) for _ in range(14)]
    priors = [rng.choice([0, 40, 900, rng.randint(0, 2500)]) for _ in counts]
    counts[3], priors[3] = 5, 2500
    if large:
        counts[9], priors[9] = large, 1100
    c = Case(priors, trees(rng, counts), hq, hkv, d, bound + hq, words=5)
    c.max_nodes = max(c.max_nodes, bound)
    c.check((0, 3))


def test_refused_on_the_gpu():
    c = Case([900], trees(random.Random(7), [40]), 32, 8, 128, 50)
    with pytest.raises(binding.RagError) as e:
        c.run(4, ws=None)
    assert e.value.status == binding.RAG_ERR_WORKSPACE
    c.mask = c.mask[:-1].contiguous()
    with pytest.raises(ValueError, match="inconsistent shapes"):
        c.run(1)
