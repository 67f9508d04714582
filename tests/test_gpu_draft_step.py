"""The serving operators together, as a loop of speculative decoding over stuffed
prompts runs them: pages taken for the prompts, their rows attending with the
documents apart, their K/V written; then step after step pages and slots for
drafted trees, their K/V written, the trees' attention, the accepted paths
kept, the other pages given back.  Every output is checked in 64 bits against
dense keys; the same steps captured in HIP graphs and replayed give the eager
bits, tables and lengths."""
import math
import random

import pytest
import torch

import draft_support as ds
from paper_2412_10543_amd import binding
from paper_2412_10543_amd.workloads import normal_bf16

pytestmark = pytest.mark.gpu

i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

HQ, HKV, D = 8, 2, 128
SCALE = 1.0 / math.sqrt(D)
PROMPTS = [(17, [100, 33], 20), (0, [250], 9), (64, [40, 40, 40], 1)]    # system prompt, documents, query
S, MAX_NODES, MAX_KEPT, WIDTH, BLOCKS = 3, 20, 6, 30, 70
CAPACITY = S * MAX_NODES


def capture(fn):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            fn()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    return g


class Server:
    """Caches, page tables and the buffers of a step, all on the GPU."""

    def __init__(self):
        self.kc = torch.full((BLOCKS, HKV, 16, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.vc = self.kc.clone()
        self.table = torch.zeros((S, WIDTH), dtype=torch.int32, device="cuda")
        self.stack = i32(random.Random(1).sample(range(BLOCKS), BLOCKS))
        self.free, self.free2, self.free3 = i32([BLOCKS]), i32([0]), i32([0])
        self.lens, self.wanted, self.held, self.after = (i32([0] * S) for _ in range(4))
        self.cu, self.cu2, self.granted = i32([0] * (S + 1)), i32([0] * (S + 1)), i32([0])
        self.slots, self.none = i32([0] * CAPACITY), i32([])
        self.q = torch.zeros((CAPACITY, HQ, D), dtype=torch.bfloat16, device="cuda")
        self.k = torch.zeros((CAPACITY, HKV, D), dtype=torch.bfloat16, device="cuda")
        self.v, self.o = self.k.clone(), torch.full_like(self.q, 7.0)
        self.mask = torch.zeros((CAPACITY, 1), dtype=torch.int64, device="cuda")
        self.nodes, self.num_kept = i32([0] * S), i32([0] * S)
        self.kept = i32([[0] * MAX_KEPT] * S)
        n = binding.rag_attn_decode_tree_workspace_size(S, MAX_NODES, HQ, HKV, D, WIDTH, num_splits=3)
        assert n > 0
        self.ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")

    def admit(self, k, v, lens):
        tokens = k.shape[0]
        slots, new = i32([0] * tokens), i32(lens)
        binding.rag_kv_pages_update(self.table, self.stack, self.free, self.lens, new, self.free2,
                                    self.held, self.cu, slots, self.granted)
        binding.rag_kv_cache_write(k, v, self.kc, self.vc, slots)
        self.free.copy_(self.free2)
        self.lens.copy_(self.held)

    def step(self):
        """Reads q, k, v, mask, nodes, kept and num_kept; writes o."""
        torch.add(self.lens, self.nodes, out=self.wanted)
        binding.rag_kv_pages_update(self.table, self.stack, self.free, self.lens, self.wanted,
                                    self.free2, self.held, self.cu, self.slots, self.granted)
        binding.rag_kv_cache_write(self.k, self.v, self.kc, self.vc, self.slots)
        binding.rag_attn_decode_paged_tree(self.q, self.kc, self.vc, self.o, self.mask, self.table,
                                           self.held, self.cu, MAX_NODES, SCALE, num_splits=3,
                                           workspace=self.ws)
        binding.rag_kv_cache_keep(self.kc, self.vc, self.table, self.lens, self.kept, self.num_kept)
        torch.add(self.lens, self.num_kept, out=self.after)
        binding.rag_kv_pages_update(self.table, self.stack, self.free2, self.held, self.after,
                                    self.free3, self.lens, self.cu2, self.none, self.granted)
        self.free.copy_(self.free3)

    def state(self):
        free = self.free.item()
        return dict(lens=self.lens.tolist(), free=free, stack=self.stack[:free].tolist(),
                    pages=[self.table[s, :ds.pages_of(n)].tolist()
                           for s, n in enumerate(self.lens.tolist())], cu=self.cu.tolist())


class Draft:
    """A step's trees and accepted paths."""

    def __init__(self, seed):
        rng = random.Random(seed)
        counts = [rng.choice([0, 1, 5, 12, MAX_NODES]) for _ in range(S)]
        counts[seed % S] = MAX_NODES
        self.parents = [ds.tree_parents(rng, n) if n else [] for n in counts]
        self.seen = [ds.ancestor_seen(p) if p else torch.zeros((0, 0), dtype=torch.bool)
                     for p in self.parents]
        self.counts, self.paths = counts, []
        for p in self.parents:
            node, path = rng.randrange(len(p)) if p else -1, []
            while node >= 0:
                path.insert(0, node)
                node = p[node]
            self.paths.append(path[:rng.randint(0, MAX_KEPT)])
        n = sum(counts)
        self.q = normal_bf16((CAPACITY, HQ, D), seed + 1, "cuda")
        self.k = normal_bf16((CAPACITY, HKV, D), seed + 2, "cuda")
        self.v = normal_bf16((CAPACITY, HKV, D), seed + 3, "cuda")
        self.mask = torch.zeros((CAPACITY, 1), dtype=torch.int64, device="cuda")
        self.mask[:n] = ds.mask_words(self.seen, 1).cuda()
        self.tokens = n

    def put(self, server):
        server.q.copy_(self.q)
        server.k.copy_(self.k)
        server.v.copy_(self.v)
        server.mask.copy_(self.mask)
        server.nodes.copy_(i32(self.counts))
        server.kept.copy_(i32([p + [-1] * (MAX_KEPT - len(p)) for p in self.paths]))
        server.num_kept.copy_(i32([len(p) for p in self.paths]))


class Dense:
    """The sequences' keys and values in plain lists."""

    def __init__(self, k, v, lens):
        self.k, self.v, at = [], [], 0
        for n in lens:
            self.k.append(k[at:at + n].cpu())
            self.v.append(v[at:at + n].cpu())
            at += n

    def step(self, draft):
        o = torch.zeros((draft.tokens, HQ, D), dtype=torch.float64)
        b, at = torch.zeros_like(o), 0
        for s, n in enumerate(draft.counts):
            k, v = (torch.cat([old[s], new[at:at + n].cpu()])
                    for old, new in ((self.k, draft.k), (self.v, draft.v)))
            prior = len(self.k[s])
            seen = torch.cat([torch.ones((n, prior), dtype=torch.bool), draft.seen[s]], 1)
            for h in range(HQ if n else 0):
                g = h // (HQ // HKV)
                o[at:at + n, h], _, b[at:at + n, h], _ = ds.attend64(
                    draft.q[at:at + n, h], k[:, g], v[:, g], seen, SCALE)
            keep = list(range(prior)) + [prior + i for i in draft.paths[s]]
            self.k[s], self.v[s] = k[keep], v[keep]
            at += n
        return o, b


def prompts():
    lens = [s + sum(d) + q for s, d, q in PROMPTS]
    rows = []
    for s, docs, query in PROMPTS:
        at = s
        rows += [(0, 0)] * s
        for n in docs:
            rows += [(s, at)] * n
            at += n
        rows += [(0, 0)] * query
    n = sum(lens)
    return lens, i32(rows), normal_bf16((n, HQ, D), 1, "cuda"), normal_bf16((n, HKV, D), 2, "cuda"), \
        normal_bf16((n, HKV, D), 3, "cuda")


def cu_of(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return i32(out)


def test_steps_against_dense_keys():
    lens, ranges, q, k, v = prompts()
    o = torch.empty_like(q)
    binding.rag_attn_prefill_varlen_ranges(q, k, v, o, None, cu_of(lens), cu_of(lens), ranges,
                                           max(lens), max(lens), SCALE)
    w = ds.reference_ranges(q, k, v, lens, lens, ranges, SCALE)
    ds.within(o, w[0], w[2], "prompts")
    server, dense = Server(), Dense(k, v, lens)
    server.admit(k, v, lens)
    assert server.granted.item() == S
    for i in range(6):
        draft = Draft(10 * i)
        draft.put(server)
        server.o.fill_(7.0)
        server.step()
        want, bound = dense.step(draft)
        torch.cuda.synchronize()
        ds.within(server.o[:draft.tokens], want, bound, f"step {i}")
        assert (server.o[draft.tokens:] == 7.0).all()
        state = server.state()
        assert state["lens"] == [len(x) for x in dense.k]
        assert sorted(state["stack"] + sum(state["pages"], [])) == list(range(BLOCKS))
        for s in range(S):
            n = len(dense.k[s])
            assert torch.equal(ds.dense_keys(server.kc, server.table, s, n), dense.k[s])
            assert torch.equal(ds.dense_keys(server.vc, server.table, s, n), dense.v[s])


def test_captured_steps_are_the_eager_ones():
    """Two servers' steps in two graphs, each with its workspace, replayed in turn and
    at once; a third server runs eagerly."""
    lens, ranges, q, k, v = prompts()
    eager, one, two = Server(), Server(), Server()
    o, o2, cu = torch.empty_like(q), torch.empty_like(q), cu_of(lens)

    def prefill(out):
        binding.rag_attn_prefill_varlen_ranges(q, k, v, out, None, cu, cu, ranges, max(lens),
                                               max(lens), SCALE)

    prefill(o)
    for s in (eager, one, two):
        s.admit(k, v, lens)
    torch.cuda.synchronize()
    graphs = [capture(one.step), capture(two.step)]
    fill = capture(lambda: prefill(o2))
    side = torch.cuda.Stream()
    for i in range(5):
        print(f"replay {i}", flush=True)
        draft = Draft(7 * i + 1)
        for s in (eager, one, two):
            draft.put(s)
            s.o.fill_(7.0)
        o2.zero_()
        eager.step()
        torch.cuda.synchronize()
        graphs[0].replay()
        if i % 2:
            torch.cuda.synchronize()
            graphs[1].replay()
        else:
            with torch.cuda.stream(side):
                graphs[1].replay()
        fill.replay()
        torch.cuda.synchronize()
        for s in (one, two):
            assert torch.equal(s.o, eager.o) and s.state() == eager.state()
        assert torch.equal(o, o2)
