"""The operators of a decoding loop over a 4-bit cache together, as one runs them: pages and slots
for the prompts and for each step's drafted chains, the projection's rows normed, rotated and
written in 4 bits, their attention, the verification of the drafts, the other pages given back; then
a prompt's next piece over keys read back from the cache.  Every output is checked in 64 bits;
the same steps captured in HIP graphs and replayed give the eager bits, tables and lengths."""
import math
import random

import pytest
import torch

import draft_support as ds
import serve_support as ss
from paper_2412_10543_amd import binding
from paper_2412_10543_amd.workloads import normal_bf16

pytestmark = pytest.mark.gpu

i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

HQ, HKV, D, ROT, VOCAB = 8, 2, 128, 64, 1003
SCALE = 1.0 / math.sqrt(D)
PROMPTS = [100, 33, 250, 1]
S, MAX_ROWS, WIDTH, BLOCKS, MOST = 4, 6, 24, 60, 600
CAPACITY = S * MAX_ROWS + 3              # (rows behind the last sequence in every step)
QW, KW = normal_bf16((D,), 91), normal_bf16((D,), 92)
CS = ss.angles(MOST, ROT)


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


def parts(qkv):
    return qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:]


class Server:
    """Caches, page tables and the buffers of a step, all on the GPU."""

    def __init__(self, with_draft):
        g = torch.Generator().manual_seed(5)
        self.kc, self.vc = (torch.randint(0, 256, (BLOCKS, HKV, 9 * D), generator=g,
                                          dtype=torch.uint8).cuda() for _ in range(2))
        self.table = torch.zeros((S, WIDTH), dtype=torch.int32, device="cuda")
        self.stack = i32(random.Random(1).sample(range(BLOCKS), BLOCKS))
        self.free, self.free2, self.free3 = i32([BLOCKS]), i32([0]), i32([0])
        self.lens, self.wanted, self.held, self.after = (i32([0] * S) for _ in range(4))
        self.cu, self.cu2, self.granted = i32([0] * (S + 1)), i32([0] * (S + 1)), i32([0])
        self.slots, self.none = i32([0] * CAPACITY), i32([])
        self.qw, self.kw, self.cs = QW.cuda(), KW.cuda(), CS.cuda()
        self.qkv = torch.zeros((CAPACITY, HQ + 2 * HKV, D), dtype=torch.bfloat16, device="cuda")
        self.q = torch.full((CAPACITY, HQ, D), 7.0, dtype=torch.bfloat16, device="cuda")
        self.o, self.pos = torch.full_like(self.q, 7.0), i32([0] * CAPACITY)
        self.logits = torch.zeros((CAPACITY, VOCAB), device="cuda")
        self.draft = torch.zeros((CAPACITY, VOCAB), device="cuda") if with_draft else None
        self.heat = torch.tensor([0.8, 0.0, 1.2, 1.0], device="cuda")
        self.u, self.tokens = torch.zeros(CAPACITY, device="cuda"), i32([0] * CAPACITY)
        self.rows, self.num_kept, self.next = i32([0] * S), i32([0] * S), i32([0] * S)
        self.kept = i32([[0] * MAX_ROWS] * S)
        self.ws = torch.zeros(binding.rag_attn_decode_kv4_workspace_size(S, MAX_ROWS, HQ, HKV, D, WIDTH),
                              dtype=torch.uint8, device="cuda")
        self.ws2 = torch.zeros(binding.rag_draft_verify_workspace_size(CAPACITY, S, VOCAB),
                               dtype=torch.uint8, device="cuda")

    def write(self, qkv, pos, slots, q, k_out=None, v_out=None):
        binding.rag_qkv_rope_write_kv4(*parts(qkv), q, pos, self.cs, slots, self.kc, self.vc, k_out, v_out,
                                       self.qw, self.kw)

    def admit(self, qkv, lens):
        """The prompts' attention, over their unquantized rows."""
        tokens = qkv.shape[0]
        slots, new = i32([0] * tokens), i32(lens)
        pos = i32([i for n in lens for i in range(n)])
        q = torch.empty((tokens, HQ, D), dtype=torch.bfloat16, device="cuda")
        k = torch.empty((tokens, HKV, D), dtype=torch.bfloat16, device="cuda")
        v, o, cu = torch.empty_like(k), torch.empty_like(q), i32([0] * (S + 1))
        binding.rag_kv_pages_update(self.table, self.stack, self.free, self.lens, new, self.free2,
                                    self.held, cu, slots, self.granted)
        self.write(qkv, pos, slots, q, k, v)
        binding.rag_attn_prefill_varlen(q, k, v, o, None, cu, cu, max(lens), max(lens), SCALE, True)
        self.free.copy_(self.free2)
        self.lens.copy_(self.held)
        return q, k, v, o

    def step(self):
        """Reads qkv, pos, logits, tokens, draft, u, rows; writes o, kept, num_kept, next."""
        torch.add(self.lens, self.rows, out=self.wanted)
        binding.rag_kv_pages_update(self.table, self.stack, self.free, self.lens, self.wanted,
                                    self.free2, self.held, self.cu, self.slots, self.granted)
        self.write(self.qkv, self.pos, self.slots, self.q)
        binding.rag_attn_decode_paged_kv4(self.q, self.kc, self.vc, self.o, self.table, self.held, SCALE,
                                          self.cu, MAX_ROWS, self.ws)
        binding.rag_draft_verify(self.logits, self.tokens, self.cu, self.heat, self.u, self.kept,
                                 self.num_kept, self.next, draft_probs=self.draft, workspace=self.ws2)
        torch.add(self.lens, self.num_kept, out=self.after)
        binding.rag_kv_pages_update(self.table, self.stack, self.free2, self.held, self.after,
                                    self.free3, self.lens, self.cu2, self.none, self.granted)
        self.free.copy_(self.free3)

    def state(self):
        free = self.free.item()
        return dict(lens=self.lens.tolist(), free=free, stack=self.stack[:free].tolist(),
                    pages=[self.table[s, :ds.pages_of(n)].tolist()
                           for s, n in enumerate(self.lens.tolist())], cu=self.cu.tolist(),
                    kept=self.kept.tolist(), num=self.num_kept.tolist(), next=self.next.tolist())


class Draft:
    """A step's rows, logits and drafted chains."""

    def __init__(self, seed):
        r = random.Random(seed)
        self.rows = [r.choice([0, 1, 3, MAX_ROWS]) for _ in range(S)]
        self.rows[seed % S] = MAX_ROWS
        logits, self.tokens, _, self.cu, _, u, draft = ss.verify_case(seed, self.rows, VOCAB, True)
        n = self.n = len(logits)
        pad = lambda x: torch.cat([x, torch.full((CAPACITY - n,) + x.shape[1:], math.nan)])  # noqa: E731
        self.logits, self.draft, self.u = pad(logits), pad(draft), pad(u)
        self.qkv = normal_bf16((CAPACITY, HQ + 2 * HKV, D), seed + 1)

    def positions(self, lens):
        return [m + i for m, n in zip(lens, self.rows) for i in range(n)]

    def put(self, server, lens):
        server.qkv.copy_(self.qkv)
        server.logits.copy_(self.logits)
        if server.draft is not None:
            server.draft.copy_(self.draft)
        server.u.copy_(self.u)
        server.tokens.copy_(i32(self.tokens + [0] * (CAPACITY - self.n)))
        server.rows.copy_(i32(self.rows))
        server.pos.copy_(i32(self.positions(lens) + [1 << 30] * (CAPACITY - self.n)))
        server.o.fill_(7.0)
        server.q.fill_(7.0)


def turned(qkv, positions):
    """(K rows in 64 bits, their bound, V rows) of new tokens."""
    _, k, v = parts(qkv[:len(positions)].cpu())
    want, bound = ss.reference_rope(k, KW, 1e-6, torch.tensor(positions), CS, False)
    return want, bound, v.double()


def check_pages(server, history, what):
    """Every sequence's rows in its pages, half a step and what rounding the scale adds (0.56 s)
    from those of the history."""
    for s, rows in enumerate(history):
        pages = server.table[s, :ds.pages_of(len(rows[0]))].long().cpu()
        for cache, want, bound, values in ((server.kc, rows[0], rows[1], False),
                                           (server.vc, rows[2], 0 * rows[1], True)):
            got, steps = (x[pages].reshape(-1, HKV, D)[:len(want)] for x in ss.unpack(cache.cpu(), D, values))
            over = (got - want).abs() - bound - 0.5586 * steps
            assert over.max() <= 0, (what, s, over.max())


@pytest.mark.parametrize("with_draft", [False, True])
def test_steps_in_64_bits(with_draft):
    server = Server(with_draft)
    qkv = normal_bf16((sum(PROMPTS), HQ + 2 * HKV, D), 1, "cuda")
    q, k, v, o = server.admit(qkv, PROMPTS)
    assert server.granted.item() == S
    want = ds.reference_ranges(q, k, v, PROMPTS, PROMPTS, i32([(0, 0)] * sum(PROMPTS)), SCALE)
    ds.within(o, want[0], want[2], "prompts")
    new = turned(qkv, [i for n in PROMPTS for i in range(n)])
    at, history = 0, []
    for n in PROMPTS:
        history.append([x[at:at + n] for x in new])
        at += n
    check_pages(server, history, "prompts")
    for i in range(5):
        draft, lens = Draft(10 * i + 3), server.lens.tolist()
        draft.put(server, lens)
        server.step()
        torch.cuda.synchronize()
        held = [m + n for m, n in zip(lens, draft.rows)]
        n = draft.n
        assert server.cu.tolist() == draft.cu and server.held.tolist() == held
        pos = draft.positions(lens)
        want, bound = ss.reference_rope(parts(draft.qkv[:n])[0], QW, 1e-6, torch.tensor(pos), CS, False)
        ds.within(server.q[:n], want, bound, f"q of step {i}")
        want, bound = ss.reference_kv4(server.q[:n], server.kc, server.vc, server.table.cpu(), held,
                                       draft.rows, SCALE)
        ds.within(server.o[:n], want, bound, f"step {i}")
        assert (server.o[n:] == 7.0).all() and (server.q[n:] == 7.0).all()
        kept, num, nxt = ss.reference_verify(
            draft.logits[:n].numpy(), draft.tokens, draft.cu, server.heat.tolist(), draft.u[:n].tolist(),
            MAX_ROWS, draft=draft.draft[:n].numpy() if with_draft else None)
        assert (server.kept.tolist(), server.num_kept.tolist(), server.next.tolist()) == (kept, num, nxt)
        new = turned(draft.qkv, pos)
        for s in range(S):                 # (a chain's kept rows are its first)
            a = draft.cu[s]
            history[s] = [torch.cat([old, x[a:a + num[s]]]) for old, x in zip(history[s], new)]
        assert server.lens.tolist() == [len(x[0]) for x in history]
        check_pages(server, history, f"step {i}")
    # a piece of 40 more tokens for every sequence, over the keys read back
    lens = server.lens.tolist()
    total = [m + 40 for m in lens]
    cu_k, cu_q = i32([sum(total[:s]) for s in range(S + 1)]), i32([40 * s for s in range(S + 1)])
    k = torch.full((sum(total), HKV, D), math.nan, dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    qkv = normal_bf16((40 * S, HQ + 2 * HKV, D), 77, "cuda")
    q = torch.empty((40 * S, HQ, D), dtype=torch.bfloat16, device="cuda")
    slots = i32([0] * (40 * S))
    binding.rag_kv_pages_update(server.table, server.stack, server.free, server.lens, i32(total),
                                server.free2, server.held, server.cu, slots, server.granted)
    server.write(qkv, i32([m + i for m in lens for i in range(40)]), slots, q)
    binding.rag_kv4_read(server.kc, server.vc, server.table, cu_k, k, v)
    o = torch.empty_like(q)
    binding.rag_attn_prefill_varlen(q, k, v, o, None, cu_q, cu_k, 40, max(total), SCALE, True)
    want = ds.reference_ranges(q, k, v, [40] * S, total, i32([(0, 0)] * (40 * S)), SCALE)
    ds.within(o, want[0], want[2], "piece")
    # the same rows straight from the pages, up to the rounding of the rows read to bf16
    o2 = torch.empty_like(q)
    ws = torch.zeros(binding.rag_attn_decode_kv4_workspace_size(S, 40, HQ, HKV, D, WIDTH),
                     dtype=torch.uint8, device="cuda")
    binding.rag_attn_decode_paged_kv4(q, server.kc, server.vc, o2, server.table, i32(total), SCALE, cu_q, 40,
                                      ws)
    want = ss.reference_kv4(q, server.kc, server.vc, server.table.cpu(), total, [40] * S, SCALE)
    ds.within(o2, want[0], want[1], "piece from the pages")


@pytest.mark.parametrize("with_draft", [False, True])
def test_captured_steps_are_the_eager_ones(with_draft):
    """Two servers' steps in two graphs, each with its workspaces, replayed in turn and at once; a
    third server runs eagerly."""
    servers = [Server(with_draft) for _ in range(3)]
    eager, one, two = servers
    qkv = normal_bf16((sum(PROMPTS), HQ + 2 * HKV, D), 1, "cuda")
    for s in servers:
        s.admit(qkv, PROMPTS)
    torch.cuda.synchronize()
    graphs = [capture(one.step), capture(two.step)]
    side = torch.cuda.Stream()
    for i in range(5):
        print(f"replay {i}", flush=True)
        draft, lens = Draft(7 * i + 1), eager.lens.tolist()
        for s in servers:
            draft.put(s, lens)
        eager.step()
        torch.cuda.synchronize()
        graphs[0].replay()
        if i % 2:
            torch.cuda.synchronize()
            graphs[1].replay()
        else:
            with torch.cuda.stream(side):
                graphs[1].replay()
        torch.cuda.synchronize()
        for s in (one, two):
            assert torch.equal(s.o, eager.o) and torch.equal(s.q, eager.q)
            assert torch.equal(s.kc, eager.kc) and torch.equal(s.vc, eager.vc)
            assert s.state() == eager.state()


def test_calls_on_three_streams_at_once():
    """Each with its caches and workspaces; the same bits as alone."""
    servers = [Server(True) for _ in range(3)]
    qkv = normal_bf16((sum(PROMPTS), HQ + 2 * HKV, D), 1, "cuda")
    for s in servers:
        s.admit(qkv, PROMPTS)
    drafts = [Draft(100 + i) for i in range(3)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s, d in zip(servers, drafts):
        d.put(s, PROMPTS)
    torch.cuda.synchronize()
    for s, t in zip(servers, streams):
        with torch.cuda.stream(t):
            s.step()
    torch.cuda.synchronize()
    for s, d in zip(servers, drafts):
        alone = Server(True)
        alone.admit(qkv, PROMPTS)
        d.put(alone, PROMPTS)
        torch.cuda.synchronize()
        alone.step()
        torch.cuda.synchronize()
        assert torch.equal(s.o, alone.o) and torch.equal(s.kc, alone.kc) and s.state() == alone.state()


def test_prefix_pages_in_several_tables():
    """Sequences whose tables begin with the same pages attend them alike, and read them alike."""
    lens = [200, 70, 96]
    kc, vc, table = ss.random_pool(lens, HKV, D, 11)
    table[1:, :4] = table[0, :4]
    q = normal_bf16((3, HQ, D), 12, "cuda")
    o = torch.empty_like(q)
    ws = torch.zeros(binding.rag_attn_decode_kv4_workspace_size(3, 1, HQ, HKV, D, table.shape[1]),
                     dtype=torch.uint8, device="cuda")
    binding.rag_attn_decode_paged_kv4(q, kc.cuda(), vc.cuda(), o, table.cuda(), i32(lens), SCALE, workspace=ws)
    want, bound = ss.reference_kv4(q, kc, vc, table, lens, [1] * 3, SCALE)
    ds.within(o, want, bound, "shared pages")
    k = torch.empty((64 * 3, HKV, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    binding.rag_kv4_read(kc.cuda(), vc.cuda(), table.cuda(), i32([0, 64, 128, 192]), k, v)
    for x in (k, v):
        assert torch.equal(x[:64], x[64:128]) and torch.equal(x[:64], x[128:])
