"""rag_attn_prefill_varlen_ranges on the GPU against 64 bits, element by element
within the bound that the arithmetic gives (draft_support)."""
import math
import random

import pytest
import torch

import draft_support as ds
import gpu_support as G
from paper_2412_10543_amd import binding
from paper_2412_10543_amd.workloads import normal_bf16

pytestmark = pytest.mark.gpu

i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731


def cu(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return i32(out)


def inputs(lens_q, lens_k, hq, hkv, d, seed, q_scale=1.0):
    return (normal_bf16((sum(lens_q), hq, d), seed, "cuda", q_scale),
            normal_bf16((sum(lens_k), hkv, d), seed + 1, "cuda"),
            normal_bf16((sum(lens_k), hkv, d), seed + 2, "cuda"))


def run(q, k, v, lens_q, lens_k, ranges, want_lse=True, stream=None):
    o = torch.full_like(q, float("nan"))
    lse = torch.full((q.shape[1], q.shape[0]), float("nan"), device="cuda") if want_lse else None
    binding.rag_attn_prefill_varlen_ranges(q, k, v, o, lse, cu(lens_q), cu(lens_k), ranges,
                                           max(lens_q), max(lens_k), 1.0 / math.sqrt(q.shape[2]),
                                           stream=stream)
    return o, lse


def check(q, k, v, lens_q, lens_k, ranges):
    ranges = i32(ranges).reshape(-1, 2)
    o, lse = run(q, k, v, lens_q, lens_k, ranges)
    wo, wl, bo, bl = ds.reference_ranges(q, k, v, lens_q, lens_k, ranges, 1.0 / math.sqrt(q.shape[2]))
    torch.cuda.synchronize()
    ds.within(o, wo, bo, "o")
    empty = wl == -math.inf
    assert (lse.cpu()[empty] == -math.inf).all()
    assert (o.transpose(0, 1)[empty.cuda()] == 0).all()
    bl[empty] = math.nan
    ds.within(lse, wl, bl, "lse")
    o2, _ = run(q, k, v, lens_q, lens_k, ranges, want_lse=False)
    assert torch.equal(torch.nan_to_num(o2), torch.nan_to_num(o))
    return o


def doc_ranges(shared, docs, query):
    out, at = [(0, 0)] * shared, shared
    for n in docs:
        out += [(shared, at)] * n
        at += n
    return out + [(0, 0)] * query


HEADS = [(4, 2, 64), (32, 8, 128), (2, 2, 128), (6, 2, 64), (20, 4, 128), (7, 1, 64), (16, 2, 128),
         (16, 1, 64)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_documents(hq, hkv, d):
    prompts = [(17, [100, 33, 64], 20), (0, [5, 130], 1), (64, [64, 64, 64], 64), (3, [1, 1, 1], 0),
               (200, [], 7)]
    lens = [s + sum(x) + y for s, x, y in prompts]
    check(*inputs(lens, lens, hq, hkv, d, 1), lens, lens, sum((doc_ranges(*p) for p in prompts), []))


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257, 700])
def test_lengths(n):
    lens = [n, 1, max(1, n - 3)]
    rng = random.Random(n)
    r = []
    for x in lens:
        cut = rng.randint(0, x)
        r += doc_ranges(cut // 2, [cut - cut // 2], x - cut)
    check(*inputs(lens, lens, 8, 2, 128, n), lens, lens, r)


def test_prefix_and_window():
    lens = [333, 90, 400]
    r = [(100, 0)] * 333 + [(90, 0)] * 90 + [(4, p - 49) for p in range(400)]
    check(*inputs(lens, lens, 8, 2, 128, 5), lens, lens, r)
    check(*inputs(lens, lens, 8, 8, 64, 6), lens, lens, r)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 2, 64)])
def test_tokens_behind_windows_are_sequences_of_one_row(hq, hkv, d):
    """A generated token's row alone over its packed keys, windows of 50 keys and
    the first 4: what the row would see as a prompt's last."""
    lens = [1, 2, 50, 54, 55, 400, 1000]
    q, k, v = inputs(lens, lens, hq, hkv, d, 17)
    at = torch.tensor(lens).cumsum(0) - 1
    alone = check(q[at.cuda()].contiguous(), k, v, [1] * len(lens), lens, [(4, n - 50) for n in lens])
    whole = i32([(4, p - 49) for n in lens for p in range(n)])
    want, _, bound, _ = ds.reference_ranges(q, k, v, lens, lens, whole, 1.0 / math.sqrt(d))
    ds.within(alone, want[at], bound[at])


@pytest.mark.parametrize("seed", range(6))
def test_any_ranges(seed):
    """Values in and out of range, empty rows, fewer and more rows than keys, a
    sequence without rows, one without keys."""
    rng = random.Random(seed)
    lens_q = [rng.choice([1, 7, 64, 150]), 0, 40, rng.randint(1, 200), 5]
    lens_k = [rng.choice([1, 64, 300]), 9, 13, rng.randint(1, 400), 0]
    r = []
    for nq, nk in zip(lens_q, lens_k):
        for _ in range(nq):
            r.append((rng.choice([0, -3, nk, nk + 9, 1 << 30, rng.randint(0, nk)]),
                      rng.choice([0, -9, nk, 1 << 30, rng.randint(0, nk), rng.randint(0, nk)])))
    hq, hkv, d = rng.choice(HEADS)
    check(*inputs(lens_q, lens_k, hq, hkv, d, seed), lens_q, lens_k, r)


def test_rows_that_see_nothing():
    lens = [70, 130]
    r = [(0, 1 << 30)] * 70 + [(0, 500 if p % 3 else 0) for p in range(130)]
    o = check(*inputs(lens, lens, 8, 2, 128, 3), lens, lens, r)
    assert (o[:70] == 0).all()


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("side", [1, 2])
def test_unseen_values_never_arrive(value, side):
    """A document holds `value`: its rows from there on and the query's may, the
    other documents' do not."""
    lens = [16 + 50 + 70 + 90 + 30]
    r = doc_ranges(16, [50, 70, 90], 30)
    x = list(inputs(lens, lens, 8, 2, 128, 9))
    x[side][16 + 50 + 40, :, 3] = value
    x[side][16 + 10, 0, 60] = value
    ranges = i32(r)
    o, lse = run(*x, lens, lens, ranges)
    wo, _, bo, _ = ds.reference_ranges(*x, lens, lens, ranges, 1.0 / math.sqrt(128))
    assert 0 < torch.isnan(bo).double().mean() < 0.7
    ds.within(o, wo, bo)


@pytest.mark.parametrize("q_scale", [0.0, 8.0, 40.0])
def test_flat_and_peaky_scores(q_scale):
    lens = [500]
    check(*inputs(lens, lens, 8, 2, 128, 2, q_scale), lens, lens, doc_ranges(40, [200, 200], 60))


def test_plain_causal_is_the_prefill():
    lens = [300, 77]
    q, k, v = inputs(lens, lens, 8, 2, 128, 8)
    o, lse = run(q, k, v, lens, lens, i32([(0, 0)] * 377))
    po, pl = torch.empty_like(o), torch.empty_like(lse)
    binding.rag_attn_prefill_varlen(q, k, v, po, pl, cu(lens), cu(lens), 300, 300, 1 / math.sqrt(128))
    wo, wl, bo, bl = ds.reference_ranges(q, k, v, lens, lens, i32([(0, 0)] * 377), 1 / math.sqrt(128))
    for got in (o, po):
        ds.within(got, wo, bo)
    for got in (lse, pl):
        ds.within(got, wl, bl)


def test_document_keys_do_not_depend_on_other_documents():
    """A document's rows are the same bits alone behind the system prompt and
    among others at the same place."""
    q, k, v = inputs([400], [400], 8, 2, 128, 4)
    o, _ = run(q, k, v, [400], [400], i32(doc_ranges(64, [64, 128, 100], 44)))
    k[64:128], v[64:128] = float("nan"), float("inf")
    o2, _ = run(q, k, v, [400], [400], i32(doc_ranges(64, [64, 128, 100], 44)))
    assert torch.equal(o[128:356], o2[128:356]) and torch.equal(o[:64], o2[:64])


def test_rows_behind_the_last_sequence_stay():
    lens = [100, 33]
    q, k, v = inputs([133 + 40], [133], 8, 2, 64, 3)
    o = torch.full_like(q, 7.0)
    lse = torch.full((8, 173), 7.0, device="cuda")
    r = i32(doc_ranges(0, [100], 0) + doc_ranges(3, [20], 10) + [(0, 0)] * 40)
    binding.rag_attn_prefill_varlen_ranges(q, k, v, o, None, cu(lens), cu(lens), r, 100, 100, 0.125)
    torch.cuda.synchronize()
    assert (o[133:] == 7.0).all() and not (o[:133] == 7.0).all() and (lse == 7.0).all()
    # with a log-sum-exp, of the sequences' rows
    packed = torch.full((8, 133), 7.0, device="cuda")
    binding.rag_attn_prefill_varlen_ranges(q, k, v, o, packed, cu(lens), cu(lens), r, 100, 100, 0.125)
    _, want, _, bound = ds.reference_ranges(q[:133], k, v, lens, lens, r[:133], 0.125)
    ds.within(packed, want, bound)
    assert (o[133:] == 7.0).all()
    for bad in (lse[:7], torch.full((8, 174), 7.0, device="cuda")):
        with pytest.raises(ValueError, match="inconsistent shapes"):
            binding.rag_attn_prefill_varlen_ranges(q, k, v, o, bad, cu(lens), cu(lens), r, 100, 100, 0.125)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (32, 8, 128)])
@pytest.mark.parametrize("lens", [[100, 33], [1], [64, 64, 257]])
def test_nothing_is_written_behind_the_log_sum_exps(hq, hkv, d, lens):
    """They stand at the front of a longer buffer; q and o have rows behind the last
    sequence."""
    n = sum(lens)
    q, k, v = inputs([n + 40], [n], hq, hkv, d, 3)
    buf = torch.full((hq * n + 3000,), 7.0, device="cuda")
    lse, o = buf[:hq * n].view(hq, n), torch.full_like(q, 7.0)
    r = i32(sum(([(x // 3, x // 2)] * x for x in lens), []) + [(0, 0)] * 40)
    binding.rag_attn_prefill_varlen_ranges(q, k, v, o, lse, cu(lens), cu(lens), r, max(lens), max(lens),
                                           1.0 / math.sqrt(d))
    wo, wl, bo, bl = ds.reference_ranges(q[:n], k, v, lens, lens, r[:n], 1.0 / math.sqrt(d))
    torch.cuda.synchronize()
    empty = wl == -math.inf
    assert (lse.cpu()[empty] == -math.inf).all()
    bl[empty] = math.nan
    ds.within(lse, wl, bl, "lse")
    ds.within(o[:n], wo, bo, "o")
    assert (buf[hq * n:] == 7.0).all() and (o[n:] == 7.0).all()


def test_offsets_past_32_bits():
    """A window over a packed batch whose last rows lie beyond 2^31 elements."""
    hq, hkv, d, n = 64, 1, 128, 2 ** 31 // (64 * 128) + 200
    q = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda")
    q.normal_()
    k, v = (normal_bf16((n, hkv, d), i, "cuda") for i in (1, 2))
    p = torch.arange(n, device="cuda", dtype=torch.int32)
    ranges = torch.stack([torch.full_like(p, 2), p - 30], 1).contiguous()
    o, lse = run(q, k, v, [n], [n], ranges)
    torch.cuda.synchronize()
    at = torch.tensor([0, 5, 2 ** 31 // (64 * 128) - 1, 2 ** 31 // (64 * 128) + 1, n - 1])
    for i in at.tolist():
        seen = torch.tensor(sorted({0, 1} | set(range(max(0, i - 30), i + 1))))
        seen = seen[seen < n]
        for h in (0, 63):
            x, y, b, bl = ds.attend64(q[i:i + 1, h], k[seen, 0], v[seen, 0],
                                      torch.ones((1, len(seen)), dtype=torch.bool), 1 / math.sqrt(d))
            ds.within(o[i:i + 1, h], x, b)
            ds.within(lse[h, i:i + 1], y, bl)


def test_another_stream():
    lens = [200]
    q, k, v = inputs(lens, lens, 8, 2, 128, 6)
    r = doc_ranges(10, [90, 60], 40)
    a, _ = run(q, k, v, lens, lens, i32(r))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b, _ = run(q, k, v, lens, lens, i32(r))
    c, _ = run(q, k, v, lens, lens, i32(r), stream=s)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c)


ITEMS = [
    # (prompts as (system prompt, documents, query), hq, hkv, d)
    ([(17, [100, 33, 300], 40), (3, [700], 9), (0, [40], 0)], 8, 2, 128),
    ([(40, [400, 1, 64], 300)], 8, 4, 64),
    ([(0, [900, 900], 33), (1, [], 0)], 2, 2, 128),
    ([(200, [90] * 5, 7)], 16, 1, 64),
]


@pytest.mark.parametrize("case", range(len(ITEMS)))
@pytest.mark.parametrize("kind", ["documents", "any", "nan"])
def test_several_tiles_a_workgroup(case, kind):
    """Tiles that one workgroup runs one after another are the bits of tiles of their
    own: long and short ones, ones without a key, ones with values that must not
    arrive."""
    prompts, hq, hkv, d = ITEMS[case]
    lens = [s + sum(x) + y for s, x, y in prompts]
    r = sum((doc_ranges(*p) for p in prompts), [])
    x = inputs(lens, lens, hq, hkv, d, 60 + case)
    if kind == "any":
        rng = random.Random(case)
        at = 0
        for n in lens:
            for a in range(at, at + n, 50):              # the same for 50 rows, or none
                e = rng.choice([(0, 1 << 30), (rng.randint(0, n), rng.randint(0, n)), (0, 0)])
                r[a:min(a + 50, at + n)] = [e] * (min(a + 50, at + n) - a)
            at += n
    if kind == "nan":
        for t, row in ((1, lens[0] // 3), (2, lens[0] // 2), (2, 1)):
            x[t][row, :, 7] = math.nan
    ranges = i32(r).reshape(-1, 2)
    with G.env("RAG_ATTN_PF_ITEMS", 1):
        o1, l1 = run(*x, lens, lens, ranges)
    wo, _, bo, _ = ds.reference_ranges(*x, lens, lens, ranges, 1.0 / math.sqrt(d))
    ds.within(o1, wo, bo)
    for items in (2, 3, 5, 32):
        print(f"items {items}", flush=True)
        with G.env("RAG_ATTN_PF_ITEMS", items):
            o, lse = run(*x, lens, lens, ranges)
        torch.cuda.synchronize()
        # (a NaN is one, of whatever bits)
        assert torch.equal(torch.isnan(o), torch.isnan(o1))
        assert torch.equal(o.nan_to_num(9.0).view(torch.int16), o1.nan_to_num(9.0).view(torch.int16))
        assert torch.equal(torch.isnan(lse), torch.isnan(l1))
        assert torch.equal(lse.nan_to_num(9.0), l1.nan_to_num(9.0))


def test_a_launch_of_many_tiles():
    """More tiles than workgroups are made for one by one."""
    lens = [5000, 100]
    q, k, v = inputs(lens, lens, 32, 32, 64, 70)
    q = q.repeat(1, 4, 1)                                # 128 heads on 32: 4 to a workgroup
    r = i32(doc_ranges(30, [60] * 82, 50) + doc_ranges(0, [40, 40], 20))
    o, _ = run(q, k, v, lens, lens, r)
    with G.env("RAG_ATTN_PF_ITEMS", 1):
        o1, _ = run(q, k, v, lens, lens, r)
    assert torch.equal(o, o1)
    sub = [0, 3, 127]                                    # q heads, and the kv heads they read
    w = ds.reference_ranges(q[:, sub].contiguous(), k[:, [0, 0, 31]].contiguous(),
                            v[:, [0, 0, 31]].contiguous(), lens, lens, r, 1.0 / 8)
    ds.within(o[:, sub], w[0], w[2])
