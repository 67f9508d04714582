"""The 4-bit cache on the GPU: rows read back, and attention against the 64-bit
reference, element by element inside the bound of its arithmetic."""
import math
import random

import pytest
import torch

import serve_support as ss
from draft_support import pages_of, within
from paper_2412_10543_amd import binding

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return _i32(cu)


def _workspace(S, rows, hq, hkv, d, width=1):
    n = binding.rag_attn_decode_kv4_workspace_size(S, rows, hq, hkv, d, width)
    return torch.zeros(n, dtype=torch.uint8, device="cuda")


def _attend(q, kc, vc, table, kv, rows, ws=None, single=None):
    S, hq, hkv, d = len(kv), q.shape[1], kc.shape[1], q.shape[2]
    o = torch.full_like(q, math.nan)
    single = max(rows, default=0) == 1 and min(rows) == 1 if single is None else single
    ws = _workspace(S, max(rows), hq, hkv, d, table.shape[1]) if ws is None else ws
    binding.rag_attn_decode_paged_kv4(q, kc, vc, o, table, _i32(kv), 1 / math.sqrt(d),
                                      None if single else _cu(rows), max(rows), ws)
    torch.cuda.synchronize()
    assert int(ws[:4096 * 4].count_nonzero()) == 0          # the counters are zero again
    return o


def _case(kv, rows, hq, hkv, d, seed, k_scale=1.0, poison=True):
    kc, vc, table = ss.random_pool(kv, hkv, d, seed, k_scale, poison)
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn((sum(rows), hq, d), generator=g).bfloat16()
    return q.cuda(), kc.cuda(), vc.cuda(), table.cuda()


def _check(kv, rows, hq, hkv, d, seed, k_scale=1.0):
    q, kc, vc, table = _case(kv, rows, hq, hkv, d, seed, k_scale)
    o = _attend(q, kc, vc, table, kv, rows)
    want, bound = ss.reference_kv4(q, kc, vc, table.cpu(), kv, rows, 1 / math.sqrt(d))
    within(o, want, bound, f"kv {kv} rows {rows}")


HEADS = [(32, 8, 128), (4, 2, 64), (64, 8, 128), (14, 2, 64), (16, 16, 128), (20, 4, 128), (40, 1, 64)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("kv", [[1], [2], [15], [16], [17], [31], [32], [33], [300], [1000, 1, 77, 513],
                                [4782], [700] * 9])
def test_one_row_a_sequence(hq, hkv, d, kv):
    _check(kv, [1] * len(kv), hq, hkv, d, seed=len(kv) + kv[0])


@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_chains(hq, hkv, d):
    r = random.Random(hq)
    for most, count in ((2, 5), (4, 3), (5, 4), (9, 4), (17, 3), (40, 2)):
        rows = [r.randint(0, most) for _ in range(count)] + [most]
        kv = [n + r.choice([0, 0, 1, 30, 500, 1300]) for n in rows]
        _check(kv, rows, hq, hkv, d, seed=most)


@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (2, 2, 128), (3, 1, 128)])
def test_numbers_of_pairs_around_the_tiles_of_16(hq, hkv, d):
    """Sequences on both sides of every number of tiles, some cut into pieces, in one batch; with those
    beside them that have no keys to cut."""
    group = hq // hkv
    rows = [(p + group - 1) // group for p in (16, 17, 32, 33, 48, 49, 64, 65, 1, 8, 130)] + [0, 1]
    r = random.Random(hq)
    kv = [n + r.choice([0, 1, 30, 500, 2500]) for n in rows[:-2]] + [77, 1]
    _check(kv, rows, hq, hkv, d, seed=31)
    order = list(range(len(kv)))
    r.shuffle(order)
    _check([kv[i] + 600 * (rows[i] > 0) for i in order], [rows[i] for i in order], hq, hkv, d, seed=32)


@pytest.mark.parametrize("k_scale", [4.0, 12.0])
def test_peaked_scores(k_scale):
    _check([900, 40, 3000], [1, 3, 2], 8, 2, 128, 5, k_scale)


@pytest.mark.parametrize("hq", [8, 20])
def test_scale_so_small_that_all_keys_are_alike(hq):
    """The least scale above 0: the mean of the values."""
    kv = [40, 700]
    q, kc, vc, table = _case(kv, [1, 1], hq, 2, 128, 9)
    o, ws = torch.full_like(q, math.nan), _workspace(2, 1, hq, 2, 128)
    binding.rag_attn_decode_paged_kv4(q, kc, vc, o, table, _i32(kv), 2.0 ** -149, workspace=ws)
    torch.cuda.synchronize()
    want, bound = ss.reference_kv4(q, kc, vc, table.cpu(), kv, [1, 1], 2.0 ** -149)
    within(o, want, bound, "mean")


def test_sequences_without_keys_or_rows():
    """kv 0 with a row each gives 0; sequences without rows are passed over; rows behind the
    last sequence stay."""
    q, kc, vc, table = _case([0, 20, 0], [1, 1, 1], 8, 2, 64, 3)
    o = _attend(q, kc, vc, table, [0, 20, 0], [1, 1, 1])
    assert (o[0] == 0).all() and (o[2] == 0).all() and torch.isfinite(o[1]).all() and (o[1] != 0).any()
    q, kc, vc, table = _case([50, 0, 20], [3, 0, 1], 8, 2, 64, 4)
    q = torch.cat([q, q])
    o = _attend(q, kc, vc, table, [50, 0, 20], [3, 0, 1])
    assert torch.isfinite(o[:4]).all() and o[4:].isnan().all()


@pytest.mark.parametrize("S,rows", [(1, 1), (5, 1), (3, 0)])
def test_tables_without_pages(S, rows):
    """The workspace that the library asks for, none, is what the call takes: zeros, or no rows."""
    hq, hkv, d = 32, 8, 128
    assert binding.rag_attn_decode_kv4_workspace_size(S, 9, hq, hkv, d, 0) == 0
    q = torch.randn((S, hq, d)).bfloat16().cuda()
    kc, vc = (torch.empty((0, hkv, 9 * d), dtype=torch.uint8, device="cuda") for _ in range(2))
    o, table = torch.full_like(q, math.nan), torch.empty((S, 0), dtype=torch.int32, device="cuda")
    cu = None if rows else _i32([0] * (S + 1))
    for _ in range(2):
        binding.rag_attn_decode_paged_kv4(q, kc, vc, o, table, _i32([0] * S), 0.1, cu, 9)
        torch.cuda.synchronize()
        assert (o == 0).all() if rows else o.isnan().all()


@pytest.mark.parametrize("S", [200, 1024, 1025])
def test_many_sequences(S):
    """Up to 1024 sequences share all keys; with one more none is cut."""
    r = random.Random(S)
    kv = [r.choice([1, 17, 40, 100]) for _ in range(S)]
    kv[S // 2] = 3000
    _check(kv, [1] * S, 4, 2, 64, seed=S)


@pytest.mark.parametrize("most,group", [(1, 4), (2, 4), (4, 4), (8, 4), (40, 4)])
def test_many_chains_that_none_is_cut_of(most, group):
    """More than 1024 sequences, with rows for every form and for several tiles."""
    r = random.Random(most)
    rows = [r.choice([0, 1, most]) for _ in range(1030)]
    kv = [n + r.choice([0, 1, 20, 70]) for n in rows]
    kv[500] += 1500
    _check(kv, rows, group, 1, 64, seed=most)


@pytest.mark.parametrize("hkv", [300, 600, 4100])
def test_many_kv_heads(hkv):
    """One workgroup a kv head for all sequences, and more kv heads than there are counters for."""
    _check([100, 1, 333], [1, 1, 1], hkv, hkv, 64, seed=hkv)
    _check([40, 9, 70], [3, 0, 9], hkv, hkv, 64, seed=hkv + 1)


def test_cuts_do_not_depend_on_the_others():
    """A sequence alone, among others and in another order: the same numbers up to the
    bound; runs repeat bit by bit, and one workspace serves calls of any sizes."""
    hq, hkv, d = 32, 8, 128
    kv, rows = [2500, 90, 6000, 700, 1], [1, 4, 2, 9, 1]
    q, kc, vc, table = _case(kv, rows, hq, hkv, d, 8)
    ws = _workspace(len(kv), 9, hq, hkv, d)
    a = _attend(q, kc, vc, table, kv, rows, ws)
    one = _attend(q[:1].contiguous(), kc, vc, table[:1].contiguous(), kv[:1], [1], ws)
    b = _attend(q, kc, vc, table, kv, rows, ws)
    assert torch.equal(a, b)
    want, bound = ss.reference_kv4(q, kc, vc, table.cpu(), kv, rows, 1 / math.sqrt(d))
    within(a, want, bound)
    within(one, want[:1], bound[:1])
    order = [3, 0, 4, 2, 1]
    at = [sum(rows[:i]) for i in range(5)]
    index = [at[i] + j for i in order for j in range(rows[i])]
    c = _attend(q[index].contiguous(), kc, vc, table[order].contiguous(), [kv[i] for i in order],
                [rows[i] for i in order], ws)
    within(c, want[index], bound[index])


@pytest.mark.parametrize("kv,rows", [([9000, 40], [1, 1]), ([5000, 700, 3, 2500], [9, 17, 1, 33]),
                                     ([300] * 1030, [1] * 1030)])
def test_in_place(kv, rows):
    """o = q: cut sequences, several tiles, and launches that cut none."""
    hq, hkv, d = (32, 8, 128) if len(kv) < 1000 else (4, 2, 64)
    q, kc, vc, table = _case(kv, rows, hq, hkv, d, 14)
    o = _attend(q, kc, vc, table, kv, rows)
    for _ in range(3):
        p, ws = q.clone(), _workspace(len(kv), max(rows), hq, hkv, d)
        binding.rag_attn_decode_paged_kv4(p, kc, vc, p, table, _i32(kv), 1 / math.sqrt(d), _cu(rows),
                                          max(rows), ws)
        assert torch.equal(o, p)


def test_physical_order_of_pages_changes_nothing():
    kv, hq, hkv, d = [1234, 600], 8, 2, 128
    q, kc, vc, table = _case(kv, [1, 1], hq, hkv, d, 9, poison=False)
    o = _attend(q, kc, vc, table, kv, [1, 1])
    perm = torch.randperm(kc.shape[0], device="cuda")
    back = torch.empty_like(perm)
    back[perm] = torch.arange(len(perm), device="cuda")
    p = _attend(q, kc[perm].contiguous(), vc[perm].contiguous(), back[table.long()].int(), kv, [1, 1])
    assert torch.equal(o, p)


def test_what_a_row_does_not_see_never_reaches_it():
    """The keys of later rows, NaN and all; a NaN key that a row sees makes it NaN."""
    hq, hkv, d = 8, 2, 128
    kv, rows = [300], [6]
    q, kc, vc, table = _case(kv, rows, hq, hkv, d, 10)
    o = _attend(q, kc, vc, table, kv, rows)
    page, at = int(table[0, 297 // 16]), 297 % 16
    for cache in (kc, vc):
        for g in range(d // 64):
            cache[page, :, 8 * d + 4 * (16 * g + at):][:, :4] = 0xff         # s = NaN, zero NaN
        p = _attend(q, kc, vc, table, kv, rows)
        assert torch.equal(p[:3], o[:3]) and p[3:].isnan().all()


def test_equals_the_bf16_cache_s_attention_on_the_same_values():
    """Attention over the values that the codes stand for, in a bf16 cache: both calls lie
    inside their bounds of the same reference, so that they differ by at most the sum."""
    kv, hq, hkv, d = [800, 33, 2100], 32, 8, 128
    q, k4, v4, table = _case(kv, [1] * 3, hq, hkv, d, 11, poison=False)
    o = _attend(q, k4, v4, table, kv, [1] * 3)
    kc, vc = (next(iter(ss.unpack(c, d, values))).permute(0, 2, 1, 3).float().bfloat16().contiguous().cuda()
              for c, values in ((k4, False), (v4, True)))
    p = torch.empty_like(q)
    n = binding.rag_attn_decode_workspace_size(3, hq, hkv, d, table.shape[1])
    binding.rag_attn_decode_paged(q, kc, vc, p, table, _i32(kv), 1 / math.sqrt(d),
                                  workspace=torch.zeros(max(n, 1), dtype=torch.uint8, device="cuda"))
    # values rounded to bf16 (2^-9 on average, a score of about 1 from 128 of them): 2e-2 as everywhere
    assert (o.float() - p.float()).abs().max() <= 2e-2


@pytest.mark.parametrize("hkv,d", [(8, 128), (2, 64), (1, 128), (3, 64)])
@pytest.mark.parametrize("lens", [[1], [16], [15, 17], [0, 33, 0, 5, 160], [700, 1, 2, 3, 90] * 7, [5000]])
def test_rows_read_back(hkv, d, lens):
    kc, vc, table = ss.random_pool([max(n, 1) for n in lens], hkv, d, len(lens), poison=True)
    total = sum(lens)
    out = [torch.full((total + 3, hkv, d), -7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    binding.rag_kv4_read(kc.cuda(), vc.cuda(), table.cuda(), _cu(lens), *out)
    for cache, values, got in ((kc, False, out[0]), (vc, True, out[1])):
        rows, _ = ss.unpack(cache, d, values)
        want = [rows[table[s, :pages_of(n)].long()].reshape(-1, hkv, d)[:n] for s, n in enumerate(lens)]
        assert torch.equal(got.cpu()[:total], torch.cat(want).float().bfloat16())
        assert (got[total:] == -7).all()


@pytest.mark.parametrize("hkv,d,pages", [(8, 128, 2100), (8, 128, 4200), (8, 64, 8300), (7, 64, 2800),
                                         (6, 128, 4200), (3, 64, 8300), (20, 64, 2800), (20, 128, 1700)])
def test_rows_of_many_keys_read_back(hkv, d, pages):
    """Over tables that repeat a few pages."""
    r = random.Random(pages)
    kc, vc, _ = ss.random_pool([16 * 50], hkv, d, pages)
    lens = [16 * (pages // 2) + 5, 0, 16 * (pages // 3), 1, 16 * (pages // 6) - 3, 77]
    width = max(map(pages_of, lens))
    table = torch.tensor([[r.randrange(kc.shape[0]) for _ in range(width)] for _ in lens], dtype=torch.int32)
    total = sum(lens)
    out = [torch.full((total + 3, hkv, d), -7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    binding.rag_kv4_read(kc.cuda(), vc.cuda(), table.cuda(), _cu(lens), *out)
    for cache, values, got in ((kc, False, out[0]), (vc, True, out[1])):
        rows = next(iter(ss.unpack(cache, d, values))).float().bfloat16().cuda()
        at = 0
        for s, n in enumerate(lens):
            want = rows[table[s, :pages_of(n)].long().cuda()].reshape(-1, hkv, d)[:n]
            assert torch.equal(got[at:at + n], want), (s, values)
            at += n
        assert (got[total:] == -7).all()


def test_page_numbers_behind_two_gigabytes():
    """Offsets in a pool of over 4 GiB a cache are 64-bit."""
    hkv, d, kv = 8, 128, 40
    blocks = (5 << 30) // (9 * d * hkv)
    kc4, vc4, table = ss.random_pool([kv], hkv, d, 12)
    big = [torch.empty((blocks, hkv, 9 * d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    far = torch.tensor([[blocks - 1, blocks - 3, 7]], dtype=torch.int32)
    for src, dst in ((kc4, big[0]), (vc4, big[1])):
        for i in range(3):
            dst[int(far[0, i])] = src[int(table[0, i])].cuda()
    q = torch.randn((1, 32, d)).bfloat16().cuda()
    a = _attend(q, kc4.cuda(), vc4.cuda(), table.cuda(), [kv], [1])
    b = _attend(q, *big, far.cuda(), [kv], [1])
    assert torch.equal(a, b)
    rows = [[torch.empty((kv, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
    binding.rag_kv4_read(kc4.cuda(), vc4.cuda(), table.cuda(), _cu([kv]), *rows[0])
    binding.rag_kv4_read(*big, far.cuda(), _cu([kv]), *rows[1])
    assert torch.equal(rows[0][0], rows[1][0]) and torch.equal(rows[0][1], rows[1][1])
    k = torch.randn((16, hkv, d)).bfloat16().cuda()
    slots = (blocks - 2) * 16 + torch.arange(16, dtype=torch.int32, device="cuda")
    binding.rag_qkv_rope_write_kv4(None, k, k, None, None, None, slots, *big)
    small = torch.zeros((1, hkv, 9 * d), dtype=torch.uint8, device="cuda")
    small_v = small.clone()
    binding.rag_qkv_rope_write_kv4(None, k, k, None, None, None, slots - (blocks - 2) * 16, small, small_v)
    assert torch.equal(big[0][blocks - 2], small[0]) and torch.equal(big[1][blocks - 2], small_v[0])


def test_shapes_are_refused():
    q, kc, vc, table = _case([40], [1], 8, 2, 64, 1)
    ws, kv, o = _workspace(1, 1, 8, 2, 64), _i32([40]), torch.empty_like(q)

    def call(**kw):
        a = dict(q=q, k_cache=kc, v_cache=vc, o=o, block_tables=table, kv_lens=kv, softmax_scale=0.1,
                 workspace=ws)
        a.update(kw)
        binding.rag_attn_decode_paged_kv4(**a)

    call()
    for kw in (dict(q=q.float()), dict(k_cache=kc[..., :64]), dict(v_cache=vc[:1]), dict(o=o[:, :4]),
               dict(block_tables=table.long()), dict(kv_lens=_i32([40, 40])), dict(workspace=None),
               dict(workspace=ws[:100]), dict(cu_seqlens_q=_i32([0, 1, 2])), dict(workspace=ws.cpu()),
               dict(q=q[:, :7].contiguous(), o=o[:, :7].contiguous())):
        with pytest.raises((ValueError, TypeError, binding.RagError)):
            call(**kw)
    k = torch.empty((40, 2, 64), dtype=torch.bfloat16, device="cuda")
    for args in ((kc, vc, table, _cu([40]), k[:, :1].contiguous(), k), (kc, vc, table, _cu([20, 20]), k, k.clone()),
                 (kc, vc[..., 8:].contiguous(), table, _cu([40]), k, k.clone())):
        with pytest.raises((ValueError, binding.RagError)):
            binding.rag_kv4_read(*args)


@pytest.mark.parametrize("max_rows,hq,hkv,d", [(1, 32, 8, 128), (2, 8, 2, 64), (5, 8, 2, 128), (17, 4, 1, 128)])
def test_rows_past_the_host_s_bound_stay_inside_the_workspace(max_rows, hq, hkv, d):
    """A broken precondition (a sequence of more rows than max_seqlen_q), which the call is not
    told of: it writes neither behind its workspace nor the rows past the bound, and sequences
    inside it are attended as alone."""
    rows, kv = [max_rows + 8, max_rows, 1, 3 * max_rows + 40], [5000, 3000, 700, 9000]
    q, kc, vc, table = _case(kv, rows, hq, hkv, d, 21)
    size = binding.rag_attn_decode_kv4_workspace_size(4, max_rows, hq, hkv, d, table.shape[1])
    store = torch.zeros(size + (1 << 20), dtype=torch.uint8, device="cuda")
    store[size:] = 0x5a
    o = torch.full_like(q, math.nan)
    for _ in range(2):
        binding.rag_attn_decode_paged_kv4(q, kc, vc, o, table, _i32(kv), 1 / math.sqrt(d), _cu(rows), max_rows,
                                          store[:size])
        torch.cuda.synchronize()
        assert (store[size:] == 0x5a).all() and int(store[:4096 * 4].count_nonzero()) == 0
    want, bound = ss.reference_kv4(q, kc, vc, table.cpu(), kv, rows, 1 / math.sqrt(d))
    for s in range(4):
        at = sum(rows[:s])
        n = min(rows[s], max_rows)
        if n == rows[s]:
            within(o[at:at + n], want[at:at + n], bound[at:at + n], f"sequence {s}")
        else:
            assert torch.isfinite(o[at:at + n]).all()
            assert o[at + n:at + rows[s]].isnan().all()
