"""rag_draft_verify on the GPU against the 64-bit reference, one node after another:
every kept node, count and token is the same."""
import math
import random

import numpy as np
import pytest
import torch

import serve_support as ss
from paper_2412_10543_amd import binding

pytestmark = pytest.mark.gpu

COUNTERS = 2 * 16384


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _workspace(rows, S, vocab):
    return torch.zeros(binding.rag_draft_verify_workspace_size(rows, S, vocab), dtype=torch.uint8,
                       device="cuda")


def _verify(logits, tokens, parents, cu, heat, uniforms, draft, max_kept, ws=None):
    S, rows = len(cu) - 1, logits.shape[0]
    ws = _workspace(rows, S, logits.shape[1]) if ws is None else ws
    kept = torch.full((S, max_kept), -9, dtype=torch.int32, device="cuda")
    num, nxt = _i32([-9] * S), _i32([-9] * S)
    binding.rag_draft_verify(logits, _i32(tokens), _i32(cu),
                             torch.tensor(heat, dtype=torch.float32, device="cuda"),
                             torch.as_tensor(uniforms, dtype=torch.float32).cuda(), kept, num, nxt,
                             parents=None if parents is None else _i32(parents), draft_probs=draft,
                             workspace=ws)
    torch.cuda.synchronize()
    assert int(ws[:COUNTERS * 4].count_nonzero()) == 0       # the counters are zero again
    return kept.tolist(), num.tolist(), nxt.tolist()


def _check(lens, vocab, chain, with_draft, wide, padded=0, max_kept=None, seed=0, **kw):
    logits, tokens, parents, cu, heat, u, draft = ss.verify_case(seed, lens, vocab, chain, **kw)
    max_kept = max(lens + [1]) if max_kept is None else max_kept
    store = torch.full((len(logits), vocab + padded), math.nan,
                       dtype=torch.float32 if wide else torch.bfloat16, device="cuda")
    store[:, :vocab] = logits
    probs = torch.full((len(logits), vocab + padded), math.nan, device="cuda")
    probs[:, :vocab] = draft
    got = _verify(store[:, :vocab], tokens, None if chain else parents, cu, heat, u,
                  probs[:, :vocab] if with_draft else None, max_kept)
    # (the temperatures that the kernel has are fp32)
    heat = torch.tensor(heat, dtype=torch.float32).tolist()
    want = ss.reference_verify(logits.numpy(), tokens, cu, heat, u.tolist(), max_kept,
                               None if chain else parents, draft.numpy() if with_draft else None)
    assert got == tuple(want)
    return want


VOCABS = [1, 7, 100, 4095, 4096, 4097, 8200, 33001]


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("padded", [0, 1, 8])
def test_trees(vocab, wide, padded):
    for seed in range(3):
        lens = [1, 5, 0, 12, 30, 2, 0]
        _check(lens, vocab, False, False, wide, padded, seed=seed)


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("with_draft", [False, True])
def test_chains(vocab, wide, with_draft):
    for seed in range(3):
        _check([0, 1, 4, 9, 2, 6, 17], vocab, True, with_draft, wide, padded=seed, seed=seed)


@pytest.mark.parametrize("with_draft", [False, True])
def test_drafts_that_fit_are_kept_to_the_end(with_draft):
    """Drafts as the model draws them, or drawn from its own probabilities: whole paths, and no
    longer than they may be."""
    n, vocab = 20, 500
    logits, tokens, _, cu, heat, u, draft = ss.verify_case(3, [n] * 6, vocab, True, heats=(0.0, 0.3))
    heat = torch.tensor(heat).float().tolist()
    for row in range(6 * n):
        if row % n:
            w, best = ss._weights(logits[row - 1].numpy(), heat[row // n])
            draft[row] = torch.from_numpy(w / w.sum()).float() if w.sum() else draft[row]
            tokens[row] = ss._token(logits[row - 1].numpy(), heat[row // n], float(u[row - 1]))
    for max_kept in (1, 2, 5, 19, 20, 40):
        got = _verify(logits.cuda(), tokens, None, cu, heat, u, draft.cuda() if with_draft else None, max_kept)
        want = ss.reference_verify(logits.numpy(), tokens, cu, heat, u.tolist(), max_kept,
                                   draft=draft.numpy() if with_draft else None)
        assert got == tuple(want) and got[1] == [min(max_kept, n)] * 6


@pytest.mark.parametrize("chain,with_draft", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("max_kept", [1, 2, 3])
def test_paths_that_may_not_be_longer(chain, with_draft, max_kept):
    """The last node that may be kept counts as having no children, refused or not."""
    for seed in range(4):
        _check([9, 1, 4, 0, 12, 3, 3, 2, 7], 900, chain, with_draft, True, max_kept=max_kept, seed=seed)


def test_long_chains_and_trees():
    """More nodes than the walk holds at a time, rows more than four at a time."""
    _check([1500, 3], 40, False, False, True, seed=1, heats=(0.0,))
    n, vocab = 1200, 30
    logits, tokens, _, cu, heat, u, draft = ss.verify_case(2, [n, 37], vocab, True, heats=(0.0,))
    for row in range(n + 37):
        if row not in (0, n):
            tokens[row] = int(logits[row - 1].argmax())
    for d in (None, draft):
        got = _verify(logits.cuda(), tokens, None, cu, heat, u, None if d is None else d.cuda(), n)
        want = ss.reference_verify(logits.numpy(), tokens, cu, heat, u.tolist(), n,
                                   draft=None if d is None else d.numpy())
        assert got == tuple(want) and got[1] == [n, 37]


def test_greedy_ties_take_the_lowest_index():
    vocab = 9000
    logits = torch.zeros((3, vocab))
    logits[0, [8999, 17, 5000]] = 2.0
    logits[1, [4096, 4095]] = 3.0
    for wide in (False, True):
        x = logits.cuda() if wide else logits.bfloat16().cuda()
        got = _verify(x, [0, 17, 4095], None, [0, 3], [0.0], [0.5] * 3, None, 3)
        assert got == ([[0, 1, 2]], [3], [0])


def test_masked_and_unusual_logits():
    """-inf masks a token, NaN counts as -inf; rows of nothing else, and with +inf, give the
    first index of their maximum; drawn with numbers at both ends of [0, 1)."""
    vocab, inf, nan = 5000, math.inf, math.nan
    g = torch.Generator().manual_seed(2)
    x = torch.randn((10, vocab), generator=g)
    x[0, :4990] = -inf
    x[1] = -inf
    x[1, 4321] = 0.0
    x[2] = -inf
    x[3] = nan
    x[4, 100:] = nan
    x[5, 77] = inf
    x[5, 99] = inf
    x[6] = 1e30
    x[7] = -3e38
    x[8, :] = -200.0
    x[8, 3000] = 200.0
    x[9, 0] = nan
    last = 1 - 2.0 ** -24
    for u in (0.0, 0.25, float(torch.tensor(0.77)), last):  # (fp32, as the kernel has them)
        for heat in (0.0, 1.0, 0.01, 1e-45, inf):
            cu = list(range(11))
            got = _verify(x.cuda(), [0] * 10, None, cu, [heat] * 10, [u] * 10, None, 1)
            want = ss.reference_verify(x.numpy(), [0] * 10, cu, [heat] * 10, [u] * 10, 1) \
                if heat in (0.0, 1.0) else None
            token = got[2]
            assert token[1] == 4321 and token[2] == 0 and token[3] == 0 and token[5] == 77
            assert token[0] >= 4990 and token[4] < 100 and token[9] > 0
            # (with u = 0 the first token that has any weight, here e^-400)
            assert token[8] == 3000 or heat == inf or u == 0.0
            assert want is None or got == tuple(want), (u, heat)


@pytest.mark.parametrize("heat", [1e-45, 1e-30, 0.01, 1e30, math.inf])
def test_draws_at_the_ends_of_the_temperatures(heat):
    """Masked, constant and far-apart rows against weights by hand: where T is infinite every finite
    logit weighs 1, where it is least the largest ones do."""
    vocab, inf = 5000, math.inf
    g = torch.Generator().manual_seed(12)
    x = torch.randn((6, vocab), generator=g)
    x[1, :4990] = -inf
    x[2] = 1e30
    x[3] = -3e38
    x[3, 5::7] = -inf
    x[4, ::2] = 3e38
    x[4, 1::2] = -3e38
    x[5, 17:] = math.nan
    heat = float(torch.tensor(heat))
    for u in (0.0, 0.25, 0.77, 1 - 2.0 ** -24):
        u, want = float(torch.tensor(u)), []
        for row in x.double().numpy():
            some = np.isfinite(row)
            far = np.where(some, row - row[some].max(), 0)
            w = np.where(some, 1.0 if heat == inf else np.exp(np.maximum(far / heat, -1e4)), 0.0)
            want.append(ss._pick(w, u))
        got = _verify(x.cuda(), [0] * 6, None, list(range(7)), [heat] * 6, [u] * 6, None, 1)
        # (with u = 0 a weight that is 0 for one and e^-700 for the other would count)
        assert u == 0.0 and heat == float(torch.tensor(0.01)) or got[2] == want, (u, heat)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("vocab", [3, 5000])
def test_rows_of_nan_and_masks_alone(vocab, wide):
    """NaN counts as -inf also where nothing else is left: the first index of the maximum is 0,
    whichever of the two stands there."""
    inf, nan = math.inf, math.nan
    rows = [[nan] + [-inf] * (vocab - 1), [-inf] + [nan] * (vocab - 1), [nan] * (vocab - 1) + [-inf],
            [nan] * vocab, [-inf] * vocab, [nan, -inf] + [nan] * (vocab - 2)]
    x = torch.tensor(rows)
    x = x if wide else x.bfloat16()
    n, u = len(rows), 0.6
    for heat in (0.0, 1.0):
        assert _verify(x.cuda(), [0] * n, None, list(range(n + 1)), [heat] * n, [u] * n, None, 1) == \
            ([[0]] * n, [1] * n, [0] * n)
        # chains of two: token 0 is what such a row says, 1 is not
        q = torch.full((2 * n, vocab), 1.0 / vocab).cuda()
        y = x.repeat_interleave(2, 0).cuda()
        for token in (0, 1):
            tokens = [9, token] * n
            cu, h, us = list(range(0, 2 * n + 1, 2)), [heat] * n, [u] * (2 * n)
            for draft in (None, q):
                got = _verify(y, tokens, None, cu, h, us, draft, 2)
                want = ss.reference_verify(y.float().cpu().numpy(), tokens, cu, h, us, 2,
                                           draft=None if draft is None else q.cpu().numpy())
                assert got == tuple(want) and got[1] == [1 if token else 2] * n and got[2] == [0] * n


@pytest.mark.parametrize("chain,with_draft", [(False, False), (True, False), (True, True)])
def test_offsets_past_the_rows_leave_the_workspace_as_it_was(chain, with_draft):
    """A broken precondition (a last sequence that ends behind num_rows), which the call is not told
    of: the sequence has the rows that there are, and the next call's counters are zero."""
    lens, vocab = [4, 1, 9], 700
    logits, tokens, parents, cu, heat, u, draft = ss.verify_case(3, lens, vocab, chain, heats=(1.0,))
    ws = _workspace(14, 3, vocab)
    args = (tokens, None if chain else parents)
    want = ss.reference_verify(logits.numpy(), tokens, cu, heat, u.tolist(), 9, None if chain else parents,
                               draft.numpy() if with_draft else None)
    q = draft.cuda() if with_draft else None
    for end in (14, 23, 1 << 20, 14):                       # (_verify looks at the counters)
        assert _verify(logits.cuda(), *args, cu[:3] + [end], heat, u, q, 9, ws) == tuple(want)


def test_numbers_outside_the_interval_stay_in_the_vocabulary():
    x = torch.randn((4, 5000)).cuda()
    q = torch.softmax(torch.randn((4, 5000)), 1).cuda()
    for draft in (None, q):
        for u in (1.0, 2.0, -1.0, math.nan, math.inf):
            kept, num, nxt = _verify(x, [0, 1, 2, 3], None, [0, 4], [1.0], [u] * 4, draft, 4)
            assert 0 <= nxt[0] < 5000 and 1 <= num[0] <= 4


def test_tokens_outside_the_vocabulary_are_not_kept():
    x = torch.randn((3, 600)).cuda()
    q = torch.softmax(torch.randn((3, 600)), 1).cuda()
    for draft in (None, q):
        for heat in (0.0, 1.0):
            for bad in (-1, 600, 1 << 30, -(1 << 31)):
                got = _verify(x, [0, bad, 5], None, [0, 3], [heat], [0.5] * 3, draft, 3)
                assert got[0] == [[0, -1, -1]] and got[1] == [1]


def test_drafter_that_equals_the_model():
    """max(p - q, 0) is empty: nothing is refused, and a refused token (u at its end) is drawn
    from p."""
    g = torch.Generator().manual_seed(4)
    x = torch.randn((2, 800), generator=g)
    q = torch.softmax(x.double(), 1).float()[[1, 0]]        # row 1: what row 0 says
    got = _verify(x.cuda(), [0, 5], None, [0, 2], [1.0], [0.4, 0.999], q.cuda(), 2)
    want = ss.reference_verify(x.numpy(), [0, 5], [0, 2], [1.0], [float(torch.tensor(0.4)),
                               float(torch.tensor(0.999))], 2, draft=q.numpy())
    assert got == tuple(want)
    zero = torch.zeros_like(q)
    zero[1, 5] = 1e30                                       # refuses, and takes 5 out of p
    got = _verify(x.cuda(), [0, 5], None, [0, 2], [1.0], [0.4, 0.999], zero.cuda(), 2)
    want = ss.reference_verify(x.numpy(), [0, 5], [0, 2], [1.0], [float(torch.tensor(0.4)),
                               float(torch.tensor(0.999))], 2, draft=zero.numpy())
    assert got == tuple(want) and got[2][0] != 5
    full = torch.full_like(q, 1e30)                         # nothing is left: p itself
    got = _verify(x.cuda(), [0, 5], None, [0, 2], [1.0], [0.4, 0.999], full.cuda(), 2)
    want = ss.reference_verify(x.numpy(), [0, 5], [0, 2], [1.0], [float(torch.tensor(0.4)),
                               float(torch.tensor(0.999))], 2, draft=full.numpy())
    assert got == tuple(want)


def test_temperatures_near_a_logit_s_last_place():
    """Neighbouring logits that lie hundreds to thousands of powers of 2 apart: the largest ones alone
    are drawn, as likely as each other."""
    heat = [1e-9, 3e-9, 6e-9, 7e-9, 8e-9, 9e-9, 1e-8, 1.05e-8, 1.1e-8, 2e-8, 1e-7, 1e-6] * 4
    g = torch.Generator().manual_seed(8)
    x = 100 - 2.0 ** -17 * torch.randint(0, 4, (48, 5000), generator=g)
    x[:, 70] = 100
    u, cu = torch.rand(48, generator=g), list(range(49))
    got = _verify(x.cuda(), [0] * 48, None, cu, heat, u, None, 1)
    assert all(x[i, t] == 100 for i, t in enumerate(got[2][:36]))
    heat = torch.tensor(heat, dtype=torch.float32).tolist()
    assert got == tuple(ss.reference_verify(x.numpy(), [0] * 48, cu, heat, u.tolist(), 1))


def test_large_vocabulary_flat_logits():
    """Every one of 150,001 tokens is as likely as the others up to a little: a draw turns on
    the sixth digit of the sums."""
    g = torch.Generator().manual_seed(6)
    x = (0.01 * torch.randn((64, 150001), generator=g))
    u = torch.rand(64, generator=g)
    cu = list(range(65))
    for wide in (True, False):
        y = x if wide else x.bfloat16()
        got = _verify(y.cuda(), [0] * 64, None, cu, [1.0] * 64, u, None, 1)
        assert got == tuple(ss.reference_verify(y.float().numpy(), [0] * 64, cu, [1.0] * 64, u.tolist(), 1))


def test_large_vocabulary_flat_drafts():
    g = torch.Generator().manual_seed(7)
    x = 0.01 * torch.randn((32, 100003), generator=g)
    q = torch.softmax(0.01 * torch.randn((32, 100003), generator=g), 1)
    u = torch.rand(32, generator=g)
    u[1::2] = 0.9999                                        # (mostly refused)
    tokens = torch.randint(0, 100003, (32,), generator=g).tolist()
    cu = list(range(0, 33, 2))
    got = _verify(x.cuda(), tokens, None, cu, [1.0] * 16, u, q.cuda(), 2)
    want = ss.reference_verify(x.numpy(), tokens, cu, [1.0] * 16, u.tolist(), 2, draft=q.numpy())
    assert got == tuple(want)


def _lens(rows, S, seed):
    """S lengths that have `rows` nodes together, of at least 1 where there are enough."""
    r = random.Random(seed)
    lens = [1] * min(rows, S) + [0] * (S - rows)
    r.shuffle(lens)
    for _ in range(rows - S):
        lens[r.randrange(S)] += 1
    return lens


# A wave has one, two or four loads of 512 logits of a row, from 17 and from 33 rows of 128,077 tokens on,
# and in the draws behind chains from 15 and from 29 sequences on: all pairs of them.
@pytest.mark.parametrize("rows,S", [(12, 5), (14, 15), (10, 30), (30, 8), (32, 16), (30, 30), (40, 5), (50, 16),
                                    (131, 20), (70, 33), (300, 48)])
@pytest.mark.parametrize("wide", [False, True])
def test_batches_over_a_large_vocabulary(rows, S, wide):
    vocab = 128077
    for chain, with_draft in ((True, True), (True, False), (False, False)):
        if rows == 300 and not (wide and chain):
            continue
        _check(_lens(rows, S, rows), vocab, chain, with_draft, wide, padded=3, seed=S + rows, near=1.0)


def test_flat_logits_and_drafts_in_a_batch_of_chains():
    """As the flat ones above, at the longest segments: 40 chains, all sums of 128,077 tokens alike."""
    g = torch.Generator().manual_seed(17)
    S, n, vocab = 40, 4, 128077
    x = 0.01 * torch.randn((S * n, vocab), generator=g)
    q = torch.softmax(0.01 * torch.randn((S * n, vocab), generator=g), 1)
    u = torch.rand(S * n, generator=g)
    u[1::n] = torch.where(torch.arange(S) % 2 == 0, u[1::n], 0.9999)          # (half of them: mostly refused)
    tokens = torch.randint(0, vocab, (S * n,), generator=g).tolist()
    cu = list(range(0, S * n + 1, n))
    for draft in (None, q):
        got = _verify(x.cuda(), tokens, None, cu, [1.0] * S, u, None if draft is None else q.cuda(), n)
        want = ss.reference_verify(x.numpy(), tokens, cu, [1.0] * S, u.tolist(), n,
                                   draft=None if draft is None else q.numpy())
        assert got == tuple(want)


def test_one_workspace_for_calls_of_any_sizes():
    ws = _workspace(400, 50, 9000)
    r = random.Random(1)
    for i in range(8):
        chain = i % 2 == 0
        lens = [r.randint(0, 12) for _ in range(r.randint(1, 30))] + [1]
        vocab = r.choice([50, 4096, 9000])
        logits, tokens, parents, cu, heat, u, draft = ss.verify_case(i, lens, vocab, chain)
        d = draft.cuda() if i % 4 == 0 else None
        got = _verify(logits.cuda(), tokens, None if chain else parents, cu, heat, u, d, 12, ws)
        heat = torch.tensor(heat, dtype=torch.float32).tolist()
        want = ss.reference_verify(logits.numpy(), tokens, cu, heat, u.tolist(), 12,
                                   None if chain else parents, None if d is None else draft.numpy())
        assert got == tuple(want), i


def test_rows_behind_the_last_sequence_and_many_empty_sequences():
    logits, tokens, parents, cu, heat, u, draft = ss.verify_case(5, [3, 4], 300, True)
    more = torch.full((9, 300), math.nan)
    x = torch.cat([logits, more]).cuda()
    cu = [0] * 300 + cu[1:] + [7] * 300
    heat = [1.0] * 299 + heat + [1.0] * 300
    for d in (None, torch.cat([draft, more]).cuda()):
        got = _verify(x, tokens + [0] * 9, None, cu, heat, torch.cat([u, torch.rand(9)]), d, 4)
        want = ss.reference_verify(logits.numpy(), tokens, cu, torch.tensor(heat).float().tolist(),
                                   u.tolist(), 4, draft=None if d is None else draft.numpy())
        assert got == tuple(want)
    got = _verify(x[:0], [], None, [0, 0, 0], [1.0, 0.0], torch.rand(0), None, 2)
    assert got == ([[-1, -1]] * 2, [0, 0], [-1, -1])


def test_shapes_are_refused():
    x = torch.randn((4, 100)).cuda()
    t = dict(logits=x, tokens=_i32([0] * 4), cu_seqlens_q=_i32([0, 4]), temperature=torch.ones(1).cuda(),
             uniforms=torch.rand(4).cuda(), kept=_i32([[0] * 4]), num_kept=_i32([0]), next_token=_i32([0]),
             workspace=_workspace(4, 1, 100))
    binding.rag_draft_verify(**t)
    for kw in (dict(logits=x.half()), dict(logits=x.t()), dict(logits=x[:, ::2]), dict(tokens=_i32([0] * 3)),
               dict(temperature=torch.ones(2).cuda()), dict(uniforms=torch.rand(4)), dict(kept=_i32([0] * 4)),
               dict(draft_probs=x[:, :50]), dict(draft_probs=x.bfloat16()), dict(parents=_i32([0] * 3)),
               dict(draft_probs=x.clone(), parents=_i32([0] * 4)), dict(workspace=None),
               dict(kept=t["num_kept"][:, None]), dict(logits=x[:2].expand(4, 2, 100)[:, 0])):
        with pytest.raises((ValueError, TypeError, binding.RagError)):
            binding.rag_draft_verify(**{**t, **kw})
