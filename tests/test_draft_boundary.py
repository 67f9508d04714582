"""The page, tree, keep and key-range entry points on the CPU: bad host
arguments are refused with the documented status before anything is enqueued,
documented no-ops return RAG_OK, and the references of the GPU tests agree with
brute force.  No call here reaches a launch."""
import math
import os
import random

import pytest
import torch

import brute
import draft_support as ds
from paper_2412_10543_amd import binding

needs_lib = pytest.mark.skipif(not os.path.exists(binding.LIBRARY),
                               reason="librag_attn.so not built")
FAKE = 0x100000
BAD, NO, WS, OK = (binding.RAG_ERR_INVALID_ARG, binding.RAG_ERR_UNSUPPORTED,
                   binding.RAG_ERR_WORKSPACE, binding.RAG_OK)


def _says(status, want):
    assert status == want
    assert (binding.rag_last_error() == "") == (want == OK)


@needs_lib
@pytest.mark.parametrize("kw,status", [
    (dict(num_free=None), BAD), (dict(num_free_out=None), BAD), (dict(cu=None), BAD),
    (dict(granted=None), BAD), (dict(old=None), BAD), (dict(new=None), BAD), (dict(lens=None), BAD),
    (dict(table=None), BAD), (dict(stack=None), BAD), (dict(slots=None), BAD),
    (dict(S=-1), BAD), (dict(tokens=-1), BAD), (dict(width=-1), BAD), (dict(blocks=-1), BAD),
    (dict(num_free_out=FAKE + 64), BAD), (dict(lens=FAKE + 128), BAD), (dict(lens=FAKE + 192), BAD),
    (dict(granted=FAKE + 64), BAD),
    (dict(bs=32), NO), (dict(S=4097), NO), (dict(tokens=1 << 30), NO), (dict(blocks=(1 << 27) + 1), NO),
    (dict(width=1 << 27), NO),
])
def test_pages_refusals(kw, status):
    a = dict(table=FAKE, stack=FAKE + 32, num_free=FAKE + 64, old=FAKE + 128, new=FAKE + 192, S=4,
             width=8, blocks=100, bs=16, tokens=64, num_free_out=FAKE + 256, lens=FAKE + 320,
             cu=FAKE + 384, slots=FAKE + 448, granted=FAKE + 512)
    a.update(kw)
    _says(binding.lib().rag_kv_pages_update(*a.values(), None), status)


# the arrays of rag_kv_pages_update and their int32 values for 4 rows, 8 pages a row, 100 pages
# and 64 slots; the call writes those of the first line
PAGES_ARRAYS = dict(table=32, stack=100, num_free_out=1, lens=4, cu=5, slots=64, granted=1,
                    num_free=1, old=4, new=4)
PAGES_WRITTEN = list(PAGES_ARRAYS)[:7]


@needs_lib
@pytest.mark.parametrize("a,b", [(a, b) for i, a in enumerate(PAGES_WRITTEN)
                                 for b in list(PAGES_ARRAYS)[i + 1:]])
def test_pages_refuse_a_written_array_that_overlaps_another(a, b):
    """Every workgroup reads the inputs while others write: whole, by the first
    value and by the last."""
    at = {name: FAKE + 4096 * i for i, name in enumerate(PAGES_ARRAYS)}
    order = ["table", "stack", "num_free", "old", "new", "S", "width", "blocks", "bs", "tokens",
             "num_free_out", "lens", "cu", "slots", "granted"]
    for shift in (0, PAGES_ARRAYS[b] - 1, 1 - PAGES_ARRAYS[a]):
        v = dict(at, S=4, width=8, blocks=100, bs=16, tokens=64)
        v[a] = at[b] + 4 * shift
        _says(binding.lib().rag_kv_pages_update(*(v[n] for n in order), None), BAD)
        assert "overlap" in binding.rag_last_error()


@needs_lib
@pytest.mark.parametrize("kw,status", [
    (dict(kc=None), BAD), (dict(vc=None), BAD), (dict(table=None), BAD), (dict(base=None), BAD),
    (dict(kept=None), BAD), (dict(n=None), BAD), (dict(S=-1), BAD), (dict(max_kept=-1), BAD),
    (dict(hkv=0), BAD), (dict(kc=FAKE + 8), BAD), (dict(vc=FAKE + 2), BAD), (dict(blocks=-1), BAD),
    (dict(d=96), NO), (dict(bs=8), NO), (dict(S=1 << 30, hkv=8), NO),
    (dict(S=0), OK), (dict(max_kept=0), OK), (dict(width=0), OK),
])
def test_keep_refusals(kw, status):
    a = dict(kc=FAKE, vc=FAKE, table=FAKE, base=FAKE, kept=FAKE, n=FAKE, S=4, width=8, max_kept=5,
             blocks=100, hkv=8, d=128, bs=16)
    a.update(kw)
    _says(binding.lib().rag_kv_cache_keep(*a.values(), None), status)


@needs_lib
@pytest.mark.parametrize("kw,status", [
    (dict(q=None), BAD), (dict(kc=None), BAD), (dict(vc=None), BAD), (dict(o=None), BAD),
    (dict(mask=None), BAD), (dict(table=None), BAD), (dict(kv=None), BAD), (dict(cu=None), BAD),
    (dict(S=-1), BAD), (dict(nodes=-1), BAD), (dict(words=-1), BAD), (dict(splits=-1), BAD),
    (dict(nodes=65), BAD), (dict(words=0), BAD), (dict(hq=12), BAD), (dict(hkv=0), BAD),
    (dict(scale=0.0), BAD), (dict(scale=math.nan), BAD), (dict(scale=math.inf), BAD),
    (dict(q=FAKE + 8), BAD), (dict(o=FAKE + 4), BAD), (dict(mask=FAKE + 4), BAD),
    (dict(width=0), BAD), (dict(d=80), NO), (dict(bs=32), NO),
    (dict(nodes=1 << 20, words=1 << 14), NO), (dict(width=1 << 27), NO),
    (dict(splits=4), WS), (dict(splits=4, ws=FAKE, ws_bytes=100), WS),
    (dict(splits=4, ws=FAKE + 64, ws_bytes=1 << 40), BAD),
    (dict(S=0), OK), (dict(nodes=0), OK),
])
def test_tree_refusals(kw, status):
    a = dict(q=FAKE, kc=FAKE, vc=FAKE, o=FAKE, mask=FAKE, table=FAKE, kv=FAKE, cu=FAKE, S=2,
             nodes=10, words=1, width=64, blocks=300, hq=32, hkv=8, d=128, bs=16, scale=0.088,
             splits=1, ws=None, ws_bytes=0)
    a.update(kw)
    _says(binding.lib().rag_attn_decode_paged_tree(*a.values(), None), status)


@needs_lib
@pytest.mark.parametrize("kw,status", [
    (dict(q=None), BAD), (dict(k=None), BAD), (dict(v=None), BAD), (dict(o=None), BAD),
    (dict(cu_q=None), BAD), (dict(cu_k=None), BAD), (dict(ranges=None), BAD), (dict(S=-1), BAD),
    (dict(max_q=-1), BAD), (dict(max_k=-1), BAD), (dict(hq=6, hkv=4), BAD), (dict(scale=-1.0), BAD),
    (dict(k=FAKE + 8), BAD), (dict(ranges=FAKE + 4), BAD), (dict(d=256), NO),
    (dict(S=1 << 20, max_q=1 << 20), NO), (dict(S=0), OK), (dict(max_q=0), OK),
])
def test_ranges_refusals(kw, status):
    a = dict(q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=None, cu_q=FAKE, cu_k=FAKE, ranges=FAKE, S=1,
             max_q=16, max_k=16, hq=4, hkv=2, d=64, scale=0.125)
    a.update(kw)
    _says(binding.lib().rag_attn_prefill_varlen_ranges(*a.values(), None), status)


@needs_lib
def test_tree_workspace_sizes():
    f = binding.rag_attn_decode_tree_workspace_size
    assert f(0, 8, 32, 8, 128, 64) == f(4, 0, 32, 8, 128, 64) == f(4, 8, 30, 8, 128, 64) == 0
    assert f(4, 8, 32, 8, 128, 0) == 0 and f(4, 8, 32, 8, 128, 64, num_splits=1) == 0
    one = 4 * 8 * 32 * 129 * 4
    for n in (2, 3, 16):
        assert n * one <= f(4, 8, 32, 8, 128, 64, num_splits=n) < n * one + 1024
    for s in (1, 7, 64):                  # large enough for any choice, never beyond 64 pieces
        assert f(s, 64, 32, 8, 128, 2300) <= 64 * s * 64 * 32 * 129 * 4 + 1024


@needs_lib
@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (4, 2, 64), (64, 8, 128), (25, 1, 128), (14, 2, 64),
                                      (600, 600, 128), (900, 900, 64)])
@pytest.mark.parametrize("splits", [0, 1, 2, 3, 64])
def test_tree_workspace_of_the_largest_step_serves_every_smaller_one(hq, hkv, d, splits):
    axes = [(1, 2, 4, 8, 16, 17, 63, 64, 65, 100, 255, 256, 257, 1000, 100000),
            (1, 2, 7, 8, 16, 17, 31, 32, 33, 64, 65, 100, 127, 128, 130, 300, 1000),
            (1, 15, 16, 29, 31, 32, 33, 64, 100, 125, 126, 127, 128, 650, 2300, 1 << 20)]
    size = {(s, n, w): binding.rag_attn_decode_tree_workspace_size(s, n, hq, hkv, d, w,
                                                                   num_splits=splits)
            for s in axes[0] for n in axes[1] for w in axes[2]}
    for at in size:
        for i, axis in enumerate(axes):
            k = axis.index(at[i]) + 1
            if k < len(axis):
                more = (*at[:i], axis[k], *at[i + 1:])
                assert size[at] <= size[more], (at, more)


@needs_lib
def test_binding_refuses_what_is_not_on_the_gpu():
    i32 = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    c = torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16)
    t = torch.zeros((4, 2), dtype=torch.int32)
    for call in (lambda: binding.rag_kv_pages_update(t, i32, i32[:1], i32, i32, i32[:1], i32, i32,
                                                     i32, i32[:1]),
                 lambda: binding.rag_kv_cache_keep(c, c, t, i32, t, i32),
                 lambda: binding.rag_attn_decode_paged_tree(x, c, c, x, t.long(), t, i32, i32, 1, 1.0),
                 lambda: binding.rag_attn_prefill_varlen_ranges(x, x, x, x, None, i32, i32, t, 4, 4,
                                                                1.0)):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()
    for first in (None, [1, 2], 7):
        with pytest.raises(TypeError, match="q must be a torch.Tensor"):
            binding.rag_attn_prefill_varlen_ranges(first, x, x, x, None, i32, i32, t, 4, 4, 1.0)


# ---------------------------------------------------------------------------
# the references themselves
# ---------------------------------------------------------------------------
def test_reference_against_brute_force():
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn((n, 8), generator=g, dtype=torch.float64) for n in (5, 9, 9))
    seen = torch.rand((5, 9), generator=g) < 0.5
    seen[2] = False
    o, lse, bo, _ = ds.attend64(q, k, v, seen, 0.4)
    assert (o[2] == 0).all() and lse[2] == -math.inf and (bo >= 0).all()
    for i in (0, 1, 3, 4):
        at = [j for j in range(9) if seen[i, j]]
        want, ll = brute.attend([q[i].tolist()], k[at].tolist(), v[at].tolist(), 0.4, causal=False)
        assert torch.allclose(o[i], torch.tensor(want[0], dtype=torch.float64), atol=1e-12)
        assert abs(lse[i].item() - ll[0]) < 1e-12


def test_reference_ignores_unseen_values_and_marks_seen_ones():
    q, k, v = torch.ones((2, 4)), torch.ones((3, 4)), torch.ones((3, 4))
    v[1, 2] = math.nan
    k[2, 0] = math.inf
    seen = torch.tensor([[True, False, False], [True, True, False]])
    o, _, b, _ = ds.attend64(q, k, v, seen, 1.0)
    assert (o[0] == 1).all() and torch.isfinite(b[0]).all() and torch.isnan(b[1]).all()


def test_range_masks():
    assert ds.range_seen(3, 5, [(2, 3), (0, 9), (-4, -1)]).tolist() == [
        [True, True, False, False, False], [False] * 5, [True] * 5]
    assert ds.range_seen(2, 1, [(0, 0), (0, 0)]).tolist() == [[False], [True]]   # p = -1, 0


def test_mask_words_round_trip():
    rng = random.Random(5)
    parents = ds.tree_parents(rng, 70)
    seen = ds.ancestor_seen(parents)
    w = ds.mask_words([seen], 2, fill=-1)
    for i in range(70):
        bits = (int(w[i, 0]) & (1 << 64) - 1) | (int(w[i, 1]) & (1 << 64) - 1) << 64
        assert [bool(bits >> j & 1) for j in range(70)] == seen[i].tolist()
        assert bits >> 70 == (1 << 58) - 1
    node, path = 69, set()
    while node >= 0:
        path.add(node)
        node = parents[node]
    assert {j for j in range(70) if seen[69, j]} == path


def test_reference_pages_by_hand():
    # row 0 gives back pages 7 and 8 (keeps 5), row 1 grows by two pages, row 2 not
    r = ds.reference_pages([[5, 7, 8], [9, 0, 0], [1, 2, 0]], [3, 4, 0, 0, 0, 0], 2, [40, 16, 20],
                           [10, 41, 24], 100)
    assert r["table"] == [[5, 7, 8], [9, 8, 7], [1, 2, 0]]
    assert r["free"] == 2 and r["lens"] == [10, 41, 24] and r["cu"] == [0, 0, 25, 29]
    assert r["granted"] == 3
    assert r["slots"][:2] == [128, 129] and r["slots"][24] == 7 * 16 + 8
    assert r["slots"][25:29] == [2 * 16 + 4, 2 * 16 + 5, 2 * 16 + 6, 2 * 16 + 7]
    # a capacity of 25 slots: the last row does not fit
    r = ds.reference_pages([[5, 7, 8], [9, 0, 0], [1, 2, 0]], [3, 4, 0, 0, 0, 0], 2, [40, 16, 20],
                           [10, 41, 24], 25)
    assert r["granted"] == 2 and r["lens"] == [10, 41, 20] and r["cu"] == [0, 0, 25, 25]
