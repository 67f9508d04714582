"""The entry points of the new tokens' way into the caches, of the 4-bit cache and of
the verification on the CPU: bad host arguments are refused with the documented status
before anything is enqueued, documented no-ops return RAG_OK, and the references of the
GPU tests agree with brute force.  No call here reaches a launch."""
import math
import os
import random

import numpy as np
import pytest
import torch

import serve_support as ss
from paper_2412_10543_amd import binding

needs_lib = pytest.mark.skipif(not os.path.exists(binding.LIBRARY),
                               reason="librag_attn.so not built")
FAKE = 1 << 40
STEP = 1 << 32                   # between the arrays of a call
BAD, NO, WS, OK = (binding.RAG_ERR_INVALID_ARG, binding.RAG_ERR_UNSUPPORTED,
                   binding.RAG_ERR_WORKSPACE, binding.RAG_OK)


def _says(status, want):
    assert status == want, (status, binding.rag_last_error())
    assert (binding.rag_last_error() == "") == (want == OK)


def _at(i):
    return FAKE + i * STEP


ROPE = dict(q=_at(0), k=_at(1), v=_at(2), qs=4096, ks=1024, vs=1024, qo=_at(3), ko=_at(4), vo=_at(5),
            kc=_at(6), vc=_at(7), slots=_at(8), pos=_at(9), cs=_at(10), most=1000, rot=128, inter=0,
            qw=_at(11), kw=_at(12), eps=1e-6, T=5, hq=32, hkv=8, d=128, bs=16, blocks=100)


@needs_lib
@pytest.mark.parametrize("kv4", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(k=None), BAD), (dict(v=None), BAD), (dict(q=None), BAD), (dict(qo=None), BAD),
    (dict(q=None, qo=None), BAD), (dict(ko=None), BAD), (dict(vo=None), BAD), (dict(kc=None), BAD),
    (dict(vc=None), BAD), (dict(slots=None), BAD), (dict(pos=None), BAD), (dict(cs=None), BAD),
    (dict(slots=None, kc=None, vc=None, ko=None, vo=None), BAD),
    (dict(T=-1), BAD), (dict(hq=-1), BAD), (dict(hq=0), BAD), (dict(hkv=0), BAD), (dict(blocks=-1), BAD),
    (dict(most=0), BAD), (dict(rot=0), BAD), (dict(rot=144), BAD), (dict(inter=2), BAD),
    (dict(eps=-1.0), BAD), (dict(eps=math.nan), BAD), (dict(eps=math.inf), BAD),
    (dict(qs=4088), BAD), (dict(ks=1028), BAD), (dict(vs=0), BAD), (dict(vs=-1024), BAD),
    (dict(qs=1 << 41), BAD),
    (dict(q=_at(0) + 8), BAD), (dict(k=_at(1) + 2), BAD), (dict(kc=_at(6) + 8), BAD),
    (dict(cs=_at(10) + 4), BAD), (dict(qw=_at(11) + 8), BAD), (dict(qo=_at(3) + 8), BAD),
    (dict(d=96), NO), (dict(bs=32), NO), (dict(rot=72), NO), (dict(blocks=(1 << 27) + 1), NO),
    (dict(hq=1 << 17, qs=1 << 24), NO),
    (dict(T=0), OK), (dict(T=0, k=None, slots=None), OK),
])
def test_rope_refusals(kv4, kw, status):
    a = dict(ROPE, **kw)
    if kv4 and a["slots"] is None and a["T"] > 0:
        status = BAD
    L = binding.lib()
    call = L.rag_qkv_rope_write_kv4 if kv4 else L.rag_qkv_rope_write
    _says(call(*a.values(), None), status)


@needs_lib
@pytest.mark.parametrize("a,b,bytes_b", [
    ("qo", "q", 5 * 8192), ("qo", "k", 5 * 2048), ("ko", "q", 5 * 8192), ("ko", "k", 5 * 2048),
    ("vo", "v", 5 * 2048), ("kc", "k", 5 * 2048), ("vc", "qo", 5 * 8192), ("kc", "vc", 100 * 8 * 4096),
    ("ko", "vo", 5 * 2048), ("vo", "k", 5 * 2048)])
def test_rope_refuses_outputs_that_overlap(a, b, bytes_b):
    for shift in (16, bytes_b - 16, -16):
        x = dict(ROPE)
        x[a] = x[b] + shift
        _says(binding.lib().rag_qkv_rope_write(*x.values(), None), BAD)
        assert "overlap" in binding.rag_last_error()


@needs_lib
@pytest.mark.parametrize("b,bytes_b", [("slots", 20), ("pos", 20), ("cs", 1000 * 128 * 4), ("qw", 256),
                                       ("kw", 256)])
@pytest.mark.parametrize("a", ["qo", "ko", "vo", "kc", "vc"])
def test_rope_refuses_outputs_over_its_other_inputs(a, b, bytes_b):
    """Slots, positions, angles and weights, in part or whole, in either call."""
    L = binding.lib()
    for call in (L.rag_qkv_rope_write, L.rag_qkv_rope_write_kv4):
        for shift in (0, 16 * ((bytes_b - 1) // 16), -16):
            x = dict(ROPE)
            x[a] = x[b] + shift
            _says(call(*x.values(), None), BAD)
            assert "overlap" in binding.rag_last_error()


READ = dict(kc=_at(0), vc=_at(1), table=_at(2), cu=_at(3), k=_at(4), v=_at(5), T=100, S=3, width=10,
            blocks=50, hkv=8, d=128, bs=16)


@needs_lib
@pytest.mark.parametrize("kw,status", [
    (dict(kc=None), BAD), (dict(vc=None), BAD), (dict(table=None), BAD), (dict(cu=None), BAD),
    (dict(k=None), BAD), (dict(v=None), BAD), (dict(T=-1), BAD), (dict(S=-1), BAD),
    (dict(width=-1), BAD), (dict(blocks=-1), BAD), (dict(hkv=0), BAD), (dict(kc=_at(0) + 8), BAD),
    (dict(k=_at(4) + 2), BAD), (dict(d=32), NO), (dict(bs=8), NO), (dict(width=1 << 27), NO),
    (dict(T=(1 << 31) - 1, hkv=1000), NO),
    (dict(T=0), OK), (dict(S=0), OK), (dict(width=0), OK),
])
def test_read_refusals(kw, status):
    _says(binding.lib().rag_kv4_read(*dict(READ, **kw).values(), None), status)


@needs_lib
@pytest.mark.parametrize("a,b,bytes_b", [
    ("k", "v", 100 * 2048), ("k", "kc", 50 * 8 * 1152), ("v", "vc", 50 * 8 * 1152), ("k", "vc", 50 * 8 * 1152),
    ("v", "table", 120), ("k", "table", 120), ("v", "cu", 16), ("k", "cu", 16)])
def test_read_refuses_outputs_that_overlap(a, b, bytes_b):
    for shift in (0, 16 * ((bytes_b - 1) // 16), -16):
        x = dict(READ)
        x[a] = x[b] + shift
        _says(binding.lib().rag_kv4_read(*x.values(), None), BAD)
        assert "overlap" in binding.rag_last_error()


ATTN = dict(q=_at(0), kc=_at(1), vc=_at(2), o=_at(3), table=_at(4), kv=_at(5), cu=_at(6), S=4, rows=3,
            width=20, blocks=100, hq=32, hkv=8, d=128, bs=16, scale=0.088, ws=_at(7), ws_bytes=1 << 30)


@needs_lib
@pytest.mark.parametrize("kw,status", [
    (dict(q=None), BAD), (dict(kc=None), BAD), (dict(vc=None), BAD), (dict(o=None), BAD),
    (dict(table=None), BAD), (dict(kv=None), BAD), (dict(S=-1), BAD), (dict(rows=-1), BAD),
    (dict(width=-1), BAD), (dict(hq=12), BAD), (dict(hq=0), BAD), (dict(hkv=0), BAD),
    (dict(scale=0.0), BAD), (dict(scale=math.nan), BAD), (dict(scale=math.inf), BAD),
    (dict(q=_at(0) + 8), BAD), (dict(o=_at(3) + 4), BAD), (dict(vc=_at(2) + 8), BAD),
    (dict(ws=_at(7) + 64), BAD), (dict(d=256), NO), (dict(bs=32), NO), (dict(rows=1 << 19), NO),
    (dict(blocks=(1 << 27) + 1), NO), (dict(ws=None), WS), (dict(ws_bytes=100), WS),
    (dict(S=0), OK), (dict(rows=0), OK),
])
def test_attention_refusals(kw, status):
    _says(binding.lib().rag_attn_decode_paged_kv4(*dict(ATTN, **kw).values(), None), status)


@needs_lib
@pytest.mark.parametrize("cu", [_at(6), None])
@pytest.mark.parametrize("a", ["o", "ws"])
@pytest.mark.parametrize("b,bytes_b", [("q", 4 * 8192), ("kc", 100 * 8 * 1152), ("vc", 100 * 8 * 1152),
                                       ("table", 320), ("kv", 16), ("cu", 20), ("ws", 4096), ("o", 4 * 8192)])
def test_attention_refuses_outputs_that_overlap(a, b, bytes_b, cu):
    if a == b or (b == "cu" and cu is None):
        return
    if cu and b in ("q", "o"):
        bytes_b = 8192                         # (a row at least)
    step = 256 if a == "ws" else 16
    for shift in (0, step * ((bytes_b - 1) // step), -step):
        if (a, b, shift) != ("o", "q", 0):     # (in place)
            x = dict(ATTN, cu=cu)
            x[a] = x[b] + shift
            _says(binding.lib().rag_attn_decode_paged_kv4(*x.values(), None), BAD)
            assert "overlap" in binding.rag_last_error()


@needs_lib
@pytest.mark.parametrize("x", [None, 3, np.zeros((2, 2), dtype=np.int32)])
@pytest.mark.parametrize("call,count,first", [
    ("rag_kv_pages_update", 10, "block_tables"), ("rag_kv_cache_keep", 6, "k_cache"),
    ("rag_kv4_read", 6, "k_cache"), ("rag_draft_verify", 8, "logits"), ("rag_qkv_rope_write", 6, "k"),
    ("rag_attn_decode_paged_kv4", 6, "q"), ("rag_attn_decode_paged_tree", 8, "q"),
    ("rag_attn_prefill_varlen_ranges", 8, "q")])
def test_arguments_that_are_no_tensors_are_named(call, count, first, x):
    """No tensor among them: the first is refused by its name, as it is among tensors."""
    more = {"rag_attn_decode_paged_kv4": (0.1,), "rag_attn_decode_paged_tree": (4, 0.1),
            "rag_attn_prefill_varlen_ranges": (8, 8, 0.1)}.get(call, ())
    with pytest.raises(TypeError, match=f"^{first} must be a torch.Tensor"):
        getattr(binding, call)(*[x] * count, *more)


@needs_lib
def test_attention_of_chains_is_told_their_length():
    """A length that the call took for granted would be a bound that longer chains break."""
    q = torch.zeros((4, 8, 64), dtype=torch.bfloat16)
    cache, i = torch.zeros((3, 2, 576), dtype=torch.uint8), torch.zeros((2, 1), dtype=torch.int32)
    args = (q, cache, cache.clone(), q.clone(), i, i[:, 0], 0.1)
    with pytest.raises(ValueError, match="max_seqlen_q"):
        binding.rag_attn_decode_paged_kv4(*args, cu_seqlens_q=torch.tensor([0, 1, 4], dtype=torch.int32))


@needs_lib
def test_launches_of_too_many_threads_are_refused():
    """A launch takes less than 2^32 threads: 2^24 workgroups of 256."""
    L = binding.lib()
    most = (1 << 31) - 1
    kw = dict(ROPE, hq=1, hkv=1, d=64, rot=64, qs=64, ks=64, vs=64, T=most)
    for i, name in enumerate(("q", "k", "v", "qo", "ko", "vo", "kc", "vc")):
        kw[name] = FAKE + i * (1 << 40)
    _says(L.rag_qkv_rope_write(*kw.values(), None), NO)
    _says(L.rag_kv4_read(*dict(READ, T=most, hkv=8).values(), None), NO)
    kw = dict(ATTN, S=1 << 19, hkv=32, cu=None)
    _says(L.rag_attn_decode_paged_kv4(*kw.values(), None), NO)
    kw = dict(VERIFY, T=1 << 20, V=1 << 20, ls=1 << 20, parents=None, ws_bytes=1 << 60)
    for i, name in enumerate(("logits", "tokens", "cu", "heat", "u", "kept", "n", "nxt", "ws")):
        kw[name] = FAKE + i * (1 << 44)
    _says(L.rag_draft_verify(*kw.values(), None), NO)


@needs_lib
def test_tables_wider_than_the_plan_counts():
    """Where the plan's places fit in 32 bits at the widest table that is taken, and did not at
    wider ones: 512 shares, each at least the longest tile's 62nd part, a block counted four times."""
    widest = 1 << 26
    longest = (widest // 2 + 24) * 4
    assert 512 * ((longest + 61) // 62) < 1 << 31 < 512 * (((1 << 26) - 1 + 24) * 4 // 62)
    assert 16 * (widest + 2 * 64) < 1 << 31              # a key of the last pages requested
    L = binding.lib()
    for width, want in ((widest, WS), (widest + 1, NO), ((1 << 27) - 1, NO)):
        _says(L.rag_attn_decode_paged_kv4(*dict(ATTN, S=1, width=width, ws=None).values(), None), want)
        n = binding.rag_attn_decode_kv4_workspace_size(1, 3, 32, 8, 128, width)
        assert (n > 0) == (want == WS)


@needs_lib
def test_attention_workspace_serves_smaller_calls():
    size = binding.rag_attn_decode_kv4_workspace_size
    for hq, hkv, d in ((32, 8, 128), (64, 8, 128), (14, 2, 64), (512, 512, 128)):
        last = 0
        for rows in (1, 2, 3, 4, 8, 9, 16, 17, 100):
            now = size(1, rows, hq, hkv, d, 10)
            assert now >= last > -1 and now > 0
            assert now == size(1024, rows, hq, hkv, d, 5000) == size(5000, rows, hq, hkv, d, 1)
            last = now
    for bad in ((0, 1, 32, 8, 128, 10), (1, 0, 32, 8, 128, 10), (1, 1, 32, 0, 128, 10),
                (1, 1, 30, 8, 128, 10), (1, 1, 32, 8, 96, 10), (1, 1, 32, 8, 128, 0)):
        assert size(*bad) == 0
    assert size(1, 1, 32, 8, 128, 10, 32) == 0


@needs_lib
def test_attention_workspace_is_of_its_heads():
    """Why the promise of smaller calls is one for the same heads: shares per kv head are whole
    workgroups, and fewer kv heads have more rows of q heads each."""
    size = binding.rag_attn_decode_kv4_workspace_size
    assert size(1, 1, 4, 4, 128, 10) > size(1, 1, 5, 5, 128, 10)
    assert size(1, 1, 256, 256, 128, 10) > size(1, 1, 300, 300, 128, 10)
    assert size(1, 1, 32, 8, 128, 10) > size(1, 1, 32, 32, 128, 10)
    header = open(os.path.join(os.path.dirname(binding.__file__), "..", "include", "rag_attn.h")).read()
    words = " ".join(header.replace("*", " ").split())
    assert "rag_attn_decode_paged_kv4 calls of these sizes and, with the same heads, of smaller ones" in words
    assert "for the same arguments or, with the same heads, for larger sizes" in words


VERIFY = dict(logits=_at(0), wide=0, ls=1000, draft=None, ds=0, tokens=_at(2), parents=_at(3), cu=_at(4),
              heat=_at(5), u=_at(6), kept=_at(7), n=_at(8), nxt=_at(9), T=20, S=4, V=1000, most=8,
              ws=_at(10), ws_bytes=1 << 30)


@needs_lib
@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), BAD), (dict(tokens=None), BAD), (dict(cu=None), BAD), (dict(heat=None), BAD),
    (dict(u=None), BAD), (dict(kept=None), BAD), (dict(n=None), BAD), (dict(nxt=None), BAD),
    (dict(T=-1), BAD), (dict(S=-1), BAD), (dict(V=0), BAD), (dict(most=-1), BAD), (dict(most=0), BAD),
    (dict(wide=2), BAD), (dict(ls=999), BAD), (dict(logits=_at(0) + 2), BAD),
    (dict(draft=_at(1), ds=999, parents=None), BAD), (dict(draft=_at(1) + 4, ds=1000, parents=None), BAD),
    (dict(ws=_at(10) + 128), BAD), (dict(kept=_at(2)), BAD), (dict(n=_at(4)), BAD),
    (dict(nxt=_at(8) + 12), BAD), (dict(kept=_at(10)), BAD), (dict(ws=_at(0)), BAD),
    (dict(draft=_at(1), ds=1000), NO), (dict(T=(1 << 20) + 1), NO), (dict(S=16385), NO),
    (dict(V=(1 << 28) + 1, ls=1 << 29), NO),
    (dict(ws=None), WS), (dict(ws_bytes=1000), WS), (dict(S=0), OK),
])
def test_verify_refusals(kw, status):
    _says(binding.lib().rag_draft_verify(*dict(VERIFY, **kw).values(), None), status)


@needs_lib
def test_verify_workspace_serves_smaller_calls():
    size = binding.rag_draft_verify_workspace_size
    steps = [(1, 1, 1), (5, 1, 4096), (5, 2, 4097), (300, 64, 128000), (300, 65, 128000),
             (1 << 20, 16384, 200000)]
    sizes = [size(*x) for x in steps]
    assert sizes == sorted(sizes) and sizes[0] > 0
    for bad in ((-1, 1, 10), (1, -1, 10), (1, 1, 0), ((1 << 20) + 1, 1, 10), (1, 16385, 10), (1, 1, (1 << 28) + 1)):
        assert size(*bad) == 0


# ---------------------------------------------------------------------------
# the references
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("values", [False, True])
def test_page_reference_round_trip(d, values):
    """Codes put in a page one by one come back, alone and all at once, whatever the order of
    the tokens; every nibble and parameter has a place of its own."""
    r = random.Random(d + values)
    rows = torch.randn((16, d), generator=torch.Generator().manual_seed(d)).bfloat16()
    rows[3] = 0
    rows[5, 64 * (d // 64) - 64:] = rows[5, :64].abs() + 1       # 0 is its least value
    page = bytearray(r.randbytes(9 * d))
    for t in r.sample(range(16), 16):
        ss.page_put(page, d, t, values, ss.quantize(rows[t].tolist()))
    cache = torch.tensor(list(page), dtype=torch.uint8).reshape(1, 1, 9 * d)
    (all_rows, steps) = ss.unpack(cache, d, values)
    for t in range(16):
        want = ss.quantize(rows[t].tolist())
        assert ss.page_get(page, d, t, values) == want
        flat = [s * (c - z) for codes, z, s in want for c in codes]
        assert all_rows[0, t, 0].tolist() == flat
        step = torch.tensor([s for _, _, s in want for _ in range(64)], dtype=torch.float64)
        assert (torch.tensor(flat, dtype=torch.float64) - rows[t].double()).abs().le(0.5586 * step).all()   # 1/2 + 15 2^-8
        assert steps[0, t, 0].tolist() == step.tolist()


def test_rope_reference_against_complex_turns():
    g = torch.Generator().manual_seed(5)
    x = torch.randn((7, 3, 64), generator=g).bfloat16()
    w = torch.randn(64, generator=g).bfloat16()
    pos = torch.randint(0, 50, (7,), generator=g)
    cs = ss.angles(50, 32)
    for inter in (False, True):
        got, _ = ss.reference_rope(x, w, 1e-5, pos, cs, inter)
        n = x.double() * w.double() / torch.sqrt(x.double().square().mean(2, keepdim=True) + 1e-5)
        a, b = (n[..., 0:32:2], n[..., 1:32:2]) if inter else (n[..., :16], n[..., 16:32])
        z = torch.complex(a, b) * torch.complex(cs[pos][:, None, :16].double(), cs[pos][:, None, 16:].double())
        want = torch.stack([z.real, z.imag], -1).flatten(2) if inter else torch.cat([z.real, z.imag], 2)
        assert torch.allclose(got[..., :32], want, rtol=1e-12, atol=1e-12)
        assert torch.equal(got[..., 32:], n[..., 32:])
        # the rotation keeps lengths, as cos and sin in fp32 do
        assert torch.allclose(got.norm(dim=2), n.norm(dim=2), rtol=1e-6)


def test_verified_text_is_distributed_as_the_model_s():
    """Over many random numbers the first token behind the root has the model's
    probabilities, whatever the drafter proposed: with its probabilities, and without."""
    vocab, n = 5, 40000
    g = torch.Generator().manual_seed(9)
    logits = torch.randn((1, vocab), generator=g)
    p = torch.softmax(logits[0].double(), 0)
    q = torch.softmax(1.5 * torch.randn(vocab, generator=g), 0)
    x = torch.multinomial(q, n, replacement=True, generator=g).tolist()
    u = torch.rand((n, 2), generator=g)
    for draft in (None, torch.stack([q, q])):
        counts = np.zeros(vocab)
        for i in range(n):
            kept, num, nxt = ss.reference_verify([logits[0].tolist()] * 2, [0, x[i]], [0, 2], [1.0],
                                                 u[i].tolist(), 2, draft=draft)
            counts[x[i] if num[0] == 2 else nxt[0]] += 1
        # five standard deviations of a binomial
        assert (np.abs(counts / n - p.numpy()) < 5 * np.sqrt(p.numpy() / n)).all()
