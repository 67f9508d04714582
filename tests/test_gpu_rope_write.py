"""rag_qkv_rope_write and rag_qkv_rope_write_kv4 on the GPU: every output against the
64-bit reference, the caches bit by bit, and what must stay as it was."""
import math

import pytest
import torch

import serve_support as ss
from paper_2412_10543_amd import binding

pytestmark = pytest.mark.gpu

MARK = -7.0


def _draw(shape, g, scale=1.0):
    return (scale * torch.randn(shape, generator=g)).bfloat16()


def _case(T, hq, hkv, d, rot, seed, norm=True, pad=0.0, most=300, blocks=None):
    """Parts of one projection's rows, slots in random order, some tokens padding."""
    g = torch.Generator().manual_seed(seed)
    blocks = blocks or (T + 15) // 16 + 3
    qkv = _draw((T, hq + 2 * hkv, d), g, 1.5)
    slots = torch.randperm(blocks * 16, generator=g)[:T].int()
    slots[torch.rand(T, generator=g) < pad] = -1
    pos = torch.randint(0, most, (T,), generator=g).int()
    pos[slots < 0] = 1 << 30                     # not looked at
    c = dict(qkv=qkv, q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], slots=slots, pos=pos,
             cs=ss.angles(most, rot) if rot else None, blocks=blocks,
             qw=_draw((d,), g) if norm else None, kw=_draw((d,), g) if norm else None)
    return c


def _gpu(x):
    return None if x is None else x.cuda()


def _run(c, d, kv4, interleaved=False, eps=1e-6, rows_out=True, with_q=True):
    T, hkv = c["k"].shape[:2]
    qkv = c["qkv"].cuda()
    hq = c["q"].shape[1]
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    new = lambda h: torch.full((T, h, d), MARK, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    out = dict(q=new(hq) if with_q else None, k=new(hkv) if rows_out else None,
               v=new(hkv) if rows_out else None)
    if kv4:
        g = torch.Generator().manual_seed(1)
        caches = [torch.randint(0, 256, (c["blocks"], hkv, 9 * d), generator=g, dtype=torch.uint8)
                  for _ in range(2)]
    else:
        caches = [torch.full((c["blocks"], hkv, 16, d), MARK, dtype=torch.bfloat16) for _ in range(2)]
    out["before"] = caches
    kc, vc = (x.cuda() for x in caches)
    call = binding.rag_qkv_rope_write_kv4 if kv4 else binding.rag_qkv_rope_write
    call(q if with_q else None, k, v, out["q"], _gpu(c["pos"]) if c["cs"] is not None else None,
         _gpu(c["cs"]), _gpu(c["slots"]), kc, vc, k_out=out["k"], v_out=out["v"],
         q_weight=_gpu(c["qw"]) if with_q else None, k_weight=_gpu(c["kw"]), eps=eps,
         interleaved=interleaved)
    torch.cuda.synchronize()
    assert torch.equal(qkv.cpu().view(torch.int16), c["qkv"].view(torch.int16))
    out.update(kc=kc.cpu(), vc=vc.cpu(), **{n: None if out[n] is None else out[n].cpu() for n in "qkv"})
    return out


def _check_rows(c, out, interleaved, eps=1e-6):
    real = c["slots"] >= 0
    pos = torch.where(real, c["pos"], 0) if c["cs"] is not None else None
    for name, x, w in (("q", c["q"], c["qw"]), ("k", c["k"], c["kw"])):
        want, bound = ss.reference_rope(x, w, eps, pos, c["cs"], interleaved)
        over = ((out[name].double() - want).abs() - bound)[real]
        assert over.numel() == 0 or over.max() <= 0, (name, over.max())
        assert (out[name][~real] == MARK).all()
    assert torch.equal(out["v"][real], c["v"][real])
    assert (out["v"][~real] == MARK).all()


SHAPES = [(32, 8, 128), (4, 2, 64), (14, 2, 64), (5, 1, 128), (16, 16, 128), (1, 1, 64)]


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("T", [1, 2, 5, 33, 260])
@pytest.mark.parametrize("interleaved", [False, True])
def test_bf16_rows_and_cache(hq, hkv, d, T, interleaved):
    for i, rot in enumerate((d, d // 2, 16, 48)):
        c = _case(T, hq, hkv, d, rot, seed=T * 10 + i, norm=i % 2 == 0, pad=0.2 if T > 2 else 0.0)
        out = _run(c, d, False, interleaved)
        _check_rows(c, out, interleaved)
        for cache, before, rows in ((out["kc"], out["before"][0], out["k"]),
                                    (out["vc"], out["before"][1], out["v"])):
            want = before.clone()
            for t, s in enumerate(c["slots"].tolist()):
                if s >= 0:
                    want[s // 16, :, s % 16] = rows[t]
            assert torch.equal(cache, want)


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("T", [1, 3, 18])
def test_kv4_pages(hq, hkv, d, T):
    """Every byte of the pools: the codes of the rounded rows, one token at a time."""
    for i, rot in enumerate((d, 32)):
        c = _case(T, hq, hkv, d, rot, seed=T * 10 + i, norm=i == 0, pad=0.2 if T > 2 else 0.0, blocks=3)
        out = _run(c, d, True, interleaved=i == 1)
        _check_rows(c, out, i == 1)
        for cache, before, rows, values in ((out["kc"], out["before"][0], out["k"], False),
                                            (out["vc"], out["before"][1], out["v"], True)):
            pages = [[bytearray(before[b, h].numpy().tobytes()) for h in range(hkv)] for b in range(3)]
            for t, s in enumerate(c["slots"].tolist()):
                if s >= 0:
                    for h in range(hkv):
                        ss.page_put(pages[s // 16][h], d, s % 16, values, ss.quantize(rows[t, h].tolist()))
            want = torch.tensor([[list(p) for p in row] for row in pages], dtype=torch.uint8)
            assert torch.equal(cache, want)


@pytest.mark.parametrize("d", [64, 128])
def test_kv4_of_unusual_values(d):
    """Zeros, one sign only, steps far apart, the least and greatest bf16, NaN and
    infinities: a group's own value and the other groups' are as documented."""
    g = torch.Generator().manual_seed(3)
    rows = torch.randn((16, d), generator=g).bfloat16()
    big, tiny = 3.38e38, 1e-40
    rows[0] = 0
    rows[1] = rows[1].abs()
    rows[2] = -rows[2].abs()
    rows[3, :64] *= 1e30
    rows[4, :64] = torch.tensor([big, -big] * 32).bfloat16()
    rows[5, :64] = tiny
    rows[6, :64] = torch.tensor([9.3e-41, -9.3e-41] + [0.0] * 62).bfloat16()
    rows[7, 5] = math.nan
    rows[8, 6] = math.inf
    rows[9, 63] = -math.inf
    rows[10] = torch.arange(d).bfloat16() / 4    # ties
    rows[11] = -torch.arange(d).bfloat16() / 8 + 3.5
    rows[12, 0] = 1e20
    rows[13, :] = 1.0
    rows[14, :] = -2.0
    kv = rows[:, None].cuda()
    kc = torch.full((1, 1, 9 * d), 0x5a, dtype=torch.uint8, device="cuda")
    vc = kc.clone()
    slots = torch.arange(16, dtype=torch.int32, device="cuda")
    binding.rag_qkv_rope_write_kv4(None, kv, kv, None, None, None, slots, kc, vc)
    for cache, values in ((kc, False), (vc, True)):
        page = bytearray(cache.cpu().numpy().tobytes())
        for t in range(16):
            for got, want in zip(ss.page_get(page, d, t, values), ss.quantize(rows[t].tolist())):
                if math.isnan(want[2]):
                    assert math.isnan(got[2]) and math.isfinite(got[1]) and set(got[0]) == {0}
                else:
                    assert got == want, (t, values)
    cu = torch.tensor([0, 16], dtype=torch.int32, device="cuda")
    table = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    k, v = torch.empty_like(kv), torch.empty_like(kv)
    binding.rag_kv4_read(kc, vc, table, cu, k, v)
    for x in (k.cpu()[:, 0], v.cpu()[:, 0]):
        for t in range(16):
            want = torch.tensor([math.nan if z is None else s * (c - z)
                                 for codes, z, s in ss.quantize(rows[t].tolist()) for c in codes],
                                dtype=torch.float64).float().bfloat16()
            assert torch.equal(x[t].isnan(), want.isnan())
            assert torch.equal(x[t][~want.isnan()], want[~want.isnan()])


def test_copies_stay_bit_by_bit():
    """Without norm and rotation, and in channels that are not turned: NaN, infinities and
    all others as they were; the call equals rag_kv_cache_write."""
    T, hq, hkv, d = 40, 4, 2, 128
    c = _case(T, hq, hkv, d, 0, seed=4, norm=False)
    c["qkv"][3, :, 100] = math.nan
    c["qkv"][5, :, 90] = math.inf
    c["qkv"][6, :, 127] = -math.inf
    out = _run(c, d, False)
    kc = torch.full((c["blocks"], hkv, 16, d), MARK, dtype=torch.bfloat16, device="cuda")
    vc = kc.clone()
    binding.rag_kv_cache_write(c["k"].contiguous().cuda(), c["v"].contiguous().cuda(), kc, vc,
                               c["slots"].cuda())
    bits = lambda x: x.cpu().view(torch.int16)  # noqa: E731
    assert torch.equal(bits(out["kc"]), bits(kc)) and torch.equal(bits(out["vc"]), bits(vc))
    assert torch.equal(bits(out["q"]), bits(c["q"].contiguous()))
    c["cs"], c["pos"] = ss.angles(300, 32), c["pos"]
    out = _run(c, d, False)
    assert torch.equal(bits(out["q"][..., 32:].contiguous()), bits(c["q"][..., 32:].contiguous()))
    assert torch.equal(bits(out["k"][..., 32:].contiguous()), bits(c["k"][..., 32:].contiguous()))


@pytest.mark.parametrize("kv4", [False, True])
def test_parts_of_the_call_alone(kv4):
    """K and V without Q; without packed rows; rows without a cache; in place."""
    T, hq, hkv, d = 50, 6, 2, 128
    c = _case(T, hq, hkv, d, 64, seed=6)
    full = _run(c, d, kv4)
    for kw in (dict(with_q=False), dict(rows_out=False), dict(with_q=False, rows_out=False)):
        part = _run(c, d, kv4, **kw)
        assert torch.equal(part["kc"], full["kc"]) and torch.equal(part["vc"], full["vc"])
        for n in "qkv":
            assert part[n] is None or torch.equal(part[n], full[n])
    q, k, v = (c[n].contiguous().cuda() for n in "qkv")
    binding.rag_qkv_rope_write(q, k, v, q, c["pos"].cuda(), c["cs"].cuda(), k_out=k, v_out=v,
                               q_weight=c["qw"].cuda(), k_weight=c["kw"].cuda())
    assert torch.equal(q.cpu(), full["q"]) and torch.equal(k.cpu(), full["k"])
    assert torch.equal(v.cpu(), c["v"])


def test_norms_of_small_and_large_rows():
    """eps counts beside small rows; large rows' squares do not overflow where fp32 holds
    them; a row of zeros stays zero."""
    T, hq, hkv, d = 6, 2, 1, 64
    c = _case(T, hq, hkv, d, 64, seed=7)
    c["qkv"][0] *= 1e-4
    c["qkv"][1] *= 1e15
    c["qkv"][2] = 0
    out = _run(c, d, False, eps=1e-5)
    _check_rows(c, out, False, eps=1e-5)
    assert (out["q"][2] == 0).all()


# Launches whose waves have every second to every eleventh step of a token's heads.
@pytest.mark.parametrize("T,hq,hkv,d", [(400, 32, 8, 128), (700, 32, 8, 128), (1500, 32, 8, 128),
                                        (2700, 32, 8, 128), (2300, 14, 2, 64), (1400, 30, 5, 64)])
def test_tokens_whose_heads_some_waves_share(T, hq, hkv, d):
    c = _case(T, hq, hkv, d, d // 2, seed=T, pad=0.05)
    out, four = _run(c, d, False), _run(c, d, True)
    _check_rows(c, out, False)
    assert torch.equal(out["q"], four["q"]) and torch.equal(out["k"], four["k"])
    real = c["slots"] >= 0
    at = c["slots"][real].long()
    for cache, before, rows in ((out["kc"], out["before"][0], out["k"]), (out["vc"], out["before"][1], out["v"])):
        want = before.clone()
        want[at // 16, :, at % 16] = rows[real]
        assert torch.equal(cache, want)
    # the 4-bit pages: those that calls of a few tokens each write
    kc, vc = (x.cuda() for x in four["before"])
    qkv = c["qkv"].cuda()
    for a in range(0, T, 18):
        part = slice(a, min(a + 18, T))
        binding.rag_qkv_rope_write_kv4(None, qkv[part, hq:hq + hkv], qkv[part, hq + hkv:], None,
                                       c["pos"][part].cuda(), c["cs"].cuda(), c["slots"][part].cuda(), kc, vc,
                                       k_weight=c["kw"].cuda())
    assert torch.equal(four["kc"], kc.cpu()) and torch.equal(four["vc"], vc.cpu())


@pytest.mark.parametrize("T,hq,hkv,d", [(4500, 32, 8, 128), (9001, 4, 2, 64)])
def test_many_tokens(T, hq, hkv, d):
    """Launches that walk over a token's heads in one wave: the same rows as few tokens."""
    c = _case(T, hq, hkv, d, d, seed=8, pad=0.05)
    out = _run(c, d, False)
    kv4 = _run(c, d, True)
    assert torch.equal(out["q"], kv4["q"]) and torch.equal(out["k"], kv4["k"])
    some = torch.randperm(T)[:40].sort().values
    few = {n: c[n] for n in ("cs", "qw", "kw", "blocks")}
    few.update(qkv=c["qkv"][some], q=c["q"][some], k=c["k"][some], v=c["v"][some],
               slots=c["slots"][some], pos=c["pos"][some])
    part = _run(few, d, False)
    for n in "qkv":
        assert torch.equal(part[n], out[n][some])
    _check_rows(few, part, False)
    real = c["slots"] >= 0
    at = c["slots"][real].long()
    assert torch.equal(out["kc"].permute(0, 2, 1, 3).reshape(-1, hkv, d)[at], out["k"][real])
    assert torch.equal(out["vc"].permute(0, 2, 1, 3).reshape(-1, hkv, d)[at], c["v"][real])
    # the 4-bit pages: hi - lo is up to 15 s (1 + 2^-8), s being rounded to bf16, and z is off by
    # up to 1/2, so that hi / s + z is up to 15 (1 + 2^-8) + 1/2: the code 15 stands for a value
    # at most (1/2 + 15 2^-8) s = 0.5586 s below it; all others round by s / 2
    for cache, rows, values in ((kv4["kc"], out["k"], False), (kv4["vc"], out["v"], True)):
        got, steps = (x.reshape(-1, hkv, d)[at] for x in ss.unpack(cache, d, values))
        assert ((got - rows[real].double()).abs() <= 0.5586 * steps).all()
        step = rows[real].double().unflatten(2, (-1, 64))
        step = (step.amax(3).clamp(min=0) - step.amin(3).clamp(max=0)) / 15
        assert ((steps.unflatten(2, (-1, 64))[..., 0] - step).abs() <= 2.0 ** -8 * step).all()


def test_shapes_are_refused():
    T, hq, hkv, d = 4, 4, 2, 64
    c = {n: _gpu(x) if isinstance(x, torch.Tensor) else x for n, x in _case(T, hq, hkv, d, 64, 9).items()}
    kc = torch.zeros((c["blocks"], hkv, 16, d), dtype=torch.bfloat16, device="cuda")
    k4 = torch.zeros((c["blocks"], hkv, 9 * d), dtype=torch.uint8, device="cuda")
    qo = torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda")

    def call(**kw):
        a = dict(q=c["q"], k=c["k"], v=c["v"], q_out=qo, positions=c["pos"], cos_sin=c["cs"],
                 slot_mapping=c["slots"], k_cache=kc, v_cache=kc.clone())
        a.update(kw)
        binding.rag_qkv_rope_write(**a)

    call()
    for kw in (dict(q=c["q"].float()), dict(q=c["q"][:3]), dict(v=c["v"][:, :1]), dict(q_out=qo[:, :2]),
               dict(positions=c["pos"].long()), dict(positions=c["pos"][:2]), dict(k_cache=k4),
               dict(k_cache=kc[:, :1]), dict(k=c["k"].transpose(1, 2).contiguous().transpose(1, 2)),
               dict(slot_mapping=c["slots"].cpu()), dict(q_weight=torch.ones(32, device="cuda").bfloat16()),
               dict(cos_sin=c["cs"].double()), dict(k=c["k"][0]), dict(k_out=qo[:, :2].contiguous())):
        with pytest.raises((ValueError, TypeError, binding.RagError)):
            call(**kw)
    with pytest.raises(binding.RagError):                  # its own row, twice
        binding.rag_qkv_rope_write(c["q"], c["k"], c["v"], qo, c["pos"], c["cs"], c["slots"], kc, kc)
