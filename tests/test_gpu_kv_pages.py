"""rag_kv_pages_update and rag_kv_cache_keep on the GPU, bit for bit against the
references, one page or one row after another."""
import random

import pytest
import torch

import draft_support as ds
from paper_2412_10543_amd import binding
from paper_2412_10543_amd.workloads import normal_bf16

pytestmark = pytest.mark.gpu

i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731


def layout(rng, old, width, spare):
    """Tables of rows of these lengths over shuffled pages, other entries -7; the
    free stack with garbage behind its pages."""
    blocks = sum(map(ds.pages_of, old)) + spare
    ids = list(range(blocks))
    rng.shuffle(ids)
    table = []
    for n in old:
        p = ds.pages_of(n)
        table.append(ids[:p] + [-7] * (width - p))
        ids = ids[p:]
    return table, ids + [-9] * (blocks - len(ids)), len(ids)


def update(table, stack, num_free, old, new, capacity, width, stream=None):
    t = i32(table) if table else torch.zeros((0, width), dtype=torch.int32, device="cuda")
    s, S = i32(stack), len(old)
    out = {n: torch.full((k,), -5, dtype=torch.int32, device="cuda")
           for n, k in (("free", 1), ("lens", S), ("cu", S + 1), ("slots", capacity), ("granted", 1))}
    binding.rag_kv_pages_update(t, s, i32([num_free]), i32(old), i32(new), out["free"], out["lens"],
                                out["cu"], out["slots"], out["granted"], stream=stream)
    torch.cuda.synchronize()
    r = {n: x.tolist() for n, x in out.items()}
    return dict(r, table=t.tolist(), stack=s.tolist(), free=r["free"][0], granted=r["granted"][0])


def check(table, stack, num_free, old, new, capacity, width):
    got = update(table, stack, num_free, old, new, capacity, width)
    want = ds.reference_pages(table, stack, num_free, old, new, capacity)
    for name in want:
        assert got[name] == want[name], name
    return want


@pytest.mark.parametrize("rows", [1, 2, 63, 64, 65, 255, 256, 257, 700, 4096])
@pytest.mark.parametrize("fit", ["all", "pages", "slots", "table"])
def test_random_batches(rows, fit):
    rng = random.Random(rows * 7 + len(fit))
    old = [rng.choice([0, 1, 15, 16, 17, rng.randint(0, 200)]) for _ in range(rows)]
    new = [max(0, n + rng.choice([0, 1, 16, -1, -17, -n, rng.randint(-90, 90)])) for n in old]
    width = max(map(ds.pages_of, old + new)) + 1
    need = sum(max(0, ds.pages_of(b) - ds.pages_of(a)) for a, b in zip(old, new))
    tokens = sum(max(0, b - a) for a, b in zip(old, new))
    table, stack, n = layout(rng, old, width, need if fit != "pages" else need // 5)
    if fit == "table":
        new[rng.randrange(rows)] = width * 16 + 1
    check(table, stack, n, old, new, tokens // 2 if fit == "slots" else tokens + rng.choice([0, 3, 1500]),
          width)


def test_nothing_to_do():
    assert check([], [4, 2, 0, 1, 3], 5, [], [], 9, 3)["cu"] == [0]
    assert check([], [4, 2, 0, 1, 3], 5, [], [], 0, 3)["free"] == 5
    assert check([[3, -7], [-7, -7]], [0, 1, 2, -9], 3, [16, 0], [16, 0], 0, 2)["granted"] == 2
    # no page at all, and a row that wants one
    assert check([[-7]], [], 0, [0], [1], 4, 1)["granted"] == 0
    # growth inside a page that is held takes none; with no slot for it, it waits
    assert check([[0]], [-9], 0, [3], [16], 13, 1)["granted"] == 1
    assert check([[0]], [-9], 0, [3], [16], 12, 1)["lens"] == [3]


def test_given_pages_are_taken_at_once():
    rng = random.Random(2)
    table, stack, n = layout(rng, [160, 0, 32], 12, 0)
    want = check(table, stack, n, [160, 0, 32], [0, 150, 40], 500, 12)
    # ten pages given, ten taken by row 1: row 2 would need an eleventh
    assert want["granted"] == 2 and want["free"] == 0 and want["lens"] == [0, 150, 32]


def test_lengths_beyond_any_sum():
    """Rows that ask for more than 32-bit sums hold are refused, those before them
    are served."""
    big = 2 ** 31 - 1
    check([[-7] * 3] * 5, list(range(20)), 20, [0] * 5, [17, big, big, big, big], 100, 3)
    check([[-7] * 3] * 3, list(range(20)), 20, [0] * 3, [big, 5, big], 100, 3)


def test_one_long_row_among_short_ones():
    rng = random.Random(4)
    old = [rng.randint(1, 60) for _ in range(40)]
    new = list(old)
    new[17] = 70001
    for i in range(0, 40, 3):
        new[i] += 1
    table, stack, n = layout(rng, old, 4400, 4500)
    check(table, stack, n, old, new, 70100, 4400)


def test_long_rows_that_end():
    """Many more pages come back than the slots' workgroups would put away."""
    rng = random.Random(11)
    old = [rng.randint(20000, 36000) for _ in range(30)] + [40, 7, 0]
    new = [0] * 29 + [17, 41, 0, 50]
    table, stack, n = layout(rng, old, 2300, 3)
    want = check(table, stack, n, old, new, 60, 2300)
    assert want["granted"] == 33 and want["free"] > 30000


def test_many_steps_keep_every_page_once():
    rng = random.Random(9)
    rows, width, blocks = 33, 20, 300
    table, stack, free, old = [[-7] * width for _ in range(rows)], list(range(blocks)), blocks, [0] * rows
    for step in range(25):
        new = [max(0, n + rng.choice([1, 5, 40, -3, -n])) for n in old]
        want = check(table, stack, free, old, new, 900, width)
        table, stack, free, old = want["table"], want["stack"], want["free"], want["lens"]
        held = [p for r, n in zip(table, old) for p in r[:ds.pages_of(n)]]
        assert sorted(held + stack[:free]) == list(range(blocks))


def test_arrays_side_by_side_in_one_buffer():
    """A program's step state as one allocation: arrays may touch, and the two inputs
    may be one."""
    rng = random.Random(5)
    old = [20, 0, 47, 16, 3]
    table, stack, n = layout(rng, old, 6, 20)
    for new in ([33, 50, 10, 17, 0], old):
        parts = [sum(table, []), stack, [n], [-5], [-5] * 5, [-5] * 6, [-5] * 80, [-5]] + \
            ([old] if new is old else [old, new])
        buf, at, views = i32(sum(parts, [])), 0, []
        for x in parts:
            views.append(buf[at:at + len(x)])
            at += len(x)
        t, s, free, free_out, lens, cu, slots, granted, o = views[:9]
        binding.rag_kv_pages_update(t.view(5, 6), s, free, o, views[-1], free_out, lens, cu, slots,
                                    granted)
        want = ds.reference_pages(table, stack, n, old, new, 80)
        got = [t.view(5, 6).tolist(), s.tolist(), free_out.item(), lens.tolist(), cu.tolist(),
               slots.tolist(), granted.item()]
        assert got == [want[x] for x in ("table", "stack", "free", "lens", "cu", "slots", "granted")]
        assert free.item() == n and o.tolist() == old and views[-1].tolist() == list(new)


# ---------------------------------------------------------------------------
# keep
# ---------------------------------------------------------------------------
def keep(base, kept, hkv, d, seed, max_kept=None, width_extra=0):
    """GPU and reference caches (as bits) after the accepted nodes moved."""
    rng = random.Random(seed)
    nodes = [max(k, default=-1) + 1 + rng.randint(0, 3) for k in kept]
    pages = [ds.pages_of(b + n) for b, n in zip(base, nodes)]
    width = max(pages + [1]) + width_extra
    ids = list(range(sum(pages) + 3))
    rng.shuffle(ids)
    table = []
    for p in pages:
        table.append(ids[:p] + [ids[-1]] * (width - p))
        ids = ids[p:]
    blocks = sum(pages) + 3
    kc, vc = (normal_bf16((blocks, hkv, 16, d), seed + i, "cuda") for i in (1, 2))
    kc.view(torch.int16).view(-1)[::97] = 0x7fc1          # NaN payloads move too
    most = max(map(len, kept)) if max_kept is None else max_kept
    refs = []
    for c in (kc, vc):
        x = c.clone().view(torch.int16).cpu()
        old = x.clone()
        for s, path in enumerate(kept):
            for i, node in enumerate(path):
                a, b = base[s] + node, base[s] + i
                x[table[s][b // 16], :, b % 16] = old[table[s][a // 16], :, a % 16]
        refs.append(x)
    rows = [list(p) + [-1] * (most - len(p)) for p in kept]
    binding.rag_kv_cache_keep(kc, vc, i32(table), i32(base), i32(rows).reshape(len(kept), most),
                              i32(list(map(len, kept))))
    torch.cuda.synchronize()
    return [(kc.view(torch.int16).cpu(), refs[0]), (vc.view(torch.int16).cpu(), refs[1])]


@pytest.mark.parametrize("hkv,d", [(1, 64), (2, 64), (8, 128), (3, 128)])
@pytest.mark.parametrize("seed", range(4))
def test_keep_random_paths(hkv, d, seed):
    rng = random.Random(seed)
    rows = rng.choice([1, 5, 40])
    kept = [sorted(rng.sample(range(64), rng.choice([0, 1, 2, 7, 8, 9, 16, 17, 33]))) for _ in range(rows)]
    base = [rng.choice([0, 1, 15, 16, 17, rng.randint(0, 300)]) for _ in range(rows)]
    for got, want in keep(base, kept, hkv, d, seed, max_kept=max(1, max(map(len, kept))), width_extra=seed):
        assert torch.equal(got, want)


def test_keep_places_that_are_sources():
    """Every node one place on (a place is the next one's source), all of them, none."""
    kept = [list(range(1, 60)), list(range(40)), [], [0], [63], list(range(0, 64, 2))]
    for got, want in keep([13, 16, 5, 0, 31, 7], kept, 8, 128, 3):
        assert torch.equal(got, want)
