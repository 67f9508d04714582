"""Child process of test_gpu_draft_checks.py: run with RAG_ATTN_CHECK=1 in the
environment (the library reads it once per process), call each entry point of
the drafted-token operators, the page tables and the prefill with key ranges
with valid device arrays and with arrays that break one documented
precondition, and print {case: status} as one JSON line.

In this mode the library copies the device index arrays to the host and
checks them before anything is enqueued, so the invalid cases never reach a
kernel.
"""
import json
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import torch  # noqa: E402

from paper_2412_10543_amd import binding  # noqa: E402
from paper_2412_10543_amd.workloads import normal_bf16, paged_pool  # noqa: E402

assert os.environ.get("RAG_ATTN_CHECK") == "1"
i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
out = {}


def run(name, fn):
    try:
        fn()
        torch.cuda.synchronize()
        out[name] = binding.RAG_OK
    except binding.RagError as e:
        out[name] = e.status


hq, hkv, d = 8, 2, 64
lens = [40, 300, 17]
pool = paged_pool(lens, hkv, d, 5, device="cuda")
table, blocks = pool.block_tables, pool.num_blocks
q = normal_bf16((20, hq, d), 1, "cuda")
mask = torch.full((20, 1), -1, dtype=torch.int64, device="cuda")


def entry(row, col, value):
    t = table.clone()
    t[row, col] = value
    return t


def tree(kv=lens, cu=(0, 5, 15, 20), t=table, max_nodes=10):
    return lambda: binding.rag_attn_decode_paged_tree(
        q, pool.k_cache, pool.v_cache, torch.empty_like(q), mask, t, i32(kv), i32(cu), max_nodes,
        d ** -0.5, num_splits=1)


run("tree_valid", tree())
run("tree_more_nodes_than_keys", tree(kv=[40, 300, 4]))
run("tree_keys_past_table", tree(kv=[40, table.shape[1] * 16 + 1, 17]))
run("tree_cu_decreases", tree(cu=[0, 5, 3, 12]))
run("tree_over_max_nodes", tree(max_nodes=9))
run("tree_page_too_large", tree(t=entry(1, 18, blocks)))
run("tree_page_negative", tree(t=entry(0, 0, -1)))
run("tree_unused_entry_ignored", tree(t=entry(2, 2, -1)))


def keep(base=(35, 290, 12), kept=((0, 2), (1, 9), (0, -1)), num=(2, 2, 1), t=table):
    return lambda: binding.rag_kv_cache_keep(pool.k_cache, pool.v_cache, t, i32(base), i32(kept), i32(num))


run("keep_valid", keep())
run("keep_more_than_max", keep(num=[2, 3, 1]))
run("keep_not_increasing", keep(kept=[(0, 2), (9, 9), (0, -1)]))
run("keep_past_table", keep(base=[35, table.shape[1] * 16 - 5, 12]))
run("keep_negative_base", keep(base=[-1, 290, 12]))
run("keep_page_too_large", keep(t=entry(1, 18, blocks)))
run("keep_page_before_the_nodes_ignored", keep(t=entry(1, 3, blocks)))


def pages(t=((0, 1, -7), (2, -7, -7)), stack=(5, 3, 4, -9, -9, -9), free=3, old=(20, 16), new=(33, 0)):
    return lambda: binding.rag_kv_pages_update(
        i32(t), i32(stack), i32([free]), i32(old), i32(new), i32([0]), i32([0, 0]), i32([0] * 3),
        i32([0] * 40), i32([0]))


run("pages_valid", pages())
run("pages_free_page_held", pages(stack=(5, 3, 1, -9, -9, -9)))
run("pages_held_twice", pages(t=((0, 0, -7), (2, -7, -7))))
run("pages_no_page_of_the_pool", pages(t=((0, 6, -7), (2, -7, -7))))
run("pages_more_free_than_pool", pages(free=7))
run("pages_old_past_table", pages(old=(49, 16)))
run("pages_negative_new", pages(new=(33, -1)))


def ranges(cq=(0, 40, 100), ck=(0, 40, 100), mq=60, mk=60):
    x = normal_bf16((100, hq, d), 1, "cuda")
    y = normal_bf16((100, hkv, d), 2, "cuda")
    return lambda: binding.rag_attn_prefill_varlen_ranges(
        x, y, y, torch.empty_like(x), None, i32(cq), i32(ck), i32([(0, 0)] * 100), mq, mk, d ** -0.5)


run("ranges_valid", ranges())
run("ranges_not_monotone", ranges(cq=(0, 50, 40)))
run("ranges_over_max_seqlen", ranges(mk=50))
run("ranges_more_rows_than_keys", ranges(ck=(0, 30, 90)))

print(json.dumps(out), flush=True)
