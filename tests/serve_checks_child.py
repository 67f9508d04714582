"""Child process of test_gpu_serve_checks.py: run with RAG_ATTN_CHECK=1 in the environment (the
library reads it once per process), call each entry point of the new tokens' way into the caches, of
the 4-bit cache and of the verification with valid device arrays and with arrays that break
one documented precondition, and print {case: status} as one JSON line.

In this mode the library copies the device index arrays to the host and checks them before
anything is enqueued, so the invalid cases never reach a kernel.
"""
import json
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import torch  # noqa: E402

from paper_2412_10543_amd import binding  # noqa: E402
from paper_2412_10543_amd.workloads import normal_bf16  # noqa: E402

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


HQ, HKV, D, BLOCKS = 8, 2, 64, 9
bf16 = [torch.zeros((BLOCKS, HKV, 16, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
four = [torch.zeros((BLOCKS, HKV, 9 * D), dtype=torch.uint8, device="cuda") for _ in range(2)]
cos_sin = torch.ones((50, 32), device="cuda")


def rope(kv4, slots=(3, -1, 143, 16), pos=(0, 1 << 30, 49, 5)):
    q, k = normal_bf16((4, HQ, D), 1, "cuda"), normal_bf16((4, HKV, D), 2, "cuda")
    call = binding.rag_qkv_rope_write_kv4 if kv4 else binding.rag_qkv_rope_write
    return lambda: call(q, k, k, torch.empty_like(q), i32(pos), cos_sin, i32(slots), *(four if kv4 else bf16))


for kv4, name in ((False, "rope"), (True, "rope4")):
    run(name + "_valid", rope(kv4))
    run(name + "_slot_past_pool", rope(kv4, slots=(3, -1, 144, 16)))
    run(name + "_slot_twice", rope(kv4, slots=(3, -1, 3, 16)))
    run(name + "_position_past_table", rope(kv4, pos=(0, 1, 50, 5)))
    run(name + "_position_negative", rope(kv4, pos=(-1, 1, 49, 5)))

TABLE = ((0, 1, -7), (2, 3, 4), (5, -7, -7))


def read(cu=(0, 20, 68, 70), t=TABLE):
    k = torch.empty((72, HKV, D), dtype=torch.bfloat16, device="cuda")
    return lambda: binding.rag_kv4_read(*four, i32(t), i32(cu), k, torch.empty_like(k))


run("read_valid", read())
run("read_not_monotone", read(cu=(0, 20, 10, 12)))
run("read_not_from_0", read(cu=(1, 20, 68, 70)))
run("read_past_rows", read(cu=(0, 30, 70, 75)))
run("read_keys_past_table", read(cu=(0, 0, 49, 50)))
run("read_page_past_pool", read(t=((0, 9, -7), (2, 3, 4), (5, -7, -7))))
run("read_page_negative", read(cu=(0, 33, 68, 70)))


def attend(kv=(20, 48, 2), cu=(0, 5, 5, 7), t=TABLE, rows=5):
    q = normal_bf16((3 if cu is None else 7, HQ, D), 3, "cuda")
    ws = torch.zeros(binding.rag_attn_decode_kv4_workspace_size(3, rows, HQ, HKV, D, 3),
                     dtype=torch.uint8, device="cuda")
    return lambda: binding.rag_attn_decode_paged_kv4(
        q, *four, torch.empty_like(q), i32(t), i32(kv), 0.1, None if cu is None else i32(cu), rows, ws)


run("attend_valid", attend())
run("attend_one_row_valid", attend(cu=None, kv=(20, 0, 1)))
run("attend_sequence_without_rows_not_looked_at", attend(kv=(20, 4000, 2)))
run("attend_more_rows_than_keys", attend(kv=(4, 48, 2)))
run("attend_keys_past_table", attend(kv=(49, 48, 2)))
run("attend_negative_keys", attend(cu=None, kv=(20, -1, 1)))
run("attend_cu_decreases", attend(cu=(0, 5, 4, 7)))
run("attend_over_max_rows", attend(rows=4))
run("attend_page_past_pool", attend(t=((0, 1, -7), (2, 3, 4), (9, -7, -7))))
run("attend_page_negative", attend(t=((0, -1, -7), (2, 3, 4), (5, -7, -7))))


def verify(cu=(0, 3, 3, 8), tokens=(-9, 1, 99, -9, 0, 5, 6, 7), parents=(0, 0, 0, 9, 0, 1, 1, 3)):
    logits, u = torch.zeros((10, 100), device="cuda"), torch.zeros(10, device="cuda")
    pad = lambda x: i32(list(x) + [-5, -5])  # noqa: E731
    ws = torch.zeros(binding.rag_draft_verify_workspace_size(10, 3, 100), dtype=torch.uint8, device="cuda")
    return lambda: binding.rag_draft_verify(
        logits, pad(tokens), i32(cu), torch.ones(3, device="cuda"), u, i32([[0] * 4] * 3), i32([0] * 3),
        i32([0] * 3), parents=None if parents is None else pad(parents), workspace=ws)


run("verify_valid", verify())
run("verify_chain_valid", verify(parents=None))
run("verify_cu_decreases", verify(cu=(0, 5, 4, 8)))
run("verify_past_rows", verify(cu=(0, 3, 3, 11)))
run("verify_token_past_vocabulary", verify(tokens=(-9, 1, 100, -9, 0, 5, 6, 7)))
run("verify_token_negative", verify(tokens=(-9, 1, 99, -9, -1, 5, 6, 7)))
run("verify_parent_itself", verify(parents=(0, 0, 0, 9, 0, 2, 1, 3)))
run("verify_parent_negative", verify(parents=(0, -1, 0, 9, 0, 1, 1, 3)))

print(json.dumps(out), flush=True)
