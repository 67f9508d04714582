"""Debug mode (RAG_ATTN_CHECK=1) on a host without memory for the copies of a call's
device arrays: the call returns a status, as no C++ exception leaves the library.  In
child processes, which have little address space left and allocate the copies before
they read anything from the device."""
import os
import subprocess
import sys

import pytest

from paper_2412_10543_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import resource, sys
sys.path.insert(0, {root!r})
from paper_2412_10543_amd import binding
L, F, S = binding.lib(), 0x100000, 1 << 28
used = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (used + (256 << 20),) * 2)
status = {call}
print(status, binding.rag_last_error())
"""

CALLS = {
    "prefill": "L.rag_attn_prefill_varlen(F, F, F, F, None, F, F, S, 1, 1, 1, 1, 64, 1.0, 1, None)",
    "decode": "L.rag_attn_decode_paged(F, F, F, F, F, F, None, S, S, 1, 1, 100, 1, 1, 64, 16, 1.0, 1, None, 0, "
              "None)",
    "write": "L.rag_kv_cache_write(F, F, F, F, F, S, 1, 64, 16, 100, None)",
    "ranges": "L.rag_attn_prefill_varlen_ranges(F, F, F, F, None, F, F, F, S, 1, 1, 1, 1, 64, 1.0, None)",
    "tree": "L.rag_attn_decode_paged_tree(F, F, F, F, F, F, F, F, S, 1, 1, 1, 100, 1, 1, 64, 16, 1.0, 1, None, 0, "
            "None)",
    "keep": "L.rag_kv_cache_keep(F, F, F, F, F, F, S, 1, 1, 100, 1, 64, 16, None)",
}


@pytest.mark.skipif(not os.path.exists(binding.LIBRARY), reason="librag_attn.so not built")
@pytest.mark.parametrize("name", CALLS)
def test_no_exception_leaves_the_library(name):
    r = subprocess.run([sys.executable, "-c", CHILD.format(root=ROOT, call=CALLS[name])],
                       env=dict(os.environ, RAG_ATTN_CHECK="1"), capture_output=True, text=True,
                       timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    status, message = r.stdout.strip().split(" ", 1)
    assert int(status) == binding.RAG_ERR_HIP and "debug copy" in message
