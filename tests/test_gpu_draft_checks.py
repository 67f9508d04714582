"""Debug mode (RAG_ATTN_CHECK=1) of the drafted-token operators, the page tables
and the prefill with key ranges: arrays that break a documented precondition
are refused before anything is enqueued, in a child process because the library
reads the variable once."""
import json
import os
import subprocess
import sys

import pytest

from paper_2412_10543_amd import binding

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
OK, BAD = binding.RAG_OK, binding.RAG_ERR_INVALID_ARG
FINE = {"tree_valid", "tree_unused_entry_ignored", "keep_valid", "keep_page_before_the_nodes_ignored",
        "pages_valid", "ranges_valid", "ranges_more_rows_than_keys"}


def test_debug_mode_checks_device_arrays():
    r = subprocess.run([sys.executable, "-u", os.path.join(HERE, "draft_checks_child.py")],
                       env=dict(os.environ, RAG_ATTN_CHECK="1"), capture_output=True, text=True,
                       timeout=240)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    got = json.loads([x for x in r.stdout.splitlines() if x.startswith("{")][-1])
    assert len(got) == 26
    assert got == {name: OK if name in FINE else BAD for name in got}
