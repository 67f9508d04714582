"""Debug mode (RAG_ATTN_CHECK=1) of the new tokens' way into the caches, of the 4-bit cache and of
the verification: arrays that break a documented precondition are refused before anything is
enqueued, in a child process because the library reads the variable once."""
import json
import os
import subprocess
import sys

import pytest

from paper_2412_10543_amd import binding

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
OK, BAD = binding.RAG_OK, binding.RAG_ERR_INVALID_ARG
FINE = {"attend_sequence_without_rows_not_looked_at"}


def test_debug_mode_checks_device_arrays():
    r = subprocess.run([sys.executable, "-u", os.path.join(HERE, "serve_checks_child.py")],
                       env=dict(os.environ, RAG_ATTN_CHECK="1"), capture_output=True, text=True,
                       timeout=240)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    got = json.loads([x for x in r.stdout.splitlines() if x.startswith("{")][-1])
    assert len(got) == 35
    assert got == {name: OK if name in FINE or name.endswith("_valid") else BAD for name in got}
