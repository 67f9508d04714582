"""Which of the package's native parts a use of it needs: the planners and the calls
that check their tensors in Python need librag_attn.so alone, the library's build no
torch."""
import importlib
import os
import subprocess
import sys

import pytest

from paper_2412_10543_amd import binding, build

HERE = os.path.dirname(os.path.abspath(__file__))

CHILD = """
import sys
sys.path.insert(0, {root!r})
sys.modules["paper_2412_10543_amd._marshal"] = None        # as if it were not built
import torch
from paper_2412_10543_amd import binding
assert binding.rag_plan_prompts("stuff", [32], [2], 128) == ([0, 288], [0])
assert binding.rag_attn_decode_tree_workspace_size(1, 8, 32, 8, 128, 64, num_splits=2) > 0
x = torch.zeros(4, dtype=torch.int32)
for _ in range(2):
    try:
        binding.rag_kv_pages_update(x.view(2, 2), x, x, x, x, x, x, x, x, x)
    except ImportError as e:
        print("refused:", e)
"""


@pytest.mark.skipif(not os.path.exists(binding.LIBRARY), reason="librag_attn.so not built")
def test_planners_without_the_tensor_checks():
    r = subprocess.run([sys.executable, "-c", CHILD.format(root=os.path.dirname(HERE))],
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = r.stdout.splitlines()
    assert len(lines) == 2 and all("refused:" in x and "__graft_entry__.build()" in x for x in lines)


@pytest.mark.parametrize("torch_there", [False, True])
def test_library_builds_without_torch(monkeypatch, torch_there):
    commands = []
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, **kw: commands.append(" ".join(cmd)))
    monkeypatch.setattr(build.os, "replace", lambda a, b: None)
    importlib.import_module("torch.utils.cpp_extension")
    if not torch_there:
        for name in [n for n in sys.modules if n == "torch" or n.startswith("torch.")]:
            monkeypatch.setitem(sys.modules, name, None)
    assert build.build() == build.LIBRARY
    for src in build.SOURCES:
        assert sum(os.path.join(build.CSRC, src) in x for x in commands) == 1
    assert sum("marshal.cpp" in x for x in commands) == torch_there
