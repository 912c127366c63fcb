"""Workspace sizes of arguments past the stated limits: 0, as for other invalid ones."""
from __future__ import annotations

import subprocess
import sys

import pytest

CODE = """
import ctypes
from paper_2112_13896_amd import _lib
P = 0x100000
def size(page=1024, heads=2, d=64, qt=_lib.CS_BF16, tokens=1, q_heads=4, batch=1, width=4, max_len=0):
    cache = ctypes.byref(_lib.Q8Cache(P, P, P, P, 4, heads, page, d))
    return _lib.lib().cs_paged_attention_workspace_bytes(cache, qt, tokens, q_heads, batch, width,
                                                         max_len)
print(size({args}))
"""


@pytest.mark.parametrize("args,zero", [
    ("width=1 << 30", True), ("width=(1 << 20) + 1", True), ("width=1 << 20", False),
    ("page=16, width=(1 << 31) - 1", True), ("width=1 << 28", True),
    ("tokens=1 << 30", True), ("heads=65536, q_heads=65536", True), ("width=4096", False)])
def test_attention(args, zero):
    """In a process of its own: a size that is computed for such an axis may divide by zero."""
    p = subprocess.run([sys.executable, "-c", CODE.replace("{args}", args)], capture_output=True,
                       text=True, timeout=120)
    assert p.returncode == 0, (p.returncode, p.stderr)
    assert (int(p.stdout) == 0) == zero
