"""The decoder block example with a 4-bit cache, rotary positions and steps planned on the GPU runs."""
from __future__ import annotations

import importlib.util
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(__file__), "..", "examples", "decoder_block.py")


@pytest.mark.parametrize("args", [["--bits", "4"], ["--rotary"], ["--planned"],
                                  ["--bits", "4", "--rotary", "--planned"]])
@pytest.mark.parametrize("sizes", [(3, 70, 4), (5, 300, 70), (1, 1, 1)])
def test_example(args, sizes, monkeypatch, capsys):
    """Ends by itself when an output is wrong."""
    spec = importlib.util.spec_from_file_location("decoder_block", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    batch, prompt, tokens = map(str, sizes)
    monkeypatch.setattr(sys, "argv", [PATH, "--batch", batch, "--prompt", prompt, "--tokens", tokens,
                                      *args])
    example.main()
    assert "against 32-bit floats" in capsys.readouterr().out
