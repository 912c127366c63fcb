"""A step without sequences: nothing to do, and no error."""
from __future__ import annotations

import ctypes

from paper_2112_13896_amd import _lib
from paper_2112_13896_amd._lib import CS_BF16, CS_ERR_ARG, CS_OK

P = 0x100000            # an aligned address that is never dereferenced


def test_no_sequences():
    def call(tokens=0, batch=0, width=0):
        cache = ctypes.byref(_lib.Q8Cache(P, P, P, P, 4, 2, 16, 64))
        return _lib.lib().cs_paged_attention(cache, CS_BF16, P, 256, 64, tokens, 4, batch, P, width, P,
                                             P, 0, 0.1, 0, P, P, 0, None)
    assert call() == call(batch=3) == call(width=3) == call(batch=2, width=3) == CS_OK
    for kw in (dict(tokens=1), dict(tokens=1, batch=1), dict(tokens=1, width=1), dict(batch=-1),
               dict(width=-1)):
        assert call(**kw) == CS_ERR_ARG, kw
