"""CPU models of the 8-bit kernels' LDS places: every chunk that is staged lies where it is read,
inside its buffer, and no two chunks share a place."""
from __future__ import annotations

import pytest


def chunk_turn(row: int) -> int:
    return (row ^ (row >> 3 & 3)) & 7


@pytest.mark.parametrize("rows", [64, 128, 256])
def test_linear_tile_operands(rows):
    """linear_q8_tile: lane order of the loads, permuted in their addresses, against the reads."""
    place = {}
    for piece in range(rows * 8):                            # 16 bytes each, in LDS order
        row = piece // 8
        place[piece * 16] = (row, (piece ^ chunk_turn(row)) & 7)
    assert len(place) == rows * 8
    for first in range(0, rows, 32):
        for s in range(4):
            for lane in range(64):
                r, h = lane % 32, lane // 32
                at = (first + r) * 128 + ((2 * s + h) ^ chunk_turn(r)) * 16
                assert place[at] == (first + r, 2 * s + h)


@pytest.mark.parametrize("DT", [64, 128, 256])
def test_attention_keys_and_values(DT):
    """attention_many: what four wavefronts stage of 64 keys against what a lane reads."""
    def key_turn(k):
        return chunk_turn(k) if DT == 64 else k & 15
    buffer = 64 * DT * 2
    keys, values = {}, {}
    KB, PR, VD = DT // 64, DT // 16, DT // 64
    for half in range(2):
        for lane in range(64):
            k_key, k_ch = lane // PR, lane % PR * 16
            row = (32 * half + k_key) * DT * 2
            bits = 16 * ((k_ch // 8) ^ key_turn(32 * half + k_key))
            for p in range(2 * KB):
                key = p // KB * 16 + p % KB * (64 // PR)
                at, turn = row + key * DT * 2, 16 * key_turn(key)
                for i in range(2):
                    a = at + (bits ^ turn ^ 16 * i)
                    assert a not in keys and a < buffer
                    keys[a] = (32 * half + k_key + key, k_ch // 8 + i)
            v_ch = lane % 16 * 4 * VD
            g = 4 * half + lane // 16
            bits = 16 * (g ^ chunk_turn(v_ch))
            for c in range(4 * VD):
                a = v_ch * 128 + c * 128 + (bits ^ 16 * chunk_turn(c))
                assert a not in values and a < buffer
                values[a] = (v_ch + c, g)
    assert len(keys) == 64 * DT // 8 and len(values) == DT * 8
    KA = 4 if DT == 64 else 8
    for lane in range(64):
        r, h = lane % 32, lane // 32
        for u in range(2):
            for k in range(DT // 16):
                a = r * DT * 2 + ((2 * (k % KA) + h) ^ key_turn(r)) * 16 + 32 * u * DT * 2 \
                    + k // KA * 256
                assert keys[a] == (32 * u + r, 2 * k + h)
        for v in range(4):
            for ct in range(DT // 32):
                a = r * 128 + ((2 * v + h) ^ chunk_turn(r)) * 16 + ct * 32 * 128
                assert values[a] == (32 * ct + r, 2 * v + h)


def test_attention_key_order():
    """A lane's weights of 16 keys and the values' chunk beside them name the same keys."""
    for s in range(4):
        for h in range(2):
            logits = [32 * (s // 2) + 8 * (i // 4) + 4 * h + i % 4
                      for i in range(8 * (s % 2), 8 * (s % 2) + 8)]
            staged = [16 * s + 4 * h + i // 4 * 8 + i % 4 for i in range(8)]
            assert logits == staged
