"""The attention's workspace: no call of at most batch x max_rows rows needs more than 2^18 (head_dim + 2) bytes, though fewer rows may need more than
many (they get more key chunks)."""
import os
import random

import pytest

import paper_2602_24174_amd as T

pytestmark = pytest.mark.skipif(not os.path.exists(T.LIB_PATH), reason="libtasc.so is not built")


def need(batch, kv_heads, share, hd, max_rows, max_kv, rows=None):
    return T.tasc_kv4_attention_workspace_bytes(batch, batch * max_rows if rows is None else rows, kv_heads * share, kv_heads, hd, max_rows, max_kv)


def test_bound():
    rng = random.Random(5)
    size = lambda most: max(1, int(most ** rng.random()))
    largest = 0
    for _ in range(20000):
        kv_heads, share, hd = size(64), size(40), rng.choice((32, 64, 128))
        batch, max_rows, max_kv = size(65535 // kv_heads), size(20000), size(1 << 30)
        n = need(batch, kv_heads, share, hd, max_rows, max_kv)
        assert n <= (1 << 18) * (hd + 2), (batch, kv_heads, share, hd, max_rows, max_kv, n)
        largest = max(largest, n / (hd + 2))
    assert largest > 1 << 15                                  # (the bound is not far from what is met)


def test_fewer_rows_may_need_more():
    assert need(32, 8, 4, 128, 1, 4096) == 0 < need(16, 8, 4, 128, 1, 4096)
    assert need(4, 2, 6, 128, 2048, 2500) == 0 < need(4, 2, 6, 128, 512, 2500)
