"""Attention calls by the kernel that they are meant to reach: (batch, kv_heads, heads, head_dim, max_rows, max_kv) and the order they get, (waves that share
pairs, key chunks).  tests/test_kv4_order.py holds the rule to this list, so a rule that changes cannot leave a kernel untested unseen."""

ROWS = {                                                     # waves with rows of their own (1), for every head_dim and share
    "hd32": ((41, 2, 12, 32, 150, 260), (1, 1)),
    "hd32_alone": ((64, 4, 4, 32, 250, 260), (1, 1)),
    "hd64": ((41, 2, 14, 64, 129, 200), (1, 1)),
    "hd128": ((41, 2, 12, 128, 130, 200), (1, 1)),
    "least_pairs": ((86, 8, 16, 64, 33, 70), (1, 1)),         # 66 pairs: three of a workgroup's four waves have some
}
FOUR = {                                                     # up to 16 pairs of more heads than eight waves each would fill the chip with
    "hd32": ((130, 2, 6, 32, 1, 200), (4, 1)),
    "hd64": ((130, 2, 8, 64, 4, 300), (4, 1)),
    "hd128": ((130, 2, 8, 128, 3, 130), (4, 1)),
    "chunks": ((130, 2, 4, 128, 1, 2100), (4, 2)),
    "very_many": ((300, 8, 32, 64, 1, 70), (4, 1)),           # as many as would fill the chip with rows of their own, if they had any
}
TWO = {
    "many_heads": ((260, 8, 32, 128, 5, 100), (2, 1)),        # 20 pairs
    "two_tiles": ((130, 8, 16, 64, 32, 100), (2, 1)),         # 64 pairs
    "split": ((2, 3, 9, 64, 9, 768), (2, 3)),
}
