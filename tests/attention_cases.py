"""Batches of the attention that are cut into runs, joined and planned, and the kernels that are to serve them: run on the GPU in test_gpu_attention_cut.py, their kernels
looked at on the CPU in test_attention_routes.py."""


def many_short_and_some_long(seqs, rows, long, seed):
    """`rows` rows in each of `seqs` sequences of 5 to 40 tokens, and some much longer ones."""
    new = [rows] * seqs
    lengths = [5 + (seed * 7 + 11 * i) % 36 for i in range(seqs)]
    for at, n in long.items():
        lengths[at] = n
    new[3] = 0
    return new, lengths


ROWS_BEFORE, ROWS_BEHIND = 1, 2
CUT = [dict(new=[70], lengths=[6000], heads=2, kv_heads=1, dim=64, page=64, causal=False, window=2500),
       dict(new=[70], lengths=[6000], heads=2, kv_heads=1, dim=64, page=50, causal=False),
       dict(new=[300, 65], lengths=[3000, 5000], heads=2, kv_heads=2, dim=128, page=16, name="f16", causal=False),
       dict(new=[40], lengths=[9000], heads=4, kv_heads=1, dim=256, page=64, v_fmt="fp4"),
       dict(new=[40], lengths=[4000], heads=4, kv_heads=1, dim=200, page=24, name="f16", causal=False)]
PLANNED = [dict(zip(("new", "lengths"), many_short_and_some_long(300, 3, {7: 7000, 299: 2500, 120: 900}, 1)), heads=16, kv_heads=1, dim=64, page=64),
           dict(zip(("new", "lengths"), many_short_and_some_long(257, 3, {0: 5000, 256: 3000}, 2)), heads=32, kv_heads=2, dim=128, page=16, k_fmt="fp4", window=2000),
           dict(zip(("new", "lengths"), many_short_and_some_long(260, 5, {100: 4000, 101: 4000}, 3)), heads=8, kv_heads=1, dim=128, page=40, name="f16", causal=False),
           dict(zip(("new", "lengths"), many_short_and_some_long(258, 3, {200: 3000}, 4)), heads=14, kv_heads=1, dim=256, page=64, v_fmt="fp4")]


def tokens(case):
    return ROWS_BEFORE + sum(case["new"]) + ROWS_BEHIND
