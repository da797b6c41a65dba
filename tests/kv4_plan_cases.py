"""Calls of the attention over the 4-bit cache that reach every pair of its two kernels, and what the work
plan picks for them: tests/test_kv4_plan_cases.py holds the plan to that on the CPU, tests/test_gpu_kv4_attn_plans.py
runs them.

Row tiles of 16 rows a workgroup, whether tiles' keys are split ("split": all of them, "tail": the last ones), and
which kernel joins the shares ("group": a workgroup a row, "wave": a wave a row)."""
from collections import namedtuple

Call = namedtuple("Call", "tiles split join B Nq H Hkv d n L W")

PARITY = [
    # tiles, split, join, B, Nq, H, Hkv, d, n, chunk_len, window
    Call(1, "none", None, 1, 200, 3, 1, 64, 333, 16, 2),
    Call(1, "none", None, 2, 17, 1, 1, 128, 300, 300, -1),
    Call(1, "split", "group", 2, 1, 4, 2, 128, 5003, 5003, -1),
    Call(1, "split", "group", 1, 3, 5, 1, 64, 2001, 1, -1),
    Call(1, "split", "wave", 16, 5, 32, 4, 128, 5003, 5003, -1),
    Call(1, "split", "wave", 1, 2039, 1, 1, 64, 2431, 1, -1),
    Call(1, "tail", "group", 33, 1, 33, 33, 64, 1500, 1500, -1),
    Call(2, "none", None, 1, 523, 8, 1, 128, 737, 737, 0),
    Call(2, "none", None, 1, 1026, 4, 1, 64, 1026, 1026, -1),
    Call(2, "split", "group", 1, 349, 4, 1, 128, 3049, 58, -1),
    Call(2, "split", "group", 1, 1371, 1, 1, 64, 4336, 37, -1),
    Call(2, "split", "wave", 1, 1017, 2, 1, 128, 2789, 2789, 2),
    Call(2, "split", "wave", 1, 3120, 1, 1, 64, 5003, 5003, -1),
    Call(2, "tail", "group", 1, 2137, 8, 1, 128, 2774, 72, -1),
    Call(2, "tail", "wave", 1, 2384, 8, 1, 128, 3691, 1, -1),
    Call(2, "tail", "wave", 1, 2303, 8, 2, 64, 3412, 1, -1),
    Call(4, "none", None, 1, 1046, 8, 1, 128, 2186, 252, -1),
    Call(4, "none", None, 3, 541, 8, 1, 64, 872, 349, 2),
    Call(4, "split", "group", 1, 1635, 1, 1, 128, 13966, 13966, 1),
    Call(4, "split", "group", 1, 922, 2, 1, 64, 12335, 1, -1),
    Call(4, "split", "wave", 4, 300, 8, 1, 128, 9001, 1, -1),
    Call(4, "split", "wave", 1, 700, 8, 1, 64, 9001, 1, -1),
    Call(4, "tail", "group", 1, 1025, 32, 4, 128, 1025, 1025, 0),
    Call(4, "tail", "wave", 3, 1454, 8, 1, 128, 1454, 1454, -1),
    Call(4, "tail", "wave", 3, 1452, 8, 1, 64, 1452, 1452, 1),
]

# token-causal and chunked calls in which a workgroup's rows differ in what they see
VISIBILITY = [
    Call(2, "none", None, 1, 1900, 9, 9, d, 2500, 1, -1) for d in (64, 128)
] + [
    Call(2, "tail", "group", 1, 1900, 9, 9, d, 6000, 1, -1) for d in (64, 128)
] + [
    Call(4, "none", None, 1, 4700, 8, 8, d, 4700, 1, 500) for d in (64, 128)
] + [
    Call(4, "split", "wave", 1, 1700, 2, 2, d, 9001, 1, -1) for d in (64, 128)
] + [
    Call(4, "tail", "group", 2, 4300, 4, 2, d, 4300, 1, -1) for d in (64, 128)
] + [
    Call(4, "tail", "wave", 1, 4000, 10, 5, d, 4000, 1, -1) for d in (64, 128)
]


def name(c):
    return f"{c.tiles}-{c.split}-{c.join}-B{c.B}q{c.Nq}H{c.H}of{c.Hkv}d{c.d}n{c.n}L{c.L}W{c.W}"
