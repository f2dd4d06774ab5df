"""Shapes of windowed attention in which requests are taken in the order of their rows, with the plan that each must get
(test_window_plans.py pins it on the host, test_gpu_window_by_rows.py runs it)."""

PLAN = ("waves", "block_rows", "row_blocks", "splits", "split_tiles", "by_rows", "few")

# R, block, Hq, Hkv, d, dtype, max_kv_len, window, sinks, kv_split -> plan
BY_ROWS = [
    ((17, 16, 32, 8, 128, "bf16", 2100, 2000, 4, 0), (4, 128, 1, 3, 11, 1, 0)),         # 51 (request, split)s
    ((63, 16, 32, 8, 128, "bf16", 2100, 2000, 4, 1 << 20), (4, 128, 1, 1, 33, 1, 0)),   # whole lists, 63
    ((64, 16, 32, 8, 64, "bf16", 2100, 2000, 4, 0), (4, 128, 1, 1, 33, 1, 0)),
    ((64, 16, 32, 8, 128, "bf16", 2100, 2000, 4, 256), (4, 128, 1, 9, 4, 1, 0)),
    ((63, 8, 32, 8, 128, "bf16", 4200, 4000, 4, 0), (4, 128, 1, 1, 65, 1, 0)),          # up to 32 rows, not shared by four waves
    ((64, 8, 32, 8, 64, "bf16", 2100, 2000, 4, 0), (4, 128, 1, 1, 33, 1, 1)),           # shared by four waves
    ((17, 16, 64, 4, 128, "bf16", 8200, 8000, 4, 0), (8, 256, 1, 3, 43, 1, 0)),         # eight waves
    ((63, 16, 64, 4, 128, "bf16", 8200, 8000, 4, 0), (8, 256, 1, 2, 64, 1, 0)),
    ((64, 16, 64, 4, 64, "bf16", 8200, 8000, 4, 1 << 20), (8, 256, 1, 1, 128, 1, 0)),
    ((21, 16, 64, 2, 64, "bf16", 8200, 8000, 4, 0), (8, 256, 2, 6, 22, 1, 0)),          # two row blocks
    ((17, 4, 32, 8, 128, "f32", 8200, 8000, 4, 0), (4, 16, 1, 5, 26, 1, 0)),
    ((63, 4, 32, 8, 64, "f32", 2100, 2000, 4, 1 << 20), (4, 16, 1, 1, 33, 1, 0)),
    ((64, 8, 28, 7, 100, "f32", 2100, 2000, 4, 1 << 20), (4, 32, 1, 1, 33, 1, 0)),      # blocks of 32 rows
]

# (shape, plan) of neighbours that are not: more requests than lanes, one row each, too little to do
IN_ORDER = [
    ((65, 16, 32, 8, 128, "bf16", 2100, 2000, 4, 0), (4, 128, 1, 1, 33, 0, 0)),
    ((64, 1, 32, 8, 128, "bf16", 4200, 4000, 4, 0), (4, 128, 1, 1, 65, 0, 0)),
    ((17, 16, 32, 8, 128, "bf16", 1100, 1000, 4, 0), (4, 128, 1, 3, 6, 0, 0)),
    ((6, 16, 8, 2, 64, "bf16", 720, 100, 4, 0), (4, 128, 1, 1, 4, 0, 0)),
    ((8, 5, 32, 8, 128, "f32", 16384, 512, 1, 0), (4, 16, 2, 6, 2, 0, 0)),
]


def in_order(shape, plan):
    """The same lists in a batch of 65 requests, which are taken in their own order: (shape, plan)"""
    R, block, Hq, Hkv, d, dtype, max_kv, window, sinks, _ = shape
    return (65, block, Hq, Hkv, d, dtype, max_kv, window, sinks, 64 * plan[4]), plan[:5] + (0,) + plan[6:]


def line(shape):
    R, block, Hq, Hkv, d, dtype, max_kv, window, sinks, split = shape
    return f"{R} {block} {Hq} {Hkv} {d} {int(dtype == 'f32')} {max_kv} {window} {sinks} {split}\n"
