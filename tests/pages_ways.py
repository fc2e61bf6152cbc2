"""Sizes that reach every launch of the attention over pages, and how each is
divided: (type, head_dim, page, heads, key heads, entries, rows, prefix, tail,
way, rows a workgroup of the prefix, of the tails, several ranges of the
prefix, of the tails)."""

ENTRIES, PARTS, PAIRS = 0, 1, 2

WAYS = [
    # fp32: entries by themselves in 32 rows, then both parts
    ("f32", 64, 16, 8, 1, 45, 48, 17, 5, ENTRIES, 0, 32, False, False),
    ("f32", 64, 32, 256, 32, 2, 31, 3153, 2, ENTRIES, 0, 32, False, True),
    ("f32", 128, 16, 8, 2, 21, 122, 19, 3, ENTRIES, 0, 32, False, False),
    ("f32", 64, 16, 1, 1, 3, 1, 211, 284, PARTS, 16, 16, False, False),
    ("f32", 64, 32, 2, 1, 3, 3, 77, 551, PARTS, 16, 16, False, True),
    ("f32", 64, 16, 4, 1, 3, 4, 1036, 593, PARTS, 16, 16, True, True),
    ("f32", 128, 16, 2, 1, 3, 3, 155, 159, PARTS, 16, 16, False, False),
    ("f32", 128, 32, 1, 1, 3, 1, 99, 574, PARTS, 16, 16, False, True),
    ("f32", 64, 16, 32, 32, 54, 11, 140, 2, PARTS, 32, 16, False, False),
    ("f32", 128, 16, 256, 32, 63, 1, 70, 1, PARTS, 32, 16, False, False),
    ("f32", 64, 32, 8, 8, 68, 33, 324, 26, PARTS, 32, 32, False, False),
    ("f32", 64, 16, 24, 3, 18, 39, 3304, 39, PARTS, 32, 32, True, False),
    ("f32", 128, 64, 8, 8, 53, 42, 390, 6, PARTS, 32, 32, False, False),
    # bf16, heads of 64
    ("bf16", 64, 16, 1, 1, 3, 1, 293, 241, PARTS, 16, 16, False, False),
    ("bf16", 64, 32, 1, 1, 3, 2, 140, 507, PARTS, 16, 16, False, True),
    ("bf16", 64, 64, 1, 1, 4, 1, 800, 544, PARTS, 16, 16, True, True),
    ("bf16", 64, 32, 1, 1, 3, 6, 110, 503, PARTS, 32, 16, False, True),
    ("bf16", 64, 16, 2, 1, 3, 3, 2843, 488, PARTS, 32, 16, True, False),
    ("bf16", 64, 16, 1, 1, 1, 17, 743, 538, PARTS, 32, 32, True, True),
    ("bf16", 64, 16, 1, 1, 3, 15, 236, 339, PARTS, 128, 16, False, False),
    ("bf16", 64, 64, 8, 1, 3, 2, 530, 539, PARTS, 128, 16, True, True),
    ("bf16", 64, 16, 1, 1, 3, 31, 783, 583, PARTS, 128, 32, True, True),
    ("bf16", 64, 16, 4, 2, 65, 51, 193, 260, PARTS, 128, 128, False, False),
    ("bf16", 64, 16, 1, 1, 3, 50, 524, 513, PARTS, 128, 128, True, True),
    ("bf16", 64, 128, 4, 4, 5, 40, 230, 60, PAIRS, 0, 0, False, False),
    # bf16, heads of 128
    ("bf16", 128, 16, 1, 1, 3, 1, 180, 348, PARTS, 16, 16, False, False),
    ("bf16", 128, 16, 1, 1, 3, 1, 604, 37, PARTS, 16, 16, True, False),
    ("bf16", 128, 16, 2, 1, 3, 4, 95, 442, PARTS, 32, 16, False, False),
    ("bf16", 128, 64, 1, 1, 26, 1, 3600, 39, PARTS, 32, 16, True, False),
    ("bf16", 128, 16, 2, 2, 10, 2, 4107, 832, PARTS, 32, 16, True, True),
    ("bf16", 128, 32, 1, 1, 1, 18, 100, 530, PARTS, 32, 32, False, True),
    ("bf16", 128, 32, 4, 1, 3, 3, 110, 487, PARTS, 128, 16, False, False),
    ("bf16", 128, 16, 1, 1, 14, 4, 7439, 660, PARTS, 128, 16, True, True),
    ("bf16", 128, 64, 4, 1, 64, 1, 8000, 700, PARTS, 128, 16, True, True),
    ("bf16", 128, 16, 1, 1, 3, 24, 110, 451, PARTS, 128, 32, False, False),
    ("bf16", 128, 16, 8, 1, 3, 3, 81, 538, PARTS, 128, 32, False, True),
    ("bf16", 128, 16, 1, 1, 3, 17, 508, 520, PARTS, 128, 32, True, True),
    ("bf16", 128, 32, 1, 1, 3, 40, 250, 440, PARTS, 128, 128, False, True),
    ("bf16", 128, 64, 2, 1, 3, 19, 560, 139, PARTS, 128, 128, True, False),
    ("bf16", 128, 16, 8, 1, 5, 4, 203, 40, PAIRS, 0, 0, False, False),
]


def division(plan):
    """A kv_attention_plan as the last five values of a case."""
    return plan.way, plan.prefix_rows, plan.tail_rows, plan.prefix_ranges > 1, plan.tail_ranges > 1
