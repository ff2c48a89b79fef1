"""Sizes of the language-model operators' tests, chosen so that every kernel that a call can launch is launched by one of them; which
that are is the library's to say (ceca_describe_text_launch)."""
from paper_2306_00256_amd import binding as B

CODE = {"float32": B.TYPE_F32, "bfloat16": B.TYPE_BF16, "float16": B.TYPE_F16}
VEC = {"float32": 4, "bfloat16": 8, "float16": 8}

# (type, n, T, h): columns per lane by the width, positions per wavefront by the number of rows
LOOKUPS = [(d, n, T, h) for d in CODE for h in (40, 100, 300) for n, T in ((3, 50), (4, 4200))]

# (type, n, T, V, h, accumulate, floats between tables, floats between a table's rows)
GRADIENTS = [(d, 2, T, 70, h, acc, 0, 0) for d in CODE for h in (40, 100, 300) for T in (50, 200, 900) for acc in (False, True)]       # not sorted
GRADIENTS += [(d, 3, 1500, 333, h, acc, 0, 0) for d in CODE for h in (40, 100, 300) for acc in (False, True)]
GRADIENTS += [("bfloat16", n, T, 2500, 100, acc, 0, 0) for n, T in ((6, 1000), (2, 1900), (2, 3900), (2, 7900), (2, 9000), (1, 70000)) for acc in (False, True)]
GRADIENTS += [(d, 2, 270_000, 2500, 3, acc, 0, 0) for d in ("float32", "bfloat16") for acc in (False, True)]
# zeros beside the sort and on their own (over 2^24 floats), in one piece and table by table, and row by row
GRADIENTS += [("bfloat16", 3, T, 2001, 36, False, 5, 0) for T in (1500, 9000)]
GRADIENTS += [("float16", 2, T, 70001, 130, False, apart, 0) for T in (1500, 9000) for apart in (0, 3)]
GRADIENTS += [(d, 3, T, 1203, h, acc, apart, 3) for d, h in (("float32", 50), ("bfloat16", 300)) for T in (1500, 9000) for acc in (False, True) for apart in (0, 7)]

# (type, rows, V): packs per row at the upper half of every tile, odd numbers of columns; rows that are split over workgroups and read twice
_PACKS = [(50, 31), (200, 31), (1000, 31), (2000, 70), (2900, 70), (4000, 70), (6000, 70), (8000, 70), (12000, 519), (16000, 519)]
DISTILLATIONS = [(d, rows, packs * VEC[d] + VEC[d] - 1) for d in CODE for packs, rows in _PACKS]
DISTILLATIONS += [(d, rows, V) for d in CODE for rows, V in ((5, 70001), (261, 140001), (200, 140001), (20, 5 * VEC[d] * 256 + 1))]

# (type, rows, V, K)
TOPS = [(d, rows, packs * VEC[d] + VEC[d] - 1, K) for d in CODE for packs, rows, K in ((50, 40, 20), (200, 40, 64), (400, 2100, 30), (900, 2100, 100), (900, 300, 100), (2000, 300, 64), (3900, 300, 64))]
TOPS += [(d, 3, V, K) for d in CODE for V, K in ((100001, 50), (600001, 256))]


def lookup_keys(case):
    d, n, T, h = case
    return {("lookup", d) + B.ceca_describe_text_launch(B.TEXT_EMBED, CODE[d], n, T, 9, h)[:2]}


def gradient_keys(case):
    d, n, T, V, h, acc, apart, pitch = case
    flags = (B.TEXT_ACCUMULATE if acc else 0) | (B.TEXT_APART if apart else 0) | (B.TEXT_PITCH if pitch else 0)
    vec, few, keys, tile, zeros, sums = B.ceca_describe_text_launch(B.TEXT_GRAD, CODE[d], n, T, V, h, flags)
    if few:
        return {("few", d, vec, few, acc)}
    return {("walk", d, vec, acc), ("join", vec, acc), ("sort", keys, tile, sums), ("pitch", bool(pitch), acc)} | ({("zeros", zeros, keys > 0, bool(apart) and zeros < 3)} if not acc else set())


def distillation_keys(case):
    d, rows, V = case
    out = set()
    for flag in (0, B.TEXT_WITH_GRAD):
        threads, packs, loop, parts = B.ceca_describe_text_launch(B.TEXT_DISTILL, CODE[d], 1, rows, V, 8, flag)[:4]
        out.add(("distill", d, threads, packs, loop, parts > 1, bool(flag)))
    return out


def top_keys(case):
    d, rows, V, K = case
    threads, packs, parts, merges = B.ceca_describe_text_launch(B.TEXT_TOP, CODE[d], 1, rows, V, K, 0)[:4]
    return {("top", d, threads, packs), ("merge", d, min(merges, 2))}
