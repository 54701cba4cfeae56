"""The launch plans of calls over an 8-bit cache, written plainly: the chunk
length and chunks of a traversal, the workspace bytes of the longest chunks, and
how full attention cuts its tiles (shared by the tests that name a plan or a
cut, so that their cases cannot leave it unseen)."""
from __future__ import annotations

TILE, WAVES = 64, 4


def chunks(g, groups, t_cap, block, *, test=True, compact=False):
    """(blocks in a chunk, chunks of the longest traversal) over codes."""
    rec, tpb = (g * 128 + 2 * g) * 4, block // TILE
    half_tiles = 3 * 4096 if g >= 8 or test else 3 * 32 * 288
    buffers = 0 if g >= 8 and tpb == 1 else half_tiles + 16
    few, heavy = test and groups <= 8 and t_cap >= 768, test and g == 16 and t_cap >= 128
    c_max = min(16, ((156 if few or heavy else 78) * 1024 - buffers) // (2 * rec))
    while c_max > 1 and (c_max + 2) // 3 * tpb > 16:
        c_max -= 1
    c = min(c_max, 12 if not test else 15 if few else 9)
    if c >= 3:
        c -= c % 3
    while c > 3 and ((not heavy and groups * -(-t_cap // c) < 64) or (not compact and 5 * c > t_cap)):
        c -= 3
    lead, blocks = (4, 3) if test and c > 3 else (0, c)
    n = -(-t_cap // blocks) if t_cap <= lead * blocks else lead + -(-(t_cap - lead * blocks) // c)
    return c, n


def least_bytes(g, groups, t_cap, block):
    """Workspace bytes of the plan with the longest chunks, with the test."""
    n = chunks(g, groups, t_cap, block, compact=True)[1]
    up = lambda x: (x + 255) // 256 * 256  # noqa: E731
    record = (g * 128 + 2 * g + 63) // 64 * 64
    return up(8) + up(8 * 32 * 8) + up(8 * groups) + up(8 * groups * n) + up(groups * n * 2 * record * 4)


def cut(tiles, heads, g, t_cap, block, cus):
    """How full attention cuts units (sequences, or with a list per head groups)
    of `tiles` tiles each, every one `heads` times: "each" (a wavefront to every
    group), "wave line", "line", "parts" or "whole" (a workgroup to every group).
    Two workgroups share a CU."""
    groups, total, longest = len(tiles) * heads, sum(tiles) * heads, max(tiles)
    cap = groups * t_cap * (block // TILE)
    most = min(2 * cus, groups * chunks(g, groups, t_cap, block, test=False)[1], -(-cap // WAVES) + groups)
    if groups > most:
        waves = most * WAVES
        return "each" if -(-groups // waves) * (2 + longest) <= (total + 3 * groups) // waves + 3 else "wave line"
    if 2 * groups <= most:
        return "line" if total > 16 * most else "parts"
    return "whole" if longest <= (total + 8 * groups) // most + 6 else "line"
