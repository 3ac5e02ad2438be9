"""A model of how a pair of CTAs of the int8 GEMM (csrc/linear_i8.cu) hands converted blocks to the thread that issues the
pair's UMMAs, over every interleaving of a small run: who orders what for whom, and that every run ends.

Both CTAs' converter teams write their half of a block and arrive at rank 0's barrier, whose UMMA thread waits there.  In
the PTX memory model a release of CTA scope synchronises with threads of its own CTA alone, wherever the barrier stands;
between CTAs both sides need cluster scope.
"""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_00712_gb300", "csrc")


class Violation(AssertionError):
    pass


def synchronises(release, acquire, same_cta):
    return same_cta or (release == "cluster" and acquire == "cluster")


def explore(blocks, teams, fst, release, acquire="cluster"):
    """release: the scope at which rank 1's converters release their half of a block; acquire: of rank 0's wait."""
    # blocks that each team of each rank has converted; UMMAs issued, and done (committed to both CTAs)
    start = (((0,) * teams,) * 2, 0, 0)
    seen, stack, ends = set(), [start], 0
    while stack:
        s = stack.pop()
        if s in seen:
            continue
        seen.add(s)
        steps, issued, done = s
        nxt = []
        for r in (0, 1):
            for k in range(teams):
                g = k + steps[r][k] * teams
                if g < blocks and done >= g - fst + 1:      # the stage's last UMMAs have been committed
                    mine = steps[r][:k] + (steps[r][k] + 1,) + steps[r][k + 1:]
                    nxt.append(((mine, steps[1]) if r == 0 else (steps[0], mine), issued, done))
        if issued < blocks and all(steps[r][issued % teams] > issued // teams for r in (0, 1)):
            for r, scope in ((0, "cta"), (1, release)):
                if not synchronises(scope, acquire, r == 0):
                    raise Violation(f"UMMAs of block {issued} are not ordered behind rank {r}'s half")
            nxt.append((steps, issued + 1, done))
        if done < issued:
            nxt.append((steps, issued, done + 1))
        if done == blocks:
            ends += 1
        elif not nxt:
            raise Violation(f"deadlock at {s}")
        stack.extend(nxt)
    assert ends
    return len(seen)


@pytest.mark.parametrize("blocks,teams,fst", [(9, 3, 4), (8, 3, 3), (6, 2, 4), (5, 1, 2)])
def test_both_halves_are_ordered_before_the_umma(blocks, teams, fst):
    assert explore(blocks, teams, fst, "cluster") > blocks


@pytest.mark.parametrize("release,acquire", [("cta", "cluster"), ("cluster", "cta"), ("cta", "cta")])
def test_both_sides_need_cluster_scope(release, acquire):
    with pytest.raises(Violation, match="rank 1"):
        explore(9, 3, 4, release, acquire)


def test_the_sources_release_to_other_ctas_at_cluster_scope():
    # an arrival at another CTA's barrier releases at cluster scope itself, or stands behind a fence that does
    found = 0
    for f in sorted(os.listdir(CSRC)):
        for statement in re.findall(r"asm volatile\((.*?)\);", open(os.path.join(CSRC, f)).read(), re.S):
            for op in re.findall(r"mbarrier\.arrive[\w.:]*", statement):
                if "shared::cluster" in op:
                    found += 1
                    before = statement[:statement.index(op)]
                    assert ".release.cluster." in op or (".relaxed.cluster." in op and "fence.release." in before and
                                                         ".cluster;" in before), f"{f}: {op}"
    assert found


def test_the_pairs_waits_acquire_at_cluster_scope():
    ptx = open(os.path.join(CSRC, "ptx.cuh")).read()
    body = ptx[ptx.index("bool mbar_try_wait_cluster("):]
    assert "mbarrier.try_wait.parity.acquire.cluster." in body[:body.index("\n}")]
    gemm = open(os.path.join(CSRC, "linear_i8.cu")).read()
    assert "warp_wait<PAIR>(f16f0 " in gemm and "warp_wait<PAIR>(acce0 " in gemm
