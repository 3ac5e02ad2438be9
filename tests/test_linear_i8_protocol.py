"""A model of the barriers that the int8 GEMM's loads, converter teams and UMMA thread meet at (csrc/linear_i8.cu), over
every interleaving of a small run.

Loads of blocks 0, 1, ... go into `rst` stages in order and land in any order.  Team k converts blocks k, k + teams, ...:
it waits for the block's stage of codes and for its fp16 stage (of `fst`), by the parity of the phase that it expects,
as the hardware tests it (true as soon as the phase in progress has the other parity), then writes.  The UMMA
thread takes the blocks in order; a stage is free again when the UMMAs that read it are done.

Checked: a team reads only codes of its block, writes only stages whose last block has been read, and every run ends.
The rule of the kernel (rst a multiple of the teams, fst at least their number) is what makes both hold.
"""
import pytest


class Violation(AssertionError):
    pass


def passes(phase_in_progress, n):
    """A wait for phase n to complete, by its parity."""
    return (phase_in_progress & 1) != (n & 1)


def explore(blocks, teams, rst, fst):
    # state: loads issued, loads in flight, landed count per codes stage, steps of each team (two a block: its codes' wait
    # passed, converted), releases per codes stage, blocks converted and not yet read, UMMAs done
    start = (0, frozenset(), (0,) * rst, (0,) * teams, (0,) * rst, frozenset(), 0)
    seen, stack, ends = set(), [start], 0
    while stack:
        s = stack.pop()
        if s in seen:
            continue
        seen.add(s)
        issued, flight, landed, steps, released, ready, done = s
        nxt = []
        if issued < blocks and released[issued % rst] >= issued // rst:
            nxt.append((issued + 1, flight | {issued}, landed, steps, released, ready, done))
        for b in flight:
            at = list(landed)
            at[b % rst] += 1
            nxt.append((issued, flight - {b}, tuple(at), steps, released, ready, done))
        for k in range(teams):
            g = k + steps[k] // 2 * teams
            if g >= blocks:
                continue
            if steps[k] % 2 == 0:
                if passes(landed[g % rst], g // rst):
                    nxt.append((issued, flight, landed, steps[:k] + (steps[k] + 1,) + steps[k + 1:], released, ready, done))
                continue
            freed = max(0, -(-(done - g % fst) // fst)) if done > g % fst else 0      # UMMAs of this stage that are done
            if not passes(freed, g // fst - 1):
                continue
            if landed[g % rst] != g // rst + 1:
                raise Violation(f"block {g} is converted with {landed[g % rst]} loads landed in its stage")
            if g >= fst and done <= g - fst:
                raise Violation(f"block {g} overwrites an fp16 stage that is still read")
            st, rel = list(steps), list(released)
            st[k] += 1
            rel[g % rst] += 1
            nxt.append((issued, flight, landed, tuple(st), tuple(rel), ready | {g}, done))
        if done in ready:
            nxt.append((issued, flight, landed, steps, released, ready - {done}, done + 1))
        if done == blocks:
            ends += 1
        elif not nxt:
            raise Violation(f"deadlock at {s}")
        stack.extend(nxt)
    assert ends
    return len(seen)


@pytest.mark.parametrize("teams,rst,fst", [(3, 6, 4), (3, 3, 4), (2, 4, 3), (3, 6, 3), (1, 2, 2)])
def test_the_kernels_rule_holds(teams, rst, fst):
    assert explore(10, teams, rst, fst) > 10


@pytest.mark.parametrize("teams,rst,fst", [(4, 3, 4), (2, 3, 4), (3, 4, 4)])
def test_stages_that_no_team_knows_are_found(teams, rst, fst):
    with pytest.raises(Violation):
        explore(10, teams, rst, fst)
