"""The protocol by which two warps of an attention kernel exchange a number per row, walked through in every order of their steps.

Program of a warp, for each exchange n: (wait for the tensor cores) -- write n to its place -- meet -- read the other's place.
The waits order nothing between the two warps here: the scores of the next blocks may be there already."""
import pytest


def reachable(start, steps):
    """Every state that can be reached; a state without steps is final."""
    seen, todo = {start}, [start]
    while todo:
        state = todo.pop()
        for nxt in steps(state):
            if nxt not in seen:
                seen.add(nxt)
                todo.append(nxt)
    return seen


@pytest.mark.parametrize("places,right", [(1, False), (2, True)])
def test_a_number_is_read_before_its_place_is_written_again(places, right):
    """One place for each warp is not enough; two in turn are."""
    N, wrong = 5, []

    def steps(state):
        pcs, slots = state                                          # pc of a warp: 3 n + (0 write, 1 meet, 2 read)
        out = []
        for w in (0, 1):
            n, at = divmod(pcs[w], 3)
            if n == N:
                continue
            new_pcs, new_slots = list(pcs), [list(s) for s in slots]
            new_pcs[w] += 1
            if at == 0:
                new_slots[w][n % places] = n
            elif at == 1:
                if pcs[1 - w] < 3 * n + 1:                          # the other one has not arrived
                    continue
            elif slots[1 - w][n % places] != n:
                wrong.append(state)
            out.append((tuple(new_pcs), tuple(tuple(s) for s in new_slots)))
        return out
    empty = tuple((-1,) * places for _ in range(2))
    states = reachable(((0, 0), empty), steps)
    assert any(s[0] == (3 * N, 3 * N) for s in states) and bool(wrong) != right
