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


@pytest.mark.parametrize("farewell", [None, "giving up", "always"])
def test_no_meeting_is_waited_for_that_nobody_comes_to(farewell):
    """Either warp may give up at any of its waits, and then says farewell (a flag, and an arrival without waiting): the other
    one's next meeting ends all the same and tells it so.  Without the farewell there is a state in which a warp waits for good;
    with one at the regular end, too, a warp may take its last meeting for the farewell and lose what it has."""
    N = 3

    # a warp: (n, at, alone); at: "wait" (for the tensor cores, may give up), "meet", "in" (arrived), "look" (at the flag),
    # "flag", "arrive", "end"
    def steps(state):
        warps, left, pending, gave_up = state                       # pending: who has arrived at the open generation
        out = []

        def go(w, warp, left=left, pending=pending, other=None, gave_up=gave_up):
            new = [warps[0], warps[1]]
            new[w] = warp
            if other is not None:
                new[1 - w] = other
            out.append((tuple(new), left, pending, gave_up))

        def arrive(w, waits):
            """The next state of both warps when w arrives; the generation closes at the second arrival."""
            n, at, alone = warps[w]
            mine = (n, "in" if waits else "end", alone)
            if not pending:
                go(w, mine, pending=((w, waits),))
                return
            (v, other_waits), = pending
            assert v != w
            if waits:                                               # the flags are read behind the meeting
                mine = (n, "look", alone)
            go(w, mine, pending=(), other=(warps[v][0], "look", warps[v][2]) if other_waits else None)
        for w in (0, 1):
            n, at, alone = warps[w]
            if at == "wait":
                go(w, (n, "meet" if n < N else "flag" if farewell == "always" else "end", alone))
                go(w, (n, "flag" if farewell else "end", alone), gave_up=True)
            elif at == "meet":
                arrive(w, True)
            elif at == "look":
                gone = bool(farewell) and bool(left[1 - w])
                go(w, (n, "end", True) if gone else (n + 1, "wait", False))
            elif at == "flag":
                go(w, (n, "arrive", alone), left=(1, left[1]) if w == 0 else (left[0], 1))
            elif at == "arrive":
                arrive(w, False)
        return out
    states = reachable((((0, "wait", False),) * 2, (0, 0), (), False), steps)
    final = [s for s in states if not steps(s)]
    stuck = [s for s in final if any(warp[1] != "end" for warp in s[0])]
    lost = [s for s in final if not s[3] and any(warp[2] for warp in s[0])]
    assert bool(stuck) == (farewell is None) and bool(lost) == (farewell == "always")
    if farewell:                                                    # at most an arrival that nobody waits for is left over
        assert all(not waits for s in final for _, waits in s[2])
