"""The order in which the chunk kernel's roles pass an item of query rows on, as a model: every interleaving is gone through.

A barrier is the number of its completed phases, and a wait sees the last one's parity alone, as mbarrier.try_wait.parity does.  K, V and the
weights' columns are taken to be there always, so the model allows more interleavings than the kernel.  Roles: `pages` announces items and
their Q (pages warp and the warps that split Q), `mma` issues scores and products, `soft` 0 and 1 are the two streams' softmax warps."""
import itertools

import pytest

SLOTS = 2


def stuck(items, soft_waits_for):
    """Whether some interleaving ends with a role waiting for good.  items: tiles of the two streams, by item."""
    names = ["Q", "QE"] + [f"{n}{j}" for n in ("SF", "PF") for j in (0, 1)] + [f"{n}{s}{x}" for n, x in (("IF", ""), ("IE", "a"), ("IE", "b")) for s in range(SLOTS)]
    at = {n: i for i, n in enumerate(names)}

    def pages():
        nq = 0
        for k, (n0, n1) in enumerate(items):
            s = k % SLOTS
            if k >= SLOTS:                                     # both streams have let go of the slot's last item
                yield "wait", f"IE{s}a", (k // SLOTS - 1) & 1
                yield "wait", f"IE{s}b", (k // SLOTS - 1) & 1
            yield "done", f"IF{s}"
            if n0 or n1:
                if nq:
                    yield "wait", "QE", (nq - 1) & 1
                yield "done", "Q"
                nq += 1

    def mma():
        nq, tiles = 0, [0, 0]
        for n in items:
            if not any(n):
                continue
            yield "wait", "Q", nq & 1
            nq += 1
            for t in range(max(n)):
                on = [j for j in (0, 1) if t < n[j]]
                for j in on:
                    yield "done", f"SF{j}"
                if t == max(n) - 1:
                    yield "done", "QE"
                for j in on:
                    yield "wait", f"PF{j}", tiles[j] & 1
                    tiles[j] += 1

    def soft(j):
        done = nq = 0
        for k, n in enumerate(items):
            yield "wait", f"IF{k % SLOTS}", (k // SLOTS) & 1
            if soft_waits_for == "Q" and any(n):
                yield "wait", "Q", nq & 1
                nq += 1
            if soft_waits_for == "SF" and n[j]:
                yield "wait", f"SF{j}", done & 1
            for _ in range(n[j]):
                yield "wait", f"SF{j}", done & 1
                yield "done", f"PF{j}"
                done += 1
            yield "done", f"IE{k % SLOTS}{'ab'[j]}"

    roles = [list(r) for r in (pages(), mma(), soft(0), soft(1))]
    seen, todo = set(), [((0,) * 4, (0,) * len(names))]
    while todo:
        state = todo.pop()
        if state in seen:
            continue
        seen.add(state)
        pcs, phases = state
        moved = False
        for i, role in enumerate(roles):
            if pcs[i] == len(role):
                continue
            step = role[pcs[i]]
            b = at[step[1]]
            if step[0] == "wait" and phases[b] % 2 == step[2]:        # the phase of that parity is not complete
                continue
            moved = True
            now = phases if step[0] == "wait" else phases[:b] + (phases[b] + 1,) + phases[b + 1:]
            todo.append((pcs[:i] + (pcs[i] + 1,) + pcs[i + 1:], now))
        if not moved and any(pc < len(r) for pc, r in zip(pcs, roles)):
            return True
    return False


SHAPES = [s for s in itertools.product([(0, 0), (1, 0), (0, 1), (1, 1), (2, 1)], repeat=4)]


def test_streams_that_wait_for_their_first_scores_never_get_stuck():
    assert not any(stuck(list(s), "SF") for s in SHAPES)


@pytest.mark.parametrize("items", [[(1, 0), (1, 0), (1, 1)], [(0, 1), (1, 0), (0, 1)]])
def test_streams_that_wait_for_q_itself_can_be_lapped(items):
    """Why the kernel does not: a stream without a tile may come to the wait when two further phases are over or one too many is."""
    assert stuck(items, "Q")
