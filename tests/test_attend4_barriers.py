"""The order in which the warps of attention over the 4-bit cache meet at their barriers, read from the kernel's
source and tried in every interleaving, without a GPU: with waits for products that end, and after waits that gave
up, when nothing but the barriers themselves holds a warp back."""
import os
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_26004_gb300", "csrc",
                      "kernel_attend4_tensor.cuh")
WARPS = 4


def the_kernels_order():
    """(barrier of a step's keys, the step's events): events are "keys" (warps 1 to 3 arrive), "scores" (warp 0 waits
    there), "all" (the CTA's barrier) and "weights" (warp 1 waits, the others arrive; with their barrier)."""
    text = open(SOURCE).read()
    ways = [[int(n) for n in re.findall(r"barrier_%s<(\d+)>" % how, re.search(r"auto %s = .*?};" % name, text, re.S).group(0))]
            for name, how in (("keys_turned", "arrive"), ("start_scores", "sync"))]
    assert ways[0] == ways[1] and len(ways[0]) <= 2  # of odd steps and of even ones, or of all
    step = re.search(r"for \(int t = t0; t < t1; \+\+t\) \{(.*?)// the rows' sums over the threads", text, re.S).group(1)
    events = []
    for m in re.finditer(r"keys_turned\(|start_scores\(|__syncthreads_or\(raise|barrier_sync<(.*?)>\(\);", step):
        word = m.group(0)
        events.append(("keys", None) if word.startswith("keys") else ("scores", None) if word.startswith("start")
                      else ("all", None) if word.startswith("__") else ("weights", int(m.group(1))))
    assert sorted(e for e, _ in events) == ["all", "keys", "scores", "weights"]
    return (lambda step: ways[0][0 if step & 1 else -1]), events


def programs(steps, gave_up, events, keys_at):
    """Each warp's actions of an item and the first of the next one."""
    all_ = [[] for _ in range(WARPS)]

    def keys(step):
        for w in range(1, WARPS):
            all_[w].append(("arrive", keys_at(step)))

    def scores(step):
        all_[0] += [("sync", keys_at(step)), ("start", step)]

    for item in range(2):
        first = item * steps
        keys(first)
        scores(first)
        for t in range(first, first + steps):
            more = t + 1 < first + steps
            for w in range(WARPS):
                if not gave_up:
                    all_[w].append(("wait", t))  # (for the scores of this step)
            for event, how in events:
                if event == "keys" and more:
                    keys(t + 1)
                elif event == "scores" and more:
                    scores(t + 1)
                elif event == "all":
                    for w in range(WARPS):
                        all_[w].append(("sync", 0))
                elif event == "weights":
                    for w in range(WARPS):
                        all_[w].append(("sync" if w == 1 else "arrive", how))
        for w in range(WARPS):
            all_[w].append(("sync", 0))
    return all_


def stuck(all_):
    """The first state found in which warps are left that none can move, or None; and no barrier may end with
    arrivals that nobody waited for."""
    start = ((0,) * WARPS, (), -1, (False,) * WARPS)  # places, arrivals at barriers, the last step started, asleep
    seen, todo = {start}, [start]
    while todo:
        state = todo.pop()
        places, counts, begun, asleep = state
        moves = []
        for w in range(WARPS):
            if asleep[w] or places[w] == len(all_[w]):
                continue
            what, n = all_[w][places[w]]
            if what == "wait" and begun < n:
                continue
            at, c, sleep, last = list(places), dict(counts), list(asleep), begun
            at[w] += 1
            if what == "start":
                last = n
            elif what in ("arrive", "sync"):
                c[n] = c.get(n, 0) + 1
                sleep[w] = what == "sync"
                if c[n] == WARPS:
                    del c[n]
                    for v in range(WARPS):
                        if sleep[v] and all_[v][at[v] - 1] == ("sync", n):
                            sleep[v] = False
            moves.append((tuple(at), tuple(sorted(c.items())), last, tuple(sleep)))
        if not moves and (any(p < len(a) for p, a in zip(places, all_)) or any(asleep) or counts):
            return state
        for m in moves:
            if m not in seen:
                seen.add(m)
                todo.append(m)
    return None


@pytest.mark.parametrize("gave_up", [False, True])
@pytest.mark.parametrize("steps", [1, 2, 5])
def test_no_order_of_the_warps_leaves_one_waiting(steps, gave_up):
    keys_at, events = the_kernels_order()
    assert stuck(programs(steps, gave_up, events, keys_at)) is None


@pytest.mark.parametrize("order", [("keys", "scores", "all", "weights"), ("keys", "all", "scores", "weights")])
def test_one_barrier_for_all_steps_would_not_do(order):
    """After a wait that gave up a warp arrives a second time in the place of one that has not come, in either order;
    the search finds it.  With waits that end, and with a barrier for odd steps, there is none."""
    events = [(e, 3 if e == "weights" else None) for e in order]
    assert stuck(programs(5, True, events, lambda step: 1)) is not None
    assert stuck(programs(5, False, events, lambda step: 1)) is None
    assert stuck(programs(5, True, events, lambda step: 1 + (step & 1))) is None
