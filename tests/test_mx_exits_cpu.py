"""How CTAs of the few-token kernel leave when a wait has given up.  The kernel's steps on that way are read from its source, and every order in which
the roles can take them is tried: no GPU runs it."""
import re
from pathlib import Path

SOURCE = (Path(__file__).resolve().parent.parent / "paper_2601_22716_b200" / "csrc" / "lords_mx_stream.cu").read_text()
CODE = re.sub(r"//[^\n]*", "", SOURCE)
KERNEL = CODE[CODE.index("lords_mxfp4_stream_kernel(const __grid_constant__"):CODE.index("struct StreamVariant")]
ADD_UP = CODE[CODE.index("bool add_up("):CODE.index("lords_mxfp4_stream_kernel(const __grid_constant__")]


def runs(programs, enabled, allowed):
    """Every order of the roles' steps.  `programs`: role -> steps; a step may run when enabled(role, step, done) holds, `done` the steps taken so far as
    {(role, step)}.  Returns the orders that break `allowed(role, step, done)`, and those that end with a role stuck."""
    broken, stuck, seen = [], [], set()

    def go(at, done, order):
        if (at, done) in seen:
            return
        seen.add((at, done))
        moved = False
        for k, (role, steps) in enumerate(programs.items()):
            if at[k] == len(steps):
                continue
            step = steps[at[k]]
            if not enabled(role, step, done):
                continue
            moved = True
            if not allowed(role, step, done):
                broken.append(order + [(role, step)])
                continue
            go(at[:k] + (at[k] + 1,) + at[k + 1:], done | {(role, step)}, order + [(role, step)])
        if not moved and any(at[k] < len(s) for k, s in enumerate(programs.values())):
            stuck.append(order)

    go((0,) * len(programs), frozenset(), [])
    return broken, stuck


def test_a_receiver_stays_while_others_may_send():
    """A CTA whose wait for the others' sums gave up: stores into its shared memory come before it is gone."""
    end = KERNEL[KERNEL.rindex("record_give_up"):]
    stays = re.search(r"if \(alone\)\s*\{[^}]*barrier\.cluster\.arrive[^}]*barrier\.cluster\.wait[^}]*\}", end) is not None
    # `alone` is set where that wait gave up, and nowhere else
    assert not stays or re.findall(r"alone = ([^;]*);", KERNEL) == ["false", "!ok"]
    for senders in (1, 3):
        for gave_up_too in range(senders + 1):         # some of the others wait in vain as well: they stay likewise
            programs = {"receiver": ["give up"] + (["arrive", "wait"] if stays else []) + ["exit"]}
            for s in range(senders):
                programs[f"sender {s}"] = ["send"] + (["arrive", "wait"] if stays and s < gave_up_too else []) + ["exit"]

            def enabled(role, step, done):
                # a cluster barrier's wait: every thread that has not exited has arrived
                return step != "wait" or all((r, "arrive") in done or (r, "exit") in done for r in programs)

            def allowed(role, step, done):
                return step != "send" or ("receiver", "exit") not in done

            broken, stuck = runs(programs, enabled, allowed)
            assert not stuck and not broken, (senders, gave_up_too, broken[:1], stuck[:1])
