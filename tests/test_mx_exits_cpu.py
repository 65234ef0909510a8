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


def test_tensor_memory_goes_back_when_nothing_writes_it():
    """The epilogue's wait for the accumulator gave up while the issuer was still at work: its columns are freed, and read, only when that has ended."""
    threads = {int(k) for k in re.findall(r"bar\.(?:sync|red\.or\.pred q,) 1, (\d+)", CODE)}
    assert len(threads) == 1
    # the roles that meet at the named barrier before the columns are freed: four epilogue warps, the one that frees, and the issuer if it takes part
    issuer = KERNEL[KERNEL.index("warp == 1"):KERNEL.index("warp >= kConvWarp0", KERNEL.index("warp == 1"))]
    tail = issuer[issuer.rindex("umma_commit(bar_acc"):]
    issuer_meets = "sums_read(" in tail
    assert threads == {32 * (5 + issuer_meets)}
    free = KERNEL[KERNEL.rindex("sums_read("):KERNEL.rindex("tmem_dealloc(")]
    waits = re.search(r"mbar_wait_warp\(bar_acc\b", free) is not None
    # what the epilogue does once its wait has given up: does it still load the accumulator?
    reads = [c for c in re.findall(r"([^;{}]*)[;{]\s*tmem_ld_32x16\(", ADD_UP) if "!failed" not in c]
    programs = {
        "epilogue": ["give up"] + (["read"] if reads else []) + ["meet"],
        "issuer": ["issue", "issue again", "commit"] + (["meet"] if issuer_meets else []),
        "tensor core": ["finish"],                    # the MMAs and copies that the issuer has committed
        "owner": ["meet", "met"] + (["see them finish"] if waits else []) + ["free"],
    }
    meeting = [r for r in programs if "meet" in programs[r]]

    def enabled(role, step, done):
        if step == "met":
            return all((r, "meet") in done for r in meeting)
        if step == "finish":
            return ("issuer", "commit") in done
        return step != "see them finish" or ("tensor core", "finish") in done

    def allowed(role, step, done):
        if step in ("issue", "issue again"):
            return ("owner", "free") not in done
        if step in ("read", "free"):                  # while MMAs may write the columns
            return ("tensor core", "finish") in done
        return True

    broken, stuck = runs(programs, enabled, allowed)
    assert not stuck and not broken, (broken[:1], stuck[:1])
