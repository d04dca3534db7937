"""What the linear layer's entry points launch, recorded without a GPU."""
import pytest

import linear_sizes as sizes
from _launches import POINTERS, record


@pytest.fixture(scope="module")
def tmp(tmp_path_factory):
    return tmp_path_factory.mktemp("recorder")


# one call of each kernel that stages more than 64 KiB
LARGE = [dict(op="linear", m=8192, c=4096, k=4096), dict(op="linear", m=198, c=8192, k=4096, bits=4),
         dict(op="linear", m=2003, c=2048, k=8192, adapters=5, rank=128),
         dict(op="grad_input", m=8192, c=4096, k=4096), dict(op="grad_weight", m=777, c=1411, k=1003)]


def test_lds_limits_are_raised_on_every_device(tmp):
    """A kernel with more than 64 KiB of LDS asks for it on each device before its first
    launch there, and not again."""
    there = [{"device": 0}, *LARGE, *LARGE, {"device": 3}, *LARGE, {"device": 0}, *LARGE]
    raised = set()
    for step, (status, events) in zip(there, record(tmp, there)["events"]):
        assert status == 0
        assert ("op" in step) == any(e[0] == "launch" for e in events)
        for kind, device, name, *rest in events:
            if kind == "attribute":
                assert (device, name) not in raised
                raised.add((device, name))
            elif int(rest[2]) > 64 * 1024:
                assert (device, name) in raised, f"{name} on device {device}"
    assert {d for d, _ in raised} == {"0", "3"} and len(raised) >= 8


def test_a_refused_lds_limit_is_asked_for_again(tmp):
    """The call that could not raise it says so and launches nothing; the next one tries anew."""
    for call in (LARGE[0], LARGE[3]):
        (_, _), (status, events), (again, then) = record(tmp, [{"refuse": 1}, call, call])["events"]
        assert status == -4 and not events
        assert again == 0 and [e[0] for e in then] == ["attribute", "launch"]


def test_what_holds_nothing_overlaps_nothing(tmp):
    """A gradient of no rows, or a workspace that the call does not need, may point
    anywhere: within an output or an input too."""
    steps = [dict(op="grad_weight", m=0, c=64, k=32, dy=POINTERS[8] + 64),
             dict(op="linear", m=32, c=256, k=32, workspace=POINTERS[0] + 64),
             dict(op="linear", m=32, c=256, k=32, workspace=POINTERS[8] + 64),
             dict(op="grad_input", m=32, c=64, k=32, workspace=POINTERS[0] + 64)]
    assert [status for status, _ in record(tmp, steps)["events"]] == [0] * len(steps)


OURS = ("quantize_rows", "linear_few", "linear_tile", "adapter_rows", "grad_tile", "grad_sum")


def _forms(step, events):
    """Each kernel that the call launched, in the form that its results take there."""
    names = [e[2] for e in events if e[0] == "launch"]
    split = any("grad_sum" in n for n in names)
    for kind, _, name, *rest in events:
        if kind != "launch":
            continue
        if "grad_tile" in name:
            yield name, "split" if split else "whole"
        elif "adapter_rows" in name:
            yield name, "whole" if rest[0].split()[1] == "1" else "split"
        elif "linear_tile" in name and step["adapters"]:
            yield name, "64 ranks" if step["rank"] <= 64 else "more ranks"
        else:
            yield name, ""


def test_the_parity_tests_sizes_launch_every_kernel(tmp):
    """The sizes that the GPU tests compare reach every kernel that the library holds, in
    every form; a model of times that changes may not take one from them, or leave one
    that no call reaches."""
    steps = [dict(op="rows", m=m, c=c, dtype=t) for m, c in sizes.ROWS for t in range(3)]
    for t in (0, 1):
        steps += [dict(op="linear", m=m, c=c, k=k, bits=bits, adapters=n, rank=rank, dtype=t)
                  for m, c, k, bits, n, rank in sizes.LINEAR]
        steps += [dict(op="grad_input", m=m, c=c, k=k, bits=bits, dtype=t) for m, c, k, bits in sizes.GRAD_INPUT]
        steps += [dict(op="grad_weight", m=m, c=c, k=k, dtype=t) for m, c, k in sizes.GRAD_WEIGHT]
    done = record(tmp, steps)
    reached = set()
    for step, (status, events) in zip(steps, done["events"]):
        assert status == 0, step
        reached.update(_forms(step, events))
    want = set()
    for name in done["kernels"]:
        if any(o in name for o in OURS):
            if "grad_tile" in name or "adapter_rows" in name:
                want.update({(name, "whole"), (name, "split")})
            elif "linear_tile" in name and "true" in name:
                want.update({(name, "64 ranks"), (name, "more ranks")})
            else:
                want.add((name, ""))
    assert len(want) > 200 and not want - reached, "\n".join(map(str, sorted(want - reached)))
