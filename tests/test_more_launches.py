"""What the entry points around the linear layer launch, recorded without a GPU."""
import pytest

import around_sizes as sizes
from _more_launches import record

OURS = ("norm_to_rows", "norm_backward", "norm_gain_sum", "groups_rows", "groups_tiles", "groups_back", "experts_rows",
        "experts_tiles", "experts_back_rows", "experts_back_weights")   # (expert_groups_rows and _tiles by their ends)
FIELDS = ("op", "m", "c", "k", "bits", "group", "scales", "experts", "dtype")


@pytest.fixture(scope="module")
def tmp(tmp_path_factory):
    return tmp_path_factory.mktemp("recorder")


def _forms(events):
    names = [e[2] for e in events if e[0] == "launch"]
    split = any("grad_sum" in n for n in names)
    for name in names:
        yield name, "split" if split and "groups_back" in name else ""


def test_the_parity_tests_sizes_launch_every_kernel(tmp):
    """No kernel that the GPU tests' sizes do not reach, and none that no call reaches."""
    steps = [dict(zip(FIELDS, s)) for s in sizes.PRODUCTS]
    steps += [dict(op=op, m=4, c=c, dtype=t, residual=r) for op in ("norm", "norm_grad") for c in sizes.NORMS
              for t in range(3) for r in (False, True)]
    done = record(tmp, steps)
    reached = set()
    for step, (status, events) in zip(steps, done["events"]):
        assert status == 0, step
        reached.update(_forms(events))
    want = set()
    for name in done["kernels"]:
        if any(o in name for o in OURS):
            want.add((name, ""))
            if "groups_back" in name:
                want.add((name, "split"))
    assert len(want) > 250 and not want - reached, "\n".join(map(str, sorted(want - reached)))


def test_launches_stay_within_the_limits(tmp):
    """Fewer than 2^32 threads, and a grid's other axes within 65535, at the extremes of
    rows, outputs and experts."""
    steps = []
    for m in (1, 17, 4096, 65536, 1 << 20, 1 << 22):
        for k in (1, 16, 512, 1 << 13):
            for experts in (0, 1, 64, 4096):
                for group in (0, 32, 128):
                    if k * max(experts, 1) > 1 << 22 or not (group or experts):
                        continue
                    for op in ("forward", "grad_input", "grad_weight") if experts else ("forward", "grad_input"):
                        steps.append(dict(op=op, m=m, c=256, k=k, bits=4, group=0 if op == "grad_weight" else group, experts=experts))
    launched = 0
    for step, (status, events) in zip(steps, record(tmp, steps)["events"]):
        assert status in (0, -2), step   # (a result too large is refused)
        for kind, _, name, *rest in events:
            if kind == "launch":
                x, y, z = map(int, rest[0].split())
                assert x * y * z * int(rest[1]) < 1 << 32 and y <= 65535 and z <= 65535, (step, name, rest)
                assert int(rest[2]) <= 160 * 1024, (step, name, rest)
                launched += 1
    assert launched > 300


def test_lds_limits_are_raised_on_every_device(tmp):
    large = [dict(op="forward", m=4096, c=4096, k=4096, group=128), dict(op="forward", m=16, c=4096, k=4096, group=128),
             dict(op="forward", m=4096, c=1024, k=1024, experts=8, bits=8), dict(op="grad_input", m=4096, c=4096, k=4096, group=32),
             dict(op="grad_weight", m=4096, c=1024, k=1024, experts=8)]
    there = [{"device": 0}, *large, *large, {"device": 3}, *large, {"device": 0}, *large]
    raised = set()
    for step, (status, events) in zip(there, record(tmp, there)["events"]):
        assert status == 0 and ("op" in step) == any(e[0] == "launch" for e in events)
        for kind, device, name, *rest in events:
            if kind == "attribute":
                assert (device, name) not in raised
                raised.add((device, name))
            elif int(rest[2]) > 64 * 1024:
                assert (device, name) in raised, f"{name} on device {device}"
    assert {d for d, _ in raised} == {"0", "3"} and len(raised) >= 8
