"""What the norm launches at the extremes of its sizes, and which products are refused as too
large, recorded without a GPU."""
import pytest

from _more_launches import record

ROWS = (1, 2, 3, 5, 255, 4097, 1 << 20, (1 << 22) - 1, 1 << 22)
WIDTHS = (1, 7, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 8192, 8193, 131071)


@pytest.fixture(scope="module")
def tmp(tmp_path_factory):
    return tmp_path_factory.mktemp("recorder")


def _launches(events):
    """Name, workgroups, threads and LDS bytes of each launch; grids have one axis."""
    for kind, _, name, *rest in events:
        if kind == "launch":
            x, y, z = map(int, rest[0].split())
            assert y == z == 1 and int(rest[2]) <= 160 * 1024
            yield name, x, int(rest[1])


@pytest.mark.parametrize("residual", [False, True])
def test_norm_takes_every_row(tmp, residual):
    """As many workgroups as rows, or a quarter of it where a wave takes one, whatever the
    size; fewer than 2^31 threads a launch."""
    steps = [dict(op="norm", m=m, c=c, dtype=t, residual=residual) for m in ROWS for c in WIDTHS for t in (0, 1)]
    for step, (status, events) in zip(steps, record(tmp, steps)["events"]):
        assert status == 0, step
        rows = 0
        for name, blocks, threads in _launches(events):
            assert "norm_to_rows" in name and threads == 256 and blocks * threads <= 1 << 31, step
            rows += blocks * (4 if step["c"] <= 2048 else 1)
        assert step["m"] <= rows < step["m"] + 4, step


@pytest.mark.parametrize("residual", [False, True])
def test_norms_gradient_keeps_its_partial_sums_few(tmp, residual):
    """One launch over the rows, of 512 workgroups at most and none without rows of its own,
    and one that covers the columns."""
    steps = [dict(op="norm_grad", m=m, c=c, dtype=t, residual=residual) for m in ROWS for c in WIDTHS for t in (0, 1)]
    for step, (status, events) in zip(steps, record(tmp, steps)["events"]):
        assert status == 0, step
        (rows, blocks, threads), (sums, columns, _) = _launches(events)
        waves = next(w for w, most in ((1, 512), (2, 1024), (4, 2048), (8, 4096), (16, 1 << 30)) if step["c"] <= most)
        assert "norm_backward" in rows and "norm_gain_sum" in sums
        assert threads == (1024 if waves == 16 else 512)
        assert 1 <= blocks <= min(512, -(-step["m"] * waves * 64 // threads)), step
        assert (columns - 1) * 32 < step["c"] <= columns * 32


def _too_large(op, m, c, k, experts):
    """More than 2^22 tiles of 64 x 64, one more counted for each expert that may have rows."""
    if op == "grad_weight":
        return experts * -(-k // 64) * -(-c // 64) > 1 << 22
    cols = k if op == "forward" else c
    return -(-(m + 64 * min(m, experts)) // 64) * -(-cols // 64) > 1 << 22


def test_products_are_refused_for_their_tiles_alone(tmp):
    steps, want = [], []
    for op in ("forward", "grad_input", "grad_weight"):
        for m in (1, 65, 70000, 1 << 20, 1 << 22):
            for c, k in ((256, 1), (256, 4096), (256, 4160), (4160, 64), (65536, 256), (8192, 8192), (131064, 1024)):
                for experts in (0, 1, 3, 512, 4096):
                    if k * max(experts, 1) > 1 << 22 or (op == "grad_weight" and not experts):
                        continue
                    for bits, group in ((8, 0), (4, 0), (4, 64)):
                        if (op == "grad_weight" and bits == 4) or not (group or experts):
                            continue
                        steps.append(dict(op=op, m=m, c=c, k=k, bits=bits, group=group, experts=experts))
                        want.append(_too_large(op, m, c, k, experts))
    assert any(want) and not all(want)
    for step, refused, (status, events) in zip(steps, want, record(tmp, steps)["events"]):
        assert status == (-2 if refused else 0), step
        grids = [list(map(int, e[3].split())) for e in events if e[0] == "launch"]
        assert bool(grids) == (not refused) and all(y <= 65535 and z == 1 for _, y, z in grids), step
