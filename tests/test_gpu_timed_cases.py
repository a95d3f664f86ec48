"""The timed cases of perf/operators.py as a program calls them: passes of
several prepared states in turn, and their order with the caller's own work."""
import pytest
import torch

from gpu_common import log

pytestmark = pytest.mark.gpu


@pytest.fixture
def cases():
    from perf import operators as M
    M.own = True
    yield M, {c["name"]: c for c in M.listed()}
    M.own = False
    for pair in M._pair.values():
        pair.close()
    M._pair.clear()


def same(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_states_of_two_splits_run_in_turn(cases):
    """Preparing a co-run case of another split leaves the states prepared before as they were."""
    M, by_name = cases
    c = by_name["kv8-mixed-corun"]
    a, b = M.prepare(c, 1), M.prepare(dict(c, cus_decode=64), 2)
    first = []
    for k in range(3):
        got = [M.run(s).clone() for s in (a, b)]
        first = first or got
        assert all(same(x, y) for x, y in zip(got, first)), f"turn {k}"
        log(f"  turn {k}: both splits ran")


@pytest.mark.parametrize("own_stream", [False, True])
def test_corun_pass_is_ordered_with_the_callers_stream(cases, own_stream):
    """A pass sees what the caller's stream wrote before it (late, behind other
    work), and what follows on that stream sees its outputs."""
    M, by_name = cases
    c = by_name["kv8-mixed-corun"]
    x, y = M.prepare(c, 1), M.prepare(c, 2)
    q = [s["x"]["q"].clone() for s in (x, y)]
    torch.cuda.synchronize()
    want = []
    for new in q:
        x["x"]["q"].copy_(new)
        torch.cuda.synchronize()
        out = M.run(x)
        torch.cuda.synchronize()
        want.append(out.clone())
    assert not same(*want)
    busy = torch.randn(8192, 8192, device="cuda", dtype=torch.bfloat16)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream() if own_stream else torch.cuda.current_stream()):
        for k in range(4):
            for _ in range(5):
                busy @ busy                       # the copy below waits for these
            x["x"]["q"].copy_(q[k % 2])
            got = M.run(x).clone()
            torch.cuda.current_stream().synchronize()
            assert same(got, want[k % 2]), f"pass {k}"
            log(f"  pass {k}: in order")
