"""The losses' kernel timers cover all that a call launches."""
import pytest

from gpu_util import say, torch_dev

pytestmark = pytest.mark.gpu


def timed(call, n=5):
    """(time of n calls in one piece, {group: mean of its records}) in ms."""
    from paper_1802_08021_amd import sparcml as S
    torch, _ = torch_dev()
    for _ in range(2):
        call.run()
    torch.cuda.synchronize()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    S.timing_enable(True)
    try:
        a.record()
        for _ in range(n):
            call.run()
        b.record()
        torch.cuda.synchronize()
        groups = {g: S.timing_read(g) for g in (S.TIMER_LOSS_ROWS, S.TIMER_LOSS_GRAD)}
    finally:
        S.timing_enable(False)
    return a.elapsed_time(b) / n, {g: t for g, t in groups.items() if t is not None}


def calls(T, V, kind="float32"):
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    x = torch.randn(T, V, device=dev, dtype=getattr(torch, kind))
    label = torch.zeros(T, dtype=torch.int32, device=dev)
    f = torch.rand(T, device=dev)
    return {"policy": S.PolicyLossCall(x, label, -f, f, f), "policy forward": S.PolicyLossCall(x, label, -f, f, f, dlogits=None),
            "pairs": S.PreferenceLossCall(x, label, [0, T // 2, T]),
            "pairs forward": S.PreferenceLossCall(x, label, [0, T // 2, T], dlogits=None),
            "logprob": S.TokenLogprobCall(x, label)}


def test_groups_add_up_to_the_call():
    """Many short rows, where the sums over them take their share: between
    records lie a few microseconds of a call of hundreds."""
    for name, call in calls(1 << 20, 3).items():
        whole, groups = timed(call)
        say(f"[timers] {name}: {whole:.3f} ms, groups {groups}")
        assert whole > 0.1
        assert sum(groups.values()) > 0.9 * whole, name


def test_joined_slices_have_a_record():
    from paper_1802_08021_amd import sparcml as S
    for name, call in calls(3, 200000).items():
        _, groups = timed(call)
        assert set(groups) == {S.TIMER_LOSS_ROWS, S.TIMER_LOSS_GRAD}, name
