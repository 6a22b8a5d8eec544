"""The 8-bit second moment over thousands of steps.  A root r is rounded
without bias, so r^2 lies above v by the rounding's variance: at most one code
step times the way that v moves the root,

    unit |r' - r| <= (r' / 8) (1 - beta2) |g^2 - v| / (r' + r) <= (1 - beta2) |g^2 - v| / 8,

so that with V its mean once settled and G the mean of g^2, V <= G + (G + V) /
8, V <= 9/7 G; and never below G but for the noise of the mean."""
import numpy as np
import pytest

from gpu_util import say, to_np, torch_dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("beta2,steps", [(0.99, 1500), (0.999, 9000)])
@pytest.mark.parametrize("share", [1.0, 1 / 32])
def test_second_moment_settles(beta2, steps, share):
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    n = 1 << 16
    gen = torch.Generator(device=dev).manual_seed(1)
    p, grad = [torch.zeros(n, device=dev)], [torch.zeros(n, device=dev)]
    calls = []
    for bits in (8, 32):
        m, v, *scale = S.adamw_state(p, bits)
        calls.append((S.AdamwCall(p, grad, m, v, **dict(zip(("m_scale", "v_scale"), scale))), v, scale))
    last = max(1, int(1 / (1 - beta2)))  # means over the last of the steps
    sums = np.zeros(2)
    for step in range(1, steps + 1):
        torch.randn(n, device=dev, generator=gen, out=grad[0])
        if share < 1:
            grad[0].mul_(torch.rand(n, device=dev, generator=gen) < share)
        for call, _, _ in calls:
            call.run(lr=0.0, step=step, beta2=beta2, seed=7)
        if step > steps - last:
            eight, scale, wide = calls[0][1][0], calls[0][2][1], calls[1][1][0]
            r = eight.float().view(-1, 256) * scale[0][:, None]
            sums += [float(r.double().square().sum()), float(wide.double().sum())]
        if step % 500 == 0:
            torch.cuda.synchronize()
    ratio = sums[0] / sums[1]
    say(f"[moments] beta2 {beta2}, share {share}: 8 bits / 32 bits = {ratio:.4f}")
    # Noise of the ratio: an element's moment varies by sqrt((1 - beta2) k) of
    # its mean, k the gradient's kurtosis (3 / share), in both forms; 6 sigma.
    noise = 6 * np.sqrt(2 * (1 - beta2) * 3 / share / n)
    assert 1 - noise <= ratio <= 9 / 7 + noise
