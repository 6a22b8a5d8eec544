"""The fine-tuning example end to end (losses, selection with error feedback,
sparse sum over the ranks, norm, AdamW): it learns its task, with 8-bit
moments as with 32-bit ones, and the update that it makes is that of the
summed gradient."""
import numpy as np
import pytest

import train_ref as R
from gpu_util import say, to_np, torch_dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 32])
def test_example_learns(bits):
    from paper_1802_08021_amd.finetune import Trainer
    torch_dev()
    t = Trainer(vocab=64, hidden=32, tokens=128, state_bits=bits, kb=32)
    first = t.preference_step().tolist()
    for _ in range(29):
        last = t.preference_step().tolist()
    say(f"[finetune] {bits} bits: preference loss {first[0]:.3f} -> {last[0]:.3f}")
    assert abs(first[0] - np.log(2)) < 1e-3  # the policy is its own reference
    assert last[0] < 0.5 * first[0] and last[1] > 0.9
    rewards = [float(t.policy_step()[1]) for _ in range(30)]
    say(f"[finetune] {bits} bits: right answers {rewards[0]:.3f} -> {rewards[-1]:.3f}")
    assert np.mean(rewards[-5:]) > np.mean(rewards[:5]) + 0.1


def test_step_is_the_update_of_the_summed_selection():
    from paper_1802_08021_amd.finetune import Trainer
    torch, _ = torch_dev()
    t = Trainer(vocab=32, hidden=16, ranks=3, tokens=64, state_bits=32, kb=8)
    for _ in range(3):
        before = to_np(t.flat).copy()
        m, v = (np.concatenate([to_np(x).reshape(-1) for x in s]) for s in (t.update._keep[2], t.update._keep[3]))
        t.policy_step()
        total = np.zeros(before.size)
        for r in range(3):
            np.add.at(total, to_np(t.select.idx[r]).view(np.uint32), to_np(t.select.val[r]).astype(np.float64))
        summed = to_np(t.reduce.out_val)
        np.testing.assert_allclose(summed, total, rtol=1e-6, atol=1e-9)
        norm, factor = to_np(t.update.out)
        np.testing.assert_allclose(norm, np.linalg.norm(summed.astype(np.float64)), rtol=1e-6)
        decay = np.repeat(np.float32([0.0, 0.01, 0.0]), t.sizes)
        after = np.empty_like(before)
        for part in range(3):  # decay is a number a tensor
            at = slice(sum(t.sizes[:part]), sum(t.sizes[:part + 1]))
            after[at] = R.adamw(before[at], summed[at], m[at], v[at], lr=t.lr, step=t.steps, beta2=0.99,
                                decay=decay[at][0], factor=factor, bits=32)[0]
        np.testing.assert_array_equal(to_np(t.flat), after)
