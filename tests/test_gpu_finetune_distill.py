"""The fine-tuning example's steps that score and distil: the gradients that
they leave are the formulas' (by fp64 differentiation of the same model), and
the example runs."""
import numpy as np
import pytest

from gpu_util import say, torch_dev

pytestmark = pytest.mark.gpu

u = 2.0 ** -24  # half a step of fp32


def trainer(ranks=2, tokens=96, seed=0, **kw):
    from paper_1802_08021_amd.finetune import Trainer
    t = Trainer(vocab=48, hidden=24, ranks=ranks, tokens=tokens, kb=16, bucket=64, seed=seed, **kw)
    t.flat.add_(torch_dev()[0].randn(t.flat.shape, device=t.dev, generator=t.gen), alpha=0.3)
    return t


def model64(t):
    """The model's parameters in fp64 on the CPU, as leaves."""
    return [p.detach().double().cpu().clone().requires_grad_() for p in t.views(t.flat)]


def check_gradients(t, rank, leaves, h, dz, rel):
    """The rank's row against the leaves' gradients.  Each logit's derivative may
    be off by `rel` (|dz| here: a bound of it); the products after it sum V, T and
    a token's terms in fp32, tanh and 1 - h^2 are within 8 roundings."""
    V, D, T = t.V, t.D, h.shape[0]
    W = leaves[1].detach().abs()
    h = h.detach().abs()
    off = rel * dz
    got = [g.double().cpu() for g in t.views(t.grads[rank])]
    x = t.seen[rank].cpu()
    zero = W.new_zeros(V, D)
    bounds = [zero.index_add(0, x, (off + (V + T + 8) * u * dz) @ W.t()),
              h.t() @ (off + (T + 8) * u * dz),
              (off + T * u * dz).sum(0)]
    for name, g, leaf, bound in zip(("hidden", "output", "bias"), got, leaves, bounds):
        worst = ((g - leaf.grad).abs() / (bound + 1e-30)).max()
        say(f"[finetune] rank {rank} {name}: {float(worst):.3f} of the bound")
        assert bool(((g - leaf.grad).abs() <= bound + 1e-12).all()), name


def forward64(t, leaves, x):
    h = leaves[0][x].tanh()
    z = h @ leaves[1] + leaves[2]
    # the fp32 logits: D products and a bias, tanh within 4 roundings
    err = (t.D + 6) * u * float((h.detach().abs() @ leaves[1].detach().abs() + leaves[2].detach().abs()).max())
    return h, z, err


def steps_off(t):
    """step() left out; the tokens of each rank are kept as they are drawn."""
    t.seen = []
    draw = t.draw

    def note(*shape):
        t.seen.append(draw(*shape))
        return t.seen[-1]
    t.draw, t.step = note, lambda: None


@pytest.mark.parametrize("top,hard,beta", [(5, 0.0, 0.0), (48, 0.0, 1.0), (1, 0.25, 0.0), (16, 0.5, 0.5)])
def test_distill_step_gradients(top, hard, beta):
    from paper_1802_08021_amd import sparcml as S
    torch, _ = torch_dev()
    t, teacher = trainer(), trainer(seed=1)
    steps_off(t)
    stats = t.distill_step(teacher, top=top, hard=hard, beta=beta).cpu().double()
    losses = []
    for rank in range(t.P):
        x = t.seen[rank]
        told = S.token_scores(teacher.logits(x)[1], top=top)
        ids, lq = told["top_id"].cpu().long(), told["top_logp"].cpu().double()
        leaves = model64(t)
        h, z, err = forward64(t, leaves, x.cpu())
        lp = torch.log_softmax(z, 1)
        q = torch.cat([lq.exp(), (1 - lq.exp().sum(1, keepdim=True)).clamp_min(2.0 ** -24)], 1)
        p = lp.exp().gather(1, ids)
        on = torch.zeros_like(lp).scatter(1, ids, 1.0)
        p = torch.cat([p, (lp.exp() * (1 - on)).sum(1, keepdim=True)], 1)
        if top == t.V:  # (nothing is left beside the list)
            q, p = q[:, :top], p[:, :top]
        m = beta * q + (1 - beta) * p
        if beta == 0:
            div = (q * (q.log() - p.log())).sum(1)
        elif beta == 1:
            div = (p * (p.log() - q.log())).sum(1)
        else:
            div = (beta * q * (q.log() - m.log()) + (1 - beta) * p * (p.log() - m.log())).sum(1)
        nll = -lp.gather(1, t.right(x).cpu()[:, None])[:, 0]
        loss = ((1 - hard) * div + hard * nll).mean()
        loss.backward()
        losses.append(float(loss.detach()))
        # |dz|: (1 - hard) |f_v - p_v F| + hard |p_v - [right]|, |f| <= q or p |ln|
        size = 1.0 if beta == 0 else float((p.log() - q.log()).abs().max().detach()) + 1.0
        dz = lp.exp().detach() * (2 * size) / t.T
        dz = dz.scatter_add(1, ids, q[:, :top].detach() * size / t.T).scatter_add(1, t.right(x).cpu()[:, None], dz.new_full((t.T, 1), hard / t.T))
        check_gradients(t, rank, leaves, h, dz, 4 * err + 64 * u)
    want = float(np.mean(losses))
    say(f"[finetune] distil {top} {hard} {beta}: loss {float(stats[0]):.6f}, {want:.6f}")
    size = 1.0 if beta == 0 else size
    assert abs(float(stats[0]) - want) <= (4 * err + 64 * u) * (size + abs(want) + 10)


def test_entropy_moves_the_policy_step_by_its_gradient():
    torch, _ = torch_dev()
    worth = 0.125
    rows = []
    for e in (0.0, worth):
        t = trainer()
        steps_off(t)
        t.policy_step(e)
        rows.append(t.grads.clone())
    more = t.grads
    more.copy_(rows[1] - rows[0])
    for rank in range(t.P):
        leaves = model64(t)
        h, z, err = forward64(t, leaves, t.seen[rank].cpu())
        lp = torch.log_softmax(z, 1)
        (worth * (lp.exp() * lp).sum(1)).mean().backward()  # minus the entropy
        # |dz| = e p |ln p + H| / T; what was subtracted and the policy's own part
        # (at most 2 p + [token]) were rounded once each
        large = float(lp.detach().abs().max()) + float(np.log(t.V))
        dz = lp.exp().detach() * (worth * large + 2) / t.T + 1.0 / t.T
        check_gradients(t, rank, leaves, h, dz, 4 * err * worth * large + 64 * u)


def test_distill_step_updates_and_the_example_runs(capsys):
    from paper_1802_08021_amd.finetune import main
    torch, _ = torch_dev()
    t, teacher = trainer(ranks=3, state_bits=32), trainer(seed=1)
    before, other = t.flat.clone(), teacher.flat.clone()
    stats = t.distill_step(teacher).tolist()
    torch.cuda.synchronize()
    assert np.isfinite(stats).all() and 0 < stats[3] <= 1.00001
    assert bool((t.flat != before).any()) and bool(torch.isfinite(t.flat).all())
    assert bool((teacher.flat == other).all())
    main(["--pairs-steps", "1", "--policy-steps", "10", "--distill-steps", "10", "--entropy", "0.01"])
    out = capsys.readouterr().out
    assert "policy  10:" in out and "distil  10:" in out
