"""The learner's operators as they are used together: an actor fills the ring, the learner draws a batch, computes returns, the policy's
log probabilities and their gradient, the recurrent layer's gradients, orthogonalises the update and publishes it, and the actor goes on
with the new model.  Every stage is checked against the definitions in 64 bits on the same inputs."""
import numpy as np
import pytest
import torch

from paper_2205_05248_b200 import binding, workloads

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_one_learner_iteration(precision):
    cfg = workloads.small_config(H=64, D=16, E=96, n=4, A=8, C=192, L=24, T=60, precision=precision,
                                 env=dict(done_thresh24=1 << 20))
    w = workloads.make_weights(cfg)
    actor = binding.Actor(cfg)
    actor.set_weights(w)
    actor.rollout(cfg["env"], cfg["T"], 0.3)
    s = actor.ring_sample(0, 48)
    B, L, n, A = 48, cfg["L"], cfg["n"], cfg["A"]

    # returns of the batch: reward + 0.97 * what follows, cut where a game ended, padded steps left out
    gamma = torch.full((1, 1, 1), 0.97, device="cuda").expand(B, L, 1)
    ret = binding.marl_linear_scan(gamma, s["reward"].view(B, L, 1), done=s["done"], length=s["len"], form="raw", reverse=True)["y"]
    want = torch.zeros(B, L + 1, dtype=torch.float64, device="cuda")
    for t in reversed(range(L)):
        live = t < s["len"]
        v = s["reward"][:, t].double() + 0.97 * want[:, t + 1] * (s["done"][:, t] == 0)
        want[:, t] = torch.where(live, v, torch.zeros_like(v))
    assert float((ret[:, :, 0].double() - want[:, :L]).abs().max()) < 2e-5

    # log probabilities of the recorded actions: a padded step is an empty row
    r = binding.marl_policy_logprob(s["q"], s["action"], avail=s["avail"], temperature=0.5, top=2)
    live = (torch.arange(L, device="cuda")[None, :] < s["len"][:, None])[:, :, None].expand(B, L, n)
    assert bool((r["logp"][~live] == 0).all()) and bool((r["top_index"][~live] == -1).all()) and bool(torch.isfinite(r["logp"]).all())
    z = (s["q"].double() / 0.5).masked_fill(s["avail"] == 0, -float("inf"))
    lp = torch.log_softmax(z, -1).gather(-1, s["action"].long()[..., None])[..., 0]
    assert float((r["logp"].double() - lp)[live].abs().max()) < 1e-5
    # the greedy alternative is the action of every decision that was not explored, up to the actor's tie band
    best = s["q"].masked_fill(s["avail"] == 0, -float("inf")).max(-1).values
    picked = s["q"].gather(-1, r["top_index"][..., :1].clamp(min=0).long())[..., 0]
    assert torch.equal(picked[live], best[live])

    # policy gradient of sum(advantage * logp) + 0.01 entropy, back through a gated recurrence over the episodes
    adv = ret.expand(B, L, n).contiguous()
    dq = binding.marl_policy_logprob_backward(s["q"], s["action"], r["stats"], r["entropy"], g_logp=adv,
                                              g_entropy=torch.full((B, L, n), 0.01, device="cuda"), avail=s["avail"], temperature=0.5)
    assert bool((dq[~live] == 0).all()) and float(dq[live].sum(-1).abs().max()) < 1e-3      # a gradient of probabilities sums to 0
    gate = torch.randn(B, L, n * A, device="cuda")
    x = s["q"].view(B, L, n * A)
    k = binding.marl_linear_scan(gate, x, done=s["done"], length=s["len"], keep=True)
    d = binding.marl_linear_scan_backward(gate, x, k["states"], dq.view(B, L, n * A), done=s["done"], length=s["len"])
    assert bool(torch.isfinite(d["dgate"]).all()) and bool((d["dx"].view(B, L, n, A)[~live] == 0).all())

    # an update of the four matrices, orthogonalised and published
    names = ("W1", "W_ih", "W_hh", "W2")
    g = torch.Generator().manual_seed(1)
    upd = binding.marl_orthogonalise([torch.randn(*w[k].shape, generator=g).cuda() for k in names])
    for u in upd:
        sv = torch.linalg.svdvals(u.double())
        assert 0.3 < float(sv.min()) and float(sv.max()) < 1.3
    new = dict(w)
    for k, u in zip(names, upd):
        new[k] = np.ascontiguousarray(w[k] - 0.02 * u.cpu().numpy(), dtype=np.float32)
    actor.publish_weights(new, 2, cfg["T"])
    actor.rollout(cfg["env"], 4, 0.3)
    st, _ = actor.status()
    assert st == 0 and actor.weights_version == 2
    actor.destroy()
