"""The learner's calls together, as a learner makes them: score stored tokens, take the rows behind the scores, the loss and its
gradient with the coefficients of the scores, and put the stepped head back in place."""
import numpy as np
import pytest
import torch

import paper_2603_18464_amd as P
import workloads as W
from oracle.loss_oracle import Loss, target
from tests.parity import device_inputs
from tests.test_gpu_parity import make_policy, ragged_obs

pytestmark = pytest.mark.gpu


def setup(dtype, K=5, batch=6):
    shape = W.PolicyShape(2, 256, 2, 128, 704, 1024, dtype=dtype)
    wl = W.Workload("Tl", 41, shape, batch=batch, n_patches=30, instr_len=(0, 9), n_tokens=K)
    weights = W.make_weights(shape, wl.seed)
    obs = ragged_obs(wl, [30, 1, 17, 30, 2, 29][:batch], [0, 3, 9, 4, 1, 5][:batch], seed=77)
    pol = make_policy(wl, weights, extra_seq=K)
    dev = device_inputs(pol, obs)
    return wl, weights, pol, (dev["patch_emb"], obs["cu_patch"], dev["instr_ids"], obs["cu_instr"])


def within(got, want, bound):
    err = (got.double() - want).abs()
    assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [1, 5])
def test_a_policy_gradient_step_of_the_head(dtype, K):
    wl, weights, pol, args = setup(dtype, K)
    s, B = wl.shape, wl.batch
    gen = torch.Generator().manual_seed(5)
    tokens = torch.randint(0, s.n_action_bins, (B, K), generator=gen, dtype=torch.int32).to(pol.device)
    mu = (-5.0 + torch.rand(B, K, generator=gen)).to(pol.device)
    advantage = torch.randn(B, K, generator=gen).to(pol.device)
    tau = 1.3
    sc = pol.score_tokens(*args, tokens, temperature=tau, mu_logp=mu, sigma=0.5, want_logits=True)
    h = pol.action_hidden(B, K)
    again = pol.action_hidden(B, K)                                  # (may be asked for again)
    head = pol.to_device(weights["lm_head"])[s.action_id0:]
    assert torch.equal(h, again)
    # the scores' logits from the rows, which are rounded to the storage type here, and summed over d in float32 there
    z = h.double() @ head.double().T
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    bound_z = (h.double().abs() @ head.double().abs().T) * (half * 1.01 + s.d_model * 2.0 ** -24) + 1e-30
    within(sc["logits"].reshape(B * K, -1), z, bound_z)
    # the loss is minus the log-probability
    loss, lse = P.token_loss(h, head, tokens.reshape(-1), temperature=tau)
    o = Loss(h, head, target(s.n_action_bins, labels=tokens.reshape(-1)), tau)
    want_loss, _, b_loss, _ = o.loss_bounds()
    within(loss, want_loss, b_loss)
    within(-sc["logp"].reshape(-1), want_loss, b_loss + 2 * bound_z.max(1).values / tau)
    # gradient of -(omega rho A) log pi, by the coefficients of the scores, against the formula
    g = -(sc["weight"] * advantage).reshape(-1)
    coef = (g * -1.0).contiguous()
    gh, gw = P.token_loss_grad(h, head, tokens.reshape(-1), lse, coef, temperature=tau)
    (wh, bh), (ww, bw) = o.grad_bounds(coef)
    within(gh, wh, bh)
    within(gw, ww, bw)
    # a step, put back in place while nothing runs; the next scores are those of the new head on the same rows
    new = pol.to_device(weights["lm_head"]).clone()
    new[s.action_id0:] -= (0.01 * gw.float() / gw.float().abs().max()).to(new.dtype)
    pol.drain_begin()
    pol.update_begin()
    with pytest.raises(P.VlaError):
        pol.action_hidden(B, K)                                      # weights are being written
    pol.update_tensors({"lm_head": new})
    pol.update_commit()
    with pytest.raises(P.VlaError):
        pol.action_hidden(B, K)                                      # rows of the old weights
    sc2 = pol.score_tokens(*args, tokens, temperature=tau)
    h2 = pol.action_hidden(B, K)
    assert torch.equal(h2, h)                                        # (the head has no part in them)
    o2 = Loss(h2, new[s.action_id0:], target(s.n_action_bins, labels=tokens.reshape(-1)), tau)
    want2, _, b2, _ = o2.loss_bounds()
    within(-sc2["logp"].reshape(-1), want2, b2 + 2 * bound_z.max(1).values * 1.1 / tau)
    pol.close()


def test_distillation_from_a_policy_into_another_ones_head():
    """Teacher logits from one policy's scores, the student's rows and head from another."""
    wl, weights, pol, args = setup("bf16")
    s, B, K = wl.shape, wl.batch, wl.n_tokens
    tokens = torch.zeros((B, K), dtype=torch.int32, device=pol.device)
    top = pol.score_tokens(*args, tokens, want_logits=True)["logits"].reshape(B * K, -1).topk(20)
    top_logits, top_ids = top.values.contiguous(), top.indices.to(torch.int32)
    pol.load_weights(W.make_weights(s, wl.seed + 3))
    with pytest.raises(P.VlaError):
        pol.action_hidden(B, K)
    pol.policy_step_parallel(*args, K, 7)
    h = pol.action_hidden(B, K)
    with pytest.raises(P.VlaError):
        pol.action_hidden(B, K + 1)
    head = pol.to_device(W.make_weights(s, wl.seed + 3)["lm_head"])[s.action_id0:]
    loss, lse = P.distill_loss(h, head, top_logits, top_ids, temperature=2.0)
    o = Loss(h, head, target(s.n_action_bins, top_logits=top_logits, top_ids=top_ids, tau=2.0), 2.0)
    want, _, b, _ = o.loss_bounds()
    within(loss, want, b)
    coef = torch.full((B * K,), 1.0 / (B * K), device=pol.device)
    gh, gw = P.distill_loss_grad(h, head, top_logits, top_ids, lse, coef, temperature=2.0)
    (wh, bh), (ww, bw) = o.grad_bounds(coef)
    within(gh, wh, bh)
    within(gw, ww, bw)
    pol.prefill(*args)                                               # overwrites the workspace
    with pytest.raises(P.VlaError):
        pol.action_hidden(B, K)
    pol.close()
