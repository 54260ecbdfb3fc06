"""Inner loop of RAPID (Alg. 1, procedure IW-GRPG) on a synthetic bandit: one inference batch, H
off-policy updates of the LM head, each on its own mini-batch.

As in Alg. 1 the inference batch Z (hidden states, sampled tokens, rewards, behaviour log-probs
stored with the initial W = mu) is cut into H = N_inference / N_step mini-batches of whole groups,
which the inner loop walks through in order (Sec. 3.2; Alg. 1, the loop over mini-batches).  Step h
calls rapid_iw_pg_loss_fwd_bwd on mini-batch h with the current W against the stored log mu, then
takes one gradient step (rapid_sgd_step, or rapid_adamw_step: the optimiser family of the paper's runs).  Step 1 is on-policy (all ratios exactly 1); the
staleness of Sec. 4.3 (mean |log clipped weight|) and the clip proportion grow with h, the trend of
the paper's study of the number of inner steps.  Everything numeric runs in the library; this
module only sequences calls and slices tensors.

With --tied the policy is a tied table instead of a head on given states (workloads.make_tied_workload): every step looks its
hidden states up in the current table and adds the lookup's gradient to the head's, and the behaviour policy is the
table's 8-bit copy, as an engine that generates in 8 bits serves it.  Its log-probs differ from the table's own by that
rounding, which the ratios of step 1 show: staleness is small there, not 0.

    python -m paper_2510_03515_amd.iw_grpg [--inner-steps 8] [--lr 0.02] [--optimizer sgd|adamw] [--logits-cache] [--tied]
"""
from __future__ import annotations

import argparse

import torch

from . import binding as rb
from . import workloads as wl


def _is_reward(w, lp, logp_b):
    """Self-normalised importance-sampling estimate, on the whole inference batch, of the expected
    reward of the policy that gives its tokens the log-probs lp (equals the batch's mean reward for lp = log mu)."""
    s, _ = rb.rapid_seq_logratio(lp, logp_b, w["mask"])
    # With the whole batch as one group and no clip, the unclipped baseline of Eq. (4) is (1/N) sum rho R:
    # once with the rewards, once with rewards of 1 (then it is the mean ratio); their quotient is the estimate.
    one_group = torch.zeros_like(w["group_ids"])
    ones = torch.ones_like(w["rewards"])
    num = rb.rapid_group_advantage(w["rewards"], one_group, 1, seq_logratio=s, eta=float("inf"))["adv"]
    den = rb.rapid_group_advantage(ones, one_group, 1, seq_logratio=s, eta=float("inf"))["adv"]
    return (w["rewards"][0] - num[0]).item() / (1.0 - den[0]).item()


def iw_grpg(w, inner_steps=8, lr=0.02, eta=2.0, coef_mode=1, logits_cache=False, optimizer="sgd"):
    """Runs Alg. 1's IW-GRPG on the workload dict `w` (device tensors of workloads.make_workload with
    sigma = 0 and tokens_from = "cur": the batch is sampled from W itself, and group_ids = n // G).
    The number of prompts must be a multiple of `inner_steps`.  Returns (per-step log, summary dict,
    final weights in the workload dtype).

    coef_mode 1 (clipped outer weight) is the default here: with the unclipped ratio of coef_mode 0
    a few generations whose ratio has grown dominate the later steps.  logits_cache (bf16 only): the
    backward of every step contracts the probability ratios its forward kept instead of regenerating
    the logits.  optimizer: "sgd" (plain descent with step lr) or "adamw" (lr is then AdamW's; its per-element
    step is about lr whatever the gradient's size, so it wants a far smaller value than SGD's)."""
    spec = w["spec"]
    K, G, H = w["K"], spec.G, int(inner_steps)
    assert K % H == 0, "prompts must divide into equal mini-batches"
    Kh, Nh = K // H, (K // H) * G
    W = w["W"].clone()
    master = W.float().contiguous()
    exp_avg, exp_avg_sq = (torch.zeros_like(master), torch.zeros_like(master)) if optimizer == "adamw" else (None, None)
    logp_b, _ = rb.rapid_logprob_fwd(w["hidden"], W, w["tokens"], w["mask"])   # log mu, stored at "inference"
    score = lambda: rb.rapid_logprob_fwd(w["hidden"], W, w["tokens"], w["mask"])[0]
    reward_mu = _is_reward(w, score(), logp_b)
    gid_local = w["group_ids"][:Nh].contiguous()                                # 0 .. Kh-1 in every mini-batch
    buf = rb.IwPgBuffers(w["hidden"][:Nh], W, Kh, logits_cache=logits_cache)
    log = []
    for h in range(H):
        sl = slice(h * Nh, (h + 1) * Nh)
        out = rb.rapid_iw_pg_loss_fwd_bwd(w["hidden"][sl], W, w["tokens"][sl], w["mask"][sl], logp_b[sl],
                                          w["rewards"][sl], gid_local, Kh, buffers=buf, eta=eta,
                                          coef_mode=coef_mode, logits_cache=logits_cache)
        log.append(_log_entry(h, out))
        if optimizer == "adamw":
            rb.rapid_adamw_step(master, out.dW, exp_avg, exp_avg_sq, h + 1, lr, w_out=W)
        else:
            rb.rapid_sgd_step(master, out.dW, lr, w_out=W)
    torch.cuda.synchronize()
    summary = dict(reward_behaviour=reward_mu, reward_final_is_estimate=_is_reward(w, score(), logp_b))
    return log, summary, W


def _log_entry(h, out):
    dg = out.read_diag()
    return dict(step=h + 1, loss=out.loss.item(), staleness=dg["mean_abs_log_w"],
                clip_fraction=dg["n_clipped"] / dg["n_sequences"], max_abs_s=dg["max_abs_s"])


def served_in_8_bits(rows):
    """Rows [R,d] as a policy kept in 8 bits multiplies them: through rapid_quantize_fp8 and back, fp32."""
    q = rb.rapid_quantize_fp8(rows.contiguous(), w_layout=rb.W_VD)
    blocks = q.values.shape[1] // 128
    scale = torch.exp2(q.scales[:, :blocks].float() - 127.0)
    return (q.values.float().view(rows.shape[0], blocks, 128) * scale[:, :, None]).view(rows.shape[0], -1)[:, :rows.shape[1]]


def iw_grpg_tied(w, inner_steps=8, lr=0.02, eta=2.0, coef_mode=1, logits_cache=False, optimizer="sgd"):
    """iw_grpg on a tied table: `w` is the dict of workloads.make_tied_workload (device tensors, tokens drawn from the table
    served in 8 bits).  The table's gradient is the head's (dW, [V,d]) plus the lookup's, which is added to it in place."""
    spec, scale = w["spec"], w["scale"]
    K, G, H = w["K"], spec.G, int(inner_steps)
    assert K % H == 0, "prompts must divide into equal mini-batches"
    Kh, Nh = K // H, (K // H) * G
    E = w["table"].clone()
    master = E.float().contiguous()
    exp_avg, exp_avg_sq = (torch.zeros_like(master), torch.zeros_like(master)) if optimizer == "adamw" else (None, None)
    E8 = rb.rapid_quantize_fp8(E, w_layout=rb.W_VD)

    def score():            # of the current table's 8-bit copy
        return rb.rapid_logprob_fwd_fp8(rb.rapid_embedding_fwd(E, w["inputs"], w["mask"], scale=scale), E8, w["tokens"], w["mask"])[0]

    logp_b = score()        # log mu, stored at "inference"
    reward_mu = _is_reward(w, logp_b, logp_b)
    gid_local = w["group_ids"][:Nh].contiguous()
    hidden = torch.empty((Nh, spec.T, spec.d), dtype=E.dtype, device=E.device)
    buf = rb.IwPgBuffers(hidden, E, Kh, w_layout=rb.W_VD, logits_cache=logits_cache)
    ws = rb.alloc_workspace(rb.rapid_workspace_bytes(rb.OP_EMBEDDING_BWD, Nh, spec.T, spec.d, spec.V, 1, rb._dtype_code(E)), E.device)
    log = []
    for h in range(H):
        sl = slice(h * Nh, (h + 1) * Nh)
        inputs, mask = w["inputs"][sl], w["mask"][sl]
        rb.rapid_embedding_fwd(E, inputs, mask, scale=scale, out=hidden)
        out = rb.rapid_iw_pg_loss_fwd_bwd(hidden, E, w["tokens"][sl], mask, logp_b[sl], w["rewards"][sl], gid_local, Kh, buffers=buf,
                                          eta=eta, coef_mode=coef_mode, w_layout=rb.W_VD, logits_cache=logits_cache)
        rb.rapid_embedding_bwd(out.dhidden, inputs, mask, spec.V, scale=scale, dtable=out.dW, accumulate=True, workspace=ws)
        log.append(_log_entry(h, out))
        if optimizer == "adamw":
            rb.rapid_adamw_step(master, out.dW, exp_avg, exp_avg_sq, h + 1, lr, w_out=E)
        else:
            rb.rapid_sgd_step(master, out.dW, lr, w_out=E)
    rb.rapid_quantize_fp8(E, w_layout=rb.W_VD, out=E8)
    final = score()
    torch.cuda.synchronize()
    return log, dict(reward_behaviour=reward_mu, reward_final_is_estimate=_is_reward(w, final, logp_b)), E


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--inner-steps", type=int, default=8)
    ap.add_argument("--lr", type=float, default=None, help="default 0.02 for sgd, 2e-4 for adamw")
    ap.add_argument("--optimizer", default="sgd", choices=["sgd", "adamw"])
    ap.add_argument("--dtype", default="bf16", choices=["bf16", "f32"])
    ap.add_argument("--logits-cache", action="store_true", help="bf16 only: keep the forward's ratios for the backward")
    ap.add_argument("--tied", action="store_true", help="a tied table as the policy, its 8-bit copy as the behaviour policy")
    args = ap.parse_args()
    rb.load()
    spec = wl.small_spec("bandit", args.dtype, d=256, V=4096, prompts=64, G=8, len_lo=8, len_hi=48, sigma=0.0,
                         reward="bernoulli", tokens_from="cur")
    if args.tied:
        run, w = iw_grpg_tied, wl.make_tied_workload(spec, seed=0, device="cuda", scale=spec.d ** 0.5, as_served=served_in_8_bits)
    else:
        run, w = iw_grpg, wl.make_workload(spec, seed=0, device="cuda")
    lr = args.lr if args.lr is not None else 0.02 if args.optimizer == "sgd" else 2e-4
    log, summary, _ = run(w, inner_steps=args.inner_steps, lr=lr, logits_cache=args.logits_cache, optimizer=args.optimizer)
    print("step  loss        staleness  clip_frac  max|s|")
    for r in log:
        print(f"{r['step']:4d}  {r['loss']:+.4e}  {r['staleness']:.4f}     {r['clip_fraction']:.3f}      {r['max_abs_s']:.3f}")
    print(f"mean reward of the batch (behaviour policy) {summary['reward_behaviour']:.4f}; "
          f"importance-sampling estimate for the final policy {summary['reward_final_is_estimate']:.4f}")


if __name__ == "__main__":
    main()
