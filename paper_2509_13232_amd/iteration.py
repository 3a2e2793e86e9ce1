"""Whole SPO iterations of a toy policy, from the tracker's prompts to new weights, through the library's calls alone:

    python -m paper_2509_13232_amd.iteration [--iterations 30] [--normalise] [--step adamw [--state-bits 8]]

The policy is one trained projection P before a fixed LM head W: hidden = features(prompt, position) P.  With --normalise a layer
normalisation with trained weight and bias stands between P and the head (``spo_norm_fwd``, ``spo_norm_bwd``).  A prompt is a fixed
random state per position (and a constant, which all prompts share), a response R tokens, each drawn from the K likeliest of
its position.  A response is rewarded if at least half of its tokens are from the vocabulary's first quarter.  An iteration

  * draws prompts (``spo_sample_prompts``),
  * forms each position's alternatives (``spo_logprob_fwd`` on logits, top_k) and draws the response's tokens from them,
  * takes the behaviour log-probs and the entropy from the hidden states (``spo_logprob_fwd`` with the head),
  * turns rewards into advantages and updates the tracker (``spo_advantages``, ``spo_tracker_update``),
  * adds the gradients of the PPO-clip loss and of an entropy bonus (``spo_pg_loss_fwd``, ``spo_pg_loss_bwd``,
    ``spo_logprob_bwd``) and takes one momentum step on P (``spo_muon_update``), a few times over.  The normalisation's weight and
    bias take an AdamW step; with --step adamw so do P and the head, which then is trained too, with the gradients' norm held
    below 1 (``spo_grad_norm``, ``spo_adamw_update``).

The features, the drawing from the alternatives and the two products with P are plain torch.
"""
import argparse

import torch

from . import binding as spo


class Policy:
    def __init__(self, prompts=64, tokens=16, hidden=256, vocab=4000, top_k=16, seed=0, device="cuda", normalise=False, step="muon", state_bits=32):
        g = torch.Generator().manual_seed(seed)
        self.prompts, self.tokens, self.vocab, self.top_k = prompts, tokens, vocab, top_k
        x = torch.randn((prompts, tokens, hidden), generator=g)
        x[:, :, :8] = 1.0
        self.x = x.to(device, torch.bfloat16)
        self.P = (torch.randn((hidden, hidden), generator=g) * hidden ** -0.5).to(device)
        self.W = (torch.randn((vocab, hidden), generator=g) * hidden ** -0.5).to(device, torch.bfloat16)
        self.momentum = torch.zeros_like(self.P)
        self.alpha, self.beta = spo.spo_tracker_init(torch.full((prompts,), 0.5, device=device), 0.875)
        self.draws = torch.Generator(device=device).manual_seed(seed + 1)
        self.norm = (torch.ones(hidden, device=device), torch.zeros(hidden, device=device)) if normalise else None
        self.train_head = step == "adamw"
        self.master = self.W.float() if self.train_head else None     # the head's weights, of which W is the copy that products take
        # what AdamW steps are for, in the order of gradients()
        self.adamw = ([self.P, self.master] if self.train_head else []) + list(self.norm or ())
        self.copies = [self.W if t is self.master else None for t in self.adamw]
        self.decay = [0.1 if t.dim() == 2 else 0.0 for t in self.adamw]
        self.states = [spo.adamw_state(t, state_bits) for t in self.adamw]
        self.steps = torch.zeros(1, dtype=torch.int64, device=device)

    def normalisation(self, x):
        return spo.make_norm_desc(x @ self.P.to(torch.bfloat16), *self.norm)

    def hidden(self, x):
        if self.norm:
            return spo.spo_norm_fwd(self.normalisation(x), want_stats=False)[0]
        return x @ self.P.to(torch.bfloat16)


def respond(policy, idx):
    """Responses to the prompts idx, their tokens drawn from the likeliest: a batch of what the loss needs of them."""
    x = policy.x[idx.long()].flatten(0, 1)
    h = policy.hidden(x)
    alternatives = spo.make_logprob_desc(None, None, None, logits=h @ policy.W.t(), top_k=policy.top_k)
    _, _, _, ids, logp = spo.spo_logprob_fwd(alternatives)
    pick = torch.multinomial(torch.exp(logp), 1, generator=policy.draws)
    target = ids.gather(1, pick)[:, 0].contiguous()
    old_logp, _, entropy, _, _ = spo.spo_logprob_fwd(spo.make_logprob_desc(h, policy.W, target))
    good = (target < policy.vocab // 4).float().view(-1, policy.tokens).mean(dim=1)
    return dict(idx=idx, x=x, target=target, old_logp=old_logp, entropy=entropy, reward=(good >= 0.5).float(),
                cu_seqlens=torch.arange(idx.numel() + 1, dtype=torch.int32, device=x.device) * policy.tokens)


def gradients(policy, batch, adv, entropy_bonus):
    """Of (PPO-clip loss - entropy_bonus * mean entropy), fp32: d/dP, d/dW if the head is trained, then those of the normalisation."""
    x, train_head = batch["x"], policy.train_head
    if policy.norm:
        norm = policy.normalisation(x)
        h, mean, rstd = spo.spo_norm_fwd(norm)
    else:
        h = policy.hidden(x)
    T = h.shape[0]
    loss = spo.make_desc(h, policy.W, batch["target"], batch["old_logp"], None, adv, batch["cu_seqlens"], 0.2, 0.28)
    _, logp, lse, _ = spo.spo_pg_loss_fwd(loss)
    d_h, d_W = spo.spo_pg_loss_bwd(loss, logp, lse, d_hidden_dtype=torch.float32, want_d_W=train_head)
    if entropy_bonus:
        score = spo.make_logprob_desc(h, policy.W, batch["target"])
        _, lse, entropy, _, _ = spo.spo_logprob_fwd(score)
        d_entropy = torch.full((T,), -entropy_bonus / T, device=h.device)
        d_bonus, _ = spo.spo_logprob_bwd(score, lse, entropy, d_entropy=d_entropy, d_hidden_dtype=torch.float32, want_d_W=train_head,
                                         d_W=d_W, accumulate_dW=train_head)
        d_h += d_bonus
    rest = [d_W] if train_head else []
    if policy.norm:
        d_h, *of_norm = spo.spo_norm_bwd(norm, mean, rstd, d_h, dx=d_h)
        rest += of_norm
    return [x.t().float() @ d_h, *rest]


def gradient(policy, batch, adv, entropy_bonus):
    """d/dP of (PPO-clip loss - entropy_bonus * mean entropy), fp32."""
    return gradients(policy, batch, adv, entropy_bonus)[0]


def update(policy, grads, lr=0.02, mu=0.9, adamw_lr=3e-3, max_norm=1.0):
    """One step on all that is trained."""
    if not policy.train_head:
        spo.spo_muon_update(policy.P, policy.momentum, grads[0], lr, mu=mu)
        grads = grads[1:]
    if policy.adamw:
        desc = spo.make_adamw_desc(policy.adamw, grads, policy.states, weight_decay=policy.decay, copies=policy.copies)
        norm = spo.spo_grad_norm(desc)
        spo.spo_adamw_update(desc, adamw_lr, policy.steps, grad_norm=norm, max_norm=max_norm)


def iterate(policy, iteration, batch_size=32, steps=2, lr=0.02, mu=0.9, entropy_bonus=1e-3):
    """One iteration; returns (mean reward, mean entropy of the responses' tokens)."""
    idx = spo.spo_sample_prompts(policy.alpha, policy.beta, batch_size, seed=7, iteration=iteration)
    batch = respond(policy, idx)
    _, adv, _ = spo.spo_advantages(policy.alpha, policy.beta, idx, batch["reward"], eps_norm=1e-6)
    for _ in range(steps):
        update(policy, gradients(policy, batch, adv, entropy_bonus), lr, mu)
    after, _, _, _, _ = spo.spo_logprob_fwd(spo.make_logprob_desc(policy.hidden(batch["x"]), policy.W, batch["target"]))
    kl = (batch["old_logp"] - after).view(-1, policy.tokens).mean(dim=1).clamp(min=0.0)
    spo.spo_tracker_update(policy.alpha, policy.beta, idx, batch["reward"], kl, 0.06, 0.875, 0.96)
    return float(batch["reward"].mean()), float(batch["entropy"].mean())


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--iterations", type=int, default=30)
    ap.add_argument("--normalise", action="store_true", help="a layer normalisation before the head")
    ap.add_argument("--step", choices=["muon", "adamw"], default="muon", help="adamw: of P and of the head")
    ap.add_argument("--state-bits", type=int, choices=[32, 8], default=32, help="of the AdamW steps' moments")
    args = ap.parse_args()
    policy = Policy(normalise=args.normalise, step=args.step, state_bits=args.state_bits)
    for i in range(args.iterations):
        reward, entropy = iterate(policy, i)
        value = float((policy.alpha / (policy.alpha + policy.beta)).mean())
        print(f"iteration {i:3d}  reward {reward:.3f}  tracked success {value:.3f}  entropy {entropy:.3f}", flush=True)


if __name__ == "__main__":
    main()
