"""A small policy trained by its own samples, through the library from hidden states to hidden states:

    python -m paper_2512_06547_amd.example

The policy is an embedding, a norm and a vocabulary head: enough to need every operator around a language model's head, and
small enough that nothing else is in the way.  A step draws a group of answers to each prompt as a serving process does,
from a copy of the weights that is some steps old and has its head in 4 bits:

    norm_fwd -> w4_linear -> adjust_logits (penalties, temperature, grammar mask) -> sample (tokens and their log-probs)

trains on them, the policy being the adjusted one that the tokens were drawn from:

    norm_fwd -> head -> adjust_logits -> loss_fwd_bwd -> adjust_logits_bwd -> head's gradients -> norm_bwd

and takes a step of AdamW on fp32 weights, whose bfloat16 copies are the model's, and of which w4_quantize makes the next head in
4 bits:

    grad_norm -> adamw_step -> w4_quantize

The reward is the share of even tokens in an answer, so a rising mean reward says that the whole chain points the right way.
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass

import torch

from . import binding as a3po

RMS = a3po.A3PO_NORM_RMS


@dataclass
class Policy:
    embed: torch.Tensor  # [V, H], the model's dtype
    gamma: torch.Tensor  # [H] of the norm
    head: torch.Tensor   # [V, H]
    version: int = 0


@dataclass
class Sampling:
    """What the adjusted policy is, the same for every sequence here (the library takes a value a row)."""
    repetition: float = 1.2
    frequency: float = 0.1
    presence: float = 0.1
    temperature: float = 0.9
    allowed: torch.Tensor | None = None  # int32 [ceil(V / 32)] bits

    def rows(self, history, start, length, prompt):
        n, dev = start.numel(), start.device
        value = lambda v: torch.full((n,), v, dtype=torch.float32, device=dev)
        return dict(history=history, hist_start=start, hist_len=length, prompt_len=prompt, repetition=value(self.repetition),
                    frequency=value(self.frequency), presence=value(self.presence), temperature=value(self.temperature),
                    allowed=self.allowed)


def new_policy(V, H, dtype, device, seed=0):
    g = torch.Generator().manual_seed(seed)
    make = lambda *shape: torch.randn(*shape, generator=g).to(device=device, dtype=dtype)
    # (the embeddings share a direction: what is learnt behind one token then holds behind another)
    return Policy(make(V, H) + 1, torch.ones(H, dtype=dtype, device=device), make(V, H) * H ** -0.5)


def quantize_w4(weight, group):
    """codes uint8 [N, H/2], scales float32 and zero points uint8 [N, H/group] for w4_linear: the nearest of 16 evenly spaced
    values between each group's extremes, zero among them."""
    return a3po.w4_quantize(weight, group, zeros=True)


def rollout(policy, sampling, prompts, new_tokens, group=128, generator=None):
    """Draws new_tokens behind each prompt [S, P].  -> history int32 [S, P + new_tokens], logp float32 [S, new_tokens].
    A ValueError where a row leaves no token to draw."""
    S, P = prompts.shape
    dev, total = prompts.device, P + new_tokens
    history = torch.zeros(S, total, dtype=torch.int32, device=dev)
    history[:, :P] = prompts
    start = torch.arange(S, dtype=torch.int64, device=dev) * total
    prompt = torch.full((S,), P, dtype=torch.int32, device=dev)
    gamma = policy.gamma.bfloat16()
    codes, scales, zeros = quantize_w4(policy.head, group)
    logp = torch.empty(S, new_tokens, device=dev)
    for i in range(new_tokens):
        length = torch.full((S,), P + i, dtype=torch.int32, device=dev)
        hidden = policy.embed[history[:, P + i - 1].long()].bfloat16()
        hidden, _, _ = a3po.norm_fwd(hidden, gamma, kind=RMS, out=hidden, want_stats=False)
        logits = a3po.w4_linear(hidden, codes, scales, zeros, group=group, out_dtype=torch.float32)
        rows = sampling.rows(history.view(-1), start, length, prompt)
        u = a3po.adjust_logits(logits, out=logits, want_lse=False, **rows)["out"]
        drawn = a3po.sample(u, torch.rand(S, generator=generator, device=dev))  # (u is adjusted: no temperature is left to apply)
        token, logp[:, i] = drawn["token"], drawn["logp"]
        history[:, P + i] = token
    if bool((history < 0).any()):  # (rows whose mask or weights leave nothing: as an index, -1 would be a token elsewhere or none)
        raise ValueError("no token to draw: a row of the adjusted logits is all masked, or holds NaN or +inf")
    return history, logp


def gradients(policy, sampling, history, logp_behav, versions, rewards, P, G, clip_eps=0.2):
    """One pass over the answers: the loss and its gradients with respect to the hidden states, gamma and the head."""
    S, total = history.shape
    new, dev = total - P, history.device
    at = torch.arange(S * new, device=dev)
    seq, place = at // new, at % new
    rows = sampling.rows(history.view(-1), (seq * total).contiguous(), (P + place).int(),
                         torch.full((S * new,), P, dtype=torch.int32, device=dev))
    source = history[:, P - 1:-1].reshape(-1).long()
    chosen = history[:, P:].reshape(-1).contiguous()
    hidden = policy.embed[source]
    normed, _, rstd = a3po.norm_fwd(hidden, policy.gamma, kind=RMS)
    logits = normed @ policy.head.t()
    # (not in the logits' place: the gradient asks for the sign that a penalised logit had)
    u = a3po.adjust_logits(logits, out_dtype=torch.float32, want_lse=False, **rows)["out"]
    advantages = a3po.grpo_advantages(rewards, G, seq.int())
    mask = torch.ones(S * new, dtype=torch.uint8, device=dev)
    out = a3po.loss_fwd_bwd(u, chosen, logp_behav.reshape(-1), versions, policy.version, advantages, mask, clip_eps, dlogits=u)
    dz = a3po.adjust_logits_bwd(out["dlogits"], logits, **rows)
    back = a3po.norm_bwd(dz @ policy.head, hidden, policy.gamma, rstd, kind=RMS)
    return dict(loss=out["loss"], stats=out["stats"], source=source, dhidden=back["dx"], dgamma=back["dweight"],
                dhead=dz.t() @ normed)


class Trainer:
    """The fp32 weights behind a policy, and AdamW's states for them."""

    def __init__(self, policy, lr, bits=32, max_norm=1.0, weight_decay=0.0):
        self.names, self.lr, self.max_norm, self.weight_decay, self.steps = ("embed", "gamma", "head"), lr, max_norm, weight_decay, 0
        self.master = [getattr(policy, k).float() for k in self.names]
        states = [a3po.adamw_state(p, bits) for p in self.master]
        self.exp_avgs, self.exp_avg_sqs = [s[0] for s in states], [s[1] for s in states]
        self.scales = None if bits == 32 else [s[2] for s in states]

    def step(self, policy, got):
        """One update from what gradients() gave; policy's weights become bfloat16 copies of the new ones."""
        embed = torch.zeros_like(self.master[0]).index_add_(0, got["source"], got["dhidden"].float())
        grads = [embed, got["dgamma"], got["dhead"].float()]
        self.steps += 1
        a3po.adamw_step(self.master, grads, self.exp_avgs, self.exp_avg_sqs, scales=self.scales, copies=[getattr(policy, k) for k in self.names],
                        step=self.steps, lr=self.lr, weight_decay=self.weight_decay, norm=a3po.grad_norm(grads), max_norm=self.max_norm,
                        seed=self.steps)
        policy.version += 1


def even_share(history, P):
    return (history[:, P:] % 2 == 0).float().mean(1)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--prompts", type=int, default=16)
    ap.add_argument("--group", type=int, default=8, help="answers a prompt")
    ap.add_argument("--new-tokens", type=int, default=32)
    ap.add_argument("--lag", type=int, default=2, help="steps that the sampling weights are behind by, at most")
    ap.add_argument("--lr", type=float, default=0.02)
    ap.add_argument("--state-bits", type=int, default=32, choices=(32, 8), help="of AdamW's states")
    args = ap.parse_args(argv)
    dev, P = "cuda", 8
    policy = new_policy(args.vocab, args.hidden, torch.bfloat16, dev)
    trainer = Trainer(policy, args.lr, args.state_bits)
    sampling = Sampling()
    g, gpu = torch.Generator().manual_seed(1), torch.Generator(device=dev).manual_seed(1)
    behaviour, shares = policy, []
    for step in range(args.steps):
        if step % (args.lag + 1) == 0:
            behaviour = Policy(policy.embed.clone(), policy.gamma.clone(), policy.head.clone(), policy.version)
        prompts = torch.randint(0, args.vocab, (args.prompts, P), generator=g, dtype=torch.int32)
        history, logp = rollout(behaviour, sampling, prompts.repeat_interleave(args.group, 0).to(dev), args.new_tokens,
                                generator=gpu)
        rewards = even_share(history, P)
        versions = torch.full((logp.numel(),), behaviour.version, dtype=torch.int32, device=dev)
        got = gradients(policy, sampling, history, logp, versions, rewards, P, args.group)
        trainer.step(policy, got)
        shares.append(float(rewards.mean()))
        print(f"step {step}: version {behaviour.version} of {policy.version - 1}, even tokens {shares[-1]:.3f}, "
              f"loss {float(got['loss']):+.4f}, clipped {a3po.stats_to_dict(got['stats'])['n_clipped']}", flush=True)
    return shares


if __name__ == "__main__":
    main()
