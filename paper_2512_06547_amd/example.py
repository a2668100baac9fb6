"""A small policy trained by its own samples, through the library from hidden states to hidden states:

    python -m paper_2512_06547_amd.example

The policy is an embedding, a norm and a vocabulary head: enough to need every operator around a language model's head, and
small enough that nothing else is in the way.  A step draws a group of answers to each prompt as a serving process does,
from a copy of the weights that is some steps old and has its head in 4 bits:

    norm_fwd -> w4_linear -> adjust_logits (penalties, temperature, grammar mask; log-probs of the drawn tokens)

and trains on them, the policy being the adjusted one that the tokens were drawn from:

    norm_fwd -> head -> adjust_logits -> loss_fwd_bwd -> adjust_logits_bwd -> head's gradients -> norm_bwd

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
    N, H = weight.shape
    w = weight.float().view(N, H // group, group)
    low, high = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
    scales = ((high - low) / 15).clamp(min=1e-12)
    zeros = torch.round(-low / scales).clamp(0, 15)
    q = (torch.round(w / scales[..., None]) + zeros[..., None]).clamp(0, 15).to(torch.uint8).view(N, H // 2, 2)
    return (q[..., 0] | q[..., 1] << 4).contiguous(), scales.contiguous(), zeros.to(torch.uint8).contiguous()


def rollout(policy, sampling, prompts, new_tokens, group=128, generator=None):
    """Draws new_tokens behind each prompt [S, P].  -> history int32 [S, P + new_tokens], logp float32 [S, new_tokens]."""
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
        noise = torch.empty_like(u).exponential_(generator=generator).clamp_(min=1e-30).log_()  # (the largest u - noise is a sample)
        token = (u - noise).argmax(1).int()
        logp[:, i] = a3po.token_logprobs(u, token, want_lse=False, want_chosen_logit=False)[0]
        history[:, P + i] = token
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
    ap.add_argument("--lr", type=float, default=2.0)
    args = ap.parse_args(argv)
    dev, P = "cuda", 8
    policy = new_policy(args.vocab, args.hidden, torch.bfloat16, dev)
    master = {k: getattr(policy, k).float() for k in ("embed", "gamma", "head")}
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
        master["embed"].index_add_(0, got["source"], got["dhidden"].float(), alpha=-args.lr)
        master["head"] -= args.lr * got["dhead"].float()
        master["gamma"] -= args.lr * got["dgamma"]
        for k, v in master.items():
            setattr(policy, k, v.to(torch.bfloat16))
        policy.version += 1
        shares.append(float(rewards.mean()))
        print(f"step {step}: version {behaviour.version} of {policy.version - 1}, even tokens {shares[-1]:.3f}, "
              f"loss {float(got['loss']):+.4f}, clipped {a3po.stats_to_dict(got['stats'])['n_clipped']}", flush=True)
    return shares


if __name__ == "__main__":
    main()
