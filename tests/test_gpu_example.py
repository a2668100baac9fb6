"""The example's chain of operators: its rollout against the policy computed in 64 bits, its gradients against 64-bit
differentiation of the loss written out, and its reward."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2512_06547_amd import example


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def bits_of(allowed):
    words = torch.zeros((allowed.numel() + 31) // 32, dtype=torch.int64)
    at = allowed.nonzero()[:, 0]
    words.index_add_(0, at // 32, 1 << (at % 32))
    return torch.where(words >= 1 << 31, words - (1 << 32), words).int()


def adjusted(z, history, P, sampling, allowed):
    """The adjusted logits of [S, new, V] raw ones, differentiable; history [S, P + new] int64."""
    S, new, V = z.shape
    rows = []
    for s in range(S):
        for i in range(new):
            seen = torch.zeros(V, dtype=torch.bool)
            seen[history[s, :P + i]] = True
            n = torch.bincount(history[s, P:P + i], minlength=V).double()
            u = z[s, i]
            u = torch.where(seen, torch.where(u > 0, u / sampling.repetition, u * sampling.repetition), u)
            u = u - sampling.frequency * n - sampling.presence * (n > 0)
            rows.append((u / sampling.temperature).masked_fill(~allowed, -math.inf))
    return torch.stack(rows).view(S, new, V)


def normed(x, gamma):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gamma


def make(V, dtype):
    policy = example.new_policy(V, 256, dtype, "cuda", seed=4)
    allowed = torch.rand(V, generator=torch.Generator().manual_seed(5)) < 0.7
    # values that 32 bits hold exactly, so that the reference uses the same
    return policy, allowed, example.Sampling(1.25, 0.125, 0.25, 0.75, bits_of(allowed).cuda())


def test_rollout_draws_from_the_adjusted_policy_and_tells_its_log_probs():
    """The normalised hidden values are bfloat16: a value whose fp32 result lies at a rounding boundary may take the other
    neighbour, 2^-8 of it.  Logits move by no more than that share of sum |x w|, their log-softmax by twice as much."""
    V, P, new, S, group = 700, 5, 12, 6, 64
    policy, allowed, sampling = make(V, torch.bfloat16)
    prompts = torch.randint(0, V, (S, P), generator=torch.Generator().manual_seed(6), dtype=torch.int32)
    history, logp = example.rollout(policy, sampling, prompts.cuda(), new, group, torch.Generator("cuda").manual_seed(7))
    history, logp = history.cpu().long(), logp.cpu().double()
    assert torch.equal(history[:, :P], prompts.long()) and allowed[history[:, P:]].all()
    codes, scales, zeros = (t.cpu() for t in example.quantize_w4(policy.head, group))
    q = torch.stack((codes & 15, codes >> 4), 2).view(V, -1, group).double()
    w = ((q - zeros[..., None].double()) * scales[..., None].double()).view(V, -1)
    assert ((w - policy.head.cpu().double()).abs().view(V, -1, group) <= 1.001 * scales[..., None].double()).all()
    x = normed(policy.embed.cpu().double()[history[:, P - 1:-1]], policy.gamma.cpu().double()).bfloat16().double()
    u = adjusted(x @ w.t(), history, P, sampling, allowed)
    ref = torch.log_softmax(u, 2).gather(2, history[:, P:, None])[..., 0]
    bar = 2 * 2.0 ** -8 * (x.abs() @ w.abs().t()).amax(2) * sampling.repetition / sampling.temperature + 1e-5 * (1 + ref.abs())
    assert ((logp - ref).abs() <= bar).all()
    assert (logp - ref).abs().median() <= 1e-5 * (1 + ref.abs().max()), "few values lie at a rounding boundary"


def test_gradients_are_those_of_the_loss_of_the_adjusted_policy():
    """float32 throughout: a log-prob is held to 1e-5 (1 + |logp|), below 2e-4 here, which is the relative error of a token's
    weight and of a probability; the products' sums of up to 700 terms and the norm's add less than 1e-4.  Bar: 1e-3 of the
    gradient's norm.  No token's ratio is within 1e-3 of the clip range's ends."""
    V, P, new, S, G, clip = 700, 5, 12, 8, 4, 0.2
    policy, allowed, sampling = make(V, torch.float32)
    g = torch.Generator().manual_seed(8)
    prompts = torch.randint(0, V, (S, P), generator=g)
    answers = allowed.nonzero()[:, 0][torch.randint(0, int(allowed.sum()), (S, new), generator=g)]
    answers[:, 3:] = torch.where(torch.rand(S, new - 3, generator=g) < 0.3, answers[:, :1], answers[:, 3:])
    history = torch.cat((prompts, answers), 1)
    policy.version, rewards = 7, torch.randn(S, generator=g)
    versions = torch.randint(3, 8, (S * new,), generator=g, dtype=torch.int32)

    embed, gamma, head = (getattr(policy, k).cpu().double() for k in ("embed", "gamma", "head"))
    x = embed[history[:, P - 1:-1]].requires_grad_()
    gamma.requires_grad_(), head.requires_grad_()
    u = adjusted(normed(x, gamma) @ head.t(), history, P, sampling, allowed)
    logp = torch.log_softmax(u, 2).gather(2, answers[..., None])[..., 0]
    behav = (logp.detach() + 0.5 * torch.randn(S, new, generator=g)).float()
    age = (7 - versions.view(S, new)).clamp(min=1).double()
    prox = (behav.double() / age + (1 - 1 / age) * logp).detach()
    ratio, weight = (logp - prox).exp(), (prox - behav.double()).exp()
    r = rewards.double().view(-1, G)
    adv = ((r - r.mean(1, keepdim=True)) / (r.std(1, unbiased=False, keepdim=True) + 1e-6)).view(S, 1)
    assert ((ratio - 1).abs() - clip).abs().min() > 1e-3
    loss = -(weight * torch.minimum(ratio * adv, ratio.clamp(1 - clip, 1 + clip) * adv)).mean()
    loss.backward()

    got = example.gradients(policy, sampling, history.int().cuda(), behav.cuda(), versions.cuda(), rewards.cuda(), P, G, clip)
    assert abs(float(got["loss"]) - float(loss.detach())) <= 1e-3 * float((weight * ratio.detach() * adv.abs()).mean())
    for name, ref in (("dhidden", x.grad.view(S * new, -1)), ("dgamma", gamma.grad), ("dhead", head.grad)):
        assert ((got[name].cpu().double() - ref).norm() <= 1e-3 * ref.norm()), name


def test_reward_rises():
    shares = example.main(["--steps", "16", "--prompts", "8", "--new-tokens", "16"])
    assert sum(shares[-3:]) / 3 > sum(shares[:3]) / 3 + 0.1
