"""The operators that close the loop, together as the example uses them: a step of training from the gradients that the loss left to
the 4-bit head that the next rollout draws through."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2512_06547_amd import example

from test_gpu_adamw import a3po, reference  # noqa: E402, F401


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_from_gradients_to_the_next_head(a3po, bits):  # noqa: F811
    """Masters are those of AdamW in 64 bits on the gradients given (the bar of the step's own tests, the clip factor's five roundings
    in it), the model's weights their copies, and the 4-bit head that of the copies; the draws' log-probs agree with those of the
    adjusted policy that the loss is taken of (each to the library's 1e-5 (1 + |logp|))."""
    V, P, new, S, G = 300, 4, 6, 8, 4
    policy = example.new_policy(V, 64, torch.bfloat16, "cuda", seed=3)
    trainer = example.Trainer(policy, 0.01, bits, max_norm=0.05, weight_decay=0.1)
    sampling = example.Sampling()
    prompts = torch.randint(0, V, (S, P), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    history, logp = example.rollout(policy, sampling, prompts, new, 64, torch.Generator("cuda").manual_seed(2))
    assert history.min() >= 0 and history.max() < V and (logp <= 0).all()
    rewards = example.even_share(history, P)
    got = example.gradients(policy, sampling, history, logp, torch.zeros(S * new, dtype=torch.int32, device="cuda"), rewards, P, G)
    before = [m.clone() for m in trainer.master]
    embed = torch.zeros_like(before[0]).index_add_(0, got["source"], got["dhidden"].float())
    grads = [g.cpu() for g in (embed, got["dgamma"], got["dhead"].float())]
    norm = sum(float(g.double().square().sum()) for g in grads) ** 0.5
    assert norm > 0.05, "the step clips"
    trainer.step(policy, got)
    for name, m, p, g in zip(trainer.names, trainer.master, before, grads):
        zero = torch.zeros(p.shape, dtype=torch.float64)
        ref, _, _, bar, _, _ = reference(p.cpu(), g, zero, zero, 1, 0.05 / (norm + 1e-6), lr=0.01, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)
        # (adding up rows of the embedding's gradient has an order: elements whose sum nearly cancels may differ by more)
        off = (m.cpu().double() - ref).abs()
        assert (off <= bar + 1e-6 * 0.01).float().mean() > 0.999, name
        assert torch.equal(getattr(policy, name), m.bfloat16()), name
    codes, scales, zeros = example.quantize_w4(policy.head, 64)
    value = (torch.stack((codes & 15, codes >> 4), 2).view(V, -1, 64).float() - zeros[..., None].float()) * scales[..., None]
    assert ((value - policy.head.float().view(V, -1, 64)).abs() <= 1.001 * scales[..., None]).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_the_example_runs(bits):
    shares = example.main(["--steps", "3", "--prompts", "2", "--group", "4", "--new-tokens", "4", "--vocab", "200", "--hidden", "128", "--state-bits", str(bits)])
    assert len(shares) == 3 and all(0 <= s <= 1 for s in shares)
