"""What the example does with a policy that leaves no token to draw: it says so, where a token of -1 would be an index later on."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2512_06547_amd import example


@pytest.mark.parametrize("how", ["mask", "weights", "one row's weights"])
def test_a_rollout_without_a_token_to_draw_is_refused(how):
    V, P, S = 200, 4, 6
    policy = example.new_policy(V, 64, torch.bfloat16, "cuda", seed=3)
    sampling = example.Sampling()
    prompts = torch.arange(S * P, dtype=torch.int32, device="cuda").view(S, P)
    if how == "mask":
        sampling.allowed = torch.zeros((V + 31) // 32, dtype=torch.int32, device="cuda")
    elif how == "weights":
        policy.gamma[5] = float("nan")
    else:
        policy.embed[int(prompts[2, -1])] = float("nan")
    with pytest.raises(ValueError, match="no token"):
        example.rollout(policy, sampling, prompts, 3, 64, torch.Generator("cuda").manual_seed(2))


def test_a_mask_that_leaves_one_token():
    V, P, S = 200, 4, 6
    policy = example.new_policy(V, 64, torch.bfloat16, "cuda", seed=3)
    allowed = torch.zeros((V + 31) // 32, dtype=torch.int32, device="cuda")
    allowed[3] = 1 << 7
    history, logp = example.rollout(policy, example.Sampling(allowed=allowed), torch.zeros(S, P, dtype=torch.int32, device="cuda"), 3, 64)
    assert (history[:, P:] == 103).all() and (logp.abs() <= 2.0 ** -36).all()
