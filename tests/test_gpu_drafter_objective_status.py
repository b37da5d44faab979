"""GPU: a drafter head's objective leaves the status of the head's forward pass as it was and has one of its own."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_the_forward_passes_status_outlives_the_objective():
    from paper_2506_14158_b200 import drafter, s4c

    B, T, V, K = 2, 3, 1000, 4
    head = drafter.DrafterHead(drafter.random_weights(V, 256, 4, 2, 64, 384, "cuda", seed=3), B, T, 4, 2, 64, 64, k=2, train=True)
    i32 = dict(dtype=torch.int32, device="cuda")
    kc, vc = (torch.randn(B, 2, 64, 64, device="cuda").bfloat16() for _ in range(2))
    head.forward(torch.ones(B, T, **i32), torch.randn(B * T, 256, device="cuda").bfloat16(), torch.full((B,), 5, **i32),
                 torch.tensor([[-1, 0, 0]] * B, **i32), kc, vc)
    head.status_head.fill_(s4c.SEQ_TIMEOUT)  # as the forward pass would have left it had a wait of its LM head run out
    head.status_logits.fill_(77)
    out = head.objective(torch.randint(0, V, (B * T, K), **i32), torch.randn(B * T, K, device="cuda"))
    torch.cuda.synchronize()
    assert head.status_head.item() == s4c.SEQ_TIMEOUT
    assert out["status_logits"].item() == 0 and (out["status"] == 0).all() and torch.isfinite(out["loss"]).all()
