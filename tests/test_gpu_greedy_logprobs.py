"""GPU: the LM head with log probabilities in the place of the greedy one -- the choice, its logit and the call's status are what
s4c_lm_head_greedy writes, in a call of its own and in the target's pass."""
import pytest
import torch

from parity import Guarded, dev
from test_gpu_logprobs_round import _pass

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,V", [(1, 1), (26, 4100), (128, 5001), (129, 5001), (517, 1001)])
@pytest.mark.parametrize("top", [0, 3, 8])
def test_what_the_greedy_head_writes(R, V, top):
    from paper_2506_14158_b200 import s4c

    g = torch.Generator(device="cuda").manual_seed(R + V)
    h = torch.randn(R, 128, generator=g, device="cuda").bfloat16()
    w = torch.randn(V, 128, generator=g, device="cuda").bfloat16()
    if R > 20:
        h[5] = float("nan")  # a row without a choice
        w[V // 3] = w[V // 2]  # ties
    want = s4c.lm_head_greedy(h, w)
    out = dict(choice=Guarded((R,), torch.int32, fill=-7), max_logit=Guarded((R,), torch.float32, fill=7.0),
               call_status=Guarded((1,), torch.int32, fill=77))
    for tok in (None, torch.full((R,), -1, dtype=torch.int32, device="cuda")):
        s4c.lm_head_logprobs(h, w, tok, 1.0, top, **{k: v.t for k, v in out.items()})
        torch.cuda.synchronize()
        for k, v in out.items():
            v.check(k)
        assert torch.equal(out["choice"].t, want["token"]) and torch.equal(out["max_logit"].t, want["max_logit"])
        assert out["call_status"].t.item() == 0 and want["status"].item() == 0


@pytest.mark.parametrize("top", [0, 5])
def test_the_pass_says_how_its_head_went(top):
    w, plain, tv, parent, tokens, cache_len, (B, T, V, L, md) = _pass(top, False)
    for p in (plain, tv):
        p.status_head.fill_(77), p.max_logit.fill_(float("nan"))
        p.forward(dev(tokens), dev(cache_len.copy()), dev(parent), max_cache_len=L)
    torch.cuda.synchronize()
    assert plain.status_head.item() == 0 and tv.status_head.item() == 0
    assert torch.equal(tv.max_logit, plain.max_logit)
