"""The failure path of the LM head with log probabilities, exercised without any GPU fault: s4c_selftest_lm_head_timeout runs the real launch with the
hidden states of one vocabulary tile never requested.  The products' wait for them runs out (200 ms), every role of that CTA leaves its loop, and
the call must return normally, flagged, with nothing that the workspace held before in its outputs, and leave the stream fit for the next call."""
import numpy as np
import pytest
import torch

from test_gpu_lm_head_logprobs import grid, logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,V,H,top,tile", [
    (26, 60, 128, 4, 0),         # one tile: nothing is computed
    (26, 100, 128, 4, 0),        # two tiles
    (26, 32000, 1024, 8, 5),     # a CTA's only tile
    (3, 40000, 64, 0, 148 + 3),  # a CTA's second tile, fewer slices than stages
    (128, 40000, 2048, 8, 2),    # a CTA's first tile of several, more slices than stages
    (256, 40000, 1024, 5, 148 + 7),
])
def test_a_wait_that_runs_out_ends_the_call_cleanly(R, V, H, top, tile):
    from paper_2506_14158_b200 import s4c

    rng = np.random.default_rng(R + V)
    h, w = grid(rng, R, V, H)
    x = logits(h, w)
    h, w = h.cuda(), w.cuda()
    i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.float32, device="cuda")
    out = dict(entropy=torch.zeros(R, **f32), top_token=torch.full((R, top), 7, **i32), top_logprob=torch.zeros(R, top, **f32),
               choice=torch.full((R,), 7, **i32), max_logit=torch.zeros(R, **f32), status=torch.zeros(R, **i32), call_status=torch.full((1,), 64, **i32))
    ws = torch.full((s4c.lm_head_logprobs_workspace_bytes(R, V, H, top),), 0x7F, dtype=torch.uint8, device="cuda")  # logits of 3.39e38, tokens of 2^31
    s4c.selftest_lm_head_timeout(h, w, *[out[k] for k in ("entropy", "top_token", "top_logprob", "choice", "max_logit", "status", "call_status")], ws, tile)
    torch.cuda.synchronize()  # returns: nothing hung, no error is pending
    got = {k: v.cpu().numpy() for k, v in out.items()}
    assert got["call_status"][0] == s4c.SEQ_TIMEOUT and (got["status"] & s4c.SEQ_TIMEOUT).all()
    assert np.isnan(got["entropy"]).all() and (got["top_token"] == -1).all() and np.isneginf(got["top_logprob"]).all()
    n = 148  # the CTAs of a launch, one per SM: all tiles but those of the one that gave up are there
    if V < 64:
        assert (got["choice"] == -1).all() and np.isneginf(got["max_logit"]).all()
    else:
        widths = [128] if R > 128 else range(64, 257, 32)
        bn = min(widths, key=lambda b: (-(-(-(-V // b)) // n) * b, -b))  # the tile's width, as the launch chooses it
        others = np.arange(V) // bn % n != tile % n
        best = np.where(others, x, -np.inf).max(1)
        c = got["choice"]
        assert ((c >= 0) & (c < V)).all()
        np.testing.assert_array_equal(got["max_logit"], x[np.arange(R), c])
        assert (got["max_logit"] >= best).all()
    # the same stream, the same workspace, right away: an ordinary call
    o = s4c.lm_head_logprobs(h, w, None, 1.0, top, choice=out["choice"], max_logit=out["max_logit"], call_status=out["call_status"], workspace=ws)
    want = s4c.lm_head_greedy(h, w)
    torch.cuda.synchronize()
    assert out["call_status"].item() == 0 and (o["status"] == 0).all()
    assert torch.equal(out["choice"], want["token"]) and torch.equal(out["max_logit"], want["max_logit"])
    np.testing.assert_array_equal(out["max_logit"].cpu().numpy(), x.max(1))
