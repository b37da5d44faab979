"""GPU parity: log probabilities at every temperature that the header allows, against the float64 oracle: from 4.3e-39 (1.45 / temperature is just
finite) to float32's greatest value, with logits masked by -inf and by the type's lowest value, and logits up to the type's own ends.

Tolerance: tests/test_gpu_logprobs.py's (an exponent's roundings are relative to it at any temperature)."""
import numpy as np
import pytest
import torch

import oracle

from test_gpu_logprobs import TYPES, check, run

pytestmark = pytest.mark.gpu
TEMPERATURES = [4.3e-39, 1e-38, 1.6e-38, 3e-31, 1e-30, 2e-30, 1e-5, 1e18, 7e29, 1.4e30, 1.5e30, 2.5e36, 3e36, 1e38, 1.3e38, 3.4e38, 3.4028234e38]


def rows(V, dtype):
    rng = np.random.default_rng(V)
    base = rng.standard_normal(V).astype(np.float32) * 3
    n = np.arange(V)
    ends = float(torch.finfo(TYPES[dtype]).max)
    return np.stack([
        base,
        np.where(rng.random(V) < 0.5, -np.inf, base),
        np.where(n == V // 2, 1.0, -np.inf),
        np.where(rng.random(V) < 0.5, -ends, base),
        np.where(n % 3 == 0, 0.0, -1.0),                         # the maximum 0, met several times
        np.where(n % 5 == 0, -0.0, -np.inf),
        np.where(n % 3 == 0, ends, -ends),                       # differences that leave float32
        np.where(n % 3 == 0, ends, np.where(n % 3 == 1, -np.inf, ends / 2)),
        np.where(n % 2 == 0, -ends, -np.inf),
        np.where(n % 7 == 0, np.nan, base),
        np.full(V, -np.inf)]).astype(np.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [3, 97, 5001, 40003])
@pytest.mark.parametrize("many", [False, True])
def test_rows_at_the_ends_of_the_temperatures(dtype, V, many):
    x = torch.from_numpy(rows(V, dtype)).to(TYPES[dtype])
    if many and V <= 5001:  # more rows than SMs: other thread counts serve a row
        x = x.repeat(15, 1)
    elif many:
        x = x[:3]           # few long rows: by clusters
    tok = np.arange(x.shape[0]) * 7 % V
    for tau in TEMPERATURES:
        tau = float(np.float32(tau))
        got = run(x.cuda(), tok, tau, 5)
        check(got, oracle.token_logprobs(x.double().numpy(), tok, tau, 5), V, 5)


def test_a_walk_at_the_ends_of_the_temperatures():
    from paper_2506_14158_b200 import s4c

    V = 5001
    x = torch.from_numpy(rows(V, "f32"))[:9].view(1, 9, V)
    tokens = np.arange(9, dtype=np.int32)[None] * 11
    path, accept_len, next_token = np.arange(9, dtype=np.int32)[None], np.array([8], np.int32), np.array([5], np.int32)
    d = lambda a: torch.from_numpy(a).cuda()
    emitted = np.concatenate([tokens[0, 1:], next_token])
    for tau in TEMPERATURES:
        tau = float(np.float32(tau))
        got = s4c.tree_logprobs(x.cuda(), d(tokens), d(path), d(accept_len), d(next_token), tau, 4)
        check({k: v[0] for k, v in got.items()}, oracle.token_logprobs(x[0].double().numpy(), emitted, tau, 4), V, 4)


@pytest.mark.parametrize("R,V", [(3, 1), (26, 1000), (26, 4101), (130, 4101)])
def test_the_lm_head_at_the_ends_of_the_temperatures(R, V):
    """States of one 1 each, so that logits[r, v] = weight[v, r % 64] exactly: the columns' values are those of the rows above."""
    from paper_2506_14158_b200 import s4c

    H = 64
    h = torch.zeros(R, H, dtype=torch.bfloat16)
    h[torch.arange(R), torch.arange(R) % H] = 1
    kinds = rows(V, "bf16")[[0, 3, 4, 6, 8]]  # (infinities and NaN of one column would meet the zeros of every state)
    w = torch.from_numpy(kinds[np.arange(H) % len(kinds)].T.copy()).to(torch.bfloat16)
    masked = np.isneginf(w.double().numpy())
    w[torch.from_numpy(masked)] = 0.0
    h[:, H - 1], w[:, H - 1] = 1, 0.0
    if V > 2:
        w[V // 2:V // 2 + V // 8, H - 1] = -np.inf  # masked for every row: the maximum is elsewhere
    x = w[:, :H - 1].double().numpy()[:, np.arange(R) % H % (H - 1)].T.copy()
    x[np.arange(R) % H == H - 1] = 0.0
    if V > 2:
        x[:, V // 2:V // 2 + V // 8] = -np.inf
    tok = (np.arange(R) * 7 % V).astype(np.int32)
    for tau in TEMPERATURES:
        tau = float(np.float32(tau))
        got = s4c.lm_head_logprobs(h.cuda(), w.cuda(), torch.from_numpy(tok).cuda(), tau, 5)
        check(got, oracle.token_logprobs(x, tok, tau, 5), V, 5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [97, 5001, 70001])
def test_masks_of_both_kinds_around_one_token(dtype, V):
    """Threads that meet nothing but -inf and the type's lowest value, beside the one that has the row's maximum."""
    n, low = np.arange(V), float(torch.finfo(TYPES[dtype]).min)
    mixed = np.where(n % 2 == 0, low, -np.inf)
    x = np.stack([np.where(n == 1, 0.0, mixed), np.where(n == V - 1, -3.0, mixed), np.where(n == V // 2, 1e36, mixed), np.where(n == 3, -1e36, mixed)])
    x = torch.from_numpy(x.astype(np.float32)).to(TYPES[dtype])
    tok = np.array([1, 2, V // 2, 0])
    for tau in (0.5, 1.0, 2.0, 100.0, 1e20, 1e29, 2e30, 3e38):
        tau = float(np.float32(tau))
        check(run(x.cuda(), tok, tau, 3), oracle.token_logprobs(x.double().numpy(), tok, tau, 3), V, 3)
