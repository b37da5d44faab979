"""GPU: every column of a row is counted once in the softmax statistics, in every place where it can lie -- the first and the last of a tile, of a run of
32, of the remainder behind the last whole run or vector, of each group of epilogue warps, of each block's share.

The columns are dealt out to the rows at random: a column has mass (logits 0, -1/2, -1, -3/2) in exactly one row and lies 200 below in all others, where
its term is 0 in float32.  A row's sum is then that of its n columns, a column left out or counted twice moves it by more than
e^-1.5 / n relative, and n is small.

Tolerance: of tests/test_gpu_logprobs.py's bound of a sum, S_TOL(V) = 2^-24 (V / 128 + 64) + 2^-22 + 2.1 (24 + log2 V) 2^-24 with V / 128 additions on the
longest chain, the n terms that are not 0 make at most n roundings whatever the order: S_TOL at V = 128 n.  (n = 250: 2.4e-5, against the
8.9e-4 of one column.)"""
import math

import numpy as np
import pytest
import torch

import oracle

from test_gpu_logprobs import TYPES, s_tol

pytestmark = pytest.mark.gpu


def deal(R, V):
    """logits [R,V] float64, the rows' numbers of columns, one column of each row, and the columns' order of the lowest bits"""
    rng = np.random.default_rng(R * 1000 + V)
    owner = rng.permutation(np.arange(V) % R)
    x = np.full((R, V), -200.0)
    x[owner, np.arange(V)] = -0.5 * (rng.integers(0, 4, V))
    first = np.array([np.flatnonzero(owner == r)[rng.integers(0, (owner == r).sum())] for r in range(R)])
    for r in range(R):  # (the maximum is 0 in every row, so that a term is what it says)
        x[r, first[r]] = 0.0
    return x, np.bincount(owner, minlength=R), first.astype(np.int32)


def compare(got, x, n, tok, rows=slice(None)):
    want = oracle.token_logprobs(x[rows], tok[rows], 1.0, 0)
    tol = np.array([s_tol(128 * m) for m in n[rows]])
    miss = math.exp(-1.5) / n[rows]
    assert (4 * tol < miss).all(), "the case cannot tell a missing column"  # (which moves ln S, and so logprob, by `miss`)
    lp, h = got["logprob"].double().cpu().numpy(), got["entropy"].double().cpu().numpy()
    assert (got["status"] == 0).all()
    assert (np.abs(lp - want["logprob"]) <= tol + 2.0 ** -22 * np.abs(want["logprob"])).all(), np.abs(lp - want["logprob"]).max()
    assert (np.abs(h - want["entropy"]) <= tol * (1 + 2 * want["entropy"])).all(), np.abs(h - want["entropy"]).max()


@pytest.mark.parametrize("R,V,top", [(26, 1001, 0), (26, 4100, 5), (64, 7003, 8), (100, 9001, 3), (128, 5001, 8), (128, 20003, 0), (129, 5001, 1), (256, 20000, 8),
                                     (256, 40007, 5), (300, 40000, 0), (96, 32000, 5), (120, 128256 // 4, 8)])
def test_the_lm_head_counts_every_column_once(R, V, top):
    """States that are rows of the unit matrix: logits[r, v] = weight[v, r]."""
    from paper_2506_14158_b200 import s4c

    x, n, tok = deal(R, V)
    H = (R + 63) // 64 * 64
    h, w = torch.zeros(R, H, dtype=torch.bfloat16), torch.zeros(V, H, dtype=torch.bfloat16)
    h[torch.arange(R), torch.arange(R)] = 1
    w[:, :R] = torch.from_numpy(x.T.copy()).to(torch.bfloat16)
    got = s4c.lm_head_logprobs(h.cuda(), w.cuda(), torch.from_numpy(tok).cuda(), 1.0, top)
    compare(got, x, n, tok)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,V,top,off", [(150, 700, 5, 0), (200, 3001, 5, 1), (200, 6000, 0, 3), (157, 16384, 20, 0), (300, 50001, 5, 1), (400, 100003, 0, 5)])
def test_rows_count_every_column_once(dtype, R, V, top, off):
    """All rows in one call, and some of them in calls of one and of three, which share a row out to several blocks."""
    from paper_2506_14158_b200 import s4c

    x, n, tok = deal(R, V)
    buf = torch.zeros(off + R * V, dtype=TYPES[dtype], device="cuda")
    d = buf[off:].view(R, V)
    d.copy_(torch.from_numpy(x))
    t = torch.from_numpy(tok).cuda()
    compare(s4c.token_logprobs(d, t, 1.0, top), x, n, tok)
    for r in list(range(0, R - 3, R // 6)) + [R - 3]:
        for rows in (slice(r, r + 1), slice(r, r + 3)):
            compare(s4c.token_logprobs(d[rows], t[rows], 1.0, top), x, n, tok, rows)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,V,off", [(150, 700, 0), (200, 3001, 1), (157, 16384, 0), (300, 50001, 1), (400, 100003, 5)])
def test_distillation_counts_every_column_once(dtype, R, V, off):
    """A label's loss is -ln p1, a single teacher entry's tau^2 (-ln p): with the gradient (rows kept) and without (rows streamed)."""
    from paper_2506_14158_b200 import s4c

    x, n, tok = deal(R, V)
    buf = torch.zeros(off + R * V, dtype=TYPES[dtype], device="cuda")
    d = buf[off:].view(R, V)
    d.copy_(torch.from_numpy(x))
    t, zero = torch.from_numpy(tok).cuda(), torch.zeros(R, 1, device="cuda")
    tol = np.array([s_tol(128 * m) for m in n])
    for rows in (slice(0, R), slice(1, 2), slice(R - 3, R)):
        for tau in (1.0, 2.0, 0.7):
            y = x[rows] / float(np.float32(tau))  # (at tau = 2 a term of the others is e^-100, 0 in float32 too)
            own = np.arange(R)[rows]
            lse = np.log(np.exp(y).sum(1))
            want_teacher = float(np.float32(tau)) ** 2 * (lse - x[own, tok[rows]] / float(np.float32(tau)))
            want_label = np.log(np.exp(x[rows]).sum(1)) - x[own, tok[rows]]
            for grad in (None, True):
                a = s4c.distill_topk(d[rows], t[rows].view(-1, 1), zero[rows], None, tau, 1.0, 0.0, grad=grad)["loss"].double().cpu().numpy()
                b = s4c.distill_topk(d[rows], None, None, t[rows], tau, 0.0, 1.0, grad=grad)["loss"].double().cpu().numpy()
                both = s4c.distill_topk(d[rows], t[rows].view(-1, 1), zero[rows], t[rows], tau, 1.0, 1.0, grad=grad)["loss"].double().cpu().numpy()
                lim = lambda w, s: s * tol[rows] + 2.0 ** -22 * np.abs(w)
                assert (np.abs(a - want_teacher) <= lim(want_teacher, tau ** 2)).all()
                assert (np.abs(b - want_label) <= lim(want_label, 1)).all()
                assert (np.abs(both - want_teacher - want_label) <= lim(want_teacher + want_label, 1 + tau ** 2)).all()
