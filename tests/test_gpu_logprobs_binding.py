"""GPU: what the log-probability and distillation calls are to the program around them -- to autograd, the allocator, other streams and other threads."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def teacher(R, V, K, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, V, (R, K), generator=g, device="cuda", dtype=torch.int32), torch.randn(R, K, generator=g, device="cuda")


@pytest.mark.parametrize("backward", [False, True])
def test_a_gradient_in_the_place_of_saved_logits_is_refused_by_autograd(backward):
    """A soft cap saves its output; the gradient written over it must not be taken for it on the way back."""
    from paper_2506_14158_b200 import s4c

    def head():
        x = torch.randn(6, 301, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).requires_grad_(True)
        return x, 30 * torch.tanh(x / 30), torch.tanh(x / 30)

    def grad(z, out):
        if not backward:
            return s4c.distill_topk(z, *teacher(6, 301, 4), grad=out)["grad"]
        stats = s4c.distill_topk(z, *teacher(6, 301, 4))["stats"]
        return s4c.distill_topk_backward(z, *teacher(6, 301, 4), stats, torch.ones(6, device="cuda"), grad=None if out is True else out)

    x, z, _ = head()
    g = grad(z, True)
    z.backward(g)          # a gradient of its own: as ever
    want = x.grad
    x, z, _ = head()
    before = z._version
    g2 = grad(z, z.detach())
    assert z._version > before and torch.equal(g2, g)
    z.backward(g2)         # (the product saved no output: its logits may go)
    assert torch.equal(x.grad, want)
    x, _, capped = head()  # (tanh's own output)
    g3 = grad(capped, capped.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        capped.backward(g3)


def test_outputs_that_are_given_count_as_written():
    from paper_2506_14158_b200 import s4c

    R, V = 3, 40
    x, i = torch.randn(R, V, device="cuda"), torch.zeros(R, dtype=torch.int32, device="cuda")
    f, n = lambda *s: torch.empty(*s, device="cuda"), lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")
    out = dict(logprob=f(R), entropy=f(R), top_token=n(R, 2), top_logprob=f(R, 2), status=n(R))
    s4c.token_logprobs(x, i, 1.0, 2, **out)
    assert all(t._version == 1 for t in out.values()) and x._version == 0
    s4c.lm_head_logprobs(torch.zeros(R, 64, device="cuda").bfloat16(), torch.zeros(V, 64, device="cuda").bfloat16(), i, 1.0, 2, **out,
                         choice=(c := n(R)), max_logit=(m := f(R)), call_status=(s := n(1)))
    assert all(t._version == 2 for t in out.values()) and c._version == m._version == s._version == 1
    d = dict(loss=f(R), stats=f(R, 4), status=n(R), grad=f(R, V))
    s4c.distill_topk(x, *teacher(R, V, 3), **d)
    assert all(t._version == 1 for t in d.values()) and x._version == 0
    with torch.inference_mode():
        y, out = torch.randn(R, V, device="cuda"), dict(logprob=f(R), entropy=f(R), status=n(R))
    s4c.token_logprobs(y, i, **out)
    s4c.distill_topk(y, *teacher(R, V, 3), grad=y)
    torch.cuda.synchronize()
    assert torch.isfinite(out["logprob"]).all()


CALLS = ["token_logprobs", "tree_logprobs", "lm_head_logprobs", "distill_topk", "distill_topk_backward"]


@pytest.mark.parametrize("call", CALLS)
def test_outputs_made_for_another_stream_are_that_streams(call):
    """A tensor of the current stream is given back with work on its way into it; a call on another stream, which does not wait for that work, makes
    outputs of the same sizes: none of them may lie there."""
    from paper_2506_14158_b200 import s4c

    R, V = 2000, 33
    x, i = torch.randn(R, V, device="cuda"), torch.zeros(R, dtype=torch.int32, device="cuda")
    tok, val = teacher(R, V, 3)
    h, w = torch.randn(R, 64, device="cuda").bfloat16(), torch.randn(V, 64, device="cuda").bfloat16()
    t4 = torch.zeros(20, 100, dtype=torch.int32, device="cuda")
    paths = torch.full((20, 100), -1, dtype=torch.int32, device="cuda")
    paths[:, 0] = 0
    zero = torch.zeros(20, dtype=torch.int32, device="cuda")
    st, scale = s4c.distill_topk(x, tok, val)["stats"], torch.ones(R, device="cuda")
    run = {
        "token_logprobs": lambda s: s4c.token_logprobs(x, i, 1.0, 2, stream=s),
        "tree_logprobs": lambda s: s4c.tree_logprobs(x.view(20, 100, V), t4, paths, zero, zero, 1.0, 2, stream=s),
        "lm_head_logprobs": lambda s: s4c.lm_head_logprobs(h, w, i, 1.0, 2, stream=s),
        "distill_topk": lambda s: s4c.distill_topk(x, tok, val, grad=True, stream=s),
        "distill_topk_backward": lambda s: dict(grad=s4c.distill_topk_backward(x, tok, val, st, scale, stream=s)),
    }[call]
    want = {k: v.clone() for k, v in run(None).items() if v is not None}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    victims = [torch.empty_like(v) for v in want.values() for _ in range(3)]
    torch.cuda._sleep(100_000_000)  # (about 50 ms in front of the writes below)
    for v in victims:
        v.fill_(9)
    del v, victims
    got = run(side)
    side.synchronize()
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(got[k], want[k]), k


def test_calls_of_different_sizes_from_several_threads():
    """Kept rows of 35 KB and of 131 KB a block by one kernel, whose limit of shared memory is the kernel's, not the call's.  Through the C ABI, whose
    calls run side by side."""
    import ctypes

    from paper_2506_14158_b200 import s4c
    from paper_2506_14158_b200._build import lib_path

    fn = ctypes.CDLL(lib_path()).s4c_distill_topk
    vp, i, f, ll = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_longlong
    fn.argtypes = [vp, ll, vp, vp, i, vp, i, i, i, f, f, f, vp, vp, vp, vp, ll, vp, vp]
    p = lambda t: vp(t.data_ptr())
    codes, start, rows, keep = [], threading.Barrier(6), [], []
    for V in (262144, 70000) * 3:
        x, grad, loss, stats = torch.randn(1, V, device="cuda"), torch.empty(1, V, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, 4, device="cuda")
        tok, val = teacher(1, V, 3)
        want = s4c.distill_topk(x, tok, val, grad=True)
        stream = torch.cuda.Stream()
        args = (p(x), ll(V), p(tok), p(val), i(3), None, i(1), i(V), i(0), f(1.0), f(1.0), f(1.0), p(loss), p(stats), None, p(grad), ll(V), None, vp(stream.cuda_stream))
        rows.append((args, want["loss"], loss, want["grad"], grad))
        keep.append((x, stats, tok, val, stream))
    torch.cuda.synchronize()

    def calls(args):
        start.wait()
        for _ in range(400):
            codes.append(fn(*args))

    threads = [threading.Thread(target=calls, args=(r[0],)) for r in rows]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert len(codes) == 2400 and codes.count(0) == 2400, codes.count(7)
    for _, want, loss, want_grad, grad in rows:
        assert torch.equal(want, loss) and torch.equal(want_grad, grad)


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="a workspace on another device takes two")
def test_a_workspace_on_another_device_is_refused():
    from paper_2506_14158_b200 import s4c

    h, w = torch.zeros(4, 64, device="cuda:0").bfloat16(), torch.zeros(100, 64, device="cuda:0").bfloat16()
    ws = torch.empty(s4c.lm_head_logprobs_workspace_bytes(4, 100, 64, 2), dtype=torch.uint8, device="cuda:1")
    with pytest.raises(ValueError, match="workspace is on cuda:1"):
        s4c.lm_head_logprobs(h, w, None, 1.0, 2, workspace=ws)


@pytest.mark.parametrize("call", ["token_logprobs", "lm_head_logprobs", "distill_topk"])
def test_a_captured_call_on_a_named_stream_makes_the_graphs_memory(call):
    """Outputs and workspaces made under capture, on the capturing stream given by name, and on one that was forked from it, live in the graph."""
    from paper_2506_14158_b200 import s4c

    R, V = 50, 3001
    x, i = torch.randn(R, V, device="cuda"), torch.zeros(R, dtype=torch.int32, device="cuda")
    h, w = torch.randn(R, 64, device="cuda").bfloat16(), torch.randn(V, 64, device="cuda").bfloat16()
    tok, val = teacher(R, V, 3)
    run = {"token_logprobs": lambda s: s4c.token_logprobs(x, i, 1.0, 2, stream=s), "lm_head_logprobs": lambda s: s4c.lm_head_logprobs(h, w, i, 1.0, 2, stream=s),
           "distill_topk": lambda s: s4c.distill_topk(x, tok, val, grad=True, stream=s)}[call]
    run(None)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        here = torch.cuda.current_stream()
        a = run(here)
        side.wait_stream(here)
        b = run(side)
        here.wait_stream(side)
    others = [torch.full((R, V), 9.0, device="cuda") for _ in range(8)] + [torch.full((R,), 9, device="cuda") for _ in range(64)]
    for t in (x, h):
        t.copy_(torch.randn_like(t))
    graph.replay()
    torch.cuda.synchronize()
    want = run(None)
    assert all((t == 9).all() for t in others)
    for k, v in want.items():
        if v is not None:
            assert torch.equal(a[k], v) and torch.equal(b[k], v), k
