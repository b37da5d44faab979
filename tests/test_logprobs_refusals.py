"""What the verify pass and step refuse of log probabilities when they are asked for, not when they run (no GPU needed)."""
import pytest


def test_a_pass_refuses_alternatives_that_its_route_has_not(s4c_lib):
    from paper_2506_14158_b200 import target

    for top, stochastic in [(9, False), (20, False), (-1, False), (65, True), (-1, True)]:
        with pytest.raises(ValueError, match="top_logprobs must be 0 to 8"):
            target.TargetVerify(None, 1, 8, 4, 2, 64, 64, [], [], 4, stochastic=stochastic, top_logprobs=top)
    one = object.__new__(target.TargetVerify)
    one.top_logprobs = 20
    with pytest.raises(ValueError, match="at most 8 alternatives"):
        one.forward(None, None, None, temperature=0.0)


def test_a_step_refuses_what_its_run_would(s4c_lib):
    from paper_2506_14158_b200.verify import VerifyStep

    step = object.__new__(VerifyStep)
    for kw in (dict(top=65), dict(top=-1), dict(top=3, temperature=0.0), dict(top=3, temperature=float("inf")), dict(top=3, temperature=float("nan"))):
        with pytest.raises(ValueError):
            step.set_logprobs(**kw)
    assert not vars(step)


def test_a_gradient_whose_weight_leaves_float32_is_refused(s4c_lib):
    """The gradient's coefficient is teacher_weight temperature: beyond float32 every entry would be infinite or NaN."""
    from test_abi_logprobs import P, _entry

    far = 1 << 30
    fwd = _entry(s4c_lib, "s4c_distill_topk", [("x", P), ("ld", 100), ("tt", P), ("tl", P), ("K", 8), ("c", None), ("R", 3), ("V", 100), ("dt", 0),
                                            ("tau", 1e10), ("wt", 1e30), ("wl", 1.0), ("loss", P), ("stats", None), ("g", None), ("grad", far), ("gld", 100),
                                            ("st", None), ("s", None)])
    bwd = _entry(s4c_lib, "s4c_distill_topk_backward", [("x", P), ("ld", 100), ("tt", P), ("tl", P), ("K", 8), ("c", None), ("R", 3), ("V", 100), ("dt", 0),
                                                     ("tau", 1e10), ("wt", -1e30), ("wl", 1.0), ("stats", P), ("g", P), ("grad", far), ("gld", 100), ("s", None)])
    assert fwd() == 2 and bwd() == 2 and fwd(wt=-1e30) == 2
