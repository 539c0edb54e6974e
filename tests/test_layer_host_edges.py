"""Refusals of the package's calls around the attention memory (no GPU: nothing is launched)."""
import pytest
import torch
from torch.autograd import forward_ad


def test_tangents_are_refused():
    import paper_1609_01882_amd as psc
    x, w = torch.zeros((2, 1, 8)), torch.ones(8)
    rope = psc.Rotary(8, device="cpu")
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))  # noqa: E731
        for call in (lambda: rope(dual(x)), lambda: rope(x, out=dual(x)), lambda: rope.inverse(dual(x)), lambda: psc.residual_norm(dual(x), before=w),
                     lambda: psc.residual_norm(x, dual(x), before=w), lambda: psc.residual_norm(x, before=dual(w)), lambda: psc.residual_norm(x, x, after=dual(w)),
                     lambda: psc.residual_norm(x, x, gate=dual(x))):
            with pytest.raises(psc.PscError, match="tangent"):
                call()
            with torch.no_grad(), pytest.raises(psc.PscError, match="tangent"):     # (which leaves tangents as they are)
                call()
        with pytest.raises(psc.PscError, match="tangent"):
            rope(dual(x).requires_grad_())
        # others are not meant: host tensors are refused for what they are
        with pytest.raises(psc.PscError, match="CUDA"):
            psc.residual_norm(x, before=w)


def test_assembly_that_writes_m0_says_so():
    import glob
    import os
    import re
    import paper_1609_01882_amd as psc
    source, found = os.path.join(os.path.dirname(psc.__file__), "csrc"), 0
    for name in glob.glob(os.path.join(source, "*")):
        with open(name) as f:
            text = f.read()
        for statement in re.findall(r"\basm\b[^;]*;", text):
            if re.search(r"s_mov_b32 m0", statement):
                found += 1
                assert statement.count('"m0"') == 1, (os.path.basename(name), statement)
    assert found >= 2


def test_factors_that_32_bits_do_not_hold():
    import paper_1609_01882_amd as psc
    assert psc.Rotary(8, factor=-3.4e38, device="cpu").factor == -3.4e38
    for factor in (3.5e38, -1e39, float("inf"), float("nan")):
        with pytest.raises(psc.PscError):
            psc.Rotary(8, factor=factor, device="cpu")
