"""Host-side checks of the calibration command's training options: they reach the decoder stack, or are refused."""
import sys

import pytest
import torch

from paper_2608_01847_amd import calib
from test_calib_arguments import run  # noqa: F401  (fixture)


def test_decoder_stack_takes_them(run):  # noqa: F811
    seen, out = run("--variants", "crs_dgs", "--loss", "ce", "--post-norm", "--max-grad-norm", "0.5")
    assert (seen[0]["loss"], seen[0]["post_norm"], seen[0]["max_grad_norm"]) == ("ce", True, 0.5)
    assert (out["loss"], out["post_norm"], out["max_grad_norm"]) == ("ce", True, 0.5)
    seen, out = run("--variants", "crs_dgs")
    assert (seen[0]["loss"], seen[0]["post_norm"], seen[0]["max_grad_norm"]) == ("kl_top", False, None)


@pytest.mark.parametrize("args", [("--max-grad-norm", "0"), ("--max-grad-norm", "-1"), ("--max-grad-norm", "nan"), ("--loss", "mse")])
def test_values_that_are_none(run, args):  # noqa: F811
    with pytest.raises(SystemExit) as e:
        run(*args)
    assert e.value.code == 2


@pytest.mark.parametrize("args", [("--loss", "ce"), ("--post-norm",), ("--max-grad-norm", "1.0")])
@pytest.mark.parametrize("other", [(), ("--kl-top-stack",)])
def test_other_loops_refuse_them(monkeypatch, args, other):
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(sys, "argv", ["calib", *other, *args])
    with pytest.raises(SystemExit) as e:
        calib.main()
    assert e.value.code == 2


def test_unknown_loss():
    with pytest.raises(ValueError):
        calib.DecoderStack(0, "crs_dgs", loss="mse", device="cpu")
