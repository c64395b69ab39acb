"""Host-side checks of the calibration command: what it is asked for reaches the loop, or is refused."""
import json
import sys

import pytest
import torch

from paper_2608_01847_amd import calib


@pytest.fixture()
def run(monkeypatch, capsys):
    seen = []

    def epoch(fmt, variant, steps, **kw):
        seen.append({"fmt": fmt, "variant": variant, "steps": steps, **kw})
        return {"eval_before": {}, "eval_after": {}, "train_curve": [1.0, 0.5], "seconds": 1.0}

    monkeypatch.setattr(calib, "decoder_epoch", epoch)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)

    def go(*args):
        monkeypatch.setattr(sys, "argv", ["calib", "--decoder-stack", *args])
        seen.clear()
        calib.main()
        return list(seen), json.loads(capsys.readouterr().out)

    return go


def test_decoder_stack_takes_its_arguments(run):
    seen, out = run("--variants", "rtn,crs_dgs", "--steps", "3", "--vocab", "5000", "--x-kind", "student_t3",
                    "--workload", "block8192_mxfp4")
    assert [s["variant"] for s in seen] == ["rtn", "crs_dgs"] and out["x_kind"] == "student_t3"
    for s in seen:
        assert (s["steps"], s["vocab"], s["x_kind"], s["hidden"], s["heads"]) == (3, 5000, "student_t3", 8192, (64, 8))
    seen, out = run("--variants", "rtn")
    assert seen[0]["x_kind"] == out["x_kind"] == "lowrank"


@pytest.mark.parametrize("args", [("--tokens", "512"), ("--eval-tokens", "512"), ("--kl-top-stack",),
                                  ("--workload", "linear256_mxfp4_f32")])
def test_decoder_stack_refuses_what_it_would_not_use(run, args):
    with pytest.raises(SystemExit) as e:
        run(*args)
    assert e.value.code == 2
