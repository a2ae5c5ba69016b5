"""The calibration of the device model's launch overhead and memory bandwidth
on the operators of a single-token step: the fit on the CPU, the command on
the GPU."""
import json

import numpy as np
import pytest

from paper_2111_05426_amd import calibrate
from paper_2111_05426_amd.workloads import DeviceSpec


def test_fit_recovers_exact_constants():
    nbytes = np.array([1e3, 5e4, 1e6, 3e7, 2e9])
    (launch, rate), worst = calibrate.fit_roofline(nbytes, 7e-6 + nbytes / 5.1e12)
    assert abs(launch / 7e-6 - 1) < 1e-9 and abs(rate / 5.1e12 - 1) < 1e-9 and worst < 1e-9


def test_fit_keeps_constants_non_negative():
    nbytes = np.array([1e6, 2e6, 4e6])
    (launch, rate), _ = calibrate.fit_roofline(nbytes, np.array([1e-5, 1e-5, 1e-5]))
    assert launch > 0 and rate == np.inf
    (launch, rate), _ = calibrate.fit_roofline(nbytes, nbytes / 1e12 - 1e-7)
    assert launch == 0 and 0 < rate < np.inf


def test_shapes():
    s = calibrate.DECODE_SHAPES
    assert len(set(s)) == len(s) and all(h * d in (768, 1536) for _, _, h, d in s)


@pytest.mark.gpu
def test_command(tmp_path, capsys):
    """The command runs the three operators on every shape; its constants go
    into a device model that the library takes."""
    import torch

    from paper_2111_05426_amd import dsim
    from paper_2111_05426_amd.workloads import TINY_MLP
    path = tmp_path / "decode.json"
    assert calibrate.main(["--op", "decode", "--reps", "2", "--out", str(path)]) == 0
    printed, out = json.loads(capsys.readouterr().out), json.loads(path.read_text())
    assert printed["decode"] == out["decode"]
    assert {r["op"] for r in out["samples"]} == {"append", "attention", "logits"}
    assert len(out["samples"]) == 3 * len(calibrate.DECODE_SHAPES) and all(r["seconds"] > 0 for r in out["samples"])
    c = out["decode"]
    assert c["launch_s"] >= 0 and 1e9 < c["mem_bytes_per_s"] < 1e15
    device = DeviceSpec(launch_s=c["launch_s"], mem_bytes_per_s=c["mem_bytes_per_s"])
    strat = dsim.dsim_create_grid(TINY_MLP.model, TINY_MLP.grid)
    res = dsim.alloc_results(len(strat), int(strat[:, 2].max()))
    dsim.dsim_simulate_parametric(TINY_MLP.model, torch.from_numpy(strat).cuda(), device, res)
    assert bool((res["makespan"] > 0).all())
