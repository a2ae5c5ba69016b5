"""The calibration on the operators of a single-token step reads from memory:
the timed calls' tensors, on the CPU with the operators replaced; what the
command fits, on the GPU."""
import json

import pytest
import torch

from paper_2111_05426_amd import calibrate, ops


def test_copies():
    cache = calibrate.LAST_LEVEL_CACHE
    for nbytes in (1, 1000, 10 ** 6, 10 ** 8, cache - 1, cache, 2 * cache, 2 * cache + 1, 10 ** 10):
        for reps in (1, 2, 20, 1000):
            n = calibrate._copies(nbytes, reps)
            # a call for itself, or two caches' worth of other calls' tensors since the last use
            assert 1 <= n <= reps and (n == reps or (n - 1) * nbytes >= 2 * cache)


@pytest.mark.parametrize("shape,reps", [((2, 64, 2, 32), 7), ((3, 100, 2, 16), 40), ((1, 16, 1, 64), 50)])
def test_timed_calls_share_no_tensors(monkeypatch, shape, reps):
    """With a last-level cache of 64 KB."""
    monkeypatch.setattr(calibrate, "LAST_LEVEL_CACHE", 1 << 16)
    monkeypatch.setattr(calibrate, "DECODE_VOCAB", 101)
    touched = []

    def rows(t):
        return {(t.data_ptr(), t.numel() * t.element_size())}

    def places(cache, table, positions):
        page = calibrate.DECODE_PAGE
        return {(cache["k"].data_ptr(), int(table[b, p // page]) * page + p % page)
                for b, ps in enumerate(positions) for p in ps}
    monkeypatch.setattr(ops, "dsim_kv_append", lambda cache, table, k, v, seq, pos, rope, q, q_out: touched.append(
        rows(k) | rows(v) | rows(q) | rows(q_out) | places(cache, table, [[int(p)] for p in pos])))
    monkeypatch.setattr(ops, "dsim_paged_attention", lambda q, cache, table, lens, out, workspace: touched.append(
        rows(q) | rows(out) | places(cache, table, [range(int(n)) for n in lens])))
    monkeypatch.setattr(ops, "dsim_logit_adjust", lambda x, y, history, **kw: touched.append(
        rows(x) | rows(y) | rows(history)))
    gen = torch.Generator().manual_seed(0)
    for op, nbytes, calls in calibrate._decode_calls(*shape, torch.float16, reps, gen, "cpu"):
        del touched[:]
        for call in calls:
            call()
        assert len(calls) == calibrate._copies(nbytes, reps) and len(touched) == len(calls)
        for i, a in enumerate(touched):
            for b in touched[:i]:
                assert not a & b, op


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
def test_fitted_bandwidth_is_the_memorys(tmp_path, capsys, dtype):
    """No more than the 6.5 TB/s that reads alone reach on MI355X, no less than
    half of them, and no sample above the memory's 8 TB/s; a launch overhead
    of 1 to 20 us."""
    path = tmp_path / "decode.json"
    assert calibrate.main(["--op", "decode", "--dtype", dtype, "--out", str(path)]) == 0
    out = json.loads(path.read_text())
    print(capsys.readouterr().out)
    assert 3.2e12 < out["decode"]["mem_bytes_per_s"] < 6.5e12
    assert 1e-6 < out["decode"]["launch_s"] < 20e-6
    assert all(s["bytes"] / s["seconds"] < 8e12 for s in out["samples"])
