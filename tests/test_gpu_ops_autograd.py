"""Autograd sees what the single-token step's operators write."""
import pytest
import torch

from paper_2111_05426_amd import ops
from test_gpu_ops import gpu  # noqa: F401

pytestmark = pytest.mark.gpu

I32 = torch.int32


def calls():
    """name: (call, tensors that it writes)"""
    def z(*s, dtype=torch.float32):
        return torch.zeros(*s, dtype=dtype, device="cuda")
    cache = dict(k=z(4, 16, 2, 64), v=z(4, 16, 2, 64))
    table, rows, q, q_out = z(3, 2, dtype=I32), z(3, 2, 64), z(3, 4, 64), z(3, 4, 64)
    seq, status = torch.arange(3, dtype=I32, device="cuda"), z(3, dtype=I32)
    out, lse, ws = z(3, 4, 64), z(3, 4), ops.alloc_paged_attention_workspace(4, 2, 64)
    x, y = z(2, 100), z(2, 100)
    return {
        "append": (lambda: ops.dsim_kv_append(cache, table, rows, rows, seq, seq, q=q, q_out=q_out, status=status),
                   [cache["k"], cache["v"], q_out, status], [table, rows, seq, q]),
        "attention": (lambda: ops.dsim_paged_attention(q, cache, table, seq, out, lse=lse, status=status, workspace=ws),
                      [out, lse, status, ws], [q, cache["k"], cache["v"], table, seq]),
        "logits": (lambda: ops.dsim_logit_adjust(x, y), [y], [x]),
        "logits in place": (lambda: ops.dsim_logit_adjust(x, x), [x], [])}


@pytest.mark.parametrize("name", ["append", "attention", "logits", "logits in place"])
def test_versions(name):
    call, written, read = calls()[name]
    before, kept = [t._version for t in written], [t._version for t in read]
    call()
    assert all(t._version > n for t, n in zip(written, before)) and [t._version for t in read] == kept


@pytest.mark.parametrize("name", ["append", "attention", "logits"])
def test_written_after_it_was_saved(name):
    """A buffer that another operation's backward pass needs and the operator
    writes: an error, as with any in-place write, not a wrong gradient."""
    call, written, _ = calls()[name]
    w = torch.ones((), device="cuda", requires_grad=True)
    y = sum((w * t).sum() for t in written if t.is_floating_point())
    call()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_refused_calls_write_nothing():
    x = torch.zeros(2, 100, device="cuda")
    wide = torch.zeros(2, 200, device="cuda")
    with pytest.raises(ops.DsimError):
        ops.dsim_logit_adjust(wide[:, :100], torch.as_strided(x, (2, 100), (1, 1)))   # rows that overlap
    assert x._version == 0


def test_tensors_of_inference_mode():
    """They keep no versions; they are written inside and outside of it."""
    with torch.inference_mode():
        x = torch.zeros(2, 100, device="cuda")
        bias = dict(bias_id=torch.full((2, 1), 3, dtype=I32, device="cuda"), bias=torch.ones(2, 1, device="cuda"))
        ops.dsim_logit_adjust(x, x, **bias)
    ops.dsim_logit_adjust(x, x, **bias)
    with torch.inference_mode():
        plain = torch.zeros(2, 100, device="cuda")
    y = torch.zeros(2, 100, device="cuda")
    with torch.inference_mode():
        ops.dsim_logit_adjust(plain, y, **bias)
    assert x[:, 3].tolist() == [2.0, 2.0] and y[:, 3].tolist() == [1.0, 1.0]
