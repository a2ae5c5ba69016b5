"""More refusals of the single-token step's operators, on the host: arguments
that are in range one by one but not in what the kernels make of them.  CPU
only."""
import ctypes as C

import pytest
import torch

from paper_2111_05426_amd import dsim, ops
from test_ops import FAKE, L, append_args, cache, refused, rows  # noqa: F401



@pytest.mark.parametrize("scale", [3e38, -3e38, 2.0 ** 127, float("inf"), -float("inf"), float("nan")])
def test_attention_scale_that_overflows(L, scale):   # noqa: F811
    """Times log2 e it would be infinite, and products of 0 then NaN."""
    rc = L.dsim_paged_attention(C.byref(cache()), 2, C.byref(rows()), C.byref(rows()), 4, FAKE, scale, 0, None, None,
                                None, 0, None)
    assert rc == -1 and "scale" in dsim.dsim_last_error(), (rc, dsim.dsim_last_error())


def test_attention_largest_scale(L):   # noqa: F811
    """2^126 is taken (and the next thing, the workspace, refused)."""
    for scale in (2.0 ** 126, -2.0 ** 126):
        rc = L.dsim_paged_attention(C.byref(cache()), 2, C.byref(rows()), C.byref(rows()), 4, FAKE, scale, 0, None, None,
                                    None, 0, None)
        assert rc == -3 and "workspace" in dsim.dsim_last_error()


def test_tensors_that_carry_a_tangent():
    """Forward-mode derivatives would end in the operators without a word."""
    import torch.autograd.forward_ad as forward
    args = append_args()
    x = torch.zeros(2, 100)
    attention = dict(q=args["q"][:3], cache=args["cache"], block_table=torch.zeros(3, 2, dtype=torch.int32),
                     seq_len=torch.zeros(3, dtype=torch.int32), out=torch.zeros(3, 4, 64, dtype=torch.float16),
                     workspace=torch.zeros(9, dtype=torch.uint8))
    with forward.dual_level():
        for fn, kw, name in ((ops.dsim_kv_append, args, "k"), (ops.dsim_paged_attention, attention, "q"),
                             (ops.dsim_logit_adjust, dict(logits=x, out=torch.zeros(2, 100)), "logits")):
            dual = forward.make_dual(kw[name], torch.ones_like(kw[name]))
            refused(name + " carries a tangent", fn, **{**kw, name: dual})
            with torch.no_grad():   # does not end them
                refused(name + " carries a tangent", fn, **{**kw, name: dual})
            refused("GPU", fn, **{**kw, name: forward.unpack_dual(dual).primal})
