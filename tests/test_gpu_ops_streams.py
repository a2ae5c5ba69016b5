"""The single-token step's operators on streams."""
import pytest
import torch

from paper_2111_05426_amd import ops
from test_gpu_ops import gpu  # noqa: F401

pytestmark = pytest.mark.gpu

I32 = torch.int32


class OtherStream:
    """As a stream of another device has them."""
    cuda_stream, device_index = 0, 1


@pytest.mark.parametrize("name", ["append", "attention", "logits"])
def test_stream_of_another_device(name):
    call = {"append": lambda **kw: ops.dsim_kv_append(cache, table, rows, rows, seq, seq, **kw),
            "attention": lambda **kw: ops.dsim_paged_attention(q, cache, table, seq, torch.empty_like(q), workspace=ws, **kw),
            "logits": lambda **kw: ops.dsim_logit_adjust(x, x, **kw)}[name]
    cache = {n: torch.zeros(4, 16, 2, 64, device="cuda") for n in ("k", "v")}
    table, rows = torch.zeros(3, 2, dtype=I32, device="cuda"), torch.zeros(3, 2, 64, device="cuda")
    q, seq = torch.zeros(3, 4, 64, device="cuda"), torch.arange(3, dtype=I32, device="cuda")
    ws, x = ops.alloc_paged_attention_workspace(4, 2, 64), torch.zeros(2, 100, device="cuda")
    with pytest.raises(ValueError, match="stream must be on cuda:0"):
        call(stream=OtherStream())
    call(stream=torch.cuda.current_stream())
    call(stream=torch.cuda.Stream())
    torch.cuda.synchronize()
