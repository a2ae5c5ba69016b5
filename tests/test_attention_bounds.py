"""The attention's allowed errors (attention_bounds.py) let plain fp32
arithmetic pass and refuse arithmetic that has lost bits.  CPU only."""
import pytest
import torch

import attention_bounds as bounds

F32 = torch.float32


def bits(x, n):
    """fp32 rounded to n mantissa bits (of 23)."""
    half, step = 1 << (22 - n), 1 << (23 - n)
    return ((x.contiguous().view(torch.int32) + half) & -step).view(F32)


def case(d, n, heads=4, seed=0):
    g = torch.Generator().manual_seed(seed)
    q = 2 * torch.randn(3, heads, d, generator=g)
    keys, values = (torch.randn(3 * (n // 16 + 1), 16, 2, d, generator=g) for _ in range(2))
    table = torch.randperm(keys.shape[0], generator=g).to(torch.int32).view(3, -1)
    return q, keys, values, table, torch.tensor([n, n // 2 + 1, 1])


def plain(q, keys, values, table, lens, scale, score=lambda x: x, weight=lambda x: x, inputs=lambda x: x):
    """fp32 step by step, keys in tiles of 16 with a running maximum."""
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2])
    for b in range(q.shape[0]):
        n = int(lens[b])
        j = torch.arange(n)
        page = table[b].long()[j // 16]
        for h in range(q.shape[1]):
            c = h // (q.shape[1] // keys.shape[2])
            k, v = inputs(keys[page, j % 16, c]), values[page, j % 16, c]
            s = torch.zeros(n)
            for i in range(q.shape[2]):
                s = s + k[:, i] * inputs(q[b, h])[i]
            s = score(s * scale)
            m, total, o = torch.tensor(-float("inf")), torch.tensor(0.0), torch.zeros(q.shape[2])
            for t in range(0, n, 16):
                top = torch.maximum(m, s[t:t + 16].max())
                f, w = torch.exp(m - top), weight(torch.exp(s[t:t + 16] - top))
                total, o, m = total * f, o * f, top
                for i in range(len(w)):
                    total, o = total + w[i], o + w[i] * v[t + i]
            out[b, h], lse[b, h] = o / total, m + total.log()
    return out, lse


@pytest.mark.parametrize("d,n", [(16, 40), (64, 250), (128, 250), (256, 250), (64, 1500)])
def test_bounds(d, n):
    args = case(d, n)
    ref, ref_lse, room, lse_room = bounds.attend(*args, d ** -0.5)
    out, lse = plain(*args, d ** -0.5)
    assert bounds.within(out, ref, room) and bounds.off(out, ref, room) < 0.5
    assert torch.all((lse.double() - ref_lse).abs() <= lse_room)
    # what has 10 bits of 23, as 16-bit floats and shortened matrix formats have, and 14
    for n_bits in (10, 14):
        for lost in ("score", "weight", "inputs"):
            out, lse = plain(*args, d ** -0.5, **{lost: lambda x: bits(x, n_bits)})
            assert not bounds.within(out, ref, room), (lost, n_bits)


def test_sixteen_bit_weights_are_refused():
    """Weights of 16 bits (two bf16 numbers) under many keys."""
    args = case(64, 2000, heads=2, seed=1)
    ref, _, room, _ = bounds.attend(*args, 0.125)

    def two(w):
        first = (w.view(torch.int32) & -65536).view(F32)
        return first + (w - first).bfloat16().float()
    errors = [bounds.off(plain(*args, 0.125, weight=f)[0], ref, room) for f in (lambda w: w, two)]
    assert errors[0] < 0.5 and errors[1] > 2 * errors[0]
