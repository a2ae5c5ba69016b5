"""Plain implementations of the single-token step's operators, written from
their formulas: the cache append and the logits in the fp32 steps that the
interface states (so that results must be equal), the attention in 64 bits
with a bound on what fp32 sums may lose.  CPU only."""
import math

import torch

E4M3 = torch.float8_e4m3fn
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def rotate(x, row, interleaved):
    """x (heads, d) fp32 by one row of a rotation table (or None)."""
    if row is None:
        return x
    r = row.numel()
    c, s = row[:r // 2], row[r // 2:]
    y = x.clone()
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    y[:, a] = x[:, a] * c - x[:, b] * s
    y[:, b] = x[:, b] * c + x[:, a] * s
    return y


def to_e4m3(x):
    """fp32 to e4m3: one rounding, beyond +-448 to +-448, NaN kept."""
    return torch.where(x.isnan(), x, x.clamp(-448.0, 448.0)).to(E4M3)


def append(keys, values, table, k, v, seq, pos, rope=None, interleaved=False, q=None, q_out=None, k_scale=None,
           v_scale=None):
    """Returns keys, values (pages, slots, heads, d), q_out and status after
    the call; the arguments stay as they are."""
    keys, values = keys.clone(), values.clone()
    q_out = None if q is None else q_out.clone()
    status = torch.zeros(len(seq), dtype=torch.int32)
    slots = keys.shape[1]
    for t in range(len(seq)):
        s, p = int(seq[t]), int(pos[t])
        if s < 0:
            continue
        bad = 512 if s >= table.shape[0] else 0
        if p < 0 or p >= table.shape[1] * slots or (rope is not None and p >= rope.shape[0]):
            bad |= 256
        if not bad:
            page = int(table[s, p // slots])
            bad = 128 if page < 0 or page >= keys.shape[0] else 0
        status[t] = bad
        if bad:
            if q is not None:
                q_out[t] = math.nan
            continue
        row = None if rope is None else rope[p]
        if q is not None:
            q_out[t] = rotate(q[t].float(), row, interleaved).to(q_out.dtype)
        for cache, x, scale in ((keys, rotate(k[t].float(), row, interleaved), k_scale),
                                (values, v[t].float(), v_scale)):
            if scale is not None:
                x = x / scale[:, None]
            if cache.dtype == E4M3:
                cache.view(torch.uint8)[page, p % slots] = to_e4m3(x).view(torch.uint8)
            else:
                cache[page, p % slots] = x.to(cache.dtype)
    return keys, values, q_out, status


def attend(q, keys, values, table, seq_len, scale, window=0, k_scale=None, v_scale=None):
    """Returns (out, lse, bound) in fp64: bound is what an implementation may
    be off before its last rounding.

    Each score is a sum of d products of the inputs, exact in fp32, added in
    fp32: off by at most (d + 2) 2^-24 sum |q k| scale (the scaling's rounding
    and the maximum's subtraction among it, and twice, for the exponent to
    base 2).  A weight then is off by that relative to itself, by the
    exponential's 2^-22 and by the two-number split's 2^-15 (bf16), which is
    the coarsest; a sum of n weights adds n 2^-24, once above and once below
    the fraction, with the running maximum's rescaling another 2^-23 for each
    of n / 16 tiles."""
    n, heads, d = q.shape
    slots, kv = keys.shape[1], keys.shape[2]
    out = torch.zeros(n, heads, d, dtype=torch.float64)
    bound = torch.zeros(n, heads, d, dtype=torch.float64)
    lse = torch.full((n, heads), -math.inf, dtype=torch.float64)
    for b in range(n):
        length = int(seq_len[b])
        first = max(0, length - window) if window else 0
        if length <= first:
            continue
        j = torch.arange(first, length)
        page = table[b].long()[j // slots]
        for h in range(heads):
            c = h // (heads // kv)
            k, v = keys[page, j % slots, c].double(), values[page, j % slots, c].double()
            if k_scale is not None:
                k = k * k_scale[c].double()
            if v_scale is not None:
                v = v * v_scale[c].double()
            x = q[b, h].double()
            s = (k @ x) * scale
            p = torch.softmax(s, 0)
            out[b, h] = p @ v
            lse[b, h] = torch.logsumexp(s, 0)
            off = 4 * (d + 2) * 2.0 ** -24 * abs(scale) * (k.abs() @ x.abs()).max()
            off = off + 2.0 ** -15 + 2.0 ** -21 + (length - first) * 1.25 * 2.0 ** -23
            bound[b, h] = off * (p @ v.abs())
    return out, lse, bound


def logits(x, history=None, prompt_len=None, history_len=None, repetition=None, frequency=None, presence=None,
           bias_id=None, bias=None, mask=None):
    """The adjusted logits, each step in fp32 as the interface states."""
    n, vocab = x.shape
    y = x.float().clone()
    for b in range(n):
        if history is not None:
            length = min(max(int(history_len[b]), 0), history.shape[1])
            prompt = 0 if prompt_len is None else min(max(int(prompt_len[b]), 0), length)
            ids = history[b, :length].long()
            inside = (ids >= 0) & (ids < vocab)
            made = torch.bincount(ids[prompt:][inside[prompt:]], minlength=vocab)
            seen = torch.bincount(ids[inside], minlength=vocab) > 0
            r = repetition[b] if repetition is not None else torch.tensor(1.0)
            f = frequency[b] if frequency is not None else torch.tensor(0.0)
            p = presence[b] if presence is not None else torch.tensor(0.0)
            z = torch.where(y[b] > 0, y[b] / r, y[b] * r)
            z = z - (f * made.float() + torch.where(made > 0, p, torch.tensor(0.0)))
            y[b] = torch.where(seen, z, y[b])
        if bias_id is not None:
            last = {int(t): i for i, t in enumerate(bias_id[b]) if 0 <= int(t) < vocab}
            for t, i in last.items():
                y[b, t] = y[b, t] + bias[b, i]
        if mask is not None:
            t = torch.arange(vocab)
            y[b, (mask[b].long()[t // 32] >> (t % 32)) & 1 == 0] = -math.inf
    return y.to(x.dtype)


def same(a, b):
    """Equal values, NaN where the other has NaN."""
    if a.dtype == E4M3:
        a, b = a.float(), b.float()
    return a.dtype == b.dtype and a.shape == b.shape and bool(torch.all((a == b) | (a.isnan() & b.isnan())))
