"""Paged attention in 64 bits with what fp32 arithmetic may lose on the way to
it, by the sizes that the roundings are expected to have and not by the worst
that they could add up to.  CPU only.

u = 2^-24, a rounding's largest relative size; one rounding has a root mean
square of u / sqrt(3) of its value.
* A score is a sum of d products x_i in some order.  Over all orders the
  partial sums' squares add up to d s^2 / 3 + d |x|^2 / 6 on average, so the
  sum's roundings have a mean square of a third of that (and of |x|^2 where
  products are rounded too), times the scale.
* A weight is 2^(a - b) of the score: the argument's rounding is u (m - s) and
  the exponential's two u.
* Errors of the weights reach an output as sum p_j e_j (v_j - o): independent
  ones as the root of the squares' sum.  The scale's roundings (scale, times
  log2 e, times the keys' scale) are the same for every key: three u of s_j -
  sum p s.
* The sum of n weights rounds n times, each partial sum at most the last one's
  size; that of the weighted values likewise, its partial sums' squares at
  most o^2 + sum (p_j v_j)^2 (the first is what they end at, the second what
  they reach in any order of values that are not all of one sign).
An implementation is allowed SIGMAS times the root mean square."""
import math

import torch

U = 2.0 ** -24
SIGMAS = 8
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}   # half the smallest step


def rows(q, keys, values, table, seq_len, scale, window=0, k_scale=None, v_scale=None):
    """For each sequence with keys and each head: (b, h, products (key, d),
    values (key, d)) in 64 bits, the scales in them."""
    slots, group = keys.shape[1], q.shape[1] // keys.shape[2]
    for b in range(q.shape[0]):
        n = int(seq_len[b])
        first = max(0, n - window) if window else 0
        if n <= first:
            continue
        j = torch.arange(first, n)
        page = table[b].long()[j // slots]
        for h in range(q.shape[1]):
            c = h // group
            x = keys[page, j % slots, c].double() * q[b, h].double() * scale
            v = values[page, j % slots, c].double()
            yield (b, h, x if k_scale is None else x * k_scale[c].double(),
                   v if v_scale is None else v * v_scale[c].double())


def attend(q, keys, values, table, seq_len, scale, window=0, k_scale=None, v_scale=None):
    """Returns (out, lse, what out may be off before its rounding, what lse
    may be off), in 64 bits."""
    n_seq, heads, d = q.shape
    out, room = (torch.zeros(n_seq, heads, d, dtype=torch.float64) for _ in range(2))
    lse, lse_room = torch.full((n_seq, heads), -math.inf, dtype=torch.float64), torch.zeros(n_seq, heads).double()
    for b, h, x, v in rows(q, keys, values, table, seq_len, scale, window, k_scale, v_scale):
        s, n = x.sum(1), x.shape[0]
        p = torch.softmax(s, 0)
        o = p @ v
        x2 = (x * x).sum(1)
        e2 = (d * s * s / 3 + d * x2 / 6 + x2) / 3 + (s.max() - s) ** 2 / 3 + 4.0 / 3      # a weight's, in u^2
        away = v - o
        sums = math.sqrt(n / 3) * (o.abs() + (o * o + (p * p) @ (v * v)).sqrt())
        rms = ((p * p * e2) @ (away * away)).sqrt() + sums
        same = 3 * (p * (s - p @ s).abs()) @ away.abs()
        out[b, h], room[b, h] = o, U * (SIGMAS * rms + same + 2 * o.abs())
        lse[b, h] = torch.logsumexp(s, 0)
        lse_room[b, h] = U * (SIGMAS * (((p * p * e2).sum()).sqrt() + math.sqrt(n / 3)) + 3 * (p @ s.abs()) +
                              4 * s.abs().max() + 4 * lse[b, h].abs() + 4)
    return out, lse, room, lse_room


def off(got, ref, room):
    """The largest error of got beyond its rounding, as a part of the room."""
    got, ref = got.double(), ref.double()
    rounding = HALF_STEP[torch.float32] * (ref.abs() + room)
    return float(((got - ref).abs() / (room + rounding).clamp(min=1e-300)).max())


def within(got, ref, room):
    """Whether got, rounded once to its type, lies within the room."""
    dtype, got = got.dtype, got.double()
    return bool(torch.all((got - ref).abs() <= room + (ref.abs() + room) * HALF_STEP[dtype] + LEAST[dtype]))
