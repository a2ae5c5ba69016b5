"""Plain implementations of the operators of a step of several tokens, written
from their definitions: attention in 64 bits with a bound on what an fp32
implementation may lose, the others in whole numbers and copies.  CPU only."""
import math

import torch

import step_ops


def ranges(n, length, prefix, window, first_key):
    """First key and end of the keys of a prompt's n new tokens."""
    p = torch.arange(length - n, length)
    hi = torch.clamp(torch.maximum(p + 1, torch.tensor(prefix)), max=length)
    lo = torch.zeros_like(p) if not window else torch.clamp(p + 1 - window, min=0)
    if first_key is not None:
        lo = torch.maximum(lo, first_key.long().clamp(min=0))
    return p, lo, hi


def bits(mask, n):
    """Truth values (rows, n) of words of 32 bits."""
    j = torch.arange(n)
    return (mask.long()[:, j // 32] >> (j % 32)) & 1 == 1


def attention(q, keys, values, table, start, length, scale, tree_mask=None, depth=None, prefix_len=None, first_key=None,
              window=0, cap=0.0, slopes=None, k_scale=None, v_scale=None, weight=0.0, least=0.0, exact=True):
    """Returns (out, lse, bound, lse_bound, seen) in fp64 of every token of a
    sequence; seen: (tokens,) whether it belongs to one.

    Each score is a sum of d products of the inputs, exact in fp32, added in
    fp32: off by at most (d + 2) 2^-24 sum |q k| scale.  A capped one is off by
    the tanh's error relative to it as well (2^-20, or 2^-21 where `exact`, the
    library's), a bias by three roundings of the sum.  A weight is off by that
    relative to itself, by the exponential's 2^-21 and by `weight`, its
    rounding before the second product, or by `least` of the largest weight
    where it is too small for its type; a sum of n adds n 2^-23."""
    heads, d = q.shape[1:]
    slots, kv = keys.shape[1], keys.shape[2]
    out, bound = (torch.zeros(q.shape, dtype=torch.float64) for _ in range(2))
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    lse_bound = torch.zeros(q.shape[:2], dtype=torch.float64)
    seen = torch.zeros(q.shape[0], dtype=torch.bool)
    for s in range(table.shape[0]):
        a, n, length_s = int(start[s]), int(start[s + 1] - start[s]), int(length[s])
        if n <= 0 or length_s < 0:
            continue
        rows = slice(a, a + n)
        seen[rows] = True
        if tree_mask is not None:
            dep = torch.zeros(n, dtype=torch.long) if depth is None else depth[rows].long().clamp(min=0)
            p, total = length_s + dep, length_s + n
            place = torch.cat([torch.arange(length_s), p])
            past = torch.ones(n, length_s, dtype=torch.bool)
            if window:
                past = place[None, :length_s] > p[:, None] - window
            allowed = torch.cat([past, bits(tree_mask[rows], n)], 1)
        else:
            total = length_s
            p, lo, hi = ranges(n, length_s, 0 if prefix_len is None else int(prefix_len[s]), window,
                               None if first_key is None else first_key[rows])
            place = torch.arange(total)
            allowed = (place >= lo[:, None]) & (place < hi[:, None])
        j = torch.arange(total)
        page = table[s].long()[j // slots]
        for h in range(heads):
            c = h // (heads // kv)
            k, v = keys[page, j % slots, c].double(), values[page, j % slots, c].double()
            if k_scale is not None:
                k = k * k_scale[c].double()
            if v_scale is not None:
                v = v * v_scale[c].double()
            x = q[rows, h].double()
            score = (x @ k.t()) * scale
            err = (d + 2) * 2.0 ** -24 * abs(scale) * (x.abs() @ k.abs().t())
            if cap:
                score = cap * torch.tanh(score / cap)
                err = err + score.abs() * (2.0 ** -21 if exact else 2.0 ** -19)
            if slopes is not None:
                bias = slopes[h].double() * (p[:, None] - place).abs()
                score = score - bias
                err = err + 3 * 2.0 ** -24 * (score.abs() + bias.abs())
            score = torch.where(allowed, score, -math.inf)
            v = torch.where(allowed.any(0)[:, None], v, 0.0)
            w = torch.softmax(score, 1)
            w = torch.where(allowed, w, 0.0)   # (rows without keys)
            off = torch.where(allowed, w * (2 * err + 2.0 ** -20 + weight + total * 2.0 ** -23) + least * w.amax(1, keepdim=True), 0.0)
            out[rows, h] = w @ v
            bound[rows, h] = off @ v.abs() + off.sum(1, keepdim=True) * (w @ v.abs())
            lse[rows, h] = torch.logsumexp(score, 1)
            lse_bound[rows, h] = 2 * off.sum(1) + 1e-6 + 2.0 ** -22 * torch.where(allowed.any(1), lse[rows, h].abs(), 0.0)
    return out, lse, bound, lse_bound, seen


def append_axes(keys, values, table, k, v, seq, slot, pos, rope, sections, interleaved=False, q=None, q_out=None,
                k_scale=None, v_scale=None):
    """As step_ops.append, the rotation's row put together from the axes'."""
    keys, values = keys.clone(), values.clone()
    q_out = None if q is None else q_out.clone()
    status = torch.zeros(len(seq), dtype=torch.int32)
    slots = keys.shape[1]
    axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections))
    half = axis.numel()
    pair = torch.arange(half)
    for t in range(len(seq)):
        s, at = int(seq[t]), int(slot[t])
        if s < 0:
            continue
        bad = 512 if s >= table.shape[0] else 0
        if at < 0 or at >= table.shape[1] * slots or bool(((pos[t] < 0) | (pos[t] >= rope.shape[0])).any()):
            bad |= 256
        if not bad:
            page = int(table[s, at // slots])
            bad = 128 if page < 0 or page >= keys.shape[0] else 0
        status[t] = bad
        if bad:
            if q is not None:
                q_out[t] = math.nan
            continue
        rows = pos[t].long()[axis]
        row = torch.cat([rope[rows, pair], rope[rows, half + pair]])
        if q is not None:
            q_out[t] = step_ops.rotate(q[t].float(), row, interleaved).to(q_out.dtype)
        for cache, x, scale in ((keys, step_ops.rotate(k[t].float(), row, interleaved), k_scale),
                                (values, v[t].float(), v_scale)):
            if scale is not None:
                x = x / scale[:, None]
            if cache.dtype == step_ops.E4M3:
                cache.view(torch.uint8)[page, at % slots] = step_ops.to_e4m3(x).view(torch.uint8)
            else:
                cache[page, at % slots] = x.to(cache.dtype)
    return keys, values, q_out, status


class Pool:
    """Pages and who holds them, one thing after another."""

    def __init__(self, n_pages, rows, width, page):
        self.refs, self.held, self.page = [0] * n_pages, [0] * rows, page
        self.table = [[-1] * width for _ in range(rows)]

    def free(self):
        return [i for i, r in enumerate(self.refs) if r == 0]

    def words(self):
        n = len(self.refs)
        return [sum((self.refs[i] == 0) << (i - w) for i in range(w, min(n, w + 32))) for w in range(0, n, 32)]

    def pages(self, places):
        return -(-places // self.page)

    def reserve(self, length, want, status):
        refused = False
        left = self.free()
        for s, n in enumerate(want):
            if n < 0:
                continue
            status[s] = 0
            need = self.pages(n) - self.held[s]
            if self.pages(n) > len(self.table[s]) or length[s] < 0 or length[s] > self.held[s] * self.page:
                status[s] = 256
                continue
            if n > length[s] and length[s] % self.page:
                last = self.table[s][length[s] // self.page]
                if not 0 <= last < len(self.refs):
                    status[s] = 128
                    continue
                if self.refs[last] > 1:
                    status[s] = 2048
                    continue
            if need <= 0:
                continue
            if refused or need > len(left):
                refused = True
                status[s] = 1024
                continue
            for i in range(need):
                page = left.pop(0)
                self.refs[page] = 1
                self.table[s][self.held[s] + i] = page
            self.held[s] += need

    def release(self, rows, keep):
        for s, n in zip(rows, keep):
            if not 0 <= s < len(self.held):
                continue
            for j in range(self.pages(max(n, 0)), self.held[s]):
                page = self.table[s][j]
                self.table[s][j] = -1
                if 0 <= page < len(self.refs) and self.refs[page] > 0:
                    self.refs[page] -= 1
            self.held[s] = min(self.held[s], self.pages(max(n, 0)))

    def fork(self, length, src, dst, status, layers):
        """layers: tensors (pages, slots, ...)."""
        taken, held, refused = set(), list(self.held), False
        left = self.free()
        done = []
        targets = {d for d in dst if 0 <= d < len(held) and held[d] == 0}
        for i, (a, b) in enumerate(zip(src, dst)):
            status[i] = 0
            if b < 0:
                continue
            if b >= len(held) or not 0 <= a < len(held):
                if 0 <= b < len(held) and held[b] == 0:
                    taken.add(b)   # (the claim comes first)
                status[i] = 512
                continue
            if held[b] > 0 or b in taken:
                status[i] = 4096
                continue
            taken.add(b)
            if a in targets:
                status[i] = 512
                continue
            if length[a] < 0 or length[a] > held[a] * self.page:
                status[i] = 256
                continue
            if length[a] % self.page:
                if refused or not left:
                    refused = True
                    status[i] = 1024
                    continue
                page = left.pop(0)
                self.refs[page] = 1
            else:
                page = None
            done.append((i, a, b, page))
        for i, a, b, page in done:
            n = length[a]
            for j in range(n // self.page):
                p = self.table[a][j]
                if 0 <= p < len(self.refs):
                    self.table[b][j] = p
                    self.refs[p] += 1
                else:
                    self.table[b][j] = -1
                    status[i] |= 128
            if page is not None:
                self.table[b][n // self.page] = page
                p = self.table[a][n // self.page]
                if 0 <= p < len(self.refs):
                    for x in layers:
                        x[page, :n % self.page] = x[p, :n % self.page]
                else:
                    status[i] |= 128
            self.held[b] = self.pages(n)
            length[b] = n


def compact(layers, table, start, keep, n_keep):
    """layers: tensors (pages, slots, ...), changed; returns the status."""
    status = torch.zeros(table.shape[0], dtype=torch.int32)
    slots = layers[0].shape[1]
    before = [x.clone() for x in layers]
    for s in range(table.shape[0]):
        first, n = int(start[s]), min(max(int(n_keep[s]), 0), keep.shape[1])
        last = -1
        for j in range(n):
            k = int(keep[s, j])
            if first < 0 or k <= last or first + k >= table.shape[1] * slots:
                status[s] |= 256
                break
            last = k
            if k == j:
                continue
            to, of = int(table[s, (first + j) // slots]), int(table[s, (first + k) // slots])
            if not (0 <= to < layers[0].shape[0] and 0 <= of < layers[0].shape[0]):
                status[s] |= 128
                continue
            for x, y in zip(layers, before):
                x[to, (first + j) % slots] = y[of, (first + k) % slots]
        if first < 0:
            status[s] |= 256
    return status
