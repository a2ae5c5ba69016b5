"""Python binding of the single-token step's operators (include/dsim_ops.h):
argument marshalling only.

* dsim_kv_append: new keys and values rotated by position and written into a
  paged cache, queries rotated on the way;
* dsim_paged_attention: attention of one new token per sequence over it;
* dsim_logit_adjust: penalties for repeated tokens, biases and grammar masks.

A cache is a dict of device tensors: "k" and "v" of shape (pages, slots of a
page, heads, head_dim) with any strides whose last is 1 (alloc_kv_cache keeps
a head's slots of a page together), and for an e4m3 cache optionally
"k_scale" and "v_scale", fp32 (heads,).  Position t of sequence s lies in page
block_table[s, t // page_size], slot t % page_size.

    cache = ops.alloc_kv_cache(n_pages, 16, kv_heads, head_dim, torch.bfloat16)
    rope = ops.rope_table(max_len, head_dim)
    ws = ops.alloc_paged_attention_workspace(heads, kv_heads, head_dim)
    # every step, seq_len counting the new token
    ops.dsim_kv_append(cache, block_table, k, v, seq, seq_len - 1, rope=rope, q=q, q_out=q)
    ops.dsim_paged_attention(q, cache, block_table, seq_len, out, workspace=ws)
    ops.dsim_logit_adjust(logits, logits, history=tokens, history_len=seq_len, repetition=r)

Every call runs on the device of its tensors, on `stream` (None: that
device's current stream); its tensors must be ready there.  Like the rest of
the binding the calls raise ValueError for tensors that do not match what the
library reads or writes, and DsimError where the library refuses.
"""
import ctypes as C
from functools import lru_cache

from . import dsim
from .dsim import DsimError  # noqa: F401  (what the calls raise)

F32, F16, BF16, E4M3 = 0, 1, 2, 3
ST_BAD_PAGE, ST_BAD_POSITION, ST_BAD_SEQUENCE = 128, 256, 512


class dsim_kv_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("block_table", C.c_void_p), ("n_pages", C.c_int64), ("page_stride", C.c_int64),
                ("slot_stride", C.c_int64), ("head_stride", C.c_int64), ("table_stride", C.c_int64),
                ("dtype", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32), ("page_size", C.c_int32),
                ("n_seq", C.c_int32), ("table_width", C.c_int32)]


class dsim_rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class dsim_logits(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("out", C.c_void_p), ("logits_stride", C.c_int64),
                ("out_stride", C.c_int64), ("n_rows", C.c_int64), ("vocab", C.c_int32), ("dtype", C.c_int32),
                ("history", C.c_void_p), ("prompt_len", C.c_void_p), ("history_len", C.c_void_p),
                ("history_stride", C.c_int64), ("history_width", C.c_int32), ("n_bias", C.c_int32),
                ("repetition", C.c_void_p), ("frequency", C.c_void_p), ("presence", C.c_void_p),
                ("bias_id", C.c_void_p), ("bias", C.c_void_p), ("mask", C.c_void_p), ("mask_stride", C.c_int64)]


_lib = None


def lib():
    """libdsim.so with the operators' signatures set; raises if it has not
    been built."""
    global _lib
    if _lib is None:
        L = dsim.lib()
        P, I32, I64 = C.c_void_p, C.c_int32, C.c_int64
        L.dsim_kv_append.argtypes = [P, I64, I32, P, P, P, P, I32, P, P, P, I64, I32, I32, P, P]
        L.dsim_paged_attention_workspace.restype = C.c_size_t
        L.dsim_paged_attention_workspace.argtypes = [I32, I32, I32]
        L.dsim_paged_attention.argtypes = [P, I32, P, P, I32, P, C.c_float, I32, P, P, P, C.c_size_t, P]
        L.dsim_logit_adjust.argtypes = [P, P]
        for f in (L.dsim_kv_append, L.dsim_paged_attention, L.dsim_logit_adjust):
            f.restype = C.c_int
        _lib = L
    return _lib


@lru_cache(maxsize=None)
def _types():
    import torch
    return {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16, torch.float8_e4m3fn: E4M3}


def _fail(name, what):
    raise ValueError("%s %s" % (name, what))


class _Args:
    """The tensors of one call: each checked as it is added, all of them for
    their device at the end."""

    def __init__(self):
        self.seen = []

    def tensor(self, name, t, dtypes, shape):
        """A tensor of one of the dtypes and the shape (None entries free)
        whose last dimension is contiguous; its address."""
        try:
            dtype, got, p = t.dtype, t.shape, t.data_ptr
        except AttributeError:
            _fail(name, "must be a torch tensor")
        if dtype not in dtypes:
            _fail(name, "must be of dtype %s, not %s" % (" or ".join(str(d) for d in dtypes), dtype))
        if len(got) != len(shape) or any(w is not None and a != w for a, w in zip(got, shape)):
            _fail(name, "must have shape %s, not %s" % (shape, tuple(got)))
        if got[-1] > 1 and t.stride(-1) != 1:
            _fail(name, "must be contiguous in its last dimension")
        self.seen.append((name, t))
        return p()

    def flat(self, name, t, dtype, n):
        """A contiguous vector of n elements, or None; its address."""
        if t is None:
            return None
        return self.tensor(name, t, (dtype,), (n,))

    def run(self, fn, stream, call):
        """call(stream handle) on the device that holds every tensor."""
        import torch
        device = self.seen[0][1].device
        for name, t in self.seen:
            if t.device != device or not t.is_cuda:
                _fail(name, "must be a GPU tensor on %s, not on %s" % (
                    device if device.type == "cuda" else "the others' device", t.device))
        if device.index == torch.cuda.current_device():
            dsim._check(fn, call(_handle(stream, device)))
        else:
            with torch.cuda.device(device):
                dsim._check(fn, call(_handle(stream, device)))


def _handle(stream, device):
    if stream is None:
        import torch
        return torch.cuda.current_stream(device).cuda_stream
    return getattr(stream, "cuda_stream", stream)


def _rows(t):
    s = t.stride()
    return dsim_rows(t.data_ptr(), s[0], s[1])


def _cache(a, cache, block_table):
    import torch
    k, v = cache["k"], cache["v"]
    a.tensor("cache['k']", k, _types(), (None,) * 4)
    a.tensor("cache['v']", v, (k.dtype,), tuple(k.shape))
    if any(x != y and n > 1 for x, y, n in zip(k.stride(), v.stride(), k.shape)):
        _fail("cache['v']", "must have the strides of cache['k']")
    pages, slots, heads, d = k.shape
    table = a.tensor("block_table", block_table, (torch.int32,), (None, None))
    ks = a.flat("cache['k_scale']", cache.get("k_scale"), torch.float32, heads)
    vs = a.flat("cache['v_scale']", cache.get("v_scale"), torch.float32, heads)
    st, bt = k.stride(), block_table
    return dsim_kv_cache(k.data_ptr(), v.data_ptr(), ks, vs, table, pages, st[0], st[1], st[2], bt.stride(0),
                         _types()[k.dtype], heads, d, slots, bt.shape[0], bt.shape[1])


def alloc_kv_cache(n_pages, page_size, n_heads, head_dim, dtype, device="cuda"):
    """A cache dict (uninitialised); the slots of one head and page are next
    to each other in memory."""
    import torch
    shape = (n_pages, n_heads, page_size, head_dim)
    return {n: torch.empty(shape, dtype=dtype, device=device).transpose(1, 2) for n in ("k", "v")}


def rope_table(n_pos, rot_dim, base=10000.0, device="cuda"):
    """The rotation table (n_pos, rot_dim) fp32: rot_dim / 2 cosines, then as
    many sines, of position * base^(-2 i / rot_dim), computed in fp64."""
    import torch
    i = torch.arange(rot_dim // 2, dtype=torch.float64, device=device)
    angle = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * float(base) ** (-2.0 * i / rot_dim)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def dsim_kv_append(cache, block_table, k, v, seq, pos, rope=None, interleaved=False, q=None, q_out=None, status=None,
                   stream=None):
    """k, v: (tokens, heads, head_dim); seq, pos: int32 (tokens,), seq < 0 for
    padding; block_table: int32 (sequences, pages of a sequence); rope: fp32
    (positions, rot_dim) or None; q, q_out: (tokens, query heads, head_dim) or
    None, q_out may be q; status: int32 (tokens,) or None."""
    import torch
    a = _Args()
    c = _cache(a, cache, block_table)
    a.tensor("k", k, _types(), (None, c.n_heads, c.head_dim))
    n, dt = k.shape[0], (k.dtype,)
    a.tensor("v", v, dt, (n, c.n_heads, c.head_dim))
    seq_p = a.flat("seq", seq, torch.int32, n)
    pos_p = a.flat("pos", pos, torch.int32, n)
    if seq_p is None or pos_p is None:
        _fail("seq and pos", "are required")
    st = a.flat("status", status, torch.int32, n)
    heads = qr = qo = rope_p = None
    n_rope = rot = 0
    if (q is None) != (q_out is None):
        _fail("q and q_out", "come together")
    if q is not None:
        a.tensor("q", q, dt, (n, None, c.head_dim))
        heads = q.shape[1]
        a.tensor("q_out", q_out, dt, (n, heads, c.head_dim))
        qr, qo = _rows(q), _rows(q_out)
    if rope is not None:
        rope_p = a.tensor("rope", rope, (torch.float32,), (None, None))
        if not rope.is_contiguous():
            _fail("rope", "must be contiguous")
        n_rope, rot = rope.shape
    kr, vr = _rows(k), _rows(v)
    L = lib()
    a.run("dsim_kv_append", stream, lambda s: L.dsim_kv_append(
        C.byref(c), n, _types()[k.dtype], C.byref(kr), C.byref(vr), None if qr is None else C.byref(qr),
        None if qo is None else C.byref(qo), heads or 0, seq_p, pos_p, rope_p, n_rope, rot, 1 if interleaved else 0,
        st, s))


def dsim_paged_attention_workspace(n_q_heads, n_heads, head_dim):
    return int(lib().dsim_paged_attention_workspace(n_q_heads, n_heads, head_dim))


def alloc_paged_attention_workspace(n_q_heads, n_heads, head_dim, device="cuda"):
    """A caller-owned workspace for dsim_paged_attention (torch uint8)."""
    import torch
    return torch.empty(max(dsim_paged_attention_workspace(n_q_heads, n_heads, head_dim), 16), dtype=torch.uint8,
                       device=device)


def dsim_paged_attention(q, cache, block_table, seq_len, out, scale=None, window=0, workspace=None, lse=None,
                         status=None, stream=None):
    """q, out: (sequences, query heads, head_dim); seq_len: int32
    (sequences,), the new token included; scale: None for head_dim^-0.5;
    lse: fp32 (sequences, query heads) or None; status: int32 (sequences,) or
    None; workspace: uint8 of at least dsim_paged_attention_workspace(...)
    bytes (None: one is allocated with torch for this call)."""
    import torch
    a = _Args()
    c = _cache(a, cache, block_table)
    n = c.n_seq
    a.tensor("q", q, _types(), (n, None, c.head_dim))
    heads = q.shape[1]
    a.tensor("out", out, (q.dtype,), tuple(q.shape))
    lens = a.flat("seq_len", seq_len, torch.int32, n)
    if lens is None:
        _fail("seq_len", "is required")
    lse_p = None
    if lse is not None:
        lse_p = a.tensor("lse", lse, (torch.float32,), (n, heads))
        if not lse.is_contiguous():
            _fail("lse", "must be contiguous")
    st = a.flat("status", status, torch.int32, n)
    qr, o = _rows(q), _rows(out)
    if scale is None:
        scale = float(c.head_dim) ** -0.5
    L = lib()
    own = workspace is None
    if own:
        workspace = alloc_paged_attention_workspace(heads, c.n_heads, c.head_dim, device=q.device)
    a.tensor("workspace", workspace, (torch.uint8,), (None,))
    if own and stream is not None and q.is_cuda:
        # its memory may be handed out again only after that stream's work
        workspace.record_stream(stream if hasattr(stream, "cuda_stream")
                                else torch.cuda.ExternalStream(stream, device=q.device))
    a.run("dsim_paged_attention", stream, lambda s: L.dsim_paged_attention(
        C.byref(c), _types()[q.dtype], C.byref(qr), C.byref(o), heads, lens, scale, window, lse_p, st,
        workspace.data_ptr(), workspace.numel(), s))


def dsim_logit_adjust(logits, out, history=None, prompt_len=None, history_len=None, repetition=None, frequency=None,
                      presence=None, bias_id=None, bias=None, mask=None, stream=None):
    """logits, out: (rows, vocab), out may be logits; history: int32 (rows,
    width) token numbers, of which history_len (rows,) count, the first
    prompt_len (rows,) as the prompt; repetition, frequency, presence: fp32
    (rows,); bias_id, bias: int32 and fp32 (rows, biases); mask: int32 (rows,
    ceil(vocab / 32)), bit t % 32 of word t // 32 set where t is allowed."""
    import torch
    a = _Args()
    x = a.tensor("logits", logits, tuple(_types())[:3], (None, None))
    n, vocab = logits.shape
    y = a.tensor("out", out, (logits.dtype,), (n, vocab))
    i32, f32 = torch.int32, torch.float32
    s = dsim_logits(x, y, logits.stride(0), out.stride(0), n, vocab, _types()[logits.dtype])
    if history is not None:
        s.history = a.tensor("history", history, (i32,), (n, None))
        s.history_stride, s.history_width = history.stride(0), history.shape[1]
    s.history_len = a.flat("history_len", history_len, i32, n)
    s.prompt_len = a.flat("prompt_len", prompt_len, i32, n)
    s.repetition = a.flat("repetition", repetition, f32, n)
    s.frequency = a.flat("frequency", frequency, f32, n)
    s.presence = a.flat("presence", presence, f32, n)
    if history is not None and s.history_width == 0:
        s.history = s.history_len   # (no token is read)
    if (bias_id is None) != (bias is None):
        _fail("bias_id and bias", "come together")
    if bias_id is not None:
        s.bias_id = a.tensor("bias_id", bias_id, (i32,), (n, None))
        s.n_bias = bias_id.shape[1]
        s.bias = a.tensor("bias", bias, (f32,), (n, s.n_bias))
        if not (bias_id.is_contiguous() and bias.is_contiguous()):
            _fail("bias_id and bias", "must be contiguous")
    if mask is not None:
        s.mask = a.tensor("mask", mask, (i32,), (n, (vocab + 31) // 32))
        s.mask_stride = mask.stride(0)
    L = lib()
    a.run("dsim_logit_adjust", stream, lambda h: L.dsim_logit_adjust(C.byref(s), h))
