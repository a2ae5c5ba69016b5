"""The single-token step's operators on the host: what include/dsim_ops.h
declares is exported, the C entry points refuse bad arguments before any
launch, the binding refuses tensors that do not match, and the plain
implementations that the GPU tests compare with agree with torch's own.
CPU only: no call here reaches a GPU."""
import ctypes as C
import os
import re

import pytest
import torch

import step_ops as plain
from paper_2111_05426_amd import build, dsim, ops

HEADER = os.path.join(build.INCLUDE, "dsim_ops.h")
F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
I32 = torch.int32
P, I4, I8 = C.c_void_p, C.c_int32, C.c_int64


class Cache(C.Structure):
    _fields_ = [("k", P), ("v", P), ("k_scale", P), ("v_scale", P), ("block_table", P), ("n_pages", I8),
                ("page_stride", I8), ("slot_stride", I8), ("head_stride", I8), ("table_stride", I8), ("dtype", I4),
                ("n_heads", I4), ("head_dim", I4), ("page_size", I4), ("n_seq", I4), ("table_width", I4)]


class Rows(C.Structure):
    _fields_ = [("data", P), ("row_stride", I8), ("head_stride", I8)]


class Logits(C.Structure):
    _fields_ = [("logits", P), ("out", P), ("logits_stride", I8), ("out_stride", I8), ("n_rows", I8), ("vocab", I4),
                ("dtype", I4), ("history", P), ("prompt_len", P), ("history_len", P), ("history_stride", I8),
                ("history_width", I4), ("n_bias", I4), ("repetition", P), ("frequency", P), ("presence", P),
                ("bias_id", P), ("bias", P), ("mask", P), ("mask_stride", I8)]


FAKE = 1 << 20   # a device address that is never followed


@pytest.fixture(scope="module")
def L():
    ops.lib()
    lib = C.CDLL(dsim.LIB_PATH)
    lib.dsim_kv_append.argtypes = [P, I8, I4, P, P, P, P, I4, P, P, P, I8, I4, I4, P, P]
    lib.dsim_paged_attention_workspace.restype = C.c_size_t
    lib.dsim_paged_attention_workspace.argtypes = [I4, I4, I4]
    lib.dsim_paged_attention.argtypes = [P, I4, P, P, I4, P, C.c_float, I4, P, P, P, C.c_size_t, P]
    lib.dsim_logit_adjust.argtypes = [P, P]
    return lib


def test_exports_every_declared_function(L):
    with open(HEADER) as f:
        names = re.findall(r"DSIM_API\s+[\w\s\*]*?\b(dsim_\w+)\s*\(", f.read())
    assert set(names) == {"dsim_kv_append", "dsim_paged_attention_workspace", "dsim_paged_attention",
                          "dsim_logit_adjust"}
    for n in names:
        assert hasattr(L, n) and hasattr(ops, n), n


def cache(**over):
    d = dict(k=FAKE, v=FAKE, block_table=FAKE, n_pages=8, page_stride=2 * 16 * 64, slot_stride=64,
             head_stride=16 * 64, table_stride=4, dtype=2, n_heads=2, head_dim=64, page_size=16, n_seq=3,
             table_width=4)
    d.update(over)
    return Cache(**d)


def rows(**over):
    return Rows(**{**dict(data=FAKE, row_stride=256, head_stride=64), **over})


BAD_CACHES = [
    (dict(dtype=4), "dtype"), (dict(dtype=-1), "dtype"), (dict(n_heads=0), "n_heads"), (dict(n_heads=2000), "n_heads"),
    (dict(head_dim=72), "head_dim"), (dict(head_dim=0), "head_dim"), (dict(head_dim=272), "head_dim"),
    (dict(page_size=0), "page_size"), (dict(page_size=(1 << 20) + 1), "page_size"), (dict(n_pages=-1), "n_pages"),
    (dict(n_pages=1 << 31), "n_pages"), (dict(n_seq=-1), "n_seq"), (dict(n_seq=(1 << 20) + 1), "n_seq"),
    (dict(table_width=-1), "table"), (dict(table_stride=3), "overlap"), (dict(table_stride=1 << 61), "table"),
    (dict(page_size=1 << 20, table_width=1 << 12, table_stride=1 << 12), "2^31"),
    (dict(slot_stride=60), "16 bytes"), (dict(page_stride=-2048), ">= 0"), (dict(head_stride=1 << 61), "16 bytes"),
    (dict(slot_stride=1024), "overlap"), (dict(slot_stride=0), "overlap"), (dict(page_stride=1024), "overlap"),
    (dict(k=0), "NULL"), (dict(v=FAKE + 8), "aligned"), (dict(k_scale=FAKE), "e4m3"), (dict(block_table=0), "NULL")]


@pytest.mark.parametrize("i", range(len(BAD_CACHES)))
def test_cache_refused(L, i):
    over, word = BAD_CACHES[i]
    c, r = cache(**over), rows()
    rc = L.dsim_kv_append(C.byref(c), 4, 2, C.byref(r), C.byref(r), None, None, 0, FAKE, FAKE, None, 0, 0, 0, None, None)
    assert rc < 0 and word in dsim.dsim_last_error(), dsim.dsim_last_error()
    if word == "overlap" and "table_stride" not in over:
        return   # rows that are only read may
    rc = L.dsim_paged_attention(C.byref(c), 2, C.byref(r), C.byref(r), 4, FAKE, 1.0, 0, None, None, FAKE, 1 << 40, None)
    assert rc < 0 and word in dsim.dsim_last_error(), dsim.dsim_last_error()


def test_append_refused(L):
    def call(word, n=4, dtype=2, k=rows(), v=rows(), q=None, q_out=None, heads=0, seq=FAKE, pos=FAKE, rope=None, n_rope=0,
             rot=0, inter=0, c=cache()):
        ref = lambda x: None if x is None else C.byref(x)   # noqa: E731
        rc = L.dsim_kv_append(ref(c), n, dtype, ref(k), ref(v), ref(q), ref(q_out), heads, seq, pos, rope, n_rope, rot,
                              inter, None, None)
        assert rc < 0 and word in dsim.dsim_last_error(), dsim.dsim_last_error()
    call("NULL", c=None)
    call("dtype", dtype=1)
    call("dtype", dtype=3, c=cache(dtype=3))
    call("dtype", dtype=0, c=cache(dtype=3))
    call("n_tok", n=-1)
    call("n_tok", n=1 << 31)
    call("rot_dim", rot=12, rope=FAKE, n_rope=9)
    call("rot_dim", rot=72, rope=FAKE, n_rope=9)
    call("interleaved", inter=2)
    call("come together", rot=64)
    call("come together", rope=FAKE, n_rope=5)
    call("n_rope", rope=FAKE, rot=64, n_rope=-1)
    call("aligned", rope=FAKE + 4, rot=64, n_rope=4)
    call("come together", q=rows())
    call("n_q_heads", q=rows(), q_out=rows(), heads=0)
    call("q_out", q=rows(row_stride=512), q_out=rows(row_stride=192), heads=4)
    call("in place", q=rows(row_stride=512), q_out=rows(), heads=4)
    call("in place", q=rows(row_stride=512), q_out=rows(row_stride=512, head_stride=128), heads=4)
    call("k must", k=None)
    call("v", v=rows(data=FAKE + 2))
    call("16 bytes", k=rows(head_stride=68))
    call("seq and pos", seq=None)
    call("seq and pos", pos=None)
    # nothing to do is no error, whatever the rows are
    r = L.dsim_kv_append(C.byref(cache()), 0, 2, None, None, None, None, 0, None, None, None, 0, 0, 0, None, None)
    assert r == 0


def test_attention_refused(L):
    def call(code, word, dtype=2, q=rows(), out=rows(), heads=4, lens=FAKE, scale=1.0, window=0, ws=FAKE,
             ws_bytes=1 << 40, c=cache()):
        ref = lambda x: None if x is None else C.byref(x)   # noqa: E731
        rc = L.dsim_paged_attention(ref(c), dtype, ref(q), ref(out), heads, lens, scale, window, None, None, ws, ws_bytes,
                                    None)
        assert rc == code and word in dsim.dsim_last_error(), (rc, dsim.dsim_last_error())
    call(-1, "NULL", c=None)
    call(-1, "dtype", dtype=0)
    call(-2, "n_q_heads", heads=3)
    call(-2, "n_q_heads", heads=0)
    call(-2, "n_q_heads", heads=1026)
    call(-1, "scale", scale=float("nan"))
    call(-1, "scale", scale=float("inf"))
    call(-1, "window", window=-1)
    call(-1, "q", q=None)
    call(-1, "out", out=rows(data=0))
    call(-1, "overlap", out=rows(row_stride=0))
    call(-1, "overlap", out=rows(row_stride=128))
    call(-1, "in place", out=rows(row_stride=1024))
    call(-1, "in place", q=rows(row_stride=512), out=rows(row_stride=512, head_stride=128))
    call(-1, "seq_len", lens=None)
    need = L.dsim_paged_attention_workspace(4, 2, 64)
    assert need > 0
    call(-3, "workspace", ws_bytes=need - 1)
    call(-3, "workspace", ws=None)
    call(-1, "aligned", ws=FAKE + 8)
    for bad in ((4, 3, 64), (0, 0, 64), (2, 4, 64), (4, 2, 60), (4, 2, 512), (2048, 2, 64)):
        assert L.dsim_paged_attention_workspace(*bad) == 0
    assert L.dsim_paged_attention(C.byref(cache(n_seq=0)), 2, None, None, 4, None, 1.0, 0, None, None, None, 0, None) == 0


def test_logits_refused(L):
    def call(word, **over):
        d = dict(logits=FAKE, out=FAKE, logits_stride=100, out_stride=100, n_rows=2, vocab=100, dtype=1, history=FAKE,
                 history_len=FAKE, history_stride=5, history_width=5, bias_id=FAKE, bias=FAKE, n_bias=3, mask=FAKE,
                 mask_stride=4)
        d.update(over)
        rc = L.dsim_logit_adjust(C.byref(Logits(**d)), None)
        assert rc < 0 and word in dsim.dsim_last_error(), dsim.dsim_last_error()
    assert L.dsim_logit_adjust(None, None) < 0
    call("dtype", dtype=3)
    call("vocab", vocab=0)
    call("vocab", vocab=(1 << 30) + 1)
    call("n_rows", n_rows=-1)
    call("n_rows", n_rows=1 << 21)
    call("n_bias", n_bias=-1)
    call("n_bias", n_bias=4097)
    call("history_width", history_width=1 << 30)
    call("NULL", logits=0)
    call("NULL", out=0)
    call("overlap", logits_stride=99)
    call("overlap", out_stride=0)
    call("too large", out_stride=1 << 60)
    call("too large", n_rows=1 << 20, vocab=1 << 30, logits_stride=1 << 30, out_stride=1 << 30, mask_stride=1 << 25,
         history_stride=8)
    call("aligned", logits=FAKE + 1)
    call("in place", out_stride=128)
    call("history", history=0)
    call("history", history_len=0)
    call("history", history_stride=4)
    call("history", history=0, history_len=0, presence=FAKE)
    call("bias", bias=0)
    call("bias", bias_id=0)
    call("mask", mask_stride=3)


# ---------------------------------------------------------------------------
# The binding
# ---------------------------------------------------------------------------
def refused(word, fn, *args, **kw):
    with pytest.raises(ValueError) as e:
        fn(*args, **kw)
    assert word in str(e.value), str(e.value)


def append_args(device="cpu", **over):
    z = lambda *s, dtype=F16: torch.zeros(*s, dtype=dtype, device=device)   # noqa: E731
    d = dict(cache=dict(k=z(4, 16, 2, 64), v=z(4, 16, 2, 64)), block_table=z(3, 2, dtype=I32), k=z(5, 2, 64),
             v=z(5, 2, 64), seq=z(5, dtype=I32), pos=z(5, dtype=I32), rope=z(32, 64, dtype=F32), q=z(5, 4, 64),
             q_out=z(5, 4, 64), status=z(5, dtype=I32))
    d.update(over)
    return d


@pytest.mark.parametrize("device", ["cpu", "meta"])
def test_append_binding(device):
    z = lambda *s, dtype=F16: torch.zeros(*s, dtype=dtype, device=device)   # noqa: E731

    def bad(word, **over):
        refused(word, ops.dsim_kv_append, **append_args(device, **over))
    bad("GPU")
    bad("required", cache=dict(k=z(4, 16, 2, 64)))
    bad("dict", cache=None)
    bad("torch tensor", cache=dict(k=5, v=5))
    bad("shape", cache=dict(k=z(4, 16, 128), v=z(4, 16, 128)))
    bad("dtype", cache=dict(k=z(4, 16, 2, 64, dtype=torch.float64), v=z(4, 16, 2, 64)))
    bad("dtype", cache=dict(k=z(4, 16, 2, 64), v=z(4, 16, 2, 64, dtype=BF16)))
    bad("strides", cache=dict(k=z(4, 16, 2, 64), v=z(4, 2, 16, 64).transpose(1, 2)))
    bad("last dimension", cache=dict(k=z(4, 16, 64, 2).transpose(2, 3), v=z(4, 16, 64, 2).transpose(2, 3)))
    bad("shape", cache=dict(k=z(4, 16, 2, 64), v=z(4, 16, 2, 64), k_scale=z(3, dtype=F32)))
    bad("dtype", block_table=z(3, 2, dtype=torch.int64))
    bad("shape", block_table=z(3, dtype=I32))
    bad("shape", k=z(5, 3, 64))
    bad("shape", v=z(4, 2, 64))
    bad("dtype", v=z(5, 2, 64, dtype=F32))
    bad("dtype", k=z(5, 2, 64, dtype=E4M3))
    bad("shape", seq=z(4, dtype=I32))
    bad("dtype", pos=z(5, dtype=torch.int64))
    bad("contiguous", pos=z(10, dtype=I32)[::2])
    bad("required", seq=None)
    bad("together", q_out=None)
    bad("shape", q_out=z(5, 3, 64))
    bad("dtype", q=z(5, 4, 64, dtype=BF16))
    bad("dtype", rope=z(32, 64))
    bad("contiguous", rope=z(64, 32, dtype=F32).t())
    bad("rope", rope=z(32, 128, dtype=F32))
    bad("shape", status=z(6, dtype=I32))


def test_attention_binding():
    z = lambda *s, dtype=F16: torch.zeros(*s, dtype=dtype)   # noqa: E731

    def bad(word, **over):
        d = dict(q=z(3, 4, 64), cache=dict(k=z(4, 16, 2, 64), v=z(4, 16, 2, 64)), block_table=z(3, 2, dtype=I32),
                 seq_len=z(3, dtype=I32), out=z(3, 4, 64), workspace=z(1 << 22, dtype=torch.uint8))
        d.update(over)
        refused(word, ops.dsim_paged_attention, **d)
    bad("GPU")
    bad("GPU", workspace=None)
    bad("shape", q=z(2, 4, 64))
    bad("shape", out=z(3, 2, 64))
    bad("dtype", out=z(3, 4, 64, dtype=BF16))
    bad("shape", seq_len=z(4, dtype=I32))
    bad("dtype", workspace=z(100))
    bad("window", window=-1)
    bad("window", window=1 << 31)
    bad("shape", lse=z(3, 3, dtype=F32))
    bad("contiguous", lse=z(4, 3, dtype=F32).t())
    bad("dtype", status=z(3))
    bad("required", q=None)
    bad("torch tensor", q=None, workspace=None)
    bad("shape", q=z(3, 4), workspace=None)
    bad("dict", cache=None, workspace=None)
    bad("heads", q=z(3, 3, 64), workspace=None)
    with pytest.raises(TypeError):
        ops.dsim_paged_attention(z(3, 4, 64), dict(k=z(4, 16, 2, 64), v=z(4, 16, 2, 64)), z(3, 2, dtype=I32),
                                 z(3, dtype=I32), z(3, 4, 64), scale="x", workspace=z(9, dtype=torch.uint8))


def test_tensors_that_require_a_gradient():
    """No operator has a backward pass: refused while gradients are recorded."""
    q, cache = torch.zeros(3, 4, 64, dtype=F16, requires_grad=True), append_args()["cache"]
    args = dict(q=q * 1, cache=cache, block_table=torch.zeros(3, 2, dtype=I32), seq_len=torch.zeros(3, dtype=I32),
                out=torch.zeros(3, 4, 64, dtype=F16), workspace=torch.zeros(9, dtype=torch.uint8))
    k, x = torch.zeros(5, 2, 64, dtype=F16, requires_grad=True), torch.zeros(2, 100, requires_grad=True)
    for what, fn, kw in (("q", ops.dsim_paged_attention, args), ("k", ops.dsim_kv_append, append_args(k=k)),
                         ("logits", ops.dsim_logit_adjust, dict(logits=x, out=torch.zeros(2, 100))),
                         ("out", ops.dsim_logit_adjust, dict(logits=x.detach(), out=x))):
        refused(what + " requires a gradient", fn, **kw)
        with torch.no_grad():
            refused("GPU", fn, **kw)
        with torch.inference_mode():
            refused("GPU", fn, **kw)


def test_logits_binding():
    z = lambda *s, dtype=F32: torch.zeros(*s, dtype=dtype)   # noqa: E731

    def bad(word, **over):
        d = dict(logits=z(2, 100), out=z(2, 100), history=z(2, 7, dtype=I32), history_len=z(2, dtype=I32),
                 prompt_len=z(2, dtype=I32), repetition=z(2), frequency=z(2), presence=z(2),
                 bias_id=z(2, 3, dtype=I32), bias=z(2, 3), mask=z(2, 4, dtype=I32))
        d.update(over)
        refused(word, ops.dsim_logit_adjust, **d)
    bad("GPU")
    bad("dtype", logits=z(2, 100, dtype=torch.float64))
    bad("shape", out=z(2, 99))
    bad("dtype", out=z(2, 100, dtype=F16))
    bad("last dimension", logits=z(100, 2).t())
    bad("shape", history=z(3, 7, dtype=I32))
    bad("dtype", history=z(2, 7, dtype=torch.int64))
    for name in ("history_len", "prompt_len", "repetition", "frequency", "presence"):
        bad("shape", **{name: z(3, dtype=I32 if name.endswith("len") else F32)})
        bad("dtype", **{name: z(2, dtype=F16)})
    bad("together", bias=None)
    bad("shape", bias=z(2, 4))
    bad("shape", mask=z(2, 3, dtype=I32))


def test_rope_table():
    t = ops.rope_table(5, 8, device="cpu")
    assert t.shape == (5, 8) and t.dtype == F32
    for p in range(5):
        for i in range(4):
            a = torch.tensor(p * 10000.0 ** (-i / 4), dtype=torch.float64)
            assert t[p, i] == a.cos().float() and t[p, 4 + i] == a.sin().float()


# ---------------------------------------------------------------------------
# The plain implementations
# ---------------------------------------------------------------------------
def test_plain_attention_agrees_with_torch():
    g = torch.Generator().manual_seed(0)
    q, keys, values = (torch.randn(*s, generator=g) for s in ((2, 4, 32), (6, 8, 2, 32), (6, 8, 2, 32)))
    table = torch.tensor([[5, 1, 0], [2, 4, 3]], dtype=I32)
    out, lse, bound = plain.attend(q, keys, values, table, torch.tensor([20, 7]), 0.3)
    for b, n in enumerate((20, 7)):
        k, v = (x[table[b].long()].flatten(0, 1)[:n].repeat_interleave(2, dim=1).double() for x in (keys, values))
        ref = torch.nn.functional.scaled_dot_product_attention(q[b][:, None].double(), k.transpose(0, 1),
                                                               v.transpose(0, 1), scale=0.3)[:, 0]
        assert torch.allclose(out[b], ref, rtol=1e-12, atol=1e-12)
        assert torch.allclose(lse[b].exp(), ((k * q[b].double()).sum(-1) * 0.3).exp().sum(0), rtol=1e-12)
    assert (bound > 0).all() and bound.max() < 1e-3


def test_plain_logits_by_hand():
    x = torch.tensor([[1.0, -2.0, 3.0, 4.0, 5.0, -6.0]])
    i = lambda *v: torch.tensor([v], dtype=I32)   # noqa: E731
    f = lambda v: torch.tensor([v])               # noqa: E731
    y = plain.logits(x, history=i(0, 1, 2, 2, 9, 5), prompt_len=i(2)[0], history_len=i(5)[0], repetition=f(2.0),
                     frequency=f(0.5), presence=f(0.25), bias_id=i(3, 3, -1, 2), bias=torch.tensor([[9., 10., 1., 1.]]),
                     mask=i(0b101111))
    # 0, 1: prompt; 2: twice generated, then biased; 3: the last bias; 4: masked; 5: behind the history's end
    assert y.tolist() == [[0.5, -4.0, 3.0 / 2 - (1.0 + 0.25) + 1.0, 14.0, -float("inf"), -6.0]]


def test_plain_append_by_hand():
    keys = torch.zeros(3, 2, 1, 16)
    k = torch.arange(16.0).view(1, 1, 16) + 1
    rope = torch.cat([torch.zeros(2, 4), torch.ones(2, 4)], dim=1)   # a quarter turn
    a = plain.append(keys, keys, torch.tensor([[2, 1]], dtype=I32), k, k, torch.tensor([0]), torch.tensor([1]), rope)
    assert a[0][2, 1, 0].tolist() == [-5., -6., -7., -8., 1., 2., 3., 4.] + list(range(9, 17))
    assert a[1][2, 1, 0].tolist() == list(range(1, 17)) and a[3].tolist() == [0]
    b = plain.append(keys, keys, torch.tensor([[2, 1]], dtype=I32), k, k, torch.tensor([0]), torch.tensor([1]), rope,
                     interleaved=True)
    assert b[0][2, 1, 0, :8].tolist() == [-2., 1., -4., 3., -6., 5., -8., 7.]
    c = plain.append(keys, keys, torch.tensor([[2, 3]], dtype=I32), k, k, torch.tensor([0]), torch.tensor([3]))
    assert c[3].tolist() == [128] and not c[0].any()
