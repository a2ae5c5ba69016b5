"""The operators of a step of several tokens on the host: what
include/dsim_multi_ops.h declares is exported, the C entry points refuse bad
arguments before any launch, the binding refuses tensors that do not match, and
the plain implementations that the GPU tests compare with agree with torch's
own.  CPU only: no call here reaches a GPU."""
import ctypes as C
import math
import os
import re

import pytest
import torch

import multi_ops_plain as plain
from paper_2111_05426_amd import build, dsim, ops
from test_ops import BAD_CACHES, FAKE, Rows, append_args, cache, refused, rows

HEADER = os.path.join(build.INCLUDE, "dsim_multi_ops.h")
F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
I32 = torch.int32
P, I4, I8 = C.c_void_p, C.c_int32, C.c_int64


class Queries(C.Structure):
    _fields_ = [("q", Rows), ("out", Rows), ("n_tok", I8), ("start", P), ("len", P), ("slopes", P), ("lse", P),
                ("status", P), ("workspace", P), ("ws_bytes", C.c_size_t), ("scale", C.c_float), ("cap", C.c_float),
                ("dtype", I4), ("n_q_heads", I4), ("window", I4)]


class Pool(C.Structure):
    _fields_ = [("refs", P), ("free", P), ("held", P), ("block_table", P), ("n_pages", I8), ("table_stride", I8),
                ("n_seq", I4), ("table_width", I4), ("page_size", I4)]


@pytest.fixture(scope="module")
def L():
    ops.lib()
    lib = C.CDLL(dsim.LIB_PATH)
    lib.dsim_kv_append_axes.argtypes = [P, I8, I4, P, P, P, P, I4, P, P, P, I4, P, P, I8, I4, I4, P, P]
    lib.dsim_prompt_attention_workspace.restype = C.c_size_t
    lib.dsim_prompt_attention_workspace.argtypes = [I8, I4, I4, I4, I4]
    lib.dsim_prompt_attention.argtypes = [P, P, P, P, P]
    lib.dsim_tree_attention.argtypes = [P, P, P, I8, I4, P, P]
    lib.dsim_kv_reserve.argtypes = [P, P, P, P, P]
    lib.dsim_kv_release.argtypes = [P, I8, P, P, P, P]
    lib.dsim_kv_fork.argtypes = [P, I4, P, P, I8, P, P, P, P]
    lib.dsim_kv_copy_pages.argtypes = [P, I4, I8, P, P, P]
    lib.dsim_kv_compact.argtypes = [P, I4, P, P, I8, I4, P, P, P]
    return lib


def ref(x):
    return None if x is None else C.byref(x)


def expect(word, rc):
    assert rc < 0 and word in dsim.dsim_last_error(), (rc, word, dsim.dsim_last_error())


def test_exports_every_declared_function(L):
    with open(HEADER) as f:
        names = re.findall(r"DSIM_API\s+[\w\s\*]*?\b(dsim_\w+)\s*\(", f.read())
    assert set(names) == {"dsim_kv_append_axes", "dsim_prompt_attention_workspace", "dsim_prompt_attention",
                          "dsim_tree_attention", "dsim_kv_reserve", "dsim_kv_release", "dsim_kv_fork",
                          "dsim_kv_copy_pages", "dsim_kv_compact"}
    for n in names:
        assert hasattr(L, n) and hasattr(ops, n), n


def queries(**over):
    d = dict(q=rows(), out=rows(data=FAKE << 4), n_tok=5, start=FAKE, len=FAKE, workspace=FAKE, ws_bytes=1 << 40, scale=1.0,
             dtype=2, n_q_heads=4)
    return Queries(**{**d, **over})


BAD_QUERIES = [
    (dict(dtype=1), "dtype"), (dict(dtype=3), "dtype"), (dict(n_q_heads=3), "n_q_heads"), (dict(n_q_heads=0), "n_q_heads"),
    (dict(n_q_heads=1 << 20), "n_q_heads"), (dict(n_tok=-1), "n_tok"), (dict(n_tok=1 << 29), "n_tok"),
    (dict(n_tok=(1 << 29) - 63), "n_tok"), (dict(n_tok=1 << 62), "n_tok"),
    (dict(scale=math.inf), "scale"), (dict(scale=math.nan), "scale"), (dict(scale=-2.0 ** 127), "scale"),
    (dict(cap=-1.0), "cap"), (dict(cap=math.inf), "cap"), (dict(cap=math.nan), "cap"), (dict(cap=2.0 ** -61), "cap"),
    (dict(window=-1), "window"), (dict(q=rows(data=0)), "q"), (dict(q=rows(data=FAKE + 2)), "q"),
    (dict(q=rows(row_stride=-256)), "q"), (dict(q=rows(head_stride=68)), "q"), (dict(out=rows(data=0)), "out"),
    (dict(out=rows(data=FAKE << 4, row_stride=64)), "out"), (dict(out=rows(data=FAKE, row_stride=512)), "in place"),
    (dict(start=0), "start"), (dict(len=0), "len"), (dict(workspace=0), "workspace"), (dict(ws_bytes=100), "workspace"),
    (dict(workspace=FAKE + 8), "aligned")]


@pytest.mark.parametrize("i", range(len(BAD_QUERIES)))
def test_queries_refused(L, i):
    over, word = BAD_QUERIES[i]
    c, q = cache(), queries(**over)
    expect(word, L.dsim_prompt_attention(ref(c), ref(q), None, None, None))
    expect(word, L.dsim_tree_attention(ref(c), ref(q), FAKE, 2, 2, FAKE, None))


@pytest.mark.parametrize("i", range(len(BAD_CACHES)))
def test_cache_refused(L, i):
    over, word = BAD_CACHES[i]
    c, q = cache(**over), queries()
    many = (type(c) * 2)(c, c)
    if not (word == "overlap" and "table_stride" not in over):   # (rows that are only read may)
        expect(word, L.dsim_prompt_attention(ref(c), ref(q), None, None, None))
        expect(word, L.dsim_tree_attention(ref(c), ref(q), FAKE, 2, 2, FAKE, None))
    expect(word, L.dsim_kv_compact(many, 2, FAKE, FAKE, 4, 4, FAKE, None, None))
    r = rows()
    expect(word, L.dsim_kv_append_axes(ref(c), 4, 2, ref(r), ref(r), None, None, 0, FAKE, FAKE, None, 0, None, None, 0, 0, 0,
                                       None, None))
    if not set(over) & {"table_width", "table_stride", "n_seq", "block_table"}:
        expect(word, L.dsim_kv_copy_pages(many, 2, 4, FAKE, FAKE, None))
        expect(word, L.dsim_kv_fork(many, 2, ref(pool()), FAKE, 4, FAKE, FAKE, FAKE, None))


def test_attention_refused(L):
    c, q = cache(), queries()
    expect("cache", L.dsim_prompt_attention(None, ref(q), None, None, None))
    expect("queries", L.dsim_prompt_attention(ref(c), None, None, None, None))
    expect("cache", L.dsim_tree_attention(None, ref(q), FAKE, 2, 2, FAKE, None))
    expect("mask is NULL", L.dsim_tree_attention(ref(c), ref(q), None, 2, 2, FAKE, None))
    expect("mask_words", L.dsim_tree_attention(ref(c), ref(q), FAKE, 2, 0, FAKE, None))
    expect("mask_words", L.dsim_tree_attention(ref(c), ref(q), FAKE, 1 << 27, (1 << 26) + 1, FAKE, None))
    expect("mask", L.dsim_tree_attention(ref(c), ref(q), FAKE, 1, 2, FAKE, None))
    expect("mask", L.dsim_tree_attention(ref(c), ref(q), FAKE, -2, 2, FAKE, None))
    expect("mask", L.dsim_tree_attention(ref(c), ref(q), FAKE, 1 << 61, 2, FAKE, None))
    for over in (dict(window=3), dict(slopes=FAKE)):
        expect("depth", L.dsim_tree_attention(ref(c), ref(queries(**over)), FAKE, 2, 2, None, None))
    # no sequences: nothing to do
    none = cache(n_seq=0)
    assert L.dsim_prompt_attention(ref(none), ref(q), None, None, None) == 0
    assert L.dsim_tree_attention(ref(none), ref(q), FAKE, 2, 2, FAKE, None) == 0


def test_workspace_size(L):
    f = L.dsim_prompt_attention_workspace
    assert f(100, 3, 4, 2, 64) > 0 and f(0, 0, 1, 1, 16) > 0
    for bad in ((-1, 3, 4, 2, 64), (5, -1, 4, 2, 64), (5, (1 << 20) + 1, 4, 2, 64), (5, 3, 4, 3, 64), (5, 3, 0, 0, 64),
                (5, 3, 4, 2, 72), (5, 3, 4, 2, 272), (5, 3, 4, 2, 0), (1 << 29, 3, 4, 2, 64), (1 << 40, 3, 4, 2, 64),
                (5, 3, 2048, 2, 64)):
        assert f(*bad) == 0, bad
    need = f(5, 3, 4, 2, 64)
    c = cache()
    expect("workspace needs %d bytes" % need, L.dsim_prompt_attention(ref(c), ref(queries(ws_bytes=need - 1)), None, None, None))
    # what the blocks need does not shrink with the rows
    assert f(1 << 20, 1, 8, 8, 128) < 1 << 30


def test_axes_refused(L):
    def call(word, n=4, n_axes=2, sections=(16, 16), pos=FAKE, rope=FAKE, n_rope=9, rot=64, seq=FAKE, slot=FAKE):
        s = None if sections is None else (I4 * max(len(sections), 1))(*sections)
        r = rows()
        rc = L.dsim_kv_append_axes(ref(cache()), n, 2, ref(r), ref(r), None, None, 0, seq, slot, pos, n_axes, s, rope, n_rope,
                                   rot, 0, None, None)
        expect(word, rc)
    call("n_axes", n_axes=0)
    call("n_axes", n_axes=5, sections=(8, 8, 8, 4, 4))
    call("sections is NULL", sections=None)
    call("sections must be >= 0", sections=(40, -8))
    call("sum to", sections=(16, 15))
    call("sum to", sections=(2 ** 31 - 1, 2 ** 31 - 1))
    call("pos is NULL", pos=None)
    call("n_tok", n=-1)
    call("seq and pos", seq=None)
    call("rot_dim", rot=12)


def pool(**over):
    d = dict(refs=FAKE, free=FAKE, held=FAKE, block_table=FAKE, n_pages=8, table_stride=4, n_seq=3, table_width=4,
             page_size=16)
    return Pool(**{**d, **over})


BAD_POOLS = [
    (dict(page_size=0), "page_size"), (dict(page_size=(1 << 20) + 1), "page_size"), (dict(n_pages=-1), "n_pages"),
    (dict(n_pages=1 << 31), "n_pages"), (dict(n_seq=-1), "n_seq"), (dict(n_seq=(1 << 20) + 1), "n_seq"),
    (dict(table_width=-1), "table"), (dict(table_stride=3), "overlap"), (dict(table_stride=-4), "table"),
    (dict(table_stride=1 << 61), "table"), (dict(page_size=1 << 20, table_width=1 << 12, table_stride=1 << 12), "2^31"),
    (dict(refs=0), "NULL"), (dict(free=0), "NULL"), (dict(held=0), "NULL"), (dict(block_table=0), "NULL")]


@pytest.mark.parametrize("i", range(len(BAD_POOLS)))
def test_pool_refused(L, i):
    over, word = BAD_POOLS[i]
    p = pool(**over)
    expect(word, L.dsim_kv_reserve(ref(p), FAKE, FAKE, FAKE, None))
    expect(word, L.dsim_kv_release(ref(p), 4, FAKE, FAKE, None, None))
    expect(word, L.dsim_kv_fork(ref(cache()), 1, ref(p), FAKE, 4, FAKE, FAKE, FAKE, None))


def test_pages_refused(L):
    p, c = pool(), cache()
    for at in range(3):
        args = [FAKE if i != at else None for i in range(3)]
        expect("must not be NULL", L.dsim_kv_reserve(ref(p), *args, None))
    expect("pool is NULL", L.dsim_kv_reserve(None, FAKE, FAKE, FAKE, None))
    assert L.dsim_kv_reserve(ref(pool(n_seq=0)), None, None, None, None) == 0
    expect("n must", L.dsim_kv_release(ref(p), -1, FAKE, FAKE, None, None))
    expect("n must", L.dsim_kv_release(ref(p), 1 << 31, FAKE, FAKE, None, None))
    expect("must not be NULL", L.dsim_kv_release(ref(p), 4, None, FAKE, None, None))
    expect("must not be NULL", L.dsim_kv_release(ref(p), 4, FAKE, None, None, None))
    assert L.dsim_kv_release(ref(p), 0, None, None, None, None) == 0

    def fork(word, layers=c, n_layers=1, pool_=p, n=4, args=(FAKE,) * 4):
        expect(word, L.dsim_kv_fork(ref(layers), n_layers, ref(pool_), args[0], n, args[1], args[2], args[3], None))
    fork("layers is NULL", layers=None)
    fork("n_layers", n_layers=0)
    fork("n_layers", n_layers=1025)
    fork("pool is NULL", pool_=None)
    fork("same pages", pool_=pool(n_pages=9))
    fork("same pages", pool_=pool(page_size=8))
    fork("n must", n=-1)
    for at in range(4):
        fork("must not be NULL", args=[FAKE if i != at else None for i in range(4)])
    assert L.dsim_kv_fork(ref(c), 1, ref(p), None, 0, None, None, None, None) == 0

    expect("layers is NULL", L.dsim_kv_copy_pages(None, 1, 4, FAKE, FAKE, None))
    expect("n must", L.dsim_kv_copy_pages(ref(c), 1, -1, FAKE, FAKE, None))
    expect("must not be NULL", L.dsim_kv_copy_pages(ref(c), 1, 4, None, FAKE, None))
    expect("must not be NULL", L.dsim_kv_copy_pages(ref(c), 1, 4, FAKE, None, None))
    assert L.dsim_kv_copy_pages(ref(c), 1, 0, None, None, None) == 0

    def compact(word, start=FAKE, keep=FAKE, stride=4, width=4, n_keep=FAKE, layers=c):
        expect(word, L.dsim_kv_compact(ref(layers), 1, start, keep, stride, width, n_keep, None, None))
    compact("must not be NULL", start=None)
    compact("must not be NULL", keep=None)
    compact("must not be NULL", n_keep=None)
    compact("keep", stride=3)
    compact("keep", stride=-4)
    compact("keep", width=-1)
    compact("keep_width", width=(1 << 30) + 1, stride=1 << 31)
    compact("keep", stride=1 << 61)
    compact("NULL", layers=cache(block_table=0))
    assert L.dsim_kv_compact(ref(cache(n_seq=0)), 1, None, None, 4, 4, None, None, None) == 0


@pytest.mark.parametrize("over", [dict(dtype=1), dict(n_heads=1), dict(head_dim=32), dict(page_size=8), dict(n_pages=7),
                                  dict(page_stride=4096), dict(head_stride=2048, page_stride=4096)])
def test_layers_that_differ(L, over):
    many = (type(cache()) * 3)(cache(), cache(), cache(**over))
    expect("same shape", L.dsim_kv_copy_pages(many, 3, 4, FAKE, FAKE, None))
    expect("same shape", L.dsim_kv_compact(many, 3, FAKE, FAKE, 4, 4, FAKE, None, None))


# ---------------------------------------------------------------------------
# The binding
# ---------------------------------------------------------------------------
def z(*s, dtype=F16):
    return torch.zeros(*s, dtype=dtype)


def attention_args(tree, **over):
    d = dict(q=z(5, 4, 64), cache=dict(k=z(4, 16, 2, 64), v=z(4, 16, 2, 64)), block_table=z(3, 2, dtype=I32),
             start=z(4, dtype=I32), out=z(5, 4, 64), workspace=z(1 << 20, dtype=torch.uint8))
    d.update(dict(context_len=z(3, dtype=I32), tree_mask=z(5, 1, dtype=I32)) if tree else dict(seq_len=z(3, dtype=I32)))
    return {**d, **over}


@pytest.mark.parametrize("tree", [False, True])
def test_attention_binding(tree):
    fn = ops.dsim_tree_attention if tree else ops.dsim_prompt_attention

    def bad(word, **over):
        refused(word, fn, **attention_args(tree, **over))
    bad("GPU")
    bad("GPU", workspace=None)
    bad("shape", q=z(5, 4, 32))
    bad("shape", q=z(4, 64))
    bad("shape", out=z(5, 2, 64))
    bad("dtype", out=z(5, 4, 64, dtype=BF16))
    bad("dtype", q=z(5, 4, 64, dtype=E4M3))
    bad("shape", start=z(3, dtype=I32))
    bad("dtype", start=z(4, dtype=torch.int64))
    bad("shape", **{"context_len" if tree else "seq_len": z(4, dtype=I32)})
    bad("shape", slopes=z(3, dtype=F32))
    bad("dtype", slopes=z(4))
    bad("dtype", workspace=z(100))
    bad("window", window=-1)
    bad("window", window=1 << 31)
    bad("cap", cap=math.nan)
    bad("scale", scale=math.nan)
    bad("shape", lse=z(5, 3, dtype=F32))
    bad("contiguous", lse=z(4, 5, dtype=F32).t())
    bad("shape", status=z(5, dtype=I32))
    bad("required", q=None)
    bad("torch tensor", q=None, workspace=None)
    bad("dict", cache=None, workspace=None)
    bad("shape", q=z(5, 4), workspace=None)
    bad("heads", q=z(5, 3, 64), workspace=None)
    if tree:
        bad("shape", tree_mask=z(4, 1, dtype=I32))
        bad("dtype", tree_mask=z(5, 1, dtype=torch.int64))
        bad("shape", depth=z(4, dtype=I32))
        bad("required", tree_mask=None)
    else:
        bad("shape", prefix_len=z(5, dtype=I32))
        bad("shape", first_key=z(3, dtype=I32))
        bad("dtype", first_key=z(5, dtype=torch.int64))
    with pytest.raises(TypeError):
        fn(**attention_args(tree, scale="x"))


def test_workspace_binding():
    assert ops.dsim_prompt_attention_workspace(5, 3, 4, 2, 64) > 0
    assert ops.dsim_prompt_attention_workspace(-5, 3, 4, 2, 64) == 0
    assert ops.dsim_prompt_attention_workspace(5, 1 << 40, 4, 2, 64) == 0
    assert ops.alloc_prompt_attention_workspace(5, 3, 4, 2, 64, device="cpu").dtype == torch.uint8


def axes_args(**over):
    a = append_args()
    a["slot"], a["pos"] = a.pop("pos"), z(5, 2, dtype=I32)
    return {**a, "sections": (20, 12), **over}


def test_axes_binding():
    def bad(word, **over):
        refused(word, ops.dsim_kv_append_axes, **axes_args(**over))
    bad("GPU")
    bad("GPU", rope=None, pos=None, sections=None)
    bad("shape", slot=z(4, dtype=I32))
    bad("shape", pos=z(5, dtype=I32))
    bad("shape", pos=z(4, 2, dtype=I32))
    bad("columns", pos=z(5, 5, dtype=I32), sections=(8, 8, 8, 4, 4))
    bad("columns", pos=z(5, 0, dtype=I32), sections=())
    bad("contiguous", pos=z(2, 5, dtype=I32).t())
    bad("dtype", pos=z(5, 2, dtype=torch.int64))
    bad("required", pos=None)
    bad("required with several", sections=None)
    bad("entry for each", sections=(32,))
    bad("need rope", rope=None)
    bad("need rope", rope=None, pos=None)
    bad("rope", rope=z(32, 0, dtype=F32))
    bad("together", q_out=None)
    with pytest.raises(TypeError):
        ops.dsim_kv_append_axes(**axes_args(sections=5))
    with pytest.raises(TypeError):
        ops.dsim_kv_append_axes(**axes_args(sections=("a", "b")))


def test_pages_binding():
    def pool_(**over):
        return {**dict(refs=z(40, dtype=I32), free=z(2, dtype=I32), held=z(3, dtype=I32)), **over}
    table, three, four = z(3, 2, dtype=I32), z(3, dtype=I32), z(4, dtype=I32)
    layer = dict(k=z(40, 16, 2, 64), v=z(40, 16, 2, 64))

    def reserve(word, pool=None, block_table=table, page_size=16, seq_len=three, new_len=three, status=three):
        refused(word, ops.dsim_kv_reserve, pool or pool_(), block_table, page_size, seq_len, new_len, status)
    reserve("GPU")
    refused("dict", ops.dsim_kv_reserve, None, table, 16, three, three, three)
    reserve("required", pool=dict(refs=three))
    reserve("shape", pool=pool_(free=three))
    reserve("shape", pool=pool_(held=four))
    reserve("dtype", pool=pool_(refs=z(40)))
    reserve("contiguous", pool=pool_(refs=z(80, dtype=I32)[::2]))
    reserve("dtype", block_table=z(3, 2))
    reserve("page_size", page_size=0)
    reserve("page_size", page_size=1 << 40)
    reserve("shape", seq_len=four)
    reserve("shape", new_len=four)
    reserve("required", status=None)
    with pytest.raises(TypeError):
        ops.dsim_kv_reserve(pool_(), table, "x", three, three, three)

    refused("GPU", ops.dsim_kv_release, pool_(), table, 16, four, four)
    refused("shape", ops.dsim_kv_release, pool_(), table, 16, four, three)
    refused("shape", ops.dsim_kv_release, pool_(), table, 16, four, four, three)
    refused("dtype", ops.dsim_kv_release, pool_(), table, 16, z(4), four)

    def fork(word, layers=layer, pool=None, src=four, dst=four, status=four, seq_len=three):
        refused(word, ops.dsim_kv_fork, layers, pool or pool_(), table, seq_len, src, dst, status)
    fork("GPU")
    fork("GPU", layers=[layer, layer])
    fork("layers", layers=[])
    fork("layers", layers=None)
    fork("dict", layers=[layer, None])
    fork("shape", dst=three)
    fork("required", status=None)
    fork("shape", seq_len=four)

    refused("GPU", ops.dsim_kv_copy_pages, layer, four, four)
    refused("shape", ops.dsim_kv_copy_pages, layer, four, three)
    refused("GPU", ops.dsim_kv_compact, (layer,), table, three, z(3, 5, dtype=I32), three)
    refused("shape", ops.dsim_kv_compact, layer, table, three, z(4, 5, dtype=I32), three)
    refused("shape", ops.dsim_kv_compact, layer, table, four, z(3, 5, dtype=I32), three)
    refused("last dimension", ops.dsim_kv_compact, layer, table, three, z(5, 3, dtype=I32).t(), three)
    refused("shape", ops.dsim_kv_compact, layer, table, three, z(3, 5, dtype=I32), three, four)


def calls():
    """Each operator with its arguments and a name of a floating one."""
    table, three = z(3, 2, dtype=I32), z(3, dtype=I32)
    return [(ops.dsim_prompt_attention, attention_args(False), "q"), (ops.dsim_tree_attention, attention_args(True), "q"),
            (ops.dsim_kv_append_axes, axes_args(), "k"),
            (ops.dsim_prompt_attention, attention_args(False, slopes=z(4, dtype=F32)), "slopes")], table, three


def test_tensors_that_require_a_gradient():
    """No operator has a backward pass: refused while gradients are recorded."""
    for fn, kw, name in calls()[0]:
        x = kw[name].clone().requires_grad_()
        refused(name + " requires a gradient", fn, **{**kw, name: x})
        with torch.no_grad():
            refused("GPU", fn, **{**kw, name: x})
    table, three = calls()[1:]
    layer = dict(k=z(4, 16, 2, 64).requires_grad_(), v=z(4, 16, 2, 64))
    refused("requires a gradient", ops.dsim_kv_copy_pages, layer, three, three)
    refused("requires a gradient", ops.dsim_kv_compact, layer, table, three, z(3, 5, dtype=I32), three)


def test_tensors_that_carry_a_tangent():
    import torch.autograd.forward_ad as forward
    with forward.dual_level():
        for fn, kw, name in calls()[0]:
            dual = forward.make_dual(kw[name], torch.ones_like(kw[name]))
            refused(name + " carries a tangent", fn, **{**kw, name: dual})


# ---------------------------------------------------------------------------
# The plain implementations
# ---------------------------------------------------------------------------
def test_plain_prompt_agrees_with_torch():
    g = torch.Generator().manual_seed(0)
    n, d = 11, 16
    q, k, v = (torch.randn(n, h, d, generator=g, dtype=torch.float64) for h in (4, 2, 2))
    table = torch.tensor([[1, 0, 2]], dtype=I32)
    keys, values = (torch.zeros(4, 4, 2, d, dtype=torch.float64) for _ in range(2))
    for j in range(n):
        keys[table[0, j // 4], j % 4], values[table[0, j // 4], j % 4] = k[j], v[j]
    out, lse, _, _, seen = plain.attention(q, keys, values, table, torch.tensor([0, n]), torch.tensor([n]), d ** -0.5)
    want = torch.nn.functional.scaled_dot_product_attention(
        q.transpose(0, 1), k.transpose(0, 1).repeat_interleave(2, 0), v.transpose(0, 1).repeat_interleave(2, 0), is_causal=True)
    assert seen.all() and torch.allclose(out, want.transpose(0, 1), atol=1e-12)
    # a chain of drafted tokens is a prompt's end
    sees = torch.tril(torch.ones(5, 5)).long()
    mask = (sees << torch.arange(5)).sum(1, keepdim=True).to(I32)
    tree, tree_lse, _, _, _ = plain.attention(q[6:], keys, values, table, torch.tensor([0, 5]), torch.tensor([6]), d ** -0.5,
                                              tree_mask=mask, depth=torch.arange(5))
    assert torch.allclose(tree, out[6:], atol=1e-12) and torch.allclose(tree_lse, lse[6:], atol=1e-12)


def test_plain_masks_by_hand():
    _, lo, hi = plain.ranges(3, 5, 0, 2, None)
    assert lo.tolist() == [1, 2, 3] and hi.tolist() == [3, 4, 5]
    _, lo, hi = plain.ranges(3, 5, 4, 0, torch.tensor([-2, 3, 9]))
    assert lo.tolist() == [0, 3, 9] and hi.tolist() == [4, 4, 5]
    assert plain.bits(torch.tensor([[5, -(1 << 31)]], dtype=I32), 64)[0].nonzero().flatten().tolist() == [0, 2, 63]


def test_plain_compact_by_hand():
    x = torch.arange(8.0).view(2, 4, 1)
    status = plain.compact([x], torch.tensor([[1, 0]], dtype=I32), torch.tensor([1]), torch.tensor([[1, 3, 6, 2]]), torch.tensor([4]))
    # places 0 to 7 hold 4 5 6 7 0 1 2 3; 2, 4 and 7 move to 1, 2 and 3
    assert x.flatten().tolist() == [0, 1, 2, 3, 4, 6, 0, 3] and status.tolist() == [256]
