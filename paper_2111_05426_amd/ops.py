"""Python binding of the operators of a single-token step (include/dsim_ops.h)
and of a step of several tokens (include/dsim_multi_ops.h): argument
marshalling only.

* dsim_kv_append: new keys and values rotated by position and written into a
  paged cache, queries rotated on the way;
* dsim_paged_attention: attention of one new token per sequence over it;
* dsim_logit_adjust: penalties for repeated tokens, biases and grammar masks;
* dsim_prompt_attention: attention of the new tokens of prompts, chunks of them
  and packed documents over the cache, their own keys among them;
* dsim_tree_attention: of a tree of drafted tokens over its context and itself;
* dsim_kv_append_axes: the append with the rotation's positions apart from the
  places in the cache, on up to four axes;
* dsim_kv_reserve, dsim_kv_release, dsim_kv_fork, dsim_kv_copy_pages: the pages
  of a cache and who holds them;
* dsim_kv_compact: kept tokens of a sequence move to its front.

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

Pages are dealt out by a pool, and a draft of several tokens per sequence is
checked in one step:

    pool = ops.alloc_page_pool(n_pages, rows)
    ops.dsim_kv_reserve(pool, block_table, 16, seq_len, seq_len + nodes, status)
    ops.dsim_kv_append_axes(cache, block_table, k, v, seq, slot, depth_position, rope, q=q, q_out=q)
    ops.dsim_tree_attention(q, cache, block_table, start, seq_len, tree_mask, out, depth=depth)
    # the accepted path, node numbers in ascending order, moves to the context's end
    ops.dsim_kv_compact(layers, block_table, seq_len, path, n_accepted)
    ops.dsim_kv_release(pool, block_table, 16, row, seq_len + n_accepted)

Every call runs on the device of its tensors, on `stream` (a torch stream or
a raw handle; None: that device's current stream), where its tensors must be
ready.  Like the rest of the binding the calls raise ValueError for tensors
that do not match what the library reads or writes, before any launch, and
DsimError where the library refuses.  None has a derivative: a tensor that
requires a gradient is refused while gradients are recorded, and one that
carries a tangent; what a call writes counts as changed in place.  The checks
and the call are host C++ (binding/, built as _ops.so); there
is no fallback.
"""
from . import dsim
from .dsim import DsimError  # noqa: F401  (what the calls raise)

ST_BAD_PAGE, ST_BAD_POSITION, ST_BAD_SEQUENCE = 128, 256, 512
ST_NO_PAGE, ST_SHARED_PAGE, ST_IN_USE = 1024, 2048, 4096

_native = None


def lib():
    """The compiled binding; raises ImportError if it has not been built."""
    global _native
    if _native is None:
        import torch  # noqa: F401  (the binding and the library use its HIP runtime)
        dsim.lib()
        try:
            from . import _ops
        except ImportError as e:
            raise ImportError("the operators' binding is not built (run python -m paper_2111_05426_amd.build): %s" % e)
        _native = _ops
    return _native


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
    (_native or lib()).kv_append(cache, block_table, k, v, seq, pos, rope, interleaved, q, q_out, status, stream)


def dsim_paged_attention_workspace(n_q_heads, n_heads, head_dim):
    return (_native or lib()).paged_attention_workspace(n_q_heads, n_heads, head_dim)


def alloc_paged_attention_workspace(n_q_heads, n_heads, head_dim, device="cuda"):
    """A caller-owned workspace for dsim_paged_attention (torch uint8)."""
    import torch
    return torch.empty(max(dsim_paged_attention_workspace(n_q_heads, n_heads, head_dim), 16), dtype=torch.uint8,
                       device=device)


def _workspace(q, cache, stream):
    """A workspace for one call, its memory not handed out again before
    `stream` has passed the call."""
    import torch
    if not torch.is_tensor(q):
        raise ValueError("q must be a torch tensor")
    if not isinstance(cache, dict) or not torch.is_tensor(cache.get("k")):
        raise ValueError("cache must be a dict of torch tensors")
    if q.dim() != 3 or cache["k"].dim() != 4:
        raise ValueError("q must have shape (sequences, query heads, head_dim), not %s" % (tuple(q.shape),))
    need = dsim_paged_attention_workspace(q.shape[1], cache["k"].shape[2], q.shape[2])
    if need == 0:
        raise ValueError("q must have a multiple of the cache's heads, heads of a size that the operator takes")
    workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    if stream is not None and q.is_cuda:
        workspace.record_stream(stream if hasattr(stream, "cuda_stream")
                                else torch.cuda.ExternalStream(stream, device=q.device))
    return workspace


def dsim_paged_attention(q, cache, block_table, seq_len, out, scale=None, window=0, workspace=None, lse=None,
                         status=None, stream=None):
    """q, out: (sequences, query heads, head_dim), out may be q; seq_len: int32
    (sequences,), the new token included; scale: None for head_dim^-0.5;
    lse: fp32 (sequences, query heads) or None; status: int32 (sequences,) or
    None; workspace: uint8 of at least dsim_paged_attention_workspace(...)
    bytes (None: one is allocated with torch for this call)."""
    if workspace is None:
        workspace = _workspace(q, cache, stream)
    (_native or lib()).paged_attention(q, cache, block_table, seq_len, out, scale, window, workspace, lse, status,
                                       stream)


def dsim_logit_adjust(logits, out, history=None, prompt_len=None, history_len=None, repetition=None, frequency=None,
                      presence=None, bias_id=None, bias=None, mask=None, stream=None):
    """logits, out: (rows, vocab), out may be logits; history: int32 (rows,
    width) token numbers, of which history_len (rows,) count, the first
    prompt_len (rows,) as the prompt; repetition, frequency, presence: fp32
    (rows,); bias_id, bias: int32 and fp32 (rows, biases); mask: int32 (rows,
    ceil(vocab / 32)), bit t % 32 of word t // 32 set where t is allowed."""
    (_native or lib()).logit_adjust(logits, out, history, prompt_len, history_len, repetition, frequency, presence,
                                    bias_id, bias, mask, stream)


# ---------------------------------------------------------------------------
# A step of several tokens (include/dsim_multi_ops.h)
# ---------------------------------------------------------------------------
def dsim_kv_append_axes(cache, block_table, k, v, seq, slot, pos, rope, sections=None, interleaved=False, q=None,
                        q_out=None, status=None, stream=None):
    """dsim_kv_append with a token's place in the cache, slot: int32 (tokens,),
    apart from what it is rotated by, pos: int32 (tokens, axes).  sections: the
    rotated pairs of each axis, rot_dim / 2 in all (None: one axis); rope and
    pos None: nothing is rotated."""
    (_native or lib()).kv_append_axes(cache, block_table, k, v, seq, slot, pos, rope, sections, interleaved, q, q_out,
                                      status, stream)


def dsim_prompt_attention_workspace(n_tokens, n_seq, n_q_heads, n_heads, head_dim):
    return (_native or lib()).prompt_attention_workspace(n_tokens, n_seq, n_q_heads, n_heads, head_dim)


def alloc_prompt_attention_workspace(n_tokens, n_seq, n_q_heads, n_heads, head_dim, device="cuda"):
    """A caller-owned workspace for dsim_prompt_attention and
    dsim_tree_attention calls of these sizes (torch uint8)."""
    import torch
    return torch.empty(max(dsim_prompt_attention_workspace(n_tokens, n_seq, n_q_heads, n_heads, head_dim), 16),
                       dtype=torch.uint8, device=device)


def _rows_workspace(q, cache, block_table, stream):
    """A workspace for one call, as _workspace."""
    import torch
    if not torch.is_tensor(q) or not torch.is_tensor(block_table):
        raise ValueError("q and block_table must be torch tensors")
    if not isinstance(cache, dict) or not torch.is_tensor(cache.get("k")):
        raise ValueError("cache must be a dict of torch tensors")
    if q.dim() != 3 or cache["k"].dim() != 4 or block_table.dim() != 2:
        raise ValueError("q must have shape (tokens, query heads, head_dim), not %s" % (tuple(q.shape),))
    need = dsim_prompt_attention_workspace(q.shape[0], block_table.shape[0], q.shape[1], cache["k"].shape[2], q.shape[2])
    if need == 0:
        raise ValueError("q must have a multiple of the cache's heads, heads of a size that the operator takes, and "
                         "fewer than 2^31 rows")
    workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    if stream is not None and q.is_cuda:
        workspace.record_stream(stream if hasattr(stream, "cuda_stream")
                                else torch.cuda.ExternalStream(stream, device=q.device))
    return workspace


def dsim_prompt_attention(q, cache, block_table, start, seq_len, out, scale=None, window=0, cap=0.0, slopes=None,
                          prefix_len=None, first_key=None, workspace=None, lse=None, status=None, stream=None):
    """q, out: (tokens, query heads, head_dim), out may be q; start: int32
    (sequences + 1,), tokens start[s] to start[s + 1] - 1 are the last ones of
    sequence s; seq_len: int32 (sequences,), those included; scale: None for
    head_dim^-0.5; cap: scores become cap * tanh(score / cap); slopes: fp32
    (query heads,), of the bias by distance; prefix_len: int32 (sequences,),
    keys that every token sees; first_key: int32 (tokens,), where the token's
    document begins; lse: fp32 (tokens, query heads); status: int32
    (sequences,); workspace: uint8 of at least
    dsim_prompt_attention_workspace(...) bytes (None: one is allocated with
    torch for this call)."""
    if workspace is None:
        workspace = _rows_workspace(q, cache, block_table, stream)
    (_native or lib()).prompt_attention(q, cache, block_table, start, seq_len, out, scale, window, cap, slopes, prefix_len,
                                        first_key, workspace, lse, status, stream)


def dsim_tree_attention(q, cache, block_table, start, context_len, tree_mask, out, depth=None, scale=None, window=0,
                        cap=0.0, slopes=None, workspace=None, lse=None, status=None, stream=None):
    """As dsim_prompt_attention, for drafted tokens whose keys lie behind a
    context of context_len: int32 (sequences,) keys.  tree_mask: int32 (tokens,
    words), bit m % 32 of word m // 32 set where the token attends to node m of
    its sequence; depth: int32 (tokens,), for windows and slopes."""
    if workspace is None:
        workspace = _rows_workspace(q, cache, block_table, stream)
    (_native or lib()).tree_attention(q, cache, block_table, start, context_len, tree_mask, out, depth, scale, window, cap,
                                      slopes, workspace, lse, status, stream)


def alloc_page_pool(n_pages, n_seq, device="cuda"):
    """A pool of n_pages pages that n_seq rows of a block table may hold, all
    of them free: a dict of "refs" (pages,), "free" (bits of the pages that
    nobody holds, in 32-bit words) and "held" (rows,), int32."""
    import torch
    free = torch.full(((n_pages + 31) // 32,), -1, dtype=torch.int32, device=device)
    if n_pages % 32:
        free[-1] = (1 << n_pages % 32) - 1
    return {"refs": torch.zeros(n_pages, dtype=torch.int32, device=device), "free": free,
            "held": torch.zeros(n_seq, dtype=torch.int32, device=device)}


def dsim_kv_reserve(pool, block_table, page_size, seq_len, new_len, status, stream=None):
    """Pages for new_len: int32 (rows,) places in every row (negative: left
    alone), of which seq_len are in use; status: int32 (rows,)."""
    (_native or lib()).kv_reserve(pool, block_table, page_size, seq_len, new_len, status, stream)


def dsim_kv_release(pool, block_table, page_size, row, keep_len, status=None, stream=None):
    """Rows row: int32 (n,) (negative: none) give back what lies behind their
    first keep_len: int32 (n,) places; status: int32 (n,) or None."""
    (_native or lib()).kv_release(pool, block_table, page_size, row, keep_len, status, stream)


def dsim_kv_fork(layers, pool, block_table, seq_len, src, dst, status, stream=None):
    """Rows dst: int32 (n,) become second holders of rows src's seq_len places,
    with copies of pages that end in the middle; layers: a cache or a list of
    them; seq_len: int32 (rows,), set for dst; status: int32 (n,)."""
    (_native or lib()).kv_fork(layers, pool, block_table, seq_len, src, dst, status, stream)


def dsim_kv_copy_pages(layers, src, dst, stream=None):
    """Pages dst: int32 (n,) of every layer become what pages src are."""
    (_native or lib()).kv_copy_pages(layers, src, dst, stream)


def dsim_kv_compact(layers, block_table, start, keep, n_keep, status=None, stream=None):
    """Places start + keep[:, j], j < n_keep, of every sequence move to start +
    j; start, n_keep: int32 (sequences,); keep: int32 (sequences, width),
    ascending; status: int32 (sequences,) or None."""
    (_native or lib()).kv_compact(layers, block_table, start, keep, n_keep, status, stream)
