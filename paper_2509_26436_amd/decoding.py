"""The decoding step on 4-bit operands: MXFP4 quantization and linear layers, rotary positions,
and attention of one new token a sequence over a paged cache; head norms, attention of prompts and of
drafted tokens' trees over the same cache (include/quartz.h, "decoding").

As in the rest of the package, the functions named like the C entry points take raw integers and
return the status code; the tensor helpers check their tensors (``ValueError``), allocate outputs on
the inputs' device (as memory of ``stream``, where one is given) and raise ``QuartzError`` on a
non-OK status.  They launch on the inputs' device, whichever device is current.  Outputs and
workspaces that share memory with an input are a ``ValueError`` too.  Nothing is recorded for
autograd: outputs require no gradient, whatever the inputs do (``rotary(inverse=True)`` is there for
a caller's own backward pass).  The helpers' marshalling is compiled: a decoding step is many calls
of a few microseconds.
"""
from __future__ import annotations

import ctypes

import paper_2509_26436_amd as _q

ROTARY_SCALINGS = ("linear", "base", "parts")

P, I64, I32, F32, F64, SZ = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float,
                             ctypes.c_double, ctypes.c_size_t)
_SIGNATURES = {
    "quartz_mxfp4_quantize": ([P, I64, I64, I64, P, P, P], I32),
    "quartz_mxfp4_dequantize": ([P, P, I64, I64, P, I64, P], I32),
    "quartz_mxfp4_linear": ([P] * 6 + [I64] * 4 + [I32, P], I32),
    "quartz_mxfp4_linear_workspace_bytes": ([I64, I64], SZ),
    "quartz_mxfp4_linear_bf16": ([P, I64, P, P, P, P, I64, I64, I64, I64, I32, P, SZ, P], I32),
    "quartz_mxfp4_linear_kernel": ([I64, I64, I64, P], I32),
    "quartz_rotary_frequencies": ([I64, F64, I32, F64, F64, F64, F64, P], I32),
    "quartz_rotary": ([P, P] + [I64] * 8 + [P, P, I32, I32, F32, P], I32),
    "quartz_paged_append": ([P, P] + [I64] * 7 + [P, P, P, I64, I32, F32, P, P, I32, F32, F32, I64, I64,
                                                  I64, P, I64, I64, I64, P], I32),
    "quartz_paged_attention_workspace_bytes": ([I64] * 7, SZ),
    "quartz_paged_attention": ([P, P] + [I64] * 8 + [P, P, I32, F32, F32, I64, I64, I64, P, I64, I64, P,
                                                     F32, I64, P, SZ, P], I32),
    "quartz_head_norm_rotary": (([P, P] + [I64] * 5 + [P]) * 2 + [I64] * 3 + [P, I64, I64, P, P, I32, I32, F32, F32, P],
                                I32),
    "quartz_paged_prompt_workspace_bytes": ([I64] * 7, SZ),
    "quartz_paged_prompt_attention": ([P, P] + [I64] * 9 + [P, P, I32, F32, F32, I64, I64, I64, P, I64, I64, P, P,
                                                            F32, I64, F32, P, P, P, SZ, P], I32),
    "quartz_paged_tree_attention": ([P, P] + [I64] * 9 + [P, P, I32, F32, F32, I64, I64, I64, P, I64, I64, P, P,
                                                          P, I64, I64, F32, F32, P, SZ, P], I32),
    "quartz_paged_keep": ([P, P, I64, I64, I64, P, P, I32] + [I64] * 5 + [P, I64, I64, P], I32),
}


def bind(lib):
    """Argument types of this module's entry points."""
    for name, (args, result) in _SIGNATURES.items():
        f = getattr(lib, name)
        f.argtypes, f.restype = args, result


# ----------------------------------------------------------- raw C entry points

def quartz_mxfp4_quantize(x, M, K, ldx, codes, scales, stream) -> int:
    return _q.load().quartz_mxfp4_quantize(x, M, K, ldx, codes, scales, stream)


def quartz_mxfp4_dequantize(codes, scales, M, K, y, ldy, stream) -> int:
    return _q.load().quartz_mxfp4_dequantize(codes, scales, M, K, y, ldy, stream)


def quartz_mxfp4_linear(a_codes, a_scales, w_codes, w_scales, bias, y, M, N, K, ldy, epilogue,
                        stream) -> int:
    return _q.load().quartz_mxfp4_linear(a_codes, a_scales, w_codes, w_scales, bias, y, M, N, K, ldy,
                                         epilogue, stream)


def quartz_mxfp4_linear_workspace_bytes(M, K) -> int:
    return int(_q.load().quartz_mxfp4_linear_workspace_bytes(M, K))


def quartz_mxfp4_linear_bf16(x, ldx, w_codes, w_scales, bias, y, M, N, K, ldy, epilogue, workspace,
                             workspace_bytes, stream) -> int:
    return _q.load().quartz_mxfp4_linear_bf16(x, ldx, w_codes, w_scales, bias, y, M, N, K, ldy,
                                              epilogue, workspace, workspace_bytes, stream)


def quartz_mxfp4_linear_kernel(M, N, K, kernel) -> int:
    return _q.load().quartz_mxfp4_linear_kernel(M, N, K, kernel)


def quartz_rotary_frequencies(rot, base, scaling, factor, low, high, original, freqs) -> int:
    return _q.load().quartz_rotary_frequencies(rot, base, scaling, factor, low, high, original, freqs)


def quartz_rotary(x, y, tokens, heads, d, rot, x_token, x_head, y_token, y_head, positions, freqs,
                  layout, inverse, magnitude, stream) -> int:
    return _q.load().quartz_rotary(x, y, tokens, heads, d, rot, x_token, x_head, y_token, y_head,
                                   positions, freqs, layout, inverse, magnitude, stream)


def quartz_paged_append(k, v, tokens, heads, d, k_token, k_head, v_token, v_head, positions, sequences,
                        freqs, rot, layout, magnitude, k_cache, v_cache, cache_type, k_scale, v_scale,
                        pages, page_size, page_stride, table, table_rows, table_pages, table_stride,
                        stream) -> int:
    return _q.load().quartz_paged_append(k, v, tokens, heads, d, k_token, k_head, v_token, v_head,
                                         positions, sequences, freqs, rot, layout, magnitude, k_cache,
                                         v_cache, cache_type, k_scale, v_scale, pages, page_size,
                                         page_stride, table, table_rows, table_pages, table_stride,
                                         stream)


def quartz_paged_attention_workspace_bytes(sequences, heads, kv_heads, d, page_size, table_pages,
                                           window) -> int:
    return int(_q.load().quartz_paged_attention_workspace_bytes(sequences, heads, kv_heads, d, page_size,
                                                                table_pages, window))


def quartz_paged_attention(q, o, sequences, heads, kv_heads, d, q_token, q_head, o_token, o_head,
                           k_cache, v_cache, cache_type, k_scale, v_scale, pages, page_size, page_stride,
                           table, table_pages, table_stride, lengths, scale, window, workspace,
                           workspace_bytes, stream) -> int:
    return _q.load().quartz_paged_attention(q, o, sequences, heads, kv_heads, d, q_token, q_head, o_token,
                                            o_head, k_cache, v_cache, cache_type, k_scale, v_scale, pages,
                                            page_size, page_stride, table, table_pages, table_stride,
                                            lengths, scale, window, workspace, workspace_bytes, stream)


def quartz_head_norm_rotary(q, q_out, q_heads, q_token, q_head, q_out_token, q_out_head, q_weight, k, k_out,
                            k_heads, k_token, k_head, k_out_token, k_out_head, k_weight, tokens, d, rot, positions,
                            axis_count, axis_stride, axes, freqs, layout, norm, eps, magnitude, stream) -> int:
    return _q.load().quartz_head_norm_rotary(q, q_out, q_heads, q_token, q_head, q_out_token, q_out_head, q_weight,
                                             k, k_out, k_heads, k_token, k_head, k_out_token, k_out_head, k_weight,
                                             tokens, d, rot, positions, axis_count, axis_stride, axes, freqs, layout,
                                             norm, eps, magnitude, stream)


def quartz_paged_prompt_workspace_bytes(tokens, sequences, heads, kv_heads, d, page_size, table_pages) -> int:
    return int(_q.load().quartz_paged_prompt_workspace_bytes(tokens, sequences, heads, kv_heads, d, page_size,
                                                             table_pages))


def quartz_paged_prompt_attention(q, o, tokens, sequences, heads, kv_heads, d, q_token, q_head, o_token, o_head,
                                  k_cache, v_cache, cache_type, k_scale, v_scale, pages, page_size, page_stride,
                                  table, table_pages, table_stride, starts, lengths, scale, window, cap, slopes,
                                  prefix, workspace, workspace_bytes, stream) -> int:
    return _q.load().quartz_paged_prompt_attention(q, o, tokens, sequences, heads, kv_heads, d, q_token, q_head,
                                                   o_token, o_head, k_cache, v_cache, cache_type, k_scale, v_scale,
                                                   pages, page_size, page_stride, table, table_pages, table_stride,
                                                   starts, lengths, scale, window, cap, slopes, prefix, workspace,
                                                   workspace_bytes, stream)


def quartz_paged_tree_attention(q, o, tokens, sequences, heads, kv_heads, d, q_token, q_head, o_token, o_head,
                                k_cache, v_cache, cache_type, k_scale, v_scale, pages, page_size, page_stride, table,
                                table_pages, table_stride, starts, lengths, tree, tree_words, tree_stride, scale, cap,
                                workspace, workspace_bytes, stream) -> int:
    return _q.load().quartz_paged_tree_attention(q, o, tokens, sequences, heads, kv_heads, d, q_token, q_head,
                                                 o_token, o_head, k_cache, v_cache, cache_type, k_scale, v_scale,
                                                 pages, page_size, page_stride, table, table_pages, table_stride,
                                                 starts, lengths, tree, tree_words, tree_stride, scale, cap,
                                                 workspace, workspace_bytes, stream)


def quartz_paged_keep(first, kept, sequences, most, kept_stride, k_cache, v_cache, cache_type, heads, d, pages,
                      page_size, page_stride, table, table_pages, table_stride, stream) -> int:
    return _q.load().quartz_paged_keep(first, kept, sequences, most, kept_stride, k_cache, v_cache, cache_type, heads,
                                       d, pages, page_size, page_stride, table, table_pages, table_stride, stream)


# ------------------------------------------------------------------- tensor helpers

_native_module = None


def _native():
    """The compiled half of the helpers (csrc/decoding_binding.cpp); raises if it is missing."""
    global _native_module
    if _native_module is None:
        _q._torch()
        _q.load()
        try:
            from . import _decoding
        except ImportError as e:
            raise RuntimeError("the compiled binding _decoding.so is missing or does not load; build it "
                               "with `python paper_2509_26436_amd/build.py`") from e
        _native_module = _decoding
    return _native_module


class _On:
    """The stream a call was given, as the current one (its device too)."""

    def __init__(self, stream, tensor):
        if tensor.device != stream.device:
            raise ValueError(f"the stream is of {stream.device}, the tensors are on {tensor.device}")
        self._context = _q._torch().cuda.stream(stream)

    def __enter__(self):
        self._context.__enter__()

    def __exit__(self, *error):
        self._context.__exit__(*error)


class MxTensor:
    """An MXFP4 tensor of ``rows`` x ``K`` (include/quartz.h has the format): activations, or a
    linear layer's weight [N, K].  ``codes``: uint8 [K/32, rows, 16], ``scales``: uint8
    [ceil(K/128), rows, 4]."""
    __slots__ = ("codes", "scales", "rows", "K")

    def __init__(self, codes, scales, rows: int, K: int):
        _native().check_mx(codes, scales, rows, K)
        self.codes, self.scales, self.rows, self.K = codes, scales, rows, K

    def __repr__(self):
        return f"MxTensor({self.rows} x {self.K}, {self.codes.device})"


def mxfp4_quantize(x, out: MxTensor | None = None, stream=None) -> MxTensor:
    """bf16 [M, K] (unit column stride, K a multiple of 64, 16-byte aligned rows) to MXFP4:
    activations, or a weight [N, K] once per layer."""
    if stream is not None:
        with _On(stream, x):
            return mxfp4_quantize(x, out)
    if out is None:
        codes, scales = _native().quantize_new(x)
        return MxTensor(codes, scales, *x.shape)
    _native().quantize_into(x, out.codes, out.scales, out.rows, out.K)
    return out


def mxfp4_dequantize(t: MxTensor, out=None, stream=None):
    """The bf16 values [rows, K] that an MXFP4 tensor stands for."""
    if stream is not None:
        with _On(stream, t.codes):
            return mxfp4_dequantize(t, out)
    return _native().dequantize(t.codes, t.scales, t.rows, t.K, out)


def mxfp4_workspace(M: int, K: int, device):
    """Workspace of ``mxfp4_linear`` on bf16 activations [M, K], or None where it needs none."""
    n = quartz_mxfp4_linear_workspace_bytes(M, K)
    return _q._torch().empty((n,), dtype=_q._torch().uint8, device=device) if n else None


def mxfp4_linear(x, w: MxTensor, bias=None, epilogue: int = 0, out=None, stream=None, workspace=None):
    """y bf16 [M, N] = act(x w^T + bias) with both operands in MXFP4: ``x`` an MxTensor, or bf16
    activations [M, K], which the call quantizes (into ``workspace`` from ``mxfp4_workspace``, else
    one of its own; few tokens need none).  Writes ``out``, a bf16 [M, >= N] view with unit column
    stride, if given."""
    if stream is not None:
        with _On(stream, w.codes):
            return mxfp4_linear(x, w, bias, epilogue, out, None, workspace)
    if isinstance(x, MxTensor):
        return _native().linear_mx(x.codes, x.scales, x.rows, x.K, w.codes, w.scales, w.rows, w.K, bias,
                                   epilogue, out)
    return _native().linear_bf16(x, w.codes, w.scales, w.rows, w.K, bias, epilogue, out, workspace)


MX_KERNELS = ("direct", "tiled")


def mxfp4_linear_kernel(M: int, N: int, K: int) -> dict:
    """The kernel that ``mxfp4_linear`` launches for these sizes (quartz_mxfp4_linear_kernel, host
    only): kernel (one of MX_KERNELS), tile rows (tokens) and columns, and whether bf16 activations
    are quantized within it."""
    out = (ctypes.c_int32 * 4)()
    status = quartz_mxfp4_linear_kernel(M, N, K, ctypes.addressof(out))
    if status:
        raise _q.QuartzError(status, "quartz_mxfp4_linear_kernel")
    return {"kernel": MX_KERNELS[out[0]], "rows": out[1], "cols": out[2], "fused": bool(out[3])}


def rotary_frequencies(rot: int, base: float = 10000.0, scaling: str = "linear", factor: float = 1.0,
                       low: float = 1.0, high: float = 32.0, original: float = 4096.0, device="cuda"):
    """Frequencies of ``rot`` rotated channels for ``rotary`` and ``paged_append``: int64 [rot/2],
    turns a position in units of 2^-64, on ``device``.  ``scaling`` and ``factor`` stretch them for
    longer contexts (quartz_rotary_frequencies; low, high and original belong to "parts")."""
    torch = _q._torch()
    if scaling not in ROTARY_SCALINGS:
        raise ValueError(f"scaling must be one of {ROTARY_SCALINGS}")
    host = torch.empty((max(rot, 0) // 2,), dtype=torch.int64)
    status = quartz_rotary_frequencies(rot, base, ROTARY_SCALINGS.index(scaling), factor, low, high,
                                       original, host.data_ptr())
    if status:
        raise _q.QuartzError(status, "quartz_rotary_frequencies")
    return host.to(device)


def rotary(x, positions, freqs, layout: str = "half", inverse: bool = False, magnitude: float = 1.0,
           out=None, stream=None):
    """Rotary positions on x bf16 [tokens, heads, d] (any token and head strides): the first
    2 len(freqs) channels of every head turned by its token's position, the others copied.
    ``positions``: int32 [tokens].  ``layout`` pairs channels: "half" (i, i + len(freqs)) or
    "interleaved" (2i, 2i + 1).  ``inverse=True`` is the transposed map: it takes the gradient of
    the output to that of the input (a caller's own backward pass calls it).  ``out`` may be x."""
    if stream is not None:
        with _On(stream, x):
            return rotary(x, positions, freqs, layout, inverse, magnitude, out)
    return _native().rotary(x, positions, freqs, layout, inverse, magnitude, out)


class PagedCache:
    """A layer's keys and values in pages, [pages, heads, page_size, d] of bf16 or float8_e4m3fn
    (pages may be strided), and the sequences' page table, int32 [sequences, pages of the longest].
    A stored value stands for itself times its scale."""
    __slots__ = ("k", "v", "table", "k_scale", "v_scale")

    def __init__(self, k, v, table, k_scale: float = 1.0, v_scale: float = 1.0):
        _native().check_cache(k, v, table, k_scale, v_scale)
        self.k, self.v, self.table, self.k_scale, self.v_scale = k, v, table, k_scale, v_scale


def paged_append(cache: PagedCache, k, v, positions, sequences=None, freqs=None, layout: str = "half",
                 magnitude: float = 1.0, stream=None) -> None:
    """Writes the keys and values of new tokens, bf16 [tokens, heads, d] (any token and head
    strides), into the places of ``positions`` (int32 [tokens]) of ``sequences`` (int32 [tokens],
    rows of the table; None: token t is of sequence t).  ``freqs`` turns the keys on the way, as
    ``rotary`` does.  Tokens without a place (negative positions, pages that are none) are skipped.
    The cache's keys and values must be distinct memory, and none of the inputs'."""
    if stream is not None:
        with _On(stream, k):
            return paged_append(cache, k, v, positions, sequences, freqs, layout, magnitude)
    _native().append(cache.k, cache.v, cache.table, cache.k_scale, cache.v_scale, k, v, positions, sequences,
                     freqs, layout, magnitude)


def paged_attention_workspace(sequences: int, heads: int, cache: PagedCache, window: int = 0):
    """Workspace of ``paged_attention`` for these sizes, or None where it needs none."""
    _, kv_heads, page, d = cache.k.shape
    torch = _q._torch()
    with torch.cuda.device(cache.k.device):      # sized for its compute units
        n = quartz_paged_attention_workspace_bytes(sequences, heads, kv_heads, d, page, cache.table.shape[1],
                                                   window)
    return torch.empty((n,), dtype=torch.uint8, device=cache.k.device) if n else None


def paged_attention(q, cache: PagedCache, lengths, scale: float | None = None, window: int = 0, out=None,
                    workspace=None, stream=None):
    """Attention of one new token a sequence over the first ``lengths`` (int32 [sequences], on the
    GPU) positions of its pages, or the last ``window`` of them: q bf16 [sequences, heads, d] ->
    bf16 [sequences, heads, d].  heads is a multiple of the cache's heads (neighbouring query heads
    share one); ``scale`` is 1 / sqrt(d) by default.  A sequence of length 0 gives zeros.  The kernel
    is chosen by the table's width (or the window): a table as wide as the longest sequence of a
    few hundred keys takes one launch."""
    if stream is not None:
        with _On(stream, q):
            return paged_attention(q, cache, lengths, scale, window, out, workspace)
    return _native().attention(cache.k, cache.v, cache.table, cache.k_scale, cache.v_scale, q, lengths, scale,
                               window, out, workspace)


def head_norm_rotary(q, k, positions, freqs, q_weight=None, k_weight=None, eps: float | None = 1e-6, axes=None,
                     layout: str = "half", magnitude: float = 1.0, out=None, stream=None):
    """The heads of queries and keys (bf16 [tokens, heads, d], any token and head strides; ``k`` may be
    None), each normed by its root mean square, scaled by its weight (bf16 [d]) and turned as by
    ``rotary``, in one pass: returns both.  ``positions``: int32 [tokens], or [axes, tokens] for
    positions of several axes, of which pair i takes axis ``axes[i]`` (int32 [len(freqs)]; frequencies
    of each axis' own pairs one after the other).  ``eps=None``: turned only.  ``out``: a pair of
    outputs (either may be None, or its input)."""
    if stream is not None:
        with _On(stream, q):
            return head_norm_rotary(q, k, positions, freqs, q_weight, k_weight, eps, axes, layout, magnitude, out)
    q_out, k_out = (None, None) if out is None else out
    return _native().head_norm_rotary(q, k, positions, freqs, q_weight, k_weight, eps, axes, layout, magnitude,
                                      q_out, k_out)


def paged_prompt_workspace(tokens: int, heads: int, cache: PagedCache):
    """Workspace of ``paged_prompt_attention`` and ``paged_tree_attention`` for these sizes, or None
    where they need none."""
    _, kv_heads, page, d = cache.k.shape
    torch = _q._torch()
    with torch.cuda.device(cache.k.device):      # sized for its compute units
        n = quartz_paged_prompt_workspace_bytes(tokens, cache.table.shape[0], heads, kv_heads, d, page,
                                                cache.table.shape[1])
    return torch.empty((n,), dtype=torch.uint8, device=cache.k.device) if n else None


def paged_prompt_attention(q, cache: PagedCache, starts, lengths, scale: float | None = None, window: int = 0,
                           cap: float = 0.0, slopes=None, prefix=None, out=None, workspace=None, stream=None):
    """Attention of the new tokens of prompts over their pages: q bf16 [tokens, heads, d] -> bf16
    [tokens, heads, d].  Sequence b (a row of the table) has the tokens ``starts[b]`` to
    ``starts[b + 1] - 1`` (int32 [sequences + 1]) at the last places of its ``lengths[b]`` (int32
    [sequences]) keys, which ``paged_append`` has written before.  A token sees its own position and
    those before it, the last ``window`` of them if that is set, and the first ``prefix[b]`` (int32
    [sequences]) of its sequence.  ``cap`` caps scores, cap tanh(s / cap); ``slopes`` (fp32 [heads])
    takes slope |distance| off them.  ``scale`` is 1 / sqrt(d) by default.  A token that sees nothing
    gets zeros; rows of no sequence are left as they are."""
    if stream is not None:
        with _On(stream, q):
            return paged_prompt_attention(q, cache, starts, lengths, scale, window, cap, slopes, prefix, out, workspace)
    return _native().prompt_attention(cache.k, cache.v, cache.table, cache.k_scale, cache.v_scale, q, starts, lengths,
                                      None, scale, window, cap, slopes, prefix, out, workspace)


def paged_tree_attention(q, cache: PagedCache, starts, lengths, tree, scale: float | None = None, cap: float = 0.0,
                         out=None, workspace=None, stream=None):
    """Attention of trees of drafted tokens over their pages: as ``paged_prompt_attention``, but a token
    sees every place before its sequence's new ones, and of those the ones whose bits are set in its
    ``tree`` words (int64 [tokens, words]; bit i % 64 of word i // 64: the sequence's new token i, the
    token itself among them).  The nodes of a tree lie in the cache's places one after the other,
    whatever positions their keys were turned by; ``paged_keep`` moves the accepted ones."""
    if stream is not None:
        with _On(stream, q):
            return paged_tree_attention(q, cache, starts, lengths, tree, scale, cap, out, workspace)
    if tree is None:
        raise ValueError("tree must be a tensor")
    return _native().prompt_attention(cache.k, cache.v, cache.table, cache.k_scale, cache.v_scale, q, starts, lengths,
                                      tree, scale, 0, cap, None, None, out, workspace)


def paged_keep(cache: PagedCache, first, kept, stream=None) -> None:
    """Moves the accepted tokens of trees to the places behind their sequences: place ``first[b] +
    kept[b, i]`` to ``first[b] + i`` (int32 [sequences] and [sequences, most], a row of the table a
    sequence), as if all were read before any is written.  Entries below i (-1 where there are no more)
    move nothing."""
    if stream is not None:
        with _On(stream, cache.k):
            return paged_keep(cache, first, kept)
    _native().keep(cache.k, cache.v, cache.table, cache.k_scale, cache.v_scale, first, kept)
