"""Binding of include/mcf_cache.h: what the softmax chain needs around it where keys and values are kept between calls.
Tensors go through the extension module _mcf_cache (csrc/mcf_torch_cache.cpp).

Rows are [tokens, heads, size] (norm_rotate: also [batch, tokens, heads, size]), float16 or bfloat16, with a packed last
dimension and otherwise any strides that are multiples of 8 elements, so that slices of one projection serve as they are.
All calls are asynchronous on `stream` (None: torch's current one) and can be captured into a graph.  The order of another stream behind the
current one is the caller's to see to; the memory of what a call there reads, writes and returns is kept until both streams are through with it.
norm_rotate is recorded for autograd where its operands ask for it; append_cache and cache_attention are not, their results have no gradients.
"""
from typing import NamedTuple

from .binding import McfError, _stream_ptr, load_library

_mod = None
_function = None  # norm_rotate for autograd


class KVCache(NamedTuple):
    """Keys and values in pages of 16, 32, 64 or 128 tokens, 8 bits each: k and v float8_e4m3fn [pages, heads, page_size, size],
    k_scale and v_scale float32 [pages, heads]; what is held is k * k_scale.  Heads of 64, 80, 96, 128, 192 or 256."""
    k: object
    v: object
    k_scale: object
    v_scale: object


def kv_cache(pages, heads, page_size, size, device="cuda"):
    """An empty KVCache."""
    import torch
    return KVCache(*(torch.zeros((pages, heads, page_size, size), dtype=torch.float8_e4m3fn, device=device) for _ in range(2)),
                   *(torch.zeros((pages, heads), dtype=torch.float32, device=device) for _ in range(2)))


def _native():
    """The extension module; raises if it has not been built (there is no fallback path)."""
    global _mod
    if _mod is None:
        import torch  # noqa: F401  (the extension links against its libraries)
        load_library()
        try:
            from . import _mcf_cache
        except ImportError as e:
            raise McfError(-1, f"the extension module _mcf_cache is missing or does not load ({e}): build it with "
                               "`python -m paper_2506_22169_amd.build`; there is no fallback") from e
        _mcf_cache.set_error(McfError)
        _mod = _mcf_cache
    return _mod


def _stream(stream):
    return None if stream is None else _stream_ptr(stream).value or 0


def norm_rotate(q, k=None, cos=None, sin=None, positions=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, q_out=None,
                k_out=None, stream=None):
    """mcf_norm_rotate: for every row of q and k the RMS norm with its weight [size] (None: none), then the rotation by the
    row of cos and sin (float32 [positions, rotary / 2]; None: none) that its position names, in one pass.
    positions: int32 or int64 [tokens] or [batch, tokens]; None counts the tokens of a batch row from 0; one outside of
    the tables gives NaN.  The pairs are (j, j + rotary / 2), or (2j, 2j + 1) with interleaved.  Returns (q_out, k_out), None
    without k; the outputs may be q and k themselves.
    Where q, k or a weight requires a gradient and torch records, the gradients are norm_rotate_backward's, which autograd runs on the stream that was
    torch's current one.  Such a call is refused with q_out or k_out and while its stream is captured: a captured training step calls
    norm_rotate under torch.no_grad() and norm_rotate_backward itself."""
    out = (_mod or _native()).norm_rotate(q, k, cos, sin, positions, q_weight, k_weight, eps, interleaved, q_out, k_out, _stream(stream))
    return out if out is not NotImplemented else _recorded().apply(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, stream)


def _recorded():
    """norm_rotate as a function of autograd's."""
    global _function
    if _function is None:
        import torch

        class NormRotate(torch.autograd.Function):
            @staticmethod
            def forward(ctx, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, stream):
                ctx.save_for_backward(q, k, q_weight, k_weight, cos, sin, positions)
                ctx.rest = eps, interleaved
                return _native().norm_rotate(q, k, cos, sin, positions, q_weight, k_weight, eps, interleaved, None, None, _stream(stream))

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, dq, dk):
                q, k, q_weight, k_weight, cos, sin, positions = ctx.saved_tensors
                if torch.cuda.is_current_stream_capturing():  # (autograd's own streams beside the captured one can end the process)
                    raise McfError(2, "recorded gradients are not captured: norm_rotate_backward is")
                dq, dk = (t if t is None or _laid_out(t) else t.contiguous() for t in (dq, dk))  # (the gradient of a sum is one number, expanded)
                gq, gk, gqw, gkw = norm_rotate_backward(dq, dk, q, k, cos, sin, positions, q_weight, k_weight, *ctx.rest)
                gqw, gkw = (g if g is None else g.to(w.dtype) for g, w in ((gqw, q_weight), (gkw, k_weight)))
                return gq, gk, gqw, gkw, None, None, None, None, None, None

        _function = NormRotate
    return _function


def _laid_out(t):
    """Whether rows have a layout that the calls take."""
    return t.stride(-1) == 1 and t.data_ptr() % 16 == 0 and all(s % 8 == 0 for s, n in zip(t.stride()[:-1], t.shape) if n > 1)


def norm_rotate_backward(dq, dk, q, k=None, cos=None, sin=None, positions=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False,
                         q_out=None, k_out=None, stream=None):
    """mcf_norm_rotate_backward: from the gradients dq, dk of norm_rotate's results and its operands, the gradients
    (of q, of k, of q_weight, of k_weight), the weights' in float32; None for what is not there.  q_out and k_out, where the first
    two go, may be dq and dk."""
    return (_mod or _native()).norm_rotate_backward(dq, dk, q, k, cos, sin, positions, q_weight, k_weight, eps, interleaved, q_out, k_out,
                                                    _stream(stream))


def append_cache(cache, k, v, table, lengths, starts=None, cos=None, sin=None, k_weight=None, q=None, q_weight=None, eps=1e-6,
                 interleaved=False, q_out=None, stream=None):
    """mcf_cache_append: keys and values [tokens, heads, size] of the newest tokens of every sequence go into `cache`, the keys
    normed and rotated as norm_rotate does, with the token's place in its sequence as the position.

    table int32 [sequences, pages]: the pages of each sequence (a number outside of the cache: no page); lengths int32
    [sequences]: its tokens, the new ones the last of them; starts int32 [sequences + 1]: whose rows are whose
    (starts[b] .. starts[b + 1] - 1, ascending; None: one row each).  Rows outside of every sequence are left alone.
    The scale of a page and head is a power of two from its largest value; in a page that holds earlier tokens it only
    grows, and those are rounded again when it does.  A page that is written belongs to one sequence.
    q [tokens, q_heads, size], q_weight: the queries of the same tokens get their norm and rotation in the same launch; returns
    q_out (may be q; rows outside of every sequence are undefined where the call makes it), None without q."""
    return (_mod or _native()).append_cache(cache, k, v, table, lengths, starts, cos, sin, k_weight, q, q_weight, eps, interleaved, q_out,
                                            _stream(stream))


def cache_attention(q, cache, table, lengths, scale, starts=None, causal=True, out=None, stream=None):
    """mcf_cache_attention: softmax(scale Q K^T) V of every row of q [tokens, q_heads, size] over the tokens of its sequence in
    `cache` (table, lengths, starts as append_cache takes them), those up to itself with causal.  Query head h reads head
    h / (q_heads / heads) of the cache.  A row that sees no token is zeros; rows outside of every sequence are left as they were
    in `out` (and are undefined where the call makes it).  One kernel serves a call, by the mean number of rows: single tokens
    against long sequences and long prompts go faster in calls of their own (up to six times: 8 tokens against 130000 beside a prompt of 512)."""
    return (_mod or _native()).cache_attention(q, cache, table, lengths, scale, starts, causal, out, _stream(stream))
