"""Buffer plumbing around include/stem_decode.h: rotary positions, a paged KV cache for what follows a pre-filled prompt, and
decoding steps of many requests that share it.  No arithmetic here."""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import decode_binding as db


class _Turn(torch.autograd.Function):
    """Rotary._run as a node of autograd's graph: the gradients of either map are the other map of the gradients."""

    @staticmethod
    def forward(ctx, rotary, positions, q, k, backward):
        ctx.rotary, ctx.is_backward = rotary, backward
        ctx.save_for_backward(positions)
        ctx.set_materialize_grads(False)
        out = rotary._run(q, k, positions, None, None, backward)
        ctx.mark_non_differentiable(*(y for y, needed in zip(out, ctx.needs_input_grad[2:4]) if y is not None and not needed))
        return out

    @staticmethod
    def backward(ctx, grad_q, grad_k):
        # gradients come with any strides (one number for all rows, for instance): what the library does not take is copied
        grads = [g if g is None or db.usable_rows(g) else g.clone(memory_format=torch.contiguous_format) for g in (grad_q, grad_k)]
        if grads[0] is None and grads[1] is None:
            return None, None, None, None, None
        return (None, None, *_Turn.apply(ctx.rotary, *ctx.saved_tensors, *grads, not ctx.is_backward), None)


class Rotary:
    """Rotary positions of heads of `head_dim` values, of which the first `rotary_dim` turn (None: all), in the "half" or
    "interleaved" layout, with frequencies scaled for long contexts by one of decode_binding.SCALINGS (low, high: as
    stem_rotary_frequencies has them)."""

    def __init__(self, head_dim: int, rotary_dim: Optional[int] = None, theta: float = 10000.0, layout: str = "half",
                 scaling: str = "none", factor: float = 1.0, trained_length: float = 0.0, low: float = 1.0,
                 high: Optional[float] = None, device="cuda"):
        self.head_dim, self.rotary_dim, self.layout = int(head_dim), int(head_dim if rotary_dim is None else rotary_dim), layout
        turns, self.attention_factor = db.stem_rotary_frequencies(self.rotary_dim, theta, scaling, factor, trained_length, low, high)
        if self.rotary_dim > self.head_dim or self.head_dim % 8 or self.head_dim > db.STEM_MAX_HEAD_DIM or layout not in db.LAYOUTS:
            raise ValueError("there are no positions of %d of %d values, layout %r" % (self.rotary_dim, self.head_dim, layout))
        self.turns = turns.to(device)

    @classmethod
    def none(cls, head_dim: int, device="cuda") -> "Rotary":
        """Positions that turn nothing: keys and queries (of finite values) stay as they are."""
        r = cls(head_dim, 2, device=device)
        r.turns.zero_()
        return r

    def _shape(self, q, k, q_out, k_out=None) -> db.RotaryShape:
        shape = db.RotaryShape.from_tensors(q, k, self.rotary_dim, self.layout, q_out, k_out)
        if shape.c.head_dim != self.head_dim:
            raise ValueError("heads of %d values, and positions made for %d" % (shape.c.head_dim, self.head_dim))
        return shape

    def _turn(self, q, k, positions, q_out, k_out, backward: bool) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
        if torch.is_grad_enabled() and any(x is not None and x.requires_grad for x in (q, k)):
            if q_out is not None or k_out is not None:
                raise ValueError("outputs that are given carry no gradients: call under torch.no_grad, or without them")
            return _Turn.apply(self, positions, q, k, backward)
        return self._run(q, k, positions, q_out, k_out, backward)

    def _run(self, q, k, positions, q_out, k_out, backward: bool) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
        q_out = torch.empty_like(q) if q_out is None and q is not None else q_out
        k_out = torch.empty_like(k) if k_out is None and k is not None else k_out
        shape = self._shape(q, k, q_out, k_out)
        db.stem_rotary(shape, q, k, positions, self.turns, self.attention_factor, q_out, k_out, backward)
        return q_out, k_out

    def apply(self, q, k, positions: torch.Tensor, q_out=None, k_out=None):
        """q [T, Hq, d] and k [T, Hkv, d] (either may be None) turned by positions int32 [T]; into new tensors unless q_out and
        k_out are given, which may be q and k themselves.  New tensors carry q's and k's gradients."""
        return self._turn(q, k, positions, q_out, k_out, False)

    def backward(self, grad_q, grad_k, positions: torch.Tensor, grad_q_out=None, grad_k_out=None):
        """The gradients of apply's inputs from those of its outputs."""
        return self._turn(grad_q, grad_k, positions, grad_q_out, grad_k_out, True)


class Turned:
    """Whether the buffers for a prompt's turned queries and keys hold them."""

    def __init__(self, done: bool):
        self.done = done

    def need(self) -> None:
        if not self.done:
            raise RuntimeError("queries and keys have not been turned by their positions: run() or rotate() first")


class PagedCache:
    """Keys and values of up to `requests` requests in `num_pages` pages of `page_size` tokens, at most `pages_per_request` each, with the
    block tables, lengths and free pages that go with them, all on the GPU.  `tokens` is the number of rows of a step's tensors: a step has
    at most that many new tokens.  `position_offset`: the position of a request's first token.  Where it is not given, the first
    StemDecode with rotary positions that is made of the cache sets it to the length of its prefix; a cache that begins before that
    begins at 0.  A cache is one layer's, and its books are its own: each layer of a model has one, and they all take the same steps."""

    def __init__(self, requests: int, num_pages: int, page_size: int, pages_per_request: int, num_kv_heads: int, head_dim: int,
                 tokens: Optional[int] = None, position_offset: Optional[int] = None, dtype: torch.dtype = torch.bfloat16, device="cuda"):
        self.requests, self.tokens = int(requests), int(tokens if tokens is not None else requests)
        if self.tokens > db.MAX_TOKENS:
            raise ValueError("a step has at most %d rows" % db.MAX_TOKENS)
        self.k_pages, self.v_pages = (torch.empty(num_pages, page_size, num_kv_heads, head_dim, dtype=dtype, device=device)
                                      for _ in range(2))
        self.pages = db.PageShape.from_tensors(self.k_pages, self.v_pages)
        self.shape = db.TableShape(requests, page_size, num_pages, pages_per_request, self.tokens, position_offset or 0)
        self._offset_open = position_offset is None        # whether the first position may still be set
        self.offset_given = position_offset is not None
        self.max_suffix = int(pages_per_request) * int(page_size)

        def whole(*sizes, value=0):
            return torch.full(sizes, value, dtype=torch.int32, device=device)

        self.table = whole(self.requests, pages_per_request, value=-1)
        self.lens, self.cu_new, self.status = whole(self.requests), whole(self.requests + 1), whole(4)
        self.positions, self.slots = whole(max(self.tokens, 1)), whole(max(self.tokens, 1), value=-1)
        self.ring = torch.arange(num_pages, dtype=torch.int32, device=device)
        self.ring_state = torch.tensor([0, num_pages], dtype=torch.int32, device=device)
        self.workspace = torch.empty(db.stem_block_table_workspace_bytes(self.shape), dtype=torch.uint8, device=device)

    def advance(self, new_lens: Optional[torch.Tensor] = None, max_new: int = 0) -> None:
        """Room for a step: new_lens int32 [requests] new tokens (None: one each; negative: the request has finished and its pages
        go back), each at most max_new (0: any number).  Brings lens, table, cu_new, positions and slots up to date; a step for which
        there is no room changes none of the first two, has no tokens and says so in status (see refused)."""
        self.shape.c.max_new = max_new
        self._offset_open = False
        db.stem_block_table(self.shape, self.lens, new_lens, self.ring_state, self.ring, self.table, self.lens, self.ring_state,
                            self.cu_new, self.positions, self.slots, self.status, self.workspace)

    def begin_behind(self, length: int) -> None:
        """The requests' first position is `length`, unless another was given when the cache was made.  Raises if the cache has begun, or
        has been set to begin, elsewhere."""
        offset = self.shape.c.position_offset
        if self.offset_given or offset == length:
            return
        if not self._offset_open or offset:
            raise ValueError("the cache's positions begin at %d, behind a prefix of %d tokens" % (offset, length))
        # (the sizes as they would be from the start, which the library may refuse)
        c = self.shape.c
        db.stem_block_table_workspace_bytes(db.TableShape(c.requests, c.page_size, c.num_pages, c.pages_per_request, c.token_capacity, length))
        c.position_offset = length

    def refused(self) -> Tuple[int, int, int, int]:
        """What the last step lacked: pages; requests with unusable lengths, too long for their row or of more new tokens than allowed;
        tokens beyond the step's rows; room for pages given back.  Waits for the GPU."""
        return tuple(self.status.tolist())

    def _rows_shape(self, rotary: Rotary, q, k, v, q_out) -> db.RotaryShape:
        """The shape of a step's rows.  Raises unless they go with the cache and with each other."""
        if k.shape[0] != self.tokens:
            raise ValueError("a step's tensors have %d rows here, as many as the cache was made for" % self.tokens)
        shape = rotary._shape(q, k, q_out)
        if k.dtype != self.k_pages.dtype or k.shape[1:] != self.k_pages.shape[2:]:
            raise ValueError("k does not go with the cache's pages")
        if v.shape != k.shape or v.stride() != k.stride() or v.dtype != k.dtype:
            raise ValueError("v has to be of k's sizes, strides and type")
        dev = self.k_pages.device
        if not k.device == v.device == rotary.turns.device == dev or q is not None and not q.device == q_out.device == dev:
            raise ValueError("a step's tensors have to be on the cache's device")
        db.need_usable_rows(shape, q, k, v, q_out)
        return shape

    def append(self, rotary: Rotary, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
               q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """The step's new rows, q [tokens, Hq, d], k and v [tokens, Hkv, d] in the order of the requests: q and k turned, k and v
        written to the pages.  Rows behind the last new token are left alone."""
        if q is not None and q_out is None:
            q_out = torch.empty_like(q)
        self._write(self._rows_shape(rotary, q, k, v, q_out), rotary, q, k, v, q_out)
        return q_out

    def _write(self, shape: db.RotaryShape, rotary: Rotary, q, k, v, q_out) -> None:
        db.stem_rotary_append(shape, self.pages, q, k, v, self.positions, self.slots, rotary.turns, rotary.attention_factor, q_out,
                              self.k_pages, self.v_pages)


class StemDecode:
    """Decoding steps of the requests of a PagedCache behind a prefix that they share: prefix_k, prefix_v [L, Hkv, d], its keys turned
    already, as StemPrefill leaves them.  With rotary positions, new tokens stand behind the prefix, at L and on, unless the cache was
    made with a position_offset (for keys whose positions do not begin at 0).  One object is one sequence of steps: its buffers
    belong to one step at a time.  A step may be captured into a graph and replayed."""

    def __init__(self, prefix_k: torch.Tensor, prefix_v: torch.Tensor, num_q_heads: int, cache: PagedCache,
                 rotary: Optional[Rotary] = None, max_new: int = 1, softmax_scale: Optional[float] = None,
                 want_lse: bool = False):
        d, dev, dtype = prefix_k.shape[2], prefix_k.device, prefix_k.dtype
        self.prefix_k, self.prefix_v, self.cache = prefix_k, prefix_v, cache
        self.turned = Turned(True)
        self.rotary = rotary if rotary is not None else Rotary.none(d, dev)
        if self.rotary.head_dim != d:
            raise ValueError("heads of %d values, and positions made for %d" % (d, self.rotary.head_dim))
        self.softmax_scale = float(softmax_scale if softmax_scale is not None else d ** -0.5)
        self.max_new = int(max_new)
        self.q = torch.zeros(cache.tokens, num_q_heads, d, dtype=dtype, device=dev)      # turned
        self.out = torch.zeros_like(self.q)
        self.lse = torch.zeros(num_q_heads, cache.tokens, dtype=torch.float32, device=dev) if want_lse else None
        self.shape = db.PrefixShape.from_tensors(self.q, prefix_k, cache.pages, cache.table, max_new, cache.max_suffix)
        # all that the library could refuse of a step, but for its rows: a step that has begun is one that ends
        db.need_usable_prefix(self.shape, prefix_k, prefix_v, self.softmax_scale)
        if any(t.device != cache.k_pages.device for t in (prefix_k, prefix_v, self.rotary.turns)):
            raise ValueError("the prefix and the positions have to be on the cache's device")
        if num_q_heads + 2 * prefix_k.shape[1] > db.MAX_HEADS:
            raise ValueError("a token has at most %d heads in all" % db.MAX_HEADS)
        self.workspace = torch.empty(db.stem_prefix_attn_workspace_bytes(self.shape), dtype=torch.uint8, device=dev)
        if rotary is not None:
            cache.begin_behind(prefix_k.shape[0])

    def attend(self) -> torch.Tensor:
        """Attention of self.q's rows, whose keys and values are in the cache, to the prefix and to their requests' tokens."""
        self.turned.need()
        c = self.cache
        db.stem_prefix_attn(self.shape, self.q, self.prefix_k, self.prefix_v, c.k_pages, c.v_pages, c.table, c.lens, c.cu_new,
                            self.softmax_scale, self.out, self.lse, self.workspace)
        return self.out

    def step(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, new_lens: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One step: room for the new tokens, their keys and values into the cache, their attention.  Rows as in PagedCache.append; a
        step with more than max_new tokens of a request is one without room.  Returns self.out, whose rows behind the last new token
        keep what they held."""
        self.turned.need()
        shape = self.cache._rows_shape(self.rotary, q, k, v, self.q)      # (what it refuses leaves the cache as it was)
        self.cache.advance(new_lens, self.max_new)
        self.cache._write(shape, self.rotary, q, k, v, self.q)
        return self.attend()
