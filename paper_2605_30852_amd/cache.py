"""A paged KV cache of several sequences: the spd_cache calls of include/spd.h over torch tensors.

PyTorch only allocates device memory and provides the current stream; every computation runs in libspd.so.
Index arguments are int32 tensors on the cache's device, and every call is asynchronous on that device's current
stream, so a run of calls can be captured into a graph."""
from __future__ import annotations

import ctypes as ct
from typing import Optional, Tuple

import torch

from . import binding as B

PAGE = 16
_FORK_WORKSPACE = 256
_DTYPES = {torch.float32: B.SPD_F32, torch.bfloat16: B.SPD_BF16}


def _optional(name: str, t: Optional[torch.Tensor], dtype: torch.dtype, size: Optional[int] = None, gpu: Optional[int] = None) -> int:
    """A rule's tensor, of any size on any GPU where a call has not said which."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.dim() != 1 or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of one dimension on a GPU")
    if size is not None and (t.shape[0] != size or t.get_device() != gpu):
        raise ValueError(f"the rule's {name} must have {size} entries on the cache's device")
    return t.data_ptr()


class _Rule:
    """Attributes that may be set anew between calls, and the structs made of them that calls pass on: none outlives a change of an
    attribute, a struct is never written again, and one made beside a change goes into the dict that the change has replaced."""

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        self.__dict__["_made"] = {}


def _lies(t: Optional[torch.Tensor], at: Optional[int], size: Optional[int], gpu: Optional[int]) -> bool:
    """Whether a rule's tensor, of so many entries on this GPU, still lies where the struct says."""
    return t is None or (t.data_ptr() == at and t.shape[0] == size and t.get_device() == gpu)


class AttentionRule(_Rule):
    """A rule for `prompt_attention` and `prefix_attention`. The row of key p sees the first open_lens[i] keys of its sequence
    (batch sequence i; also those behind p), and the keys of [max(first[row], p - window + 1), p]: `first` gives each row the
    first key of its document (one behind p: a padding row), window 0 is none. cap: a score s becomes cap tanh(s / cap), 0: not.
    slopes: fp32 [heads], slopes[head] |p - key| is taken from it. Index tensors are int32; the tensors stay the caller's and are
    read by every call under the rule; attributes may be set anew between calls."""

    def __init__(self, cap: float = 0.0, slopes: Optional[torch.Tensor] = None, window: int = 0,
                 first: Optional[torch.Tensor] = None, open_lens: Optional[torch.Tensor] = None):
        self.cap, self.window, self.slopes, self.first, self.open_lens = cap, window, slopes, first, open_lens
        self.check()

    def check(self, rows: Optional[int] = None, seqs: Optional[int] = None, heads: Optional[int] = None,
              gpu: Optional[int] = None) -> "B.spd_attention_rule":
        """What a call of so many rows, sequences and heads passes on: the attributes as they are now."""
        made = self._made
        c = made.get(0)
        slopes, first, opened = self.slopes, self.first, self.open_lens
        if c is not None and _lies(slopes, c.slopes, heads, gpu) and _lies(first, c.first, rows, gpu) and _lies(opened, c.open_lens, seqs, gpu):
            return c
        cap, window = self.cap, self.window
        if not (cap == 0 or 2.0 ** -20 <= cap <= 2.0 ** 20):
            raise ValueError("cap must be 0 or in [2^-20, 2^20]")
        if not 0 <= window < 1 << 31:
            raise ValueError("window must be in [0, 2^31)")
        c = made[0] = B.spd_attention_rule(cap, window, _optional("slopes", slopes, torch.float32, heads, gpu),
                                           _optional("first", first, torch.int32, rows, gpu),
                                           _optional("open_lens", opened, torch.int32, seqs, gpu))
        return c


class HeadRule(_Rule):
    """What `append_heads` makes of the heads of q and k: x / sqrt(mean(x^2) + eps) * gain (fp32 [head_dim]; None: as it is), then
    the rotation of its first dims, in half layout (dims i and i + half of them) or interleaved (2i and 2i + 1)."""

    def __init__(self, q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None, eps: float = 1e-6,
                 interleaved: bool = False):
        self.q_gain, self.k_gain, self.eps, self.interleaved = q_gain, k_gain, eps, interleaved
        self.check()

    def check(self, head_dim: Optional[int] = None, gpu: Optional[int] = None, rot: int = 0) -> "B.spd_head_rule":
        """What a call with heads of head_dim passes on, rot dims of which turn: the attributes as they are now."""
        made = self._made
        c = made.get(rot)
        q_gain, k_gain = self.q_gain, self.k_gain
        if c is None or not (_lies(q_gain, c.q_gain, head_dim, gpu) and _lies(k_gain, c.k_gain, head_dim, gpu)):
            c = made[rot] = B.spd_head_rule(_optional("q_gain", q_gain, torch.float32, head_dim, gpu),
                                            _optional("k_gain", k_gain, torch.float32, head_dim, gpu), self.eps, rot,
                                            1 if self.interleaved else 0)
        return c


class PagedCache:
    """kv: [layers][pages][2][KV heads][16][head_dim] (fp32 or bf16); page_table: int32 [sequences][pages of one];
    lens: int32 [sequences]; refs: int32 [pages], or None if no call changes the pages. The tensors stay the
    caller's, and hold the state: sequence s has lens[s] keys, in the pages of its row of the table."""

    def __init__(self, kv: torch.Tensor, page_table: torch.Tensor, lens: torch.Tensor,
                 refs: Optional[torch.Tensor] = None):
        if kv.dim() != 6 or kv.shape[2] != 2 or kv.shape[4] != PAGE or kv.dtype not in _DTYPES:
            raise ValueError("kv must be a float32 or bfloat16 tensor [layers][pages][2][KV heads][16][head_dim]")
        if not kv.is_cuda or not kv.is_contiguous():
            raise ValueError("kv must be contiguous, on a GPU")
        self.kv, self.page_table, self.lens, self.refs = kv, page_table, lens, refs
        self.device = kv.device
        self._gpu = kv.get_device()
        self.n_layers, self.num_pages, _, self.n_kv_heads, _, self.head_dim = kv.shape
        self._index("page_table", page_table, 2)
        self.max_seqs, self.max_pages = page_table.shape
        self._index("lens", lens, 1, self.max_seqs)
        if refs is not None:
            self._index("refs", refs, 1, self.num_pages)
        self.c = B.spd_cache(kv.data_ptr(), page_table.data_ptr(), lens.data_ptr(), refs.data_ptr() if refs is not None else None,
                             self.n_layers, self.num_pages, self.max_seqs, self.max_pages, self.n_kv_heads, self.head_dim,
                             _DTYPES[kv.dtype])
        B.spd_cache_workspace(self.c, 1)  # checks the description
        self._ws_bytes = {}

    @classmethod
    def empty(cls, n_layers: int, num_pages: int, n_kv_heads: int, head_dim: int, max_seqs: int, max_pages: int,
              dtype: torch.dtype = torch.bfloat16, device="cuda") -> "PagedCache":
        """A cache without sequences; the pages' contents are whatever the memory held."""
        i32 = dict(dtype=torch.int32, device=device)
        return cls(torch.empty((n_layers, num_pages, 2, n_kv_heads, PAGE, head_dim), dtype=dtype, device=device),
                   torch.full((max_seqs, max_pages), -1, **i32), torch.zeros(max_seqs, **i32), torch.zeros(num_pages, **i32))

    # ------------------------------------------------------------------------------------------------ pages
    def reserve(self, seqs: torch.Tensor, add: torch.Tensor) -> torch.Tensor:
        """Sequence seqs[i] grows by add[i] keys; returns the status word (int32[1], SPD_CACHE_DONE or why nothing
        changed). A page that others hold too is copied before its sequence writes into it."""
        n = self._entries(seqs, add)
        return self._change(n, lambda st, ws, wb, s: B.spd_cache_reserve(self.c, seqs.data_ptr(), add.data_ptr(), n, st, ws, wb, s))

    def fork(self, src: torch.Tensor, dst: torch.Tensor, keep: torch.Tensor) -> torch.Tensor:
        """The empty sequence dst[i] becomes the first keep[i] keys of src[i], sharing its pages; returns the status."""
        n = self._entries(src, dst, keep)
        return self._change(n, lambda st, ws, wb, s: B.spd_cache_fork(self.c, src.data_ptr(), dst.data_ptr(), keep.data_ptr(), n,
                                                                      st, ws, wb, s), _FORK_WORKSPACE)

    def truncate(self, seqs: torch.Tensor, keep: torch.Tensor) -> torch.Tensor:
        """Sequence seqs[i] keeps its first keep[i] keys (0: none) and lets go of its other pages; returns the status."""
        n = self._entries(seqs, keep)
        return self._change(n, lambda st, ws, wb, s: B.spd_cache_truncate(self.c, seqs.data_ptr(), keep.data_ptr(), n, st, ws, wb, s), 0)

    def compact(self) -> torch.Tensor:
        """Moves the held pages to the lowest ids; returns their number (int32[1])."""
        return self._change(1, lambda live, ws, wb, s: B.spd_cache_compact(self.c, live, ws, wb, s))

    # ------------------------------------------------------------------------------------------------ rows
    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, seqs: torch.Tensor, cu_rows: torch.Tensor,
               q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
               rope: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Optional[torch.Tensor]:
        """Writes a batch's rows k, v [rows][KV heads][head_dim] into their pages. rope: (cos, sin), fp32
        [positions][head_dim / 2], rotates k and, if given, q [rows][heads][head_dim], which is returned (in q_out, or a new tensor)."""
        return self._append(layer, k, v, seqs, cu_rows, q, q_out, rope, None)

    def append_heads(self, layer: int, k: torch.Tensor, v: torch.Tensor, seqs: torch.Tensor, cu_rows: torch.Tensor, rule: HeadRule,
                     q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                     rope: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Optional[torch.Tensor]:
        """`append` with the rule's norms of the heads of k and q, and its rotation: rope is (cos, sin), fp32 [positions][half of
        the dims that turn], the first ones of a head, a multiple of 16."""
        return self._append(layer, k, v, seqs, cu_rows, q, q_out, rope, rule)

    def _append(self, layer, k, v, seqs, cu_rows, q, q_out, rope, rule):
        rows, n = k.shape[0], self._batch(seqs, cu_rows)
        ks, vs = self._rows("k", k, rows, k.dtype, self.n_kv_heads), self._rows("v", v, rows, k.dtype, self.n_kv_heads)
        qp = op = qs = os_ = hq = 0
        if q is not None:
            hq = q.shape[1] if q.dim() == 3 else 0
            qs = self._rows("q", q, rows, k.dtype, hq)
            if q_out is None:
                q_out, os_ = torch.empty(q.shape, dtype=q.dtype, device=self.device), hq * self.head_dim
            else:
                os_ = self._rows("q_out", q_out, rows, k.dtype, hq)
            qp, op = q.data_ptr(), q_out.data_ptr()
        elif q_out is not None:
            raise ValueError("q_out without q")
        cos = sin = places = half = 0
        if rope is not None:
            places, half = rope[0].shape[0], self.head_dim // 2 if rule is None or rope[0].dim() != 2 else rope[0].shape[1]
            for x in rope:
                if x.dtype is not torch.float32 or x.shape != (places, half) or x.get_device() != self._gpu or not x.is_contiguous():
                    raise ValueError("rope must be two contiguous float32 tensors [positions][head_dim / 2] on the cache's device")
            cos, sin = rope[0].data_ptr(), rope[1].data_ptr()
        if rule is not None:
            r = rule.check(self.head_dim, self._gpu, 2 * half)
            if rows:
                self._on_device(lambda s: B.spd_cache_append_heads(self.c, layer, k.data_ptr(), ks, v.data_ptr(), vs, qp, qs, op, os_,
                                                                   hq, _DTYPES[k.dtype], r, cos, sin, places, seqs.data_ptr(),
                                                                   cu_rows.data_ptr(), n, rows, s))
        elif rows:
            self._on_device(lambda s: B.spd_cache_append(self.c, layer, k.data_ptr(), ks, v.data_ptr(), vs, qp, qs, op, os_, hq,
                                                         _DTYPES[k.dtype], cos, sin, places, seqs.data_ptr(), cu_rows.data_ptr(),
                                                         n, rows, s))
        return q_out

    def prompt_attention(self, layer: int, q: torch.Tensor, seqs: torch.Tensor, cu_rows: torch.Tensor,
                         out: Optional[torch.Tensor] = None, max_len: int = 0, rule: Optional[AttentionRule] = None) -> torch.Tensor:
        """Causal attention of a batch's packed rows q [rows][heads][head_dim], the newest keys of their sequences.
        fp32 q: any cache, fp32 arithmetic; bf16 q: a bf16 cache, and the probabilities are rounded to bf16 as the output is.
        max_len: keys of the longest sequence, if known. Rows of `out` behind the last sequence are left as they are.
        rule: which keys a row sees, and what becomes of its scores (its tensors: [rows] and [sequences] of this batch); bf16 q: the
        tanh of a cap up to 55 is right to 4e-5 of itself."""
        rows, n = q.shape[0], self._batch(seqs, cu_rows)
        hq, qs, out, os_ = self._query(q, rows, out)
        r = rule.check(rows, n, hq, self._gpu) if rule is not None else None
        if rows:
            dt = _DTYPES[q.dtype]
            if r is not None:
                wb = self._bytes(("ruled prompt", hq, dt, n, rows, max_len), B.spd_prompt_attention_ruled_workspace)
                ws, wp = self._workspace(wb)
                self._on_device(lambda s: B.spd_prompt_attention_ruled(self.c, layer, q.data_ptr(), qs, out.data_ptr(), os_, hq, dt,
                                                                       seqs.data_ptr(), cu_rows.data_ptr(), n, rows, max_len, r, wp, wb, s))
                return out
            wb = self._bytes(("prompt", hq, dt, n, rows, max_len), B.spd_prompt_attention_workspace)
            ws, wp = self._workspace(wb)
            self._on_device(lambda s: B.spd_prompt_attention(self.c, layer, q.data_ptr(), qs, out.data_ptr(), os_, hq, dt,
                                                             seqs.data_ptr(), cu_rows.data_ptr(), n, rows, max_len, wp, wb, s))
        return out

    def prefix_attention(self, layer: int, q: torch.Tensor, seqs: torch.Tensor, cu_groups: Optional[torch.Tensor] = None,
                         prefix_lens: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                         max_len: int = 0, rule: Optional[AttentionRule] = None) -> torch.Tensor:
        """Decode attention, row i of q [sequences][heads][head_dim] over all keys of seqs[i]. Rows cu_groups[j] ..
        cu_groups[j + 1] - 1 share their first prefix_lens[j] keys, which are read once for all of them. rule: as for
        prompt_attention, a row being a sequence's."""
        n = self._entries(seqs)
        hq, qs, out, os_ = self._query(q, n, out)
        ng = cg = pl = 0
        if cu_groups is not None or prefix_lens is not None:
            if cu_groups is None or prefix_lens is None:
                raise ValueError("cu_groups and prefix_lens come together")
            ng = self._batch(prefix_lens, cu_groups)
            if ng:
                cg, pl = cu_groups.data_ptr(), prefix_lens.data_ptr()
        dt = _DTYPES[q.dtype]
        if rule is not None:
            r = rule.check(n, n, hq, self._gpu)
            wb = self._bytes(("ruled prefix", hq, dt, n, ng, max_len), B.spd_prefix_attention_ruled_workspace)
            ws, wp = self._workspace(wb)
            self._on_device(lambda s: B.spd_prefix_attention_ruled(self.c, layer, q.data_ptr(), qs, out.data_ptr(), os_, hq, dt,
                                                                   seqs.data_ptr(), n, cg, pl, ng, max_len, r, wp, wb, s))
            return out
        wb = self._bytes(("prefix", hq, dt, n, ng, max_len), B.spd_prefix_attention_workspace)
        ws, wp = self._workspace(wb)
        self._on_device(lambda s: B.spd_prefix_attention(self.c, layer, q.data_ptr(), qs, out.data_ptr(), os_, hq, dt,
                                                         seqs.data_ptr(), n, cg, pl, ng, max_len, wp, wb, s))
        return out

    # ------------------------------------------------------------------------------------------------ marshalling
    def _index(self, name: str, t: torch.Tensor, dim: int = 1, size: Optional[int] = None) -> None:
        if t.dtype is not torch.int32 or t.get_device() != self._gpu or t.dim() != dim or not t.is_contiguous() or \
                (size is not None and t.shape[0] != size):
            raise ValueError(f"{name} must be a contiguous int32 tensor of {dim} dimension(s)"
                             + (f" and {size} entries" if size is not None else "") + " on the cache's device")

    def _entries(self, first: torch.Tensor, *others: torch.Tensor) -> int:
        self._index("index", first)
        n = first.shape[0]
        for t in others:
            self._index("index", t, 1, n)
        return n

    def _batch(self, seqs: torch.Tensor, cu: torch.Tensor) -> int:
        self._index("seqs", seqs)
        n = seqs.shape[0]
        self._index("cu", cu, 1, n + 1)
        return n

    def _rows(self, name: str, t: torch.Tensor, rows: int, dtype: torch.dtype, heads: int) -> int:
        """The stride between the rows of [rows][heads][head_dim]."""
        dh = self.head_dim
        if t.dtype is not dtype or t.shape != (rows, heads, dh) or t.get_device() != self._gpu or dtype not in _DTYPES:
            st = None
        else:
            st = t.stride()
        if st is None or st[2] != 1 or (heads > 1 and st[1] != dh):
            raise ValueError(f"{name} must be [{rows} rows][{heads} heads][{dh}] of {dtype} (float32 or bfloat16) on the "
                             "cache's device, the heads of a row one after the other")
        return st[0] if rows > 1 else heads * dh

    def _query(self, q: torch.Tensor, rows: int, out: Optional[torch.Tensor]):
        hq = q.shape[1] if q.dim() == 3 else 0
        qs = self._rows("q", q, rows, q.dtype, hq)
        if out is None:
            return hq, qs, torch.empty(q.shape, dtype=q.dtype, device=self.device), hq * self.head_dim
        return hq, qs, out, self._rows("out", out, rows, q.dtype, hq)

    def _bytes(self, key, fn) -> int:
        n = self._ws_bytes.get(key)
        if n is None:
            if len(self._ws_bytes) >= 4096:
                self._ws_bytes.clear()
            n = self._ws_bytes[key] = fn(self.c, *key[1:])
        return n

    def _workspace(self, nbytes: int):
        """Of the current stream's pool, whose blocks are 512-byte aligned; free again when the call has returned, as the stream orders
        its next user behind it."""
        if nbytes == 0:
            return None, 0
        ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        return ws, ws.data_ptr()

    def _change(self, n: int, call, wb: Optional[int] = None) -> torch.Tensor:
        """wb: the workspace's bytes, if not those for n sequences."""
        word = torch.empty(1, dtype=torch.int32, device=self.device)
        if wb is None:
            wb = self._bytes(("pages", n), B.spd_cache_workspace) if n >= 1 else 0
        ws, wp = self._workspace(wb)
        self._on_device(lambda s: call(word.data_ptr(), wp, wb, s))
        return word

    def _on_device(self, call) -> None:
        """call(stream) with the cache's device current: the library launches on the current one. (The raw stream is
        torch.cuda.current_stream().cuda_stream without the object, 2 us less a call.)"""
        i = self._gpu
        if torch._C._cuda_getDevice() == i:
            call(torch._C._cuda_getCurrentRawStream(i))
        else:
            with torch.cuda.device(self.device):
                call(torch._C._cuda_getCurrentRawStream(i))
