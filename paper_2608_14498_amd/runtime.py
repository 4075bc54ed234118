"""Device-side convenience layer: torch owns the memory, the HIP library computes.

``DeviceModel`` uploads seeded host weights once, binds them with rp_create and
offers prefix / suffix / decode calls that allocate outputs and workspaces with
torch and call the C entry points on a torch stream.  ``PagedKV`` does the same for
a rollout cache in pages.  Nothing here computes any part of the method.
"""
from __future__ import annotations

from typing import Optional, Sequence

import numpy as np
import torch

from . import binding as rb
from .configs import ModelShape


def to_device(a: Optional[np.ndarray], device) -> Optional[torch.Tensor]:
    """Upload a stored host tensor (float32, int32, or bf16 bit patterns as uint16)."""
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a))
    if a.dtype == np.uint16:
        t = t.view(torch.bfloat16)
    return t.to(device, non_blocking=False)


def stream_ptr(stream: Optional[torch.cuda.Stream] = None) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def prompt_positions(cu: Sequence[int], token_ids: np.ndarray) -> np.ndarray:
    """Packed positions of every scorable prompt token: text tokens (id >= 0) that are
    not the first token of their sequence (host int32)."""
    ids = np.asarray(token_ids)
    first = np.zeros(len(ids), bool)
    first[np.asarray(cu[:-1], np.int64)] = True
    return np.nonzero((ids >= 0) & ~first)[0].astype(np.int32)


_DTYPE_NAMES = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}


def _i32_dev(t: Optional[torch.Tensor], what: str, numel: Optional[int], device) -> Optional[torch.Tensor]:
    """t as it is, checked: the C side sees an address only."""
    if t is None:
        return None
    if t.dtype is not torch.int32 or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{what} must be a contiguous int32 tensor on {device}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{what} has {t.numel()} elements, not {numel}")
    return t


class PagedKV:
    """A rollout cache in pages (rp_pages): pools k, v [L, n_pages, page_size, Hkv, Dh], page table
    [n_seqs, table_ld], lengths [n_seqs] and reference counts [n_pages] (int32), all device tensors
    that the object keeps and its calls update in stream order."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, length: torch.Tensor, refs: torch.Tensor):
        if k.dim() != 5 or k.shape != v.shape or k.dtype != v.dtype or k.dtype not in _DTYPE_NAMES:
            raise ValueError("k and v are [L, n_pages, page_size, Hkv, Dh], both float32, bfloat16 or float16")
        if not k.is_contiguous() or not v.is_contiguous() or v.device != k.device:
            raise ValueError("k and v must be contiguous, on one device")
        if table.dim() != 2:
            raise ValueError("table is [n_seqs, table_ld]")
        self.device = k.device
        self._index = k.get_device()
        _i32_dev(table, "table", None, self.device)
        _i32_dev(length, "length", table.shape[0], self.device)
        _i32_dev(refs, "refs", k.shape[1], self.device)
        self.k, self.v, self.table, self.length, self.refs = k, v, table, length, refs
        L, P, ps, H, D = k.shape
        self.pages = rb.make_pages(k, v, P * ps * H * D, _DTYPE_NAMES[k.dtype], L, H, D, P, ps, table, length, refs,
                                   table.shape[0], table.shape[1])

    @classmethod
    def empty(cls, n_layers: int, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, n_seqs: int,
              table_ld: int, dtype=torch.bfloat16, device: str = "cuda"):
        """An empty pool."""
        shape = (n_layers, n_pages, page_size, n_kv_heads, head_dim)
        k, v = torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device)
        ints = lambda fill, *s: torch.full(s, fill, dtype=torch.int32, device=device)
        return cls(k, v, ints(-1, n_seqs, table_ld), ints(0, n_seqs), ints(0, n_pages))

    def _call(self, fn, stream, *args):
        """fn(pages, stream, *args) with the pool's device current."""
        if torch.cuda.current_device() != self._index:
            with torch.cuda.device(self.device):
                return fn(self.pages, stream_ptr(stream), *args)
        # (the current stream's address without a Stream object: a rollout step makes many small calls)
        return fn(self.pages, torch._C._cuda_getCurrentRawStream(self._index) if stream is None else stream.cuda_stream, *args)

    def _empty(self, stream, shape, dtype=torch.int32) -> torch.Tensor:
        """A tensor of the stream that the call runs on: its memory is handed on behind that call."""
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def _ints(self, t, what, stream, *shape):
        if t is None:
            return self._empty(stream, shape)
        n = 1
        for x in shape:
            n *= x
        return _i32_dev(t, what, n, self.device)

    def _workspace(self, ws, stream, nbytes):
        if ws is None:
            return self._empty(stream, max(nbytes(), 256), torch.uint8)
        if ws.dtype is not torch.uint8 or not ws.is_contiguous() or ws.device != self.device:
            raise ValueError(f"workspace must be a contiguous uint8 tensor on {self.device}")
        return ws

    def _rows(self, K, V, rows: int) -> rb.RpKV:
        """Packed rows [L, ..., Hkv, Dh] of the pool's type."""
        L, _, _, H, D = self.k.shape
        for t in (K, V):
            if t.dtype != self.k.dtype or t.device != self.device or not t.is_contiguous():
                raise ValueError("K and V must be contiguous, of the pool's type and device")
            if t.numel() != L * rows * H * D:
                raise ValueError(f"K and V hold {t.numel()} elements, not {L} layers of {rows} rows of {H} x {D}")
        return rb.make_kv(K, V, rows * H * D)

    def append(self, seqs: Sequence[int], cu: Sequence[int], K, V, missing=None, stream=None) -> torch.Tensor:
        """Rows cu[i] .. cu[i+1] of K, V [L, cu[-1], Hkv, Dh] become the next tokens of sequence
        seqs[i].  Returns missing [n]: 0, or why sequence i stayed as it was (rollplex.h)."""
        if len(cu) != len(seqs) + 1:
            raise ValueError("cu has one entry more than seqs")
        missing = self._ints(missing, "missing", stream, len(seqs))
        self._call(rb.rp_pages_append, stream, len(seqs), seqs, cu, self._rows(K, V, int(cu[-1])), missing)
        return missing

    def fork(self, src: Sequence[int], dst: Sequence[int], missing=None, stream=None) -> torch.Tensor:
        """Sequence dst[i] gives its pages back and becomes a copy of src[i] that shares its full pages."""
        if len(src) != len(dst):
            raise ValueError("src and dst have the same length")
        missing = self._ints(missing, "missing", stream, len(dst))
        self._call(rb.rp_pages_fork, stream, len(dst), src, dst, missing)
        return missing

    def free(self, seqs: Sequence[int], stream=None) -> None:
        self._call(rb.rp_pages_free, stream, len(seqs), seqs)

    def compact_workspace(self) -> torch.Tensor:
        return torch.empty(rb.rp_pages_compact_workspace_bytes(self.pages), dtype=torch.uint8, device=self.device)

    def compact(self, n_live=None, workspace=None, stream=None) -> torch.Tensor:
        """Moves the pages in use to the lowest ids; returns their number (int32 [1])."""
        n_live = self._ints(n_live, "n_live", stream, 1)
        ws = self._workspace(workspace, stream, lambda: rb.rp_pages_compact_workspace_bytes(self.pages))
        self._call(rb.rp_pages_compact, stream, n_live, ws, ws.numel())
        return n_live

    def attention_workspace(self, B: int, N: int, n_q_heads: int) -> torch.Tensor:
        n = rb.rp_tree_attention_workspace_bytes(self.pages, B, N, n_q_heads)
        return torch.empty(n, dtype=torch.uint8, device=self.device)

    def tree_attention(self, layer: int, q, k_new, v_new, mask=None, n_nodes=None, scale: Optional[float] = None,
                       out=None, workspace=None, stream=None) -> torch.Tensor:
        """Attention of q [B, N, Hq, Dh] (the rows may lie apart) over the first B sequences' cached
        tokens of a layer and the new tokens k_new, v_new [B, N, Hkv, Dh] that mask (int32
        [B, N, ceil(N / 32)], bit j for token j; None: the tokens up to its own) shows."""
        _, _, _, H, D = self.k.shape
        if q.dim() != 4 or q.shape[3] != D or q.dtype != self.k.dtype or q.device != self.device:
            raise ValueError(f"q is [B, N, Hq, {D}] of the pool's type and device")
        B, N, Hq, _ = q.shape
        # (the stride of a dimension of one element says nothing)
        if q.stride(3) != 1 or (Hq > 1 and q.stride(2) != D) or (B > 1 and N > 1 and q.stride(0) != N * q.stride(1)):
            raise ValueError("q: heads must be contiguous and rows evenly spaced")
        q_ld = q.stride(1) if N > 1 else q.stride(0) if B > 1 else Hq * D
        for t in (k_new, v_new):
            if t.shape != (B, N, H, D) or t.dtype != q.dtype or t.device != self.device or not t.is_contiguous():
                raise ValueError(f"k_new and v_new are contiguous [{B}, {N}, {H}, {D}] of the pool's type and device")
        if out is None:
            out = self._empty(stream, (B, N, Hq, D), q.dtype)
        elif out.shape != q.shape or out.dtype != q.dtype or out.device != self.device or not out.is_contiguous():
            raise ValueError("out is contiguous, of q's shape, type and device")
        _i32_dev(mask, "mask", B * N * ((N + 31) // 32), self.device)
        _i32_dev(n_nodes, "n_nodes", B, self.device)
        ws = self._workspace(workspace, stream, lambda: rb.rp_tree_attention_workspace_bytes(self.pages, B, N, Hq))
        self._call(rb.rp_tree_attention, stream, layer, B, N, Hq, n_nodes, mask, q, q_ld, k_new, v_new,
                   D ** -0.5 if scale is None else scale, out, ws, ws.numel())
        return out

    def commit(self, token_ids, parents, next_ids, K, V, n_nodes=None, accepted=None, n_accepted=None, token_out=None,
               missing=None, stream=None):
        """Appends the drafted tokens (token_ids, parents [B, N], K, V [L, B * N, Hkv, Dh]) that next_ids
        [B, N] confirm.  Returns (accepted [B, N], n_accepted [B], token_out [B], missing [B])."""
        B, N = token_ids.shape
        for t, what in ((token_ids, "token_ids"), (parents, "parents"), (next_ids, "next_ids")):
            _i32_dev(t, what, B * N, self.device)
        _i32_dev(n_nodes, "n_nodes", B, self.device)
        accepted = self._ints(accepted, "accepted", stream, B, N)
        n_accepted, token_out = self._ints(n_accepted, "n_accepted", stream, B), self._ints(token_out, "token_out", stream, B)
        missing = self._ints(missing, "missing", stream, B)
        self._call(rb.rp_tree_commit, stream, B, N, n_nodes, token_ids, parents, next_ids, self._rows(K, V, B * N),
                   accepted, n_accepted, token_out, missing)
        return accepted, n_accepted, token_out, missing


class DeviceModel:
    """Weights resident in HBM plus a model handle of the HIP library."""

    def __init__(self, host_weights, max_position: int, device: str = "cuda", weight_layout: int = 0):
        """weight_layout (rb.RP_WO_TRANSPOSED | rb.RP_W_DOWN_TRANSPOSED) stores those row-parallel
        projections transposed, [in, out], as a training engine's shards would lay them out."""
        m: ModelShape = host_weights.model
        self.shape = m
        self.device = torch.device(device)
        self.dtype = {"bf16": torch.bfloat16, "f16": torch.float16}.get(m.dtype, torch.float32)
        self.max_position = int(max_position)
        up = lambda a: to_device(a, self.device)
        self.embed = up(host_weights.embed)
        self.lm_head = up(host_weights.lm_head)
        self.final_norm = up(host_weights.final_norm)
        stored_t = {"wo": weight_layout & rb.RP_WO_TRANSPOSED, "w_down": weight_layout & rb.RP_W_DOWN_TRANSPOSED}
        self.layers = [{k: up(np.ascontiguousarray(v.T) if stored_t.get(k) else v) for k, v in lw.items()}
                       for lw in host_weights.layers]
        p = rb._ptr
        arr = (rb.RpLayerWeights * m.n_layers)()
        for i, lw in enumerate(self.layers):
            for name, _ in rb.RpLayerWeights._fields_:
                setattr(arr[i], name, p(lw.get(name)))
        self._layer_arr = arr
        self._weights = rb.RpWeights(p(self.embed), p(self.final_norm), p(self.lm_head), arr)
        self.config = rb.make_config(m, self.max_position, weight_layout)
        self.handle = rb.rp_create(self.config, self._weights)

    def close(self):
        if getattr(self, "handle", None):
            rb.rp_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---------------------------------------------------------------- helpers
    def alloc_kv(self, rows: int):
        m = self.shape
        shape = (m.n_layers, rows, m.n_kv_heads, m.head_dim)
        k = torch.empty(shape, dtype=self.dtype, device=self.device)
        v = torch.empty(shape, dtype=self.dtype, device=self.device)
        return k, v

    def workspace(self, nbytes: int) -> torch.Tensor:
        return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=self.device)

    # ---------------------------------------------------------------- passes
    def prefix(self, cu: Sequence[int], token_ids: torch.Tensor, visual: Optional[torch.Tensor],
               kv=None, h_last=None, hidden_out=None, workspace=None, stream=None, positions=None,
               mrope_section=None, flags: int = 0):
        """Prefix pass.  Returns (K, V, h_last) with K/V [L, T, Hkv, Dh].  With positions
        (device int32 [3, T]) and mrope_section, RoPE uses multimodal 3-D positions; flags
        (rb.RP_PREFIX_LAST_ROWS_ONLY) select options of rp_prefix_forward_flags."""
        m = self.shape
        B, T = len(cu) - 1, int(cu[-1])
        K, V = kv if kv is not None else self.alloc_kv(T)
        if h_last is None:
            h_last = torch.empty((B, m.d_model), dtype=torch.float32, device=self.device)
        nbytes = rb.rp_prefix_workspace_bytes(self.handle, B, cu)
        ws = workspace if workspace is not None else self.workspace(nbytes)
        n_visual = 0 if visual is None else visual.shape[0]
        if flags:
            rb.rp_prefix_forward_flags(self.handle, stream_ptr(stream), B, cu, token_ids, visual, n_visual,
                                       positions, mrope_section, flags, rb.make_kv(K, V, K[0].numel()), h_last,
                                       hidden_out, ws, ws.numel())
        elif positions is None:
            rb.rp_prefix_forward(self.handle, stream_ptr(stream), B, cu, token_ids, visual, n_visual,
                                 rb.make_kv(K, V, K[0].numel()), h_last, hidden_out, ws, ws.numel())
        else:
            rb.rp_prefix_forward_mrope(self.handle, stream_ptr(stream), B, cu, token_ids, visual, n_visual,
                                       positions, mrope_section, rb.make_kv(K, V, K[0].numel()), h_last,
                                       hidden_out, ws, ws.numel())
        return K, V, h_last

    def suffix(self, prefix_cu, suffix_cu, K, V, h_last, response_ids, logprobs=None, workspace=None,
               stream=None):
        B, R = len(prefix_cu) - 1, int(suffix_cu[-1])
        if logprobs is None:
            logprobs = torch.empty(max(R, 1), dtype=torch.float32, device=self.device)[:R]
        nbytes = rb.rp_suffix_workspace_bytes(self.handle, B, prefix_cu, suffix_cu)
        ws = workspace if workspace is not None else self.workspace(nbytes)
        rb.rp_suffix_logprob(self.handle, stream_ptr(stream), B, prefix_cu, suffix_cu,
                             rb.make_kv(K, V, K[0].numel()), h_last, response_ids, logprobs, ws, ws.numel())
        return logprobs

    def suffix_grouped(self, prefix_cu, prefix_of_suffix, suffix_cu, K, V, h_last, response_ids, logprobs=None,
                       workspace=None, stream=None, flags: int = 0, rope_pos0=None):
        """Suffix pass where suffix s reads prefix prefix_of_suffix[s] (shared prefixes);
        flags = rb.RP_SUFFIX_FUSED_LOGPROB scores without storing the logits; rope_pos0[p]
        is the rotary position of the first response token after prefix p (default P_p)."""
        P, S, R = len(prefix_cu) - 1, len(suffix_cu) - 1, int(suffix_cu[-1])
        if logprobs is None:
            logprobs = torch.empty(max(R, 1), dtype=torch.float32, device=self.device)[:R]
        nbytes = rb.rp_suffix_grouped_workspace_bytes(self.handle, P, prefix_cu, S, prefix_of_suffix, suffix_cu,
                                                      flags)
        ws = workspace if workspace is not None else self.workspace(nbytes)
        rb.rp_suffix_logprob_grouped(self.handle, stream_ptr(stream), P, prefix_cu, S, prefix_of_suffix,
                                     suffix_cu, rope_pos0, flags, rb.make_kv(K, V, K[0].numel()), h_last,
                                     response_ids, logprobs, ws, ws.numel())
        return logprobs

    def prompt_logprobs(self, cu, token_ids, hidden, positions, logprobs=None, workspace=None, stream=None,
                        flags: int = 0):
        """Teacher-forced log-probs of the prompt tokens at packed positions (device int32),
        scored from the prefix pass's hidden_out (device fp32 [T, d])."""
        B, n = len(cu) - 1, int(positions.numel())
        if logprobs is None:
            logprobs = torch.empty(max(n, 1), dtype=torch.float32, device=self.device)[:n]
        nbytes = rb.rp_prompt_logprob_workspace_bytes(self.handle, n, flags)
        ws = workspace if workspace is not None else self.workspace(nbytes)
        rb.rp_prompt_logprob(self.handle, stream_ptr(stream), B, cu, token_ids, hidden, n, positions, flags,
                             logprobs, ws, ws.numel())
        return logprobs

    def decode(self, cache_k, cache_v, kv_len, token_ids, logits=None, next_ids=None, workspace=None,
               stream=None):
        B, cap = cache_k.shape[1], cache_k.shape[2]
        if next_ids is None:
            next_ids = torch.empty(B, dtype=torch.int32, device=self.device)
        nbytes = rb.rp_decode_workspace_bytes(self.handle, B, cap)
        ws = workspace if workspace is not None else self.workspace(nbytes)
        rb.rp_decode_step(self.handle, stream_ptr(stream), B, rb.make_kv(cache_k, cache_v, cache_k[0].numel()),
                          cap, kv_len, token_ids, logits, next_ids, ws, ws.numel())
        return next_ids

    def tree_step(self, cache: PagedKV, token_ids, parents=None, n_nodes=None, pos0=None, draft=None, logits=None,
                  next_ids=None, workspace=None, stream=None):
        """One pass over new tokens token_ids [B, N] of the cache's first B sequences (trees by
        parents [B, N]; None: chains).  Returns (next_ids [B, N], K, V [L, B * N, Hkv, Dh] of the new tokens,
        for PagedKV.commit)."""
        B, N = token_ids.shape
        if cache.device != self.embed.device:
            raise ValueError(f"the cache is on {cache.device}, the model on {self.embed.device}")
        for t, what, n in ((token_ids, "token_ids", B * N), (parents, "parents", B * N), (n_nodes, "n_nodes", B),
                           (pos0, "pos0", B), (next_ids, "next_ids", B * N)):
            _i32_dev(t, what, n, cache.device)
        if logits is not None and (logits.dtype != torch.float32 or logits.numel() != B * N * self.shape.vocab or
                                   not logits.is_contiguous() or logits.device != cache.device):
            raise ValueError("logits is a contiguous float32 tensor [B, N, V]")
        K, V = draft if draft is not None else [
            cache._empty(stream, (cache.k.shape[0], B * N) + cache.k.shape[3:], cache.k.dtype) for _ in "kv"]
        next_ids = cache._ints(next_ids, "next_ids", stream, B, N)
        ws = cache._workspace(workspace, stream, lambda: rb.rp_tree_step_workspace_bytes(self.handle, B, N))
        rows = cache._rows(K, V, B * N)
        cache._call(lambda pages, st: rb.rp_tree_step(self.handle, st, pages, B, N, n_nodes, token_ids, parents, pos0,
                                                      rows, logits, next_ids, ws, ws.numel()), stream)
        return next_ids, K, V
