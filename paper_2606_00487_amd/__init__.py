"""TAPS draft-tree verification hot path on MI355X (gfx950).

Thin Python binding over libtaps.so (include/taps.h): argument marshalling
only, every step of the path runs in the HIP kernels.  PyTorch provides device
memory and the current stream.

    sel = Selector(batch, block, vocab, K, budget, dtype=BF16, kind=LOGITS)
    tree = sel(marginals)                       # taps_select
    att = TreeAttention(batch, budget, Hq, Hkv, head_dim, max_ctx)
    O = att(Q, K, V, kv_offset, ctx_len, tree.parent, tree.n_nodes)   # tree_verify_attn
    walk = AcceptWalk(batch, budget, block)
    path, path_len, bonus = walk(tree, target_tokens)                 # accept_walk
    com = KVCommit(batch, budget, block, Hkv, head_dim, max_ctx)
    new_ctx, tokens, n = com(K, V, kv_offset, ctx_len, tree, path, path_len, bonus)  # kv_commit
    lay = VerifyLayer(batch, budget, Hq, Hkv, head_dim, hidden, max_ctx)
    Y = lay(X, LayerWeights(Wq, Wk, Wv, Wo, q_norm, k_norm), K, V, kv_offset, ctx_len, tree)

Around the round, over a paged cache:

    res = PagedKVReserve(batch, max_pages, num_pages, page_rows, max_new)
    held, n_free, short, slots = res(block_table, held, ctx_len, n_new, free_pages, n_free)
    PagedKVAppend(Hkv, head_dim, page_rows)(K_new, V_new, slots, K_pages, V_pages)
    dec = PagedDecodeAttention(batch, Hq, Hkv, head_dim, max_len, page_rows)
    O = dec(Q, K_pages, V_pages, block_table, kv_len)                 # decode_attn_paged
    smp = TokenSampler(batch, budget, vocab)
    target_tokens, probs = smp(logits, u, tree.n_nodes, temperature=T, top_p=p)   # taps_sample
"""
from __future__ import annotations

import ctypes
import dataclasses

import torch

from . import _lib
from ._lib import (TAPS_BF16 as BF16, TAPS_FP32 as FP32, TAPS_LOGITS as LOGITS,  # noqa: F401
                   TAPS_PROBS as PROBS, TAPS_SCORER_LEARNED as LEARNED,
                   TAPS_SCORER_MARGINAL as MARGINAL, TAPS_SCORER_SIBLING as SIBLING, TapsError,
                   load)

_TORCH_DT = {BF16: torch.bfloat16, FP32: torch.float32}


def _ptr(t: torch.Tensor | None) -> int | None:
    return None if t is None else t.data_ptr()


# torch's own bindings (not public) give the current stream's handle itself: a
# torch.cuda.Stream object for each of a round's calls costs more than the rest of the call's
# arguments together.  A torch without them takes the public call.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream() -> int:
    if _raw_stream is None or _device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


def _need(t: torch.Tensor, name: str, dtype, shape=None):
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise TypeError(f"{name}: expected a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if shape is not None and t.shape != shape:   # a torch.Size is a tuple
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")


@dataclasses.dataclass
class TreeBuffers:
    """Device arrays of taps_tree (see include/taps.h)."""
    parent: torch.Tensor
    token: torch.Tensor
    depth: torch.Tensor
    rank: torch.Tensor
    q_reach: torch.Tensor
    n_nodes: torch.Tensor
    topk_idx: torch.Tensor
    topk_val: torch.Tensor

    @staticmethod
    def empty(batch, block, K, budget, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        return TreeBuffers(
            parent=torch.empty(batch, budget, **i32), token=torch.empty(batch, budget, **i32),
            depth=torch.empty(batch, budget, **i32), rank=torch.empty(batch, budget, **i32),
            q_reach=torch.empty(batch, budget, dtype=torch.float64, device=device),
            n_nodes=torch.empty(batch, **i32), topk_idx=torch.empty(batch, block, K, **i32),
            topk_val=torch.empty(batch, block, K, dtype=torch.float32, device=device))

    def struct(self) -> _lib.Tree:
        return _lib.Tree(_ptr(self.parent), _ptr(self.token), _ptr(self.depth), _ptr(self.rank),
                         _ptr(self.q_reach), _ptr(self.n_nodes), _ptr(self.topk_idx),
                         _ptr(self.topk_val))


@dataclasses.dataclass
class ScorerWeights:
    """Device weights of the learned-scorer hook (taps_scorer_mlp): float32 emb [vocab][d],
    W1 [h][2d+3], b1 [h], w2 [h], the float b2 and int32 root_token [batch]."""
    emb: torch.Tensor
    W1: torch.Tensor
    b1: torch.Tensor
    w2: torch.Tensor
    b2: float
    root_token: torch.Tensor

    def struct(self) -> _lib.ScorerMLP:
        d, h = self.emb.shape[1], self.W1.shape[0]
        _need(self.emb, "emb", torch.float32)
        _need(self.W1, "W1", torch.float32, (h, 2 * d + 3))
        _need(self.b1, "b1", torch.float32, (h,))
        _need(self.w2, "w2", torch.float32, (h,))
        _need(self.root_token, "root_token", torch.int32)
        return _lib.ScorerMLP(_ptr(self.emb), _ptr(self.W1), _ptr(self.b1), _ptr(self.w2),
                              float(self.b2), _ptr(self.root_token), d, h)


class Selector:
    """taps_select: top-K, Eq. 1-3 and the budgeted prefix-closed selection of Alg. 1."""

    def __init__(self, batch, block, vocab, K, budget, dtype=BF16, kind=LOGITS, lambda1=1.0,
                 lambda2=0.125, tau=0.0, beta=1.0, scorer=SIBLING, mlp=None, device="cuda"):
        """scorer: SIBLING (sibling softmax over the K candidates), MARGINAL (the drafter's
        full-vocabulary marginal: the scoring ablation) or LEARNED (the learned-scorer hook,
        whose weights `mlp` (ScorerWeights) must stay alive while the Selector is used)."""
        self.lib = load()
        self.mlp = mlp
        self._mlp_struct = mlp.struct() if mlp is not None else None
        self.p = _lib.SelectParams(batch, block, vocab, K, budget, dtype, kind, lambda1, lambda2,
                                   tau, beta, scorer,
                                   ctypes.pointer(self._mlp_struct) if mlp is not None else None)
        _lib.check(self.lib, "taps_select_validate", self.lib.taps_select_validate(ctypes.byref(self.p)))
        self.ws_bytes = self.lib.taps_select_workspace_bytes(ctypes.byref(self.p))
        nbytes = self.ws_bytes + self.lib.taps_select_tables_bytes(ctypes.byref(self.p))
        self.ws = torch.empty(max(nbytes, 8), dtype=torch.uint8, device=device)
        self.tree = TreeBuffers.empty(batch, block, K, budget, device)
        self._tree_struct = self.tree.struct()

    def __call__(self, marginals: torch.Tensor, tree: TreeBuffers | None = None) -> TreeBuffers:
        p = self.p
        _need(marginals, "marginals", _TORCH_DT[p.dtype], (p.batch, p.block, p.vocab))
        t = tree or self.tree
        st = t.struct() if tree is not None else self._tree_struct
        _lib.check(self.lib, "taps_select",
                   self.lib.taps_select(_ptr(marginals), ctypes.byref(p), ctypes.byref(st),
                                        _ptr(self.ws), self.ws.numel(), _stream()))
        return t

    def noalloc(self, marginals: torch.Tensor, tree: TreeBuffers | None = None) -> TreeBuffers:
        """taps_select_noalloc: the same selection with the library's static scratch instead
        of this Selector's workspace (for callers that cannot allocate)."""
        p = self.p
        _need(marginals, "marginals", _TORCH_DT[p.dtype], (p.batch, p.block, p.vocab))
        t = tree or self.tree
        st = t.struct() if tree is not None else self._tree_struct
        _lib.check(self.lib, "taps_select_noalloc",
                   self.lib.taps_select_noalloc(_ptr(marginals), ctypes.byref(p),
                                                ctypes.byref(st), _stream()))
        return t


class TreeAttention:
    """tree_verify_attn: tree-masked verification attention."""

    def __init__(self, batch, budget, Hq, Hkv, head_dim, max_ctx, dtype=BF16, scale=None,
                 device="cuda"):
        self.lib = load()
        self.shape = (batch, budget, Hq, Hkv, head_dim, max_ctx, dtype)
        self.scale = float(scale if scale is not None else head_dim ** -0.5)
        _lib.check(self.lib, "tree_verify_attn_validate",
                   self.lib.tree_verify_attn_validate(batch, budget, Hq, Hkv, head_dim, max_ctx,
                                                      dtype, self.scale))
        self.ws_bytes = self.lib.tree_verify_attn_workspace_bytes(batch, budget, Hq, Hkv,
                                                                  head_dim, max_ctx, dtype)
        self.ws = torch.empty(max(self.ws_bytes, 16), dtype=torch.uint8, device=device)
        self._home = _stream() if self.ws.is_cuda else None   # the stream whose calls share ws

    def __call__(self, Q, K, V, kv_offset, ctx_len, parent, n_nodes, out=None, events=None):
        """events: optional (begin, end) torch.cuda.Event pair recorded around the main
        attention kernel only (tree_verify_attn_timed)."""
        stream, ws = _stream(), self.ws
        batch, budget, Hq, Hkv, hd, max_ctx, dtype = self.shape
        tdt = _TORCH_DT[dtype]
        _need(Q, "Q_tree", tdt, (batch, budget, Hq, hd))
        _need(K, "K_cache", tdt)
        _need(V, "V_cache", tdt, K.shape)
        if K.dim() != 3 or K.shape[1:] != (Hkv, hd):
            raise ValueError(f"K_cache: expected [rows, {Hkv}, {hd}], got {tuple(K.shape)}")
        _need(kv_offset, "kv_offset", torch.int64, (batch,))
        _need(ctx_len, "ctx_len", torch.int32, (batch,))
        _need(parent, "tree_parent", torch.int32, (batch, budget))
        _need(n_nodes, "n_nodes", torch.int32, (batch,))
        O = out if out is not None else torch.empty_like(Q)
        _need(O, "O", tdt, (batch, budget, Hq, hd))
        if dtype == FP32 and self.ws_bytes and stream != self._home:
            # fp32 calls of one object may overlap on several streams: scratch of their own
            ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=Q.device)
        args = (_ptr(Q), _ptr(K), _ptr(V), _ptr(kv_offset), _ptr(ctx_len), _ptr(parent),
                _ptr(n_nodes), batch, budget, Hq, Hkv, hd, max_ctx, dtype, self.scale, _ptr(O),
                _ptr(ws), self.ws_bytes, stream)
        if events is None:
            _lib.check(self.lib, "tree_verify_attn", self.lib.tree_verify_attn(*args))
        else:
            _lib.check(self.lib, "tree_verify_attn_timed", self.lib.tree_verify_attn_timed(
                *args, events[0].cuda_event, events[1].cuda_event))
        return O


class PagedTreeAttention:
    """tree_verify_attn_paged: tree_verify_attn over a paged KV cache (bf16, head_dim 128)."""

    def __init__(self, batch, budget, Hq, Hkv, max_ctx, page_rows, scale=None, device="cuda"):
        self.lib = load()
        hd = 128
        self.shape = (batch, budget, Hq, Hkv, hd, max_ctx)
        self.page_rows = int(page_rows)
        self.scale = float(scale if scale is not None else hd ** -0.5)
        self.ws_bytes = self.lib.tree_verify_attn_paged_workspace_bytes(
            batch, budget, Hq, Hkv, hd, max_ctx, self.page_rows)
        self.ws = torch.empty(max(self.ws_bytes, 16), dtype=torch.uint8, device=device)

    def __call__(self, Q, K_pages, V_pages, block_table, ctx_len, parent, n_nodes, out=None,
                 events=None):
        """K_pages, V_pages: [num_pages, page_rows, Hkv, 128] bf16; block_table: [batch,
        max_pages] int32 page ids (request b's logical row r at page block_table[b, r //
        page_rows], slot r % page_rows).  events: optional (begin, end) pair recorded around
        the main attention kernel only (tree_verify_attn_paged_timed)."""
        batch, budget, Hq, Hkv, hd, max_ctx = self.shape
        _need(Q, "Q_tree", torch.bfloat16, (batch, budget, Hq, hd))
        _need(K_pages, "K_pages", torch.bfloat16)
        if K_pages.dim() != 4 or K_pages.shape[1:] != (self.page_rows, Hkv, hd):
            raise ValueError(f"K_pages: expected [pages, {self.page_rows}, {Hkv}, {hd}], "
                             f"got {tuple(K_pages.shape)}")
        _need(V_pages, "V_pages", torch.bfloat16, K_pages.shape)
        _need(block_table, "block_table", torch.int32)
        if block_table.dim() != 2 or block_table.shape[0] != batch:
            raise ValueError(f"block_table: expected [{batch}, max_pages], "
                             f"got {tuple(block_table.shape)}")
        _need(ctx_len, "ctx_len", torch.int32, (batch,))
        _need(parent, "tree_parent", torch.int32, (batch, budget))
        _need(n_nodes, "n_nodes", torch.int32, (batch,))
        O = out if out is not None else torch.empty_like(Q)
        _need(O, "O", torch.bfloat16, (batch, budget, Hq, hd))
        args = (_ptr(Q), _ptr(K_pages), _ptr(V_pages), K_pages.shape[0], self.page_rows,
                _ptr(block_table), block_table.shape[1], _ptr(ctx_len), _ptr(parent),
                _ptr(n_nodes), batch, budget, Hq, Hkv, hd, max_ctx, BF16, self.scale, _ptr(O),
                _ptr(self.ws), self.ws_bytes, _stream())
        if events is None:
            _lib.check(self.lib, "tree_verify_attn_paged", self.lib.tree_verify_attn_paged(*args))
        else:
            _lib.check(self.lib, "tree_verify_attn_paged_timed",
                       self.lib.tree_verify_attn_paged_timed(*args, events[0].cuda_event,
                                                             events[1].cuda_event))
        return O


class AcceptWalk:
    """accept_walk: greedy acceptance of the longest matching root path."""

    def __init__(self, batch, budget, block, device="cuda"):
        self.lib = load()
        self.batch, self.budget, self.block = batch, budget, block
        self.path = torch.empty(batch, block + 1, dtype=torch.int32, device=device)
        self.path_len = torch.empty(batch, dtype=torch.int32, device=device)
        self.bonus = torch.empty(batch, dtype=torch.int32, device=device)

    def __call__(self, tree: TreeBuffers, target_tokens: torch.Tensor):
        _need(target_tokens, "target_tokens", torch.int32, (self.batch, self.budget))
        st = tree.struct()
        _lib.check(self.lib, "accept_walk", self.lib.accept_walk(
            ctypes.byref(st), self.batch, self.budget, self.block, _ptr(target_tokens),
            _ptr(self.path), _ptr(self.path_len), _ptr(self.bonus), _stream()))
        return self.path, self.path_len, self.bonus


class KVCommit:
    """kv_commit: the accepted path's tree K/V rows move to the rows after the context
    (in place), and the round's emitted tokens."""

    def __init__(self, batch, budget, block, Hkv, head_dim, max_ctx, dtype=BF16, device="cuda"):
        self.lib = load()
        self.shape = (batch, budget, block, Hkv, head_dim, max_ctx, dtype)
        self.new_ctx = torch.empty(batch, dtype=torch.int32, device=device)
        self.committed = torch.empty(batch, block + 1, dtype=torch.int32, device=device)
        self.n_committed = torch.empty(batch, dtype=torch.int32, device=device)

    def __call__(self, K, V, kv_offset, ctx_len, tree: TreeBuffers, path, path_len, bonus):
        batch, budget, block, Hkv, hd, max_ctx, dtype = self.shape
        tdt = _TORCH_DT[dtype]
        _need(K, "K_cache", tdt)
        _need(V, "V_cache", tdt, K.shape)
        if K.dim() != 3 or K.shape[1:] != (Hkv, hd):
            raise ValueError(f"K_cache: expected [rows, {Hkv}, {hd}], got {tuple(K.shape)}")
        _need(kv_offset, "kv_offset", torch.int64, (batch,))
        _need(ctx_len, "ctx_len", torch.int32, (batch,))
        _need(tree.token, "tree.token", torch.int32, (batch, budget))
        _need(path, "path", torch.int32, (batch, block + 1))
        _need(path_len, "path_len", torch.int32, (batch,))
        _need(bonus, "bonus", torch.int32, (batch,))
        st = tree.struct()
        _lib.check(self.lib, "kv_commit", self.lib.kv_commit(
            _ptr(K), _ptr(V), _ptr(kv_offset), _ptr(ctx_len), ctypes.byref(st), _ptr(path),
            _ptr(path_len), _ptr(bonus), batch, budget, block, Hkv, hd, max_ctx, dtype,
            _ptr(self.new_ctx), _ptr(self.committed), _ptr(self.n_committed), _stream()))
        return self.new_ctx, self.committed, self.n_committed


class PagedKVCommit:
    """kv_commit_paged: kv_commit on a paged cache (pools [num_pages, page_rows, Hkv,
    head_dim] and a block table [batch, max_pages], as for PagedTreeAttention)."""

    def __init__(self, batch, budget, block, Hkv, head_dim, max_ctx, page_rows, dtype=BF16,
                 device="cuda"):
        self.lib = load()
        self.shape = (batch, budget, block, Hkv, head_dim, max_ctx, dtype)
        self.page_rows = int(page_rows)
        self.new_ctx = torch.empty(batch, dtype=torch.int32, device=device)
        self.committed = torch.empty(batch, block + 1, dtype=torch.int32, device=device)
        self.n_committed = torch.empty(batch, dtype=torch.int32, device=device)

    def __call__(self, K_pages, V_pages, block_table, ctx_len, tree: TreeBuffers, path, path_len,
                 bonus):
        batch, budget, block, Hkv, hd, max_ctx, dtype = self.shape
        tdt = _TORCH_DT[dtype]
        _need(K_pages, "K_pages", tdt)
        _need(V_pages, "V_pages", tdt, K_pages.shape)
        if K_pages.dim() != 4 or K_pages.shape[1:] != (self.page_rows, Hkv, hd):
            raise ValueError(f"K_pages: expected [pages, {self.page_rows}, {Hkv}, {hd}], "
                             f"got {tuple(K_pages.shape)}")
        _need(block_table, "block_table", torch.int32)
        if block_table.dim() != 2 or block_table.shape[0] != batch:
            raise ValueError(f"block_table: expected [{batch}, max_pages], "
                             f"got {tuple(block_table.shape)}")
        _need(ctx_len, "ctx_len", torch.int32, (batch,))
        _need(tree.token, "tree.token", torch.int32, (batch, budget))
        _need(path, "path", torch.int32, (batch, block + 1))
        _need(path_len, "path_len", torch.int32, (batch,))
        _need(bonus, "bonus", torch.int32, (batch,))
        st = tree.struct()
        _lib.check(self.lib, "kv_commit_paged", self.lib.kv_commit_paged(
            _ptr(K_pages), _ptr(V_pages), K_pages.shape[0], self.page_rows, _ptr(block_table),
            block_table.shape[1], _ptr(ctx_len), ctypes.byref(st), _ptr(path), _ptr(path_len),
            _ptr(bonus), batch, budget, block, Hkv, hd, max_ctx, dtype, _ptr(self.new_ctx),
            _ptr(self.committed), _ptr(self.n_committed), _stream()))
        return self.new_ctx, self.committed, self.n_committed


@dataclasses.dataclass
class LayerWeights:
    """Device bf16 weights of one attention layer (taps_layer_weights), row-major [out][in]:
    Wq [Hq*hd][hidden], Wk and Wv [Hkv*hd][hidden], Wo [hidden][Hq*hd], q_norm and k_norm
    [hd]."""
    Wq: torch.Tensor
    Wk: torch.Tensor
    Wv: torch.Tensor
    Wo: torch.Tensor
    q_norm: torch.Tensor
    k_norm: torch.Tensor
    rope_theta: float = 1e6
    norm_eps: float = 1e-6

    def struct(self) -> _lib.LayerWeights:
        hidden = self.Wq.shape[1]
        for name in ("Wq", "Wk", "Wv", "Wo", "q_norm", "k_norm"):
            _need(getattr(self, name), name, torch.bfloat16)
        _need(self.Wo, "Wo", torch.bfloat16, (hidden, self.Wq.shape[0]))
        return _lib.LayerWeights(_ptr(self.Wq), _ptr(self.Wk), _ptr(self.Wv), _ptr(self.Wo),
                                 _ptr(self.q_norm), _ptr(self.k_norm), float(self.rope_theta),
                                 float(self.norm_eps), hidden)


class VerifyLayer:
    """verify_layer: one attention layer of the target over the selected trees
    (projections, per-head RMSNorm, rotary positions by tree depth, tree attention,
    output projection)."""

    def __init__(self, batch, budget, Hq, Hkv, head_dim, hidden, max_ctx, scale=None,
                 device="cuda"):
        self.lib = load()
        self.scale = float(scale if scale is not None else head_dim ** -0.5)
        self.shape = (batch, budget, Hq, Hkv, head_dim, hidden, max_ctx)
        nbytes = self.lib.verify_layer_workspace_bytes(batch, budget, Hq, Hkv, head_dim, hidden,
                                                       max_ctx)
        if batch > 0 and nbytes == 0:
            raise TapsError("verify_layer_workspace_bytes", _lib.TAPS_ERR_UNSUPPORTED)
        self.ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        self.Y = torch.empty((batch, budget, hidden), dtype=torch.bfloat16, device=device)

    def __call__(self, X, w: LayerWeights, K, V, kv_offset, ctx_len, tree: TreeBuffers):
        batch, budget, Hq, Hkv, hd, hidden, max_ctx = self.shape
        _need(X, "X", torch.bfloat16, (batch, budget, hidden))
        _need(K, "K_cache", torch.bfloat16)
        _need(V, "V_cache", torch.bfloat16, K.shape)
        _need(kv_offset, "kv_offset", torch.int64, (batch,))
        _need(ctx_len, "ctx_len", torch.int32, (batch,))
        ws = w.struct()
        if ws.hidden != hidden:
            raise ValueError(f"weights: hidden {ws.hidden}, expected {hidden}")
        st = tree.struct()
        _lib.check(self.lib, "verify_layer", self.lib.verify_layer(
            _ptr(X), ctypes.byref(ws), _ptr(K), _ptr(V), _ptr(kv_offset), _ptr(ctx_len),
            ctypes.byref(st), batch, budget, Hq, Hkv, hd, max_ctx, self.scale, _ptr(self.Y),
            _ptr(self.ws), self.ws.numel(), _stream()))
        return self.Y


class PagedVerifyLayer:
    """verify_layer_paged: verify_layer over a paged KV cache (pools [num_pages, page_rows,
    Hkv, head_dim] and a block table [batch, max_pages], as for PagedTreeAttention)."""

    def __init__(self, batch, budget, Hq, Hkv, head_dim, hidden, max_ctx, page_rows, scale=None,
                 device="cuda"):
        self.lib = load()
        self.scale = float(scale if scale is not None else head_dim ** -0.5)
        self.shape = (batch, budget, Hq, Hkv, head_dim, hidden, max_ctx)
        self.page_rows = int(page_rows)
        nbytes = self.lib.verify_layer_paged_workspace_bytes(batch, budget, Hq, Hkv, head_dim,
                                                             hidden, max_ctx, self.page_rows)
        if batch > 0 and nbytes == 0:
            raise TapsError("verify_layer_paged_workspace_bytes", _lib.TAPS_ERR_UNSUPPORTED)
        self.ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        self.Y = torch.empty((batch, budget, hidden), dtype=torch.bfloat16, device=device)

    def __call__(self, X, w: LayerWeights, K_pages, V_pages, block_table, ctx_len,
                 tree: TreeBuffers):
        batch, budget, Hq, Hkv, hd, hidden, max_ctx = self.shape
        _need(X, "X", torch.bfloat16, (batch, budget, hidden))
        _need(K_pages, "K_pages", torch.bfloat16)
        if K_pages.dim() != 4 or K_pages.shape[1:] != (self.page_rows, Hkv, hd):
            raise ValueError(f"K_pages: expected [pages, {self.page_rows}, {Hkv}, {hd}], "
                             f"got {tuple(K_pages.shape)}")
        _need(V_pages, "V_pages", torch.bfloat16, K_pages.shape)
        _need(block_table, "block_table", torch.int32)
        if block_table.dim() != 2 or block_table.shape[0] != batch:
            raise ValueError(f"block_table: expected [{batch}, max_pages], "
                             f"got {tuple(block_table.shape)}")
        _need(ctx_len, "ctx_len", torch.int32, (batch,))
        ws = w.struct()
        if ws.hidden != hidden:
            raise ValueError(f"weights: hidden {ws.hidden}, expected {hidden}")
        st = tree.struct()
        _lib.check(self.lib, "verify_layer_paged", self.lib.verify_layer_paged(
            _ptr(X), ctypes.byref(ws), _ptr(K_pages), _ptr(V_pages), K_pages.shape[0],
            self.page_rows, _ptr(block_table), block_table.shape[1], _ptr(ctx_len),
            ctypes.byref(st), batch, budget, Hq, Hkv, hd, max_ctx, self.scale, _ptr(self.Y),
            _ptr(self.ws), self.ws.numel(), _stream()))
        return self.Y


# The calls below run on the current device and refuse tensors of another one (-1: no GPU).
_current = _device or torch.cuda.current_device


def _need_on(dev: int, t: torch.Tensor, name: str, dtype, shape=None):
    """_need, and the tensor lives on the current device `dev`."""
    if (t.dtype is dtype and t.get_device() == dev and (shape is None or t.shape == shape)
            and t.is_contiguous()):
        return
    _need(t, name, dtype, shape)
    raise ValueError(f"{name}: tensor on {t.device}, the current device is cuda:{dev}")


def _need_rows(dev: int, t: torch.Tensor, name: str, dtype, inner, steps) -> int:
    """[rows, *inner], each row contiguous (its strides are `steps`); the rows may be apart.
    Returns their distance in elements."""
    shape, strides = t.shape, t.stride()
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.get_device() != dev:
        if not t.is_cuda:
            raise TypeError(f"{name}: expected a GPU tensor")
        raise ValueError(f"{name}: tensor on {t.device}, the current device is cuda:{dev}")
    if shape[1:] != inner:
        raise ValueError(f"{name}: expected [rows, {', '.join(map(str, inner))}], got {tuple(shape)}")
    if strides[1:] != steps and any(n > 1 and a != b
                                    for n, a, b in zip(inner, strides[1:], steps)):
        raise ValueError(f"{name}: each row must be contiguous")
    return strides[0] if shape[0] > 1 else inner[0] * steps[0]


def _need_pools(dev, K_pages, V_pages, dtype, page):
    """page: (page_rows, Hkv, head_dim)"""
    _need_on(dev, K_pages, "K_pages", dtype)
    if K_pages.shape[1:] != page:
        raise ValueError(f"K_pages: expected [pages, {page[0]}, {page[1]}, {page[2]}], "
                         f"got {tuple(K_pages.shape)}")
    _need_on(dev, V_pages, "V_pages", dtype, K_pages.shape)


class PagedKVReserve:
    """kv_reserve_paged: pages for the requests' next rows, from the free-page stack into
    their block tables, and the slot map of the new rows."""

    def __init__(self, batch, max_pages, num_pages, page_rows, max_new, slot_map=True):
        """max_new: upper bound of n_new and, with slot_map, the slot map's columns."""
        self.lib = load()
        self.shape = (batch, max_pages, num_pages, int(page_rows), max_new)
        self.slot_map = slot_map

    def __call__(self, block_table, held_pages, ctx_len, n_new, free_pages, n_free):
        """block_table [batch, max_pages] and free_pages [num_pages] are updated in place.
        Returns new tensors: pages held [batch], free pages [1], requests that are short [1]
        (all int32) and the slot map [batch, max_new] int64 (None without slot_map)."""
        batch, max_pages, num_pages, page_rows, max_new = self.shape
        dev = _current()
        _need_on(dev, block_table, "block_table", torch.int32, (batch, max_pages))
        _need_on(dev, held_pages, "held_pages", torch.int32, (batch,))
        _need_on(dev, ctx_len, "ctx_len", torch.int32, (batch,))
        _need_on(dev, n_new, "n_new", torch.int32, (batch,))
        _need_on(dev, free_pages, "free_pages", torch.int32, (num_pages,))
        _need_on(dev, n_free, "n_free", torch.int32, (1,))
        # one allocation for the three; without requests the call writes nothing
        counts = block_table.new_empty(batch + 2) if batch else torch.cat(
            (n_free.clamp(0, num_pages), torch.zeros_like(n_free)))
        held, free, short = counts.split_with_sizes((batch, 1, 1))
        slots = block_table.new_empty((batch, max_new), dtype=torch.int64) if self.slot_map else None
        at = counts.data_ptr()
        _lib.check(self.lib, "kv_reserve_paged", self.lib.kv_reserve_paged(
            _ptr(block_table), max_pages, _ptr(held_pages), _ptr(ctx_len), _ptr(n_new), batch,
            max_new, _ptr(free_pages), _ptr(n_free), num_pages, page_rows, at, at + 4 * batch,
            at + 4 * batch + 4, _ptr(slots), _stream()))
        return held, free, short, slots


class PagedKVAppend:
    """kv_append_paged: new K/V rows into the page pools through a slot map."""

    def __init__(self, Hkv, head_dim, page_rows, dtype=BF16):
        self.lib = load()
        self.shape = (Hkv, head_dim, int(page_rows), dtype)
        self._page = (int(page_rows), Hkv, head_dim)
        self._row, self._steps = (Hkv, head_dim), (head_dim, 1)

    def __call__(self, K_new, V_new, slot_map, K_pages, V_pages):
        """K_new, V_new: [rows, Hkv, head_dim], rows contiguous in themselves (slices of a fused
        projection's rows are fine).  slot_map: int64 of `rows` entries in any shape."""
        Hkv, hd, page_rows, dtype = self.shape
        tdt = _TORCH_DT[dtype]
        dev = _current()
        ks = _need_rows(dev, K_new, "K_new", tdt, self._row, self._steps)
        vs = _need_rows(dev, V_new, "V_new", tdt, self._row, self._steps)
        rows = K_new.shape[0]
        _need_on(dev, slot_map, "slot_map", torch.int64)
        if V_new.shape[0] != rows or slot_map.numel() != rows:
            raise ValueError(f"K_new has {rows} rows, V_new {V_new.shape[0]}, slot_map "
                             f"{slot_map.numel()} entries")
        _need_pools(dev, K_pages, V_pages, tdt, self._page)
        _lib.check(self.lib, "kv_append_paged", self.lib.kv_append_paged(
            _ptr(K_new), _ptr(V_new), ks, vs, _ptr(slot_map), rows, Hkv, hd, dtype,
            _ptr(K_pages), _ptr(V_pages), K_pages.shape[0], page_rows, _stream()))
        return K_pages, V_pages


class PagedDecodeAttention:
    """decode_attn_paged: attention of one new token per request over a paged KV cache."""

    def __init__(self, batch, Hq, Hkv, head_dim, max_len, page_rows, dtype=BF16, scale=None):
        self.lib = load()
        self.scale = float(scale if scale is not None else head_dim ** -0.5)
        self.shape = (batch, Hq, Hkv, head_dim, max_len, int(page_rows), dtype)
        _lib.check(self.lib, "decode_attn_paged_validate",
                   self.lib.decode_attn_paged_validate(*self.shape, self.scale))
        self.ws_bytes = self.lib.decode_attn_paged_workspace_bytes(*self.shape)
        self._page = (int(page_rows), Hkv, head_dim)
        self._row, self._steps = (Hq, head_dim), (head_dim, 1)

    def __call__(self, Q, K_pages, V_pages, block_table, kv_len, out=None):
        """Q: [batch, Hq, head_dim], requests may be apart.  Each call has scratch of its own
        (from torch's allocator, on the current stream), so calls may overlap."""
        batch, Hq, Hkv, hd, max_len, page_rows, dtype = self.shape
        tdt = _TORCH_DT[dtype]
        dev = _current()
        qs = _need_rows(dev, Q, "Q", tdt, self._row, self._steps)
        if Q.shape[0] != batch:
            raise ValueError(f"Q: expected {batch} requests, got {Q.shape[0]}")
        _need_pools(dev, K_pages, V_pages, tdt, self._page)
        _need_on(dev, block_table, "block_table", torch.int32)
        if block_table.dim() != 2 or block_table.shape[0] != batch:
            raise ValueError(f"block_table: expected [{batch}, max_pages], "
                             f"got {tuple(block_table.shape)}")
        _need_on(dev, kv_len, "kv_len", torch.int32, (batch,))
        if out is None:
            O = Q.new_empty((batch, Hq, hd))
        else:
            O = out
            _need_on(dev, O, "O", tdt, (batch, Hq, hd))
        ws = Q.new_empty(self.ws_bytes, dtype=torch.uint8) if self.ws_bytes else None
        _lib.check(self.lib, "decode_attn_paged", self.lib.decode_attn_paged(
            _ptr(Q), qs, _ptr(K_pages), _ptr(V_pages), K_pages.shape[0], page_rows,
            _ptr(block_table), block_table.shape[1], _ptr(kv_len), batch, Hq, Hkv, hd, max_len,
            dtype, self.scale, _ptr(O), _ptr(ws), self.ws_bytes, _stream()))
        return O


class TokenSampler:
    """taps_sample: tokens from logits with temperature, top-k, top-p and min-p and given
    random numbers."""

    def __init__(self, batch, budget, vocab, dtype=BF16):
        """budget: rows per request (the nodes of its tree; 1 without a draft)."""
        self.lib = load()
        self.shape = (batch, budget, vocab, dtype)
        _lib.check(self.lib, "taps_sample_validate",
                   self.lib.taps_sample_validate(batch, budget, vocab, vocab, dtype))

    def __call__(self, logits, u, n_nodes=None, temperature=None, top_k=None, top_p=None,
                 min_p=None):
        """logits: [batch, budget, vocab], rows may be apart (a padded vocabulary's slice) and
        begin anywhere unless a row is whole 16-byte units (then at one); u: [batch, budget]
        float32; n_nodes: [batch] int32 or None; the settings: [batch] tensors (top_k int32, the
        others float32) or None.  Returns the tokens [batch, budget] int32 and their
        probabilities, float32."""
        batch, budget, vocab, dtype = self.shape
        if logits.shape != (batch, budget, vocab):
            raise ValueError(f"logits: expected [{batch}, {budget}, {vocab}], "
                             f"got {tuple(logits.shape)}")
        if batch > 1 and budget > 1 and logits.stride(0) != budget * logits.stride(1):
            raise ValueError("logits: all rows must be the same distance apart")
        dev, tdt = _current(), _TORCH_DT[dtype]
        if logits.is_contiguous():
            _need_on(dev, logits, "logits", tdt)
            stride = vocab
        else:
            rows = logits[0] if batch == 1 else logits[:, 0] if budget == 1 else logits.flatten(0, 1)
            stride = _need_rows(dev, rows, "logits", tdt, (vocab,), (1,))
        _need_on(dev, u, "u", torch.float32, (batch, budget))
        for t, name, dt in ((n_nodes, "n_nodes", torch.int32), (top_k, "top_k", torch.int32),
                            (temperature, "temperature", torch.float32),
                            (top_p, "top_p", torch.float32), (min_p, "min_p", torch.float32)):
            if t is not None:
                _need_on(dev, t, name, dt, (batch,))
        tokens, probs = u.new_empty((batch, budget), dtype=torch.int32), torch.empty_like(u)
        st = _lib.Sampling(_ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p))
        _lib.check(self.lib, "taps_sample", self.lib.taps_sample(
            _ptr(logits), stride, batch, budget, vocab, dtype, _ptr(n_nodes), ctypes.byref(st),
            _ptr(u), _ptr(tokens), _ptr(probs), None, 0, _stream()))
        return tokens, probs
