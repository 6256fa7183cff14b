"""Convenience wrapper that owns a context and marshals torch tensors.

Marshalling only: allocation of output tensors, struct filling, and calls
into the HIP library.  Nothing here computes any part of the drafting path.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import binding as B


def _dtype_code(dtype: str) -> int:
    return B.PRISM_BF16 if dtype == "bf16" else B.PRISM_F32


class Drafter:
    """One drafting context on the current GPU.

    `shape` is any object with the model/capacity attributes of
    prism_config (hidden, n_q_heads, n_kv_heads, head_dim, ffn, vocab,
    feat_width, rope_theta, rms_eps, dtype ("f32"/"bf16"), kv_block_size,
    batch, tree_width, tree_nodes) plus n_sets (M), n_steps and
    blocks_per_seq.
    """

    def __init__(self, shape, max_batch: Optional[int] = None, max_steps: Optional[int] = None,
                 max_blocks_per_seq: Optional[int] = None, max_new_rows: Optional[int] = None):
        self.shape = shape
        cfg = B.prism_config()
        cfg.hidden = shape.hidden
        cfg.n_q_heads = shape.n_q_heads
        cfg.n_kv_heads = shape.n_kv_heads
        cfg.head_dim = shape.head_dim
        cfg.ffn = shape.ffn
        cfg.vocab = shape.vocab
        cfg.n_sets = shape.M
        cfg.max_steps = max_steps or shape.n_steps
        cfg.feat_width = shape.feat_width
        cfg.rope_theta = shape.rope_theta
        cfg.rms_eps = shape.rms_eps
        cfg.dtype = _dtype_code(shape.dtype)
        cfg.kv_block_size = shape.kv_block_size
        cfg.max_batch = max_batch or shape.batch
        cfg.max_blocks_per_seq = max_blocks_per_seq or shape.blocks_per_seq
        cfg.tree_width = shape.tree_width
        cfg.tree_nodes = shape.tree_nodes
        cfg.max_new_rows = (max_new_rows if max_new_rows is not None
                            else getattr(shape, "max_new_rows", 0))
        self.cfg = cfg
        self.ctx = B.prism_create(cfg)
        self.device = torch.device("cuda", torch.cuda.current_device())
        self._cache_setup()

    def close(self):
        if self.ctx:
            B.prism_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # weights ------------------------------------------------------------------
    def load(self, weights, sets: Optional[Sequence[int]] = None):
        B.prism_draft_load_shared(self.ctx, weights.embed, weights.lm_head, weights.final_norm)
        ids = range(len(weights.sets)) if sets is None else sets
        for s, ps in zip(ids, weights.sets):
            self.load_set(s, ps)

    def load_set(self, s: int, ps):
        p = B.prism_param_set()
        for name in ("w_fc", "g1", "w_q", "w_k", "w_v", "w_o", "g2", "w_gate", "w_up", "w_down"):
            setattr(p, "d_" + name, B.ptr(getattr(ps, name)))
        p.feat_width = ps.feat_width
        B.prism_draft_load_params(self.ctx, s, p)

    def set_step_map(self, f_map):
        B.prism_set_step_map(self.ctx, f_map)

    # batches ------------------------------------------------------------------
    def batch(self, inp) -> B.prism_batch:
        b = B.prism_batch()
        b.batch = int(inp.tokens.shape[0])
        b.d_tokens = B.ptr(inp.tokens)
        b.d_features = B.ptr(inp.features)
        b.d_ctx_lens = B.ptr(inp.ctx_lens)
        b.d_k_pool = B.ptr(inp.k_pool)
        b.d_v_pool = B.ptr(inp.v_pool)
        b.d_block_table = B.ptr(inp.block_table)
        b.n_pool_blocks = int(inp.k_pool.shape[0])
        return self._sizes(b)

    # calls --------------------------------------------------------------------
    def chain_buffers(self, nb: int, K: int, logits=False, hidden=False):
        dev = self.device
        out = {"tokens": torch.full((nb, K), -1, dtype=torch.int32, device=dev)}
        out["logits"] = (torch.empty((nb, K, self.shape.vocab), dtype=torch.float32, device=dev)
                         if logits else None)
        out["hidden"] = (torch.empty((nb, K, self.shape.hidden), dtype=torch.float32, device=dev)
                         if hidden else None)
        return out

    def chain(self, inp, K: Optional[int] = None, logits=False, hidden=False, out=None,
              batch=None):
        K = K or self.shape.n_steps
        b = batch if batch is not None else self.batch(inp)
        if out is None:
            out = self.chain_buffers(b.batch, K, logits, hidden)
        B.prism_draft_chain(self.ctx, b, K, out["tokens"], out["logits"], out["hidden"])
        return out

    def chain_sample(self, inp, temperature: float, K: Optional[int] = None, logits=False,
                     hidden=False, out=None, batch=None):
        """Stochastic chain: tokens drawn from softmax(logits / T) with the
        uniforms inp.uniforms [B, K]; out["logp"] holds log p_draft."""
        K = K or self.shape.n_steps
        b = batch if batch is not None else self.batch(inp)
        if out is None:
            out = self.chain_buffers(b.batch, K, logits, hidden)
            out["logp"] = torch.full((b.batch, K), float("nan"), dtype=torch.float32,
                                     device=self.device)
        B.prism_draft_chain_sample(self.ctx, b, K, temperature, inp.uniforms, out["tokens"],
                                   out.get("logp"), out["logits"], out["hidden"])
        return out

    def chain_catchup(self, inp, K: Optional[int] = None, logits=False, hidden=False, out=None,
                      batch=None):
        """Chain whose step 1 is the prefill over inp.new_tokens / new_features
        (rows delimited by inp.new_offsets)."""
        K = K or self.shape.n_steps
        b = batch if batch is not None else self.batch(inp)
        if out is None:
            out = self.chain_buffers(b.batch, K, logits, hidden)
        cu = B.prism_catchup()
        cu.total_rows = int(inp.new_tokens.shape[0])
        cu.d_offsets = B.ptr(inp.new_offsets)
        cu.d_tokens = B.ptr(inp.new_tokens)
        cu.d_features = B.ptr(inp.new_features)
        B.prism_draft_chain_catchup(self.ctx, b, cu, K, out["tokens"], out["logits"],
                                    out["hidden"])
        return out

    def tree_buffers(self, nb: int, depth: int, debug=True, logits=False):
        dev = self.device
        w, v = self.shape.tree_width, self.shape.tree_nodes
        C = w + (depth - 1) * w * w
        i32 = dict(dtype=torch.int32, device=dev)
        out = {"tokens": torch.full((nb, v), -1, **i32), "parent": torch.full((nb, v), -2, **i32),
               "depth": torch.zeros((nb, v), **i32),
               "score": torch.zeros((nb, v), dtype=torch.float32, device=dev),
               "mask": torch.zeros((nb, v), dtype=torch.int64, device=dev)}
        if debug:
            out["cand_tokens"] = torch.full((nb, C), -1, **i32)
            out["cand_parent"] = torch.full((nb, C), -2, **i32)
            out["cand_score"] = torch.zeros((nb, C), dtype=torch.float32, device=dev)
            out["frontier"] = torch.full((nb, max(depth - 1, 1), w), -1, **i32)
        if logits:
            out["logits"] = torch.full((depth, nb, w, self.shape.vocab), float("nan"),
                                       dtype=torch.float32, device=dev)
        return out

    def tree(self, inp, depth: Optional[int] = None, debug=True, logits=False, out=None,
             batch=None):
        depth = depth or self.shape.n_steps
        b = batch if batch is not None else self.batch(inp)
        if out is None:
            out = self.tree_buffers(b.batch, depth, debug, logits)
        t = B.prism_tree_out()
        for k in ("tokens", "parent", "depth", "score", "mask"):
            setattr(t, "d_" + k, B.ptr(out[k]))
        for k in ("cand_tokens", "cand_parent", "cand_score", "frontier", "logits"):
            setattr(t, "d_" + k, B.ptr(out.get(k)))
        B.prism_draft_tree(self.ctx, b, depth, t)
        return out

    def score_tree(self, inp, tokens, depth, mask, out=None, batch=None):
        """Target-side scoring of B draft trees (this context holds the
        scoring model): logits [B, v+1, V] of the root and every node under
        the tree mask.  inp describes the scoring model's own sequences
        (root tokens, features, prior KV)."""
        b = batch if batch is not None else self.batch(inp)
        Bn, v = int(tokens.shape[0]), int(tokens.shape[1])
        if out is None:
            out = torch.empty((Bn, v + 1, self.shape.vocab), dtype=torch.float32,
                              device=self.device)
        B.prism_score_tree(self.ctx, b, v, tokens, depth, mask, out)
        return out

    def verify_chain(self, target_logits, draft_tokens, temperature: float = 0.0,
                     draft_logits=None, uniforms=None):
        """Sec. 2 verification of B chains of K drafts; returns kept counts
        and next tokens [B]."""
        Bn, K = int(draft_tokens.shape[0]), int(draft_tokens.shape[1])
        n = torch.empty(Bn, dtype=torch.int32, device=self.device)
        nxt = torch.empty(Bn, dtype=torch.int32, device=self.device)
        B.prism_verify_chain(self.ctx, Bn, K, temperature, target_logits, draft_logits,
                             draft_tokens, uniforms, n, nxt)
        return {"n": n, "next": nxt}

    def verify_tree(self, target_logits, tokens, parent):
        """Greedy verification of B draft trees; returns kept counts, kept
        node paths [B, nodes] (-1 padded) and next tokens."""
        Bn, v = int(tokens.shape[0]), int(tokens.shape[1])
        n = torch.empty(Bn, dtype=torch.int32, device=self.device)
        path = torch.empty((Bn, v), dtype=torch.int32, device=self.device)
        nxt = torch.empty(Bn, dtype=torch.int32, device=self.device)
        B.prism_verify_tree(self.ctx, Bn, v, target_logits, tokens, parent, n, path, nxt)
        return {"n": n, "path": path, "next": nxt}

    def step(self, k: int, inp, rows: dict, topk: int = 1, logits=False, batch=None):
        """One pass of step k on explicit rows.  `rows` holds device tensors:
        tokens, feat, seq, pos, slot and optionally feat_rows, tree_bits;
        feat is fp32 (hidden states) or the context dtype (target features)."""
        b = batch if batch is not None else self.batch(inp)
        R = int(rows["tokens"].shape[0])
        dev = self.device
        io = B.prism_step_io()
        io.rows = R
        io.d_tokens = B.ptr(rows["tokens"])
        io.d_feat = B.ptr(rows["feat"])
        io.feat_dtype = B.PRISM_BF16 if rows["feat"].dtype == torch.bfloat16 else B.PRISM_F32
        io.d_feat_rows = B.ptr(rows.get("feat_rows"))
        io.d_seq = B.ptr(rows["seq"])
        io.d_pos = B.ptr(rows["pos"])
        io.d_slot = B.ptr(rows["slot"])
        io.d_tree_bits = B.ptr(rows.get("tree_bits"))
        io.kv = __import__("ctypes").pointer(b)
        io.topk = topk
        out = {"hidden": torch.empty((R, self.shape.hidden), dtype=torch.float32, device=dev),
               "ids": torch.empty((R, topk), dtype=torch.int32, device=dev),
               "logp": torch.empty((R, topk), dtype=torch.float32, device=dev),
               "logits": (torch.empty((R, self.shape.vocab), dtype=torch.float32, device=dev)
                          if logits else None)}
        io.d_hidden_out = B.ptr(out["hidden"])
        io.d_topk_ids = B.ptr(out["ids"])
        io.d_topk_logp = B.ptr(out["logp"])
        io.d_logits = B.ptr(out["logits"])
        B.prism_draft_step(self.ctx, k, io)
        return out

    # long-context draft cache ---------------------------------------------------
    # These calls take a few microseconds on the GPU when they are small, so the
    # path to them is kept short: the sizes that the checks compare with are
    # read from the config once, and one struct per call is filled again and
    # again (a context is used by one host thread at a time).
    def _cache_setup(self):
        c = self.cfg
        self._dt = torch.bfloat16 if c.dtype == B.PRISM_BF16 else torch.float32
        self._nq, self._nkv, self._d = c.n_q_heads, c.n_kv_heads, c.head_dim
        self._bs, self._columns = c.kv_block_size, c.max_blocks_per_seq
        self._qkv = (self._nq + 2 * self._nkv) * self._d
        self._io = (B.prism_cache_rows(), B.prism_cache_attention(), B.prism_cache_selection(),
                    B.prism_cache_eviction())
        self._scratch_bytes = {}

    def _stream(self) -> int:
        return torch._C._cuda_getCurrentRawStream(self.device.index)

    def _expect(self, t, name: str, shape, dtype) -> int:
        """Data pointer of a contiguous tensor of this shape and type on the
        context's device."""
        if (type(t) is torch.Tensor and t.dtype is dtype and t.shape == shape
                and t.device == self.device and t.is_contiguous()):
            return t.data_ptr()
        if not isinstance(t, torch.Tensor):
            raise TypeError("%s must be a tensor" % name)
        if t.dtype != dtype:
            raise TypeError("%s must be %s, not %s" % (name, dtype, t.dtype))
        if t.device != self.device:
            raise ValueError("%s is on %s, the context on %s" % (name, t.device, self.device))
        if tuple(t.shape) != tuple(shape):
            raise ValueError("%s must have shape %s, not %s" % (name, tuple(shape), tuple(t.shape)))
        if not t.is_contiguous():
            raise ValueError("%s must be contiguous" % name)
        return t.data_ptr()          # a subclass of Tensor

    def _scratch(self, call: int, batch: int, max_len: int, like):
        key = (call, batch, max_len)
        n = self._scratch_bytes.get(key)
        if n is None:
            n = B.prism_cache_scratch(self.ctx, call, batch, max_len)
            if len(self._scratch_bytes) >= 1024:      # callers that pass a new bound at every step
                self._scratch_bytes.clear()
            self._scratch_bytes[key] = n
        return n, like.new_empty(-(-n // like.element_size())) if n else None

    def cache(self, lens, k_pool, v_pool, block_table) -> B.prism_batch:
        """The sequences of a cache call: lens [B] int32 slots held, pools
        [blocks, n_kv_heads, kv_block_size, head_dim], block_table
        [B, max_blocks_per_seq] int32.  Keeps the tensors alive."""
        nb, n = int(lens.shape[0]), int(k_pool.shape[0])
        pool = (n, self._nkv, self._bs, self._d)
        kv = B.prism_batch()
        kv.batch = nb
        kv.d_ctx_lens = self._expect(lens, "lens", (nb,), torch.int32)
        kv.d_k_pool = self._expect(k_pool, "k_pool", pool, self._dt)
        kv.d_v_pool = self._expect(v_pool, "v_pool", pool, self._dt)
        kv.d_block_table = self._expect(block_table, "block_table", (nb, self._columns), torch.int32)
        kv.n_pool_blocks = n
        kv.tensors = (lens, k_pool, v_pool, block_table)
        return self._sizes(kv)

    def _sizes(self, kv):
        """What the cache calls compare a batch's tensors with (the batches of
        drafting calls, batch(), can be passed to them too)."""
        n = kv.n_pool_blocks
        kv.nb, kv.slots, kv.summary = kv.batch, (n, self._nkv, self._bs), (n, self._nkv, 2, self._d)
        return kv

    def cache_append(self, kv, qkv, q_gain=None, k_gain=None, offsets=None, positions=None,
                     weights=None, out=None):
        """Normalise, rotate and append rows: qkv [T, (n_q + 2 n_kv) * d] of
        the sequences in order (rows offsets[b] .. offsets[b+1] - 1; None: one
        row each) at positions[b] (None: lens[b]) and the slots behind each
        context; weights (slot weights) are set to 0 there.  Returns the
        queries [T, n_q, d]."""
        dt, T = self._dt, qkv.shape[0]
        io = self._io[0]
        io.kv = ctypes.addressof(kv)
        io.rows = T
        io.d_qkv = self._expect(qkv, "qkv", (T, self._qkv), dt)
        io.d_q_gain = None if q_gain is None else self._expect(q_gain, "q_gain", (self._d,), dt)
        io.d_k_gain = None if k_gain is None else self._expect(k_gain, "k_gain", (self._d,), dt)
        io.d_offsets = (None if offsets is None
                        else self._expect(offsets, "offsets", (kv.nb + 1,), torch.int32))
        io.d_positions = (None if positions is None
                          else self._expect(positions, "positions", (kv.nb,), torch.int32))
        io.d_weights = (None if weights is None
                        else self._expect(weights, "weights", kv.slots, torch.float32))
        shape = (T, self._nq, self._d)
        if out is None:
            out = qkv.new_empty(shape)
            io.d_q = out.data_ptr()
        else:
            io.d_q = self._expect(out, "out", shape, dt)
        B.prism_cache_append(self.ctx, io, self._stream())
        return out

    def cache_attend(self, kv, q, n_new: int = 0, max_len: int = 0, blocks=None, weights=None,
                     lse: bool = False, out=None):
        """Attention of one query row per sequence, q [B, n_q, d], over its
        cache or over blocks [B, n_kv, n] of it; adds what every slot receives
        to weights.  Returns out [B, n_q, d] and, if asked for, lse [B, n_q]."""
        dt, nb = self._dt, kv.nb
        shape = (nb, self._nq, self._d)
        io = self._io[1]
        io.kv = ctypes.addressof(kv)
        io.n_new = n_new
        io.max_len = span = max_len
        io.d_q = self._expect(q, "q", shape, dt)
        if blocks is None:
            io.d_blocks = None
        else:
            io.n_blocks = n = int(blocks.shape[-1])
            io.d_blocks = self._expect(blocks, "blocks", (nb, self._nkv, n), torch.int32)
            if n < 1:
                raise ValueError("blocks has no entry")
            span = min(n, self._columns) * self._bs
        call = B.PRISM_CACHE_ATTEND
        io.d_weights = None
        if weights is not None:
            io.d_weights = self._expect(weights, "weights", kv.slots, torch.float32)
            call = B.PRISM_CACHE_ATTEND_WEIGHTS
        if out is None:
            out = q.new_empty(shape)
            io.d_out = out.data_ptr()
        else:
            io.d_out = self._expect(out, "out", shape, dt)
        sums = torch.empty(shape[:2], dtype=torch.float32, device=self.device) if lse else None
        io.d_lse = None if sums is None else sums.data_ptr()
        io.scratch_bytes, scratch = self._scratch(call, nb, span, q)
        io.d_scratch = None if scratch is None else scratch.data_ptr()
        B.prism_cache_attend(self.ctx, io, self._stream())
        return {"out": out, "lse": sums}

    def summary_buffer(self, kv):
        """A summary pool [blocks, n_kv, 2, d] for cache_summarize."""
        return torch.zeros(kv.summary, dtype=self._dt, device=self.device)

    def cache_summarize(self, kv, summary, n_new: int = 0, span: int = 0):
        """Write the key minima and maxima of the blocks that hold the last
        span slots (0: of every block) into summary [blocks, n_kv, 2, d]."""
        self._expect(summary, "summary", kv.summary, self._dt)
        B.prism_cache_summarize(self.ctx, kv, n_new, span, summary, self._stream())
        return summary

    def cache_select(self, kv, q, summary, n_blocks: int, n_first: int = 0, n_last: int = 0,
                     n_new: int = 0, max_len: int = 0, out=None):
        """The n_blocks blocks of largest score bound for each sequence and KV
        head, [B, n_kv, n_blocks] int32: increasing, then -1."""
        nb = kv.nb
        io = self._io[2]
        io.kv = ctypes.addressof(kv)
        io.n_new = n_new
        io.max_len = max_len
        io.d_q = self._expect(q, "q", (nb, self._nq, self._d), self._dt)
        io.d_summary = self._expect(summary, "summary", kv.summary, self._dt)
        io.n_blocks = n_blocks
        io.n_first = n_first
        io.n_last = n_last
        shape = (nb, self._nkv, max(n_blocks, 0))
        if out is None:
            out = torch.empty(shape, dtype=torch.int32, device=self.device)
            io.d_blocks = out.data_ptr()
        else:
            io.d_blocks = self._expect(out, "out", shape, torch.int32)
        io.scratch_bytes, scratch = self._scratch(B.PRISM_CACHE_SELECT, nb, max_len, q)
        io.d_scratch = scratch.data_ptr()
        B.prism_cache_select(self.ctx, io, self._stream())
        return out

    def cache_evict(self, kv, new_table, weights, n_keep: int, n_first: int = 0, n_recent: int = 0,
                    max_len: int = 0):
        """Copy the n_keep slots of largest weight to the blocks of new_table
        [B, max_blocks_per_seq].  Advance lens over appended rows before: the
        candidates are the slots below them.  Returns kept [B, n_kv, n_keep]
        (old slots) and lens [B], the lengths of the new cache; kept keys keep
        the rotation of their old positions (continue with explicit ones)."""
        nb = kv.nb
        io = self._io[3]
        io.kv = ctypes.addressof(kv)
        io.max_len = max_len
        io.d_new_table = self._expect(new_table, "new_table", (nb, self._columns), torch.int32)
        io.d_weights = self._expect(weights, "weights", kv.slots, torch.float32)
        io.n_keep = n_keep
        io.n_first = n_first
        io.n_recent = n_recent
        kept = new_table.new_empty((nb, self._nkv, max(n_keep, 0)))
        lens = new_table.new_empty(nb)
        io.d_kept = kept.data_ptr()
        io.d_new_lens = lens.data_ptr()
        io.scratch_bytes, scratch = self._scratch(B.PRISM_CACHE_EVICT, nb, max_len, weights)
        io.d_scratch = scratch.data_ptr()
        B.prism_cache_evict(self.ctx, io, self._stream())
        return {"kept": kept, "lens": lens}

    def device_status(self) -> int:
        return B.prism_device_status(self.ctx)
