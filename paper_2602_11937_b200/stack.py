"""Per-layer pattern driver: one decode step, or the prompts before it, of the attention stack of a model whose layers are each
full-context or sliding-window (the per-layer choice the paper's architecture search makes, Section
"Window attention for long-context inference").

A ``DecodeStack`` only loops over the C-ABI calls (fused quantise-and-append, with the position rotation of q and k
when it is given a rotation, then attention, per layer); every step of the path is a kernel of the library.  ``capture()`` records one step into a CUDA graph so a
36-layer step is one launch from the host's point of view.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import torch

from . import binding as B
from .paging import blocks_twice, window_keys_lost


class DecodeStack:
    def __init__(self, windows: Sequence[int], k_caches: Sequence[torch.Tensor], v_caches: Sequence[torch.Tensor],
                 seq_lens: torch.Tensor, block_tables: Sequence[Optional[torch.Tensor]], max_blocks_per_seq: int,
                 k_scales: Sequence[Optional[torch.Tensor]], v_scales: Sequence[Optional[torch.Tensor]],
                 sinks: Sequence[Optional[torch.Tensor]], kv_dtype: int = B.KV_FP8_E4M3, num_splits: int = 0,
                 rope: Optional[B.Rope] = None):
        """rope: q and k of ``step`` arrive unrotated and are rotated on their way (one table for all layers); None: they
        arrive rotated.  A sequence that a layer skips (longer than its table row, or at a position the rotation does not
        have: ``status`` says so) has no valid output in that step."""
        n = len(windows)
        assert all(len(x) == n for x in (k_caches, v_caches, block_tables, k_scales, v_scales, sinks))
        self.windows = list(windows)
        self.batch = int(seq_lens.shape[0])
        self.num_splits = num_splits
        self.sinks = list(sinks)
        self._keep = (k_caches, v_caches, seq_lens, block_tables, k_scales, v_scales)  # the views hold raw pointers
        self.descs = [B.layer_desc(window=w, kv_dtype=kv_dtype) for w in windows]
        self.views = [B.kv_view(k_caches[i], v_caches[i], seq_lens, block_table=block_tables[i],
                                max_blocks_per_seq=max_blocks_per_seq, k_scale=k_scales[i], v_scale=v_scales[i])
                      for i in range(n)]
        dev = seq_lens.device
        nbytes = max(B.puzzle_decode_attn_workspace_bytes(d, self.batch, num_splits) for d in self.descs)
        self.workspace = torch.zeros(nbytes, dtype=torch.uint8, device=dev)
        B.puzzle_decode_attn_workspace_init(self.descs[0], self.batch, self.workspace)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.rope = rope
        # the layers run one after the other, so one buffer holds each layer's rotated queries in turn
        self.q_rotated = None if rope is None else torch.empty(
            self.batch, self.descs[0].num_q_heads, self.descs[0].head_dim, dtype=torch.bfloat16, device=dev)
        self.graph = None
        self._no_rings = {}      # window layers whose tables have no block twice: those tables' versions

    def step(self, q: List[torch.Tensor], k_new: List[torch.Tensor], v_new: List[torch.Tensor],
             out: List[torch.Tensor], stream=None) -> None:
        """Append + attention for every layer, in order, on ``stream`` (all layers share one workspace, so
        their kernels run one after the other on that stream)."""
        for i in range(len(self.windows)):
            q_i = q[i]
            if self.rope is None:
                B.puzzle_kv_append(self.descs[i], self.views[i], k_new[i], v_new[i], dev_status=self.status, stream=stream)
            else:
                B.puzzle_kv_append_rope(self.descs[i], self.views[i], self.rope, q_i, k_new[i], v_new[i], self.q_rotated,
                                        dev_status=self.status, stream=stream)
                q_i = self.q_rotated
            B.puzzle_decode_attn(self.descs[i], self.views[i], q_i, self.sinks[i], out[i], None,
                                 num_splits=self.num_splits, workspace=self.workspace, dev_status=self.status,
                                 stream=stream)

    def prefill(self, q: List[torch.Tensor], k_new: List[torch.Tensor], v_new: List[torch.Tensor], starts: torch.Tensor,
                out: List[torch.Tensor], continued: bool = False, stream=None) -> None:
        """Append + attention of the prompts' tokens for every layer.  q[i], k_new[i], v_new[i]: bf16 [tokens][heads][D] of layer
        i, the tokens of all sequences behind each other (slices of one projection's output will do); starts: int32
        [batch + 1], first row of every sequence and the end of the last; out[i]: bf16 [tokens][Hq][D].  The lengths that
        the stack was made with count these tokens already.

        continued False: every sequence begins with these tokens; they attend to one another's keys and values as they are, and of
        a window layer only the tokens that a later step can see go into the cache (a ring of ``window_ring_blocks`` takes
        them).  continued True: pieces behind earlier tokens attend to the cache.  A window layer's cache then has to
        hold the window before the piece's first token together with the piece, which a ring of R blocks does for
        ``16 R + 1 - W`` tokens of a sequence; longer pieces over a ring are refused with a ValueError before anything is stored
        (give the pieces in shorter ones, or the layer a longer ring).  To know, the call looks at the tables of
        window layers and waits for the answer; not again at those that have no block twice, until torch changes them (36 layers, 8
        x 5 tokens: 790 us a call, 1290 with a look).  Not for capture: buffers are allocated as needed."""
        tokens = q[0].shape[0]
        if continued and tokens > 0:
            self._check_rings(starts, tokens, stream)
        d0 = self.descs[0]
        rotate = self.rope is not None
        room = lambda heads: torch.empty(tokens, heads, d0.head_dim, dtype=torch.bfloat16, device=q[0].device)
        q_rot, k_rot = (room(d0.num_q_heads), room(d0.num_kv_heads)) if rotate else (None, None)
        workspace = None
        if continued:
            nbytes = B.puzzle_chunk_attn_workspace_bytes(d0, self.batch, tokens)
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=q[0].device)
        if stream is not None:                       # the buffers are used there, whatever stream they were made on
            stream.wait_stream(torch.cuda.current_stream())
            for t in (q_rot, k_rot, workspace):
                if t is not None:
                    t.record_stream(stream)
        for i, w in enumerate(self.windows):
            keep = 0 if continued or w == 0 else -(-w // d0.block_size) * d0.block_size
            B.puzzle_kv_append_packed(self.descs[i], self.views[i], self.rope, q[i] if rotate else None, k_new[i], v_new[i], starts,
                                      q_rot, k_rot, keep, dev_status=self.status, stream=stream)
            q_i, k_i = (q_rot, k_rot) if rotate else (q[i], k_new[i])
            if continued:
                B.puzzle_chunk_attn(self.descs[i], self.views[i], q_i, starts, self.sinks[i], out[i], workspace=workspace,
                                    dev_status=self.status, stream=stream)
            else:
                B.puzzle_prompt_attn(self.descs[i], q_i, k_i, v_new[i], starts, self.sinks[i], out[i], dev_status=self.status,
                                     stream=stream)

    def _check_rings(self, starts: torch.Tensor, tokens: int, stream) -> None:
        _, _, seq_lens, tables, _, _ = self._keep
        version = lambda i: None if tables[i].is_inference() else tables[i]._version
        layers = [i for i, w in enumerate(self.windows) if w > 0 and tables[i] is not None and
                  (version(i) is None or self._no_rings.get(i) != version(i))]
        if not layers:
            return
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            first, end = starts[:-1].to(torch.int64), starts[1:].to(torch.int64)
            new = torch.where((first >= 0) & (end >= first) & (end <= tokens), end - first, 0)
            lost = window_keys_lost([tables[i] for i in layers], [self.windows[i] for i in layers],
                                    [self.views[i].num_blocks for i in layers], seq_lens, new, tokens).any(1)
            lost, twice = torch.stack([lost, blocks_twice([tables[i] for i in layers]).any(1)]).tolist()
        if any(lost):
            raise ValueError("a piece is too long for the ring of layer %d (window %d): its tokens would overwrite keys that its "
                             "first ones see" % (layers[lost.index(True)], self.windows[layers[lost.index(True)]]))
        self._no_rings.update((i, version(i)) for i, t in zip(layers, twice) if not t)

    def capture(self, q, k_new, v_new, out) -> "torch.cuda.CUDAGraph":
        """Records one step (with these argument tensors) into a CUDA graph; replay with ``graph.replay()``."""
        self.step(q, k_new, v_new, out)            # warm-up outside capture (first launches set attributes)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            self.step(q, k_new, v_new, out, stream=torch.cuda.current_stream())
        self.graph = g
        return g
