"""One decode step and one packed prefill through the padoc_attn C ABI, for callers holding torch
tensors. Host work here is the C1 planners (in the library) and host<->device copies of their
integer outputs; every attention step runs in the library's CUDA kernels.
"""
from __future__ import annotations

from typing import List, Optional

import numpy as np
import torch

from . import padoc_attn as pa


class DecodePlan:
    """Decode plan (C1) uploaded to the device, with its split-K workspace (C4)."""

    def __init__(self, pages, num_q_heads: int, num_kv_heads: int, head_dim: int, device, block_size: int = 16,
                 layout_streams: bool = False, split_tokens: int = 0, tc_ctas: int = 0, warp_ctas: int = 0):
        self.cfg = pa.make_decode_config(num_q_heads, num_kv_heads, head_dim, block_size, layout_streams, split_tokens,
                                         tc_ctas, warp_ctas)
        plan, self.info = pa.padoc_build_decode_plan(pages, self.cfg)
        self.plan_host = plan
        self.plan_dev = torch.from_numpy(plan.copy()).to(device)
        ws = pa.padoc_decode_workspace_size(self.info)
        self.workspace = torch.empty(max(ws, 256), dtype=torch.uint8, device=device)

    @property
    def num_streams(self) -> int:
        return self.info.num_streams

    def run(self, k_pool, v_pool, page_table, stream_table, q, scale, out, lse, stream=None):
        pa.padoc_branch_decode_attn(k_pool, v_pool, self.info, self.plan_dev, page_table, stream_table, q, scale,
                                    out, lse, self.workspace, stream)


class PrefillPlan:
    """Spans and tile map (C1) of a packed prefill, uploaded to the device."""

    def __init__(self, pages, dtype: torch.dtype, head_dim: int, device):
        code = pa.PADOC_DTYPE_BF16 if dtype == torch.bfloat16 else pa.PADOC_DTYPE_F32
        self.q_tile, self.k_tile = pa.padoc_prefill_tile_shape(code, head_dim)
        self.spans_host = pa.padoc_build_query_spans(pages)
        self.row_ptr_host, self.k_tiles_host, self.kinds_host = pa.padoc_build_tile_map(pages, self.q_tile, self.k_tile)
        self.T = int(self.spans_host.shape[0])
        self.spans = torch.from_numpy(self.spans_host.copy()).to(device)
        self.row_ptr = torch.from_numpy(self.row_ptr_host.copy()).to(device)
        nnz = max(len(self.k_tiles_host), 1)
        self.k_tiles = torch.zeros(nnz, dtype=torch.int32, device=device)
        self.kinds = torch.zeros(nnz, dtype=torch.int8, device=device)
        if len(self.k_tiles_host):
            self.k_tiles.copy_(torch.from_numpy(self.k_tiles_host.copy()))
            self.kinds.copy_(torch.from_numpy(self.kinds_host.copy()))

    def run(self, q, k, v, scale, out, lse, stream=None):
        pa.padoc_ancestor_prefill_attn(q, k, v, self.spans, self.row_ptr, self.k_tiles, self.kinds, scale, out, lse,
                                       self.q_tile, self.k_tile, stream)


class PrefillBwdPlan:
    """Spans, the query-major and key-major tile maps (C1) and the workspace of a packed prefill's
    backward, on the device."""

    def __init__(self, pages, dtype: torch.dtype, head_dim: int, num_q_heads: int, device):
        code = pa.PADOC_DTYPE_BF16 if dtype == torch.bfloat16 else pa.PADOC_DTYPE_F32
        (qq, qk), (kq, kk) = pa.padoc_prefill_bwd_tile_shapes(code, head_dim)
        spans = pa.padoc_build_query_spans(pages)
        self.T = int(spans.shape[0])
        up = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a if len(a) else np.zeros(1, dt))).to(device)
        self.spans = torch.from_numpy(spans.copy()).to(device)
        row_ptr, k_tiles, kinds = pa.padoc_build_tile_map(pages, qq, qk)
        col_ptr, q_tiles, kkinds, order = pa.padoc_build_key_tile_map(pages, kq, kk)
        self._keep = [up(row_ptr, np.int32), up(k_tiles, np.int32), up(kinds, np.int8),
                      up(col_ptr, np.int32), up(q_tiles, np.int32), up(kkinds, np.int8), up(order, np.int32)]
        self.q_map = pa.make_tile_map_dev(*self._keep[:3], qq, qk)
        self.k_map = pa.make_tile_map_dev(*self._keep[3:6], kq, kk, order=self._keep[6])
        ws = pa.padoc_prefill_bwd_workspace_size(self.T, num_q_heads)
        self.workspace = torch.empty(max(ws, 256), dtype=torch.uint8, device=device)

    def run(self, q, k, v, out, dout, lse, scale, dq, dk, dv, stream=None):
        pa.padoc_ancestor_prefill_bwd(q, k, v, out, dout, lse, self.spans, self.q_map, self.k_map, scale, dq, dk, dv,
                                      self.workspace, stream)


class RotaryPrefill:
    """One attention layer of the packed prefill from the projections on: the head norms and rotary
    positions of ``rotary`` (pa.Rotary), then the ancestor attention; with training also the gradients of
    both. grids: (page, begin, t, h, w) of the image patches among the prefix tokens, whose positions are
    padoc_build_rotary_positions'; with one axis every token has its place in the page's visible sequence."""

    def __init__(self, pages, rotary, num_q_heads: int, num_kv_heads: int, dtype: torch.dtype, device, grids=(),
                 training: bool = False):
        d = rotary.head_dim
        self.rotary = rotary
        self.fwd = PrefillPlan(pages, dtype, d, device)
        self.T = self.fwd.T
        pos, self.prefix_end = pa.padoc_build_rotary_positions(pages, grids)
        if rotary.num_axes > 3 or (rotary.num_axes < 3 and len(grids)):
            raise ValueError("a page's grids need the three axes, a page without them at most three")
        self.pos = torch.from_numpy(np.ascontiguousarray(pos[:, :rotary.num_axes])).to(device)
        new = lambda h, n=None: torch.empty((self.T, h, d), dtype=dtype, device=device)
        self.q, self.k = new(num_q_heads), new(num_kv_heads)   # normed and rotated
        self.bwd = None
        if training:
            self.bwd = PrefillBwdPlan(pages, dtype, d, num_q_heads, device)
            self.workspace = torch.empty(max(pa.padoc_qk_rotary_bwd_workspace_size(rotary, self.T), 256),
                                         dtype=torch.uint8, device=device)

    def _like(self, queries, keys, lse):
        """Refuses tensors that are not [T] rows of the layer's query or key heads, and an lse that is not [T][Hq]."""
        for like, ts in ((self.q, queries), (self.k, keys)):
            if any(t.shape != like.shape or t.dtype is not like.dtype for t in ts):
                raise ValueError("out, dout and dq must be like the layer's q, v, dk and dv like its k")
        if lse.shape != self.q.shape[:2] or lse.dtype is not torch.float32:
            raise ValueError("lse must be float32 [T][Hq]")

    def run(self, q, k, v, scale, out, lse, stream=None):
        """q / k: [T][heads][d] as the projections give them (rows may lie apart); v contiguous."""
        self._like((out,), (v,), lse)
        pa.padoc_qk_rotary(self.rotary, q, k, self.pos, self.q, self.k, stream)
        self.fwd.run(self.q, self.k, v, scale, out, lse, stream)

    def run_bwd(self, q, k, v, out, dout, lse, scale, dq, dk, dv, dq_weight=None, dk_weight=None, stream=None):
        """Gradients of the last run's q, k, v (dq, dk, dv contiguous) and, with norm weights, of these."""
        if self.bwd is None:
            raise ValueError("gradients need training=True")
        # what either step would refuse, before the first writes dq and dk
        self._like((out, dout, dq), (v, dk, dv), lse)
        pa._rotary_bwd_args(self.rotary, dq, dk, self.pos, dq, dk, q, k, dq_weight, dk_weight, self.workspace)
        rows = (q, k) if self.rotary.q_weight is not None else ()
        if any(t.data_ptr() % 16 or (self.T > 1 and t.stride(0) * t.element_size() % 16) for t in rows + (dq, dk)):
            raise ValueError("rows must start on 16-byte boundaries")
        self.bwd.run(self.q, self.k, v, out, dout, lse, scale, dq, dk, dv, stream)
        pa.padoc_qk_rotary_bwd(self.rotary, dq, dk, self.pos, dq, dk, q, k, dq_weight, dk_weight, self.workspace, stream)


class CrossPlan:
    """Cross attention of query rows over an encoder's states: the plan of segments (q_begin, q_len, k_begin, k_len)
    on the device, with its workspaces. Calls that may run at the same time (two streams, two captured graphs) need a
    CrossPlan each. It may be dropped while its calls still run, on whatever streams, but not before the last replay of
    a graph that has captured one."""

    def __init__(self, segments, num_q_heads: int, num_kv_heads: int, head_dim: int, dtype: torch.dtype, device,
                 training: bool = False, ctas: int = 0):
        self.cfg = pa.make_cross_config(num_q_heads, num_kv_heads, head_dim, dtype, training, ctas)
        plan, self.info = pa.padoc_build_cross_plan(segments, self.cfg)
        self.plan_dev = torch.from_numpy(plan.copy() if plan.size else np.zeros(1, np.int32)).to(device)
        new = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device=device)
        self.workspace = new(pa.padoc_cross_workspace_size(self.info))
        self.bwd_workspace = new(pa.padoc_cross_bwd_workspace_size(self.info)) if training else None
        self._streams = set()   # whose work keeps the memory above from being given to others

    def _keep_for(self, raw):
        # (0 and 1 are the default stream's handles)
        stream = torch.cuda.ExternalStream(raw, device=self.plan_dev.device) if raw > 1 else \
            torch.cuda.default_stream(self.plan_dev.device)
        for t in (self.plan_dev, self.workspace, self.bwd_workspace):
            if t is not None:
                t.record_stream(stream)
        self._streams.add(raw)

    def run(self, q, k, v, scale, out, lse, stream=None):
        """q [rows][Hq][d]; k, v [key rows][Hkv][d] (rows may lie apart); out like q, lse fp32 [rows][Hq]. Rows in no
        segment are left as they are."""
        raw = pa._stream_ptr(stream)
        pa.padoc_cross_attn(self.info, self.plan_dev, q, k, v, scale, out, lse, self.workspace, raw)
        if raw not in self._streams:
            self._keep_for(raw)

    def run_bwd(self, q, k, v, out, dout, lse, scale, dq, dk, dv, stream=None):
        """Gradients of run for its out and lse: dq of the segments' rows, dk and dv of every key row."""
        if self.bwd_workspace is None:
            raise ValueError("gradients need training=True")
        raw = pa._stream_ptr(stream)
        pa.padoc_cross_attn_bwd(self.info, self.plan_dev, q, k, v, out, dout, lse, scale, dq, dk, dv, self.bwd_workspace, raw)
        if raw not in self._streams:
            self._keep_for(raw)


class ChunkPrefillPlan:
    """Plan (C1) of a chunked prefill over the paged cache, uploaded: chunks of consecutive query
    tokens per stream (padoc_prefill_chunk rows), run by the decode kernels with the chunks' tokens
    as streams; ``chunk_table`` holds each chunk's private block ids (one row per chunk)."""

    def __init__(self, page_len, chunks, chunk_table, num_q_heads: int, num_kv_heads: int, head_dim: int, device,
                 block_size: int = 16, tc_ctas: int = 0, warp_ctas: int = 0):
        self.cfg = pa.make_decode_config(num_q_heads, num_kv_heads, head_dim, block_size, False, 0, tc_ctas, warp_ctas)
        self.chunks = np.ascontiguousarray(np.asarray(chunks, np.int32).reshape(-1, 4))
        plan, self.info = pa.padoc_build_chunk_prefill_plan(page_len, self.chunks, self.cfg)
        self.plan_dev = torch.from_numpy(plan.copy()).to(device)
        table = pa.padoc_expand_chunk_table(self.chunks, chunk_table,
                                            max(int(self.info.max_stream_blocks), np.asarray(chunk_table).shape[1], 1))
        self.stream_table = torch.from_numpy(table.copy()).to(device)
        ws = pa.padoc_decode_workspace_size(self.info)
        self.workspace = torch.empty(max(ws, 256), dtype=torch.uint8, device=device)

    @property
    def num_tokens(self) -> int:
        return self.info.num_streams

    def run(self, k_pool, v_pool, page_table, q, scale, out, lse, stream=None):
        """q / out: [tokens][Hq][d] in the chunks' token order; lse fp32 [tokens][Hq]."""
        pa.padoc_branch_decode_attn(k_pool, v_pool, self.info, self.plan_dev, page_table, self.stream_table, q, scale,
                                    out, lse, self.workspace, stream)


class MaskedParallelLoop:
    """Algorithm 1 (App. E.1) over the library: the host scheduler (padoc_mpd_*), the append kernel
    and the decode step on one paged KV pool, with device memory from torch.

    Per step the host asks the scheduler for the live streams and their input slots, builds the
    step's decode plan from the stream list, and sends slots, source rows, block tables and plan to
    the device in one copy from pinned memory (two staging buffers, so the host fills one while
    the previous step's copy may still read the other). The device then appends every input's K/V
    into the pool, lays out the queries and decodes every stream, all on one CUDA stream. With rotary
    (pa.Rotary) the inputs are appended normed and rotated, at positions given by source row.

    Between steps a branch can be forked with its history (fork_stream), streams and pages dropped, and the
    pool compacted or replaced by one of another size (compact, resize).

    With an encoder a page is admitted with the rows of its image's states (states); its branches have them too, or a
    range of their own (set_states: a region's crop), and cross_step is the step's cross attention over them.

    Memory that a call needs more of is allocated on that call's stream. Calls on different streams are ordered by
    the caller, the first one behind the stream that was current when the loop was made (its pool is zeroed there)."""

    def __init__(self, num_blocks: int, num_q_heads: int, num_kv_heads: int, head_dim: int, dtype: torch.dtype,
                 device, block_order=None, block_size: int = 16, tc_ctas: int = 0, warp_ctas: int = 0,
                 split_tokens: int = 0, rotary=None):
        self.mpd = pa.Mpd(num_blocks, block_size, block_order)
        self.k_pool = torch.zeros((num_blocks, num_kv_heads, block_size, head_dim), dtype=dtype, device=device)
        self.v_pool = torch.zeros_like(self.k_pool)
        self._pool = pa.make_kv_pool(self.k_pool, self.v_pool)
        self.cfg = pa.make_decode_config(num_q_heads, num_kv_heads, head_dim, block_size, False, split_tokens,
                                         tc_ctas, warp_ctas)
        self.device, self.dtype = device, dtype
        if rotary is not None and rotary.table.device != self.k_pool.device:
            raise ValueError("the rotary must be on the pool's device")
        self.rotary = rotary
        self.num_q_heads, self.head_dim = num_q_heads, head_dim
        self._stage = [None, None]
        self._stage_free = [torch.cuda.Event(), torch.cuda.Event()]
        self._turn = 0
        self._ints = torch.empty(1024, dtype=torch.int32, device=device)
        self.workspace = torch.empty(256, dtype=torch.uint8, device=device)
        self.q_step = torch.empty((64, num_q_heads, head_dim), dtype=dtype, device=device)
        self.last_info = None
        self.last_step = None
        self.last_stage = None
        self.h2d_bytes = 0                          # copied to the device by the last step, admission or move ...
        self.cross_h2d_bytes = 0                    # ... and, for its plan, by the last cross_step
        self._runner = None
        self._states = np.zeros((0, 2), np.int32)   # each stream's key rows (first, number), by stream id
        self._step_ids = None
        self._cross_ints = torch.empty(1024, dtype=torch.int32, device=device)
        self._cross_workspace = torch.empty(256, dtype=torch.uint8, device=device)
        self._cross_plan = None                     # (segments, config) and summary of the plan in _cross_ints

    def _grow(self, name, rows, stream):
        """Makes the array ``name`` at least rows long for use on ``stream``, where the old one may still be in use."""
        old = getattr(self, name)
        if old.shape[0] < rows:
            old.record_stream(stream)
            with torch.cuda.stream(stream):
                new = torch.empty((max(rows, 2 * old.shape[0]),) + tuple(old.shape[1:]), dtype=old.dtype, device=self.device)
            setattr(self, name, new)

    def _room(self, sizes, stream, to="_ints"):
        """Room for an upload of arrays of these sizes on ``stream``; returns their places and the words."""
        offs, n = [], 0
        for size in sizes:
            offs.append(n)
            n += (int(size) + 31) // 32 * 32
        b = self._turn & 1
        if self._stage[b] is None or self._stage[b].numel() < n:
            self._stage_free[b].synchronize()
            self._stage[b] = torch.empty(max(n, 2 * (0 if self._stage[b] is None else self._stage[b].numel()), 4096),
                                         dtype=torch.int32).pin_memory()
        self._grow(to, n, stream)
        return offs, n

    def _upload(self, parts, stream, to="_ints", count="h2d_bytes"):
        """Copies int32 host arrays to the device (into the array ``to``) in one transfer, each starting on a
        128-byte boundary, and notes its bytes in ``count``; returns device views."""
        offs, n = self._room([a.size for a in parts], stream, to)
        b = self._turn & 1
        self._turn += 1
        self._stage_free[b].synchronize()
        host = self._stage[b].numpy()
        for a, o in zip(parts, offs):
            host[o:o + a.size] = a.reshape(-1)
        dev = getattr(self, to)
        with torch.cuda.stream(stream):
            dev[:n].copy_(self._stage[b][:n], non_blocking=True)
        self._stage_free[b].record(stream)
        setattr(self, count, 4 * n)
        return [dev[o:o + a.size] for a, o in zip(parts, offs)]

    def _check_rows(self, k_src, q_src, v_src, pos_src):
        """Refuses source rows that the append with rotary would refuse (by an append of none of them)."""
        if k_src.shape[0] < 1:
            raise ValueError("sources must have a row")
        pa.padoc_append_rotary_inputs(self.rotary, self.k_pool, self.v_pool, k_src, v_src, pos_src, self._ints,
                                      q_src=q_src, q_dst=self.q_step, count=0)

    def add_page(self, prefix_len: int, num_forks: int, layout_eos: bool, k_src, v_src, src_rows, stream=None,
                 pos_src=None, states=(0, 0)):
        """Admits a page: its prefix K/V (rows src_rows of k_src / v_src, device tensors [rows][Hkv][d])
        go into the blocks the scheduler gives it. pos_src: int32 [rows][axes], with rotary. states: (first, number)
        of the encoder's rows that the page's streams see in cross_step. Returns (page id, new stream ids)."""
        stream = stream or torch.cuda.current_stream()
        states = self._range(*states)
        if self.rotary is not None and prefix_len > 0:   # before the scheduler admits the page
            self._check_rows(k_src, None, v_src, pos_src)
            if len(src_rows) != prefix_len:
                raise ValueError("src_rows must name a row for each prefix token")
        if prefix_len > 0:
            rows = np.asarray(src_rows, np.int32)
            if prefix_len <= self.status()[2] * self.cfg.block_size:   # (a page that does not fit is refused below)
                self._room((prefix_len, rows.size), stream)
        pid, slots, new = self.mpd.add_page(prefix_len, num_forks, layout_eos)
        if prefix_len > 0:
            slots_d, rows_d = self._upload([slots, rows], stream)
            if self.rotary is not None:
                pa.padoc_append_rotary_inputs(self.rotary, self.k_pool, self.v_pool, k_src, v_src, pos_src, slots_d,
                                              src_rows=rows_d, count=prefix_len, stream=stream)
            else:
                pa.padoc_append_inputs(self.k_pool, self.v_pool, k_src, v_src, slots_d, src_rows=rows_d, count=prefix_len,
                                       stream=stream)
        self._give_states(new, states)
        return pid, new

    @staticmethod
    def _range(first, number):
        if first < 0 or number < 0 or first + number > 2 ** 31 - 1024:
            raise ValueError("states: a range of rows")
        return int(first), int(number)

    def _give_states(self, ids, states):
        ids = [i for i in ids if i >= 0]
        if len(ids) == 0 or (states[1] == 0 and len(self._states) == 0):   # (none so far: all are empty)
            return
        if max(ids) >= len(self._states):
            more = np.zeros((max(max(ids) + 1, 2 * len(self._states), 64), 2), np.int32)
            more[:len(self._states)] = self._states
            self._states = more
        self._states[ids] = states

    def set_states(self, stream_id: int, first: int, number: int):
        """The encoder's rows that a live stream sees in cross_step from now on (and branches forked from it)."""
        if stream_id < 0:
            raise ValueError("no such stream")
        states = self._range(first, number)
        if stream_id >= len(self._states):
            self._give_states([stream_id], (0, 1))   # (room, also for an empty range)
        self._states[stream_id] = states

    def states_of(self, stream_id: int):
        """(first, number) of the encoder's rows that the stream sees."""
        return tuple(int(x) for x in self._states[stream_id]) if 0 <= stream_id < len(self._states) else (0, 0)

    def cross_step(self, ids, q, k, v, scale: float, out=None, lse=None, stream=None):
        """Cross attention of a step's tokens: row i of q [C][Hq][d] is stream ids[i]'s (in the step's order), k and v
        [rows][Hkv][d] are the encoder's (rows may lie apart). Streams that follow one another and see the same rows
        read them together. Returns (out [C][Hq][d], lse fp32 [C][Hq]). The plan is built and copied anew only when the
        streams or their states have changed. It lies in the loop's own memory, where a later call puts another, so a
        call on a stream that is being captured is refused: capture a CrossPlan over the streams' segments instead."""
        if stream is None:
            stream, capturing = torch.cuda.current_stream(), torch.cuda.is_current_stream_capturing()
        else:
            with torch.cuda.stream(stream):
                capturing = torch.cuda.is_current_stream_capturing()
        if capturing:
            raise ValueError("cross_step cannot be captured: capture a CrossPlan over the streams' segments")
        ids = np.asarray(ids, np.int64)
        if q.shape[0] != ids.size or (ids.size and ids.min() < 0):
            raise ValueError("q needs a row for each stream")
        if out is None or lse is None:
            with torch.cuda.stream(stream):
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
                lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device) if lse is None else lse
        self.cross_h2d_bytes = 0
        if ids.size == 0:
            return out, lse
        if ids.max() >= len(self._states):
            self._give_states([int(ids.max())], (0, 1))
            self._states[int(ids.max())] = 0
        mine = self._states[ids]
        first = np.flatnonzero(np.concatenate(([True], (mine[1:] != mine[:-1]).any(1))))
        segments = np.empty((first.size, 4), np.int32)
        segments[:, 0] = first
        segments[:, 1] = np.diff(np.append(first, ids.size))
        segments[:, 2:] = mine[first]
        key = (segments.tobytes(), q.shape[1], k.shape[1], q.shape[2], q.dtype)
        if self._cross_plan is None or self._cross_plan[0] != key:
            cfg = pa.make_cross_config(q.shape[1], k.shape[1], q.shape[2], q.dtype)
            plan, info = pa.padoc_build_cross_plan(segments, cfg)
            self._cross_plan = None
            self._upload([plan], stream, "_cross_ints", "cross_h2d_bytes")
            self._cross_plan = (key, info)
        info = self._cross_plan[1]
        self._grow("_cross_workspace", pa.padoc_cross_workspace_size(info), stream)
        pa.padoc_cross_attn(info, self._cross_ints, q, k, v, scale, out, lse, self._cross_workspace, stream)
        return out, lse

    def step(self, k_src, v_src, q_src, rows_of, scale: float, out=None, lse=None, stream=None, pos_src=None):
        """One iteration: every live stream appends its next input (rows_of(stream ids) gives the rows
        of k_src / v_src / q_src, and with rotary of pos_src, that hold them) and is decoded. Returns (stream ids, out [C][Hq][d],
        lse fp32 [C][Hq]); the caller ends the step with end_step. The host work is two library calls:
        padoc_mpd_prepare_step into a pinned staging buffer, and padoc_mpd_launch_step, which copies it
        to the device and launches the append and the decode."""
        stream = stream or torch.cuda.current_stream()
        if self.rotary is not None and self.status()[1]:   # before the scheduler begins the step
            if q_src is None:
                raise ValueError("a step needs q_src")
            self._check_rows(k_src, q_src, v_src, pos_src)
        b = self._turn & 1
        self._turn += 1
        self._stage_free[b].synchronize()
        if self._stage[b] is None:
            self._stage[b] = torch.empty(1 << 16, dtype=torch.int32).pin_memory()
        while True:
            try:
                st = self.mpd.prepare_step(self.cfg, self._stage[b].numpy())
                break
            except pa.PadocError as e:
                need = getattr(e, "step", None)
                if e.status != 6 or need is None or need.total_words <= self._stage[b].numel():
                    raise
                self._stage[b] = torch.empty(2 * int(need.total_words), dtype=torch.int32).pin_memory()
        host = self._stage[b].numpy()
        C = int(st.num_streams)
        self._step_ids = ids = host[st.off_stream_ids:st.off_stream_ids + C].copy()
        host[st.off_rows:st.off_rows + C] = rows_of(ids)
        n = int(st.upload_words)
        self._grow("_ints", n, stream)
        self.h2d_bytes = 4 * n
        info = st.plan
        self.last_info = info
        self.last_step = st
        self.last_stage = host
        if C == 0:
            self._stage_free[b].record(stream)
            empty = torch.empty((0, self.num_q_heads), dtype=torch.float32, device=self.device)
            return ids, torch.empty((0, self.num_q_heads, self.head_dim), dtype=self.dtype, device=self.device), empty
        self._grow("q_step", C, stream)
        self._grow("workspace", pa.padoc_decode_workspace_size(info), stream)
        if out is None or lse is None:
            with torch.cuda.stream(stream):
                if out is None:
                    out = torch.empty((C, self.num_q_heads, self.head_dim), dtype=self.dtype, device=self.device)
                if lse is None:
                    lse = torch.empty((C, self.num_q_heads), dtype=torch.float32, device=self.device)
        # one library call: the stage's copy to the device, the append and the decode
        if self.rotary is not None:
            pa.padoc_mpd_launch_step_rotary(st, self._stage[b], self._ints, self._pool, self.rotary, k_src, v_src, q_src,
                                            pos_src, self.q_step, scale, out, lse, self.workspace, stream)
        else:
            pa.padoc_mpd_launch_step(st, self._stage[b], self._ints, self._pool, k_src, v_src, q_src, self.q_step, scale,
                                     out, lse, self.workspace, stream)
        self._stage_free[b].record(stream)
        return ids, out, lse

    def run_step(self, k_src, v_src, q_src, row_of_stream, scale: float, out, lse, stream=None, pos_src=None):
        """step() as one library call (padoc_mpd_runner_step): row_of_stream is an int32 numpy table
        of each live stream's source row indexed by stream id; out [rows][Hq][d] and lse [rows][Hq]
        (rows at least the live streams) receive the outputs in step order. Returns (C, stream ids
        int32 [C], valid until the next step); end the step with end_step. With rotary, pos_src as in step."""
        if self._runner is None:
            self._runner = pa.MpdRunner(self.mpd, self.cfg, self._pool)
        if self.rotary is not None and not self._runner.rotates(self.rotary, pos_src) and self.status()[1]:
            self._runner.set_rotary(self.rotary, pos_src)
        try:
            n, ids = self._runner.step(k_src, v_src, q_src, row_of_stream, scale, out, lse, stream)
        except pa.PadocError as e:
            if e.status in (2, 4):   # past the planning: the step has begun, with the streams that the runner noted
                self._step_ids = self._runner._ids
            raise
        self.h2d_bytes = self._runner.upload_bytes
        self._step_ids = ids
        return n, ids

    def last_run_step(self):
        """(padoc_mpd_step, its staging words) of the last run_step."""
        return self._runner.last_step()

    def end_step(self, num_forks=None, eos=None, num_streams=None):
        """Each stream's output event (forks, EOS) in step order; returns the new branches' ids."""
        new = self.mpd.end_step(num_forks, eos, num_streams)
        if len(new) and len(self._states) and self._step_ids is not None:   # branches see what their stream sees
            forks = np.asarray(num_forks)           # (one number for all streams, or one each)
            ids = self._step_ids[:num_streams if forks.ndim == 0 else len(forks)]
            for parent, child in zip(np.repeat(ids, forks), new):
                self._give_states([int(child)], self.states_of(int(parent)))
        return new

    def _before_copies(self, pairs, stream):
        """Refuses what a copy of up to ``pairs`` blocks within the pool would refuse, and makes its room: the
        scheduler changes only after this."""
        if pairs == 0:
            return
        own = pa.KvPools([(self.k_pool, self.v_pool)])
        pa.padoc_copy_kv_blocks(own, self._ints, self._ints, own, 0, stream)
        self._room((pairs, pairs), stream)

    def _copy_blocks(self, src, dst, stream, pool=None):
        """Blocks src to dst of the pool (or of ``pool``, (k_pool, v_pool))."""
        if len(src):
            src_d, dst_d = self._upload([np.asarray(src, np.int32), np.asarray(dst, np.int32)], stream)
            own = pa.KvPools([(self.k_pool, self.v_pool)])
            pa.padoc_copy_kv_blocks(own if pool is None else pa.KvPools([pool]), src_d, dst_d, own, len(src), stream)

    def fork_stream(self, stream_id: int, num_copies: int = 1, stream=None):
        """Forks a live branch into num_copies more with the same history, between steps: they share its
        complete blocks and get copies of the partly filled one. Returns the new stream ids."""
        stream = stream or torch.cuda.current_stream()
        self._before_copies(max(0, min(num_copies, self.status()[2])), stream)   # (a copy takes a free block)
        new, src, dst = self.mpd.fork_stream(stream_id, num_copies)
        self._copy_blocks(src, dst, stream)
        self._give_states([int(i) for i in new], self.states_of(int(stream_id)))
        return new

    def drop_stream(self, stream_id: int):
        """Retires a live stream between steps."""
        self.mpd.drop_stream(stream_id)

    def drop_page(self, page_id: int):
        """Retires every stream of a live page between steps."""
        self.mpd.drop_page(page_id)

    def compact(self, stream=None) -> int:
        """Moves the live blocks to the pool's lowest ids, between steps. Returns their number."""
        stream = stream or torch.cuda.current_stream()
        free = self.status()[2]
        self._before_copies(min(free, self.k_pool.shape[0] - free), stream)      # (a move takes a live block to a free one)
        src, dst = self.mpd.compact()
        self._copy_blocks(src, dst, stream)
        return self.k_pool.shape[0] - free

    def resize(self, num_blocks: int, stream=None):
        """Replaces the pool by one of num_blocks blocks (at least the live ones), between steps."""
        stream = stream or torch.cuda.current_stream()
        if num_blocks < self.k_pool.shape[0] - self.status()[2]:
            raise pa.PadocError("padoc_mpd_resize", 6)
        live = self.compact(stream)
        shape = (num_blocks,) + tuple(self.k_pool.shape[1:])
        with torch.cuda.stream(stream):
            k_pool = torch.zeros(shape, dtype=self.dtype, device=self.device)
            v_pool = torch.zeros(shape, dtype=self.dtype, device=self.device)
        ids = np.arange(live, dtype=np.int32)
        self._copy_blocks(ids, ids, stream, (k_pool, v_pool))
        self.mpd.resize(num_blocks)
        if self._runner is not None:
            self._runner.close()
            self._runner = None
        for t in (self.k_pool, self.v_pool):
            t.record_stream(stream)
        self.k_pool, self.v_pool = k_pool, v_pool
        self._pool = pa.make_kv_pool(self.k_pool, self.v_pool)

    def status(self):
        return self.mpd.status()


def shard_pages(num_pages: int, rank: int, world: int) -> List[int]:
    """Pages of one rank when pages are split across ranks (pages never see each other, so a
    rank's pages need nothing from any other rank): contiguous, sizes differing by at most one."""
    if world < 1 or not (0 <= rank < world):
        raise ValueError("bad rank/world")
    base, extra = divmod(num_pages, world)
    lo = rank * base + min(rank, extra)
    return list(range(lo, lo + base + (1 if rank < extra else 0)))
