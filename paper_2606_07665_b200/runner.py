"""Device-side staging of a workload and the launch sequence of one decode step.

Only plumbing: torch tensors for device memory, the split plan from the library, and the three
C-ABI calls in order.  Every arithmetic step runs inside libac's kernels.

``DecodeStep`` stages a synthetic workload; ``PagedAttention`` (bf16 cache), ``Q4Cache`` with ``Q4DecodeStep``
(4-bit cache) and ``CachePages`` (reserve, fork, release, trim, compact, copy) work on tensors that the caller owns.
"""
from __future__ import annotations

import ctypes

import numpy as np
import torch

from . import binding as ac


def _dev_u16(a: np.ndarray, device) -> torch.Tensor:
    """uint16 bf16 bit patterns -> device int16 tensor (same bits)."""
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to(device)


def bits_of(t: torch.Tensor) -> np.ndarray:
    """Device int16 tensor -> host uint16 bit patterns."""
    return t.detach().cpu().numpy().view(np.uint16)


class DecodeStep:
    """Holds one workload on the device and enqueues RoPE+append -> attention -> merge.

    ``layout`` is "token_major" ([page, slot, head, d], the default) or "head_major"
    ([page, head, slot, d]); the kernels see only the strides.
    """

    def __init__(self, w, device="cuda:0", num_splits: int | None = None, layout: str = "token_major",
                 max_context_len: int | None = None, fused_merge: bool = True,
                 fused_step: bool = False, window: int = 0, row_order="auto", rope_variants=None,
                 sinks: int = 0):
        self.w = w
        # prelude variants the single-launch step applies (rotary_dim, interleaved, q_norm_weight,
        # k_norm_weight, norm_eps); None = the plain rotation
        if isinstance(rope_variants, str) and rope_variants == "workload":
            # the options the workload itself names, norm weights moved to the device
            self.rope_variants = {
                k: (torch.from_numpy(np.ascontiguousarray(v).view(np.int16)).to(device) if isinstance(v, np.ndarray) else v)
                for k, v in w.extra.get("rope_variants", {}).items()}
        else:
            self.rope_variants = dict(rope_variants) if rope_variants else {}
        self.window = int(window) if window else int(getattr(w, "window", 0))   # > 0: sliding window
        self.sinks = int(sinks)                        # first tokens that stay visible beside the window
        self.fused_step = bool(fused_step)             # one launch: RoPE + append + attention + merge
        self.fused_merge = bool(fused_merge) or self.fused_step
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        ac.ac_init(self.device.index if self.device.index is not None else -1)
        self.B, self.Hq, self.Hkv, self.d, self.ps = w.B, w.Hq, w.Hkv, w.d, w.page_size
        self.num_pages = w.num_pages
        self.layout = layout
        kc, vc = w.k_cache, w.v_cache
        if layout == "head_major":
            kc = np.ascontiguousarray(kc.transpose(0, 2, 1, 3))
            vc = np.ascontiguousarray(vc.transpose(0, 2, 1, 3))
            self.stride_page = self.Hkv * self.ps * self.d
            self.stride_head = self.ps * self.d
            self.stride_token = self.d
        elif layout == "token_major":
            self.stride_page = self.ps * self.Hkv * self.d
            self.stride_token = self.Hkv * self.d
            self.stride_head = self.d
        else:
            raise ValueError(layout)
        self.k_cache = _dev_u16(kc, self.device)
        self.v_cache = _dev_u16(vc, self.device)
        self.q_in = _dev_u16(w.q, self.device)
        self.q_rot = self.q_in.clone()          # rows the kernel skips (inactive) keep their input
        self.k_new = _dev_u16(w.k_new, self.device)
        self.v_new = _dev_u16(w.v_new, self.device)
        self.block_table = torch.from_numpy(w.block_table).to(self.device)
        self.context_lens = torch.from_numpy(w.context_lens).to(self.device)
        self.rope_cos = torch.from_numpy(w.rope_cos).to(self.device)
        self.rope_sin = torch.from_numpy(w.rope_sin).to(self.device)
        # Scheduling hint: requests by decreasing length (what a scheduler that knows the lengths
        # hands over with the block table).  "auto": wherever the grid is more than one wave deep -- the
        # kernel would otherwise rank the requests itself in every CTA (up to 128 rows, ~1 us) or keep
        # index order (more rows); decided in set_splits, once the grid is known.
        self._row_order_auto = isinstance(row_order, str) and row_order == "auto"
        if self._row_order_auto:
            row_order = None
        self.row_order = None if row_order is None else torch.from_numpy(np.asarray(row_order, np.int32)).to(self.device)
        self.out = torch.zeros((self.B, self.Hq, self.d), dtype=torch.int16, device=self.device)
        self.status_flag = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.max_context_len = int(max_context_len) if max_context_len else w.max_context_len
        self.set_splits(num_splits)

    def set_splits(self, num_splits: int | None) -> None:
        span = self.max_context_len
        if self.window > 0:
            span = min(span, ac.ac_window_span(self.window, self.sinks))   # tokens of a row, as the kernel counts
        if num_splits is None:
            # the lengths are on the host (the scheduler built context_lens from them): plan with them
            counts = [min(int(n) + 1, span) if n >= 0 else 0 for n in self.w.context_lens]
            num_splits, _, _ = ac.ac_decode_plan_for_lengths(counts, self.Hq, self.Hkv, self.d, self.ps,
                                                             span, ac.ac_sm_count())
        self.num_splits = int(num_splits)
        self.split_tokens = ac.ac_split_tokens(span, self.num_splits)
        if self._row_order_auto:
            deep = self.B > 1 and self.B * self.Hkv * self.num_splits > 2 * (ac.ac_sm_count() or 148)
            order = np.argsort(-self.w.context_lens.astype(np.int64), kind="stable").astype(np.int32)
            self.row_order = torch.from_numpy(order).to(self.device) if deep else None
        # sized for either merge flavour: partials, then the fused path's arrival counters
        self.workspace_bytes = ac.ac_fused_workspace_bytes(self.B, self.Hq, self.Hkv, self.d,
                                                           self.num_splits)
        self.workspace = (torch.empty(max(self.workspace_bytes, 16) // 4, dtype=torch.float32,
                                      device=self.device))
        ac.ac_fused_workspace_reset(self.workspace, self.workspace_bytes, self.B, self.Hq, self.Hkv,
                                    self.d, self.num_splits)

    # -- the three calls -----------------------------------------------------------------------
    def rope_kv_append_ex(self, stream=None, rotary_dim=0, interleaved=False, q_norm_weight=None,
                          k_norm_weight=None, norm_eps=0.0) -> None:
        """Prelude variants; norm weights are device int16 tensors holding bf16 bits."""
        ac.ac_rope_kv_append_ex(self.q_in, self.q_rot, self.k_new, self.v_new, self.k_cache, self.v_cache,
                                self.stride_page, self.stride_token, self.stride_head, self.block_table,
                                self.w.max_pages_per_seq, self.context_lens, self.rope_cos, self.rope_sin,
                                self.w.max_position, self.B, self.Hq, self.Hkv, self.d, self.ps,
                                self.num_pages, self.status_flag, stream, rotary_dim=rotary_dim,
                                interleaved=interleaved, q_norm_weight=q_norm_weight,
                                k_norm_weight=k_norm_weight, norm_eps=norm_eps)

    def rope_kv_append(self, stream=None) -> None:
        ac.ac_rope_kv_append(self.q_in, self.q_rot, self.k_new, self.v_new, self.k_cache, self.v_cache,
                             self.stride_page, self.stride_token, self.stride_head, self.block_table,
                             self.w.max_pages_per_seq, self.context_lens, self.rope_cos, self.rope_sin,
                             self.w.max_position, self.B, self.Hq, self.Hkv, self.d, self.ps,
                             self.num_pages, self.status_flag, stream)

    def attention(self, stream=None, new_tokens: int = 1, q=None) -> None:
        if self.window > 0 or self.row_order is not None:
            ac.ac_paged_decode_attn_ex(self.q_rot if q is None else q, self.k_cache, self.v_cache,
                                       self.stride_page, self.stride_token, self.stride_head,
                                       self.block_table, self.w.max_pages_per_seq, self.context_lens,
                                       new_tokens, 0.0, self.num_splits,
                                       self.workspace if self.num_splits > 1 else None,
                                       self.workspace_bytes, self.out, self.B, self.Hq, self.Hkv, self.d,
                                       self.ps, self.num_pages, self.max_context_len, self.status_flag,
                                       stream, window=self.window, fused_merge=self.fused_merge,
                                       row_order=self.row_order, sinks=self.sinks)
            return
        fn = ac.ac_paged_decode_attn_fused_merge if self.fused_merge else ac.ac_paged_decode_attn
        fn(self.q_rot if q is None else q, self.k_cache, self.v_cache,
                                self.stride_page, self.stride_token, self.stride_head, self.block_table,
                                self.w.max_pages_per_seq, self.context_lens, new_tokens, 0.0,
                                self.num_splits, self.workspace if self.num_splits > 1 else None,
                                self.workspace_bytes, self.out, self.B, self.Hq, self.Hkv, self.d,
                                self.ps, self.num_pages, self.max_context_len, self.status_flag, stream)

    def merge(self, stream=None) -> None:
        if self.num_splits > 1 and not self.fused_merge:
            ac.ac_splitkv_merge(self.workspace, self.num_splits, self.context_lens, self.out, self.B,
                                self.Hq, self.d, stream)

    def decode_step_fused(self, stream=None, **rope_variants) -> None:
        """rope_variants: rotary_dim, interleaved, q_norm_weight, k_norm_weight, norm_eps (prelude
        variants applied inside the step; norm weights are device int16 tensors holding bf16 bits)."""
        ac.ac_decode_step_fused_ex(self.q_in, self.q_rot, self.k_new, self.v_new, self.k_cache,
                                   self.v_cache, self.stride_page, self.stride_token, self.stride_head,
                                   self.block_table, self.w.max_pages_per_seq, self.context_lens,
                                   self.rope_cos, self.rope_sin, self.w.max_position, 0.0, self.num_splits,
                                   self.workspace if self.num_splits > 1 else None, self.workspace_bytes,
                                   self.out, self.B, self.Hq, self.Hkv, self.d, self.ps, self.num_pages,
                                   self.max_context_len, self.status_flag, stream, window=self.window,
                                   row_order=self.row_order, sinks=self.sinks,
                                   **{**self.rope_variants, **rope_variants})

    def step(self, stream=None) -> None:
        if self.fused_step:
            self.decode_step_fused(stream)
            return
        self.rope_kv_append(stream)
        self.attention(stream)
        self.merge(stream)

    @property
    def launches_per_step(self) -> int:
        if self.fused_step:
            return 1
        return 3 if (self.num_splits > 1 and not self.fused_merge) else 2

    def capture(self) -> torch.cuda.CUDAGraph:
        """Record one step into a CUDA graph (one graph per batch-size bucket in a serving loop)."""
        side = torch.cuda.Stream(device=self.device)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.step(side)                      # warm-up outside capture
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            self.step(side)
        return graph

    # -- results -------------------------------------------------------------------------------
    def cache_bits(self):
        k, v = bits_of(self.k_cache), bits_of(self.v_cache)
        if self.layout == "head_major":
            k = k.reshape(self.num_pages, self.Hkv, self.ps, self.d).transpose(0, 2, 1, 3)
            v = v.reshape(self.num_pages, self.Hkv, self.ps, self.d).transpose(0, 2, 1, 3)
        return k, v

    def out_f64(self) -> np.ndarray:
        b = bits_of(self.out)
        return (b.astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)

    def partials(self):
        n = self.B * self.Hq * self.num_splits
        ws = self.workspace.detach().cpu().numpy()
        po = ws[:n * self.d].reshape(self.B, self.Hq, self.num_splits, self.d)
        pl = ws[n * self.d:n * self.d + n].reshape(self.B, self.Hq, self.num_splits)
        return po, pl


class AttentionBlockStep:
    """The attention block of one decoder layer for one decode step, as three launches in a row:
    QKV projection + RoPE + KV append, paged decode attention with the merge fused in, output
    projection + residual + RMSNorm.  ``hidden`` [B,H], ``w_qkv`` [(Hq+2Hkv)*d, H], ``w_o`` [H, Hq*d],
    ``norm_weight`` [H] are uint16 arrays of bf16 bits; ``hidden`` is both the projection's input and
    the residual stream."""

    def __init__(self, w, hidden, w_qkv, w_o, norm_weight, norm_eps=1e-5, device="cuda:0",
                 num_splits: int | None = None):
        self.step_ = DecodeStep(w, device=device, num_splits=num_splits, fused_merge=True)
        st = self.step_
        self.H = int(hidden.shape[1])
        self.norm_eps = float(norm_eps)
        self.hidden = _dev_u16(hidden, st.device)
        self.w_qkv = _dev_u16(w_qkv, st.device)
        self.w_o = _dev_u16(w_o, st.device)
        self.norm_weight = _dev_u16(norm_weight, st.device)
        self.residual_out = torch.empty_like(self.hidden)
        self.normed_out = torch.empty_like(self.hidden)

    def step(self, stream=None) -> None:
        st = self.step_
        ac.ac_qkv_rope_kv_append(self.hidden, self.w_qkv, self.H, st.q_rot, st.k_cache, st.v_cache,
                                 st.stride_page, st.stride_token, st.stride_head, st.block_table,
                                 st.w.max_pages_per_seq, st.context_lens, st.rope_cos, st.rope_sin,
                                 st.w.max_position, st.B, st.Hq, st.Hkv, st.d, st.ps, st.num_pages,
                                 st.status_flag, stream)
        st.attention(stream)
        ac.ac_oproj_residual_rmsnorm(st.out, self.w_o, st.Hq * st.d, self.H, self.hidden,
                                     self.residual_out, self.norm_weight, self.norm_eps, self.normed_out,
                                     st.B, stream)


# ---- objects over the caller's tensors -----------------------------------------------------------------------
#
# They validate once what stays (pools, tables, lengths) and per call what changes, keep the plan, the workspace
# and the marshalled arguments, and enqueue on the current stream of their device (or on the one given).
#
# What an object allocates for itself stays allocated until every stream that it was used on is done with it, and for as
# long as the object lives where a captured call uses it.  So plan() and the end of an object need no synchronisation;
# only a captured graph must not be replayed beyond the objects that it calls, and a stream given as a handle must
# outlive them.

_BF16 = (torch.bfloat16, torch.int16)          # bf16 values, or their bits


def _want(t, name, shape, dtypes, device):
    """t is a contiguous tensor of this shape (a torch.Size), type and device; raises ValueError otherwise (TypeError for
    what is no tensor)."""
    try:
        if t.shape == shape and t.dtype in dtypes and t.is_contiguous() and t.device == device:
            return
    except AttributeError:
        pass
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: {type(t).__name__}, expected a tensor")
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: type {t.dtype}, expected {' or '.join(map(str, dtypes))}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{name}: on {t.device}, expected {device}")
    raise ValueError(f"{name}: not contiguous")


def _axes(layout):
    """(slot axis, head axis) of a pool [num_pages, ., ., .]."""
    if layout not in ("token_major", "head_major"):
        raise ValueError(f"layout {layout!r}, expected 'token_major' or 'head_major'")
    return (1, 2) if layout == "token_major" else (2, 1)


def _new_tokens(n):
    """1: attention over context_lens[b] + 1 tokens, the one just appended among them; 0: over the cached ones alone."""
    if n not in (0, 1):
        raise ValueError(f"new_tokens {n}, expected 0 or 1")
    return int(n)


class _OnDevice:
    """A device, ac_init on it, its streams, and what belongs to the calls on them."""

    def _bind(self, device):
        if device.type != "cuda":
            raise ValueError(f"tensors on {device}, expected a CUDA device")
        self.device, self._index, self._lib = device, device.index, ac.lib()
        self._streams = set()
        self._captured = True                              # nobody asks, unless the buffers can be replaced
        with torch.cuda.device(device):
            ac.ac_init(device.index)
            self.status_flag = torch.zeros(1, dtype=torch.int32, device=device)
            torch.cuda.current_stream().synchronize()      # zeroed whatever stream the calls run on
        self._flag = self.status_flag.data_ptr()

    def _buffers(self):
        """The tensors that calls use and nobody else holds."""
        return [self.status_flag]

    def _used_on(self, stream):
        """The buffers are in use on this stream (a handle) from now on; their memory must not go to anything else before
        that stream is past the call (the allocator looks at this when it gets them back)."""
        self._streams.add(stream)
        used = torch.cuda.ExternalStream(stream, device=self.device)
        for t in self._buffers():
            t.record_stream(used)

    def _new(self, shape, stream, dtype=torch.bfloat16):
        """A tensor that belongs to the stream that will write it, so that its memory is not handed to another one's work
        while that stream still uses it."""
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=self.device) if isinstance(stream, int) else stream):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def _enqueue(self, name, args, stream, at):
        """Calls the library with the device current; args are marshalled but for the stream, which goes in at `at`."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self._enqueue(name, args, stream, at)
        if stream is None:
            stream = _raw_stream(self._index)
            self._captured = self._captured or _current_is_captured()
        else:
            if not isinstance(stream, int):
                stream = stream.cuda_stream
            self._captured = self._captured or _is_captured(stream)
        args[at] = stream
        if stream not in self._streams:
            self._used_on(stream)
        status = getattr(self._lib, name)(*args)
        if status != 0:
            raise ac.AcError(status, name)


# the current device and stream without the wrappers (a microsecond per call)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
_current_is_captured = getattr(torch._C, "_cuda_isCurrentStreamCapturing", None) or torch.cuda.is_current_stream_capturing


def _is_captured(stream, _driver=[]):
    """Whether this stream (a handle) is being captured into a graph.  Asked of the driver: making the stream the current one to
    ask torch costs as much as the call that follows."""
    if not _driver:
        _driver.append(ctypes.CDLL("libcuda.so.1").cuStreamIsCapturing)
        _driver[0].argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int)]
    status = ctypes.c_int(0)
    return _driver[0](stream, status) == 0 and status.value != 0


class _Rows(_OnDevice):
    """A block table and context lengths, and the split plan of attention over them."""

    workspace = row_order = None
    _kept = ()

    def _replace_buffers(self):
        """Before plan() replaces the buffers: captured calls go on using the present ones."""
        if self._captured and self.workspace is not None:
            self._kept += (self._buffers(),)
        self._streams, self._captured = set(), False

    def _buffers(self):
        return [t for t in (self.status_flag, self.workspace, self.row_order) if t is not None]

    def _rows(self, block_table, context_lens, page_size, num_pages, Hq, Hkv, d):
        B = context_lens.shape[0]
        _want(context_lens, "context_lens", (B,), (torch.int32,), self.device)
        _want(block_table, "block_table", (B, block_table.shape[-1]), (torch.int32,), self.device)
        if Hq <= 0 or Hq % Hkv:
            raise ValueError(f"{Hq} query heads over {Hkv} KV heads")
        self.block_table, self.context_lens = block_table, context_lens
        self.B, self.Hq, self.Hkv, self.d = B, Hq, Hkv, d
        self.page_size, self.num_pages, self.max_pages_per_seq = page_size, num_pages, block_table.shape[1]

    def plan(self, lens_host=None, max_context_len=None, num_splits=None, row_order="auto"):
        """Chooses the splits.  ``lens_host``: the rows' cached tokens on the host (< 0: inactive), as the scheduler
        that built context_lens has them; without them every row counts ``max_context_len`` tokens (default: what
        the block table can hold).  Plan again when the lengths outgrow max_context_len: the last split takes what lies
        beyond it, which is right but slow.  Graphs captured before keep the plan that they were captured under.
        ``row_order``: the order in which the grid serves the rows, a permutation on the host, None for the kernel's own, or "auto"
        (longest first where lens_host is known and the grid is more than one wave deep)."""
        if lens_host is not None and len(lens_host) != self.B:
            raise ValueError(f"{len(lens_host)} lengths for {self.B} rows")
        if row_order is not None and not (isinstance(row_order, str) and row_order == "auto"):
            row_order = np.asarray(row_order)              # the kernels index the rows with it
            if not np.array_equal(np.sort(row_order, axis=None), np.arange(self.B)) or row_order.ndim != 1:
                raise ValueError(f"row_order: expected 'auto' or a permutation of 0 .. {self.B - 1}")
        if max_context_len is None:
            max_context_len = (max(1, max(int(n) + 1 for n in lens_host)) if lens_host is not None
                               else self.max_pages_per_seq * self.page_size)
        self.max_context_len = int(max_context_len)
        span = min(self.max_context_len, ac.ac_window_span(self.window, self.sinks))
        counts = [min(int(n) + 1, span) if n >= 0 else 0 for n in lens_host] if lens_host is not None else None
        with torch.cuda.device(self.device):
            if num_splits is None:
                num_splits = self._choose(counts, span)
            self._replace_buffers()
            self.num_splits = int(num_splits)
            self.workspace_bytes = ac.ac_fused_workspace_bytes(self.B, self.Hq, self.Hkv, self.d, self.num_splits)
            self.workspace = torch.zeros(max(self.workspace_bytes, 16) // 4, dtype=torch.float32, device=self.device)
            torch.cuda.current_stream().synchronize()      # zeroed whatever stream the calls run on
            self.row_order = None
            if isinstance(row_order, str):
                deep = self.B > 1 and self.B * self.Hkv * self.num_splits > 2 * (ac.ac_sm_count() or 148)
                if lens_host is not None and deep:
                    row_order = np.argsort(-np.asarray(lens_host, dtype=np.int64), kind="stable")
                else:
                    row_order = None
            if row_order is not None:
                self.row_order = torch.from_numpy(np.asarray(row_order, np.int32).copy()).to(self.device)
        self._options = ac._options(self.window, True, self.row_order, sinks=self.sinks)
        self._marshal()


class PagedAttention(_Rows):
    """Decode attention over a bf16 cache of the caller's, with an optional sliding window and sinks.

    ``k_cache``, ``v_cache``: [num_pages, page_size, Hkv, d] ("token_major") or [num_pages, Hkv, page_size, d].  The
    object owns its workspace: its calls, and replays of graphs captured from them, must not overlap on the GPU (one
    object per stream)."""

    def __init__(self, k_cache, v_cache, block_table, context_lens, Hq, lens_host=None, window=0, sinks=0,
                 max_context_len=None, num_splits=None, row_order="auto", layout="token_major", softmax_scale=0.0,
                 new_tokens=1):
        self._bind(k_cache.device)
        if k_cache.dim() != 4:
            raise ValueError(f"k_cache: {k_cache.dim()} dimensions, expected 4")
        _want(k_cache, "k_cache", k_cache.shape, _BF16, self.device)
        _want(v_cache, "v_cache", k_cache.shape, _BF16, self.device)
        token, head = _axes(layout)
        self.k_cache, self.v_cache, self.window, self.sinks = k_cache, v_cache, int(window), int(sinks)
        self.softmax_scale, self.new_tokens = float(softmax_scale), _new_tokens(new_tokens)
        self._strides = (k_cache.stride(0), k_cache.stride(token), k_cache.stride(head))
        self._rows(block_table, context_lens, k_cache.shape[token], k_cache.shape[0], Hq, k_cache.shape[head],
                   k_cache.shape[3])
        self._q_shape = torch.Size((self.B, self.Hq, self.d))
        self.plan(lens_host, max_context_len, num_splits, row_order)

    def _choose(self, counts, span):
        if counts is not None:
            return ac.ac_decode_plan_for_lengths(counts, self.Hq, self.Hkv, self.d, self.page_size, span)[0]
        return ac.ac_decode_plan(self.B, self.Hq, self.Hkv, self.d, self.page_size, span)[0]

    def _marshal(self):
        self._args = [None, self.k_cache.data_ptr(), self.v_cache.data_ptr(), *self._strides,
                      self.block_table.data_ptr(), self.max_pages_per_seq, self.context_lens.data_ptr(),
                      self.new_tokens, self.softmax_scale, self.num_splits, self.workspace.data_ptr(),
                      self.workspace_bytes, None, self.B, self.Hq, self.Hkv, self.d, self.page_size, self.num_pages,
                      self.max_context_len, self._flag, None, self._options]

    def attention(self, q, out=None, stream=None):
        """q: rotated queries [B, Hq, d] bf16; returns out [B, Hq, d] bf16 (allocated unless given)."""
        _want(q, "q", self._q_shape, _BF16, self.device)
        if out is None:
            out = self._new(self._q_shape, stream, q.dtype)
        else:
            _want(out, "out", self._q_shape, _BF16, self.device)
        args = self._args.copy()
        args[0], args[14] = q.data_ptr(), out.data_ptr()
        self._enqueue("ac_paged_decode_attn_ex", args, stream, -2)
        return out


class Q4Cache(_OnDevice):
    """A 4-bit paged cache over the caller's tensors (``empty`` allocates them).

    ``k_codes``, ``v_codes``: uint8 [num_pages, page_size, Hkv, d/2] ("token_major") or [num_pages, Hkv, page_size,
    d/2] ("head_major"); ``params``: bf16 [num_pages, Hkv, page_size, 2, d/group, 2] (K and V; scale, minimum)."""

    def __init__(self, k_codes, v_codes, params, page_size=None, layout="token_major"):
        self._bind(k_codes.device)
        if k_codes.dim() != 4 or params.dim() != 6:
            raise ValueError("codes have 4 dimensions, params 6")
        token, head = _axes(layout)
        self.num_pages, self.page_size, self.Hkv = k_codes.shape[0], k_codes.shape[token], k_codes.shape[head]
        self.d, self.layout = 2 * k_codes.shape[3], layout
        if page_size is not None and page_size != self.page_size:
            raise ValueError(f"codes have pages of {self.page_size} tokens, not {page_size}")
        groups = params.shape[4]
        if groups <= 0 or self.d % groups:
            raise ValueError(f"{groups} groups over {self.d} elements")
        self.group = self.d // groups
        _want(k_codes, "k_codes", k_codes.shape, (torch.uint8,), self.device)
        _want(v_codes, "v_codes", k_codes.shape, (torch.uint8,), self.device)
        _want(params, "params", (self.num_pages, self.Hkv, self.page_size, 2, groups, 2), _BF16, self.device)
        self.k_codes, self.v_codes, self.params = k_codes, v_codes, params
        self.struct = ac.q4_cache(k_codes, v_codes, params, k_codes.stride(0), k_codes.stride(token),
                                  k_codes.stride(head), self.group)

    @classmethod
    def empty(cls, num_pages, page_size, Hkv, d, group=64, layout="token_major", device="cuda:0"):
        _axes(layout)
        if group not in (32, 64, 128) or group > d:
            raise ValueError(f"group {group}: expected 32, 64 or 128, and at most {d}")
        shape = (num_pages, page_size, Hkv, d // 2) if layout == "token_major" else (num_pages, Hkv, page_size, d // 2)
        k, v = (torch.zeros(shape, dtype=torch.uint8, device=device) for _ in range(2))
        params = torch.zeros((num_pages, Hkv, page_size, 2, d // group, 2), dtype=torch.bfloat16, device=device)
        cache = cls(k, v, params, layout=layout)
        cache._allocated = (k, v, params)
        return cache

    _allocated = ()

    def _buffers(self):
        return [self.status_flag, *self._allocated]

    @property
    def pools(self):
        """(tensor, segments of a page) of the three pools, for CachePages."""
        codes = 1 if self.layout == "token_major" else self.Hkv
        return [(self.k_codes, codes), (self.v_codes, codes), (self.params, self.Hkv)]

    def _bulk(self, name, k, v, block_table, start_pos, row_offsets, stream):
        B = start_pos.shape[0]
        total = k.shape[0]
        for t, what in ((k, "k"), (v, "v")):
            _want(t, what, (total, self.Hkv, self.d), _BF16, self.device)
        _want(start_pos, "start_pos", (B,), (torch.int32,), self.device)
        _want(row_offsets, "row_offsets", (B + 1,), (torch.int32,), self.device)
        _want(block_table, "block_table", (B, block_table.shape[-1]), (torch.int32,), self.device)
        if total == 0:
            return
        self._enqueue(name, [k.data_ptr(), v.data_ptr(), self.struct, block_table.data_ptr(), block_table.shape[1],
                             start_pos.data_ptr(), row_offsets.data_ptr(), total, B, self.Hkv, self.d, self.page_size,
                             self.num_pages, self._flag, None], stream, -1)

    def store(self, k, v, block_table, start_pos, row_offsets, stream=None):
        """Quantises k, v (bf16 [tokens, Hkv, d], keys rotated): row b's tokens row_offsets[b] .. row_offsets[b+1] - 1
        go to positions start_pos[b], start_pos[b] + 1, ..."""
        self._bulk("ac_kv_store_q4", k, v, block_table, start_pos, row_offsets, stream)

    def load(self, block_table, start_pos, row_offsets, total_tokens=None, k_out=None, v_out=None, stream=None):
        """The same tokens as bf16 [tokens, Hkv, d]; outputs are allocated unless given."""
        if k_out is None or v_out is None:
            if total_tokens is None:
                raise ValueError("load needs total_tokens or both outputs")
            shape = (total_tokens, self.Hkv, self.d)
            k_out = self._new(shape, stream) if k_out is None else k_out
            v_out = self._new(shape, stream) if v_out is None else v_out
        self._bulk("ac_kv_load_q4", k_out, v_out, block_table, start_pos, row_offsets, stream)
        return k_out, v_out


class Q4DecodeStep(_Rows):
    """One decode step over a 4-bit cache: RoPE + quantised append, then attention (two launches).

    ``rope_variants``: rotary_dim, interleaved, q_norm_weight, k_norm_weight, norm_eps as in
    ``ac_rope_kv_append_ex``; the rope tables are only needed for ``append`` and ``step``.  The object owns its
    workspace: its calls, and replays of graphs captured from them, must not overlap on the GPU (one object per stream)."""

    def __init__(self, cache, block_table, context_lens, Hq, lens_host=None, window=0, sinks=0, rope_cos=None,
                 rope_sin=None, max_context_len=None, num_splits=None, row_order="auto", rope_variants=None,
                 softmax_scale=0.0, new_tokens=1):
        self._bind(cache.device)
        self.cache, self.window, self.sinks = cache, int(window), int(sinks)
        self.softmax_scale, self.new_tokens = float(softmax_scale), _new_tokens(new_tokens)
        self._rows(block_table, context_lens, cache.page_size, cache.num_pages, Hq, cache.Hkv, cache.d)
        self._q_shape, self._kv_shape = (torch.Size((self.B, h, self.d)) for h in (self.Hq, self.Hkv))
        self.rope_cos, self.rope_sin = rope_cos, rope_sin
        variants = dict(rope_variants or {})
        self._norms = (variants.get("q_norm_weight"), variants.get("k_norm_weight"))      # kept alive
        for t, what in zip(self._norms, ("q_norm_weight", "k_norm_weight")):
            if t is not None:
                _want(t, what, (self.d,), _BF16, self.device)
        self._rope = ac._rope_options(**variants)
        if (rope_cos is None) != (rope_sin is None):
            raise ValueError("rope_cos and rope_sin go together")
        if rope_cos is not None:
            rotary = int(variants.get("rotary_dim", 0)) or self.d
            for t, what in ((rope_cos, "rope_cos"), (rope_sin, "rope_sin")):
                _want(t, what, (rope_cos.shape[0], rotary // 2), (torch.float32,), self.device)
        self.plan(lens_host, max_context_len, num_splits, row_order)

    def _buffers(self):
        return super()._buffers() + self.cache._buffers()

    def _choose(self, counts, span):
        return ac.ac_decode_plan_q4(counts, self.B, self.Hq, self.Hkv, self.d, self.page_size, span)[0]

    def _marshal(self):
        shape = [self.B, self.Hq, self.Hkv, self.d, self.page_size, self.num_pages]
        table = [self.cache.struct, self.block_table.data_ptr(), self.max_pages_per_seq, self.context_lens.data_ptr()]
        self._attn_args = [None, *table, self.new_tokens, self.softmax_scale, self.num_splits,
                           self.workspace.data_ptr(), self.workspace_bytes, None, *shape, self.max_context_len,
                           self._flag, None, self._options]
        if self.rope_cos is not None:
            self._append_args = [None, None, None, None, *table, self.rope_cos.data_ptr(), self.rope_sin.data_ptr(),
                                 self.rope_cos.shape[0], *shape, self._flag, None, self._rope]

    def append(self, q_in, k_new, v_new, q_out=None, stream=None):
        """Rotates q_in [B, Hq, d] into q_out (allocated unless given, may be q_in) and writes k_new, v_new
        [B, Hkv, d] into the slot at context_lens[b]; returns q_out."""
        if self.rope_cos is None:
            raise ValueError("append needs the rope tables")
        _want(q_in, "q_in", self._q_shape, _BF16, self.device)
        _want(k_new, "k_new", self._kv_shape, _BF16, self.device)
        _want(v_new, "v_new", self._kv_shape, _BF16, self.device)
        if q_out is None:
            q_out = self._new(self._q_shape, stream, q_in.dtype)
        elif q_out is not q_in:
            _want(q_out, "q_out", self._q_shape, _BF16, self.device)
        args = self._append_args.copy()
        args[:4] = q_in.data_ptr(), q_out.data_ptr(), k_new.data_ptr(), v_new.data_ptr()
        self._enqueue("ac_rope_kv_append_q4", args, stream, -2)
        return q_out

    def attention(self, q, out=None, stream=None):
        """q: rotated queries [B, Hq, d] bf16; returns out [B, Hq, d] bf16 (allocated unless given)."""
        _want(q, "q", self._q_shape, _BF16, self.device)
        if out is None:
            out = self._new(self._q_shape, stream, q.dtype)
        else:
            _want(out, "out", self._q_shape, _BF16, self.device)
        args = self._attn_args.copy()
        args[0], args[10] = q.data_ptr(), out.data_ptr()
        self._enqueue("ac_paged_decode_attn_q4", args, stream, -2)
        return out

    def step(self, q_in, k_new, v_new, q_rot=None, out=None, stream=None):
        """append, then attention over context_lens[b] + 1 tokens."""
        if self.new_tokens != 1:
            raise ValueError(f"step attends over the token that it appends: new_tokens is {self.new_tokens}, not 1")
        return self.attention(self.append(q_in, k_new, v_new, q_rot, stream), out, stream)


class CachePages(_OnDevice):
    """Pages of any number of pools under one block table: reserve, fork, release, trim, compact, copy.

    ``pools``: contiguous tensors [num_pages, ...], each alone or with the number of segments of its page ([page,
    slot, ...]: 1; [page, head, slot, ...]: the heads).  ``block_table`` int32 [rows, max_pages_per_seq],
    ``context_lens`` int32 [rows] (< 0: unused), ``ref_counts`` int32 [num_pages] (0: free); all are updated in place.
    ``status_flag`` collects what went wrong on the device (AC_FLAG_...).  The object owns its workspace: its calls must
    not overlap on the GPU."""

    def __init__(self, pools, block_table, context_lens, ref_counts, page_size):
        self._bind(block_table.device)
        self.rows, self.max_pages_per_seq = block_table.shape
        self.num_pages, self.page_size = ref_counts.shape[0], int(page_size)
        _want(block_table, "block_table", (self.rows, self.max_pages_per_seq), (torch.int32,), self.device)
        _want(context_lens, "context_lens", (self.rows,), (torch.int32,), self.device)
        _want(ref_counts, "ref_counts", (self.num_pages,), (torch.int32,), self.device)
        self.block_table, self.context_lens, self.ref_counts = block_table, context_lens, ref_counts
        self.pools = [p if isinstance(p, tuple) else (p, 1) for p in pools]
        described = []
        for t, segments in self.pools:
            if t.shape[0] != self.num_pages:
                raise ValueError(f"a pool of {t.shape[0]} pages, ref_counts of {self.num_pages}")
            _want(t, "pool", t.shape, (t.dtype,), self.device)
            described.append((t, t.numel() // self.num_pages * t.element_size(), segments))
        self._pools = ac.page_pools(described)
        self.workspace = torch.empty(ac.ac_cache_workspace_bytes(self.rows, self.num_pages, self.rows),
                                     dtype=torch.uint8, device=self.device)
        self._room = (self.workspace.data_ptr(), self.workspace.numel())

    def _buffers(self):
        return [self.status_flag, self.workspace]

    def reserve(self, new_tokens, stream=None):
        """Pages for new_tokens more tokens of every active row, lowest free page first, rows in order.  Let the rows
        grow by that many tokens before the next call, or call trim() first."""
        self._enqueue("ac_cache_reserve",
                      [self.block_table.data_ptr(), self.max_pages_per_seq, self.context_lens.data_ptr(),
                       self.ref_counts.data_ptr(), int(new_tokens), self.rows, self.page_size, self.num_pages,
                       *self._room, self._flag, None], stream, -1)

    def fork(self, pairs, stream=None):
        """pairs: int32 [n, 2] (parent row, child row); at most as many as the table has rows."""
        n = pairs.shape[0]
        _want(pairs, "pairs", (n, 2), (torch.int32,), self.device)
        if n > self.rows:
            raise ValueError(f"{n} forks in a table of {self.rows} rows")
        if n == 0:
            return
        self._enqueue("ac_cache_fork",
                      [self._pools, len(self.pools), self.block_table.data_ptr(), self.max_pages_per_seq,
                       self.context_lens.data_ptr(), self.ref_counts.data_ptr(), pairs.data_ptr(), n, self.rows,
                       self.page_size, self.num_pages, *self._room, self._flag, None], stream, -1)

    def release(self, row_list, stream=None):
        """row_list: int32 [n]; unused and repeated rows are no-ops.  Pages reserved for the rows stay taken until trim()."""
        n = row_list.shape[0]
        _want(row_list, "row_list", (n,), (torch.int32,), self.device)
        if n == 0:
            return
        self._enqueue("ac_cache_release",
                      [self.block_table.data_ptr(), self.max_pages_per_seq, self.context_lens.data_ptr(),
                       self.ref_counts.data_ptr(), row_list.data_ptr(), n, self.rows, self.page_size, self.num_pages,
                       self._flag, None], stream, -1)

    def trim(self, stream=None):
        """Frees what was reserved and not used, for released rows too: counts the pages that the rows hold anew."""
        self._enqueue("ac_cache_trim",
                      [self.block_table.data_ptr(), self.max_pages_per_seq, self.context_lens.data_ptr(),
                       self.ref_counts.data_ptr(), self.rows, self.page_size, self.num_pages, self._flag, None], stream, -1)

    def copy(self, pairs, stream=None):
        """Copies whole pages: pairs int32 [n, 2] (source, destination)."""
        n = pairs.shape[0]
        _want(pairs, "pairs", (n, 2), (torch.int32,), self.device)
        if n == 0 or not self.pools:
            return
        self._enqueue("ac_cache_copy_pages", [self._pools, len(self.pools), pairs.data_ptr(), n, self.num_pages,
                                              self._flag, None], stream, -1)

    def compact(self, table_out=None, refs_out=None, live_out=None, stream=None):
        """Moves the live pages to the lowest ids; nothing may be reserved (trim() before it).  In place, or (both given)
        into another table and counts, so that a step in flight can still read the old ones.  ``live_out`` int32 [1] receives the number of live pages."""
        if (table_out is None) != (refs_out is None):
            raise ValueError("table_out and refs_out go together")
        if table_out is None:
            table_out, refs_out = self.block_table, self.ref_counts
        _want(table_out, "table_out", (self.rows, self.max_pages_per_seq), (torch.int32,), self.device)
        _want(refs_out, "refs_out", (self.num_pages,), (torch.int32,), self.device)
        if live_out is not None:
            _want(live_out, "live_out", (1,), (torch.int32,), self.device)
        self._enqueue("ac_cache_compact",
                      [self._pools, len(self.pools), self.block_table.data_ptr(), table_out.data_ptr(),
                       self.max_pages_per_seq, self.context_lens.data_ptr(), self.ref_counts.data_ptr(),
                       refs_out.data_ptr(), self.rows, self.page_size, self.num_pages,
                       live_out.data_ptr() if live_out is not None else None, *self._room, self._flag, None],
                      stream, -1)
