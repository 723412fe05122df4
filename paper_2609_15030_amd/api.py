"""Torch-facing helpers over the C ABI: move inputs to the device, allocate
outputs, checkpoint rows and workspace, and call the entry points.

Allocation and marshalling only; all computation happens in liblinattn.so.
"""
from __future__ import annotations

import dataclasses
from typing import Optional, Sequence

import numpy as np
import torch

from . import linattn as la
from .workloads import BF16, Inputs


@dataclasses.dataclass
class DeviceInputs:
    q: torch.Tensor
    k: torch.Tensor
    v: torch.Tensor
    g: torch.Tensor
    beta: torch.Tensor
    cu_dev: torch.Tensor
    cu_host: np.ndarray
    io_dtype: int

    @property
    def n_seqs(self) -> int:
        return len(self.cu_host) - 1

    @property
    def n_heads(self) -> int:
        return self.q.shape[1]

    @property
    def dk(self) -> int:
        return self.q.shape[2]

    @property
    def dv(self) -> int:
        return self.v.shape[2]

    @property
    def total_tokens(self) -> int:
        return int(self.cu_host[-1])


def torch_dtype(io_dtype: int):
    return torch.bfloat16 if io_dtype == la.LA_BF16 else torch.float32


def to_device(x: Inputs, device="cuda") -> DeviceInputs:
    """Exact conversion: the arrays already hold values of the storage dtype."""
    io = la.LA_BF16 if x.io_dtype == BF16 else la.LA_F32
    td = torch_dtype(io)

    def dev(a, dt):
        return torch.from_numpy(np.ascontiguousarray(a)).to(device=device, dtype=dt).contiguous()

    cu = np.ascontiguousarray(x.cu_seqlens, dtype=np.int32)
    return DeviceInputs(dev(x.q, td), dev(x.k, td), dev(x.v, td), dev(x.g, torch.float32),
                        dev(x.beta, torch.float32), dev(cu, torch.int32), cu, io)


def checkpoint_rows(lengths: Sequence[int], starts: Optional[Sequence[int]], interval: int):
    """Row offsets for the checkpoints of each sequence and the total, as the
    library numbers them (la_checkpoint_rows)."""
    cu = np.concatenate([[0], np.cumsum(np.asarray(lengths, np.int64))]).astype(np.int32)
    return la.la_checkpoint_rows(cu, None if starts is None else np.asarray(starts, np.int64), interval)


@dataclasses.dataclass
class PrefillResult:
    o: torch.Tensor
    final_state: torch.Tensor
    ckpt: Optional[torch.Tensor]
    ckpt_offsets: np.ndarray
    n_ckpt_rows: int


class Prefill:
    """Reusable buffers for repeated prefill calls of one shape."""

    def __init__(self, x: DeviceInputs, interval: int, variant: int = la.LA_GDR_LITERAL,
                 scale: float = 1.0, starts: Optional[Sequence[int]] = None,
                 emit_ckpt: bool = True):
        self.x = x
        self.shape = la.make_shape(x.n_seqs, x.n_heads, x.dk, x.dv, interval, x.io_dtype,
                                   variant, scale)
        dev = x.q.device
        lens = np.diff(x.cu_host).tolist()
        self.starts = None if starts is None else np.asarray(starts, np.int64)
        self.ckpt_offsets, self.n_ckpt_rows = checkpoint_rows(lens, starts, interval)
        self.ckpt_off_dev = torch.from_numpy(self.ckpt_offsets).to(dev)
        self.start_dev = None if starts is None else torch.from_numpy(self.starts).to(dev)
        self.o = torch.empty((x.total_tokens, x.n_heads, x.dv), dtype=x.q.dtype, device=dev)
        self.final = torch.empty((x.n_seqs, x.n_heads, x.dk, x.dv), dtype=torch.float32, device=dev)
        self.ckpt = None
        if emit_ckpt and self.n_ckpt_rows > 0:
            self.ckpt = torch.empty((self.n_ckpt_rows, x.n_heads, x.dk, x.dv), dtype=torch.float32,
                                    device=dev)
        nbytes = la.la_prefill_workspace_bytes(self.shape, x.total_tokens)
        assert nbytes > 0
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)

    def run(self, state_in: Optional[torch.Tensor] = None, stream=None) -> PrefillResult:
        """la_prefill (cold) or la_prefill_resume (with start positions)."""
        x = self.x
        ck = self.ckpt
        if self.starts is None:
            la.la_prefill(self.shape, x.q, x.k, x.v, x.g, x.beta, x.cu_dev, x.cu_host, self.o,
                          self.final, ck, self.ckpt_off_dev if ck is not None else None,
                          self.ckpt_offsets if ck is not None else None, self.workspace, stream)
        else:
            assert state_in is not None
            la.la_prefill_resume(self.shape, x.q, x.k, x.v, x.g, x.beta, x.cu_dev, x.cu_host,
                                 self.start_dev, self.starts, state_in, self.o, self.final, ck,
                                 self.ckpt_off_dev if ck is not None else None,
                                 self.ckpt_offsets if ck is not None else None, self.workspace,
                                 stream)
        return PrefillResult(self.o, self.final, ck, self.ckpt_offsets, self.n_ckpt_rows)


    def run_paged(self, pool: torch.Tensor, ckpt_page_ids: Optional[torch.Tensor] = None,
                  state_page_ids: Optional[torch.Tensor] = None, err_count: Optional[torch.Tensor] = None,
                  stream=None) -> PrefillResult:
        """la_prefill_paged: checkpoints to pool pages (rows numbered as
        ckpt_offsets), starting states from pool pages (a resume).  The
        result's ckpt is None: the checkpoints live in the pool."""
        x = self.x
        pages = la.make_pages(pool, ckpt_page_ids, state_page_ids, err_count)
        with_ck = ckpt_page_ids is not None
        la.la_prefill_paged(self.shape, pages, x.q, x.k, x.v, x.g, x.beta, x.cu_dev, x.cu_host, self.start_dev,
                            self.starts, self.o, self.final, self.ckpt_off_dev if with_ck else None,
                            self.ckpt_offsets if with_ck else None, self.workspace, stream)
        return PrefillResult(self.o, self.final, None, self.ckpt_offsets, self.n_ckpt_rows)


def prefill(x: DeviceInputs, interval: int, variant: int = la.LA_GDR_LITERAL, scale: float = 1.0,
            emit_ckpt: bool = True) -> PrefillResult:
    return Prefill(x, interval, variant, scale, None, emit_ckpt).run()


def prefill_resume(x: DeviceInputs, starts: Sequence[int], state_in: torch.Tensor, interval: int,
                   variant: int = la.LA_GDR_LITERAL, scale: float = 1.0,
                   emit_ckpt: bool = True) -> PrefillResult:
    return Prefill(x, interval, variant, scale, starts, emit_ckpt).run(state_in)


# ---------------------------------------------------------------------------
# the attention side of a hybrid cache
# ---------------------------------------------------------------------------

class AttnPrefill:
    """Causal attention of prompts: lengths, workspace and output of one batch.

    new: tokens of each sequence in the call; kv: keys of each sequence, for
    calls over a cache (run_paged; None: as many as its tokens)."""

    def __init__(self, q_heads: int, kv_heads: int, head_dim: int, new: Sequence[int],
                 kv: Optional[Sequence[int]] = None, dtype=torch.bfloat16, scale: Optional[float] = None,
                 device="cuda"):
        self.shape = la.make_attn_shape(len(new), q_heads, kv_heads, head_dim, la._dtype_of(dtype), scale)
        self.cu_host = np.concatenate([[0], np.cumsum(np.asarray(new, np.int64))]).astype(np.int32)
        self.kv_host = None if kv is None else np.ascontiguousarray(kv, dtype=np.int32)
        self.cu_dev = torch.from_numpy(self.cu_host).to(device)
        self.kv_dev = None if kv is None else torch.from_numpy(self.kv_host).to(device)
        self.o = torch.empty((int(self.cu_host[-1]), q_heads, head_dim), dtype=dtype, device=device)
        n = la.la_attn_prefill_workspace_bytes(self.shape, self.cu_host, self.kv_host)
        if n == 0:
            raise ValueError(la.last_error_message())
        self.workspace = torch.empty(n, dtype=torch.uint8, device=device)

    def run(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, stream=None) -> torch.Tensor:
        la.la_attn_prefill(self.shape, q, k, v, self.cu_dev, self.cu_host, self.o, self.workspace, stream)
        return self.o

    def run_paged(self, layer: la.LaKvLayer, q: torch.Tensor, stream=None) -> torch.Tensor:
        la.la_attn_prefill_paged(self.shape, layer, q, self.cu_dev, self.cu_host, self.kv_dev, self.kv_host, self.o,
                                 self.workspace, stream)
        return self.o


class AttnDecode:
    """Attention of one new token per sequence, up to max_kv_len keys each.

    cu_group: device int32 [n_groups + 1], the groups of consecutive sequences
    that share a prefix of at most max_prefix_len keys (None: nothing shared);
    max_group: the most sequences of a group (None: read from cu_group; n_seqs
    where its groups are all empty, since they may be filled later)."""

    def __init__(self, n_seqs: int, q_heads: int, kv_heads: int, head_dim: int, max_kv_len: int,
                 dtype=torch.bfloat16, scale: Optional[float] = None, cu_group: Optional[torch.Tensor] = None,
                 max_prefix_len: int = 0, max_group: Optional[int] = None, device="cuda"):
        self.shape = la.make_attn_shape(n_seqs, q_heads, kv_heads, head_dim, la._dtype_of(dtype), scale)
        self.max_kv_len, self.cu_group, self.max_prefix_len = int(max_kv_len), cu_group, int(max_prefix_len)
        if cu_group is not None and max_group is None:
            max_group = (int((cu_group[1:] - cu_group[:-1]).max()) if cu_group.numel() > 1 else 0) or n_seqs
        self.max_group = max_group
        self.o = torch.empty((n_seqs, q_heads, head_dim), dtype=dtype, device=device)
        n = la.la_attn_decode_workspace_bytes(self.shape, self.max_kv_len, self.max_prefix_len)
        if n == 0:
            raise ValueError(la.last_error_message())
        self.workspace = torch.empty(n, dtype=torch.uint8, device=device)

    def run(self, layer: la.LaKvLayer, q: torch.Tensor, kv_len: torch.Tensor,
            prefix_len: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """prefix_len: device int32 [n_groups], shared keys of each group."""
        groups = None
        if self.cu_group is not None and prefix_len is not None:
            groups = la.make_prefix_groups(self.cu_group, prefix_len, self.max_group, self.max_prefix_len)
        la.la_attn_decode(self.shape, layer, q, kv_len, self.max_kv_len, self.o, groups, self.workspace, stream)
        return self.o


class Rope:
    """Rotary positions of heads of head_dim: the first rotary_dim dims (None:
    all) in pairs (i, i + rotary_dim / 2) (layout "halves") or (2 i, 2 i + 1)
    ("pairs"), at frequencies base^(-2 i / rotary_dim) under a scaling
    (la.make_rope_scaling), or at given ones (radians a token, fp64)."""

    def __init__(self, head_dim: int, rotary_dim: Optional[int] = None, layout: str = "halves", base: float = 10000.0,
                 scaling: Optional[la.LaRopeScaling] = None, frequencies: Optional[np.ndarray] = None,
                 magnitude: float = 1.0, device="cuda"):
        self.head_dim, self.rotary_dim = int(head_dim), int(head_dim if rotary_dim is None else rotary_dim)
        self.layout, self.magnitude = layout, float(magnitude)
        if frequencies is None:
            frequencies = la.la_rope_frequencies(self.rotary_dim, base, scaling)
        self.frequencies = np.ascontiguousarray(frequencies, np.float64)
        self.turns = torch.from_numpy(la.la_rope_turns(self.frequencies).view(np.int64)).to(device)
        self._plans = {}                           # by type

    def apply(self, q: Optional[torch.Tensor], k: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
              k_out: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
              cu_seqlens: Optional[torch.Tensor] = None, kv_len: Optional[torch.Tensor] = None, transpose: bool = False,
              stream=None):
        """Turns q and k [T, heads, head_dim] at positions int32 [T], or at those
        of the sequences of cu_seqlens and kv_len (la_kv_write's); in place where no
        output is given.  transpose: the gradient.  Returns the outputs."""
        if q is None and k is None:
            raise ValueError("expected q, k or both")
        q_out, k_out = q if q_out is None else q_out, k if k_out is None else k_out
        dtype = (k if q is None else q).dtype
        plan = self._plans.get(dtype)
        if plan is None:
            plan = self._plans[dtype] = la.make_rope_plan(self.head_dim, self.rotary_dim, self.layout, la._dtype_of(dtype),
                                                          self.turns, self.magnitude)
        la.la_rope_apply(plan, q, q_out, k, k_out, positions, cu_seqlens, kv_len, transpose, stream)
        return q_out, k_out


class BlockPool:
    """The blocks of a cache with their table, reference counts and free list
    (la_block_pool), over tensors the caller holds; BlockPool.new makes an
    empty one."""

    def __init__(self, cache: torch.Tensor, block_tokens: int, table: torch.Tensor, ref_count: torch.Tensor,
                 free_list: torch.Tensor, free_count: torch.Tensor, err_count: Optional[torch.Tensor] = None):
        self.cache, self.block_tokens, self.table = cache, block_tokens, table
        self.ref_count, self.free_list, self.free_count, self.err_count = ref_count, free_list, free_count, err_count
        self.pool = la.make_block_pool(cache, block_tokens, table, ref_count, free_list, free_count, err_count)
        self.workspace = torch.empty(la.la_blocks_compact_workspace_bytes(cache.shape[0]), dtype=torch.uint8,
                                     device=cache.device)

    @staticmethod
    def new(n_blocks: int, block_bytes: int, block_tokens: int, n_rows: int, max_blocks: int, device="cuda") -> "BlockPool":
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)
        return BlockPool(torch.zeros((n_blocks, block_bytes), dtype=torch.uint8, device=device), block_tokens,
                         i32(n_rows, max_blocks) - 1, i32(n_blocks),
                         torch.arange(n_blocks - 1, -1, -1, dtype=torch.int32, device=device), i32(1) + n_blocks, i32(1))

    def copy(self, src_ids, dst_ids, stream=None):
        la.la_blocks_copy(self.pool, src_ids, dst_ids, stream)

    def fork(self, parent_rows, child_rows, lens, stream=None):
        la.la_blocks_fork(self.pool, parent_rows, child_rows, lens, stream)

    def extend(self, rows, lens, stream=None):
        la.la_blocks_extend(self.pool, rows, lens, stream)

    def free(self, rows, stream=None):
        la.la_blocks_free(self.pool, rows, stream)

    def compact(self, new_ids=None, stream=None):
        la.la_blocks_compact(self.pool, self.workspace, new_ids, stream)
