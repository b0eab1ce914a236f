"""Driver of token rollouts: owns the pool, the page tables and the workspaces of a paged key-value
cache for groups of trajectories and issues the library calls in the order of a rollout (prompts in,
expansion, decoding steps, prunes, release).  Allocation and streams are torch's; every number is
computed by the library's kernels.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B


class PagedCache:
    """A paged cache of up to ``max_rows`` rows of up to ``max_tokens`` tokens on the current device.

    Rows are group-major, as everywhere in the library; after ``fork`` with a fan-out the cache knows
    how many tokens a group's rows have in common, and attention reads those once per group.

    Calls run on the current stream.  The workspaces are the stream's own, so calls on several streams may overlap;
    the pool, the tables and the lengths are one, and who changes them while another stream reads them orders the two."""

    def __init__(self, n_pages: int, page_size: int, n_layers: int, n_kv_heads: int, head_dim: int, max_rows: int,
                 max_tokens: int, dtype: torch.dtype = torch.bfloat16):
        if not torch.cuda.is_available():
            raise RuntimeError("the rollout library needs a CUDA device; there is no CPU path")
        dev = torch.device("cuda", torch.cuda.current_device())
        self.dev, self.page_size, self.max_rows = dev, page_size, max_rows
        self.k, self.v = (torch.zeros(n_layers, n_pages, n_kv_heads, page_size, head_dim, device=dev, dtype=dtype) for _ in range(2))
        width = -(-max_tokens // page_size)
        self._tables = [torch.full((max_rows, width), -1, device=dev, dtype=torch.int32) for _ in range(2)]
        self._lens = [torch.zeros(max_rows, device=dev, dtype=torch.int32) for _ in range(2)]
        self._grown = torch.zeros(max_rows, device=dev, dtype=torch.int32)
        self._extended = False               # whether _grown is about the present rows
        self._cur = 0
        self.refs = torch.zeros(n_pages, device=dev, dtype=torch.int32)
        self.status = torch.zeros(1, device=dev, dtype=torch.int32)
        self.group, self.shared = 1, None
        self._spaces, self._in_graphs = {}, {}
        self.n_rows = 0

    def _describe(self):
        self.kv = B.make_kv(self.k, self.v, self.table, self.len, self._grown[: self._n_rows])

    @property
    def n_rows(self) -> int:
        return self._n_rows

    @n_rows.setter
    def n_rows(self, n: int):
        if not 0 <= n <= self.max_rows:
            raise ValueError(f"{n} rows in a cache of {self.max_rows}")
        self._n_rows = n
        self._describe()

    @property
    def table(self) -> torch.Tensor:
        return self._tables[self._cur][: self._n_rows]

    @property
    def len(self) -> torch.Tensor:
        return self._lens[self._cur][: self._n_rows]

    def _space(self, nbytes: int) -> torch.Tensor:
        """The current stream's workspace, zeroed when it is made and grown when a call asks for more.  Calls on two streams may
        overlap, so each stream has its own.  A graph under capture whose stream has none yet gets one that only the graph knows,
        since what zeroes it runs at the replay; one that a graph has been given is kept when the stream's grows."""
        stream, capturing = B._stream(None), torch.cuda.is_current_stream_capturing()
        space = self._spaces.get(stream)
        if space is None or space.nbytes < nbytes:
            space = torch.zeros(nbytes, device=self.dev, dtype=torch.uint8)
            if not capturing:
                self._spaces[stream] = space
        elif capturing:
            self._in_graphs[space.data_ptr()] = space
        return space

    def admit(self, n_rows: int) -> None:
        """Starts over with n_rows empty rows; whatever the cache held is released."""
        if not 0 <= n_rows <= self.max_rows:
            raise ValueError(f"{n_rows} rows in a cache of {self.max_rows}")
        B.kv_fork(self.kv, None, None, None, self.refs, self.refs, self._space(B.kv_fork_workspace_bytes(self.kv, 0)),
                  status=self.status)
        self._lens[self._cur].zero_()
        self._extended = False
        self.group, self.shared = 1, None
        self.n_rows = n_rows

    def extend(self, n_new) -> None:
        """Room for n_new more tokens in every row (an int, or int32 [rows]).  A row without room (``check`` reports it)
        keeps its tokens: the new ones that ``append`` and ``attend`` are given for it are left out."""
        B.kv_extend(self.kv, n_new, self.len, self.refs, self.refs, status=self.status)
        self._extended = True

    def _want_room(self) -> None:
        if not self._extended:
            raise ValueError("new tokens without room for them: extend first")

    def append(self, layer: int, k_new, v_new, start=None) -> None:
        """Keys and values of the rows' last tokens (after ``extend``)."""
        self._want_room()
        B.kv_append(self.kv, layer, k_new, v_new, start, status=self.status)

    def attend(self, layer: int, q, k_new=None, v_new=None, out=None, lse=None, scale: Optional[float] = None):
        """Attention of the rows' newest token over the cache; with k_new / v_new that token is stored on
        the way (after ``extend(1)``)."""
        if k_new is not None:
            self._want_room()
        out = torch.empty_like(q, memory_format=torch.contiguous_format) if out is None else out
        ws = self._space(B.kv_attend_workspace_bytes(self.kv, q.shape[1], self.group))
        B.kv_attend(self.kv, layer, q, out, ws, k_new=k_new, v_new=v_new, lse=lse, scale=scale, group=self.group, shared=self.shared,
                    status=self.status)
        return out

    def _fork(self, src_rows) -> None:
        n = src_rows.numel()
        if n > self.max_rows:
            raise ValueError(f"{n} rows in a cache of {self.max_rows}")
        other = self._cur ^ 1
        B.kv_fork(self.kv, src_rows, self._tables[other][:n], self._lens[other][:n], self.refs, self.refs,
                  self._space(B.kv_fork_workspace_bytes(self.kv, n)), status=self.status)
        self._cur = other
        self._extended = False
        self.n_rows = n

    def expand(self, fan: int) -> None:
        """Every row becomes a group of ``fan`` rows that share its full pages."""
        if fan < 1:
            raise ValueError("fan: at least one row of each")
        shared = torch.div(self.len, self.page_size, rounding_mode="floor") * self.page_size
        self._fork(torch.arange(self.n_rows, device=self.dev, dtype=torch.int32).repeat_interleave(fan))
        self.group, self.shared = fan, shared.to(torch.int32)

    def prune(self, src_rows, keep: int) -> None:
        """Keeps the rows that a prune has kept (pg_prune_ovf's src_rows: ``keep`` per group, group-major)
        and frees the pages of the others."""
        if keep < 1 or src_rows.numel() * self.group != self.n_rows * keep:
            raise ValueError("src_rows: `keep` rows of every group")
        self._fork(src_rows)
        self.group = keep

    def pack(self) -> None:
        """Moves the pages in use to the front of the pool."""
        B.kv_pack(self.kv, self.refs, self.refs, self.table, self._space(B.kv_pack_workspace_bytes(self.kv)), status=self.status)

    def check(self) -> None:
        """Raises PgError if a call has flagged a bad index, a full table or an exhausted pool; synchronises."""
        B.kv_status(self.status)
