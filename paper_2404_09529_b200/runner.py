"""Memory plumbing around the C-ABI calls: lays token-major tensors out as the packed (or padded)
batch, owns the device buffers and workspaces, and calls pp_pack / pp_prefill_attention /
pp_unpack_kv in order. All arithmetic of the method happens inside the library."""
from __future__ import annotations

import numpy as np
import torch

from . import binding as B


class PrefillBatch:
    """One batch of prompts on the device, ready to be prefilled.

    mode "packed": bins from pp_pack(lengths) (first-fit-decreasing, capacity = longest prompt).
    mode "padded": the full-batching baseline -- one bin per prompt in original order, every
    bin declared as a single segment of the full capacity, so all k*m rows are computed;
    unpack still copies only each prompt's true rows.
    mode "varlen": one bin per prompt in original order, each declared with its true length: the
    mask and tile skipping without the bin packing (isolates what packing adds).
    """

    SENTINEL = -1.0e30      # bf16 value that pre-fills guard regions and cache pools (guard=True)

    def __init__(self, lengths, n_q_heads: int, n_kv_heads: int, head_dim: int, rope_base: float,
                 mode: str = "packed", device: str = "cuda", softmax_scale: float = 0.0, room=0,
                 guard: bool = False, pack: "B.Packing | None" = None):
        """room (int or one int per prompt): spare rows in every prompt's cache block, so that
        cache_cap[i] = lengths[i] + room. guard: put sentinel-filled regions in front of and behind
        every buffer the library writes (O, K, both cache pools) and pre-fill the pools with the
        sentinel, so that `assert_untouched` can tell whether anything outside the documented
        outputs was written. pack: a packing made elsewhere (e.g. some bins of a packing of a whole
        stream of prompts, Packing.slice_bins) for exactly these prompts; mode is then "prepacked"."""
        self.device = torch.device(device)
        self.mode = "prepacked" if pack is not None else mode
        self._given_pack = pack
        self.lengths = np.ascontiguousarray(np.asarray(lengths, dtype=np.int32))
        self.k = int(self.lengths.shape[0])
        self.total_tokens = int(self.lengths.sum())
        self.hq, self.hkv, self.d = n_q_heads, n_kv_heads, head_dim
        self.rope_base, self.softmax_scale = rope_base, softmax_scale
        self._pack()
        R, M = self.pack.n_bins, self.pack.capacity
        dev, bf = self.device, torch.bfloat16
        self._guards = []
        self.q = torch.zeros((R, M, n_q_heads, head_dim), dtype=bf, device=dev)
        self.kk = self._alloc((R, M, n_kv_heads, head_dim), guard, 0.0)
        self.v = torch.zeros((R, M, n_kv_heads, head_dim), dtype=bf, device=dev)
        self.o = self._alloc((R, M, n_q_heads, head_dim), guard, 0.0)
        # per-prompt caches, one pool each, [Hkv, cap_i, D] blocks back to back in original order
        self.cache_cap = (self.lengths + np.asarray(room, dtype=np.int32)).astype(np.int32)
        cap_prefix = np.concatenate([[0], np.cumsum(self.cache_cap.astype(np.int64))])
        self.cache_off = (cap_prefix[:-1] * n_kv_heads * head_dim).astype(np.int64)
        pool = int(cap_prefix[-1]) * n_kv_heads * head_dim
        self.k_cache = self._alloc((pool,), guard, self.SENTINEL if guard else 0.0)
        self.v_cache = self._alloc((pool,), guard, self.SENTINEL if guard else 0.0)
        self.ws = B.Workspaces(self.params, self.pack.k, device=dev)
        # flat packed row of every real token, original prompt order
        rows = [np.arange(l, dtype=np.int64) + int(b) * M + int(off)
                for l, b, off in zip(self.lengths, self.bin_of, self.off_of)]
        self.token_rows = torch.from_numpy(np.concatenate(rows)).to(dev)

    def _alloc(self, shape, guard: bool, fill: float) -> torch.Tensor:
        """A device tensor of `shape`; with guard, the middle of a larger sentinel-filled buffer."""
        n = int(np.prod(shape))
        if not guard:
            return torch.full((n,), fill, dtype=torch.bfloat16, device=self.device).view(shape)
        g = 4096                                          # elements: keeps the payload 8 KB aligned
        whole = torch.full((n + 2 * g,), self.SENTINEL, dtype=torch.bfloat16, device=self.device)
        self._guards.append((whole, g, n))
        body = whole[g:g + n]
        body.fill_(fill)
        return body.view(shape)

    def assert_untouched(self) -> None:
        """Guard regions around O, K and the cache pools, and the spare rows [lengths[i], cap[i]) of
        every cache block, still hold the sentinel bit for bit (needs guard=True)."""
        assert self._guards, "PrefillBatch was built without guard=True"
        for whole, g, n in self._guards:
            for part in (whole[:g], whole[g + n:]):
                assert bool((part == self.SENTINEL).all()), "write outside an output buffer"
        for i in range(self.k):
            l = int(self.lengths[i])
            for c in self.caches(i):
                assert bool((c[:, l:] == self.SENTINEL).all()), f"spare cache rows of prompt {i} were written"

    def _pack(self) -> None:
        """BINPACK through the library (host)."""
        if self.mode == "prepacked":
            self.pack = self._given_pack
            self.bin_of, self.off_of = self.pack.bin_of, self.pack.off_of
        elif self.mode == "packed":
            self.pack = B.pp_pack(self.lengths, 0)
            self.bin_of, self.off_of = self.pack.bin_of, self.pack.off_of
        elif self.mode == "padded":
            m = int(self.lengths.max())
            self.pack = B.pp_pack(np.full(self.k, m, dtype=np.int32), 0)
            self.bin_of = np.arange(self.k, dtype=np.int32)
            self.off_of = np.zeros(self.k, dtype=np.int32)
        elif self.mode == "varlen":
            m = int(self.lengths.max())
            ar = np.arange(self.k, dtype=np.int32)
            self.pack = B.Packing(self.k, m, np.arange(self.k + 1, dtype=np.int32), ar.copy(),
                                  np.zeros(self.k, np.int32), self.lengths.copy(), ar.copy(),
                                  np.zeros(self.k, np.int32))
            self.bin_of, self.off_of = self.pack.bin_of, self.pack.off_of
        else:
            raise ValueError(self.mode)
        self.params = B.AttnParams(self.hq, self.hkv, self.d, self.rope_base, self.softmax_scale,
                                   self.pack.capacity, self.pack.n_bins, 0)

    def load(self, q_tok: torch.Tensor, k_tok: torch.Tensor, v_tok: torch.Tensor) -> None:
        """TENSORIZE: scatter token-major [T, H, D] tensors into the packed layout; padding rows zero."""
        for dst, src in ((self.q, q_tok), (self.kk, k_tok), (self.v, v_tok)):
            dst.zero_()
            dst.view(-1, dst.shape[2], dst.shape[3])[self.token_rows] = src.to(self.device)

    def run(self, flags: int = 0, repack: bool = False, unpack: bool = True) -> None:
        """One pass of the hot path on the current stream (asynchronous)."""
        if repack:
            self._pack()
        stream = B.current_stream()
        host_attn, host_unpack, slot = self.ws.acquire()
        self.params.flags = flags
        B.pp_prefill_attention(self.params, self.pack, self.q, self.kk, self.v, self.o, self.ws.attn_dev,
                               host_attn, self.ws.attn_bytes, self.ws.status, stream)
        if unpack:
            B.pp_unpack_kv(self.params, self.bin_of, self.off_of, self.lengths, self.kk, self.v, self.k_cache,
                           self.v_cache, self.cache_off, self.cache_cap, self.ws.unpack_dev, host_unpack,
                           self.ws.unpack_bytes, stream)
        self.ws.release(slot)

    def run_fused(self, repack: bool = False, flags: int = 0, keep_rope_table: bool = True) -> None:
        """One pass of the hot path through the fused entry point (asynchronous). q is left untouched.
        The fused workspace is written by nothing but these calls, so from the second call with the
        same capacity on, the cos/sin table in it is declared valid (PP_FLAG_KEEP_ROPE_TABLE)."""
        if repack:
            self._pack()
        stream = B.current_stream()
        _, _, slot = self.ws.acquire()
        if keep_rope_table and getattr(self, "_rope_table_capacity", None) == self.pack.capacity:
            flags |= B.PP_FLAG_KEEP_ROPE_TABLE
        self._rope_table_capacity = self.pack.capacity
        self.params.flags = flags
        B.pp_prefill_fused(self.params, self.pack, self.lengths, self.q, self.kk, self.v, self.o, self.k_cache,
                           self.v_cache, self.cache_off, self.cache_cap, self.ws.fused_dev,
                           self.ws.fused_host(slot), self.ws.fused_bytes, self.ws.status, stream)
        self.ws.release(slot)

    def run_unpack_only(self) -> None:
        stream = B.current_stream()
        _, host_unpack, slot = self.ws.acquire()
        B.pp_unpack_kv(self.params, self.bin_of, self.off_of, self.lengths, self.kk, self.v, self.k_cache,
                       self.v_cache, self.cache_off, self.cache_cap, self.ws.unpack_dev, host_unpack,
                       self.ws.unpack_bytes, stream)
        self.ws.release(slot)

    def device_status(self) -> int:
        return int(self.ws.status.item())

    # ---- views of the results, original prompt order (device tensors) ----
    def o_tokens(self) -> torch.Tensor:
        """[T, Hq, D] attention outputs of the real tokens."""
        return self.o.view(-1, self.hq, self.d)[self.token_rows]

    def rotated_tokens(self):
        """([T, Hq, D], [T, Hkv, D]): q and k as they stand in the packed buffers."""
        return (self.q.view(-1, self.hq, self.d)[self.token_rows],
                self.kk.view(-1, self.hkv, self.d)[self.token_rows])

    def caches(self, i: int):
        """(k_cache_i, v_cache_i) as [Hkv, cap_i, D] views of the pools; rows [0, lengths[i]) are filled."""
        n = int(self.cache_cap[i]) * self.hkv * self.d
        off = int(self.cache_off[i])
        shape = (self.hkv, int(self.cache_cap[i]), self.d)
        return self.k_cache[off:off + n].view(shape), self.v_cache[off:off + n].view(shape)


class DecodeBatch:
    """Per-prompt KV caches with room to grow, and one generation step at a time through
    pp_decode_step. Memory plumbing only: `adopt` copies the caches a PrefillBatch has filled into
    blocks of capacity lengths[i] + room."""

    def __init__(self, lengths, n_q_heads: int, n_kv_heads: int, head_dim: int, rope_base: float,
                 room: int = 32, device: str = "cuda", softmax_scale: float = 0.0):
        self.device = torch.device(device)
        self.lengths = np.ascontiguousarray(np.asarray(lengths, dtype=np.int32)).copy()
        self.k = int(self.lengths.shape[0])
        self.hq, self.hkv, self.d = n_q_heads, n_kv_heads, head_dim
        self.cache_cap = (self.lengths + room).astype(np.int32)
        prefix = np.concatenate([[0], np.cumsum(self.cache_cap.astype(np.int64))])
        self.cache_off = (prefix[:-1] * n_kv_heads * head_dim).astype(np.int64)
        pool = int(prefix[-1]) * n_kv_heads * head_dim
        self.k_cache = torch.zeros(pool, dtype=torch.bfloat16, device=self.device)
        self.v_cache = torch.zeros(pool, dtype=torch.bfloat16, device=self.device)
        self.params = B.AttnParams(n_q_heads, n_kv_heads, head_dim, rope_base, softmax_scale, 1, 1, 0)
        self.o = torch.zeros((self.k, n_q_heads, head_dim), dtype=torch.bfloat16, device=self.device)
        self._ws_bytes = 0
        self._ws = self._host = None

    def caches(self, i: int):
        """(k_cache_i, v_cache_i) as [Hkv, cap_i, D] views; rows [0, lengths[i]) are filled."""
        cap = int(self.cache_cap[i])
        n = cap * self.hkv * self.d
        off = int(self.cache_off[i])
        shape = (self.hkv, cap, self.d)
        return self.k_cache[off:off + n].view(shape), self.v_cache[off:off + n].view(shape)

    @classmethod
    def from_prefill(cls, prefill: PrefillBatch) -> "DecodeBatch":
        """Decode straight on the cache pools a PrefillBatch (built with room > 0) has filled: the
        hand-over from UNPACK to generation, no copy in between."""
        self = cls.__new__(cls)
        self.device = prefill.device
        self.lengths = prefill.lengths.copy()
        self.k = prefill.k
        self.hq, self.hkv, self.d = prefill.hq, prefill.hkv, prefill.d
        self.cache_cap, self.cache_off = prefill.cache_cap, prefill.cache_off
        self.k_cache, self.v_cache = prefill.k_cache, prefill.v_cache
        self.params = B.AttnParams(self.hq, self.hkv, self.d, prefill.rope_base, prefill.softmax_scale, 1, 1, 0)
        self.o = torch.zeros((self.k, self.hq, self.d), dtype=torch.bfloat16, device=self.device)
        self._ws_bytes = 0
        self._ws = self._host = None
        return self

    def adopt(self, prefill: PrefillBatch) -> None:
        for i in range(self.k):
            src_k, src_v = prefill.caches(i)
            dst_k, dst_v = self.caches(i)
            l = int(self.lengths[i])
            dst_k[:, :l].copy_(src_k[:, :l])
            dst_v[:, :l].copy_(src_v[:, :l])

    def step(self, q_new: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor) -> torch.Tensor:
        """One token per prompt: q_new [k, Hq, D], k_new / v_new [k, Hkv, D] bf16 on the device."""
        need = B.pp_decode_workspace_bytes(self.params, self.lengths)
        if need > self._ws_bytes:
            self._ws_bytes = need + (need >> 2)        # lengths grow by one per step
            self._ws = torch.empty(self._ws_bytes, dtype=torch.uint8, device=self.device)
            self._host = [torch.empty(self._ws_bytes, dtype=torch.uint8).pin_memory() for _ in range(2)]
            self._copied = [B.fence() for _ in range(2)]   # after the upload that last read each staging buffer
            self._turn = 0
        slot = self._turn & 1
        self._turn += 1
        self._copied[slot].synchronize()
        stream = B.current_stream()
        B.pp_decode_step(self.params, self.lengths, q_new, k_new, v_new, self.o, self.k_cache, self.v_cache,
                         self.cache_off, self.cache_cap, self._ws, self._host[slot], self._ws_bytes,
                         stream)
        self._copied[slot].record(stream)
        self.lengths += 1
        return self.o


class PagedCaches:
    """KV caches in pages: two pools of pages and the table that says which pages every prompt has (see
    ``pp_paged_cache`` in include/pp.h). The tensors may come from the caller, who then keeps the table; `allocate` makes
    them, and `reserve`, `share` and `release` hand pages out. Memory plumbing only."""

    TYPES = {torch.bfloat16: B.PP_CACHE_BF16, torch.float8_e4m3fn: B.PP_CACHE_E4M3}

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor, rows_first: bool = False,
                 k_scale: torch.Tensor | None = None, v_scale: torch.Tensor | None = None):
        """k_pages, v_pages: [n_pages, Hkv, page_size, D], or with rows_first [n_pages, page_size, Hkv, D]; bf16, or float8_e4m3fn
        with k_scale and v_scale (float32 [Hkv]). page_table: int32 [prompts, most pages of a prompt]."""
        head, row = (2, 1) if rows_first else (1, 2)
        if k_pages.dtype not in self.TYPES or k_pages.dim() != 4 or k_pages.stride(3) != 1:
            raise ValueError("pages are 4-D bfloat16 or float8_e4m3fn tensors, contiguous in the last dimension")
        if (v_pages.shape, v_pages.stride(), v_pages.dtype, v_pages.device) != (k_pages.shape, k_pages.stride(), k_pages.dtype, k_pages.device):
            raise ValueError("both pools have one shape, layout, type and device")
        if page_table.dtype != torch.int32 or page_table.dim() != 2 or page_table.device != k_pages.device or not page_table.is_contiguous():
            raise ValueError("the page table is a contiguous 2-D int32 tensor on the pools' device")
        self.n_pages, self.page_size = k_pages.shape[0], k_pages.shape[row]
        self.hkv, self.d = k_pages.shape[head], k_pages.shape[3]
        self.n_prompts = page_table.shape[0]
        e4m3 = k_pages.dtype == torch.float8_e4m3fn
        for scale in (k_scale, v_scale):
            if (scale is not None) != e4m3:
                raise ValueError("8-bit pages, and only they, have scales")
            if e4m3 and (scale.dtype != torch.float32 or scale.shape != (self.hkv,) or scale.device != k_pages.device or not scale.is_contiguous()):
                raise ValueError("a scale is a contiguous float32 [Hkv] tensor on the pools' device")
        self.device, self.index, self.rows_first = k_pages.device, k_pages.get_device(), rows_first
        self.k_pages, self.v_pages, self.page_table, self.k_scale, self.v_scale = k_pages, v_pages, page_table, k_scale, v_scale
        self.struct = B.PagedCache(
            k_pages.data_ptr(), v_pages.data_ptr(), k_scale.data_ptr() if e4m3 else None, v_scale.data_ptr() if e4m3 else None,
            page_table.data_ptr(), k_pages.stride(0), k_pages.stride(head), k_pages.stride(row), self.n_pages, self.page_size,
            page_table.shape[1], self.TYPES[k_pages.dtype])
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._append_params = {}
        self._count = self._users = None

    @classmethod
    def allocate(cls, n_prompts: int, n_pages: int, max_rows: int, n_kv_heads: int, head_dim: int, page_size: int = 64,
                 dtype: torch.dtype = torch.bfloat16, rows_first: bool = False, device: str = "cuda",
                 k_scale: torch.Tensor | None = None, v_scale: torch.Tensor | None = None) -> "PagedCaches":
        """Pools of n_pages zeroed pages and an empty table for n_prompts prompts of up to max_rows rows. The further layers of a
        model need no table of their own: PagedCaches(k_pages, v_pages, first.page_table), with pools of the same number of pages."""
        shape = (n_pages, page_size, n_kv_heads, head_dim) if rows_first else (n_pages, n_kv_heads, page_size, head_dim)
        pools = [torch.zeros(shape, dtype=torch.uint8 if dtype.itemsize == 1 else torch.bfloat16, device=device).view(dtype) for _ in range(2)]
        table = torch.full((n_prompts, -(-max_rows // page_size)), -1, dtype=torch.int32, device=device)
        self = cls(*pools, table, rows_first, k_scale, v_scale)
        self._table = np.full(tuple(table.shape), -1, dtype=np.int32)     # what the device table holds
        self._count = np.zeros(n_prompts, dtype=np.int64)                 # pages that each prompt has
        self._users = np.zeros(n_pages, dtype=np.int64)                   # prompts that have each page
        self._free = list(range(n_pages - 1, -1, -1))
        return self

    def _owned(self, *prompts: int) -> None:
        if self._count is None:
            raise ValueError("the table of these caches belongs to the caller")
        if not all(0 <= p < self.n_prompts for p in prompts):
            raise IndexError(f"prompts are 0 .. {self.n_prompts - 1}")

    def _write_row(self, prompt: int) -> None:
        self.page_table[prompt].copy_(torch.from_numpy(self._table[prompt].copy()))

    def reserve(self, prompt: int, rows: int) -> None:
        """Pages for rows 0 .. rows - 1 of a prompt, in addition to those it has."""
        self._owned(prompt)
        have, want = int(self._count[prompt]), -(-rows // self.page_size)
        if want > self._table.shape[1]:
            raise ValueError(f"{rows} rows do not fit the prompt's row of the page table")
        if want <= have:
            return
        if want - have > len(self._free):
            raise MemoryError(f"{want - have} pages wanted, {len(self._free)} free")
        pages = [self._free.pop() for _ in range(want - have)]
        self._table[prompt, have:want] = pages
        self._users[pages] = 1
        self._count[prompt] = want
        self._write_row(prompt)

    def share(self, source: int, prompt: int, rows: int) -> int:
        """Gives an empty prompt the pages of `source` that lie wholly within its first `rows` rows. Returns how many rows those
        are; the rows behind them are the prompt's own (append them again)."""
        self._owned(source, prompt)
        n = max(rows, 0) // self.page_size
        if self._count[prompt]:
            raise ValueError("the prompt has pages already")
        if n > self._count[source]:
            raise ValueError("the source does not have that many rows")
        self._table[prompt, :n] = self._table[source, :n]
        self._users[self._table[source, :n]] += 1
        self._count[prompt] = n
        self._write_row(prompt)
        return n * self.page_size

    def release(self, prompt: int) -> None:
        """Gives a prompt's pages back, those at least that no other prompt has."""
        self._owned(prompt)
        pages = self._table[prompt, :self._count[prompt]]
        self._users[pages] -= 1
        self._free.extend(int(p) for p in pages if self._users[p] == 0)
        self._table[prompt] = -1
        self._count[prompt] = 0
        self._write_row(prompt)

    def check_new(self, x: torch.Tensor, rows: int, heads: int, what: str) -> int:
        """The row stride of new rows [rows, heads, D]; slices of a fused projection are welcome. (As few tensor attributes as
        will do: each costs the host a tenth of a microsecond or more, and a step of a few prompts takes the GPU ten.)"""
        if x.dtype is not torch.bfloat16 or x.get_device() != self.index or x.shape != (rows, heads, self.d):
            raise ValueError(f"{what}: a bfloat16 tensor of shape {(rows, heads, self.d)} on {self.device} is wanted")
        s0, s1, s2 = x.stride()
        if s2 != 1 or (s1 != self.d and heads > 1):
            raise ValueError(f"{what}: the heads of a row lie one behind the other")
        if rows <= 1:
            return 0
        if s0 < heads * self.d:
            raise ValueError(f"{what}: every row has memory of its own")
        return s0

    def check_ints(self, x: torch.Tensor, what: str) -> int:
        """The length of a contiguous int32 vector on the pools' device."""
        if x.dtype is not torch.int32 or x.dim() != 1 or x.get_device() != self.index or not x.is_contiguous():
            raise ValueError(f"{what}: a contiguous int32 vector on the pools' device is wanted")
        return x.shape[0]

    def append(self, prompt: torch.Tensor, position: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, rope_base: float,
               rotated: bool = False) -> None:
        """Row r of k_new, v_new [rows, Hkv, D] becomes row position[r] of prompt[r] (int32 tensors on the device; prompt < 0: no
        row), its key rotated by that position unless it is rotated already. On the current stream, asynchronous."""
        rows = self.check_ints(prompt, "prompt")
        if self.check_ints(position, "position") != rows:
            raise ValueError("prompt and position have one length")
        k_stride, v_stride = self.check_new(k_new, rows, self.hkv, "k_new"), self.check_new(v_new, rows, self.hkv, "v_new")
        key = (rope_base, rotated)
        params = self._append_params.get(key)
        if params is None:
            params = B.AttnParams(self.hkv, self.hkv, self.d, rope_base, 0.0, 1, 1, B.PP_FLAG_SKIP_ROPE if rotated else 0)
            self._append_params[key] = params
        with on_device(self.device):
            B.pp_paged_append(params, self.struct, prompt, position, rows, self.n_prompts, k_new, k_stride, v_new, v_stride,
                              self.status, B.current_stream())

    def append_prefill(self, prefill: PrefillBatch, start=0) -> torch.Tensor:
        """UNPACK into pages: the rotated keys and the values of a PrefillBatch that has run, prompt i of the batch into
        prompt i here (`reserve` its rows first). start (int or one int per prompt): rows before it are left as they are, such as
        those in pages from `share`, which other prompts may be reading and which every prompt that has them would write. Returns
        the lengths, int32 on the device."""
        if (prefill.hkv, prefill.d) != (self.hkv, self.d):
            raise ValueError(f"the prefill has {prefill.hkv} KV heads of {prefill.d}, the caches {self.hkv} of {self.d}")
        if prefill.k > self.n_prompts:
            raise ValueError(f"{prefill.k} prompts, {self.n_prompts} rows of the page table")
        room = self.struct.table_stride if self._count is None else self._count[:prefill.k]
        short = np.nonzero(-(-prefill.lengths.astype(np.int64) // self.page_size) > room)[0]
        if len(short):
            raise ValueError(f"prompt {short[0]} has no pages for its {prefill.lengths[short[0]]} rows")
        start = np.broadcast_to(np.asarray(start, dtype=np.int64), (prefill.k,))
        if (start < 0).any() or (start > prefill.lengths).any():
            raise ValueError("start: rows that the prompts have")
        segment = np.full((prefill.pack.n_bins, prefill.pack.capacity), -1, dtype=np.int32)
        position = np.zeros_like(segment)
        for i, n in enumerate(prefill.lengths):
            at = slice(int(prefill.off_of[i]) + int(start[i]), int(prefill.off_of[i]) + int(n))
            segment[prefill.bin_of[i], at] = i
            position[prefill.bin_of[i], at] = np.arange(start[i], n)
        segment, position = (torch.from_numpy(x.reshape(-1)).to(self.device) for x in (segment, position))
        rows = segment.shape[0]
        self.append(segment, position, prefill.kk.view(rows, self.hkv, self.d), prefill.v.view(rows, self.hkv, self.d),
                    prefill.rope_base, rotated=True)
        return torch.from_numpy(prefill.lengths).to(self.device)

    def device_status(self) -> int:
        """What the appends found wrong first (PP_PAGED_*), or 0: waits for them. It stays until `reset_status`."""
        return int(self.status.item())

    def reset_status(self) -> None:
        """On the current stream: appends queued behind it report anew."""
        self.status.zero_()


class _Nothing:
    def __enter__(self):
        return self

    def __exit__(self, *_):
        return False


_NOTHING = _Nothing()


def on_device(device: torch.device):
    """Makes `device` the current one, where it is not (the C ABI launches on the current device)."""
    return _NOTHING if torch._C._cuda_getDevice() == device.index else torch.cuda.device(device)


class PagedDecoder:
    """Generation steps over PagedCaches through pp_paged_decode_step / pp_paged_decode_shared. Owns the workspace (of the steps
    of one stream: steps that may run at the same time want a decoder each) and the status word: to be kept until the steps that
    were queued have run, and as long as a graph that captured some."""

    def __init__(self, caches: PagedCaches, n_q_heads: int, rope_base: float, softmax_scale: float = 0.0):
        self.caches, self.hq = caches, n_q_heads
        self.params = B.AttnParams(n_q_heads, caches.hkv, caches.d, rope_base, softmax_scale, 1, 1, 0)
        self.status = torch.zeros(1, dtype=torch.int32, device=caches.device)
        # Workspaces are kept when a larger one is wanted: a captured graph may go on using them.
        self._workspaces = []
        self._sizes = {}

    def _workspace(self, k: int, n_groups: int):
        """(workspace, its bytes) for these sizes."""
        need = self._sizes.get((k, n_groups))
        if need is None:
            need = B.pp_paged_decode_workspace_bytes(self.params, k, n_groups)
            if need == 0:
                raise ValueError("no generation step for these shapes")
            self._sizes[(k, n_groups)] = need
        if not self._workspaces or self._workspaces[-1][1] < need:
            # (twice the last one at least: all that are kept take no more than the last one again, however the prompts grow in number)
            if self._workspaces:
                need = max(need, 2 * self._workspaces[-1][1])
            self._workspaces.append((torch.empty(need, dtype=torch.uint8, device=self.caches.device), need))
        return self._workspaces[-1]

    def step(self, lengths: torch.Tensor, q: torch.Tensor, k: torch.Tensor | None = None, v: torch.Tensor | None = None,
             out: torch.Tensor | None = None, groups=None) -> torch.Tensor:
        """One token for each prompt of the table's first len(lengths) rows. lengths: int32 on the device, rows that the pages hold
        (< 0: no prompt). q [n, Hq, D]; k, v [n, Hkv, D]: the new token, appended; or None: the pages hold it. groups: (group_ptr,
        shared_len), int32 on the device, where prompts share their first pages. Returns out [n, Hq, D]; on the
        current stream, asynchronous, nothing is read back. The lengths are the caller's to advance. More than 8192 prompts are
        the work of several calls of the library; groups may lie across them, but there are no more groups than prompts of a call."""
        c = self.caches
        n = c.check_ints(lengths, "lengths")
        if not 0 < n <= c.n_prompts:
            raise ValueError("lengths: one for each of at most the table's rows")
        if (k is None) != (v is None):
            raise ValueError("a new token has a key and a value")
        q_stride = c.check_new(q, n, self.hq, "q")
        k_stride = v_stride = 0
        if k is not None:
            k_stride, v_stride = c.check_new(k, n, c.hkv, "k"), c.check_new(v, n, c.hkv, "v")
        if out is None:
            out = torch.zeros((n, self.hq, c.d), dtype=torch.bfloat16, device=c.device)
        elif out.dtype is not torch.bfloat16 or out.shape != (n, self.hq, c.d) or out.get_device() != c.index or not out.is_contiguous():
            raise ValueError("out: a contiguous bfloat16 tensor of q's shape on the pools' device")
        if groups is not None:
            ptr, shared = groups
            n_groups = c.check_ints(shared, "shared_len")
            if c.check_ints(ptr, "group_ptr") != n_groups + 1:
                raise ValueError("groups: group_ptr has one entry more than shared_len")
            if n_groups == 0:
                groups = None
        calls = -(-n // B.PP_PAGED_MAX_PROMPTS)
        if groups is not None and calls > 1:
            least = n - (calls - 1) * -(-n // calls)   # prompts of the last call
            if n_groups > least:
                raise ValueError(f"groups: no more than {least} for {n} prompts")
        with on_device(c.device):
            if calls > 1:
                self._step_in_parts(calls, lengths, n, q, q_stride, k, k_stride, v, v_stride, out, groups)
            elif groups is None:
                ws, size = self._workspace(n, 0)
                B.pp_paged_decode_step(self.params, c.struct, lengths, n, q, q_stride, k, k_stride, v, v_stride, out, ws, size, self.status,
                                       B.current_stream())
            else:
                ws, size = self._workspace(n, n_groups)
                B.pp_paged_decode_shared(self.params, c.struct, lengths, n, ptr, shared, n_groups, q, q_stride, k, k_stride, v, v_stride, out,
                                         ws, size, self.status, B.current_stream())
        return out

    def device_status(self) -> int:
        """What the steps found wrong first (PP_PAGED_*, or a wait that gave up), or 0: waits for them. It stays until `reset_status`."""
        return int(self.status.item())

    def reset_status(self) -> None:
        """On the current stream: steps queued behind it report anew."""
        self.status.zero_()

    def _step_in_parts(self, calls, lengths, n, q, q_stride, k, k_stride, v, v_stride, out, groups) -> None:
        """`step` as so many calls, each for the prompts of a part of the table."""
        c, stream = self.caches, B.current_stream()
        most = -(-n // calls)
        ws, size = self._workspace(most, 0 if groups is None else groups[1].shape[0])
        if groups is not None:
            ptr, shared = groups
            bad = (ptr[1:] < ptr[:-1]).any() | (ptr[0] < 0) | (ptr[-1] > n)     # for all parts, whichever of them would show it
        for a in range(0, n, most):
            b = min(a + most, n)
            part = B.PagedCache.from_buffer_copy(c.struct)
            part.page_table += a * 4 * c.struct.table_stride
            new = (None if x is None else x[a:b] for x in (k, v))
            args = (q[a:b], q_stride, next(new), k_stride, next(new), v_stride, out[a:b], ws, size, self.status, stream)
            if groups is None:
                B.pp_paged_decode_step(self.params, part, lengths[a:b], b - a, *args)
            else:
                B.pp_paged_decode_shared(self.params, part, lengths[a:b], b - a, torch.where(bad, -1, ptr.clamp(a, b) - a), shared,
                                         shared.shape[0], *args)
