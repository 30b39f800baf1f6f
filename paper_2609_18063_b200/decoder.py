"""The expert stack: one token through L MoE layers with prediction-driven staging; and whole decoder blocks, with
latent attention over a paged cache in front of each layer-step.

A thin owner of the buffers around ``edg_stack_decode_token`` -- the per-token host loop itself (wait
for the mirrored routing, stage, enqueue the L layer-steps) runs inside the C library.  Per token
it does what the paper's decode timeline shows: the routing of every layer was predicted one token
earlier (the head owned by layer l, evaluated on that layer's input at token t, predicts layer
(l+1) mod L at token t+1); the kernels mirror it into pinned host memory, so the single hand-off of
a token needs neither a device-to-host copy nor a stream synchronisation; the stager enqueues the
copies of the missing experts on the side stream, and each layer's kernel waits only for its own
layer's copies, so later layers' copies overlap earlier layers' compute.
"""
from __future__ import annotations

import time

import torch

from . import binding as B
from . import layer_io


class StackDecoder:
    def __init__(self, desc: B.LayerDesc, store: B.Store, W_pre: torch.Tensor, prefetch: bool = True):
        """W_pre: device [L][E][H]; head l predicts the routing of layer (l+1) % L at the next token."""
        self.desc, self.store, self.W_pre, self.prefetch = desc, store, W_pre, prefetch
        self.L = store.n_layers
        K = desc.K
        self.inds = torch.zeros((2, self.L, K), dtype=torch.int32, device="cuda")
        self.gates = torch.zeros((2, self.L, K), dtype=torch.float32, device="cuda")
        # host mirrors of the two routing buffers, written by the kernels themselves (-1 = not yet)
        self.mirror = torch.full((2, self.L, K), -1, dtype=torch.int32).pin_memory()
        self.ws = layer_io.new_workspace(desc)
        self.misses = 0

    def prime(self, x_prompt: torch.Tensor) -> None:
        """Routing of token 0 from the last prompt token's layer inputs [L][H] (prefill has no
        prediction; one batched flush over all heads)."""
        L = self.L
        tmp_i = torch.zeros((L, self.desc.K), dtype=torch.int32, device="cuda")
        tmp_g = torch.zeros((L, self.desc.K), dtype=torch.float32, device="cuda")
        B.prerouter_topk(self.desc, self.W_pre, x_prompt, L, tmp_i, tmp_g, None)
        # head l feeds layer (l+1) % L
        self.inds[0] = torch.roll(tmp_i, 1, dims=0)
        self.gates[0] = torch.roll(tmp_g, 1, dims=0)
        self.mirror[0].copy_(self.inds[0])
        torch.cuda.current_stream().synchronize()

    def step(self, t: int, X: torch.Tensor, Y: torch.Tensor, logits_out=None) -> None:
        """Token t: X device bf16 [L][H] (layer inputs), Y device [L][H] (layer outputs)."""
        cur, nxt = t % 2, (t + 1) % 2
        self.misses += B.stack_decode_token(self.store, X, self.inds[cur], self.gates[cur], self.W_pre,
                                            self.inds[nxt], self.gates[nxt], logits_out, self.mirror[cur],
                                            self.mirror[nxt], Y, self.ws, prefetch=self.prefetch)


_TYPES = {B.F32: torch.float32, B.F16: torch.float16, B.BF16: torch.bfloat16}


def _refuse(bad: bool, what: str) -> None:
    if bad:
        raise ValueError(what)


def _is(t, shape, dtype, device) -> bool:
    """Whether t is a tensor like that (an address says nothing about itself: taken as given)."""
    return not isinstance(t, torch.Tensor) or (tuple(t.shape) == tuple(shape) and t.dtype == dtype and t.device == device)


class LatentCache:
    """Latent rows of all layers in pages, and which pages a request holds (device state, ``edg.pages_*``).  Lists are int32 tensors on the cache's
    device, those of one call of one length; anything else is a ValueError."""

    def __init__(self, layers: int, n_pages: int, page: int, row: int, n_seqs: int, max_pages: int, device="cuda"):
        """row: d_latent + d_rope values of bf16."""
        self.rows = torch.zeros((layers, n_pages, page, row), dtype=torch.bfloat16, device=device)
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device=device)
        self.table = torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(n_seqs, dtype=torch.int32, device=device)
        self.pool = B.make_page_pool(self.refs, self.table, self.lens, page=page)
        self.pages = B.make_page_cache(self.rows)
        self.ws = torch.zeros(B.pages_workspace_bytes(self.pool), dtype=torch.uint8, device=device)

    def _lists(self, *lists: torch.Tensor) -> None:
        for v in lists:
            _refuse(v.dtype != torch.int32 or v.device != self.lens.device or v.numel() != lists[0].numel(), "lists are int32 [n] on the cache's device")

    def reserve(self, seqs: torch.Tensor, counts: torch.Tensor) -> None:
        """Grows sequences.  A list that the pool cannot serve, or a sequence that has no room, keeps its lens and is told by status() alone: what
        appends rows afterwards takes the last positions for the new ones.  Look before it does."""
        self._lists(seqs, counts)
        B.pages_reserve(self.pool, self.pages, seqs.numel(), seqs, counts, self.ws)

    def fork(self, parents: torch.Tensor, children: torch.Tensor) -> None:
        self._lists(parents, children)
        B.pages_fork(self.pool, parents.numel(), parents, children, self.ws)

    def free(self, seqs: torch.Tensor) -> None:
        self._lists(seqs)
        B.pages_free(self.pool, seqs.numel(), seqs, self.ws)

    def compact(self) -> None:
        B.pages_compact(self.pool, self.pages, self.ws)

    def status(self) -> int:
        return B.workspace_status(self.ws)


class LatentBlock:
    """The attention half of one decoder layer: int4 projections of the hidden state to queries and latent rows, latent attention over the
    request's pages, int4 output projection.  Serves single tokens, batches of requests and prompts alike.

    ``w_q``, ``w_kv``, ``w_out``: (LinearDesc, device record) with N = heads * (d_nope + d_rope), d_latent + d_rope and H; ``w_uk`` / ``w_uv`` device
    bf16 [heads][d_nope][d_latent] / [heads][d_v][d_latent]; ``gain`` device bf16 [d_latent] or None; ``inv_freq`` device f32 [d_rope / 2].
    Adapters: an optional (A, B) behind the record.  Rows of all of them are dense.  What one call writes and the next reads is bf16: the outputs of
    ``w_q`` and ``w_kv``, and ``desc``'s; ``w_out`` writes any type.  Anything else is a ValueError."""

    def __init__(self, desc: B.LatentDesc, w_q, w_kv, w_out, w_uk, w_uv, gain, inv_freq, max_rows: int, max_seqs: int, max_new: int, max_total: int):
        self.desc, self.w_q, self.w_kv, self.w_out = desc, w_q, w_kv, w_out
        self.w_uk, self.w_uv, self.gain, self.inv_freq = w_uk, w_uv, gain, inv_freq
        h, dev, bf16 = desc.heads, w_uk.device, torch.bfloat16
        d_q, d_kv, H = h * (desc.d_nope + desc.d_rope), desc.d_latent + desc.d_rope, w_q[0].Kd
        _refuse(desc.out_dtype != B.BF16, "the output projection reads bf16: out_dtype of the attention must be bf16")
        _refuse(desc.ldq not in (0, d_q) or desc.ldkv not in (0, d_kv), "a block's queries and rows lie dense")
        for name, w, N, Kd, out in (("w_q", w_q, d_q, H, B.BF16), ("w_kv", w_kv, d_kv, H, B.BF16), ("w_out", w_out, H, h * desc.d_v, None)):
            d = w[0]
            _refuse((d.N, d.Kd) != (N, Kd), f"{name} is {d.N} x {d.Kd}, the block needs {N} x {Kd}")
            _refuse(out is not None and d.out_dtype != out, f"{name} must write bf16")
            _refuse(d.ldx not in (0, Kd) or d.ldy not in (0, N), f"{name}: a block's rows lie dense")
            _refuse(isinstance(w[1], torch.Tensor) and (w[1].device != dev or w[1].nbytes < B.linear_record_bytes(d)), f"{name}: not a record of this projection")
            _refuse(len(w) not in (2, 4) or (d.rank > 0) != (len(w) == 4), f"{name}: an adapter where the rank is not 0, and none elsewhere")
            _refuse(len(w) == 4 and not (_is(w[2], (d.rank, Kd), bf16, dev) and _is(w[3], (N, d.rank), bf16, dev)), f"{name}: A [rank][Kd] and B [N][rank] in bf16")
        _refuse(not _is(w_uk, (h, desc.d_nope, desc.d_latent), bf16, dev) or not _is(w_uv, (h, desc.d_v, desc.d_latent), bf16, dev), "w_uk and w_uv")
        _refuse(gain is not None and not _is(gain, (desc.d_latent,), bf16, dev), "gain")
        _refuse(not _is(inv_freq, (desc.d_rope // 2,), torch.float32, dev), "inv_freq")
        self.q = torch.empty((max_rows, h * (desc.d_nope + desc.d_rope)), dtype=torch.bfloat16, device=dev)
        self.kv = torch.empty((max_rows, desc.d_latent + desc.d_rope), dtype=torch.bfloat16, device=dev)
        self.q_rope = torch.empty((max_rows, h, desc.d_rope), dtype=torch.bfloat16, device=dev)
        self.a = torch.empty((max_rows, h * desc.d_v), dtype=torch.bfloat16, device=dev)
        self.bounds = (max_seqs, max_rows, max_new, max_total)
        self.ws = torch.zeros(B.latent_workspace_bytes(desc, *self.bounds), dtype=torch.uint8, device=dev)
        need = max(B.linear_workspace_bytes(w[0], max_rows) for w in (w_q, w_kv, w_out))
        self.ws_linear = torch.empty(need, dtype=torch.uint8, device=dev)

    def _project(self, w, T, x, y):
        A, Bm = (w[2], w[3]) if len(w) > 2 else (None, None)
        B.linear_int4_lora(w[0], w[1], T, x, A, Bm, y, self.ws_linear)

    def run(self, x, y, cu, lens, table, rows, max_new=1, total=None, eps=1e-6) -> None:
        """x device bf16 [T][H] (the new rows of n = cu.numel() - 1 sequences, whose places in the cache are reserved), y device [T][H] of
        ``w_out``'s type; cu, lens and table (int32) are those of the same n sequences, rows the layer's part of the cache; max_new bounds the new
        rows of a sequence, total the sum of lens.  What exceeds the block's own bounds, or does not fit it, is a ValueError, and nothing is launched."""
        n, T, d = cu.numel() - 1, x.shape[0], self.desc
        total = self.bounds[3] if total is None else total
        out, dev, i32 = self.w_out[0], self.w_uk.device, torch.int32
        if not (1 <= n <= self.bounds[0] and 1 <= T <= self.bounds[1] and 1 <= max_new <= min(self.bounds[2], T) and 0 <= total <= self.bounds[3]):
            raise ValueError(f"{n} sequences, {T} rows, {max_new} of one sequence, {total} positions: the block is made for {self.bounds}")
        if not _is(x, (T, self.w_q[0].Kd), torch.bfloat16, dev) or y.numel() != T * out.N or y.dtype != _TYPES[out.out_dtype] or y.device != dev:
            raise ValueError("x is bf16 [T][H], y [T][H] of the output projection's type")
        if not (cu.dtype == lens.dtype == table.dtype == i32 and cu.device == lens.device == table.device == dev and lens.numel() >= n
                and table.dim() == 2 and table.shape[0] >= n and table.shape[1] == d.max_pages):
            raise ValueError("cu, lens and table are int32 [n + 1], [n] and [n][max_pages]")
        if not _is(rows, (d.n_pages, d.page, d.d_latent + d.d_rope), torch.bfloat16, dev):
            raise ValueError("rows are the layer's bf16 [n_pages][page][d_latent + d_rope]")
        if not (x.is_contiguous() and y.is_contiguous() and cu.is_contiguous() and lens.is_contiguous() and table.is_contiguous() and rows.is_contiguous()):
            raise ValueError("tensors must be contiguous")
        self._project(self.w_q, T, x, self.q)
        self._project(self.w_kv, T, x, self.kv)
        B.latent_append(self.desc, n, T, cu, lens, table, self.kv, self.gain, eps, self.inv_freq, self.q, self.q_rope, rows, self.ws)
        B.latent_attention(self.desc, n, T, max_new, total, cu, lens, table, self.q, self.q_rope, self.w_uk, self.w_uv, rows, self.a, self.ws)
        self._project(self.w_out, T, self.a, y)


class BlockDecoder(StackDecoder):
    """A request through a stack of whole decoder blocks: the attention half (:class:`LatentBlock`) in front of every MoE layer-step, the
    hidden state handed on as bf16(rmsnorm(x + y)) behind each of the two.  Routing is predicted as in :class:`StackDecoder`: the head owned by
    layer l, evaluated on that layer-step's input at token t, predicts layer (l + 1) % L at token t + 1."""

    def __init__(self, desc: B.LayerDesc, store: B.Store, W_pre: torch.Tensor, blocks, cache: LatentCache, seq: int = 0):
        super().__init__(desc, store, W_pre)
        if len(blocks) != self.L or cache.rows.shape[0] != self.L:
            raise ValueError("one attention block and one layer of the cache per layer of the store")
        for b in blocks:
            d, out = b.desc, b.w_out[0]
            _refuse((out.N, out.out_dtype) != (desc.H, desc.out_dtype), "a block's output projection writes [H] of the layer's out_dtype")
            _refuse(tuple(cache.rows.shape[1:]) != (d.n_pages, d.page, d.d_latent + d.d_rope) or cache.table.shape[1] != d.max_pages, "a block's cache is another")
            _refuse(b.w_uk.device != cache.rows.device, "blocks and cache lie on one device")
        _refuse(not 0 <= seq < cache.lens.shape[0], "seq is a row of the cache's table")
        self.blocks, self.cache = blocks, cache
        dev = W_pre.device
        self._seq = torch.tensor([seq], dtype=torch.int32, device=dev)
        self._one = torch.ones(1, dtype=torch.int32, device=dev)
        self._cu = torch.tensor([0, 1], dtype=torch.int32, device=dev)
        self._lens, self._table = cache.lens[seq:seq + 1], cache.table[seq:seq + 1]
        dt = _TYPES[desc.out_dtype]
        self.o = torch.empty(desc.H, dtype=dt, device=dev)              # attention output, of the type that the next state is made from
        self.y = torch.empty((self.L, desc.H), dtype=dt, device=dev)
        self.x_moe = torch.empty((self.L, desc.H), dtype=torch.bfloat16, device=dev)
        self.x_out = torch.empty((self.L, desc.H), dtype=torch.bfloat16, device=dev)
        self._most = min(b.bounds[3] for b in blocks)                   # positions that the blocks are made for, and that the cache can hold
        self._capacity = cache.table.shape[1] * cache.rows.shape[2]
        self._grow_ws = torch.zeros_like(cache.ws)                      # its status word tells of this request's growth alone

    def _grow(self) -> None:
        """One more position, or an error with nothing of the token enqueued.  (Whether there is a page is the device's to say: this waits for its
        answer, and so for the last layer of the token before: some 30 us a token.)"""
        if self._most < self._capacity and int(self._lens) >= self._most:
            raise B.EdgError(-4, "BlockDecoder.token")
        B.pages_reserve(self.cache.pool, self.cache.pages, 1, self._seq, self._one, self._grow_ws)
        code = B.workspace_status(self._grow_ws)
        if code != 0:
            self._grow_ws[:4].zero_()
            raise B.EdgError(code, "BlockDecoder.token")

    def token(self, t: int, x: torch.Tensor, timeout_s: float = 5.0) -> torch.Tensor:
        """Token t: x device bf16 [H], the first block's input; returns the last block's output (a view that the next token overwrites).  Where the
        pool has no page for the token EdgError -3 is raised, where the sequence is full or the blocks' bound is reached -4: nothing has been
        changed then, and the token can be asked for again when pages are free."""
        _refuse(x.numel() != self.desc.H or x.dtype != torch.bfloat16 or x.device != self.o.device or not x.is_contiguous(), "x is bf16 [H]")
        cur, nxt = t % 2, (t + 1) % 2
        mirror, end = self.mirror[cur].numpy(), time.monotonic() + timeout_s
        while (mirror < 0).any():                                       # written by the heads of the token before
            if time.monotonic() > end:
                raise B.EdgError(-6, "BlockDecoder.token")
        self._grow()
        self.mirror[nxt].fill_(-1)
        for l in range(self.L):
            self.misses += B.stage_experts_to_slots(self.store, l, mirror[l])[1]
        for l, block in enumerate(self.blocks):
            block.run(x.view(1, -1), self.o, self._cu, self._lens, self._table, self.cache.rows[l])
            B.next_hidden_state(self.desc, x, self.o, self.x_moe[l])
            nl = (l + 1) % self.L
            B.moe_layer_decode_dependent(self.store, l, self.x_moe[l], self.inds[cur][l], self.gates[cur][l], self.W_pre[l], self.inds[nxt][nl],
                                         self.gates[nxt][nl], None, self.y[l], self.x_out[l], self.ws, inds_next_host_mirror_opt=self.mirror[nxt][nl])
            x = self.x_out[l]
        return x
