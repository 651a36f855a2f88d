"""ctypes binding of include/cryptogen_requests.h: what a model has learned, brought to the encrypted tokens of many requests.

Argument marshalling only, as in binding.py: every method passes data_ptr() values and the current torch stream of the
context's device to the entry point of the same name.
"""
import ctypes as C

import torch

from .binding import _REQUEST_SYMBOLS, CgError, CgSizeError, Context, _need, _params, _raw_stream

# (without the checks for a lazy start, which a live context has behind it: the smallest calls wait for the host)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_I64, _F64, _I32 = torch.int64, torch.float64, torch.int32


def _count(x) -> int:
    """A size as the entry points take it, in 32 bits; anything else is 0, which none of them accepts."""
    x = int(x)
    return x if 0 < x < 1 << 32 else 0


class Requests:
    """The plaintext side of a server: a handle of constant tables beside a Context (whose t must have slots: a prime, 1 mod 2N).

    Its creation synchronises; every other method only enqueues, and can be captured.  Threads may call one handle at once, on
    any streams: every call takes scratch of its own.  Close it before its context."""

    def __init__(self, ctx: Context):
        self.ctx, self.lib = ctx, ctx.lib
        self._index = ctx._device_index
        self.device = torch.device("cuda", self._index)
        self.n, self.k = ctx.n, ctx.k
        self._ct = 2 * self.k * self.n
        self._calls = {name: getattr(self.lib.dll, name) for name in _REQUEST_SYMBOLS}
        self.h = None
        h, prm = C.c_void_p(), _params(ctx.params)
        with torch.cuda.device(self.device):
            ctx._check(self.lib.dll.cg_req_create(C.byref(h), ctx.h, C.byref(prm)))
        self.h = h

    def close(self):
        if getattr(self, "h", None):
            with torch.cuda.device(self.device):
                self.lib.dll.cg_req_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _open(self, name):
        if not self.h or not self.ctx.h:
            raise CgError(f"{name}: the handle or its context is closed")
        return self.h

    def _ask(self, name, *args) -> int:
        """The bytes of scratch that a call needs, which the handle asks its context for."""
        return int(self._calls[name](self._open(name), *args))

    def _call(self, name, *args):
        self._open(name)
        if _current_device() == self._index:
            status = self._calls[name](self.h, _raw_stream(self._index), *args)
        else:
            with torch.cuda.device(self.device):
                status = self._calls[name](self.h, _raw_stream(self._index), *args)
        if status:
            self.ctx._check(status)

    def _at(self, t, dtype, numel: int, what: str) -> int:
        """A tensor's address (0 for None), once it is what the kernels will read or write."""
        if t is None:
            return 0
        if t.get_device() != self._index or t.dtype is not dtype or not t.is_contiguous():
            raise CgSizeError(f"{what}: a contiguous {dtype} tensor on {self.device} is needed, got {t.dtype} on {t.device}"
                              + ("" if t.is_contiguous() else ", strided"))
        if t.numel() < numel:
            _need(t, numel, what)
        return t.data_ptr()

    def _cts(self, t, count, what):
        return self._at(t, _I64, count * self._ct, what)

    def _plains(self, t, count, what):
        return self._at(t, _F64, count * self.k * self.n, what)

    def _empty(self, shape, dtype):
        return torch.empty(shape, dtype=dtype, device=self.device)

    def _workspace(self, need: int) -> torch.Tensor:
        """Scratch of one call, which keeps it until everything is enqueued: the allocator gives the memory to what is enqueued behind, and never
        to a call that another thread makes at the same time on the same stream."""
        return self._empty(need, torch.uint8)

    # ---- slots ----
    def _batch(self, slots):
        """(plaintexts, address)"""
        batch, rest = divmod(slots.numel(), self.n)
        if rest or not batch:
            raise CgSizeError(f"slots: {slots.numel()} values are no whole number of plaintexts of {self.n}")
        return batch, self._at(slots, _I64, 0, "slots")

    def slots_encode(self, slots, out=None):
        """int64 slot values [..., N], any representatives modulo t -> polynomials with coefficients in [0, t)."""
        batch, at = self._batch(slots)
        out = torch.empty_like(slots) if out is None else out
        self._call("cg_slots_encode", at, self._at(out, _I64, batch * self.n, "out"), batch)
        return out

    def slots_prepare(self, slots, out=None):
        """int64 slot values [..., N] -> prepared plaintexts, as plain_prepare makes them of polynomials."""
        batch, at = self._batch(slots)
        out = self._empty(batch * self.k * self.n, _F64) if out is None else out
        self._call("cg_slots_prepare", at, self._plains(out, batch, "out"), batch)
        return out

    # ---- projections ----
    def cpvm_diagonals(self, d1, d2) -> int:
        """Number of diagonals of a d1 x d2 matrix (0: sizes out of range)."""
        return int(self.lib.dll.cg_cpvm_diagonals(self.h, _count(d1), _count(d2)))

    def cpvm_prepare(self, units, d1, d2, w=None, a=None, b=None, a_group=1, out=None):
        """Diagonals of W_u + A_(u // a_group) B_u: w int64 [units][d1][d2], a int64 [ceil(units / a_group)][d1][rank],
        b int64 [units][rank][d2] (w, or a and b, may be left out)."""
        units, d1, d2, a_group, rank = _count(units), _count(d1), _count(d2), _count(a_group), 0
        if (a is None) != (b is None):
            raise CgSizeError("a and b come together")
        if a is not None:
            rank = a.shape[-1]
            if not a_group or a.numel() != -(-units // a_group) * d1 * rank or b.numel() != units * rank * d2:
                raise CgSizeError(f"a {tuple(a.shape)} and b {tuple(b.shape)} do not make {units} matrices of {d1} x {d2}")
        plains = units * self.cpvm_diagonals(d1, d2)
        out = self._empty(plains * self.k * self.n, _F64) if out is None else out
        need = self._ask("cg_cpvm_prepare_workspace_bytes", units, d1, d2, rank)
        ws = self._workspace(need) if need else None
        self._call("cg_cpvm_prepare", self._at(w, _I64, units * d1 * d2, "w"), self._at(a, _I64, 0, "a"), self._at(b, _I64, 0, "b"), units, a_group,
                   d1, d2, rank, self._plains(out, plains, "out"), 0 if ws is None else ws.data_ptr())
        return out

    def cpvm_requests(self, x, diags, requests, units, n_diag, d2, gk_copies, gk_block, adapters=None, pick=None, out=None,
                      block_round_bits=0):
        """y[r][u] = x_r (W_u + the adapter pick[r] asks for), as Context.cpvm_hoisted computes it for one request: adapters
        prepared [n_adapters][units][n_diag] without W, pick int32 [requests] on the GPU (anything else than 0 .. n_adapters - 1:
        none).  In rounds of three bits (block_round_bits=3) it takes about
        half the time it takes generator by generator (0), with more keys."""
        ctx, R, U, D, d2 = self.ctx, _count(requests), _count(units), _count(n_diag), _count(d2)
        out = ctx.empty_ct(R, U) if out is None else out
        ctx._need_keys(list(gk_copies) + list(gk_block))
        if len(gk_copies) != max(0, D - 1):
            raise CgSizeError(f"{D - 1} copy keys needed, {len(gk_copies)} given")
        ctx._need_fold_keys(1, d2, block_round_bits, gk_block)
        n_adapters, per = 0, U * D * self.k * self.n
        if adapters is not None:
            n_adapters = adapters.numel() // max(1, per)
            if not n_adapters or adapters.numel() != n_adapters * per:
                raise CgSizeError(f"adapters: {adapters.numel()} values are no whole number of adapters of {per}")
            if pick is None:
                raise CgSizeError("adapters come with pick")
        args = (self._cts(x, R, "x"), self._plains(diags, U * D, "diags"), self._plains(adapters, 0, "adapters"), n_adapters,
                self._at(pick, _I32, R, "pick") if n_adapters else 0, R, U, D, d2, block_round_bits,
                ctx._keys(gk_copies) if len(gk_copies) else None, ctx._keys(gk_block), self._cts(out, R * U, "out"))
        ws = self._workspace(self._ask("cg_cpvm_requests_workspace_bytes", R, U, D))
        self._call("cg_cpvm_requests", *args, ws.data_ptr())
        return out

    # ---- position biases ----
    def _tables(self, table, edges, heads):
        n = edges.numel()
        return self._at(table, _I64, n * heads, "table"), self._at(edges, _I32, 1, "edges"), n

    def score_bias(self, scores, requests, heads, n_cts, d2, pos, table, edges, out=None):
        """scores [requests][heads][n_cts] + the bias of every token's distance to pos[request]; table int64 [buckets][heads], edges int32
        [buckets] ascending.  out=scores works in place."""
        requests, heads, n_cts = _count(requests), _count(heads), _count(n_cts)
        units = requests * heads * n_cts
        out = torch.empty_like(scores) if out is None else out
        self._call("cg_score_bias", self._cts(scores, units, "scores"), requests, heads, n_cts, _count(d2),
                   self._at(pos, _I32, requests, "pos"), *self._tables(table, edges, heads), self._cts(out, units, "out"))
        return out

    def prompt_bias(self, diagonals, prompts, heads, d2, table, edges, out=None):
        """The same for the diagonals of prefill_qk, [prompts][heads][N / d2]."""
        prompts, heads, d2 = _count(prompts), _count(heads), _count(d2)
        units = prompts * heads * (self.n // max(1, d2))
        out = torch.empty_like(diagonals) if out is None else out
        self._call("cg_prompt_bias", self._cts(diagonals, units, "diagonals"), prompts, heads, d2, *self._tables(table, edges, heads),
                   self._cts(out, units, "out"))
        return out

    # ---- appends ----
    def kv_append_requests(self, cache, cache_stride_cts, requests, per, lens, rows, masks, d2, row_stride_cts=None):
        """Every request's `per` new rows into its caches at its own length: cache [requests][per][cache_stride_cts], lens int32
        [requests] on the GPU (below 0, or a full cache: left as it is), rows [requests][row_stride_cts or per]."""
        R, P, stride, d2 = _count(requests), _count(per), _count(cache_stride_cts), _count(d2)
        gap = P if row_stride_cts is None else _count(row_stride_cts)
        self._call("cg_kv_append_requests", self._cts(cache, R * P * stride, "cache"), stride, R, P,
                   self._at(lens, _I32, R, "lens"), self._cts(rows, max(0, R - 1) * gap + P, "rows"), gap,
                   self._plains(masks, self.n // max(1, d2), "masks"), d2)
