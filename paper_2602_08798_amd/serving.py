"""ctypes binding of include/cryptogen_requests.h: what a model has learned, brought to the encrypted tokens of many requests.

Argument marshalling only, as in binding.py: every method passes data_ptr() values and the current torch stream of the
context's device to the entry point of the same name.
"""
import ctypes as C

import torch

from .binding import CgSizeError, Context, _need, _params, _ptr


def _ints(t, dtype, numel: int, what: str) -> int:
    """A small integer array that the kernels read: its address (0 for None)."""
    if t is None:
        return 0
    if not (t.is_cuda and t.is_contiguous() and t.dtype == dtype):
        raise CgSizeError(f"{what}: a contiguous {dtype} tensor on the GPU is needed, got {t.dtype}")
    _need(t, numel, what)
    return t.data_ptr()


class Requests:
    """The plaintext side of a server: a handle of constant tables beside a Context (whose t must have slots: a prime, 1 mod 2N)."""

    def __init__(self, ctx: Context):
        self.ctx, self.lib = ctx, ctx.lib
        self.n, self.k = ctx.n, ctx.k
        self._ws = {}
        h, prm = C.c_void_p(), _params(ctx.params)
        with torch.cuda.device(ctx.device):
            ctx._check(self.lib.dll.cg_req_create(C.byref(h), ctx.h, C.byref(prm)))
        self.h = h

    def close(self):
        if getattr(self, "h", None):
            self.lib.dll.cg_req_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _call(self, name, *args):
        f = getattr(self.lib.dll, name)
        if torch.cuda.current_device() == self.ctx._device_index:
            self.ctx._check(f(self.h, self.ctx.stream, *args))
        else:
            with torch.cuda.device(self.ctx._device_index):
                self.ctx._check(f(self.h, self.ctx.stream, *args))

    def _workspace(self, need: int) -> torch.Tensor:
        """Scratch that is the current stream's alone.  A captured call has its own, from the graph's pool: what an eager call keeps
        may be replaced by a larger one while the graph lives."""
        if torch.cuda.is_current_stream_capturing():
            return torch.empty(need, dtype=torch.uint8, device=self.ctx.device)
        key = self.ctx.stream
        ws = self._ws.get(key)
        if ws is None or ws.numel() < need:
            self._ws.pop(key, None)
            ws = self._ws[key] = torch.empty(need, dtype=torch.uint8, device=self.ctx.device)
        return ws

    def _rows(self, count: int) -> int:
        return max(0, int(count)) * self.n

    def _empty(self, numel, dtype):
        return torch.empty(numel, dtype=dtype, device=self.ctx.device)

    # ---- slots ----
    def _batch(self, slots):
        if slots.numel() % self.n or not slots.numel():
            raise CgSizeError(f"slots: {slots.numel()} values are no whole number of plaintexts of {self.n}")
        return slots.numel() // self.n

    def slots_encode(self, slots, out=None):
        """int64 slot values [..., N], any representatives in (-2^31, 2^31) -> polynomials with coefficients in [0, t)."""
        batch = self._batch(slots)
        out = self._empty(slots.shape, torch.int64) if out is None else out
        _need(out, slots.numel(), "out")
        self._call("cg_slots_encode", _ints(slots, torch.int64, 0, "slots"), _ptr(out), batch)
        return out

    def slots_prepare(self, slots, out=None):
        """int64 slot values [batch][N] -> prepared plaintexts, as plain_prepare makes them of polynomials."""
        batch = self._batch(slots)
        out = self._empty(self._rows(batch * self.k), torch.float64) if out is None else out
        _need(out, self._rows(batch * self.k), "out (prepared)")
        self._call("cg_slots_prepare", _ints(slots, torch.int64, 0, "slots"), _ptr(out), batch)
        return out

    # ---- projections ----
    def cpvm_diagonals(self, d1, d2) -> int:
        """Number of diagonals of a d1 x d2 matrix (0: sizes out of range)."""
        return int(self.lib.dll.cg_cpvm_diagonals(self.h, d1, d2))

    def cpvm_prepare(self, units, d1, d2, w=None, a=None, b=None, a_group=1, out=None):
        """Diagonals of W_u + A_(u // a_group) B_u: w int64 [units][d1][d2], a int64 [ceil(units / a_group)][d1][rank],
        b int64 [units][rank][d2] (w, or a and b, may be left out)."""
        rank = 0
        if (a is None) != (b is None):
            raise CgSizeError("a and b come together")
        if a is not None:
            per = int(a_group) and -(-int(units) // int(a_group))
            rank = a.numel() // max(1, per * int(d1))
            if a.shape[-1] != rank or a.numel() != per * int(d1) * rank or b.numel() != int(units) * rank * int(d2):
                raise CgSizeError(f"a {tuple(a.shape)} and b {tuple(b.shape)} do not make {units} matrices of {d1} x {d2}")
        rows = self._rows(int(units) * self.cpvm_diagonals(d1, d2) * self.k)
        out = self._empty(rows, torch.float64) if out is None else out
        _need(out, rows, "out (prepared)")
        need = int(self.lib.dll.cg_cpvm_prepare_workspace_bytes(self.h, units, d1, d2, rank))
        ws = self._workspace(need) if need else None
        self._call("cg_cpvm_prepare", _ints(w, torch.int64, int(units) * int(d1) * int(d2), "w"), _ints(a, torch.int64, 0, "a"),
                   _ints(b, torch.int64, 0, "b"), units, a_group, d1, d2, rank, _ptr(out), _ptr(ws))
        return out

    def cpvm_requests(self, x, diags, requests, units, n_diag, d2, gk_copies, gk_block, adapters=None, pick=None, out=None,
                      block_round_bits=0):
        """y[r][u] = x_r (W_u + the adapter pick[r] asks for), as Context.cpvm_hoisted computes it for one request: adapters
        prepared [n_adapters][units][n_diag] without W, pick int32 [requests] on the GPU (anything else than 0 .. n_adapters - 1:
        none)."""
        ctx, R, U = self.ctx, max(0, int(requests)), max(0, int(units))
        per = self._rows(U * max(0, int(n_diag)) * self.k)
        out = ctx.empty_ct(R, U) if out is None else out
        _need(x, ctx._cts(R), "x")
        _need(diags, per, "diags (prepared)")
        _need(out, ctx._cts(R * U), "out")
        ctx._need_keys(list(gk_copies) + list(gk_block))
        if len(gk_copies) != max(0, int(n_diag) - 1):
            raise CgSizeError(f"{int(n_diag) - 1} copy keys needed, {len(gk_copies)} given")
        ctx._need_fold_keys(1, d2, block_round_bits, gk_block)
        n_adapters = 0
        if adapters is not None:
            n_adapters = adapters.numel() // max(1, per)
            if not n_adapters or adapters.numel() != n_adapters * per:
                raise CgSizeError(f"adapters: {adapters.numel()} values are no whole number of adapters of {per}")
            if pick is None:
                raise CgSizeError("adapters come with pick")
        ws = self._workspace(int(self.lib.dll.cg_cpvm_requests_workspace_bytes(self.h, R, U, n_diag)))
        self._call("cg_cpvm_requests", _ptr(x), _ptr(diags), _ptr(adapters), n_adapters,
                   _ints(pick, torch.int32, R, "pick") if n_adapters else 0, requests, units, n_diag, d2, block_round_bits,
                   ctx._keys(gk_copies) if len(gk_copies) else None, ctx._keys(gk_block), _ptr(out), _ptr(ws))
        return out

    # ---- position biases ----
    def _bias_tables(self, table, edges, heads):
        n = edges.numel()
        return (_ints(table, torch.int64, n * max(0, int(heads)), "table"), _ints(edges, torch.int32, 1, "edges"), n)

    def score_bias(self, scores, requests, heads, n_cts, d2, pos, table, edges, out=None):
        """scores [requests][heads][n_cts] + the bias of every token's distance to pos[request]; table int64 [buckets][heads], edges int32
        [buckets] ascending.  out=scores works in place."""
        cts = self.ctx._cts(max(0, int(requests)) * max(0, int(heads)) * max(0, int(n_cts)))
        out = torch.empty_like(scores) if out is None else out
        _need(scores, cts, "scores")
        _need(out, cts, "out")
        self._call("cg_score_bias", _ptr(scores), requests, heads, n_cts, d2, _ints(pos, torch.int32, max(0, int(requests)), "pos"),
                   *self._bias_tables(table, edges, heads), _ptr(out))
        return out

    def prompt_bias(self, diagonals, prompts, heads, d2, table, edges, out=None):
        """The same for the diagonals of prefill_qk, [prompts][heads][N / d2]."""
        cts = self.ctx._cts(max(0, int(prompts)) * max(0, int(heads)) * (self.n // max(1, int(d2))))
        out = torch.empty_like(diagonals) if out is None else out
        _need(diagonals, cts, "diagonals")
        _need(out, cts, "out")
        self._call("cg_prompt_bias", _ptr(diagonals), prompts, heads, d2, *self._bias_tables(table, edges, heads), _ptr(out))
        return out

    # ---- appends ----
    def kv_append_requests(self, cache, cache_stride_cts, requests, per, lens, rows, masks, d2, row_stride_cts=None):
        """Every request's `per` new rows into its caches at its own length: cache [requests][per][cache_stride_cts], lens int32
        [requests] on the GPU (below 0, or a full cache: left as it is), rows [requests][row_stride_cts or per]."""
        ctx, R, caches = self.ctx, max(0, int(requests)), max(0, int(requests)) * max(0, int(per))
        row_stride_cts = per if row_stride_cts is None else row_stride_cts
        _need(cache, ctx._cts(caches * max(0, int(cache_stride_cts))), "cache")
        _need(rows, ctx._cts(max(0, R - 1) * int(row_stride_cts) + max(0, int(per))), "rows")
        _need(masks, self._rows(self.n // max(1, int(d2)) * self.k), "masks (prepared)")
        self._call("cg_kv_append_requests", _ptr(cache), cache_stride_cts, requests, per, _ints(lens, torch.int32, R, "lens"), _ptr(rows),
                   row_stride_cts, _ptr(masks), d2)
