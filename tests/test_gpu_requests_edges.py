"""Calls at the edges of what the requests' header allows."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from tests.test_gpu_requests import _env, _ints, _matrices, say


@pytest.mark.parametrize("group", [4, (1 << 31) - 1, 1 << 31, (1 << 32) - 3, (1 << 32) - 1])
def test_one_matrix_for_all_units(group):
    """A number of units that share A beyond all there are, up to the largest the call takes, means: one A."""
    import torch
    env = _env("C1")
    units, d1, d2 = 3, 100, 64
    say(f"cpvm_prepare: {units} units, a_group {group}")
    w, a, b = (_ints(x) for x in _matrices(np.random.default_rng(4), units, d1, d2, 5, units, True))
    got = env.rq.cpvm_prepare(units, d1, d2, w, a, b, a_group=group)
    assert torch.equal(got, env.rq.cpvm_prepare(units, d1, d2, w, a, b, a_group=units))


def _signs(n, kind):
    return {"plus": np.ones(n), "minus": -np.ones(n), "alternating": 1.0 - 2 * (np.arange(n) % 2), "halves": np.where(np.arange(n) < n // 2, 1.0, -1.0)}[kind]


@pytest.mark.parametrize("name,n_diag", [("C1", 1), ("C1", 2), ("C1", 4), ("C1", 8), ("C1", 32), ("C2", 8), ("C2", 16), ("C5", 4)])
def test_sums_of_the_largest_products(name, n_diag):
    """Base and adapter diagonals of (q - 1) / 2 in size at every point, in one sign and in several, times tokens whose transforms have that size
    everywhere too: a sum of products opened, closed and opened again never gets larger."""
    import torch
    from oracle import attention, bfv
    env = _env(name)
    n, k, d2, q = env.n, env.k, 64, [int(m) for m in env.prm.q]
    half = np.array([(m - 1) // 2 for m in q], dtype=np.int64)
    gens = attention.block_generators(n, d2)
    keys = {g: env.key(900 + i) for i, g in enumerate(dict.fromkeys(g for r in attention.round_galois(n, gens, 3) for g in r))}
    block, raw = [keys[g][1] for r in attention.round_galois(n, gens, 3) for g in r], {g: x[0] for g, x in keys.items()}
    nothing = env.ctx.ksk_prepare(torch.zeros(env.prm.dnum, 2, env.ctx.L, n, dtype=torch.int64, device="cuda"))
    for token, base, plus in (("plus", "plus", "plus"), ("minus", "plus", "plus"), ("plus", "minus", "minus"), ("plus", "alternating", "alternating"),
                              ("minus", "halves", "alternating")):
        say(f"{name}: {n_diag} diagonals, token {token}, base {base}, adapter {plus}")
        # a constant has the same value at every point, and is every copy's component 0 (keys of 0 leave component 1 empty)
        x = np.zeros((1, 2, k, n), dtype=np.uint64)
        x[..., 0] = half if token == "plus" else np.array(q) - half
        w, e = (torch.as_tensor(np.broadcast_to(_signs(n, s) * half[:, None], (1, n_diag, k, n)).copy(), device="cuda") for s in (base, plus))
        got = env.host(env.rq.cpvm_requests(env.dev(x), w.view(-1), 1, 1, n_diag, d2, [nothing] * (n_diag - 1), block, adapters=e.view(-1),
                                            pick=_ints([0], torch.int32), block_round_bits=3))[0, 0]
        y = np.zeros((2, k, n), dtype=np.uint64)
        both = (_signs(n, base) + _signs(n, plus)).astype(np.int64)
        for i, m in enumerate(q):
            value = int(half[i]) * (1 if token == "plus" else -1) * int(half[i])
            for h, times in ((0, n_diag), (1, 1)):
                y[h, i] = bfv.ntt_inverse(np.array([value * int(s) * times % m for s in both], dtype=np.uint64), m)
        assert np.array_equal(got, attention.fold_by_rounds(env.orc, y, gens, raw, 3)), (token, base, plus)


@pytest.mark.parametrize("name", ["C1", "C2", "C5"])
def test_appends_of_the_largest_products(name):
    """Rows at the extremes of the residues, masks of (q - 1) / 2 in size at every point, caches of q - 1."""
    import torch
    from oracle import bfv
    from tests.test_gpu_extreme_values import patterns
    env = _env(name)
    n, k, d2, q = env.n, env.k, env.n // 2, [int(m) for m in env.prm.q]
    rows = patterns(q, n, (2,))
    lens = [1] * len(rows)                               # the second of two blocks: added to what is there
    half = np.array([(m - 1) // 2 for m in q], dtype=np.int64)
    old = np.broadcast_to(np.array(q, dtype=np.uint64)[:, None] - 1, (len(rows), 1, 1, 2, k, n)).copy()
    x = np.stack(list(rows.values()))
    points = np.array([[[bfv.ntt_forward(x[r, c, i], m) for i, m in enumerate(q)] for c in range(2)] for r in range(len(rows))])
    for kind in ("plus", "minus", "alternating"):
        say(f"{name}: masks {kind}")
        masks = torch.as_tensor(np.broadcast_to(_signs(n, kind) * half[:, None], (2, k, n)).copy(), device="cuda").view(-1)
        cache = env.dev(old)
        env.rq.kv_append_requests(cache, 1, len(rows), 1, _ints(lens, torch.int32), env.dev(x), masks, d2)
        got = env.host(cache)
        sign = _signs(n, kind).astype(np.int64)
        for r, what in enumerate(rows):
            for c in range(2):
                for i, m in enumerate(q):
                    v = np.array([int(p) * int(half[i]) * int(s) % m for p, s in zip(points[r, c, i], sign)], dtype=np.uint64)
                    want = (bfv.ntt_inverse(v, m).astype(object) + (m - 1)) % m
                    assert np.array_equal(got[r, 0, 0, c, i].astype(object), want), (what, kind, c, i)
