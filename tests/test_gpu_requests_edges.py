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


@pytest.mark.parametrize("log2n,tops", [(12, (50, 41)), (13, (41, 41, 50)), (14, (41, 50))])
def test_primes_of_different_sizes(log2n, tops):
    """Ciphertext primes just above 2^40 beside ones just below 2^50: bounds that are stated for the largest hold for the smallest too."""
    import torch
    import paper_2602_08798_amd as P
    from oracle import Oracle, attention
    from oracle.client import SlotCodec, galois_rot
    from tests.bruteforce import ntt_primes
    from workloads import Stream, pseudo_ciphertexts, pseudo_switch_key
    from workloads.params import ParamSet
    n = 1 << log2n
    pool = {41: ntt_primes(1 << 41, 2 * n, 4), 50: ntt_primes(1 << 50, 2 * n, 4)}
    q, p = tuple(pool[top].pop(0) for top in tops), (pool[50].pop(0),)
    prm = ParamSet("x", log2n, q=q, p=p)
    ctx, orc, codec, k = P.Context(prm), Oracle(prm), SlotCodec(prm), len(q)
    rq, dev, d2 = P.Requests(ctx), P.to_device, 64
    rng = np.random.default_rng(log2n)
    say(f"N = {n}: primes of {tops} bits")
    v = rng.integers(-128, 128, (9, n))
    v[0], v[1] = (prm.t - 1) // 2, -((prm.t - 1) // 2)
    polys = np.stack([codec.encode(x) for x in v])
    assert torch.equal(rq.slots_prepare(_ints(v)), ctx.plain_prepare(dev(polys)))
    x = pseudo_ciphertexts(Stream(5, 1), q, n, 2)
    x[0] = np.array(q, dtype=np.uint64)[:, None] - 1
    gens = attention.block_generators(n, d2)
    rounds = [g for r in attention.round_galois(n, gens, 3) for g in r]
    raw = {g: pseudo_switch_key(Stream(6, g), list(q) + list(p), n, prm.dnum) for g in dict.fromkeys([galois_rot(n, 1)] + rounds)}
    keys = {g: ctx.ksk_prepare(dev(r)) for g, r in raw.items()}
    diags, low = ctx.plain_prepare(dev(polys[:2])), ctx.plain_prepare(dev(polys[2:4]))
    got = P.to_host(rq.cpvm_requests(dev(x), diags, 2, 1, 2, d2, [keys[galois_rot(n, 1)]], [keys[g] for g in rounds], adapters=low,
                                     pick=_ints([0, -1], torch.int32), block_round_bits=3))
    for r in range(2):
        want = attention.cpvm_with_adapter(orc, x[r], list(polys[:2]), None if r else list(polys[2:4]), raw, d2, w=3)
        assert np.array_equal(got[r, 0], want), r
    table, edges = _ints([[100], [-100]]), _ints([0, 7], torch.int32)
    out = P.to_host(rq.score_bias(dev(x), 2, 1, 1, d2, _ints([9, n // d2 - 1], torch.int32), table, edges))
    for r, pos in enumerate((9, n // d2 - 1)):
        bias = codec.encode(attention.score_bias_values(n, d2, 0, pos, [[100], [-100]], [0, 7], 0))
        assert np.array_equal(out[r], orc.add_plain(x[r], bias)), r
    cache = dev(x)
    rq.kv_append_requests(cache, 1, 2, 1, _ints([1, 0], torch.int32), dev(x[::-1].copy()), diags, n // 2)
    got = P.to_host(cache)
    assert np.array_equal(got[0], orc.add(x[0], orc.mul_plain(x[1], polys[1]))) and np.array_equal(got[1], orc.mul_plain(x[0], polys[0]))


@pytest.mark.parametrize("name", ["C1", "C2", "C5"])
def test_any_int64_is_a_representative(name):
    """Slots, matrices, factors and tables whose values fill 64 bits give what their residues give."""
    import torch
    env = _env(name)
    n, t, rq = env.n, env.prm.t, env.rq
    rng = np.random.default_rng(17)
    ends = np.array([2 ** 63 - 1, -(2 ** 63), 2 ** 32 - 1, 2 ** 32, -(2 ** 32), -(2 ** 31), 2 ** 31, -(2 ** 31) - 1, -1, 0], dtype=np.int64)

    def wide(*shape):
        v = rng.integers(-(2 ** 63), 2 ** 63 - 1, shape, dtype=np.int64, endpoint=True)
        v.reshape(-1)[:len(ends)] = ends
        return v, v % t

    say(f"{name}: slots")
    v, r = wide(9, n)
    assert torch.equal(rq.slots_encode(_ints(v)), rq.slots_encode(_ints(r)))
    assert torch.equal(rq.slots_prepare(_ints(v)), rq.slots_prepare(_ints(r)))
    units, d1, d2 = 2, 100, 64
    w, a, b = wide(units, d1, d2), wide(1, d1, 5), wide(units, 5, d2)
    for given in ((True, False), (False, True), (True, True)):       # W as it is given, A B, W beside A B
        say(f"{name}: matrices {given}")
        got, want = (rq.cpvm_prepare(units, d1, d2, w=_ints(w[i]) if given[0] else None, a=_ints(a[i]) if given[1] else None,
                                     b=_ints(b[i]) if given[1] else None, a_group=units) for i in range(2))
        assert torch.equal(got, want), given
    many = 1 + 256 // rq.cpvm_diagonals(d1, d2)                      # so many that they are laid out by diagonals first
    w = wide(many, d1, d2)
    assert torch.equal(*(rq.cpvm_prepare(many, d1, d2, w=_ints(x)) for x in w))
    say(f"{name}: tables")
    table, edges = wide(5, 2), _ints([0, 1, 2, 3, 4], torch.int32)
    s = env.dev(env.cts(2, 2))
    assert torch.equal(*(rq.score_bias(s, 1, 2, 1, d2, _ints([4], torch.int32), _ints(x), edges) for x in table))


@pytest.mark.parametrize("name,batch", [("C1", 300), ("C1", 513), ("C1", 700), ("C2", 257), ("C5", 270)])
def test_plaintexts_of_a_last_round(name, batch):
    """The last round's plaintexts, shared by several workgroups where it leaves room, are those of a call of their own."""
    import torch
    env = _env(name)
    say(f"slots_prepare {name}: {batch}")
    v = _ints(np.random.default_rng(batch).integers(-(2 ** 31), 2 ** 31, (batch, env.n)))
    got, polys = env.rq.slots_prepare(v), env.rq.slots_encode(v)
    assert torch.equal(got, env.ctx.plain_prepare(polys))
    assert torch.equal(got.view(batch, -1)[-1], env.rq.slots_prepare(v[-1:]))


@pytest.mark.parametrize("buckets", [32, 33, 64, 65])
def test_bucket_edges_are_found_by_either_way(buckets):
    """Around the numbers of buckets from which they are searched: every distance, edges that repeat and that lie beyond the cache."""
    import torch
    from oracle import attention
    env = _env("C1")
    d2 = 64
    blocks = env.n // d2
    say(f"biases: {buckets} buckets")
    rng = np.random.default_rng(buckets)
    edges = np.sort(rng.integers(0, blocks + 20, buckets))
    table = rng.integers(-128, 128, (buckets, 1))
    x = env.cts(3, blocks)
    got = env.host(env.rq.score_bias(env.dev(x[:2]), 2, 1, 1, d2, _ints([blocks - 1, blocks // 2], torch.int32), _ints(table),
                                     _ints(edges, torch.int32)))
    for r, pos in enumerate((blocks - 1, blocks // 2)):
        assert np.array_equal(got[r], env.orc.add_plain(x[r], env.codec.encode(attention.score_bias_values(env.n, d2, 0, pos, table, edges, 0)))), r
    got = env.host(env.rq.prompt_bias(env.dev(x), 1, 1, d2, _ints(table), _ints(edges, torch.int32)))
    for u in (0, 1, blocks // 2, blocks - 1):
        assert np.array_equal(got[u], env.orc.add_plain(x[u], env.codec.encode(attention.prompt_bias_values(env.n, d2, u, table, edges, 0)))), u
