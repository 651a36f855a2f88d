"""Slots, weights, adapters, position biases and appends of many requests: bit for bit against the oracle's integers.

Everything here is a residue or an integer modulo t, so every comparison is for equality; prepared plaintexts are compared as
the doubles that the evaluator's own cg_plain_prepare makes of the oracle's polynomials."""
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import attention
from oracle.client import SlotCodec, galois_rot
from workloads import Stream
from tests.test_gpu_parity import Env


def say(msg):
    print(f"[gpu-requests] {msg}", flush=True)
    sys.stdout.flush()


_envs = {}


def _env(name):
    if name not in _envs:
        env = _envs[name] = Env(name)
        env.rq = env.P.Requests(env.ctx)
        env.codec = SlotCodec(env.prm)
    return _envs[name]


def _ints(a, dtype=None):
    import torch
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int64)).to("cuda", dtype or torch.int64)


def _lens(a):
    import torch
    return _ints(a, torch.int32)


def _slots(n, batch, t, seed):
    """Rows that exercise the range: small values, all representatives, the extremes, a single slot, constants."""
    rng = np.random.default_rng(seed)
    v = rng.integers(-(2 ** 31) + 1, 2 ** 31, (batch, n))
    kinds = [rng.integers(-128, 128, n), np.full(n, t - 1), np.full(n, (t - 1) // 2), np.full(n, -((t - 1) // 2)), np.zeros(n),
             np.where(np.arange(n) % 2, (t - 1) // 2, (t + 1) // 2), np.eye(1, n, n - 1)[0], np.full(n, 2 ** 31 - 1)]
    for i in range(min(batch - 1, len(kinds))):
        v[i] = kinds[i]
    return v.astype(np.int64)


@pytest.mark.parametrize("name,batch", [("C1", 1), ("C1", 9), ("C2", 1), ("C2", 9), ("C2", 300), ("C5", 1), ("C5", 9), ("C5", 43)])
def test_slots_are_encoded_as_the_codec_does(name, batch):
    env = _env(name)
    v = _slots(env.n, batch, env.prm.t, 3 + batch)
    say(f"slots {name}: batch {batch}")
    got = env.host(env.rq.slots_encode(_ints(v)))
    rows = range(batch) if batch <= 9 else (0, 1, batch // 2, batch - 1)
    want = {i: env.codec.encode(v[i]) for i in rows}
    for i in rows:
        assert np.array_equal(got[i], want[i]), (name, batch, i)
    import torch
    plain = env.rq.slots_prepare(_ints(v)).view(batch, env.k, env.n)
    ref = env.ctx.plain_prepare(env.dev(got)).view(batch, env.k, env.n)
    assert torch.equal(plain, ref)


@pytest.mark.parametrize("log2n,t", [(12, 40961), (12, 1032193), (13, 1032193), (14, 786433)])
def test_other_plaintext_moduli(log2n, t):
    """Small ones and the largest below 2^20, where exact products and centred values are at their bounds."""
    import paper_2602_08798_amd as P
    from tests.bruteforce import ntt_primes
    from workloads.params import ParamSet
    k = {12: 2, 13: 1, 14: 2}[log2n]
    p = ntt_primes(1 << 50, 2 << log2n, k + 1)
    prm = ParamSet("x", log2n, q=tuple(p[:k]), p=tuple(p[k:]), t=t)
    ctx, codec, n = P.Context(prm), SlotCodec(prm), prm.n
    rq = P.Requests(ctx)
    say(f"t = {t}, N = {n}")
    v = _slots(n, 9, t, t)
    got = P.to_host(rq.slots_encode(_ints(v)))
    for i in range(9):
        assert np.array_equal(got[i], codec.encode(v[i])), i
    import torch
    assert torch.equal(rq.slots_prepare(_ints(v)), ctx.plain_prepare(P.to_device(got)))
    # an adapter of the largest rank with entries of the largest size
    h = (t - 1) // 2
    a, b = np.full((1, 64, 4096), h), np.full((1, 4096, 64), -h)
    b[0, :, 0], b[0, :, 1] = h, np.arange(4096) % 2 * 2 * h - h
    M = np.zeros((64, 64), dtype=np.int64)
    M[:] = [int(sum(h * int(x) for x in b[0, :, c])) % t for c in range(64)]
    C = rq.cpvm_diagonals(64, 64)
    want = np.stack([codec.encode(attention.cpvm_weight_values(n, 64, 64, M, c)) for c in range(C)])
    assert torch.equal(rq.cpvm_prepare(1, 64, 64, a=_ints(a), b=_ints(b)), ctx.plain_prepare(P.to_device(want)))
    table, edges = np.array([[h], [-h], [t - 1], [1]]), np.array([0, 1, 2, 9])
    orc = __import__("oracle").Oracle(prm)
    from workloads import pseudo_ciphertexts
    x = pseudo_ciphertexts(Stream(5, 1), prm.q, n, 1)
    out = P.to_host(rq.score_bias(P.to_device(x), 1, 1, 1, 64, _lens([n // 64 - 1]), _ints(table), _lens(edges)))
    assert np.array_equal(out[0], orc.add_plain(x[0], codec.encode(attention.score_bias_values(n, 64, 0, n // 64 - 1, table, edges, 0))))


def test_a_modulus_without_slots_has_no_handle():
    import paper_2602_08798_amd as P
    from paper_2602_08798_amd.binding import CgError
    from dataclasses import replace
    from workloads import PRESETS
    ctx = P.Context(replace(PRESETS["C1"], t=65521))
    with pytest.raises(CgError):
        P.Requests(ctx)


def test_a_closed_handle_or_context_is_refused():
    import paper_2602_08798_amd as P
    from paper_2602_08798_amd.binding import CgError
    from workloads import PRESETS
    ctx = P.Context(PRESETS["C1"])
    first, second = P.Requests(ctx), P.Requests(ctx)
    v = _ints(np.zeros((1, ctx.n)))
    first.slots_encode(v)
    first.close()
    with pytest.raises(CgError):
        first.slots_encode(v)
    second.slots_encode(v)
    ctx.close()
    with pytest.raises(CgError):
        second.slots_encode(v)


def _matrices(rng, units, d1, d2, rank, a_group, base, lo=-128, hi=128):
    return (rng.integers(lo, hi, (units, d1, d2)) if base else None,
            rng.integers(lo, hi, (-(-units // a_group), d1, rank)) if rank else None,
            rng.integers(lo, hi, (units, rank, d2)) if rank else None)


def _weight_polys(env, d1, d2, w, a, b, u, a_group):
    C = attention.cpvm_shape(env.n, d1, d2)[2]
    M = attention.low_rank_matrix(None if w is None else w[u], None if a is None else a[u // a_group], None if b is None else b[u])
    M = np.asarray(M % env.prm.t, dtype=np.int64)
    return np.stack([env.codec.encode(attention.cpvm_weight_values(env.n, d1, d2, M, c)) for c in range(C)])


@pytest.mark.parametrize("name,d1,d2,units,rank,a_group,base", [
    ("C1", 1, 64, 1, 0, 1, True), ("C1", 768, 64, 2, 0, 1, True), ("C1", 1000, 64, 3, 5, 2, True), ("C1", 65, 128, 2, 1, 1, False),
    ("C2", 768, 64, 4, 16, 3, False), ("C2", 300, 32, 1, 67, 1, True), ("C2", 4096, 128, 1, 3, 1, False), ("C5", 768, 64, 1, 8, 1, True),
    ("C5", 2048, 16, 1, 4, 5, False), ("C2", 2048, 4, 1, 2, 1, True), ("C1", 64, 256, 1, 3, 1, False)])
def test_weights_and_adapters_become_the_diagonals_of_their_matrix(name, d1, d2, units, rank, a_group, base):
    env = _env(name)
    say(f"cpvm_prepare {name}: {units} of {d1} x {d2}, rank {rank}, base {base}")
    rng = np.random.default_rng(d1 + d2 + rank)
    w, a, b = _matrices(rng, units, d1, d2, rank, a_group, base)
    if units > 1 and rank:      # any representatives
        b[1] = rng.integers(-(2 ** 31) + 1, 2 ** 31, b[1].shape)
        a[0] = rng.integers(-(2 ** 31) + 1, 2 ** 31, a[0].shape)
    dev = [None if x is None else _ints(x) for x in (w, a, b)]
    C = env.rq.cpvm_diagonals(d1, d2)
    assert C == attention.cpvm_shape(env.n, d1, d2)[2]
    got = env.rq.cpvm_prepare(units, d1, d2, *dev, a_group=a_group).view(units, C, env.k, env.n)
    import torch
    for u in range(units):
        ref = env.ctx.plain_prepare(env.dev(_weight_polys(env, d1, d2, w, a, b, u, a_group)))
        assert torch.equal(got[u], ref.view(C, env.k, env.n)), (name, d1, d2, u)


def _projection(env, d1, d2, bits, seed):
    """(copy keys, block keys, raw keys by Galois element)"""
    n, C = env.n, attention.cpvm_shape(env.n, d1, d2)[2]
    g_copies = [galois_rot(n, c) for c in range(1, C)]
    gens = attention.block_generators(n, d2)
    g_block = [g for r in attention.round_galois(n, gens, bits) for g in r] if bits else gens
    key = {g: env.key(seed + i) for i, g in enumerate(dict.fromkeys(g_copies + g_block))}
    return [key[g][1] for g in g_copies], [key[g][1] for g in g_block], {g: x[0] for g, x in key.items()}


@pytest.mark.parametrize("name,requests,units,d1,d2,bits,adapters", [
    ("C1", 1, 1, 64, 64, 3, 0), ("C1", 3, 2, 100, 64, 0, 2), ("C2", 2, 3, 768, 64, 3, 2), ("C2", 5, 1, 300, 32, 2, 1),
    ("C5", 2, 1, 768, 64, 3, 1), ("C1", 2, 2, 30, 64, 4, 1), ("C1", 2, 1, 1500, 64, 3, 2)])
def test_projections_of_many_requests_with_adapters(name, requests, units, d1, d2, bits, adapters):
    env = _env(name)
    n, C = env.n, attention.cpvm_shape(env.n, d1, d2)[2]
    say(f"cpvm_requests {name}: {requests} x {units}, {d1} x {d2}, {C} diagonals, {bits} bits, {adapters} adapters")
    rng = np.random.default_rng(requests * 100 + units + d1)
    x = env.cts(300 + requests, requests)
    base = rng.integers(0, env.prm.t, (units * C, n)).astype(np.uint64)
    plus = rng.integers(0, env.prm.t, (adapters, units * C, n)).astype(np.uint64)
    # out of range, unused and repeated choices
    pick = [(adapters, 0, -1, 0, 2 ** 31 - 1, -(2 ** 31), adapters - 1)[r % 7] if adapters < 2 else (1, 0, -1, 1, adapters)[r % 5]
            for r in range(requests)]
    copies, block, raw = _projection(env, d1, d2, bits, 500)
    prep = lambda p: env.ctx.plain_prepare(env.dev(p))
    import torch
    extra = dict(adapters=torch.stack([prep(p) for p in plus]), pick=_lens(pick)) if adapters else {}
    got = env.host(env.rq.cpvm_requests(env.dev(x), prep(base), requests, units, C, d2, copies, block, block_round_bits=bits, **extra))
    for r in range(requests):
        for u in range(units):
            own = plus[pick[r]][u * C:(u + 1) * C] if 0 <= pick[r] < adapters else None
            want = attention.cpvm_with_adapter(env.orc, x[r], list(base[u * C:(u + 1) * C]), own, raw, d2, w=bits)
            assert np.array_equal(got[r, u], want), (name, r, u)


def test_projections_without_adapters_are_those_of_one_request():
    """... also with enough requests for the rounds' larger launches."""
    import torch
    env = _env("C2")
    d1, d2, units, requests = 768, 64, 7, 9
    C = attention.cpvm_shape(env.n, d1, d2)[2]
    say(f"cpvm_requests C2: {requests} x {units} against one by one")
    copies, block, _ = _projection(env, d1, d2, 3, 500)
    diags = env.rq.cpvm_prepare(units, d1, d2, w=_ints(np.random.default_rng(1).integers(-128, 128, (units, d1, d2))))
    x = env.dev(env.cts(7, requests))
    got = env.rq.cpvm_requests(x, diags, requests, units, C, d2, copies, block, block_round_bits=3)
    for r in range(requests):
        assert torch.equal(got[r], env.ctx.cpvm_hoisted(x[r], diags, units, C, d2, copies, block, block_round_bits=3)), r


@pytest.mark.parametrize("name,requests,units,d1,bits", [("C2", 9, 8, 64, 3), ("C2", 12, 12, 64, 3), ("C2", 8, 36, 64, 4), ("C2", 1, 576, 64, 3),
                                                        ("C1", 13, 41, 64, 3), ("C5", 9, 4, 64, 3), ("C2", 17, 1, 768, 0),
                                                        ("C1", 61, 36, 64, 3), ("C1", 140, 1, 768, 3)])
def test_large_calls_are_the_small_ones(name, requests, units, d1, bits):
    """Calls whose rounds are cut into whole rounds of the compute units and the rest, with adapters: each request against the call
    for one request with its adapter's diagonals added to the base's."""
    import torch
    env = _env(name)
    d2, q = 64, torch.tensor(env.prm.q, dtype=torch.float64, device="cuda")[:, None]
    C = attention.cpvm_shape(env.n, d1, d2)[2]
    say(f"cpvm_requests {name}: {requests} x {units}, {C} diagonals, {bits} bits")
    copies, block, _ = _projection(env, d1, d2, bits, 500)
    rng = np.random.default_rng(units)
    base = env.rq.cpvm_prepare(units, d1, d2, w=_ints(rng.integers(-128, 128, (units, d1, d2))))
    low = torch.stack([env.rq.cpvm_prepare(units, d1, d2, a=_ints(rng.integers(-128, 128, (1, d1, 3))), b=_ints(rng.integers(-128, 128, (units, 3, d2))),
                                           a_group=units) for _ in range(2)])
    x = env.dev(env.cts(7, requests))
    pick = [(0, 1, -1)[r % 3] for r in range(requests)]
    got = env.rq.cpvm_requests(x, base, requests, units, C, d2, copies, block, adapters=low, pick=_lens(pick), block_round_bits=bits)
    for r in range(requests):
        both = base.view(-1, env.k, env.n) + (low[pick[r]].view(-1, env.k, env.n) if pick[r] >= 0 else 0)
        both = torch.where(both > q / 2, both - q, torch.where(both < -q / 2, both + q, both)).contiguous()
        assert torch.equal(got[r], env.ctx.cpvm_hoisted(x[r], both, units, C, d2, copies, block, block_round_bits=bits)), r


def _bias_case(env, heads, buckets, seed, first=0):
    rng = np.random.default_rng(seed)
    edges = first + np.cumsum(np.concatenate([[0], rng.integers(1, 40, buckets - 1)]))
    table = rng.integers(-128, 128, (buckets, heads))
    table[0, 0] = 2 ** 31 - 1
    return table, edges


@pytest.mark.parametrize("name,requests,heads,n_cts,d2,buckets,first", [
    ("C1", 1, 1, 1, 64, 1, 0), ("C1", 4, 3, 2, 64, 9, 0), ("C2", 3, 2, 3, 64, 32, 0), ("C2", 2, 1, 2, 2, 7, 0), ("C2", 2, 1, 1, 2048, 3, 0),
    ("C5", 2, 2, 1, 128, 16, 3), ("C1", 2, 1, 2, 1024, 5, 1), ("C1", 3, 2, 1, 4, 4096, 0)])
def test_score_bias(name, requests, heads, n_cts, d2, buckets, first):
    env = _env(name)
    B = env.n // d2
    say(f"score_bias {name}: {requests} x {heads} x {n_cts}, d2 {d2}, {buckets} buckets")
    table, edges = _bias_case(env, heads, buckets, requests + d2, first)
    pos = ([n_cts * B - 1, 0, -1, B // 2, 2 ** 31 - 1] * requests)[:requests]
    x = env.cts(41, requests * heads * n_cts).reshape(requests, heads, n_cts, 2, env.k, env.n)
    x[0, 0, 0, :, :, 0] = 0
    x[0, 0, 0, :, :, 1] = np.asarray(env.prm.q, dtype=np.uint64) - 1
    d = env.dev(x)
    args = (requests, heads, n_cts, d2, _lens(pos), _ints(table), _lens(edges))
    got = env.host(env.rq.score_bias(d, *args))
    assert np.array_equal(env.host(d), x)
    for r in range(requests):
        for h in range(heads):
            for c in range(n_cts):
                v = attention.score_bias_values(env.n, d2, c, pos[r], table, edges, h)
                want = env.orc.add_plain(x[r, h, c], env.codec.encode(v))
                assert np.array_equal(got[r, h, c], want), (name, r, h, c)
    assert env.rq.score_bias(d, *args, out=d) is d
    assert np.array_equal(env.host(d), got)


@pytest.mark.parametrize("name,prompts,heads,d2,buckets", [("C1", 1, 1, 64, 16), ("C1", 2, 2, 512, 4), ("C2", 1, 2, 128, 32), ("C5", 1, 1, 1024, 3)])
def test_prompt_bias(name, prompts, heads, d2, buckets):
    env = _env(name)
    m = env.n // d2
    say(f"prompt_bias {name}: {prompts} x {heads}, d2 {d2}")
    table, edges = _bias_case(env, heads, buckets, 9 + d2)
    x = env.cts(43, prompts * heads * m).reshape(prompts, heads, m, 2, env.k, env.n)
    d = env.dev(x)
    got = env.host(env.rq.prompt_bias(d, prompts, heads, d2, _ints(table), _lens(edges)))
    for p in range(prompts):
        for h in range(heads):
            for u in sorted({0, 1, m // 2 - 1, m // 2, m - 1, m // 3}):
                want = env.orc.add_plain(x[p, h, u], env.codec.encode(attention.prompt_bias_values(env.n, d2, u, table, edges, h)))
                assert np.array_equal(got[p, h, u], want), (name, p, h, u)
    env.rq.prompt_bias(d, prompts, heads, d2, _ints(table), _lens(edges), out=d)
    assert np.array_equal(env.host(d), got)


@pytest.mark.parametrize("name,requests,per,stride,d2,gap", [("C1", 1, 2, 1, 64, 0), ("C1", 7, 2, 2, 64, 1), ("C2", 6, 3, 2, 64, 0), ("C5", 3, 2, 2, 128, 2),
                                                             ("C1", 4, 1, 3, 2048, 0), ("C2", 3, 1, 1, 32, 0)])
def test_appends_at_each_requests_own_length(name, requests, per, stride, d2, gap):
    env = _env(name)
    B = env.n // d2
    say(f"kv_append_requests {name}: {requests} x {per}, stride {stride}, d2 {d2}")
    lens = ([B * stride - 1, 0, B * stride, -1, B - 1, B if stride > 1 else 1, 2 ** 31 - 1, -(2 ** 31)])[:requests]
    rng = np.random.default_rng(11)
    polys = rng.integers(0, env.prm.t, (B, env.n)).astype(np.uint64)
    masks = env.ctx.plain_prepare(env.dev(polys))
    cache = env.cts(50, requests * per * stride).reshape(requests, per, stride, 2, env.k, env.n)
    rows = env.cts(51, requests * (per + gap)).reshape(requests, per + gap, 2, env.k, env.n)
    d = env.dev(cache)
    env.rq.kv_append_requests(d, stride, requests, per, _lens(lens), env.dev(rows), masks, d2, row_stride_cts=per + gap)
    got, want = env.host(d), cache.copy()
    for r, length in enumerate(lens):
        if not 0 <= length < B * stride:
            continue
        at, b = divmod(length, B)
        for c in range(per):
            new = env.orc.mul_plain(rows[r, c], polys[b])
            want[r, c, at] = env.orc.add(cache[r, c, at], new) if b else new
    assert np.array_equal(got, want)


def test_a_step_of_many_requests_captured_and_replayed():
    """Projection with adapters, append, scores, bias: captured once, replayed for tokens at new lengths.  Between the replays the
    program's own eager calls run, a larger one of them with the same handle."""
    import torch
    env = _env("C1")
    ctx, rq, n = env.ctx, env.rq, env.n
    R, H, d1, d2, stride = 2, 1, 100, 64, 2
    B, C, U = n // d2, attention.cpvm_shape(n, d1, d2)[2], 3
    rng = np.random.default_rng(5)
    copies, block, _ = _projection(env, d1, d2, 3, 500)
    fold = [env.key(700 + i)[1] for i in range(6)]
    rlk = env.key(710)[1]
    base = rq.cpvm_prepare(U, d1, d2, w=_ints(rng.integers(-128, 128, (U, d1, d2))))
    low = torch.stack([rq.cpvm_prepare(U, d1, d2, a=_ints(rng.integers(-128, 128, (1, d1, 4))), b=_ints(rng.integers(-128, 128, (U, 4, d2))),
                                       a_group=U) for _ in range(2)])
    masks = rq.slots_prepare(_ints([attention.block_mask_values(n, d2, b) for b in range(B)]))
    table, edges = _bias_case(env, H, 8, 3)
    table, edges = _ints(table), _lens(edges)
    x, pick, lens = env.dev(env.cts(60, R)), _lens([1, 0]), _lens([3, B + 5])
    cache = env.dev(env.cts(61, R * 2 * H * stride)).view(R, 2 * H, stride, 2, env.k, n)
    out = {}

    def step():
        y = rq.cpvm_requests(x, base, R, U, C, d2, copies, block, adapters=low, pick=pick, block_round_bits=3)
        q, kv = y[:, :H].contiguous(), y[:, H:].contiguous()
        rq.kv_append_requests(cache, stride, R, 2 * H, lens, kv, masks, d2)
        k_cache = cache[:, :H].contiguous()
        s = ctx.decode_scores(q, k_cache, R * H, stride, d2, rlk, fold)
        out["scores"] = rq.score_bias(s, R, H, stride, d2, lens, table, edges, out=s)

    def state(seed, i):
        return env.dev(env.cts(seed, R)), _lens([(i + 1) % 3 - 1, i % 2]), _lens([4 + 70 * i, B + 5 + i])
    cache0 = cache.clone()
    want = []
    for i in range(4):
        for a, b in zip((x, pick, lens), state(70 + i, i)):
            a.copy_(b)
        step()
        torch.cuda.synchronize()
        want.append((out["scores"].clone(), cache.clone()))
    say("capture")
    cache.copy_(cache0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    torch.cuda.synchronize()
    cache.copy_(cache0)
    for i in range(4):
        say(f"replay {i}")
        for a, b in zip((x, pick, lens), state(70 + i, i)):
            a.copy_(b)
        # eager work with a larger workspace of the same handle
        rq.cpvm_requests(env.dev(env.cts(90, 5)), base, 5, U, C, d2, copies, block, block_round_bits=3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out["scores"], want[i][0]) and torch.equal(cache, want[i][1]), i


def test_two_handles_and_two_streams_at_once():
    import torch
    env = _env("C2")
    ctx, d1, d2, R, U = env.ctx, 768, 64, 2, 2
    C = attention.cpvm_shape(env.n, d1, d2)[2]
    copies, block, _ = _projection(env, d1, d2, 3, 500)
    rng = np.random.default_rng(8)
    w = [_ints(rng.integers(-128, 128, (U, d1, d2))) for _ in range(2)]
    x = [env.dev(env.cts(80 + i, R)) for i in range(2)]
    want = [env.rq.cpvm_requests(x[i], env.rq.cpvm_prepare(U, d1, d2, w=w[i]), R, U, C, d2, copies, block, block_round_bits=3) for i in range(2)]
    other = env.P.Requests(ctx)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    say("two streams")
    for _ in range(3):
        for i, (s, rq) in enumerate(zip(streams, (env.rq, other if _ else env.rq))):
            with torch.cuda.stream(s):
                got[i] = rq.cpvm_requests(x[i], rq.cpvm_prepare(U, d1, d2, w=w[i]), R, U, C, d2, copies, block, block_round_bits=3)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    other.close()


def test_one_step_on_real_encryptions():
    """Slots, base weights and an adapter, the projection, the append, the scores and the bias on real encryptions: every stage
    decrypts to the plaintext arithmetic mod t."""
    import torch
    from oracle.client import Client
    env = _env("C2")
    prm, n, t, ctx, rq = env.prm, env.n, env.prm.t, env.ctx, env.rq
    d1, d2, U, R = 100, 64, 2, 2
    B, C = n // d2, attention.cpvm_shape(n, d1, d2)[2]
    client = Client(prm, 77, env.orc)
    rng = np.random.default_rng(21)
    g_block = [g for r in attention.round_galois(n, attention.block_generators(n, d2), 3) for g in r]
    g_fold = attention.fold_generators(n, d2)
    gks = {g: ctx.ksk_prepare(env.dev(client.galois_key(g))) for g in
           dict.fromkeys([galois_rot(n, c) for c in range(1, C)] + g_block + g_fold)}
    rlk = ctx.ksk_prepare(env.dev(client.relin_key()))
    W = rng.integers(-128, 128, (U, d1, d2))
    A, Bm = rng.integers(-8, 8, (2, 1, d1, 4)), rng.integers(-8, 8, (2, U, 4, d2))
    x = rng.integers(-128, 128, (R, d1))
    ct = env.dev(np.stack([client.encrypt_slots(attention.cpvm_token_values(n, d1, d2, v)) for v in x]))
    base = rq.cpvm_prepare(U, d1, d2, w=_ints(W))
    low = torch.stack([rq.cpvm_prepare(U, d1, d2, a=_ints(A[i]), b=_ints(Bm[i]), a_group=U) for i in range(2)])
    y = rq.cpvm_requests(ct, base, R, U, C, d2, [gks[galois_rot(n, c)] for c in range(1, C)], [gks[g] for g in g_block], adapters=low,
                         pick=_lens([1, -1]), block_round_bits=3)
    host = env.host(y)
    want = np.stack([[x[r] @ (W[u] + (A[1][0] @ Bm[1][u] if r == 0 else 0)) for u in range(U)] for r in range(R)])
    for r in range(R):
        for u in range(U):
            assert np.array_equal(client.decrypt_slots(host[r, u]), np.tile(want[r, u] % t, B)), (r, u)
    # unit 0 is the query, unit 1 the new key row; the caches start empty, one request has had tokens
    masks = rq.slots_prepare(_ints([attention.block_mask_values(n, d2, b) for b in range(B)]))
    cache = torch.zeros(R, 1, 1, 2, env.k, n, dtype=torch.int64, device="cuda")
    rows = y.view(-1)[2 * env.k * n:]                        # from request 0's unit 1 on, a request's results apart
    for lens in ([0, 0], [-1, 1]):
        rq.kv_append_requests(cache, 1, R, 1, _lens(lens), rows, masks, d2, row_stride_cts=U)
    s = ctx.decode_scores(y[:, :1].contiguous(), cache, R, 1, d2, rlk, [gks[g] for g in g_fold])
    table, edges = rng.integers(-128, 128, (4, 1)), np.array([0, 1, 2, 4])
    s = env.host(rq.score_bias(s.view(R, 1, 1, 2, env.k, n), R, 1, 1, d2, _lens([0, 1]), _ints(table), _lens(edges)))
    for r in range(R):
        got = client.decrypt_slots(s[r, 0, 0])[::d2]
        dot = int(want[r, 0] @ want[r, 1])
        for j in range(B):
            there = j <= r
            assert got[j] == (dot + int(table[r - j][0]) if there else 0) % t, (r, j)


def test_refusals():
    import torch
    from paper_2602_08798_amd.binding import CgError, CgSizeError
    env = _env("C1")
    rq, n, k = env.rq, env.n, env.k
    v = _ints(np.zeros((2, n)))
    with pytest.raises(CgSizeError):
        rq.slots_prepare(v[0, :-2].contiguous())
    with pytest.raises(CgSizeError):
        rq.slots_prepare(v.to(torch.int32))
    with pytest.raises(CgSizeError):
        rq.slots_encode(v, out=torch.empty(n, dtype=torch.int64, device="cuda"))
    with pytest.raises(CgSizeError):
        rq.slots_encode(v.t())
    with pytest.raises(CgError):
        rq.slots_encode(v, out=v)
    w = _ints(np.zeros((2, 100, 64)))
    a, b = _ints(np.zeros((1, 100, 4))), _ints(np.zeros((2, 4, 64)))
    for bad in (dict(), dict(a=a), dict(b=b), dict(w=w[0]), dict(a=a, b=b, a_group=1), dict(a=a, b=b[0], a_group=2), dict(a=a, b=b, a_group=0)):
        with pytest.raises((CgError, AssertionError)):
            rq.cpvm_prepare(2, 100, 64, **bad)
    assert rq.cpvm_diagonals(n // 2 + 1, 64) == rq.cpvm_diagonals(100, 48) == rq.cpvm_diagonals(0, 64) == rq.cpvm_diagonals(100, n // 2) == 0
    with pytest.raises(CgError):
        rq.cpvm_prepare(1, n // 2 + 1, 64, w=_ints(np.zeros((n // 2 + 1, 64))))
    x, plain = env.dev(env.cts(1, 2)), env.rq.slots_prepare(_ints(np.zeros((4, n))))
    key = env.key(1)[1]
    C = attention.cpvm_shape(n, 100, 64)[2]
    copies, block, _ = _projection(env, 100, 64, 3, 500)
    diags = rq.cpvm_prepare(1, 100, 64, w=w[0].contiguous())
    good = dict(requests=2, units=1, n_diag=C, d2=64, gk_copies=copies, gk_block=block, block_round_bits=3)
    for change in (dict(requests=3), dict(units=0), dict(units=2), dict(n_diag=C * 2), dict(gk_copies=copies + [key]), dict(gk_block=block[:-1]),
                   dict(d2=48), dict(block_round_bits=8), dict(adapters=diags), dict(adapters=diags[:-1], pick=_lens([0, 0])),
                   dict(adapters=diags, pick=_lens([0])), dict(adapters=diags, pick=_ints([0, 0])), dict(out=x)):
        with pytest.raises((CgError, AssertionError)):
            rq.cpvm_requests(x, diags, **{**good, **change})
    s, table, edges, pos = env.dev(env.cts(2, 2)), _ints([[1], [2]]), _lens([0, 3]), _lens([1])
    for bad in ((2, 1, 2, 64, pos), (1, 1, 2, 48, pos), (1, 1, 2, n // 2, pos), (1, 1, 0, 64, pos), (1, 2, 1, 64, pos), (2, 1, 1, 64, pos)):
        with pytest.raises(CgError):
            rq.score_bias(s, *bad, table, edges)
    with pytest.raises(CgError):
        rq.score_bias(s, 1, 1, 2, 64, pos, table, edges[:0])
    with pytest.raises(CgError):
        rq.score_bias(s, 1, 1, 1, 64, pos, table, edges, out=s.view(-1)[n:])          # overlaps, and is not the input
    with pytest.raises(CgSizeError):
        rq.prompt_bias(s, 1, 1, 64, table, edges)
    cache, lens = env.dev(env.cts(3, 4)), _lens([0, 0])
    masks = rq.slots_prepare(_ints(np.zeros((n // 64, n))))
    for bad in ((1, 3, 1, lens, x, masks, 64), (2, 2, 2, lens, x, masks, 64), (0, 2, 1, lens, x, masks, 64), (2, 2, 1, lens[:1], x, masks, 64),
                (2, 2, 1, lens, x, plain, 64), (2, 2, 1, lens, x, masks, 48), (2, 2, 1, lens, cache, masks, 64)):
        with pytest.raises(CgError):
            rq.kv_append_requests(cache, *bad)
    with pytest.raises(CgError):
        rq.kv_append_requests(cache, 2, 2, 1, lens, x, masks, 64, row_stride_cts=0)


@pytest.mark.parametrize("wrap", [1 << 32, -(1 << 32)])
def test_sizes_that_would_pass_in_their_low_32_bits_are_refused(wrap):
    import torch
    from paper_2602_08798_amd.binding import CgError
    env = _env("C1")
    rq, n = env.rq, env.n
    a, b = _ints(np.zeros((1, 100, 4))), _ints(np.zeros((2, 4, 64)))
    x, plain, many = env.dev(env.cts(1, 2)), rq.slots_prepare(_ints(np.zeros((n // 64, n)))), env.dev(env.cts(2, n // 64))
    copies, block, _ = _projection(env, 100, 64, 3, 500)
    C = attention.cpvm_shape(n, 100, 64)[2]
    table, edges, pos, lens = _ints([[1], [2]]), _lens([0, 3]), _lens([1, 1]), _lens([0, 0])
    cache = env.dev(env.cts(3, 4))
    out = torch.empty(4 * rq.k * n, dtype=torch.float64, device="cuda")
    calls = [lambda *s: rq.cpvm_prepare(s[0], s[1], s[2], a=a, b=b, a_group=s[3], out=out),
             lambda *s: rq.cpvm_requests(x, plain, s[0], s[1], s[2], s[3], copies, block, block_round_bits=3, out=cache),
             lambda *s: rq.score_bias(x, s[0], s[1], s[2], s[3], pos, table, edges),
             lambda *s: rq.prompt_bias(many, s[0], s[1], s[2], table, edges),
             lambda *s: rq.kv_append_requests(cache, s[0], s[1], s[2], lens, x, plain, s[3], row_stride_cts=s[4])]
    sizes = [(2, 100, 64, 2), (1, 1, C, 64), (2, 1, 1, 64), (1, 1, 64), (2, 2, 1, 64, 1)]
    for call, good in zip(calls, sizes):
        call(*good)
        for at in range(len(good)):
            bad = list(good)
            bad[at] += wrap
            with pytest.raises(CgError):
                call(*bad)
    assert rq.cpvm_diagonals(100 + wrap, 64) == rq.cpvm_diagonals(100, 64 + wrap) == 0


def test_offsets_beyond_32_bits():
    """Caches, scores, plaintexts and units of more than 2^32 bytes: what lies behind, against the small calls."""
    import torch
    env = _env("C1")
    rq, n, k, d2 = env.rq, env.n, env.k, 64
    B, ct = n // d2, 2 * k * n
    far = (5 << 30) // (8 * ct)                       # ciphertexts in 5 GiB
    rows = env.dev(env.cts(60, 2))
    masks = env.ctx.plain_prepare(env.dev(np.random.default_rng(1).integers(0, env.prm.t, (B, n)).astype(np.uint64)))
    say(f"append: stride {far}")
    old = env.dev(env.cts(61, 2)).view(2, 1, ct)
    cache = torch.zeros((2, far, ct), dtype=torch.int64, device="cuda")
    cache[:, far - 1] = old[:, 0]
    rq.kv_append_requests(cache, far, 2, 1, _lens([B * far - 1, B * (far - 1)]), rows, masks, d2)
    rq.kv_append_requests(old, 1, 2, 1, _lens([B - 1, 0]), rows, masks, d2)
    assert torch.equal(cache[:, far - 1:], old) and not cache[:, :far - 1].any()
    say(f"score_bias: {far} ciphertexts, in place")
    scores, few = cache[0], env.dev(env.cts(62, 3)).view(3, ct)
    table, edges = _bias_case(env, 1, 9, 3)
    scores[far - 3:] = few
    rq.score_bias(scores, 1, 1, far, d2, _lens([B * (far - 2) + 5]), _ints(table), _lens(edges), out=scores)
    assert torch.equal(scores[far - 3:], rq.score_bias(few, 1, 1, 3, d2, _lens([B + 5]), _ints(table), _lens(edges)))
    del cache, scores
    torch.cuda.empty_cache()
    say("slots_prepare: 65536 plaintexts")
    v = torch.zeros((65536, n), dtype=torch.int64, device="cuda")
    last = _ints(_slots(n, 9, env.prm.t, 5))
    v[-9:] = last
    plain = rq.slots_prepare(v).view(65536, -1)
    assert torch.equal(plain[-9:], rq.slots_prepare(last).view(9, -1)) and not plain[:-9].any()
    del v
    say("cpvm_requests: 65536 units")
    copies, block, _ = _projection(env, 64, d2, 3, 500)
    got = rq.cpvm_requests(rows[:1], plain, 1, 65536, 1, d2, copies, block, block_round_bits=3).view(65536, ct)
    few = rq.cpvm_requests(rows[:1], plain[-9:].contiguous(), 1, 9, 1, d2, copies, block, block_round_bits=3).view(9, ct)
    assert torch.equal(got[-9:], few) and not got[:-9].any()
