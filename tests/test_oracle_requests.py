"""Pins of the oracle's operations for many requests: what they decrypt to on small rings, and the identities the kernels rest on."""
import numpy as np
import pytest

from oracle import Oracle, attention
from oracle.bfv import interp_odd, min_psi
from oracle.client import Client, SlotCodec, galois_rot
from workloads import Stream

from .toy import toy_params


@pytest.mark.parametrize("log2n,d1,d2,rank,w", [(7, 20, 8, 3, 0), (8, 100, 16, 5, 3), (8, 5, 64, 1, 2)])
def test_a_projection_with_an_adapter_decrypts_to_the_adapted_matrix(log2n, d1, d2, rank, w):
    prm = toy_params(log2n, 3, 1, 1)
    orc, n, t = Oracle(prm), prm.n, prm.t
    cl = Client(prm, 81, orc)
    C = attention.cpvm_shape(n, d1, d2)[2]
    g = Stream(81, d1)
    W, A, B, x = g.integers(-128, 128, (d1, d2)), g.integers(-16, 16, (d1, rank)), g.integers(-16, 16, (rank, d2)), g.integers(-128, 128, d1)
    need = set(attention.cpvm_hoisted_galois(n, C, d2))
    if w:
        need |= set(attention.hoisted_fold_galois(n, d2, 1, w))
    gks = {gal: cl.galois_key(gal) for gal in sorted(need)}
    enc = lambda M: [cl.codec.encode(attention.cpvm_weight_values(n, d1, d2, np.asarray(M % t, dtype=np.int64), c)) for c in range(C)]
    ct = cl.encrypt_slots(attention.cpvm_token_values(n, d1, d2, x))
    for low in (None, attention.low_rank_matrix(None, A, B)):
        y = attention.cpvm_with_adapter(orc, ct, enc(W), None if low is None else enc(low), gks, d2, w=w)
        want = (x.astype(object) @ attention.low_rank_matrix(W, *((None, None) if low is None else (A, B)))) % t
        assert np.array_equal(cl.decrypt_slots(y), np.tile(np.array(want, dtype=np.int64), n // d2))
        assert cl.noise_budget_bits(y, cl.decrypt_poly(y)) > 20


def test_a_projection_without_an_adapter_is_the_one_of_a_single_token():
    prm = toy_params(7, 2, 1, 1)
    orc, n = Oracle(prm), prm.n
    g = Stream(82, 1)
    from workloads import pseudo_ciphertexts, pseudo_switch_key
    qp = list(prm.q) + list(prm.p)
    x = pseudo_ciphertexts(g, prm.q, n, 1)[0]
    diags = list(g.integers(0, prm.t, (4, n)).astype(np.uint64))
    need = [galois_rot(n, c) for c in range(1, 4)] + [e for r in attention.round_galois(n, attention.block_generators(n, 16), 2) for e in r]
    gks = {gal: pseudo_switch_key(g, qp, n, prm.dnum) for gal in need}
    assert np.array_equal(attention.cpvm_with_adapter(orc, x, diags, None, gks, 16, w=2), attention.cpvm_hoisted(orc, x, diags, gks, 16, w=2))


def test_buckets_begin_at_their_edges():
    table, edges = np.array([[1, 10], [2, 20], [3, 30]]), [0, 1, 4]
    assert [attention.bias_of(d, table, edges, 0) for d in (-1, 0, 1, 3, 4, 1000)] == [0, 1, 2, 2, 3, 3]
    assert [attention.bias_of(d, table, [2, 3, 4], 1) for d in (0, 1, 2, 3)] == [0, 0, 10, 20]


def test_biased_scores_decrypt_to_scores_and_biases():
    """A token at index 5 of a cache of 16: every earlier token's score has its bucket's bias, later ones are as they were; the diagonals
    of a prompt pair every query with the key token that prefill_qk puts there."""
    prm = toy_params(7, 3, 1, 1)
    orc, n, t, d = Oracle(prm), prm.n, prm.t, 8
    cl = Client(prm, 83, orc)
    B = n // d
    g = Stream(83, 1)
    table, edges = g.integers(-128, 128, (4, 1)), [0, 1, 2, 4]
    scores = g.integers(0, t, n)
    ct = cl.encrypt_slots(scores)
    got = cl.decrypt_slots(orc.add_plain(ct, cl.codec.encode(attention.score_bias_values(n, d, 0, 5, table, edges, 0))))
    want = scores.copy()
    for j in range(6):
        want[j * d] += table[sum(e <= 5 - j for e in edges) - 1][0]
    assert np.array_equal(got, want % t)
    # a prompt: token i's features are its index, so that a diagonal's slot 0 of block i shows i * j for the key token j it holds
    ids = np.zeros((B, d), dtype=np.int64)
    ids[:, 0] = np.arange(1, B + 1)
    q = cl.encrypt_slots(ids.reshape(-1))
    gks = {e: cl.galois_key(e) for e in attention.required_galois(n, d)}
    diag = attention.prefill_qk(orc, q, q, cl.relin_key(), gks, d)
    far = np.arange(B)[:, None] * 0 + 7000 + np.arange(B)[:, None]           # a bucket for every distance
    for u in (0, 1, B // 2, B - 1):
        v = attention.prompt_bias_values(n, d, u, far, list(range(B)), 0)[::d]
        j = cl.decrypt_slots(diag[u])[::d] // np.arange(1, B + 1) - 1
        want = np.where(np.arange(B) >= j, 7000 + np.arange(B) - j, 0)
        assert np.array_equal(v, want), u


@pytest.mark.parametrize("log2n,d", [(6, 2), (7, 8), (8, 16), (8, 64), (10, 256)])
def test_slots_at_the_blocks_starts_make_two_short_transforms(log2n, d):
    """The polynomial of slots b d alone is N^-1 (A_(j mod n') zeta^-j + B_(j mod n') zeta^j), n' = N / (2 d): A and B the transforms of
    n' points of the two rows' values, e = 3^(d b) being 1 + 4 d k."""
    t, n = 65537, 1 << log2n
    zeta, np_ = min_psi(n, t), n // (2 * d)
    rng = np.random.default_rng(d)
    v = rng.integers(0, t, (2, np_))
    index = [(pow(3, d * b, 2 * n) - 1) // (4 * d) for b in range(np_)]
    assert sorted(index) == list(range(np_)) and all((pow(3, d * b, 2 * n) - 1) % (4 * d) == 0 for b in range(np_))
    omega = pow(zeta, 4 * d, t)
    A = [sum(int(v[0][b]) * pow(omega, -i * index[b], t) for b in range(np_)) % t for i in range(np_)]
    B = [sum(int(v[1][b]) * pow(omega, i * index[b], t) for b in range(np_)) % t for i in range(np_)]
    got = [pow(n, -1, t) * (A[j % np_] * pow(zeta, -j, t) + B[j % np_] * pow(zeta, j, t)) % t for j in range(n)]

    class Params:
        pass
    prm = Params()
    prm.n, prm.t = n, t
    slots = np.zeros(n, dtype=np.int64)
    slots[:n // 2:d], slots[n // 2::d] = v[0], v[1]
    assert np.array_equal(np.array(got, dtype=np.uint64), SlotCodec(prm).encode(slots))


@pytest.mark.parametrize("n,d1,d2", [(4096, 100, 64), (8192, 768, 64), (8192, 300, 4), (4096, 2048, 32)])
def test_a_blocks_slots_of_a_diagonal_lie_in_one_row_of_the_skewed_matrix(n, d1, d2):
    """M laid out by (feature - column) mod tile: a block of d2 slots of a diagonal reads one row, up to the wrap at a slot row's end."""
    D1, _, C = attention.cpvm_shape(n, d1, d2)
    f, half, s = attention.cpvm_feature_of_slot(n, d1, d2), n // 2, np.arange(n)
    for c in range(C):
        shown = f[(s // half) * half + (s % half + c) % half]
        row = ((shown - s % d2) % D1).reshape(-1, d2)
        whole = np.ones(row.shape[0], dtype=bool)
        whole[half // d2 - 1::half // d2] = c == 0           # the last block of either slot row
        tiles = np.arange(row.shape[0]) * d2 % D1 == D1 - d2  # ... and of a tile, where the next tile's shift begins
        whole &= ~tiles | (c == 0)
        assert (row[whole] == row[whole][:, :1]).all(), c
