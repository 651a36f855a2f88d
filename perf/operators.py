"""The operators of a server of many requests: what a model has learned, brought to encrypted tokens.

kinds
  slots    plaintext slot values encoded: the polynomial (slots_encode) or its prepared form (slots_prepare)
  weights  the diagonals of projection matrices, of low-rank adapters, or of their sums (cpvm_prepare)
  project  the tokens of several requests times a layer's matrices, each with the adapter it asks for (cpvm_requests)
  bias     a learned relative position bias by buckets added to every request's scores (score_bias)
  prompt   the same added to the diagonals of a prompt's Q K^T (prompt_bias)
  append   every request's new rows into its caches, at its own length (kv_append_requests)

Ciphertexts, keys and block masks are uniform residues, as fresh ones look to every kernel; weights, adapters and
biases are 8-bit integers, what a quantised model holds.  Parameter sets: N = 4096, 8192 and 16384 with 2, 3 and 6
primes, the shapes around 12 heads of 64 and a hidden size of 768 or 1024.
"""
import math

import torch

own = False

DEVICE = "cuda"
_B = 1 << 50


class _Params:
    """A parameter set: ciphertext primes q, special primes p, plaintext modulus t, primes per digit alpha."""

    def __init__(self, log2n, q, p, alpha):
        self.log2n, self.q, self.p, self.alpha, self.t = log2n, q, p, alpha, 65537
        self.n, self.k, self.nsp, self.dnum = 1 << log2n, len(q), len(p), len(q) // alpha


PARAMS = {
    "n4096": _Params(12, (_B - 16383, _B - 212991), (_B - 417791,), 1),
    "n8192": _Params(13, (_B - 16383, _B - 212991, _B - 1097727), (_B - 1490943,), 1),
    "n16384": _Params(14, (_B - 2162687, _B - 2850815, _B - 3014655, _B - 3047423, _B - 3342335, _B - 3735551),
                      (_B - 4718591, _B - 5177343), 2),
}
ROUND_BITS = 3      # bits per round of the folding sums


# ---- cases ----------------------------------------------------------------------------------------------------
def listed():
    return [
        # one block mask of the small ring: the smallest call there is
        {"name": "slots_one_n4096", "kind": "slots", "params": "n4096", "batch": 1, "prepared": True},
        # the block masks of a cache at d = 64, all 128 of them
        {"name": "slots_128_masks", "kind": "slots", "params": "n8192", "batch": 128, "prepared": True},
        # one head's matrix alone, as a layer that is brought in piece by piece
        {"name": "weights_one_matrix_n4096", "kind": "weights", "params": "n4096", "units": 1, "d1": 768, "d2": 64, "base": True,
         "rank": 0, "a_group": 1},
        # an adapter of rank 16 for a layer's Q, K and V: three down-projections, each shared by 12 heads
        {"name": "weights_adapter_rank16", "kind": "weights", "params": "n8192", "units": 36, "d1": 768, "d2": 64, "base": False,
         "rank": 16, "a_group": 12},
        # one sequence, one head's Q, K and V with an adapter: few launches' worth of work
        {"name": "project_1x3", "kind": "project", "params": "n8192", "requests": 1, "units": 3, "d1": 768, "d2": 64, "adapters": 1},
        # sixteen requests with sixteen adapters through a whole layer's 36 matrices
        {"name": "project_16x36", "kind": "project", "params": "n8192", "requests": 16, "units": 36, "d1": 768, "d2": 64, "adapters": 16},
        # one request, one head, one cache ciphertext
        {"name": "bias_1x1x1", "kind": "bias", "params": "n8192", "requests": 1, "heads": 1, "n_cts": 1, "d2": 64, "buckets": 32},
        # eight requests of 12 heads, up to 512 tokens each at its own position
        {"name": "bias_8x12x4", "kind": "bias", "params": "n8192", "requests": 8, "heads": 12, "n_cts": 4, "d2": 64, "buckets": 32},
        # a prompt of 32 tokens of d = 128 at the small ring, one head
        {"name": "prompt_1x1_n4096", "kind": "prompt", "params": "n4096", "prompts": 1, "heads": 1, "d2": 128, "buckets": 16},
        # a prompt of 128 tokens, 12 heads: 1536 diagonals
        {"name": "prompt_1x12", "kind": "prompt", "params": "n8192", "prompts": 1, "heads": 12, "d2": 64, "buckets": 32},
        # one request with one head: a K and a V row
        {"name": "append_1x2_n4096", "kind": "append", "params": "n4096", "requests": 1, "per": 2, "stride": 2, "d2": 64},
        # 32 requests of 12 heads, each at its own length; some are full or not in use
        {"name": "append_32x24", "kind": "append", "params": "n8192", "requests": 32, "per": 24, "stride": 4, "d2": 64},
    ]


def _spread(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["slots", "weights", "weights", "project", "project", "bias", "prompt", "append", "append"])
    params = rng.choice(["n4096", "n8192", "n8192", "n16384"])
    big = {"n4096": 1, "n8192": 1, "n16384": 4}[params]
    case = {"kind": kind, "params": params}
    if kind == "slots":
        case.update(batch=_spread(rng, 1, 400 // big), prepared=rng.random() < 0.7)
    elif kind in ("weights", "project"):
        d1, d2 = _spread(rng, 48, 2048), rng.choice([32, 64, 64, 128])
        case.update(d1=d1, d2=d2)
        if kind == "weights":
            rank = rng.choice([0, _spread(rng, 1, 64)])
            case.update(units=_spread(rng, 1, 24 // big), base=rank == 0 or rng.random() < 0.5, rank=rank, a_group=rng.randint(1, 12))
        else:
            requests = _spread(rng, 1, 16 // big)
            case.update(requests=requests, units=_spread(rng, 1, min(24, 160 // (big * requests))), adapters=rng.randint(0, 4 // big))
    elif kind == "bias":
        case.update(requests=_spread(rng, 1, 24 // big), heads=rng.randint(1, 16), n_cts=rng.randint(1, 4), d2=rng.choice([32, 64, 64, 128]),
                    buckets=_spread(rng, 1, 64))
    elif kind == "prompt":
        case.update(prompts=1, heads=_spread(rng, 1, 12 // big), d2=rng.choice([64, 64, 128]), buckets=_spread(rng, 1, 64))
    else:
        case.update(requests=_spread(rng, 1, 24 // big), per=2 * rng.randint(1, 12), stride=rng.randint(1, 3), d2=rng.choice([32, 64, 64, 128]))
    return case


# ---- arithmetic of the plain form: residues in int64, products with a quotient from float64 ------------------------
def _mul(a, b, p):
    """a b mod p for residues below p < 2^50: the quotient is right to one, what is left fits 64 bits."""
    c = torch.round(a.double() * b.double() / p.double()).long()
    r = a * b - c * p
    return torch.where(r < 0, r + p, r)


def _add(a, b, p):
    s = a + b
    return torch.where(s >= p, s - p, s)


def _sub(a, b, p):
    s = a - b
    return torch.where(s < 0, s + p, s)


def _ntt(x, tab):
    """x [..., rows, N] modulo the rows' primes -> values at psi^(2 bitrev(j) + 1)"""
    p, w, n, m = tab["p"], tab["w"], x.shape[-1], 1
    while m < n:
        v = x.reshape(*x.shape[:-1], m, 2, n // (2 * m))
        lo, hi = v[..., 0, :], _mul(v[..., 1, :], w[:, m:2 * m, None], p[:, None])
        x = torch.stack((_add(lo, hi, p[:, None]), _sub(lo, hi, p[:, None])), -2).reshape(x.shape)
        m *= 2
    return x


def _intt(x, tab):
    p, w, n = tab["p"], tab["iw"], x.shape[-1]
    m = n // 2
    while m:
        v = x.reshape(*x.shape[:-1], m, 2, n // (2 * m))
        lo, hi = v[..., 0, :], v[..., 1, :]
        x = torch.stack((_add(lo, hi, p[:, None]), _mul(_sub(lo, hi, p[:, None]), w[:, m:2 * m, None], p[:, None])), -2).reshape(x.shape)
        m //= 2
    return _mul(x, tab["ninv"], p)


# ---- tables that a program keeps ---------------------------------------------------------------------------------
_KEPT = {}


def _root(n, p):
    """the smallest primitive 2n-th root of unity modulo the prime p"""
    x = next(g for g in range(2, 1000) if pow(g, (p - 1) // 2, p) == p - 1)
    r = pow(x, (p - 1) // (2 * n), p)
    sq, best, cur = r * r % p, r, r
    for _ in range(n - 1):
        cur = cur * sq % p
        best = min(best, cur)
    return best


def _table(n, primes):
    bits = n.bit_length() - 1
    rev = torch.tensor([int(format(i, "0%db" % bits)[::-1], 2) for i in range(n)], device=DEVICE)
    p = torch.tensor(primes, device=DEVICE)[:, None]

    def powers(bases):
        w, at = torch.ones(len(primes), 1, dtype=torch.int64, device=DEVICE), 1
        while at < n:
            step = torch.tensor([pow(b, at, q) for b, q in zip(bases, primes)], device=DEVICE)[:, None]
            w, at = torch.cat((w, _mul(w, step.expand_as(w), p)), 1), 2 * at
        return w[:, rev]

    psi = [_root(n, q) for q in primes]
    ninv = torch.tensor([pow(n, -1, q) for q in primes], device=DEVICE)[:, None]
    return {"p": p, "w": powers(psi), "iw": powers([pow(x, -1, q) for x, q in zip(psi, primes)]), "ninv": ninv, "rev": rev}


class _Ring:
    """The plain form's tables of one parameter set."""

    def __init__(self, prm):
        self.prm = prm
        n, L = prm.n, prm.k + prm.nsp
        self.qp = _table(n, list(prm.q) + list(prm.p))
        self.q = {x: (y if x == "rev" else y[:prm.k]) for x, y in self.qp.items()}
        self.t = _table(n, [prm.t])
        pw, e = 1, []
        for _ in range(n // 2):
            e.append(pw)
            pw = pw * 3 % (2 * n)
        # slot s is the value at zeta^e, e = 3^i in row 0 and -3^i in row 1: its place among the transform's outputs
        e = torch.tensor(e + [2 * n - x for x in e], device=DEVICE)
        self.place = self.t["rev"][(e - 1) // 2]
        delta = math.prod(prm.q) // prm.t
        self.delta = torch.tensor([delta % q for q in prm.q], device=DEVICE)[:, None]
        self.primes = list(prm.q) + list(prm.p)
        self.P = math.prod(prm.p)
        self.half = torch.tensor([self.P // 2 % m for m in self.primes], device=DEVICE)[:, None]
        self.pinv = torch.tensor([pow(self.P, -1, q) for q in prm.q], device=DEVICE)[:, None]
        self.L = L

    def map_values(self, g):
        """where the transform of X -> X^g takes its values from"""
        n = self.prm.n
        e = (2 * self.t["rev"] + 1) * g % (2 * n)
        return self.t["rev"][(e - 1) // 2]

    def map_ring(self, x, g):
        """X -> X^g on coefficients modulo the ciphertext primes"""
        n = self.prm.n
        e = torch.arange(n, device=DEVICE) * pow(g, -1, 2 * n) % (2 * n)
        y = x[..., e % n]
        # coefficient i comes from i / g, with the sign of that power
        return torch.where(e >= n, _sub(torch.zeros_like(y), y, self.q["p"]), y)


def _ring(name):
    if name not in _KEPT:
        _KEPT[name] = _Ring(PARAMS[name])
    return _KEPT[name]


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _encode(ring, slots):
    """slot values [..., N], any representatives -> polynomials with coefficients in [0, t)"""
    ev = torch.empty_like(slots)
    ev[..., ring.place] = slots % ring.prm.t
    return _intt(ev[..., None, :], ring.t)[..., 0, :]


def _lift(ring, poly):
    """polynomials mod t -> transforms of their centred lifts [..., k, N]"""
    t = ring.prm.t
    x = torch.where(poly > (t - 1) // 2, poly - t, poly)
    return _ntt(x[..., None, :] % ring.q["p"], ring.q)


def _centred(ring, x):
    """prepared form: canonical residues as float64, |x| <= p / 2"""
    return torch.where(x > ring.q["p"] // 2, x - ring.q["p"], x).double()


def _shape(prm, d1, d2):
    """(tile length, number of diagonals) of a projection"""
    tile = 1
    while tile < max(d1, d2, prm.n // d2):
        tile *= 2
    return tile, d2 * tile // prm.n


def _diagonals(ring, w, a, b, a_group, d1, d2):
    """slot values [units][n_diag][N] of the matrices W + A B"""
    prm = ring.prm
    tile, n_diag = _shape(prm, d1, d2)
    units = (w if w is not None else b).shape[0]
    m = torch.zeros(units, tile, d2, dtype=torch.int64, device=DEVICE)
    if w is not None:
        m[:, :d1] += w
    if a is not None:
        of = torch.arange(units, device=DEVICE) // a_group
        m[:, :d1] += torch.matmul(a.double()[of], b.double()).long()     # |entries| < 2^53: exact
    n, half = prm.n, prm.n // 2
    s, c = torch.arange(n, device=DEVICE), torch.arange(n_diag, device=DEVICE)[:, None]
    at = s // half * half + (s % half + c) % half
    feature = (at % tile + n_diag * (at // tile)) % tile
    return m[:, feature, s % d2]


def _digits(ring, c1):
    """ring elements [..., k, N] -> their digits modulo all primes, transformed: [..., dnum, L, N]"""
    prm, p = ring.prm, ring.qp["p"]
    x = c1.reshape(*c1.shape[:-2], prm.dnum, prm.alpha, 1, prm.n)
    d = x[..., 0, :, :] % p
    if prm.alpha == 2:
        qa, qb = torch.tensor(prm.q[0::2], device=DEVICE)[:, None, None], torch.tensor(prm.q[1::2], device=DEVICE)[:, None, None]
        inv = torch.tensor([pow(a, -1, b) for a, b in zip(prm.q[0::2], prm.q[1::2])], device=DEVICE)[:, None, None]
        high = _mul((x[..., 1, :, :] - x[..., 0, :, :]) % qb, inv, qb)
        d = _add(d, _mul(high % p, qa % p, p), p)
    return _ntt(d, ring.qp)


def _divide(ring, acc):
    """accumulators [..., L, N] in transformed form -> floor((A + floor(P / 2)) / P) modulo the ciphertext primes"""
    prm, q, k = ring.prm, ring.q["p"], ring.prm.k
    x = _add(_intt(acc, ring.qp), ring.half, ring.qp["p"])
    low = x[..., k:k + 1, :] % q
    if prm.nsp == 2:
        p0, p1 = prm.p
        pt = torch.tensor([p1], device=DEVICE)
        high = _mul((x[..., k + 1:, :] - x[..., k:k + 1, :]) % pt, torch.tensor([pow(p0, -1, p1)], device=DEVICE), pt)
        low = _add(low, _mul(high % q, p0 % q, q), q)
    return _mul(_sub(x[..., :k, :], low, q), ring.pinv, q)


def _inner(ring, digits, g, key):
    """digits [..., dnum, L, N] mapped by X -> X^g times a key [dnum, 2, L, N], summed: [..., 2, L, N]"""
    d = digits[..., ring.map_values(g)]
    return _mul(d[..., :, None, :, :], key, ring.qp["p"]).sum(-4) % ring.qp["p"]


def _rotate(ring, x, digits, g, key):
    u = _divide(ring, _inner(ring, digits, g, key))
    return torch.stack((_add(ring.map_ring(x[..., 0, :, :], g), u[..., 0, :, :], ring.q["p"]), u[..., 1, :, :]), -3)


def _round(ring, x, gs, keys):
    """a ciphertext and its rotations by gs, with one division"""
    digits, q = _digits(ring, x[..., 1, :, :]), ring.q["p"]
    acc, c0 = None, x[..., 0, :, :]
    for g, key in zip(gs, keys):
        part = _inner(ring, digits, g, key)
        acc = part if acc is None else _add(acc, part, ring.qp["p"])
        c0 = _add(c0, ring.map_ring(x[..., 0, :, :], g), q)
    u = _divide(ring, acc)
    return torch.stack((_add(c0, u[..., 0, :, :], q), _add(x[..., 1, :, :], u[..., 1, :, :], q)), -3)


def _rounds(prm, d2):
    """Galois elements of every round of the sum over residue classes modulo d2"""
    two_n, gens, sh = 2 * prm.n, [], d2
    while sh <= prm.n // 4:
        gens.append(pow(3, sh, two_n))
        sh *= 2
    gens.append(two_n - 1)
    count = -(-len(gens) // ROUND_BITS)
    lo, extra = divmod(len(gens), count)
    out = []
    for r in range(count):
        size = lo + (r < extra)
        mine, gens = gens[:size], gens[size:]
        out.append([math.prod(g for i, g in enumerate(mine) if m >> i & 1) % two_n for m in range(1, 1 << size)])
    return out


def _project(ring, s):
    prm, q = ring.prm, ring.q["p"]
    x, n_diag = s["x"], s["n_diag"]
    digits = _digits(ring, x[:, 1])
    copies = [x] + [_rotate(ring, x, digits, pow(3, c, 2 * prm.n), s["copies"][c - 1]) for c in range(1, n_diag)]
    total = None
    for c, copy in enumerate(copies):
        w = s["diags"][None, :, c]
        if s["adapters"] is not None:
            pick = s["pick"].long()
            has = (pick >= 0) & (pick < s["adapters"].shape[0])
            extra = s["adapters"][torch.where(has, pick, 0)][:, :, c]
            w = _add(w, torch.where(has[:, None, None, None], extra, 0), q)
        part = _mul(_ntt(copy, ring.q)[:, None], w.unsqueeze(2), q)
        total = part if total is None else _add(total, part, q)
    y = _intt(total, ring.q)
    for gs, keys in zip(s["rounds"], s["block"]):
        y = _round(ring, y, gs, keys)
    return y


def _bucket_values(dist, seen, s):
    """biases [..., heads] of distances: the table's row of the last bucket that begins at or below them"""
    at = torch.bucketize(dist, s["edges"].long(), right=True) - 1
    return torch.where((seen & (at >= 0))[..., None], s["table"][at.clamp(min=0)], 0)


def _add_slots(ring, cts, slots):
    """c0 of the ciphertexts + Delta times the encoded slots, in place"""
    m = _encode(ring, slots)[..., None, :]
    cts[..., 0, :, :] = _add(cts[..., 0, :, :], _mul(m.expand(*m.shape[:-2], ring.prm.k, -1), ring.delta, ring.q["p"]), ring.q["p"])
    return cts


def _bias(ring, s):
    prm, d2 = ring.prm, s["case"]["d2"]
    blocks = prm.n // d2
    R, H, C = s["scores"].shape[:3]
    dist = s["pos"].long()[:, None] - torch.arange(C * blocks, device=DEVICE)
    v = _bucket_values(dist, dist >= 0, s).reshape(R, C, blocks, H).permute(0, 3, 1, 2)
    slots = torch.zeros(R, H, C, prm.n, dtype=torch.int64, device=DEVICE)
    slots[..., ::d2] = v
    return _add_slots(ring, s["scores"], slots)


def _prompt(ring, s):
    prm, d2 = ring.prm, s["case"]["d2"]
    m = prm.n // d2
    half = m // 2
    i, unit = torch.arange(m, device=DEVICE), torch.arange(m, device=DEVICE)[:, None]
    j = ((i // half) ^ (unit // half)) * half + (i % half + unit % half) % half
    slots = torch.zeros(s["case"]["heads"], m, prm.n, dtype=torch.int64, device=DEVICE)
    slots[..., ::d2] = _bucket_values(i - j, i >= j, s).permute(2, 0, 1)
    return _add_slots(ring, s["scores"], slots[None])


def _append(ring, s):
    case, q = s["case"], ring.q["p"]
    blocks = ring.prm.n // case["d2"]
    lens = s["lens"].long()
    at, block = lens // blocks, lens % blocks
    fine = (lens >= 0) & (at < case["stride"])
    at, r = torch.where(fine, at, 0), torch.arange(len(lens), device=DEVICE)
    new = _intt(_mul(_ntt(s["rows"], ring.q), s["masks"][block][:, None, None], q), ring.q)
    old = s["cache"][r, :, at]
    wide = (slice(None),) + (None,) * 4
    s["cache"][r, :, at] = torch.where(fine[wide], torch.where((block == 0)[wide], new, _add(old, new, q)), old)
    return s["cache"]


# ---- inputs ----------------------------------------------------------------------------------------------------------
class _Draws:
    def __init__(self, prm, seed):
        self.prm, self.g = prm, torch.Generator(device=DEVICE)
        self.g.manual_seed(seed)

    def ints(self, lo, hi, *shape, dtype=torch.int64):
        return torch.randint(lo, hi, shape, generator=self.g, device=DEVICE, dtype=dtype)

    def residues(self, primes, *lead):
        return torch.stack([self.ints(0, p, *lead, self.prm.n) for p in primes], len(lead))

    def cts(self, *lead):
        return self.residues(self.prm.q, *lead, 2)

    def keys(self, count):
        """switching keys as generated, [count][dnum][2][L][N]"""
        return self.residues(list(self.prm.q) + list(self.prm.p), count, self.prm.dnum, 2)


def _edges(buckets):
    """First distance of every bucket: one each for the nearest, then wider and wider ones."""
    near = (buckets + 1) // 2
    return [i if i < near else int(near * (512 / near) ** ((i - near + 1) / (buckets - near + 1))) + i - near for i in range(buckets)]


def _inputs(case, seed):
    """The inputs as they are before either side lays anything out."""
    prm = PARAMS[case["params"]]
    r, s, kind = _Draws(prm, seed), {}, case["kind"]
    if kind == "slots":
        s["slots"] = r.ints(-128, 128, case["batch"], prm.n)
    elif kind == "weights":
        s.update(_matrices(r, case, case["units"], case["base"], case["rank"], case["a_group"]))
    elif kind == "project":
        _, n_diag = _shape(prm, case["d1"], case["d2"])
        R, U = case["requests"], case["units"]
        s["x"] = r.cts(R)
        s["base"] = _matrices(r, case, U, True, 0, 1)
        s["low"] = [_matrices(r, case, U, False, 8, -(-U // 3)) for _ in range(case["adapters"])]
        # every request has an adapter of its own where there are as many, some have none
        s["pick"] = (torch.randperm(R, generator=r.g, device=DEVICE) - (0 if case["adapters"] == R else 1)).int()
        s["rounds"] = _rounds(prm, case["d2"])
        s["raw_copies"], s["raw_block"] = r.keys(n_diag - 1), [r.keys(len(g)) for g in s["rounds"]]
        s["n_diag"] = n_diag
    elif kind in ("bias", "prompt"):
        blocks = prm.n // case["d2"]
        if kind == "bias":
            s["scores"] = r.cts(case["requests"], case["heads"], case["n_cts"])
            s["pos"] = r.ints(0, case["n_cts"] * blocks, case["requests"], dtype=torch.int32)
        else:
            s["scores"] = r.cts(case["prompts"], case["heads"], blocks)
        s["table"] = r.ints(-128, 128, case["buckets"], case["heads"])
        s["edges"] = torch.tensor(_edges(case["buckets"]), dtype=torch.int32, device=DEVICE)
    else:
        blocks = prm.n // case["d2"]
        s["cache"] = r.cts(case["requests"], case["per"], case["stride"])
        s["rows"] = r.cts(case["requests"], case["per"])
        # one request in eight or so is not in use, or full
        lens = r.ints(0, case["stride"] * blocks, case["requests"], dtype=torch.int32)
        lens[5::16] = -1
        lens[11::16] = case["stride"] * blocks
        s["lens"] = lens
        s["mask_slots"] = torch.zeros(blocks, prm.n, dtype=torch.int64, device=DEVICE)
        for b in range(blocks):
            s["mask_slots"][b, b * case["d2"]:(b + 1) * case["d2"]] = 1
    return s


def _matrices(r, case, units, base, rank, a_group):
    d1, d2 = case["d1"], case["d2"]
    return {"w": r.ints(-128, 128, units, d1, d2) if base else None,
            "a": r.ints(-128, 128, -(-units // a_group), d1, rank) if rank else None,
            "b": r.ints(-128, 128, units, rank, d2) if rank else None, "a_group": a_group}


_CONTEXTS = {}


def _context(name):
    """A program holds one context, and what goes with it, for as long as it runs."""
    import paper_2602_08798_amd as P
    if name not in _CONTEXTS:
        ctx = P.Context(PARAMS[name])
        _CONTEXTS[name] = ctx, P.Requests(ctx)
    return _CONTEXTS[name]


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind, d1, d2 = case["kind"], case.get("d1"), case.get("d2")
    if own:
        # what a program lays out once: keys and weights in the library's prepared form
        s["ctx"], s["rq"] = ctx, rq = _context(case["params"])
        if kind == "project":
            U, n_diag = case["units"], s["n_diag"]
            s["copies"] = [ctx.ksk_prepare(x) for x in s.pop("raw_copies")]
            s["block"] = [ctx.ksk_prepare(x) for x in torch.cat(s.pop("raw_block"))]
            s["diags"] = rq.cpvm_prepare(U, d1, d2, w=s.pop("base")["w"])
            low = s.pop("low")
            s["adapters"] = torch.empty(len(low), U * n_diag * ctx.k * ctx.n, dtype=torch.float64, device=DEVICE) if low else None
            for i, m in enumerate(low):
                rq.cpvm_prepare(U, d1, d2, a=m["a"], b=m["b"], a_group=m["a_group"], out=s["adapters"][i])
        if kind == "append":
            s["masks"] = rq.slots_prepare(s.pop("mask_slots"))
    else:
        s["ring"] = ring = _ring(case["params"])
        if kind == "project":
            s["copies"] = [_ntt(x, ring.qp) for x in s.pop("raw_copies")]
            s["block"] = [_ntt(x, ring.qp) for x in s.pop("raw_block")]
            s["diags"] = _plain_diagonals(ring, s.pop("base"), d1, d2)
            low = s.pop("low")
            s["adapters"] = torch.stack([_plain_diagonals(ring, m, d1, d2) for m in low]) if low else None
        if kind == "append":
            s["masks"] = _lift(ring, _encode(ring, s.pop("mask_slots")))
    return s


def _plain_diagonals(ring, m, d1, d2):
    return _lift(ring, _encode(ring, _diagonals(ring, m["w"], m["a"], m["b"], m["a_group"], d1, d2)))


def run(s):
    case = s["case"]
    kind, d1, d2 = case["kind"], case.get("d1"), case.get("d2")
    if own:
        rq = s["rq"]
        if kind == "slots":
            return rq.slots_prepare(s["slots"]) if case["prepared"] else rq.slots_encode(s["slots"])
        if kind == "weights":
            return rq.cpvm_prepare(case["units"], d1, d2, w=s["w"], a=s["a"], b=s["b"], a_group=s["a_group"])
        if kind == "project":
            return rq.cpvm_requests(s["x"], s["diags"], case["requests"], case["units"], s["n_diag"], d2, s["copies"], s["block"],
                                    adapters=s["adapters"], pick=s["pick"], block_round_bits=ROUND_BITS)
        if kind == "bias":
            return rq.score_bias(s["scores"], case["requests"], case["heads"], case["n_cts"], d2, s["pos"], s["table"], s["edges"],
                                 out=s["scores"])
        if kind == "prompt":
            return rq.prompt_bias(s["scores"], case["prompts"], case["heads"], d2, s["table"], s["edges"], out=s["scores"])
        rq.kv_append_requests(s["cache"], case["stride"], case["requests"], case["per"], s["lens"], s["rows"], s["masks"], d2)
        return s["cache"]
    ring = s["ring"]
    if kind == "slots":
        m = _encode(ring, s["slots"])
        return _centred(ring, _lift(ring, m)).reshape(-1) if case["prepared"] else m
    if kind == "weights":
        return _centred(ring, _plain_diagonals(ring, s, d1, d2)).reshape(-1)
    return {"project": _project, "bias": _bias, "prompt": _prompt, "append": _append}[kind](ring, s)


# ---- from the definitions, without transforms modulo primes ------------------------------------------------------------
def _halve(x, m):
    """residues -> centred representatives"""
    return torch.where(x > m // 2, x - m, x)


def _by_constant(x, c, m):
    """x c mod m for residues below 2^50, twelve bits of the constant at a time"""
    acc = torch.zeros_like(x)
    for i in range(60, -1, -12):
        acc = ((acc << 12) % m + x * ((c >> i) & 4095)) % m
    return acc


def _interpolate(prm, slots):
    """The polynomials mod t with the given slot values: the defining sum over the slots, as products with a matrix of
    powers of zeta in float64 (entries below 2^17 each: sums below 2^48)."""
    n, t = prm.n, prm.t
    zeta, pw, e = _root(n, t), 1, []
    for _ in range(n // 2):
        e.append(pw)
        pw = pw * 3 % (2 * n)
    e = torch.tensor(e + [-x for x in e], device=DEVICE)
    powers = torch.tensor([pow(zeta, i, t) for i in range(2 * n)], device=DEVICE).double()
    v, i = slots.reshape(-1, n).remainder(t).double(), torch.arange(n, device=DEVICE)
    out = [torch.remainder(v @ powers[(-e[:, None] * i[at:at + 1024]) % (2 * n)], t) for at in range(0, n, 1024)]
    return torch.remainder(torch.cat(out, 1) * pow(n, -1, t), t).long().reshape(slots.shape)


def _evaluate(prm, polys):
    """Prepared forms of polynomials mod t: their centred lifts at psi^(2 bitrev(j) + 1), powers of psi in 17-bit pieces."""
    n, bits = prm.n, prm.log2n
    x = _halve(polys.reshape(-1, n), prm.t).double()
    j = torch.tensor([2 * int(format(i, "0%db" % bits)[::-1], 2) + 1 for i in range(n)], device=DEVICE)
    rows = []
    for q in prm.q:
        psi, cur, powers = _root(n, q), 1, []
        for _ in range(2 * n):
            powers.append(cur)
            cur = cur * psi % q
        powers, cols = torch.tensor(powers, device=DEVICE), []
        for at in range(0, n, 1024):
            p = powers[torch.arange(n, device=DEVICE)[:, None] * j[at:at + 1024] % (2 * n)]
            low, mid, high = ((x @ (p >> s & 131071).double()).long() % q for s in (0, 17, 34))
            cols.append((low + _by_constant(mid, 1 << 17, q) + _by_constant(high, 1 << 34, q)) % q)
        rows.append(_halve(torch.cat(cols, 1), q))
    return torch.stack(rows, 1).double()


_PIECE = 13


def _spectrum(x, m):
    """balanced 13-bit pieces of residues modulo m, as spectra of length 2N"""
    x, parts = _halve(x, m), []
    for _ in range(4):
        low = ((x + (1 << (_PIECE - 1))) & ((1 << _PIECE) - 1)) - (1 << (_PIECE - 1))
        parts.append(low)
        x = (x - low) >> _PIECE
    return torch.fft.rfft(torch.stack(parts, -2).double(), n=2 * x.shape[-1])


def _join(acc, a, b):
    """adds the products of two spectra's pieces to acc [..., 7, N + 1]"""
    for i in range(4):
        for j in range(4):
            acc[..., i + j, :] += a[..., i, :] * b[..., j, :]
    return acc


def _gather(acc, n, m):
    """negacyclic products from their spectra, modulo m"""
    c = torch.round(torch.fft.irfft(acc, n=2 * n)).long()
    c, out = c[..., :n] - c[..., n:], 0
    for i in range(6, -1, -1):
        out = ((out * (1 << 12) % m) * 2 + c[..., i, :]) % m if i < 6 else c[..., i, :] % m
    return out


def _sigma(x, g, m):
    """X -> X^g on residues modulo m"""
    n = x.shape[-1]
    e = torch.arange(n, device=DEVICE) * g % (2 * n)
    out = torch.empty_like(x)
    out[..., e % n] = torch.where(e >= n, (m - x) % m, x)
    return out


def _switched(prm, c1, gs, keys):
    """floor((A + P/2) / P) mod q, A the sum over gs of the mapped digits of c1 times the keys: [..., 2, k, N]"""
    primes, n, k = list(prm.q) + list(prm.p), prm.n, prm.k
    sums = []
    for r, m in enumerate(primes):
        acc = torch.zeros(*c1.shape[:-2], 2, 7, n + 1, dtype=torch.complex128, device=DEVICE)
        for j in range(prm.dnum):
            d = c1[..., j * prm.alpha, :] % m
            if prm.alpha == 2:
                qa, qb = prm.q[2 * j:2 * j + 2]
                step = _by_constant((c1[..., 2 * j + 1, :] - c1[..., 2 * j, :]) % qb, pow(qa, -1, qb), qb)
                d = (d + _by_constant(step % m, qa % m, m)) % m
            for g, key in zip(gs, keys):
                _join(acc, _spectrum(_sigma(d, g, m), m)[..., None, :, :], _spectrum(key[j, :, r], m))
        sums.append((_gather(acc, n, m) + math.prod(prm.p) // 2 % m) % m)
    out = []
    for i, q in enumerate(prm.q):
        low = sums[k] % q
        if prm.nsp == 2:
            p0, p1 = prm.p
            low = (low + _by_constant(_by_constant((sums[k + 1] - sums[k]) % p1, pow(p0, -1, p1), p1) % q, p0 % q, q)) % q
        out.append(_by_constant((sums[i] - low) % q, pow(math.prod(prm.p), -1, q), q))
    return torch.stack(out, -2)


def _rotated(prm, c0, g):
    return torch.stack([_sigma(c0[..., i, :], g, q) for i, q in enumerate(prm.q)], -2)


def _exact_project(prm, case, s):
    q = torch.tensor(prm.q, device=DEVICE)[:, None]
    copies = [s["x"]]
    for c in range(1, s["n_diag"]):
        g = pow(3, c, 2 * prm.n)
        u = _switched(prm, s["x"][:, 1], [g], s["raw_copies"][c - 1:c])
        copies.append(torch.stack(((_rotated(prm, s["x"][:, 0], g) + u[:, 0]) % q, u[:, 1]), 1))
    polys = [_interpolate(prm, _exact_slots(prm, case, m)) for m in [s["base"]] + s["low"]]
    R, U = case["requests"], case["units"]
    y = torch.empty(R, U, 2, prm.k, prm.n, dtype=torch.int64, device=DEVICE)
    pick = s["pick"].tolist()
    for i, m in enumerate(prm.q):
        for u in range(U):
            acc = torch.zeros(R, 2, 7, prm.n + 1, dtype=torch.complex128, device=DEVICE)
            for c in range(s["n_diag"]):
                w = [_halve(x[u, c], prm.t) for x in polys]
                w = torch.stack([(w[0] + (w[1 + a] if 0 <= a < len(s["low"]) else 0)) % m for a in pick])
                _join(acc, _spectrum(copies[c][:, :, i], m), _spectrum(w, m)[:, None])
            y[:, u, :, i] = _gather(acc, prm.n, m)
    y = y.reshape(R * U, 2, prm.k, prm.n)
    for gs, keys in zip(s["rounds"], s["raw_block"]):
        parts = []
        for x in y.split(96 if prm.n < 16384 else 24):
            u, c0 = _switched(prm, x[:, 1], gs, keys), x[:, 0]
            c0 = c0 + sum(_rotated(prm, x[:, 0], g) for g in gs) + u[:, 0]
            parts.append(torch.stack((c0 % q, (x[:, 1] + u[:, 1]) % q), 1))
        y = torch.cat(parts)
    return y.reshape(R, U, 2, prm.k, prm.n)


def _exact_slots(prm, case, m):
    """The diagonals' slot values, one slot of the token's layout at a time."""
    tile, n_diag = _shape(prm, case["d1"], case["d2"])
    n, half = prm.n, prm.n // 2
    units = (m["w"] if m["w"] is not None else m["b"]).shape[0]
    out = torch.zeros(units, n_diag, n, dtype=torch.int64, device=DEVICE)
    for u in range(units):
        full = torch.zeros(case["d1"], case["d2"], dtype=torch.int64, device=DEVICE)
        if m["w"] is not None:
            full += m["w"][u]
        if m["a"] is not None:
            full += (m["a"][u // m["a_group"]][:, :, None] * m["b"][u][None]).sum(1)
        shows = [(s % tile + n_diag * (s // tile)) % tile for s in range(n)] if u == 0 else shows
        for c in range(n_diag):
            f = torch.tensor(shows[c:half] + shows[:c] + shows[half + c:] + shows[half:half + c], device=DEVICE)
            v = full[f.clamp(max=case["d1"] - 1), torch.arange(n, device=DEVICE) % case["d2"]]
            out[u, c] = torch.where(f < case["d1"], v, 0)
    return out


def exact(case, seed):
    prm, s, kind = PARAMS[case["params"]], _inputs(case, seed), case["kind"]
    q = torch.tensor(prm.q, device=DEVICE)[:, None]
    if kind == "slots":
        m = _interpolate(prm, s["slots"])
        return _evaluate(prm, m).reshape(-1) if case["prepared"] else m
    if kind == "weights":
        return _evaluate(prm, _interpolate(prm, _exact_slots(prm, case, s))).reshape(-1)
    if kind == "project":
        return _exact_project(prm, case, s)
    blocks = prm.n // case["d2"]
    if kind == "append":
        masks = _interpolate(prm, s["mask_slots"])
        for r, length in enumerate(s["lens"].tolist()):
            at, b = divmod(length, blocks)
            if length < 0 or at >= case["stride"]:
                continue
            for i, m in enumerate(prm.q):
                acc = torch.zeros(case["per"], 2, 7, prm.n + 1, dtype=torch.complex128, device=DEVICE)
                new = _gather(_join(acc, _spectrum(s["rows"][r, :, :, i], m), _spectrum(_halve(masks[b], prm.t) % m, m)), prm.n, m)
                s["cache"][r, :, at, :, i] = (new + (s["cache"][r, :, at, :, i] if b else 0)) % m
        return s["cache"]
    edges, heads = s["edges"].tolist(), case["heads"]

    def bias(distance, h):
        at = sum(e <= distance for e in edges) - 1
        return table[at][h] if distance >= 0 and at >= 0 else 0

    table, lead = s["table"].tolist(), s["scores"].shape[:3]
    if kind == "bias":
        pos = s["pos"].tolist()
        row = [[[bias(p - j, h) for j in range(case["n_cts"] * blocks)] for h in range(heads)] for p in pos]
    else:
        half = blocks // 2
        row = [[[bias(i - (((i // half) ^ (u // half)) * half + (i % half + u % half) % half), h) for u in range(blocks) for i in range(blocks)]
                for h in range(heads)]]
    slots = torch.zeros(*lead, prm.n, dtype=torch.int64)
    slots[..., ::case["d2"]] = torch.tensor(row).reshape(*lead, blocks)
    m = _interpolate(prm, slots.to(DEVICE))
    delta = math.prod(prm.q) // prm.t
    for i, p in enumerate(prm.q):
        s["scores"][..., 0, i, :] = (s["scores"][..., 0, i, :] + _by_constant(m, delta % p, p)) % p
    return s["scores"]


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    """Bytes: inputs once, outputs once.  Operations: a butterfly is a product (8 in FP64, a fused one counted twice) and
    two sums; modulo t a product is 4."""
    prm = PARAMS[case["params"]]
    n, k, kind, row = prm.n, prm.k, case["kind"], 8 * prm.n
    fly, small = 10 * (n // 2) * prm.log2n, 6 * (n // 2) * prm.log2n       # a row's transform modulo a prime, modulo t
    L, dnum = k + prm.nsp, prm.dnum
    if kind == "slots":
        b = case["batch"]
        return {"bytes": b * row * (1 + (k if case["prepared"] else 1)), "flops": b * (small + (k * fly if case["prepared"] else 0))}
    if kind == "weights":
        U, d1, d2, rank = case["units"], case["d1"], case["d2"], case["rank"]
        rows = U * _shape(prm, d1, d2)[1]
        inputs = (U * d1 * d2 if case["base"] else 0) + -(-U // case["a_group"]) * d1 * rank + U * rank * d2
        return {"bytes": 8 * inputs + rows * k * row, "flops": 2 * U * d1 * d2 * rank + rows * (small + k * fly)}
    if kind == "project":
        R, U, n_diag = case["requests"], case["units"], _shape(prm, case["d1"], case["d2"])[1]
        rounds = [len(g) for g in _rounds(prm, case["d2"])]
        used = min(case["adapters"], R)
        rows = 2 * k * R * (1 + U) + U * n_diag * k * (1 + used) + 2 * dnum * L * (n_diag - 1 + sum(rounds))
        transforms = R * (dnum * L + 2 * L * (n_diag - 1)) + 2 * k * R * n_diag + 2 * k * R * U + R * U * len(rounds) * (dnum + 2) * L
        products = R * (n_diag - 1) * 2 * (dnum * L + k) + R * U * 2 * k * n_diag + R * U * 2 * (sum(rounds) * dnum * L + len(rounds) * k)
        return {"bytes": rows * row, "flops": transforms * fly + 8 * products * n}
    if kind in ("bias", "prompt"):
        units = case["requests"] * case["heads"] * case["n_cts"] if kind == "bias" else case["prompts"] * case["heads"] * (n // case["d2"])
        return {"bytes": units * 2 * k * row, "flops": units * n * (4 * 2 + 10 * k)}
    # (each request's row of the masks is one of blocks at most)
    units = case["requests"] * case["per"]
    rows = units * 2 * k * 3 + min(case["requests"], n // case["d2"]) * k
    return {"bytes": rows * row, "flops": units * 2 * k * (2 * fly + 8 * n)}
