// libcryptogen_requests.so (see include/cryptogen_requests.h): tables, argument checks and launch sequences.
// Rotations go through the evaluator's public entry points.
#include "../../include/cryptogen_requests.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <initializer_list>
#include <new>
#include <tuple>
#include <vector>

// the row transforms are this library's own copies: nothing of them is exported beside the evaluator's
namespace {
#include "requests.hpp"
}
using namespace cgr;

#define CG_REQUIRE(cond) do { if (!(cond)) return CG_EINVAL; } while (0)
#define CG_TRY(expr) do { int rc_ = (expr); if (rc_ != CG_OK) return rc_; } while (0)
#define CG_API extern "C" __attribute__((visibility("default")))

struct cg_req {
    cg_ctx *ctx;
    int logn, N, k, nsp, device, n_cu;
    void *mem;            // every table
    Tables T;
};

namespace {
typedef unsigned __int128 u128;
uint64_t mul_mod(uint64_t a, uint64_t b, uint64_t m) { return (uint64_t)((u128)a * b % m); }
uint64_t pow_mod(uint64_t a, uint64_t e, uint64_t m)
{
    uint64_t r = 1;
    for (a %= m; e; e >>= 1, a = mul_mod(a, a, m))
        if (e & 1) r = mul_mod(r, a, m);
    return r;
}
uint64_t inverse_mod(uint64_t a, uint64_t m) { return pow_mod(a, m - 2, m); }
double centred(uint64_t x, uint64_t m) { return x > m / 2 ? -(double)(m - x) : (double)x; }
bool small_prime(uint64_t n)
{
    if (n < 3 || n % 2 == 0) return false;
    for (uint64_t d = 3; d * d <= n; d += 2)
        if (n % d == 0) return false;
    return true;
}
// the smallest primitive 2n-th root of unity modulo the prime p = 1 mod 2n (n a power of two); 0: none found
uint64_t smallest_root(uint64_t n, uint64_t p)
{
    for (uint64_t g = 2; g < 2000; g++) {
        const uint64_t r = pow_mod(g, (p - 1) / (2 * n), p);
        if (pow_mod(r, n, p) != p - 1) continue;
        uint64_t best = r, cur = r;
        const uint64_t sq = mul_mod(r, r, p);
        for (uint64_t i = 1; i < n; i++) {
            cur = mul_mod(cur, sq, p);
            best = std::min(best, cur);
        }
        return best;
    }
    return 0;
}
uint32_t reversed(uint32_t x, int bits)
{
    uint32_t r = 0;
    for (int i = 0; i < bits; i++) r |= ((x >> i) & 1) << (bits - 1 - i);
    return r;
}
bool aligned(const void *p, uintptr_t to = 16) { return p && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool all_aligned(std::initializer_list<const void *> ps)
{
    for (const void *p : ps) if (!aligned(p)) return false;
    return true;
}
bool overlap(const void *a, size_t na, const void *b, size_t nb)
{
    const char *x = static_cast<const char *>(a), *y = static_cast<const char *>(b);
    return x < y + nb && y < x + na;
}
bool power_of_two(uint32_t x) { return x && !(x & (x - 1)); }
int log2_of(uint32_t x) { int l = 0; while (x >>= 1) l++; return l; }
bool in_one_call(uint64_t units) { return units >= 1 && units <= (1u << 16); }
bool here(const cg_req *c)
{
    int d;
    return hipGetDevice(&d) == hipSuccess && d == c->device;
}
size_t row_bytes(const cg_req *c) { return (size_t)c->N * 8; }
size_t ct_bytes(const cg_req *c) { return 2 * (size_t)c->k * row_bytes(c); }

// the launch's own status: an error that other code left pending in the thread is neither reported as ours nor cleared
template <class... P, class... A>
int launch(void (*kernel)(P...), dim3 grid, unsigned block, size_t lds, void *s, A... args)
{
    std::tuple<P...> pack{static_cast<P>(args)...};
    void *ptrs[sizeof...(P)];
    int i = 0;
    std::apply([&](auto &...e) { ((ptrs[i++] = static_cast<void *>(&e)), ...); }, pack);
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, dim3(block), ptrs, lds, static_cast<hipStream_t>(s)) == hipSuccess
               ? CG_OK : CG_EHIP;
}
// KERNEL<LOGN, E, more> of ARGS for the handle's ring, a row to a workgroup
#define CG_LIST(...) __VA_ARGS__
#define CG_ROWS(c, rows, s, ARGS, KERNEL, ...)                                                                                        \
    ((c)->logn == 12 ? launch(KERNEL<12, 8 __VA_OPT__(, ) __VA_ARGS__>, dim3((unsigned)(rows)), 512, 0, s, CG_LIST ARGS)              \
     : (c)->logn == 13 ? launch(KERNEL<13, 8 __VA_OPT__(, ) __VA_ARGS__>, dim3((unsigned)(rows)), 1024, 0, s, CG_LIST ARGS)           \
                       : launch(KERNEL<14, 16 __VA_OPT__(, ) __VA_ARGS__>, dim3((unsigned)(rows)), 1024, 0, s, CG_LIST ARGS))

int create(cg_req *c, const cg_params *prm)
{
    const int logn = c->logn, k = c->k;
    const size_t N = c->N;
    uint64_t pr[MAXPR];
    for (int i = 0; i < k; i++) pr[i] = prm->q[i];
    pr[k] = prm->t;
    DevConst H;
    memset(&H, 0, sizeof(H));
    H.logn = logn; H.k = k; H.nsp = c->nsp; H.np = k + 1; H.tmod = (double)prm->t;
    std::vector<double> tw((k + 1) * N), itw((k + 1) * N);
    std::vector<uint16_t> place(N), pow3(N / 2);
    std::vector<float> zeta(2 * N);
    std::vector<uint64_t> pw(2 * N);
    for (int r = 0; r <= k; r++) {
        const uint64_t p = pr[r], psi = smallest_root(N, p), ninv = inverse_mod(N % p, p);
        CG_REQUIRE(psi);
        H.mod[r].p = (double)p;
        H.mod[r].u = 1.0 / (double)p;
        pw[0] = 1;
        for (size_t i = 1; i < 2 * N; i++) pw[i] = mul_mod(pw[i - 1], psi, p);
        for (size_t j = 0; j < N; j++) {
            const uint32_t e = reversed((uint32_t)j, logn);
            tw[r * N + j] = centred(pw[e], p);
            itw[r * N + j] = centred(pw[(2 * N - e) % (2 * N)], p);
        }
        H.ninv[r] = centred(ninv, p);
        H.itw1_ninv[r] = centred(mul_mod(pw[2 * N - reversed(1, logn)], ninv, p), p);
    }
    // (pw now holds the powers of zeta)
    for (size_t e = 0; e < 2 * N; e++) zeta[e] = (float)centred(pw[e], prm->t);
    uint32_t e = 1;
    for (size_t i = 0; i < N / 2; i++, e = e * 3 % (2 * (uint32_t)N)) {
        pow3[i] = (uint16_t)e;
        place[i] = (uint16_t)reversed((e - 1) / 2, logn);
        place[N / 2 + i] = (uint16_t)reversed((2 * (uint32_t)N - e - 1) / 2, logn);
    }
    // floor(Q / t) = -(Q mod t) / t modulo q_i
    uint64_t q_mod_t = 1;
    for (int i = 0; i < k; i++) q_mod_t = mul_mod(q_mod_t, pr[i] % prm->t, prm->t);
    for (int i = 0; i < k; i++) H.delta_q[i] = centred(mul_mod(pr[i] - q_mod_t, inverse_mod(prm->t, pr[i]), pr[i]), pr[i]);

    const size_t parts[] = {sizeof(DevConst), tw.size() * 8, itw.size() * 8, place.size() * 2, zeta.size() * 4, pow3.size() * 2};
    const void *from[] = {&H, tw.data(), itw.data(), place.data(), zeta.data(), pow3.data()};
    char *to[6];
    size_t total = 0;
    for (size_t n : parts) total += (n + 255) / 256 * 256;
    if (hipMalloc(&c->mem, total) != hipSuccess) {
        c->mem = nullptr;
        return CG_ENOMEM;
    }
    char *at = static_cast<char *>(c->mem);
    for (int i = 0; i < 6; i++) {
        to[i] = at;
        if (hipMemcpy(at, from[i], parts[i], hipMemcpyHostToDevice) != hipSuccess) return CG_EHIP;
        at += (parts[i] + 255) / 256 * 256;
    }
    c->T = Tables{reinterpret_cast<DevConst *>(to[0]), reinterpret_cast<double *>(to[1]), reinterpret_cast<double *>(to[2]),
                  reinterpret_cast<uint16_t *>(to[3]), reinterpret_cast<float *>(to[4]), reinterpret_cast<uint16_t *>(to[5]),
                  H.ninv[k], centred((1ull << 32) % prm->t, prm->t), logn, k};
    return hipDeviceSynchronize() == hipSuccess ? CG_OK : CG_EHIP;
}

// Prepared plaintexts of a last round that leaves compute units free are shared by several workgroups, which repeat the interpolation and
// divide the primes.  us, a workgroup each / shared.  N = 8192, three primes: 1 21.3 / 12.0, 85 23.2 / 15.2, 128 23.9 / 20.8, 288 41.4 / 32.6, 341
// 41.9 / 34.6, 600 61.0 / 58.0.  N = 4096, two primes: 1 9.5 / 7.2, 128 10.7 / 8.6, 300 16.7 / 14.5, 600 24.8 / 22.6, 1100 38.2 / 35.7; six: 300
// 34.8 / 27.1.  N = 16384, six: 1 72.2 / 22.9, 86 75.1 / 49.0, 300 153 / 120; two: 300 69.9 / 61.4.  (Where more than half the units are busy nothing is shared.)
template <bool PREPARED, class LD>
int encode(const cg_req *c, void *s, LD ld, void *out, uint32_t batch)
{
    const int cu = c->n_cu, rest = (int)batch % cu;
    int whole = (int)batch, split = 1;
    if (PREPARED && rest) {
        const int most = std::min(c->k, cu / rest), each = (c->k + most - 1) / most;      // primes a workgroup
        split = (c->k + each - 1) / each;
        whole -= rest;
    }
    const int grid = whole + ((int)batch - whole) * split;
    return CG_ROWS(c, grid, s, (ld, out, c->T, whole, split), encode_kernel, PREPARED, LD);
}

// How many of the ciphertexts that are left go through their rounds together: whole rounds of the compute units first.  The evaluator takes a
// unit's key switch on one workgroup, or its (unit, prime) rows on one each, where these nearly fill their last round; with a few units
// more, every launch of the call is of the slower kind.  us a projection of one diagonal in one call / whole rounds first, one special prime (a round: as
// many units as have a compute unit for every row).
// - N = 8192.  A round and up to a quarter: k = 3 72 units 351 / 330, k = 2 95 287 / 280, k = 4 57 497 / 392, k = 6 40 533 / 517 (and a half: 96 431 / 424, 127 344 / 348, 76
//   464 / 511, 54 599 / 675).  Two and up to a half: k = 3 144 626 / 535, k = 2 191 489 / 455, k = 4 114 900 / 613, k = 6 81 1038 / 812 (three: 192 670 / 670, 255 523 /
//   541).  Units' own rounds, from two on: k = 3 576 1972 / 1754, k = 1 608 / 563, k = 2 1212 / 1117, k = 4 2796 / 2779, k = 6 5114 / 4631; from one with three
//   digits only: k = 3 288 1091 / 1014, 384 1284 / 1241, but k = 2 288 616 / 641, k = 4 1445 / 1519.
// - N = 4096, units' own rounds from two on: k = 2 520 433 / 428, 600 500 / 489, 800 633 / 580, k = 4 600 1166 / 1137 (640 515 / 517; 300 264 / 263).
// - N = 16384, rounds and up to a quarter: k = 6, two special primes, 36 854 / 743, k = 3 72 814 / 679, k = 6 40 1226 / 1021 (and a half: 96 928 / 939, 54 1474 / 1510).
// (N = 8192 with two special primes has no such kernels: 36 398 / 429, 288 2643 / 2705.)
//
// At most so many units go together at all: the workspace is theirs (5 to 7 GB), and their kernels have long filled the chip.  us, 1 / 2 / 4 / 8 units to a
// compute unit: N = 8192 2304 units 7316 / 6820 / 6809 / 6844, N = 4096 1764 / 1601 / 1575 / 1545, N = 16384 384 units 6717 / 6668 / 6658 / 6669.
uint32_t most_together(const cg_req *c) { return (c->logn == 14 ? 1u : c->logn == 13 ? 4u : 8u) * (uint32_t)c->n_cu; }
uint32_t fold_together(const cg_req *c, uint32_t left)
{
    if (left > most_together(c)) return most_together(c);
    const uint32_t cu = (uint32_t)c->n_cu, round = std::max(1u, cu / (uint32_t)(c->k + c->nsp)), rest = left % cu, over = left % round;
    if (c->logn == 14) return left > round && 4 * over <= round ? left - over : left;
    if (c->nsp > 1) return left;
    if (left >= 2 * cu || (c->logn == 13 && c->k == 3 && left >= cu)) return (c->logn == 13 ? 10 * rest < 9 * cu : 5 * rest <= 2 * cu) ? left - rest : left;
    if (c->logn == 13 && left < cu && left > round && left < 3 * round && (left < 2 * round ? 4 : 2) * over <= round) return left - over;
    return left;
}

// generators of the sum over residue classes modulo d2: rotations by d2, 2 d2, ... N/4, then the row swap
int fold_bits(const cg_req *c, uint32_t d2) { return c->logn - 2 - log2_of(d2) + 2; }
}  // namespace

CG_API int cg_req_create(cg_req **out, cg_ctx *ctx, const cg_params *prm)
{
    CG_REQUIRE(out);
    *out = nullptr;
    CG_REQUIRE(ctx && prm && prm->q && prm->log2n >= 12 && prm->log2n <= 14 && prm->k >= 1 && prm->k <= 6 && prm->nsp >= 1 &&
               prm->nsp <= 2 && prm->alpha >= 1 && prm->k % prm->alpha == 0);
    const uint64_t N = 1ull << prm->log2n;
    CG_REQUIRE(prm->t < (1u << 20) && prm->t % (2 * N) == 1 && small_prime(prm->t));
    for (uint32_t i = 0; i < prm->k; i++) CG_REQUIRE(prm->q[i] % (2 * N) == 1 && prm->q[i] > (1ull << 40) && prm->q[i] < (1ull << 50));
    // the tables made here are used with the context's
    CG_TRY(cg_check_params(ctx, prm));
    cg_req *c = new (std::nothrow) cg_req();
    if (!c) return CG_ENOMEM;
    c->ctx = ctx;
    c->logn = (int)prm->log2n; c->N = (int)N; c->k = (int)prm->k; c->nsp = (int)prm->nsp;
    int rc = CG_EHIP;
    if (hipGetDevice(&c->device) == hipSuccess &&
        hipDeviceGetAttribute(&c->n_cu, hipDeviceAttributeMultiprocessorCount, c->device) == hipSuccess && c->n_cu >= 1) {
        try {
            rc = create(c, prm);
        } catch (const std::bad_alloc &) {
            rc = CG_ENOMEM;
        }
    }
    if (rc != CG_OK) {
        if (c->mem) (void)hipFree(c->mem);
        delete c;
        return rc;
    }
    *out = c;
    return CG_OK;
}

CG_API int cg_req_destroy(cg_req *c)
{
    if (!c) return CG_OK;
    (void)hipDeviceSynchronize();
    if (c->mem) (void)hipFree(c->mem);
    delete c;
    return CG_OK;
}

CG_API int cg_slots_encode(cg_req *c, void *stream, const int64_t *slots, uint64_t *pt, uint32_t batch)
{
    CG_REQUIRE(c && all_aligned({slots, pt}) && in_one_call(batch) && here(c));
    CG_REQUIRE(!overlap(slots, row_bytes(c) * batch, pt, row_bytes(c) * batch));
    return encode<false>(c, stream, LdSlots{slots, c->logn}, pt, batch);
}

CG_API int cg_slots_prepare(cg_req *c, void *stream, const int64_t *slots, void *plain, uint32_t batch)
{
    CG_REQUIRE(c && all_aligned({slots, plain}) && in_one_call(batch) && here(c));
    CG_REQUIRE(!overlap(slots, row_bytes(c) * batch, plain, row_bytes(c) * c->k * batch));
    return encode<true>(c, stream, LdSlots{slots, c->logn}, plain, batch);
}

// ---------------------------------------------------------------------------
// projections
// ---------------------------------------------------------------------------
static bool block_length_ok(const cg_req *c, uint32_t d2) { return power_of_two(d2) && d2 >= 2 && d2 <= (uint32_t)c->N / 4; }
static uint32_t tile_length(const cg_req *c, uint32_t d1, uint32_t d2)
{
    uint32_t tile = std::max(d2, (uint32_t)c->N / d2);
    while (tile < d1) tile *= 2;
    return tile;
}

CG_API uint32_t cg_cpvm_diagonals(const cg_req *c, uint32_t d1, uint32_t d2)
{
    if (!c || !block_length_ok(c, d2) || d1 < 1 || d1 > (uint32_t)c->N / 2) return 0;
    const uint32_t tile = tile_length(c, d1, d2);
    if (tile > (uint32_t)c->N / 2) return 0;
    const uint64_t n_diag = (uint64_t)d2 * tile / c->N;
    return n_diag <= 64 ? (uint32_t)n_diag : 0;
}

// Whether matrices are laid out by their diagonals before these are encoded.  Along a diagonal of a matrix as it is given every lane reads
// another row: us, 768 x 64 at N = 8192, straight / laid out first: 1 matrix 14.1 / 19.6, 12 25.9 / 29.7, 24 35.1 / 37.4, 32 (a plaintext for every unit) 40.3
// / 38.7, 36 51.3 / 44.3, 72 95.2 / 69.9.  At N = 4096 16 (a plaintext for every unit) 18.6 / 23.4, 20 24.0 / 26.7, 36 39.7 / 34.8, 72 68.1 / 53.0; at
// N = 16384 72 130.5 / 131.0, 144 256 / 250.  Matrices of few rows stay in the caches: 300 of 100 x 64 at N = 4096 27.4 / 34.8.
static bool skewed_first(const cg_req *c, uint64_t plaintexts, uint32_t rank) { return rank || plaintexts > (uint32_t)c->n_cu; }

CG_API size_t cg_cpvm_prepare_workspace_bytes(const cg_req *c, uint32_t units, uint32_t d1, uint32_t d2, uint32_t rank)
{
    const uint32_t n_diag = cg_cpvm_diagonals(c, d1, d2);
    if (!n_diag || !skewed_first(c, (uint64_t)units * n_diag, rank)) return 0;
    return (size_t)units * tile_length(c, d1, d2) * d2 * sizeof(float);
}

CG_API int cg_cpvm_prepare(cg_req *c, void *stream, const int64_t *w, const int64_t *a, const int64_t *b, uint32_t units,
                           uint32_t a_group, uint32_t d1, uint32_t d2, uint32_t rank, void *diags, void *ws)
{
    const uint32_t n_diag = cg_cpvm_diagonals(c, d1, d2);
    CG_REQUIRE(n_diag && units >= 1 && in_one_call((uint64_t)units * n_diag) && aligned(diags) && here(c));
    CG_REQUIRE(rank ? rank <= 4096 && a_group >= 1 && all_aligned({a, b}) && (!w || aligned(w)) : !a && !b && aligned(w));
    const bool skew = skewed_first(c, (uint64_t)units * n_diag, rank);
    CG_REQUIRE(!skew || aligned(ws));
    const uint32_t tile = tile_length(c, d1, d2);
    const size_t out = row_bytes(c) * c->k * n_diag * units, mats = (size_t)units * d1 * d2 * 8, skewed = (size_t)units * tile * d2 * sizeof(float);
    const Diagonal D{c->logn, log2_of(tile), log2_of(n_diag), log2_of(d2), (int)d1};
    CG_REQUIRE(!w || !overlap(w, mats, diags, out));
    if (!skew) return encode<true>(c, stream, LdMatrix{D, w}, diags, units * n_diag);
    CG_REQUIRE(!overlap(ws, skewed, diags, out) && (!w || !overlap(w, mats, ws, skewed)));
    if (rank) {
        const size_t na = (size_t)((units - 1) / a_group + 1) * d1 * rank * 8, nb = (size_t)units * rank * d2 * 8;
        CG_REQUIRE(!overlap(a, na, diags, out) && !overlap(b, nb, diags, out) && !overlap(a, na, ws, skewed) && !overlap(b, nb, ws, skewed));
    } else {
        a_group = 1;
    }
    a_group = std::min(a_group, units);      // (the kernel divides int32, which any larger number need not be)
    const uint32_t row_blocks = (d1 + 63) / 64;
    float *m = static_cast<float *>(ws);
    CG_TRY(launch(low_rank_kernel, dim3(units * row_blocks, (d2 + 63) / 64), 256, 0, stream, w, a, b, m, (int)a_group, (int)d1, log2_of(d2),
                  (int)rank, (int)row_blocks, (int)tile, c->T));
    return encode<true>(c, stream, LdSkewed{D, m}, diags, units * n_diag);
}

// requests whose copies are made together
static uint32_t series_together(const cg_req *c, uint32_t requests, uint32_t n_diag) { return std::min(requests, std::max(1u, most_together(c) / n_diag)); }

CG_API size_t cg_cpvm_requests_workspace_bytes(const cg_req *c, uint32_t requests, uint32_t units, uint32_t n_diag)
{
    if (!c || !in_one_call((uint64_t)requests * units) || !n_diag || n_diag > 64 || !in_one_call((uint64_t)requests * n_diag)) return 0;
    const size_t copies = n_diag - 1, batch = (size_t)requests * units, together = std::min(batch, (size_t)most_together(c));
    const size_t cts = requests * copies + (size_t)requests * n_diag + batch + together;
    const size_t series = copies ? cg_workspace_bytes(c->ctx, series_together(c, requests, n_diag) * n_diag) : 0;
    return cts * ct_bytes(c) + std::max(series, cg_workspace_bytes(c->ctx, (uint32_t)together));
}

// A quarter as many rows as compute units, and each is taken in four parts (us a projection of one request, whole rows / parts: N = 8192, 48 rows, 3 matrices
// 114.3 / 113.3, 12 151.4 / 150.2; N = 16384, 48 rows, 3 matrices 250.5 / 245.1; halves, and parts of the sums' rows, are within 0.5 % either way, as is all at N = 4096).
template <int LOGN> static int copies_in_parts(const cg_req *c, void *s, const LdCopies &ld, double *f, size_t rows)
{
    return launch(ntt_fwd_part_kernel<LOGN, 2, LdCopies, StF64Red>, dim3((unsigned)rows * 4), 1u << (LOGN - 5), 0, s, ld, StF64Red{f, LOGN}, c->T.tw, c->T.C,
                  (int)rows);
}
static int transform_copies(const cg_req *c, void *s, const LdCopies &ld, double *f, size_t rows)
{
    if (c->logn == 13 && 4 * rows <= (size_t)c->n_cu) return copies_in_parts<13>(c, s, ld, f, rows);
    if (c->logn == 14 && 4 * rows <= (size_t)c->n_cu) return copies_in_parts<14>(c, s, ld, f, rows);
    return CG_ROWS(c, rows, s, (ld, f, c->T), copies_kernel);
}

static int cpvm_requests(cg_req *c, void *stream, const uint64_t *x, const void *diags, const void *adapters, uint32_t n_adapters,
                         const int32_t *pick, uint32_t requests, uint32_t units, uint32_t n_diag, uint32_t d2,
                         uint32_t round_bits, const void *const *gk_copies, const void *const *gk_block, uint64_t *out, void *ws)
{
    const uint32_t batch = requests * units;
    const size_t ct = ct_bytes(c);
    // the rounds of the sum over residue classes, or one generator after the other
    const int bits = fold_bits(c, d2);
    std::vector<uint32_t> elts, counts;
    if (round_bits) {
        const int rounds = (bits + (int)round_bits - 1) / (int)round_bits, lo = bits / rounds, extra = bits % rounds;
        for (int r = 0; r < rounds; r++) counts.push_back((1u << (lo + (r < extra))) - 1);
    } else {
        counts.assign(bits, 1);
    }
    uint32_t n_keys = 0;
    CG_TRY(cg_round_galois(c->ctx, 1, d2, round_bits ? round_bits : 1, nullptr, 0, &n_keys));
    elts.resize(n_keys);
    CG_TRY(cg_round_galois(c->ctx, 1, d2, round_bits ? round_bits : 1, elts.data(), n_keys, &n_keys));
    uint32_t total = 0;
    for (uint32_t n : counts) total += n;
    CG_REQUIRE(total == n_keys);
    for (uint32_t i = 0; i < n_keys; i++) CG_REQUIRE(aligned(gk_block[i]));

    char *at = static_cast<char *>(ws);
    auto take = [&](size_t cts) { char *p = at; at += cts * ct; return p; };
    uint64_t *copies = reinterpret_cast<uint64_t *>(take((size_t)requests * (n_diag - 1)));
    double *f = reinterpret_cast<double *>(take((size_t)requests * n_diag));
    uint64_t *xa = reinterpret_cast<uint64_t *>(take(batch)), *xb = reinterpret_cast<uint64_t *>(take(std::min(batch, most_together(c))));
    void *rest = at;
    const size_t words = ct / 8;
    if (n_diag > 1) {
        uint32_t gs[64], e = 1;
        for (uint32_t i = 1; i < n_diag; i++) gs[i - 1] = e = e * 3 % (2u * (uint32_t)c->N);
        for (uint32_t r = 0, n; r < requests; r += n) {
            n = series_together(c, requests - r, n_diag);
            CG_TRY(cg_rotate_hoisted(c->ctx, stream, x + r * words, n_diag - 1, gs, gk_copies, copies + (size_t)r * (n_diag - 1) * words, n, rest));
        }
    }
    CG_TRY(transform_copies(c, stream, LdCopies{x, copies, (int)n_diag, c->k, c->logn}, f, (size_t)requests * n_diag * 2 * c->k));
    const uint32_t blocks = (uint32_t)(c->N / (2 * PRODUCT_THREADS)) * c->k * requests;
    // three workgroups to a compute unit are resident (one to twelve are within 1 %)
    const uint32_t parts0 = std::min(units, std::max(1u, 3 * (uint32_t)c->n_cu / blocks)), per = (units + parts0 - 1) / parts0;
    const ProductArgs A{f, static_cast<const double *>(diags), static_cast<const double *>(adapters), pick, reinterpret_cast<double *>(xa),
                        (int)n_adapters, (int)requests, (int)units, (int)n_diag, (int)per, (int)((units + per - 1) / per)};
    const unsigned grid = blocks * (unsigned)A.parts;
    switch (n_diag) {
    case 1: CG_TRY(launch(products_kernel<1, true>, dim3(grid), PRODUCT_THREADS, 0, stream, A, c->T)); break;
    case 2: CG_TRY(launch(products_kernel<2, true>, dim3(grid), PRODUCT_THREADS, 0, stream, A, c->T)); break;
    case 4: CG_TRY(launch(products_kernel<4, true>, dim3(grid), PRODUCT_THREADS, 0, stream, A, c->T)); break;
    case 8: CG_TRY(launch(products_kernel<8, true>, dim3(grid), PRODUCT_THREADS, 0, stream, A, c->T)); break;
    default: CG_TRY(launch(products_kernel<8, false>, dim3(grid), PRODUCT_THREADS, 0, stream, A, c->T));
    }
    CG_TRY(CG_ROWS(c, (size_t)batch * 2 * c->k, stream, (reinterpret_cast<double *>(xa), c->T), sums_kernel));
    for (uint32_t at_unit = 0, n; at_unit < batch; at_unit += n) {
        n = round_bits ? fold_together(c, batch - at_unit) : std::min(batch - at_unit, most_together(c));
        uint64_t *cur = xa + at_unit * words, *next = xb;
        for (size_t r = 0, first = 0; r < counts.size(); first += counts[r], r++) {
            uint64_t *to = r + 1 == counts.size() ? out + at_unit * words : next;
            if (round_bits) CG_TRY(cg_rotate_sum_hoisted(c->ctx, stream, cur, counts[r], elts.data() + first, gk_block + first, to, n, rest));
            // (three launches a generator: the evaluator's own chains, which join two rotations, have no entry point.  One request, three matrices, N = 8192:
            // 229 us, cg_cpvm_hoisted 205; in rounds of three bits 111, 117)
            else CG_TRY(cg_rotate(c->ctx, stream, cur, elts[first], gk_block[first], to, n, 1, rest));
            next = cur;
            cur = to;
        }
    }
    return CG_OK;
}

CG_API int cg_cpvm_requests(cg_req *c, void *stream, const uint64_t *x, const void *diags, const void *adapters, uint32_t n_adapters,
                            const int32_t *pick, uint32_t requests, uint32_t units, uint32_t n_diag, uint32_t d2,
                            uint32_t round_bits, const void *const *gk_copies, const void *const *gk_block, uint64_t *out, void *ws)
{
    CG_REQUIRE(c && all_aligned({x, diags, out, ws}) && requests >= 1 && units >= 1 && in_one_call((uint64_t)requests * units));
    CG_REQUIRE(block_length_ok(c, d2) && power_of_two(n_diag) && n_diag <= 64 && n_diag <= d2 && in_one_call((uint64_t)requests * n_diag));
    CG_REQUIRE(n_adapters ? aligned(adapters) && aligned(pick, 4) && n_adapters < (1u << 31) : !adapters);
    CG_REQUIRE(round_bits <= 7 && gk_block && (n_diag == 1 || gk_copies) && here(c));
    for (uint32_t i = 0; i + 1 < n_diag; i++) CG_REQUIRE(aligned(gk_copies[i]));
    const size_t n_ws = cg_cpvm_requests_workspace_bytes(c, requests, units, n_diag), n_out = ct_bytes(c) * requests * units;
    const size_t n_diags = row_bytes(c) * c->k * units * n_diag;
    CG_REQUIRE(!overlap(x, ct_bytes(c) * requests, out, n_out) && !overlap(ws, n_ws, out, n_out) && !overlap(ws, n_ws, x, ct_bytes(c) * requests));
    CG_REQUIRE(!overlap(diags, n_diags, out, n_out) && !overlap(diags, n_diags, ws, n_ws));
    CG_REQUIRE(!n_adapters || (!overlap(adapters, n_diags * n_adapters, out, n_out) && !overlap(adapters, n_diags * n_adapters, ws, n_ws) &&
                               !overlap(pick, 4 * (size_t)requests, out, n_out) && !overlap(pick, 4 * (size_t)requests, ws, n_ws)));
    try {
        return cpvm_requests(c, stream, x, diags, adapters, n_adapters, pick, requests, units, n_diag, d2, round_bits, gk_copies, gk_block,
                             out, ws);
    } catch (const std::bad_alloc &) {
        return CG_ENOMEM;
    }
}

// ---------------------------------------------------------------------------
// position biases
// ---------------------------------------------------------------------------
static int add_bias(cg_req *c, void *stream, const uint64_t *in, uint32_t groups, uint32_t heads, uint32_t n_cts, uint32_t d2,
                    const int32_t *pos, const int64_t *table, const int32_t *edges, uint32_t n_buckets, uint64_t *out)
{
    CG_REQUIRE(c && all_aligned({in, out, table}) && aligned(edges, 4) && block_length_ok(c, d2) && here(c));
    CG_REQUIRE(groups >= 1 && heads >= 1 && n_cts >= 1 && n_buckets >= 1 && n_buckets <= 4096);
    CG_REQUIRE(in_one_call((uint64_t)groups * heads) && in_one_call((uint64_t)groups * heads * n_cts));
    const uint32_t units = groups * heads * n_cts;
    const size_t n_out = ct_bytes(c) * units;
    CG_REQUIRE(in == out || !overlap(in, n_out, out, n_out));
    CG_REQUIRE((!pos || !overlap(pos, 4 * (size_t)groups, out, n_out)) && !overlap(table, 8 * (size_t)n_buckets * heads, out, n_out) &&
               !overlap(edges, 4 * (size_t)n_buckets, out, n_out));
    const BiasArgs A{in, out, pos, table, edges, (int)n_buckets, (int)heads, (int)n_cts, log2_of(d2)};
    const size_t lds = (size_t)c->N / d2 * sizeof(float);
#define CG_BIAS(K) launch(bias_kernel<K, 2>, dim3(units * (unsigned)(c->N / (4 * BIAS_THREADS))), BIAS_THREADS, lds, stream, A, c->T)
    switch (c->k) {
    case 1: return CG_BIAS(1);
    case 2: return CG_BIAS(2);
    case 3: return CG_BIAS(3);
    case 4: return CG_BIAS(4);
    case 5: return CG_BIAS(5);
    default: return CG_BIAS(6);
    }
#undef CG_BIAS
}

CG_API int cg_score_bias(cg_req *c, void *stream, const uint64_t *scores, uint32_t requests, uint32_t heads, uint32_t n_cts, uint32_t d2,
                         const int32_t *pos, const int64_t *table, const int32_t *edges, uint32_t n_buckets, uint64_t *out)
{
    CG_REQUIRE(aligned(pos, 4));
    return add_bias(c, stream, scores, requests, heads, n_cts, d2, pos, table, edges, n_buckets, out);
}

CG_API int cg_prompt_bias(cg_req *c, void *stream, const uint64_t *diags, uint32_t prompts, uint32_t heads, uint32_t d2,
                          const int64_t *table, const int32_t *edges, uint32_t n_buckets, uint64_t *out)
{
    CG_REQUIRE(c && block_length_ok(c, d2));
    return add_bias(c, stream, diags, prompts, heads, (uint32_t)c->N / d2, d2, nullptr, table, edges, n_buckets, out);
}

// ---------------------------------------------------------------------------
// appends
// ---------------------------------------------------------------------------
CG_API int cg_kv_append_requests(cg_req *c, void *stream, uint64_t *cache, uint32_t cache_stride_cts, uint32_t requests, uint32_t per,
                                 const int32_t *lens, const uint64_t *rows, uint32_t row_stride_cts, const void *masks, uint32_t d2)
{
    CG_REQUIRE(c && all_aligned({cache, rows, masks}) && aligned(lens, 4) && here(c));
    CG_REQUIRE(requests >= 1 && per >= 1 && in_one_call((uint64_t)requests * per) && cache_stride_cts >= 1 && row_stride_cts >= per);
    CG_REQUIRE(power_of_two(d2) && d2 <= (uint32_t)c->N / 2);
    const size_t caches = (size_t)requests * per, n_rows = ((size_t)(requests - 1) * row_stride_cts + per) * ct_bytes(c);
    const size_t n_cache = caches * cache_stride_cts * ct_bytes(c);
    CG_REQUIRE(!overlap(cache, n_cache, rows, n_rows) && !overlap(cache, n_cache, masks, row_bytes(c) * c->k * (c->N / d2)) &&
               !overlap(cache, n_cache, lens, 4 * (size_t)requests));
    const AppendArgs A{cache, rows, static_cast<const double *>(masks), lens, (int)per, log2_of((uint32_t)c->N / d2), cache_stride_cts,
                       row_stride_cts};
    return CG_ROWS(c, caches * 2 * c->k, stream, (A, c->T), append_kernel);
}
