// Device kernels of libcryptogen_requests.so (gfx950): slots to plaintexts, sums of plaintext products of many
// requests, position biases, appends at each request's own length.  Row transforms are those of kernels.hpp.
#pragma once
#include "kernels.hpp"

namespace cgr {
using namespace cg;

// Tables of a handle: those of the ciphertext primes and, as row k, of the plaintext modulus.
struct Tables {
    const DevConst *C;         // mod[0 .. k) ciphertext primes, mod[k] the plaintext modulus
    const double *tw, *itw;    // [k + 1][N]
    const uint16_t *place;     // slot s is output place[s] of the transform modulo t
    const float *zeta;         // zeta^e mod t, centred, e < 2N
    const uint16_t *pow3;      // 3^i mod 2N, i < N/2
    double ninv_t;             // N^-1 mod t, centred
    double two32_t;            // 2^32 mod t, centred
    int logn, k;
};
// v modulo t, exact and below 2^51 (a product of 2^31 and a residue below 2^19, and 2^32): red() leaves at most (1/2 + 2^-15) t of it, which is below
// 2^19 for every t with slots (the largest is 1032193).  Any int64 costs no more than its low half did: 128 plaintexts 20.7 us, before 20.9.
__device__ __forceinline__ double of_int64(int64_t v, double two32_t)
{
    return __builtin_fma((double)(int)(v >> 32), two32_t, (double)(uint32_t)v);
}

// workgroups of 1024 threads with rows of 8192 in at most 64 registers a thread: two of them on a compute unit
template <int LOGN, int E> constexpr int two_waves() { return LOGN == 13 && E == 8 ? 8 : min_waves<LOGN, E>(); }

// A pass of the inverse transform modulo t < 2^20.  Centred inputs are below 2^19; after s stages without a reduction a sum is below
// 2^(19 + s), its difference times a factor below 2^(39 + s) <= 2^52: every product is exact in one multiplication, and no sum is reduced (six
// instructions a butterfly, where one modulo a 50-bit prime has eight and its passes reduce).  Plan and places as inv_pass.
template <int LOGN, int E, int PASS>
__device__ __forceinline__ void small_pass(double *lds, double *out, int tid, const double *__restrict__ itw, const double *twr, double *twr_next,
                                           const ModD m, double ninv, double itw1_ninv)
{
    using P = Plan<LOGN, E>;
    constexpr int R = P::R[PASS], L = LOGN - stage_start<LOGN, E, PASS>() - R, G = E >> R, PER = (1 << R) - 1;
    constexpr bool last = PASS == 0;
    static_assert(!last || G == 1, "one group a thread in the last pass");
    auto times = [&](double x, double w) {
        const double h = x * w;
        return __builtin_fma(-__builtin_rint(h * m.u), m.p, h);
    };
    double v[G][1 << R];
    int base[G];
#pragma unroll
    for (int g = 0; g < G; g++) {
        const int at = group_index<LOGN, E, PASS>(tid, g);
        base[g] = pad(((last ? 0 : at >> L) << (L + R)) | (at & ((1 << L) - 1)));
#pragma unroll
        for (int c = 0; c < (1 << R); c++) {
            if (L > 0) v[g][c] = lds[base[g] + pad(c << L)];
            else if (c % 2 == 0) {
                const double2 x = pair_at(lds, base[g] + c);
                v[g][c] = x.x;
                v[g][c + 1] = x.y;
            }
        }
    }
#pragma unroll
    for (int g = 0; g < G; g++)
#pragma unroll
        for (int u = R - 1; u >= 0; u--) {
            const int half = 1 << (R - 1 - u);
#pragma unroll
            for (int c = 0; c < (1 << R); c++) {
                if (c & half) continue;
                const double sum = v[g][c] + v[g][c + half], d = v[g][c] - v[g][c + half];
                v[g][c] = last && u == 0 ? times(sum, ninv) : sum;
                v[g][c + half] = times(d, last && u == 0 ? itw1_ninv : twr[g * PER + (1 << u) - 1 + (c >> (R - u))]);
            }
        }
    if constexpr (last) {
#pragma unroll
        for (int c = 0; c < (1 << R); c++) out[c] = v[0][c];        // (element tid + c * T)
    } else {
        if constexpr (PASS == 1) load_tw<LOGN, E, 0, true>(itw, tid, twr_next);
        else load_tw<LOGN, E, PASS - 1, false>(itw, tid, twr_next);
#pragma unroll
        for (int g = 0; g < G; g++)
#pragma unroll
            for (int c = 0; c < (1 << R); c++) {
                if (L > 0) lds[base[g] + pad(c << L)] = v[g][c];
                else if (c % 2 == 0) pair_at(lds, base[g] + c) = make_double2(v[g][c], v[g][c + 1]);
            }
        if constexpr (PASS - 1 < P::NC) lds_barrier();
        else wave_sync();
    }
}
// The row lies in LDS, behind a barrier; results |x| <= (1/2 + 2^-18) t, element tid + c * T in out[c]
template <int LOGN, int E>
__device__ __forceinline__ void small_inv_row(double *lds, double *out, int tid, const double *__restrict__ itw, const ModD m, double ninv, double itw1_ninv)
{
    constexpr int NP = Plan<LOGN, E>::NP;
    asm volatile("" : "+v"(tid));
    double twa[TWREGS], twb[TWREGS];
    load_tw<LOGN, E, NP - 1, false>(itw, tid, twa);
    if constexpr (NP > 4) {
        small_pass<LOGN, E, 4>(lds, out, tid, itw, twa, twb, m, ninv, itw1_ninv);
        small_pass<LOGN, E, 3>(lds, out, tid, itw, twb, twa, m, ninv, itw1_ninv);
        small_pass<LOGN, E, 2>(lds, out, tid, itw, twa, twb, m, ninv, itw1_ninv);
        small_pass<LOGN, E, 1>(lds, out, tid, itw, twb, twa, m, ninv, itw1_ninv);
        small_pass<LOGN, E, 0>(lds, out, tid, itw, twa, twb, m, ninv, itw1_ninv);
    } else {
        small_pass<LOGN, E, 3>(lds, out, tid, itw, twa, twb, m, ninv, itw1_ninv);
        small_pass<LOGN, E, 2>(lds, out, tid, itw, twb, twa, m, ninv, itw1_ninv);
        small_pass<LOGN, E, 1>(lds, out, tid, itw, twa, twb, m, ninv, itw1_ninv);
        small_pass<LOGN, E, 0>(lds, out, tid, itw, twb, twa, m, ninv, itw1_ninv);
    }
}

// ---------------------------------------------------------------------------
// Slot values -> polynomial modulo t -> prepared plaintext.  The interpolation is an inverse transform modulo t of the
// values in the order of the transform's outputs; its results are centred in registers and go through one forward
// transform per ciphertext prime without leaving the workgroup.  Values are read in the order of the slots, which their
// sources hold side by side, and put in their places in LDS (read in the order of the places 300 plaintexts took 52.4 us where they took 47.9).
// Bound by vector issue: 1000 plaintexts of N = 8192 and three primes take 86 us, 21.5 ns a row transform, their 262 MB at the rate of a
// copy would take 49; in 75 registers with one workgroup to a unit 102, with the interpolation by the passes for 50-bit primes 93.6.  One plaintext
// takes 12.0 us with its primes on workgroups of their own, one after the other 21.3; its polynomial alone 7.3 (1000 of them 29.3).
// ---------------------------------------------------------------------------
struct LdSlots {
    const int64_t *v;
    int logn;
    __device__ __forceinline__ double value(int b, int slot, double two32_t) const { return of_int64(at32(v + ((size_t)b << logn), slot), two32_t); }
};
// slot `slot` of diagonal c of unit u, b = u n_diag + c: M[f][col], f the feature that the token's copy c shows there, col = slot mod d2
struct Diagonal {
    int logn, log_tile, log_diag, log_d2, d1;
    __device__ __forceinline__ int feature(int b, int slot) const
    {
        const int half = 1 << (logn - 1), n_diag = 1 << log_diag;
        const int at = (slot & half) | ((slot + (b & (n_diag - 1))) & (half - 1));
        return (at + n_diag * (at >> log_tile)) & ((1 << log_tile) - 1);
    }
    __device__ __forceinline__ int col(int slot) const { return slot & ((1 << log_d2) - 1); }
};
struct LdMatrix : Diagonal {        // int64 [units][d1][d2]
    const int64_t *m;
    __device__ __forceinline__ double value(int b, int slot, double two32_t) const
    {
        const int f = feature(b, slot);
        return f < d1 ? of_int64(m[(((size_t)(b >> log_diag) * d1 + f) << log_d2) + col(slot)], two32_t) : 0.0;
    }
};
struct LdSkewed : Diagonal {        // float [units][tile][d2], row (f - col) mod tile: the d2 slots of a block lie in one row
    const float *m;
    __device__ __forceinline__ double value(int b, int slot, double) const
    {
        const int f = feature(b, slot), row = (f - col(slot)) & ((1 << log_tile) - 1);
        return f < d1 ? (double)m[(((((size_t)(b >> log_diag)) << log_tile) + row) << log_d2) + col(slot)] : 0.0;
    }
};

// The first `whole` plaintexts take a workgroup each, those behind `split`, which share the primes and repeat the interpolation.
template <int LOGN, int E, bool PREPARED, class LD>
__global__ void __launch_bounds__((1 << LOGN) / E, (two_waves<LOGN, E>()))
encode_kernel(LD ld, void *__restrict__ out, Tables T, int whole, int split)
{
    __shared__ __align__(16) double lds[lds_doubles<LOGN>()];
    constexpr int TH = (1 << LOGN) / E;
    const int tid = threadIdx.x, k = T.k, over = (int)blockIdx.x - whole;
    const int b = over < 0 ? (int)blockIdx.x : whole + over / split, part = over < 0 ? 0 : over % split, step = over < 0 ? 1 : split;
    const ModD mt = T.C->mod[k];
    double v[E], w[E];
#pragma unroll
    for (int it = 0; it < E; it++) v[it] = ld.value(b, tid + it * TH, T.two32_t);
#pragma unroll
    for (int it = 0; it < E; it++) lds[pad((int)at_lane(T.place + it * TH, tid))] = red(v[it], mt);
    lds_barrier();
    small_inv_row<LOGN, E>(lds, w, tid, T.itw + ((size_t)k << LOGN), mt, T.C->ninv[k], T.C->itw1_ninv[k]);
    if constexpr (!PREPARED) {
        uint64_t *row = static_cast<uint64_t *>(out) + ((size_t)b << LOGN);
#pragma unroll
        for (int it = 0; it < E; it++) put_lane(row + it * TH, tid, f64_to_u64(canon(w[it], mt)));
    } else {
        // |w| <= (t - 1) / 2 < 2^19 (t is odd, so the rounded quotient of an integer is never in doubt): kept in 24 bits from prime to prime
        float lift[E];
#pragma unroll
        for (int it = 0; it < E; it++) lift[it] = (float)red(w[it], mt);
        for (int i = part; i < k; i += step) {
            const ModD m = T.C->mod[i];
            lds_barrier();      // the last pass read other waves' elements, or its chunk is still being copied out
#pragma unroll
            for (int it = 0; it < E; it++) {
                asm volatile("" : "+v"(lift[it]));      // (or the conversions leave the loop, and 64 bits stay)
                w[it] = (double)lift[it];
            }
            double *row = static_cast<double *>(out) + ((size_t)(b * k + i) << LOGN);
            // Two workgroups to a unit fall out of step with priorities in the passes, one's exchanges under the other's butterflies: one row 12.1 ->
            // 11.7, 256 rows 27.4 -> 27.0, 1000 rows 90.0 -> 88.4 (N = 8192), 31.7 -> 31.3 (1000, N = 4096). At N = 16384 a workgroup has its unit for
            // itself, and 128 rows take 51.6 with them, 49.4 without.
            fwd_row<LOGN, E, false, (LOGN < 14), 1, 1>(lds, w, v, tid, T.tw + ((size_t)i << LOGN), m);
#pragma unroll
            for (int it = 0; it < E; it += 2)
                put_lane(reinterpret_cast<cg_double2v *>(row) + 32 * it, chunk_elem<E>(tid, 0) / 2,
                         cg_double2v{red(v[it], m), red(v[it + 1], m)});
        }
    }
}

// ---------------------------------------------------------------------------
// M_u = W_u + A B_u modulo t, laid out by its diagonals: 64 x 64 entries to a workgroup on the matrix cores in FP64, exact because centred
// entries are below 2^19 and rank 2^38 below 2^53.  Bound by its loads and stores, which for a rank of 16 are a hundredth of the encoded
// diagonals': factors are brought in and centred once a workgroup, and the tile leaves through LDS, a diagonal's entries side by
// side (each lane's own entry to its own row took 16.8 us for 36 matrices of 768 x 64 at rank 16, and 34.4 at 64).
// ---------------------------------------------------------------------------
typedef double cg_double4v __attribute__((ext_vector_type(4)));
constexpr int LR_TILE = 64, LR_RANK = 16;
__global__ void __launch_bounds__(256)
low_rank_kernel(const int64_t *__restrict__ w, const int64_t *__restrict__ a, const int64_t *__restrict__ b, float *__restrict__ out, int a_group,
                int d1, int log_d2, int rank, int row_blocks, int tile, Tables T)
{
    __shared__ double as[LR_TILE][LR_RANK + 1], bs[LR_RANK][LR_TILE + 2];
    __shared__ float done[LR_TILE][LR_TILE + 1];
    const ModD mt = T.C->mod[T.k];
    const int d2 = 1 << log_d2, u = (int)blockIdx.x / row_blocks, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int f0 = ((int)blockIdx.x % row_blocks) * LR_TILE, c0 = (int)blockIdx.y * LR_TILE;
    const int i = lane & 15, q = lane >> 4;
    const int64_t *au = a + (size_t)(u / a_group) * d1 * rank, *bu = b + (size_t)u * rank * d2;
    cg_double4v acc[4] = {};
    // (W's words come in beside the products)
    const int64_t *wu = w + (((size_t)u * d1) << log_d2);
    double base[4][4];
#pragma unroll
    for (int c = 0; c < 4; c++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int f = f0 + 16 * wave + 4 * e + q, col = c0 + 16 * c + i;
            base[c][e] = w && f < d1 && col < d2 ? of_int64(at32(wu, (f << log_d2) + col), T.two32_t) : 0.0;
        }
    for (int j0 = 0; j0 < rank; j0 += LR_RANK) {
        int64_t x[4], y[4];
        const int af = f0 + (tid >> 2), aj = j0 + 4 * (tid & 3), bj = j0 + (tid >> 4), bc = c0 + 4 * (tid & 15);
#pragma unroll
        for (int e = 0; e < 4; e++) {
            x[e] = af < d1 && aj + e < rank ? au[(size_t)af * rank + aj + e] : 0;
            y[e] = bj < rank && bc + e < d2 ? bu[(size_t)bj * d2 + bc + e] : 0;
        }
        if (j0) __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; e++) {
            as[tid >> 2][4 * (tid & 3) + e] = red(of_int64(x[e], T.two32_t), mt);
            bs[tid >> 4][4 * (tid & 15) + e] = red(of_int64(y[e], T.two32_t), mt);
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < LR_RANK; n += 4) {
            if (j0 + n >= rank) break;
            const double xn = as[16 * wave + i][n + q];
#pragma unroll
            for (int c = 0; c < 4; c++) acc[c] = __builtin_amdgcn_mfma_f64_16x16x4f64(xn, bs[n + q][16 * c + i], acc[c], 0, 0, 0);
        }
    }
#pragma unroll
    for (int c = 0; c < 4; c++)
#pragma unroll
        for (int e = 0; e < 4; e++) done[16 * wave + 4 * e + q][16 * c + i] = (float)red(red(acc[c][e], mt) + base[c][e], mt);
    __syncthreads();
    // feature - column = dd - 63 within the tile: a row of the layout to a wave at a time
    float *mine = out + (((size_t)u * tile) << log_d2);
    const bool there = c0 + lane < d2;
#pragma unroll
    for (int d0 = 0; d0 < 2 * LR_TILE; d0 += 32) {
        float v[8];
#pragma unroll
        for (int n = 0; n < 8; n++) v[n] = done[(d0 + 4 * n + wave - (LR_TILE - 1) + lane) & (LR_TILE - 1)][lane];
#pragma unroll
        for (int n = 0; n < 8; n++) {
            const int f = d0 + 4 * n + wave - (LR_TILE - 1) + lane;
            if (there && f >= 0 && f < LR_TILE && f0 + f < d1) put32(mine, (((f0 + f - c0 - lane) & (tile - 1)) << log_d2) + c0 + lane, v[n]);
        }
    }
}

// ---------------------------------------------------------------------------
// The copies of all tokens, transformed: row (r, c, component, prime), copy 0 being the token itself.  768 rows of 8192 (16 requests) 24 us.
// ---------------------------------------------------------------------------
struct LdCopies {
    static constexpr int kRaw = 1;
    static constexpr bool kScatter = false;
    const uint64_t *x, *copies;
    int n_diag, k, logn;
    __device__ __forceinline__ int prime(int row, const DevConst *) const { return row % k; }
    __device__ __forceinline__ int dst_limb(int row, const DevConst *) const { return row; }
    __device__ __forceinline__ const uint64_t *row(int row) const
    {
        const int cp = row / (2 * k), r = cp / n_diag, c = cp % n_diag, in_ct = row % (2 * k);
        return c ? copies + ((size_t)((r * (n_diag - 1) + c - 1) * 2 * k + in_ct) << logn) : x + ((size_t)(r * 2 * k + in_ct) << logn);
    }
    __device__ __forceinline__ void fetch(int at, int idx, const DevConst *, uint64_t *raw) const { raw[0] = at32(row(at), idx); }
    __device__ __forceinline__ double finish(const uint64_t *raw, int, int, const ModD, const DevConst *) const { return u64_to_f64(raw[0]); }
};
template <int LOGN, int E>
__global__ void __launch_bounds__((1 << LOGN) / E, (min_waves<LOGN, E>()))
copies_kernel(LdCopies ld, double *__restrict__ out, Tables T)
{
    __shared__ __align__(16) double lds[lds_doubles<LOGN>()];
    constexpr int TH = (1 << LOGN) / E;
    const int tid = threadIdx.x, row = (int)blockIdx.x, i = row % T.k;
    const uint64_t *src = ld.row(row);
    const ModD m = T.C->mod[i];
    double v[E], w[E];
#pragma unroll
    for (int it = 0; it < E; it++) v[it] = u64_to_f64(at_lane(src + it * TH, tid));
    fwd_row<LOGN, E, false>(lds, v, w, tid, T.tw + ((size_t)i << LOGN), m);
#pragma unroll
    for (int it = 0; it < E; it += 2)
        put_lane(reinterpret_cast<cg_double2v *>(out + ((size_t)row << LOGN)) + 32 * it, chunk_elem<E>(tid, 0) / 2,
                 cg_double2v{red(w[it], m), red(w[it + 1], m)});
}

// ---------------------------------------------------------------------------
// y[r][u] = sum over c of copy_(r, c) times (diagonal_(u, c) + that of the request's adapter), transformed: a thread takes a pair of
// coefficients of one request and prime through `per` units, both components, so that a diagonal's word is read once for both and
// the copies' words (up to eight copies) stay in registers.  Bound by the diagonals' way from memory, as an adapter's are read by its
// request alone: 16 requests with an adapter each, 36 matrices of 8 diagonals, N = 8192, 1.19 GB in 246 us (4.8 TB/s, a copy reaches 5.4).  As the
// loader of the inverse transforms, a row to a workgroup, each component read the diagonals for itself and the pass took 692 us
// (with four copies' words asked for together 430 to 466), here 246 and 89 for the transforms.
// ---------------------------------------------------------------------------
struct ProductArgs {
    const double *copies, *diags, *adapters;
    const int32_t *pick;
    double *out;
    int n_adapters, requests, units, n_diag, per, parts;
};
constexpr int PRODUCT_THREADS = 256;
// at_lane for what is read once: it leaves the caches to what is read again
template <class T> __device__ __forceinline__ T at_lane_once(const T *base, int tid)
{
    auto g = (const T __attribute__((address_space(1))) *)base;
    uint32_t off = (uint32_t)tid * (uint32_t)sizeof(T);
    asm("" : "+s"(g));
    asm("" : "+v"(off));
    return __builtin_nontemporal_load((const T __attribute__((address_space(1))) *)((const char __attribute__((address_space(1))) *)g + off));
}
// C copies at a time; HELD: all there are.  PLUS: an adapter's diagonals are added, ONCE: which no other request reads
template <int C, bool HELD, bool PLUS, bool ONCE>
__device__ __forceinline__ void products_of(const cg_double2v *x, const cg_double2v *w, const cg_double2v *plus, cg_double2v *out, int n_diag,
                                            int units, int k, int logn, int lane, const ModD m)
{
    const size_t row = (size_t)1 << (logn - 1);
    cg_double2v f[C][2];
    auto fetch = [&](int c0) {
#pragma unroll
        for (int c = 0; c < C; c++)
#pragma unroll
            for (int h = 0; h < 2; h++) f[c][h] = at_lane(x + (size_t)((c0 + c) * 2 + h) * k * row, lane);
    };
    if constexpr (HELD) fetch(0);
    for (int u = 0; u < units; u++) {
        double s[4] = {0.0, 0.0, 0.0, 0.0};
        for (int c0 = 0; c0 < n_diag; c0 += C) {
            cg_double2v b[C], e[PLUS ? C : 1];
            if constexpr (!HELD) fetch(c0);
#pragma unroll
            for (int c = 0; c < C; c++) {
                b[c] = at_lane(w + (size_t)(c0 + c) * k * row, lane);
                if constexpr (PLUS) e[c] = ONCE ? at_lane_once(plus + (size_t)(c0 + c) * k * row, lane) : at_lane(plus + (size_t)(c0 + c) * k * row, lane);
            }
            // four products of a centred factor and one twice as large, or eight of two centred ones: DotSum's room
            constexpr int ROOM = PLUS ? DotSum::CANONICAL : DotSum::CENTRED;
#pragma unroll
            for (int o = 0; o < C; o += ROOM) {
                DotSum d[4];
#pragma unroll
                for (int i = 0; i < 4; i++) d[i].open(s[i]);
#pragma unroll
                for (int c = o; c < o + ROOM && c < C; c++) {
                    if constexpr (PLUS) b[c] = b[c] + e[c];
                    d[0].add(f[c][0].x, b[c].x);
                    d[1].add(f[c][0].y, b[c].y);
                    d[2].add(f[c][1].x, b[c].x);
                    d[3].add(f[c][1].y, b[c].y);
                }
#pragma unroll
                for (int i = 0; i < 4; i++) s[i] = d[i].close(m);
            }
        }
        put_lane(out, lane, cg_double2v{s[0], s[1]});
        put_lane(out + (size_t)k * row, lane, cg_double2v{s[2], s[3]});
        w += (size_t)n_diag * k * row;
        if constexpr (PLUS) plus += (size_t)n_diag * k * row;
        out += (size_t)2 * k * row;
    }
}
template <int C, bool HELD>
__global__ void __launch_bounds__(PRODUCT_THREADS)
products_kernel(ProductArgs A, Tables T)
{
    const int k = T.k, logn = T.logn, blocks = (1 << logn) / (2 * PRODUCT_THREADS);
    // neighbours on an XCD: the requests, which share the diagonals
    const int l = xcd_row((int)blockIdx.x, (int)gridDim.x, A.requests);
    const int r = l % A.requests, q = l / A.requests, part = q % A.parts, at = q / A.parts, i = at / blocks, block = at % blocks;
    const int u0 = part * A.per, n = min(A.per, A.units - u0);
    const int lane = block * PRODUCT_THREADS + (int)threadIdx.x;
    const ModD m = T.C->mod[i];
    const int own = A.adapters ? A.pick[r] : -1;
    auto row = [&](const double *p, size_t at_row) { return reinterpret_cast<const cg_double2v *>(p + (at_row << logn)); };
    const cg_double2v *x = row(A.copies, (size_t)r * A.n_diag * 2 * k + i), *w = row(A.diags, (size_t)u0 * A.n_diag * k + i);
    cg_double2v *out = reinterpret_cast<cg_double2v *>(A.out + ((((size_t)r * A.units + u0) * 2 * k + i) << logn));
    // With fewer adapters than requests some are shared and stay in the caches; as many are taken for each request's own and pass them by.  us a
    // projection of 16 requests and 36 matrices, in the caches / by them: 16 adapters 2017 / 2004, eight of two requests each 1965 / 1981, four 1944 /
    // 1955, one 1928 / 1946.
    const cg_double2v *plus = row(A.adapters, ((size_t)max(own, 0) * A.units + u0) * A.n_diag * k + i);
    if (own < 0 || own >= A.n_adapters) products_of<C, HELD, false, false>(x, w, w, out, A.n_diag, n, k, logn, lane, m);
    else if (A.n_adapters < A.requests) products_of<C, HELD, true, false>(x, w, plus, out, A.n_diag, n, k, logn, lane, m);
    else products_of<C, HELD, true, true>(x, w, plus, out, A.n_diag, n, k, logn, lane, m);
}
// Rows of such sums back in coefficients, in place: 3456 rows of 8192 in 89 us, 5.1 TB/s.
template <int LOGN, int E>
__global__ void __launch_bounds__((1 << LOGN) / E, (min_waves<LOGN, E>()))
sums_kernel(double *rows, Tables T)
{
    __shared__ __align__(16) double lds[lds_doubles<LOGN>()];
    constexpr int TH = (1 << LOGN) / E;
    const int tid = threadIdx.x, i = (int)blockIdx.x % T.k;
    double *row = rows + ((size_t)blockIdx.x << LOGN), v[E], w[E];
#pragma unroll
    for (int it = 0; it < E; it += 2) {
        const cg_double2v x = at_lane(reinterpret_cast<const cg_double2v *>(row) + 32 * it, chunk_elem<E>(tid, 0) / 2);
        v[it] = x.x;
        v[it + 1] = x.y;
    }
    const ModD m = T.C->mod[i];
    inv_row<LOGN, E, false, hundredths(DotSum::OUT)>(lds, v, StRegs{w}, 0, tid, T.itw + ((size_t)i << LOGN), m, i, T.C);
#pragma unroll
    for (int it = 0; it < E; it++) put_lane(reinterpret_cast<uint64_t *>(row) + it * TH, tid, f64_to_u64(canon(w[it], m)));
}

// ---------------------------------------------------------------------------
// Position biases.  Only slots b d2 carry one: the values at zeta^(+-e), e = 3^(d2 b) = 1 modulo 4 d2, which are the
// roots of X^n' - w and X^n' - 1/w with n' = N / (2 d2), w = zeta^n'.  So the polynomial is
//   m_j = N^-1 (A_(j mod n') zeta^-j + B_(j mod n') zeta^j),  A, B transforms of n' points of the two rows' values,
// two products a coefficient where the interpolation of any slots takes log2(N) / 2.  Bound by component 0's way from memory and
// back: 1536 ciphertexts of N = 8192 and three primes in 124 us, 4.9 TB/s; 384 in 31.5 (the words asked for behind the bias 34.9; a part of four times as many
// coefficients, with as many loads in flight, 35.6).
// ---------------------------------------------------------------------------
struct BiasArgs {
    const uint64_t *in;
    uint64_t *out;
    const int32_t *pos;        // null: the diagonals of prompts
    const int64_t *table;
    const int32_t *edges;
    int n_buckets, heads, n_cts, log_d2;
    // bias of distance `dist`, and head h
    __device__ __forceinline__ double bias(int dist, int h, const ModD mt, double two32_t) const
    {
        if (dist < 0) return 0.0;
        int lo = 0;                      // edges at or below the distance
        // A few as scalar loads at once, where a search waits for each of its steps; a prompt's workgroups, with more of them, hide more of the
        // loop.  us, loop / search, N = 8192: 384 ciphertexts of scores 8 buckets 28.2 / 28.9, 32 28.7 / 29.2, 64 29.6 / 29.3, 128 34.8 / 29.6 (one 16 5.9 / 5.8,
        // 64 7.6 / 6.0; 384 of N = 4096 and 256 tokens 32 14.3 / 13.0, 64 16.3 / 13.2); 1536 of a prompt 32 106 / 110, 64 108 / 112, 128 112 / 112.
        if (n_buckets <= (pos ? 32 : 64)) {
            for (int i = 0; i < n_buckets; i++) lo += edges[i] <= dist;
        } else {
            for (int hi = n_buckets; lo < hi;) {
                const int mid = (lo + hi) >> 1;
                if (edges[mid] <= dist) lo = mid + 1;
                else hi = mid;
            }
        }
        return lo ? red(of_int64(table[(size_t)(lo - 1) * heads + h], two32_t), mt) : 0.0;
    }
};
constexpr int BIAS_THREADS = 256;
// dynamic LDS: 2 n' floats.  A workgroup takes PAIRS pairs of coefficients a thread modulo every prime, K of them.
template <int K, int PAIRS>
__global__ void __launch_bounds__(BIAS_THREADS)
bias_kernel(BiasArgs A, Tables T)
{
    extern __shared__ float ab[];      // A, then B (centred residues below 2^19: exact)
    const int tid = threadIdx.x, logn = T.logn, N = 1 << logn;
    const int parts = N / (2 * PAIRS * BIAS_THREADS), unit = (int)blockIdx.x / parts, first = (int)blockIdx.x % parts * (2 * PAIRS * BIAS_THREADS);
    const uint64_t *in = A.in + (((size_t)unit * 2 * K) << logn) + first;
    uint64_t *out = A.out + (((size_t)unit * 2 * K) << logn) + first;
    // what the bias is added to is on its way while the bias is made
    cg_ulong2v x[PAIRS][K];
#pragma unroll
    for (int p = 0; p < PAIRS; p++)
#pragma unroll
        for (int i = 0; i < K; i++) x[p][i] = at_lane(reinterpret_cast<const cg_ulong2v *>(in + ((size_t)i << logn)) + p * BIAS_THREADS, tid);
    const int ld2 = A.log_d2, log_np = logn - 1 - ld2, np = 1 << log_np;
    const ModD mt = T.C->mod[K];
    const int c = unit % A.n_cts, h = unit / A.n_cts % A.heads, r = unit / (A.n_cts * A.heads);
    const int at_pos = A.pos ? A.pos[r] : 0;
    // values in the order that the decimation in time takes them: B's, whose roots are the reciprocals, from the other end
    for (int t = tid; t < 2 * np; t += BIAS_THREADS) {
        const int row = t >> log_np, b = t & (np - 1);
        int dist;
        if (A.pos) {
            dist = at_pos < 0 ? -1 : at_pos - (c * 2 * np + t);
        } else {
            const int sigma = c >> log_np, rot = c & (np - 1);
            dist = t - ((row ^ sigma) * np + ((b + rot) & (np - 1)));
        }
        int at = (int)(T.pow3[b << ld2] >> (ld2 + 2));      // (3^(d2 b) - 1) / (4 d2)
        if (row) at = (np - at) & (np - 1);
        ab[row * np + (int)(__brev((unsigned)at) >> (32 - log_np))] = (float)A.bias(dist, h, mt, T.two32_t);
    }
    __syncthreads();
    for (int s = 0; s < log_np; s++) {
        for (int t = tid; t < np; t += BIAS_THREADS) {
            const int row = t >> (log_np - 1), q = t & (np / 2 - 1), j = q & ((1 << s) - 1);
            float *y = ab + row * np + ((q >> s) << (s + 1)) + j;
            // omega^-j for blocks of 2^(s + 1): zeta^-(2N / 2^(s + 1) j)
            const double w = T.zeta[(2 * N - ((2 * N) >> (s + 1)) * j) & (2 * N - 1)];
            const double hi = mulmod((double)y[1 << s], w, mt), lo = (double)y[0];
            y[0] = (float)red(lo + hi, mt);
            y[1 << s] = (float)red(lo - hi, mt);
        }
        __syncthreads();
    }
#pragma unroll
    for (int p = 0; p < PAIRS; p++) {
        const int j = first + 2 * (p * BIAS_THREADS + tid);
        double m[2];
#pragma unroll
        for (int e = 0; e < 2; e++) {
            const int i = (j + e) & (np - 1);
            const double sum = (double)ab[i] * (double)T.zeta[(2 * N - j - e) & (2 * N - 1)] + (double)ab[np + i] * (double)T.zeta[j + e];
            m[e] = canon(mulmod(red(sum, mt), T.ninv_t, mt), mt);
        }
#pragma unroll
        for (int i = 0; i < K; i++) {
            const ModD q = T.C->mod[i];
            const double delta = T.C->delta_q[i];
            put_lane(reinterpret_cast<cg_ulong2v *>(out + ((size_t)i << logn)) + p * BIAS_THREADS, tid,
                     cg_ulong2v{f64_to_u64(canon(u64_to_f64(x[p][i].x) + mulmod(m[0], delta, q), q)),
                                f64_to_u64(canon(u64_to_f64(x[p][i].y) + mulmod(m[1], delta, q), q))});
        }
    }
    if (A.in != A.out) {
#pragma unroll
        for (int p = 0; p < PAIRS; p++)
#pragma unroll
            for (int i = K; i < 2 * K; i++)
                put_lane(reinterpret_cast<cg_ulong2v *>(out + ((size_t)i << logn)) + p * BIAS_THREADS, tid,
                         at_lane(reinterpret_cast<const cg_ulong2v *>(in + ((size_t)i << logn)) + p * BIAS_THREADS, tid));
    }
}

// ---------------------------------------------------------------------------
// Append at each request's own length: row (request, cache, component, prime), its transform, the product with the block's mask and the
// transform back in one workgroup.  A request whose length has no place leaves at once.  Bound by vector issue (75 % busy on 4032 rows of
// 8192, 58 ns each; their bytes alone would take 36): 64 registers a thread, so that two workgroups of 1024 threads share a unit (234 us; rows on 512
// threads 238, in 66 registers 243).  Mask and addends asked for with the row 266: loads return in order, and the passes' factors wait.
// ---------------------------------------------------------------------------
struct AppendArgs {
    uint64_t *cache;
    const uint64_t *rows;
    const double *masks;
    const int32_t *lens;
    int per, log_blocks;
    uint32_t stride, row_stride;
};
template <int LOGN, int E>
__global__ void __launch_bounds__((1 << LOGN) / E, (two_waves<LOGN, E>()))
append_kernel(AppendArgs A, Tables T)
{
    __shared__ __align__(16) double lds[lds_doubles<LOGN>()];
    constexpr int TH = (1 << LOGN) / E;
    constexpr int IN = hundredths(prod_of(FwdBound<LOGN, E, Plan<LOGN, E>::NP - 1>::out));
    const int tid = threadIdx.x, k = T.k;
    const int row = (int)blockIdx.x, i = row % k, in_ct = row % (2 * k), rc = row / (2 * k), r = rc / A.per, c = rc % A.per;
    const int len = A.lens[r];
    if (len < 0 || (uint32_t)(len >> A.log_blocks) >= A.stride) return;
    const int block = len & ((1 << A.log_blocks) - 1);
    const uint64_t *src = A.rows + ((((size_t)r * A.row_stride + c) * 2 * k + in_ct) << LOGN);
    uint64_t *dst = A.cache + ((((size_t)rc * A.stride + (len >> A.log_blocks)) * 2 * k + in_ct) << LOGN);
    const double *mask = A.masks + ((size_t)(block * k + i) << LOGN);
    const ModD m = T.C->mod[i];
    double v[E], w[E];
#pragma unroll
    for (int it = 0; it < E; it++) v[it] = u64_to_f64(at_lane(src + it * TH, tid));
    fwd_row<LOGN, E, false>(lds, v, w, tid, T.tw + ((size_t)i << LOGN), m);
#pragma unroll
    for (int it = 0; it < E; it += 2) {
        const cg_double2v f = at_lane(reinterpret_cast<const cg_double2v *>(mask) + 32 * it, chunk_elem<E>(tid, 0) / 2);
        v[it] = mulmod(w[it], f.x, m);
        v[it + 1] = mulmod(w[it + 1], f.y, m);
    }
    // (asked for before the last two passes, whose factors are scalar loads and wait behind nothing)
    uint64_t old[E];
    inv_row<LOGN, E, false, IN>(lds, v, StRegs{w}, 0, tid, T.itw + ((size_t)i << LOGN), m, i, T.C, 0, [&] {
#pragma unroll
        for (int it = 0; it < E; it++) old[it] = 0;
        if (block) {
#pragma unroll
            for (int it = 0; it < E; it++) old[it] = at_lane(dst + it * TH, tid);
        }
    });
#pragma unroll
    for (int it = 0; it < E; it++) put_lane(dst + it * TH, tid, f64_to_u64(canon(w[it] + u64_to_f64(old[it]), m)));
}

}  // namespace cgr
