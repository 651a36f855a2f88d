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
    const uint16_t *slot;      // transform output j modulo t is slot slot[j]
    const float *zeta;         // zeta^e mod t, centred, e < 2N
    const uint16_t *pow3;      // 3^i mod 2N, i < N/2
    double ninv_t;             // N^-1 mod t, centred
    int logn, k;
};

// ---------------------------------------------------------------------------
// Slot values -> polynomial modulo t -> prepared plaintext.  The interpolation is an inverse transform modulo t of the
// values in the order of the transform's outputs; its results are centred in registers and go through one forward
// transform per ciphertext prime without leaving the workgroup.
// ---------------------------------------------------------------------------
struct LdSlots {
    const int64_t *v;
    int logn;
    __device__ __forceinline__ double value(int b, int slot, const ModD) const { return (double)(int)at32(v + ((size_t)b << logn), slot); }
};
// slot `slot` of diagonal c of unit u, b = u n_diag + c: M[f][slot mod d2], f the feature that the token's copy c shows there
template <class T>
struct LdDiagonal {
    const T *m;                 // [units][d1][d2]
    int logn, log_tile, log_diag, log_d2, d1;
    __device__ __forceinline__ double value(int b, int slot, const ModD) const
    {
        const int half = 1 << (logn - 1), n_diag = 1 << log_diag, tile = 1 << log_tile;
        const int u = b >> log_diag, c = b & (n_diag - 1);
        const int at = (slot & half) | ((slot + c) & (half - 1));
        const int f = (at + n_diag * (at >> log_tile)) & (tile - 1);
        if (f >= d1) return 0.0;
        return (double)(int)m[(((size_t)u * d1 + f) << log_d2) + (slot & ((1 << log_d2) - 1))];
    }
};

template <int LOGN, int E, bool PREPARED, class LD>
__global__ void __launch_bounds__((1 << LOGN) / E, (min_waves<LOGN, E>()))
encode_kernel(LD ld, void *__restrict__ out, Tables T, int split)
{
    __shared__ __align__(16) double lds[lds_doubles<LOGN>()];
    constexpr int TH = (1 << LOGN) / E;
    const int tid = threadIdx.x, k = T.k;
    const int b = (int)blockIdx.x / split, part = (int)blockIdx.x % split;
    const ModD mt = T.C->mod[k];
    double v[E], w[E];
#pragma unroll
    for (int it = 0; it < E; it++) v[it] = red(ld.value(b, T.slot[chunk_elem<E>(tid, it)], mt), mt);
    inv_row<LOGN, E>(lds, v, StRegs{w}, 0, tid, T.itw + ((size_t)k << LOGN), mt, k, T.C);
    if constexpr (!PREPARED) {
        uint64_t *row = static_cast<uint64_t *>(out) + ((size_t)b << LOGN);
#pragma unroll
        for (int it = 0; it < E; it++) put_lane(row + it * TH, tid, f64_to_u64(canon(w[it], mt)));
    } else {
        // |w| <= (t - 1) / 2: t is odd, so the rounded quotient of an integer is never in doubt
#pragma unroll
        for (int it = 0; it < E; it++) w[it] = red(w[it], mt);
        for (int i = part; i < k; i += split) {
            const ModD m = T.C->mod[i];
            lds_barrier();      // the last pass read other waves' elements, or its chunk is still being copied out
            fwd_row<LOGN, E, false, false, 1, 1>(lds, w, v, tid, T.tw + ((size_t)i << LOGN), m);
            double *row = static_cast<double *>(out) + ((size_t)(b * k + i) << LOGN);
#pragma unroll
            for (int it = 0; it < E; it += 2)
                put_lane(reinterpret_cast<cg_double2v *>(row) + 32 * it, chunk_elem<E>(tid, 0) / 2,
                         cg_double2v{red(v[it], m), red(v[it + 1], m)});
        }
    }
}

// ---------------------------------------------------------------------------
// M_u = W_u + A B_u modulo t for the diagonals of adapters: 16 x 16 tiles on the matrix cores in FP64, exact because centred
// entries are below 2^19 and rank 2^38 below 2^53.  A wave takes 16 features and up to 64 columns.
// ---------------------------------------------------------------------------
typedef double cg_double4v __attribute__((ext_vector_type(4)));
__global__ void __launch_bounds__(256)
low_rank_kernel(const int64_t *__restrict__ w, const int64_t *__restrict__ a, const int64_t *__restrict__ b, float *__restrict__ out, int a_group,
                int d1, int d2, int rank, int row_blocks, Tables T)
{
    const ModD mt = T.C->mod[T.k];
    const int u = (int)blockIdx.x / row_blocks, lane = threadIdx.x & 63;
    const int f0 = ((int)blockIdx.x % row_blocks) * 64 + ((int)threadIdx.x >> 6) * 16, c0 = (int)blockIdx.y * 64;
    const int i = lane & 15, q = lane >> 4;
    const int64_t *au = a + (size_t)(u / a_group) * d1 * rank, *bu = b + (size_t)u * rank * d2;
    cg_double4v acc[4] = {};
    for (int j0 = 0; j0 < rank; j0 += 4) {
        const int j = j0 + q;
        const double x = f0 + i < d1 && j < rank ? red((double)(int)au[(size_t)(f0 + i) * rank + j], mt) : 0.0;
#pragma unroll
        for (int c = 0; c < 4; c++) {
            const int col = c0 + 16 * c + i;
            const double y = col < d2 && j < rank ? red((double)(int)bu[(size_t)j * d2 + col], mt) : 0.0;
            acc[c] = __builtin_amdgcn_mfma_f64_16x16x4f64(x, y, acc[c], 0, 0, 0);
        }
    }
#pragma unroll
    for (int c = 0; c < 4; c++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int f = f0 + 4 * e + q, col = c0 + 16 * c + i;
            if (f >= d1 || col >= d2) continue;
            const size_t at = ((size_t)u * d1 + f) * d2 + col;
            double v = red(acc[c][e], mt);
            if (w) v = red(v + (double)(int)w[at], mt);
            out[at] = (float)v;
        }
}

// ---------------------------------------------------------------------------
// The copies of all tokens, transformed: row (r, c, component, prime), copy 0 being the token itself
// ---------------------------------------------------------------------------
template <int LOGN, int E>
__global__ void __launch_bounds__((1 << LOGN) / E, (min_waves<LOGN, E>()))
copies_kernel(const uint64_t *__restrict__ x, const uint64_t *__restrict__ copies, double *__restrict__ out, int n_diag, Tables T)
{
    __shared__ __align__(16) double lds[lds_doubles<LOGN>()];
    constexpr int TH = (1 << LOGN) / E;
    const int tid = threadIdx.x, k = T.k;
    const int row = (int)blockIdx.x, i = row % k, cp = row / (2 * k), r = cp / n_diag, c = cp % n_diag;
    const int in_ct = row % (2 * k);
    const uint64_t *src = c ? copies + ((size_t)((r * (n_diag - 1) + c - 1) * 2 * k + in_ct) << LOGN) : x + ((size_t)(r * 2 * k + in_ct) << LOGN);
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
// y[r][u] = sum over c of copy_(r, c) times (diagonal_(u, c) + that of the request's adapter), back in coefficients: row
// (r, u, component, prime)
// ---------------------------------------------------------------------------
template <int LOGN, int E>
__global__ void __launch_bounds__((1 << LOGN) / E, (min_waves<LOGN, E>()))
project_kernel(const double *__restrict__ copies, const double *__restrict__ diags, const double *__restrict__ adapters, int n_adapters,
               const int32_t *__restrict__ pick, int units, int n_diag, uint64_t *__restrict__ out, Tables T)
{
    __shared__ __align__(16) double lds[lds_doubles<LOGN>()];
    constexpr int TH = (1 << LOGN) / E;
    const int tid = threadIdx.x, k = T.k;
    const int row = (int)blockIdx.x, i = row % k, comp = row / k % 2, ru = row / (2 * k), r = ru / units, u = ru % units;
    const ModD m = T.C->mod[i];
    const int own = adapters ? pick[r] : -1;
    const double *plus = own >= 0 && own < n_adapters ? adapters + ((((size_t)own * units + u) * n_diag * k + i) << LOGN) : nullptr;
    const double *w = diags + (((size_t)u * n_diag * k + i) << LOGN), *x = copies + (((size_t)r * n_diag * 2 * k + comp * k + i) << LOGN);
    double v[E], z[E];
#pragma unroll
    for (int it = 0; it < E; it++) v[it] = 0.0;
    for (int c = 0; c < n_diag; c++) {
#pragma unroll
        for (int it = 0; it < E; it++) {
            const int idx = chunk_elem<E>(tid, it);
            double f = at32(w + ((size_t)(c * k) << LOGN), idx);
            if (plus) f += at32(plus + ((size_t)(c * k) << LOGN), idx);
            v[it] = red(v[it], m) + mulmod(at32(x + ((size_t)(c * 2 * k) << LOGN), idx), f, m);
        }
    }
    inv_row<LOGN, E>(lds, v, StRegs{z}, 0, tid, T.itw + ((size_t)i << LOGN), m, i, T.C);
#pragma unroll
    for (int it = 0; it < E; it++) put_lane(out + ((size_t)row << LOGN) + it * TH, tid, f64_to_u64(canon(z[it], m)));
}

// ---------------------------------------------------------------------------
// Position biases.  Only slots b d2 carry one: the values at zeta^(+-e), e = 3^(d2 b) = 1 modulo 4 d2, which are the
// roots of X^n' - w and X^n' - 1/w with n' = N / (2 d2), w = zeta^n'.  So the polynomial is
//   m_j = N^-1 (A_(j mod n') zeta^-j + B_(j mod n') zeta^j),  A, B transforms of n' points of the two rows' values,
// two products a coefficient where the interpolation of any slots takes log2(N) / 2.
// ---------------------------------------------------------------------------
struct BiasArgs {
    const uint64_t *in;
    uint64_t *out;
    const int32_t *pos;        // null: the diagonals of prompts
    const int64_t *table;
    const int32_t *edges;
    int n_buckets, heads, n_cts, log_d2, parts;
    // bias of distance `dist`, and head h
    __device__ __forceinline__ double bias(int dist, int h, const ModD mt) const
    {
        if (dist < 0) return 0.0;
        int lo = 0, hi = n_buckets;      // edges[lo - 1] <= dist < edges[hi]
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (edges[mid] <= dist) lo = mid + 1;
            else hi = mid;
        }
        return lo ? red((double)(int)table[(size_t)(lo - 1) * heads + h], mt) : 0.0;
    }
};
constexpr int BIAS_THREADS = 256;
// dynamic LDS: 2 n' floats
__global__ void __launch_bounds__(BIAS_THREADS)
bias_kernel(BiasArgs A, Tables T)
{
    extern __shared__ float ab[];      // A, then B (centred residues below 2^19: exact)
    const int tid = threadIdx.x, logn = T.logn, N = 1 << logn, k = T.k;
    const int unit = (int)blockIdx.x / A.parts, part = (int)blockIdx.x % A.parts;
    const int ld2 = A.log_d2, log_np = logn - 1 - ld2, np = 1 << log_np;
    const ModD mt = T.C->mod[k];
    const int c = unit % A.n_cts, h = unit / A.n_cts % A.heads, r = unit / (A.n_cts * A.heads);
    const int p = A.pos ? A.pos[r] : 0;
    // values in the order that the decimation in time takes them: B's, whose roots are the reciprocals, from the other end
    for (int t = tid; t < 2 * np; t += BIAS_THREADS) {
        const int row = t >> log_np, b = t & (np - 1);
        int dist;
        if (A.pos) {
            dist = p - (c * 2 * np + t);
            if (p < 0) dist = -1;
        } else {
            const int sigma = c >> log_np, rot = c & (np - 1);
            dist = t - ((row ^ sigma) * np + ((b + rot) & (np - 1)));
        }
        int at = (int)(T.pow3[b << ld2] >> (ld2 + 2));      // (3^(d2 b) - 1) / (4 d2)
        if (row) at = (np - at) & (np - 1);
        ab[row * np + (log_np ? (int)(__brev((unsigned)at) >> (32 - log_np)) : 0)] = (float)A.bias(dist, h, mt);
    }
    __syncthreads();
    for (int s = 0; s < log_np; s++) {
        for (int t = tid; t < np; t += BIAS_THREADS) {
            const int row = t >> (log_np - 1), q = t & (np / 2 - 1), j = q & ((1 << s) - 1);
            float *x = ab + row * np + ((q >> s) << (s + 1)) + j;
            // omega^-j for blocks of 2^(s + 1): zeta^-(2N / 2^(s + 1) j)
            const double w = T.zeta[(2 * N - ((2 * N) >> (s + 1)) * j) & (2 * N - 1)];
            const double hi = mulmod((double)x[1 << s], w, mt), lo = (double)x[0];
            x[0] = (float)red(lo + hi, mt);
            x[1 << s] = (float)red(lo - hi, mt);
        }
        __syncthreads();
    }
    const uint64_t *in = A.in + (((size_t)unit * 2 * k) << logn);
    uint64_t *out = A.out + (((size_t)unit * 2 * k) << logn);
    const int per = N / A.parts;
    for (int j = part * per + 2 * tid; j < (part + 1) * per; j += 2 * BIAS_THREADS) {
        double m[2];
#pragma unroll
        for (int e = 0; e < 2; e++) {
            const int i = (j + e) & (np - 1);
            const double sum = (double)ab[i] * (double)T.zeta[(2 * N - j - e) & (2 * N - 1)] + (double)ab[np + i] * (double)T.zeta[j + e];
            m[e] = canon(mulmod(red(sum, mt), T.ninv_t, mt), mt);
        }
        for (int i = 0; i < k; i++) {
            const ModD q = T.C->mod[i];
            const double delta = T.C->delta_q[i];
            const cg_ulong2v x = *reinterpret_cast<const cg_ulong2v *>(in + ((size_t)i << logn) + j);
            *reinterpret_cast<cg_ulong2v *>(out + ((size_t)i << logn) + j) =
                cg_ulong2v{f64_to_u64(canon(u64_to_f64(x.x) + mulmod(m[0], delta, q), q)), f64_to_u64(canon(u64_to_f64(x.y) + mulmod(m[1], delta, q), q))};
        }
        if (A.in != A.out)
            for (int i = k; i < 2 * k; i++)
                *reinterpret_cast<cg_ulong2v *>(out + ((size_t)i << logn) + j) = *reinterpret_cast<const cg_ulong2v *>(in + ((size_t)i << logn) + j);
    }
}

// ---------------------------------------------------------------------------
// Append at each request's own length: row (request, cache, component, prime), its transform, the product with the block's mask and the
// transform back in one workgroup.  A request whose length has no place leaves at once.
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
__global__ void __launch_bounds__((1 << LOGN) / E, (min_waves<LOGN, E>()))
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
    inv_row<LOGN, E, false, IN>(lds, v, StRegs{w}, 0, tid, T.itw + ((size_t)i << LOGN), m, i, T.C);
    uint64_t old[E];
#pragma unroll
    for (int it = 0; it < E; it++) old[it] = block ? at_lane(dst + it * TH, tid) : 0;
#pragma unroll
    for (int it = 0; it < E; it++) put_lane(dst + it * TH, tid, f64_to_u64(canon(w[it] + u64_to_f64(old[it]), m)));
}

}  // namespace cgr
