// es_dense.hip -- layers of networks and their gradients on gfx950.
//
//   k_gemm        one matrix product per member, C = sum A B, with bias,
//                 activation, the gate's product and the residual applied to
//                 the accumulators before they are rounded and stored
//   k_gemm_join   the same epilogue behind a split reduction
//   k_gradz       dz = dy act'(pre) and its column sums
//   k_bias_grad   those sums added up
//
// The matrix cores hold D = A B with the rows of B^T as the lanes: the n side
// (outputs) is the instruction's A operand and the m side (inputs' rows) its B
// operand, so that a lane's four accumulators of a tile lie in one row of C.
// A wave owns 64 x 64 of C as 4 x 4 tiles; tile b of the n side takes the rows
// n = 16 (r / 4) + 4 b + r % 4 of its 64 (r: row of the instruction), so that a
// lane ends with 16 consecutive outputs of a row, stored in 16-byte pieces.
// A gated layer's 64 are 32 gates and the 32 matching others, and a lane has
// both factors of 8 consecutive outputs.
#include <hip/hip_runtime.h>
#include <math.h>

#include "es_dense.hpp"
#include "es_dense_device.hpp"

namespace esmi {

namespace {

// ---- the product ----------------------------------------------------------
constexpr int TILE = 128;  // C is cut into TILE x TILE (n: 64 outputs for a gated layer's both factors)
constexpr int LROW = 144;  // bytes of a staged row: 128 of k and a pad that spreads the rows over the banks

// 16 bytes of a row from any address, zeros behind `left` elements
template <typename T>
__device__ __forceinline__ uintx4 load16(const T* p, int64_t left)
{
    constexpr int E = 16 / sizeof(T);
    uintx4 v = {0, 0, 0, 0};
    if (left >= E) {
        __builtin_memcpy(&v, p, 16);
    } else {
        T t[E];
#pragma unroll
        for (int i = 0; i < E; ++i) t[i] = i < left ? p[i] : (T)0.f;
        __builtin_memcpy(&v, t, 16);
    }
    return v;
}

// Row of the staged n side that tile b's instruction row r takes.
template <bool GATED>
__device__ __forceinline__ int slot(int b, int r)
{
    return GATED ? 32 * (b >> 1) + 8 * (r >> 2) + 4 * (b & 1) + (r & 3) : 16 * (r >> 2) + 4 * b + (r & 3);
}

// 128 bytes of k for `rows` of one operand, staged with k contiguous.
template <typename T, bool KMAJOR, bool GATED>
struct Stage {
    static constexpr int E = 16 / sizeof(T), BK = 128 / sizeof(T);
    uintx4 v[4];

    // row `i` of the staged 128 is memory row (or column) row_of(i), -1: none
    template <typename F>
    __device__ __forceinline__ void load(const T* base, int64_t stride, int32_t k0, int32_t K, int32_t limit, F row_of)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = (int)threadIdx.x + 256 * j;
            v[j] = uintx4{0, 0, 0, 0};
            if constexpr (KMAJOR) {
                const int64_t row = row_of(c / 8);
                const int32_t k = k0 + (c % 8) * E;
                if (row >= 0 && k < K) v[j] = load16(base + row * stride + k, K - k);
            } else {
                constexpr int PER = TILE / E;  // pieces of a k row
                const int32_t k = k0 + c / PER;
                const int64_t row = row_of((c % PER) * E);
                if (row >= 0 && k < K) v[j] = load16(base + (int64_t)k * stride + row, limit - row);
            }
        }
    }
    __device__ __forceinline__ void store(unsigned char* lds) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = (int)threadIdx.x + 256 * j;
            if constexpr (KMAJOR) {
                *reinterpret_cast<uintx4*>(lds + (c / 8) * LROW + (c % 8) * 16) = v[j];
            } else {
                constexpr int PER = TILE / E;
                T t[E];
                __builtin_memcpy(t, &v[j], 16);
#pragma unroll
                for (int i = 0; i < E; ++i)
                    *reinterpret_cast<T*>(lds + ((c % PER) * E + i) * LROW + (c / PER) * (int)sizeof(T)) = t[i];
            }
        }
    }
};

template <typename T, bool AK, bool BK, bool GATED>
__global__ __launch_bounds__(256) void k_gemm(GemmArgs a)
{
    __shared__ __align__(16) unsigned char sa[TILE * LROW], sb[TILE * LROW];
    const Gemm& g = a.g;
    constexpr int KT = 128 / sizeof(T);
    constexpr int BN = GATED ? TILE / 2 : TILE;
    int64_t id = blockIdx.x;
    const int32_t tn = (int32_t)(id % a.nt);
    id /= a.nt;
    const int32_t tm = (int32_t)(id % a.mt);
    id /= a.mt;
    const int32_t split = (int32_t)(id % a.splits);
    const int64_t batch = id / a.splits;
    const int32_t m0 = tm * TILE, n0 = tn * BN;
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, q = lane / 16, l16 = lane % 16;
    const int wm = wave / 2, wn = wave % 2;
    const int64_t steps = g.red * a.kt, first = steps * split / a.splits, last = steps * (split + 1) / a.splits;
    const T* A = static_cast<const T*>(g.a) + batch * g.a_batch;
    const T* B = static_cast<const T*>(g.b) + batch * g.b_batch;
    auto row_a = [&](int i) -> int64_t { return m0 + i < g.M ? m0 + i : -1; };
    auto row_b = [&](int i) -> int64_t {
        if constexpr (GATED) {
            const int32_t n = n0 + 32 * (i / 64) + i % 32;
            return n < g.N ? n + (i / 32 % 2 ? (int64_t)g.N : 0) : -1;
        } else {
            return n0 + i < g.N ? n0 + i : -1;
        }
    };

    floatx4 acc[4][4];  // [m tile][n tile]
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    Stage<T, AK, false> va;
    Stage<T, BK, GATED> vb;
    auto fetch = [&](int64_t t) {
        const int64_t r = t / a.kt;
        const int32_t k0 = (int32_t)(t % a.kt) * KT;
        va.load(A + r * g.a_red, g.a_row, k0, g.K, g.M, row_a);
        vb.load(B + r * g.b_red, g.b_row, k0, g.K, g.N, row_b);
    };
    if (first < last) fetch(first);
    for (int64_t t = first; t < last; ++t) {
        __syncthreads();
        va.store(sa);
        vb.store(sb);
        __syncthreads();
        if (t + 1 < last) fetch(t + 1);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            uintx4 fa[4], fb[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fa[i] = *reinterpret_cast<const uintx4*>(sa + (64 * wm + 16 * i + l16) * LROW + ks * 64 + q * 16);
                fb[i] = *reinterpret_cast<const uintx4*>(sb + (64 * wn + slot<GATED>(i, l16)) * LROW + ks * 64 + q * 16);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = product<T>(fb[j], fa[i], acc[i][j]);
        }
    }

    // a lane's outputs of a row: 16 in a row, or 8 of a gated layer
    constexpr int W = GATED ? 8 : 16;
    const int64_t n = GATED ? n0 + 32 * wn + 8 * q : n0 + 64 * wn + 16 * q;
    float bz[W], bu[W];
    load_bias<T, GATED, W>(g, batch, n, bz, bu);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + 64 * wm + 16 * i + l16;
        if (m >= g.M) continue;
        float z[W], u[W];
#pragma unroll
        for (int e = 0; e < W; ++e) {
            z[e] = acc[i][e / 4][e % 4];
            u[e] = GATED ? acc[i][(e / 4 + 2) % 4][e % 4] : 0.f;
        }
        if (a.splits > 1) store_partial<GATED, W>(a, split, batch, m, n, z, u);
        else {
            float r[W];
            load_res<T, W>(a, batch, m, n, r);
            finish<T, GATED, W>(a, batch, m, n, z, u, bz, bu, r);
        }
    }
}

template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_gemm_join(GemmArgs a)
{
    const Gemm& g = a.g;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, MN = (int64_t)g.M * g.N;
    if (id >= g.batches * MN) return;
    const int64_t batch = id / MN, m = id % MN / g.N, n = id % g.N;
    const int64_t wide = GATED ? 2 * (int64_t)g.N : g.N;
    float z = 0.f, u = 0.f, bz, bu, r;
    load_bias<T, GATED, 1>(g, batch, n, &bz, &bu);
    load_res<T, 1>(a, batch, m, n, &r);
    for (int32_t s = 0; s < a.splits; ++s) {
        const float* p = a.partial + ((s * g.batches + batch) * g.M + m) * wide + n;
        z += p[0];
        if constexpr (GATED) u += p[g.N];
    }
    finish<T, GATED, 1>(a, batch, m, n, &z, &u, &bz, &bu, &r);
}

bool whole(const void* p, int64_t row, int64_t batch, int64_t rows, int64_t batches, size_t elem)
{
    return p && reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows <= 1 || row * elem % 16 == 0) &&
           (batches <= 1 || batch * elem % 16 == 0);
}

GemmArgs plan(const Gemm& g)
{
    GemmArgs a{};
    a.g = g;
    const size_t e = dtype_size(g.dtype);
    a.vec_c = whole(g.c, g.c_row, g.c_batch, g.M, g.batches, dtype_size(g.c_dtype));
    a.vec_res = whole(g.res, g.res_row, g.res_batch, g.M, g.batches, e);
    a.vec_pre = whole(g.pre, g.pre_row, g.pre_batch, g.M, g.batches, e) && (!g.gated || g.N * e % 16 == 0);
    a.splits = 1;
    if (rows_fits(g)) {
        rows_plan(a);
        return a;
    }
    if (large_fits(g)) {
        large_plan(a);
        return a;
    }
    const int32_t kt = 128 / (int32_t)e, bn = g.gated ? TILE / 2 : TILE;
    a.path = PATH_STAGED;
    a.mt = (g.M - 1) / TILE + 1;
    a.nt = (g.N - 1) / bn + 1;
    a.kt = g.K ? (g.K - 1) / kt + 1 : 0;
    const int64_t tiles = g.batches * a.mt * a.nt, steps = g.red * a.kt;
    if (tiles < 256 && steps >= 8) {
        const int64_t by_tiles = (512 + tiles - 1) / tiles, by_steps = steps / 4;
        a.splits = (int32_t)(by_tiles < by_steps ? by_tiles : by_steps);
    }
    return a;
}

template <typename T>
hipError_t launch_typed(const GemmArgs& a, hipStream_t s)
{
    const Gemm& g = a.g;
    if (a.path == PATH_ROWS) return launch_rows(a, s);
    const unsigned grid = (unsigned)(g.batches * a.splits * a.mt * a.nt);
    hipError_t e = hipSuccess;
    if (a.path == PATH_LARGE) e = launch_large(a, s);
    else if (g.gated) k_gemm<T, true, true, true><<<grid, 256, 0, s>>>(a);
    else if (g.a_kmajor && g.b_kmajor) k_gemm<T, true, true, false><<<grid, 256, 0, s>>>(a);
    else if (g.a_kmajor) k_gemm<T, true, false, false><<<grid, 256, 0, s>>>(a);
    else k_gemm<T, false, false, false><<<grid, 256, 0, s>>>(a);
    if (e == hipSuccess) e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const unsigned join = (unsigned)((g.batches * g.M * g.N + 255) / 256);
    if (g.gated) k_gemm_join<T, true><<<join, 256, 0, s>>>(a);
    else k_gemm_join<T, false><<<join, 256, 0, s>>>(a);
    return hipGetLastError();
}

// ---- dz and its column sums -----------------------------------------------
constexpr int Z_ROWS = 64;  // rows of a chunk

template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_gradz(GradZ g, int32_t colblocks, int64_t chunks)
{
    __shared__ float red[GATED ? 2 : 1][4][64];
    constexpr bool FAST = sizeof(T) == 2;
    const int64_t wide = GATED ? 2 * (int64_t)g.out : g.out;
    int64_t id = blockIdx.x;
    const int32_t cb = (int32_t)(id % colblocks);
    id /= colblocks;
    const int64_t chunk = id % chunks, n = id / chunks;
    const int32_t col = cb * 64 + threadIdx.x % 64;
    const int part = threadIdx.x / 64;
    float s0 = 0.f, s1 = 0.f;
    if (col < g.out) {
        for (int i = part; i < Z_ROWS; i += 4) {
            const int64_t row = chunk * Z_ROWS + i;
            if (row >= g.rows) break;
            const float d = widen(static_cast<const T*>(g.dy)[n * g.dy_member + row * g.dy_row + col]);
            const T* pre = static_cast<const T*>(g.pre) + n * g.pre_member + row * g.pre_row;
            T* dz = static_cast<T*>(g.dz) + (n * g.rows + row) * g.ldz;
            if constexpr (GATED) {
                const float z = widen(pre[col]), u = widen(pre[g.out + col]);
                const float dg = d * u * act_slope<FAST>(z, g.act), du = d * act_value<FAST>(z, g.act);
                s0 += dg;
                s1 += du;
                if (g.dz) {
                    dz[col] = (T)dg;
                    dz[g.out + col] = (T)du;
                }
            } else {
                const float dd = g.act == ES_ACT_NONE ? d : d * act_slope<FAST>(widen(pre[col]), g.act);
                s0 += dd;
                if (g.dz) dz[col] = (T)dd;
            }
        }
    }
    if (!g.sums) return;
    red[0][part][threadIdx.x % 64] = s0;
    if constexpr (GATED) red[GATED][part][threadIdx.x % 64] = s1;
    __syncthreads();
    if (part == 0 && col < g.out) {
        float* out = g.sums + (n * chunks + chunk) * wide;
        const int c = threadIdx.x % 64;
        out[col] = (red[0][0][c] + red[0][1][c]) + (red[0][2][c] + red[0][3][c]);
        if constexpr (GATED)
            out[g.out + col] = (red[GATED][0][c] + red[GATED][1][c]) + (red[GATED][2][c] + red[GATED][3][c]);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_bias_grad(const float* sums, int64_t members, int64_t chunks, int64_t wide, T* db,
                                                   int64_t db_member, int64_t groups)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= groups * wide) return;
    const int64_t n = id / wide, o = id % wide, count = chunks * members / groups;
    double s = 0.0;
    for (int64_t c = 0; c < count; ++c) s += (double)sums[(n * count + c) * wide + o];
    db[n * db_member + o] = (T)(float)s;
}

}  // namespace

size_t gemm_workspace_floats(const Gemm& g)
{
    const GemmArgs a = plan(g);
    return a.path != PATH_ROWS && a.splits > 1 ? (size_t)a.splits * g.batches * g.M * (g.gated ? 2 : 1) * (size_t)g.N : 0;
}

bool gemm_too_large(const Gemm& g)
{
    const GemmArgs a = plan(g);
    const __int128 most = 0x7FFFFFFF;
    if (a.path == PATH_ROWS) return (__int128)g.batches * a.nt > most;
    return (__int128)g.batches * a.splits * a.mt * a.nt > most ||
           (a.splits > 1 && (__int128)g.batches * g.M * g.N / 256 >= most);
}

hipError_t launch_gemm(const Gemm& g, float* partial, hipStream_t s)
{
    GemmArgs a = plan(g);
    a.partial = partial;
    switch (g.dtype) {
    case ES_BF16: return launch_typed<__bf16>(a, s);
    case ES_F16: return launch_typed<_Float16>(a, s);
    default: return launch_typed<float>(a, s);
    }
}

int64_t gradz_chunks(int64_t rows) { return (rows + Z_ROWS - 1) / Z_ROWS; }

hipError_t launch_gradz(const GradZ& g, hipStream_t s)
{
    const int64_t chunks = gradz_chunks(g.rows);
    const int32_t colblocks = (g.out + 63) / 64;
    const int64_t grid = g.members * chunks * colblocks;
    if (grid == 0) return hipSuccess;
    auto go = [&](auto kernel) { kernel<<<(unsigned)grid, 256, 0, s>>>(g, colblocks, chunks); };
    switch (g.dtype) {
    case ES_BF16: g.gated ? go(k_gradz<__bf16, true>) : go(k_gradz<__bf16, false>); break;
    case ES_F16: g.gated ? go(k_gradz<_Float16, true>) : go(k_gradz<_Float16, false>); break;
    default: g.gated ? go(k_gradz<float, true>) : go(k_gradz<float, false>);
    }
    return hipGetLastError();
}

hipError_t launch_bias_grad(int32_t dtype, const float* sums, int64_t members, int64_t chunks, int64_t wide, void* db,
                            int64_t db_member, hipStream_t s)
{
    const int64_t groups = members != 1 && db_member == 0 ? 1 : members;
    const unsigned grid = (unsigned)((groups * wide + 255) / 256);
    switch (dtype) {
    case ES_BF16:
        k_bias_grad<<<grid, 256, 0, s>>>(sums, members, chunks, wide, static_cast<__bf16*>(db), db_member, groups);
        break;
    case ES_F16:
        k_bias_grad<<<grid, 256, 0, s>>>(sums, members, chunks, wide, static_cast<_Float16*>(db), db_member, groups);
        break;
    default: k_bias_grad<<<grid, 256, 0, s>>>(sums, members, chunks, wide, static_cast<float*>(db), db_member, groups);
    }
    return hipGetLastError();
}

}  // namespace esmi
