// es_dense_rows.hip -- forward products of few rows (a token, a policy's
// observation), gfx950: bound by one reading of the weights.
//
// A wave owns 16 outputs: it reads 64 bytes of k of their 16 rows of w at a time,
// 16 bytes a lane, straight from memory into the operand registers of the
// matrix instruction (lane = row + 16 * piece is their layout), and the same
// piece of up to 16 rows of x, which stay in the caches.  12 to 18 pieces
// are in flight at once.  Long rows are shared by up to 16 waves of a workgroup, whose
// sums are added in their order through LDS.  Rows behind the last output or
// the last row of x are read as that last one; what they give is not stored.
// One row of 4096 -> 4096 bf16 7.9 us, 4.3 TB/s; four of 4096 -> 2 x 11264 35.0 us, 5.3
// TB/s; 256 members' row of 64 -> 256 fp32 6.5 us.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "es_dense.hpp"
#include "es_dense_device.hpp"

namespace esmi {

namespace {

constexpr int MOST_WAVES = 16;

// 16 bytes at p, or what is left of the row there
template <typename T>
__device__ __forceinline__ uintx4 piece(const T* row, int32_t k, int32_t K)
{
    constexpr int E = 16 / sizeof(T);
    uintx4 v = {0, 0, 0, 0};
    const uint32_t at = (uint32_t)k, end = (uint32_t)K;  // at + E may pass 2^31
    if (at + E <= end) {
        __builtin_memcpy(&v, row + at, 16);
    } else if (at < end) {
        T t[E];
#pragma unroll
        for (int i = 0; i < E; ++i) t[i] = at + i < end ? row[at + i] : (T)0.f;
        __builtin_memcpy(&v, t, 16);
    }
    return v;
}

template <typename T, bool ODD>
__device__ __forceinline__ uintx4 whole(const T* p)
{
    if constexpr (ODD) return load16_odd(p);
    uintx4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

// ODD: 16-bit rows of w or x at odd multiples of 2 bytes
template <typename T, bool GATED, int MT, bool ODD>
__global__ __launch_bounds__(64 * MOST_WAVES) void k_rows(GemmArgs a)
{
    __shared__ floatx4 red[MOST_WAVES][GATED ? 2 : 1][MT][64];
    const Gemm& g = a.g;
    constexpr int E = 16 / sizeof(T), CHUNK = 4 * E, U = MT == 2 ? 4 : GATED ? 6 : 8, NW = GATED ? 2 : 1;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), q = lane / 16, l16 = lane % 16;
    const int per_tile = a.splits, tiles = (int)(blockDim.x / 64) / per_tile;  // waves a tile, tiles a workgroup
    const uint32_t groups = a.nt;
    const int64_t batch = blockIdx.x / groups;
    const int32_t n0 = ((int32_t)(blockIdx.x % groups) * tiles + wave / per_tile) * 16;
    const int part = wave % per_tile;

    const T *w[NW], *x[MT];
    const int32_t n = n0 + l16 < g.N ? n0 + l16 : g.N - 1;
#pragma unroll
    for (int h = 0; h < NW; ++h)
        w[h] = static_cast<const T*>(g.b) + batch * g.b_batch + (n + (int64_t)h * g.N) * g.b_row;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int32_t m = 16 * i + l16 < g.M ? 16 * i + l16 : g.M - 1;
        x[i] = static_cast<const T*>(g.a) + batch * g.a_batch + m * g.a_row;
    }
    floatx4 acc[NW][MT];
#pragma unroll
    for (int h = 0; h < NW; ++h)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[h][i] = floatx4{0.f, 0.f, 0.f, 0.f};

    // what the epilogue adds is under way meanwhile
    const int64_t o = n0 + 4 * q;
    float bz[4], bu[4], r[MT][4];
    if (part == 0) {
        load_bias<T, GATED, 4>(g, batch, o, bz, bu);
#pragma unroll
        for (int i = 0; i < MT; ++i) load_res<T, 4>(a, batch, 16 * i + l16 < g.M ? 16 * i + l16 : g.M - 1, o, r[i]);
    }

    const int32_t per = (int32_t)a.per, c0 = part * per, c1 = a.kt - c0 < per ? a.kt : c0 + per, full = g.K / CHUNK < c1 ? g.K / CHUNK : c1;
    int32_t c = c0;
    int64_t at = (int64_t)c0 * CHUNK + E * q;
    auto batch_of = [&](auto count) {
        constexpr int N = decltype(count)::value;
        uintx4 fw[NW][N], fx[MT][N];
#pragma unroll
        for (int h = 0; h < NW; ++h)
#pragma unroll
            for (int u = 0; u < N; ++u) fw[h][u] = whole<T, ODD>(w[h] + at + u * CHUNK);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int u = 0; u < N; ++u) fx[i][u] = whole<T, ODD>(x[i] + at + u * CHUNK);
        // all of them in flight before the first is used
        __builtin_amdgcn_sched_barrier(0);
        at += N * CHUNK;
        c += N;
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
            for (int h = 0; h < NW; ++h)
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[h][i] = product<T>(fw[h][u], fx[i][u], acc[h][i]);
    };
    if (n0 < g.N) {
        while (c + U <= full) batch_of(std::integral_constant<int, U>{});
        if (U > 4 && c + 4 <= full) batch_of(std::integral_constant<int, 4>{});
        if (c + 2 <= full) batch_of(std::integral_constant<int, 2>{});
        for (; c < c1; ++c) {
            const int32_t k = c * CHUNK + E * q;
            uintx4 fx[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) fx[i] = piece(x[i], k, g.K);
#pragma unroll
            for (int h = 0; h < NW; ++h) {
                const uintx4 fw = piece(w[h], k, g.K);
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[h][i] = product<T>(fw, fx[i], acc[h][i]);
            }
        }
    }
    if (per_tile > 1) {
#pragma unroll
        for (int h = 0; h < NW; ++h)
#pragma unroll
            for (int i = 0; i < MT; ++i) red[wave][h][i][lane] = acc[h][i];
        __syncthreads();
        if (part) return;
        for (int p = 1; p < per_tile; ++p)
#pragma unroll
            for (int h = 0; h < NW; ++h)
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[h][i] += red[wave + p][h][i][lane];
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        if (16 * i + l16 >= g.M) continue;
        float z[4], u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            z[e] = acc[0][i][e];
            u[e] = GATED ? acc[NW - 1][i][e] : 0.f;
        }
        finish<T, GATED, 4>(a, batch, 16 * i + l16, o, z, u, bz, bu, r[i]);
    }
}

template <typename T, bool GATED, bool ODD>
hipError_t launch_rows_of(const GemmArgs& a, unsigned grid, unsigned threads, hipStream_t s)
{
    return launch(a.g.M <= 16 ? k_rows<T, GATED, 1, ODD> : k_rows<T, GATED, 2, ODD>, grid, threads, 0, s, a);
}

template <typename T>
hipError_t launch_typed(const GemmArgs& a, hipStream_t s)
{
    const unsigned grid = (unsigned)(a.g.batches * a.nt), threads = 64u * a.mt;
    if constexpr (sizeof(T) == 2) {
        if (a.odd_a || a.odd_b) {
            return a.g.gated ? launch_rows_of<T, true, true>(a, grid, threads, s) : launch_rows_of<T, false, true>(a, grid, threads, s);
        }
    }
    return a.g.gated ? launch_rows_of<T, true, false>(a, grid, threads, s) : launch_rows_of<T, false, false>(a, grid, threads, s);
}

}  // namespace

bool rows_fits(const Gemm& g) { return g.a_kmajor && g.b_kmajor && g.red == 1 && g.M <= 32; }

// splits: waves that share a tile's rows, each at least 8 pieces of 64 bytes;
// mt: waves of a workgroup; nt: workgroups a member.
void rows_plan(GemmArgs& a)
{
    const Gemm& g = a.g;
    a.path = PATH_ROWS;
    const int32_t chunk = 64 / (int32_t)dtype_size(g.dtype);
    a.kt = g.K ? (g.K - 1) / chunk + 1 : 0;
    int32_t share = 1;
    while (share < MOST_WAVES && a.kt >= 16 * share) share *= 2;
    a.splits = share;
    a.per = (a.kt + share - 1) / share;
    a.mt = share < 4 ? 4 : share;
    const int32_t tiles = (g.N - 1) / 16 + 1, per = a.mt / share;
    a.nt = (tiles - 1) / per + 1;
}

hipError_t launch_rows(const GemmArgs& a, hipStream_t s)
{
    switch (a.g.dtype) {
    case ES_BF16: return launch_typed<__bf16>(a, s);
    case ES_F16: return launch_typed<_Float16>(a, s);
    default: return launch_typed<float>(a, s);
    }
}

}  // namespace esmi
