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
// A gated layer's columns of a wave are half gates and half the matching others.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "es_dense.hpp"
#include "es_dense_device.hpp"

namespace esmi {

namespace {

// ---- the product ----------------------------------------------------------
// Any type, size, stride and alignment.  Four waves make a TM x TN tile of C: 128
// x 128, 64 x 64 where there are few tiles, 32 x 128 for few rows (then bound by
// the reading of B).  A step is 128 bytes of k: fetched into registers while the step
// before is multiplied, then staged in LDS.  An operand with k contiguous is staged row by row and read 16
// bytes a lane; piece c of row r lies at c ^ f(r), which spreads the lanes that a
// 16-byte read serves together ({0-3, 12-15, 20-27}, {4-11, 16-19, 28-31} and
// those + 32, measured) over all banks.
// Another one is staged as it lies, a row of m (n) per k: 16-bit fragments come
// back transposed by ds_read_b64_tr_b16 (lane i of 16 gets the four k of column
// i), fp32 ones word by word.
// Bound by the fp32 matrix rate where pieces are whole (2048^3 fp32 140 us, 123 TFLOP/s),
// by its loads and their staging where not (96 x (250 x 253) (253 x 131) fp32 35 us, 46
// TFLOP/s; 16-bit 250 TFLOP/s).
template <typename T, bool KMAJOR, int TS>
struct Staged {
    static constexpr int E = 16 / sizeof(T), KT = 128 / sizeof(T), LOADS = TS * 8 / 256;  // per lane
    // fp32: rows 4 apart lie 16 banks apart
    static constexpr int ROW = KMAJOR ? 128 : TS * (int)sizeof(T) + (sizeof(T) == 4 ? 16 : 32);
    static constexpr int BYTES = (KMAJOR ? TS : KT) * ROW;
    const T* p[LOADS];
    int32_t left[LOADS];  // not k-major: valid columns from p
    uintx4 v[LOADS];

    static __device__ __forceinline__ int f(int row)
    {
        const int a = (row >> 2) & 3;
        return (2 * a + ((row >> 1) & 1)) ^ ((a ^ (a >> 1)) & 1);
    }

    // row_of(i): the matrix's row of staged row i (inside), or, not k-major, its first column and how many are left
    template <typename F>
    __device__ __forceinline__ void init(const T* base, int64_t stride, F row_of)
    {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int c = (int)threadIdx.x + 256 * j;
            int32_t n;
            if constexpr (KMAJOR) {
                p[j] = base + row_of(c / 8, n) * stride + (c % 8) * E;
            } else {
                constexpr int PER = TS / E;
                const int64_t col = row_of((c % PER) * E, n);
                left[j] = n;
                p[j] = base + (int64_t)(c / PER) * stride + col;
            }
        }
    }
    // the step whose first k has `k_left` behind it, `at` elements from the first
    __device__ __forceinline__ void fetch(int64_t at, int32_t k_left, bool odd)
    {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int c = (int)threadIdx.x + 256 * j;
            int n;  // elements to read
            if constexpr (KMAJOR) n = k_left - (c % 8) * E;
            else n = c / (TS / E) < k_left ? left[j] : 0;
            if (n >= E) {
                if (sizeof(T) == 2 && odd) v[j] = load16_odd(p[j] + at);
                else __builtin_memcpy(&v[j], p[j] + at, 16);
            } else {
                T t[E];
#pragma unroll
                for (int i = 0; i < E; ++i) t[i] = i < n ? p[j][at + i] : (T)0.f;
                __builtin_memcpy(&v[j], t, 16);
            }
        }
    }
    __device__ __forceinline__ void store(unsigned char* lds) const
    {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int c = (int)threadIdx.x + 256 * j;
            const int at = KMAJOR ? (c / 8) * ROW + ((c % 8) ^ f(c / 8)) * 16 : (c / (TS / E)) * ROW + (c % (TS / E)) * 16;
            *reinterpret_cast<uintx4*>(lds + at) = v[j];
        }
    }
    // fragment `ks` (64 bytes of k) of staged rows (columns) base + l16
    static __device__ __forceinline__ uintx4 read(const unsigned char* lds, int base, int ks, int lane)
    {
        const int l16 = lane % 16, q = lane / 16;
        if constexpr (KMAJOR) {
            return *reinterpret_cast<const uintx4*>(lds + (base + l16) * ROW + ((4 * ks + q) ^ f(base + l16)) * 16);
        } else if constexpr (sizeof(T) == 4) {
            uintx4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = *reinterpret_cast<const uint32_t*>(lds + (16 * ks + 4 * q + i) * ROW + (base + l16) * 4);
            return v;
        } else {
            typedef short shortx4 __attribute__((ext_vector_type(4)));
            shortx4 t[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const unsigned char* at = lds + (32 * ks + 8 * q + 4 * h + (l16 >> 2)) * ROW + (base + 4 * (l16 & 3)) * 2;
                t[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)at);
            }
            uintx4 v;
            __builtin_memcpy(&v, t, 16);
            return v;
        }
    }
};

template <typename T, bool AK, bool BK, bool GATED, int TM, int TN>
__global__ __launch_bounds__(256) void k_gemm(GemmArgs a)
{
    using SA = Staged<T, AK, TM>;
    using SB = Staged<T, BK, TN>;
    constexpr int KT = 128 / sizeof(T), WAVES_M = TM >= 64 ? 2 : 1, WAVES_N = 4 / WAVES_M;
    constexpr int WM = TM / WAVES_M, WN = TN / WAVES_N, MB = WM / 16, NB = WN / 16;  // a wave's rows, columns, 16 x 16 tiles
    constexpr int OUTS = GATED ? TN / 2 : TN, STAGED = SA::BYTES + SB::BYTES, FINAL = 4 * EPILOGUE_LDS<NB>;
    __shared__ __align__(16) unsigned char lds[STAGED > FINAL ? STAGED : FINAL];
    unsigned char *sa = lds, *sb = lds + SA::BYTES;
    const Gemm& g = a.g;
    uint32_t id = blockIdx.x;
    const int32_t tn = id % a.nt;
    id /= a.nt;
    const int32_t tm = id % a.mt;
    id /= a.mt;
    const int64_t split = id % (uint32_t)a.splits, batch = id / (uint32_t)a.splits;
    const int32_t m0 = tm * TM, n0 = tn * OUTS;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const int wm = wave / WAVES_N, wn = wave % WAVES_N;
    const int64_t steps = g.red * a.kt, first = split * a.per, last = steps - first < a.per ? steps : first + a.per;
    int64_t r = a.splits > 1 ? first / a.kt : 0;
    int32_t kt = (int32_t)(first - r * a.kt);
    SA va;
    SB vb;
    // rows behind the last are read as the last: what they give is not stored
    va.init(static_cast<const T*>(g.a) + batch * g.a_batch + r * g.a_red, g.a_row, [&](int i, int32_t& n) -> int64_t {
        n = g.M - m0 - i;
        return AK && n <= 0 ? g.M - 1 : m0 + i;
    });
    vb.init(static_cast<const T*>(g.b) + batch * g.b_batch + r * g.b_red, g.b_row, [&](int i, int32_t& n) -> int64_t {
        if constexpr (GATED) {
            // a wave's rows: the gates, then the others
            const int32_t o = n0 + WN / 2 * (i / WN) + i % (WN / 2);
            return (o < g.N ? o : g.N - 1) + (i / (WN / 2) % 2 ? (int64_t)g.N : 0);
        } else {
            n = g.N - n0 - i;
            return BK && n <= 0 ? g.N - 1 : n0 + i;
        }
    });

    floatx4 acc[MB][NB];  // [m tile][n tile]
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    int64_t ra = 0, rb = 0;  // the reduction batch's offsets from r's
    auto fetch = [&]() {
        const int32_t k0 = kt * KT;
        va.fetch(ra + (AK ? (int64_t)k0 : k0 * g.a_row), g.K - k0, a.odd_a);
        vb.fetch(rb + (BK ? (int64_t)k0 : k0 * g.b_row), g.K - k0, a.odd_b);
        if (++kt == a.kt) {
            kt = 0;
            ra += g.a_red;
            rb += g.b_red;
        }
    };
    if (first < last) fetch();
    for (int64_t t = first; t < last; ++t) {
        __syncthreads();
        va.store(sa);
        vb.store(sb);
        __syncthreads();
        if (t + 1 < last) fetch();
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            uintx4 fa[MB], fb[NB];
#pragma unroll
            for (int i = 0; i < MB; ++i) fa[i] = SA::read(sa, WM * wm + 16 * i, ks, lane);
#pragma unroll
            for (int j = 0; j < NB; ++j) fb[j] = SB::read(sb, WN * wn + 16 * j, ks, lane);
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = product<T>(fb[j], fa[i], acc[i][j]);
        }
    }

    __syncthreads();  // the staged steps make room for the epilogue
    epilogue<T, GATED, MB, NB, TM == 128>(a, (int32_t)split, batch, m0 + WM * wm, n0 + (GATED ? WN / 2 : WN) * wn, acc,
                               reinterpret_cast<float*>(lds + wave * EPILOGUE_LDS<NB>), lane);
}

// Sums of the splits and the epilogue, four outputs a thread.  Few outputs leave
// the chip idle: `slices` threads then share one's splits, each in its order.
// Bound by memory, or its latency: 11.3 MB of sums of 250 x 131 outputs (86 splits) 6.6 us.
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_gemm_join(GemmArgs a, int64_t total, uint32_t quads, int32_t slices)
{
    __shared__ floatx4 red[GATED ? 2 : 1][256];
    const Gemm& g = a.g;
    const int per = 256 / slices, slice = (int)threadIdx.x / per;
    const int64_t id = (int64_t)blockIdx.x * per + threadIdx.x % per;  // [batch][m][quad of outputs]
    const bool inside = id < total;
    const int64_t row = !inside ? 0 : total <= 0xFFFFFFFFll ? (uint32_t)id / quads : id / quads;
    const int64_t batch = total <= 0xFFFFFFFFll ? (uint32_t)row / (uint32_t)g.M : row / g.M;
    const int32_t o = inside ? (int32_t)((id - row * quads) * 4) : 0, left = g.N - o;
    const int64_t m = row - batch * g.M, wide = GATED ? 2 * (int64_t)g.N : g.N;
    float z[4] = {}, u[4] = {}, bz[4], bu[4], r[4];
    if (slice == 0) {
        load_bias<T, GATED, 4>(g, batch, o, bz, bu);
        load_res<T, 4>(a, batch, m, o, r);
    }
    const int64_t pitch = g.batches * g.M * wide;
    const float* p = a.partial + row * wide + o + slice * pitch;
#pragma unroll 4
    for (int32_t s = slice; s < a.splits; s += slices, p += slices * pitch) {
        float v[4];
        load_run<float, 4>(p, left, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] += v[i];
        if constexpr (GATED) {
            load_run<float, 4>(p + g.N, left, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] += v[i];
        }
    }
    if (slices > 1) {
        red[0][threadIdx.x] = floatx4{z[0], z[1], z[2], z[3]};
        if constexpr (GATED) red[GATED][threadIdx.x] = floatx4{u[0], u[1], u[2], u[3]};
        __syncthreads();
        if (slice) return;
        for (int s = 1; s < slices; ++s) {
            const floatx4 v = red[0][threadIdx.x + s * per];
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] += v[i];
            if constexpr (GATED) {
                const floatx4 w = red[GATED][threadIdx.x + s * per];
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] += w[i];
            }
        }
    }
    if (inside) finish<T, GATED, 4>(a, batch, m, o, z, u, bz, bu, r);
}

// ---- copies in whole pieces ------------------------------------------------
// One operand as [n][rows][ld], ld a multiple of 8 elements, zeros behind its
// columns.  Bound by memory: 8192 x 4095 with 4095 x 4095 bf16 50 us, 4 TB/s.
struct PackArgs {
    const uint16_t* src;
    uint16_t* dst;
    int64_t n, rows, cols, ld, batch, row, total;  // total: pieces
};

__global__ __launch_bounds__(256) void k_pack(PackArgs a)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, per = a.ld / 8;
    if (id >= a.total) return;
    const int64_t r = a.total <= 0xFFFFFFFFll ? (uint32_t)id / (uint32_t)per : id / per;  // n * rows + row
    const int64_t n = a.total <= 0xFFFFFFFFll ? (uint32_t)r / (uint32_t)a.rows : r / a.rows;
    const int64_t c = (id - r * per) * 8, left = a.cols - c;
    const uint16_t* p = a.src + n * a.batch + (r - n * a.rows) * a.row + c;
    uintx4 v;
    if (left >= 8) {
        v = load16_odd(p);
    } else {
        uint16_t t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = i < left ? p[i] : (uint16_t)0;
        __builtin_memcpy(&v, t, 16);
    }
    *reinterpret_cast<uintx4*>(a.dst + id * 8) = v;
}

struct Packing {
    bool a, b;
    size_t a_bytes, b_bytes;
};

int64_t pack_rows(const Gemm& g, bool is_a) { return (is_a ? g.a_kmajor : g.b_kmajor) ? (is_a ? g.M : (g.gated ? 2 : 1) * (int64_t)g.N) : g.K; }
int64_t pack_cols(const Gemm& g, bool is_a) { return (is_a ? g.a_kmajor : g.b_kmajor) ? g.K : is_a ? g.M : g.N; }

// The product on copies: sets the operand's place (base: where the copy will be)
// and the bytes that it takes.
size_t pack_operand(Gemm& g, bool is_a, void* base)
{
    const int64_t rows = pack_rows(g, is_a), ld = (pack_cols(g, is_a) + 7) / 8 * 8;
    // an operand that all batches (or all terms of the reduction) share is copied once
    const int64_t batch = is_a ? g.a_batch : g.b_batch, red = is_a ? g.a_red : g.b_red;
    const int64_t n = g.batches > 1 ? (batch ? g.batches : 1) : g.red > 1 && red ? g.red : 1;
    (is_a ? g.a : g.b) = base;
    (is_a ? g.a_row : g.b_row) = ld;
    (is_a ? g.a_batch : g.b_batch) = g.batches > 1 && batch ? rows * ld : 0;
    (is_a ? g.a_red : g.b_red) = g.batches <= 1 && g.red > 1 && red ? rows * ld : 0;
    (is_a ? g.a_padded : g.b_padded) = true;
    return workspace_up((size_t)n * rows * ld * 2);
}

// Whether operands are copied for the large tiles: those that they do not take as
// they lie (both where the k of a row ends within a piece), if the staged kernel's
// further time is more than the copies' (at 250 TFLOP/s against 1100: 512 x 4095 x
// 4095 125 us staged, 37 from copies made in 20; 8192 x 4095 x 4095 404, 218 and 50;
// 256 members of 255 x 257 x 255 66, 30 and 40: left as it is).
Packing packing(const Gemm& g)
{
    Packing p{};
    if (g.dtype == ES_F32 || g.K == 0 || g.red == 0 || g.batches == 0) return p;
    const bool whole_k = g.K % 8 == 0;
    p.a = !large_takes(g, true) || (g.a_kmajor && !whole_k && !g.a_padded);
    p.b = !large_takes(g, false) || (g.b_kmajor && !whole_k && !g.b_padded);
    if (!p.a && !p.b) return p;
    Gemm h = g;
    // any aligned address serves for the look
    if (p.a) p.a_bytes = pack_operand(h, true, reinterpret_cast<void*>(WORKSPACE_ALIGN));
    if (p.b) p.b_bytes = pack_operand(h, false, reinterpret_cast<void*>(WORKSPACE_ALIGN));
    // (a copy of as many pieces as no launch holds is beyond any memory)
    if (p.a_bytes / 16 + 256 > launch_groups(1) || p.b_bytes / 16 + 256 > launch_groups(1)) return Packing{};
    const double flops = 2.0 * g.batches * g.red * g.M * (g.gated ? 2.0 : 1.0) * g.N * g.K;
    const double gain = flops * (1 / 250e12 - 1 / 1100e12), cost = 2.0 * (p.a_bytes + p.b_bytes) / 4e12 + 4e-6 * (p.a + p.b);
    if (gain <= cost || !large_fits(h)) return Packing{};
    return p;
}

hipError_t launch_pack(const Gemm& from, const Gemm& to, bool is_a, hipStream_t s)
{
    PackArgs a{};
    a.src = static_cast<const uint16_t*>(is_a ? from.a : from.b);
    a.dst = static_cast<uint16_t*>(const_cast<void*>(is_a ? to.a : to.b));
    a.rows = pack_rows(from, is_a);
    a.cols = pack_cols(from, is_a);
    a.ld = is_a ? to.a_row : to.b_row;
    const int64_t batch = is_a ? from.a_batch : from.b_batch, red = is_a ? from.a_red : from.b_red;
    a.n = from.batches > 1 ? (batch ? from.batches : 1) : from.red > 1 && red ? from.red : 1;
    a.batch = from.batches > 1 ? batch : red;
    a.row = is_a ? from.a_row : from.b_row;
    a.total = a.n * a.rows * (a.ld / 8);
    return launch(k_pack, (unsigned)((a.total + 255) / 256), 256, 0, s, a);
}

bool odd(const Gemm& g, const void* p, int64_t row, int64_t batch, int64_t red)
{
    return g.dtype != ES_F32 && (reinterpret_cast<uintptr_t>(p) % 4 || row % 2 || (g.batches > 1 && batch % 2) || (g.red > 1 && red % 2));
}

// Kernel, tiles and splits of a.g
void plan_path(GemmArgs& a)
{
    const Gemm& g = a.g;
    a.odd_a = odd(g, g.a, g.a_row, g.a_batch, g.a_red);
    a.odd_b = odd(g, g.b, g.b_row, g.b_batch, g.b_red);
    if (rows_fits(g)) return rows_plan(a);
    if (large_fits(g)) return large_plan(a);
    const int32_t kt = 128 / (int32_t)dtype_size(g.dtype);
    a.path = PATH_STAGED;
    a.kt = g.K ? (g.K - 1) / kt + 1 : 0;
    a.tile = g.M <= 32 && !(g.a_kmajor && g.b_kmajor) ? 32 : 128;
    for (;;) {
        const int32_t tn = a.tile == 64 ? 64 : 128;
        a.mt = (g.M - 1) / a.tile + 1;
        a.nt = (g.N - 1) / (g.gated ? tn / 2 : tn) + 1;
        // small tiles where large ones would leave CUs without work
        if (a.tile != 128 || g.batches * a.mt * a.nt >= 512) break;
        a.tile = 64;
    }
    const int64_t tiles = g.batches * a.mt * a.nt, steps = g.red * a.kt;
    int64_t splits = 1;
    if (tiles < 512 && steps >= 8) splits = std::min((1024 + tiles - 1) / tiles, steps / 4);
    a.per = steps ? (steps + splits - 1) / splits : 0;
    a.splits = steps ? (int32_t)((steps + a.per - 1) / a.per) : 1;
}

GemmArgs plan(const Gemm& from, void* workspace, size_t* bytes)
{
    GemmArgs a{};
    Gemm g = from;
    const Packing pk = packing(g);
    char* at = static_cast<char*>(workspace);
    if (pk.a) pack_operand(g, true, at);
    if (pk.b) pack_operand(g, false, at + pk.a_bytes);
    a.g = g;
    a.partial = reinterpret_cast<float*>(at + pk.a_bytes + pk.b_bytes);
    a.splits = 1;
    plan_path(a);
    *bytes = pk.a_bytes + pk.b_bytes;
    if (a.path != PATH_ROWS && a.splits > 1)
        *bytes += workspace_up((size_t)4 * a.splits * g.batches * g.M * (g.gated ? 2 : 1) * (size_t)g.N);
    *bytes += workspace_up((size_t)4 * 256 * 256 * a.tail * a.tail_splits);
    return a;
}

template <typename T, int TM, int TN>
hipError_t launch_staged(const GemmArgs& a, unsigned grid, hipStream_t s)
{
    const Gemm& g = a.g;
    void (*kernel)(GemmArgs) = nullptr;
    if (g.a_kmajor && g.b_kmajor) {
        if constexpr (TM >= 64)  // fewer rows have kernels of their own (es_dense_rows.hip)
            kernel = g.gated ? k_gemm<T, true, true, true, TM, TN> : k_gemm<T, true, true, false, TM, TN>;
    } else {
        kernel = g.a_kmajor ? k_gemm<T, true, false, false, TM, TN> : k_gemm<T, false, false, false, TM, TN>;
    }
    return kernel ? launch(kernel, grid, 256, 0, s, a) : hipErrorInvalidValue;
}

uint32_t join_quads(const Gemm& g) { return (uint32_t)(((int64_t)g.N + 3) / 4); }

template <typename T>
hipError_t launch_typed(const GemmArgs& a, hipStream_t s)
{
    const Gemm& g = a.g;
    if (a.path == PATH_ROWS) return launch_rows(a, s);
    const unsigned grid = (unsigned)(g.batches * a.splits * a.mt * a.nt);
    hipError_t e = hipSuccess;
    if (a.path == PATH_LARGE) e = launch_large(a, s);
    else if (a.tile == 128) e = launch_staged<T, 128, 128>(a, grid, s);
    else if (a.tile == 64) e = launch_staged<T, 64, 64>(a, grid, s);
    else e = launch_staged<T, 32, 128>(a, grid, s);
    if (e != hipSuccess || a.splits == 1) return e;
    const uint32_t quads = join_quads(g);
    const int64_t total = g.batches * g.M * quads;
    int32_t slices = 1;
    while (slices < 16 && slices * 4 <= a.splits && total * slices < 131072) slices *= 2;
    const unsigned join = (unsigned)((total * slices + 255) / 256);
    return launch(g.gated ? k_gemm_join<T, true> : k_gemm_join<T, false>, join, 256, 0, s, a, total, quads, slices);
}

int64_t threads_of(const GemmArgs& a)
{
    return a.path == PATH_ROWS ? 64 * a.mt : a.path == PATH_LARGE ? large_threads(a) : 256;
}

int64_t groups_per_batch(const GemmArgs& a)
{
    if (a.path == PATH_ROWS) return a.nt;
    return (int64_t)a.splits * a.mt * a.nt + (a.tail ? (int64_t)a.tail * (a.tail_splits - 1) : 0);
}

// The product of the batches from b on
Gemm from_batch(Gemm g, int64_t b)
{
    const int64_t e = (int64_t)dtype_size(g.dtype);
    auto in = [&](const void* p, int64_t stride) -> const void* { return p ? static_cast<const char*>(p) + b * stride * e : p; };
    g.a = in(g.a, g.a_batch);
    g.b = in(g.b, g.b_batch);
    g.bias = in(g.bias, g.bias_batch);
    g.res = in(g.res, g.res_batch);
    g.pre = const_cast<void*>(in(g.pre, g.pre_batch));
    g.c = static_cast<char*>(g.c) + b * g.c_batch * (int64_t)dtype_size(g.c_dtype);
    return g;
}

// ---- dz and its column sums -----------------------------------------------
// Bound by memory: dy and pre in, dz out.  A thread takes 16 bytes of a row and
// every 2^(8 - lx)-th row of the chunk's 64, 2^lx threads side by side.  8192 x
// 4096 bf16 44 us, 4.6 TB/s; 2048 x 2 x 5632 fp16 of a gated layer 21 us, 5.4.
//
// dz is formed in fp32 and rounded to the type once, because the matrix cores take
// both operands of a product in it: the gradients dx and dw are 1.4 times as far
// from the 64-bit ones as without (bf16 2.3e-3 against 1.65e-3 of their size, fp16
// 2.9e-4 against 2.1e-4).  Two 16-bit terms of dz would undo it for twice the
// products (8192 x 4096 -> 4096 bf16: dx 238 -> 383 us, dw 201 -> 377).  The sums
// of db take the unrounded values.
constexpr int Z_ROWS = 64;

struct GradZArgs {
    GradZ g;
    int64_t chunks;
    uint32_t colblocks;
    int32_t lx;
};

template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_gradz(GradZArgs a)
{
    constexpr int W = 16 / sizeof(T), NH = GATED ? 2 : 1;
    constexpr bool FAST = sizeof(T) == 2;
    __shared__ float red[NH][256 * W];
    const GradZ& g = a.g;
    const uint32_t cb = blockIdx.x % a.colblocks;
    const int64_t outer = blockIdx.x / a.colblocks, chunk = outer % a.chunks, n = outer / a.chunks;
    const int tx = threadIdx.x & ((1 << a.lx) - 1), ty = threadIdx.x >> a.lx, rows = 256 >> a.lx;
    const int64_t col = (((int64_t)cb << a.lx) + tx) * W, left = g.out - col;
    const T* dy = static_cast<const T*>(g.dy) + n * g.dy_member + col;
    const T* pre = static_cast<const T*>(g.pre) + n * g.pre_member + col;
    const int64_t row0 = chunk * Z_ROWS, end = g.rows - row0 < Z_ROWS ? g.rows - row0 : Z_ROWS;
    float sum[NH][W];
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int i = 0; i < W; ++i) sum[h][i] = 0.f;
    if (left > 0) {
        // one row at a time: the other waves hide its latency, and more rows in flight would cost waves
        for (int r = ty; r < end; r += rows) {
            const int64_t row = row0 + r;
            float d[W], z[W], u[W], slope[W];
            load_run<T, W>(dy + row * g.dy_row, left, d);
            if (GATED || g.act != ES_ACT_NONE) {
                load_run<T, W>(pre + row * g.pre_row, left, z);
                if constexpr (GATED) load_run<T, W>(pre + row * g.pre_row + g.out, left, u);
                activate<FAST, true, W>(g.act, z, slope);
            }
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if constexpr (GATED) {
                    u[i] *= d[i] * slope[i];
                    d[i] *= z[i];
                    sum[0][i] += u[i];
                    sum[NH - 1][i] += d[i];
                } else {
                    if (g.act != ES_ACT_NONE) d[i] *= slope[i];
                    sum[0][i] += d[i];
                }
            }
            if (g.dz) {
                T* dz = static_cast<T*>(g.dz) + (n * g.rows + row) * g.ldz + col;
                // zeros up to the end of the row's last piece
                if constexpr (GATED) {
                    store_run<T, W>(dz, left, u);
                    store_run<T, W>(dz + g.out, left, d);
                    if (left <= W)
                        for (int64_t i = 2 * (int64_t)g.out; i < g.ldz; ++i) dz[i - col] = (T)0.f;
                } else {
#pragma unroll
                    for (int i = 0; i < W; ++i)
                        if (i >= left) d[i] = 0.f;
                    store_run<T, W>(dz, W, d);
                }
            }
        }
    }
    if (!g.sums && !g.db) return;
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int i = 0; i < W; ++i) red[h][(ty * W + i) * (1 << a.lx) + tx] = sum[h][i];
    __syncthreads();
    // a column's rows in their order
    const int cols = W << a.lx;
    const int64_t wide = NH * (int64_t)g.out;
    for (int c = threadIdx.x; c < cols; c += 256) {
        const int64_t o = ((int64_t)cb << a.lx) * W + c;
        if (o >= g.out) break;
        const int at = (c % W) * (1 << a.lx) + c / W;
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            float s = 0.f;
            for (int r = 0; r < rows; ++r) s += red[h][r * cols + at];
            if (g.db) static_cast<T*>(g.db)[n * g.db_member + h * g.out + o] = (T)s;
            else g.sums[(n * a.chunks + chunk) * wide + h * g.out + o] = s;
        }
    }
}

// 16 columns side by side, blockDim.x / 16 slices of the chunks, each in its order.
// A latency: 128 chunks of 4096 columns 4.8 us.
template <typename T>
__global__ __launch_bounds__(1024) void k_bias_grad(const float* sums, int64_t count, int64_t wide, T* db, int64_t db_member,
                                                    uint32_t colblocks)
{
    __shared__ double red[1024];
    const int64_t n = blockIdx.x / colblocks, o = (int64_t)(blockIdx.x % colblocks) * 16 + threadIdx.x % 16;
    const int slice = threadIdx.x / 16, slices = blockDim.x / 16;
    double s = 0.0;
    if (o < wide) {
#pragma unroll 4
        for (int64_t c = slice; c < count; c += slices) s += (double)sums[(n * count + c) * wide + o];
    }
    red[threadIdx.x] = s;
    __syncthreads();
    if (slice || o >= wide) return;
    for (int i = 1; i < slices; ++i) s += red[threadIdx.x + 16 * i];
    db[n * db_member + o] = (T)(float)s;
}

}  // namespace

size_t gemm_workspace(const Gemm& g)
{
    size_t n = 0;
    plan(g, reinterpret_cast<void*>(WORKSPACE_ALIGN), &n);
    return n;
}

bool gemm_too_large(const Gemm& g)
{
    size_t n = 0;
    const GemmArgs a = plan(g, reinterpret_cast<void*>(WORKSPACE_ALIGN), &n);
    return groups_per_batch(a) > launch_groups(threads_of(a));
}

hipError_t launch_gemm(const Gemm& g, void* workspace, size_t bytes, hipStream_t s)
{
    size_t n = 0;
    const GemmArgs a = plan(g, workspace, &n);
    hipError_t e = n <= bytes ? hipSuccess : hipErrorInvalidValue;
    if (e != hipSuccess) return e;
    if (a.g.a != g.a) e = launch_pack(g, a.g, true, s);
    if (e == hipSuccess && a.g.b != g.b) e = launch_pack(g, a.g, false, s);
    // as many batches as a launch holds (a split product has few tiles: one launch)
    const int64_t most = launch_groups(threads_of(a)) / groups_per_batch(a);
    for (int64_t b = 0; e == hipSuccess && b < a.g.batches; b += most) {
        GemmArgs part = a;
        part.g = from_batch(a.g, b);
        part.g.batches = std::min(most, a.g.batches - b);
        switch (g.dtype) {
        case ES_BF16: e = launch_typed<__bf16>(part, s); break;
        case ES_F16: e = launch_typed<_Float16>(part, s); break;
        default: e = launch_typed<float>(part, s);
        }
    }
    return e;
}

int64_t gradz_chunks(int64_t rows) { return (rows + Z_ROWS - 1) / Z_ROWS; }

namespace {

// Columns of workgroups, 2^lx threads side by side
int64_t gradz_colblocks(const GradZ& g, int32_t* lx)
{
    const int64_t pieces = ((int64_t)g.out * dtype_size(g.dtype) + 15) / 16;
    *lx = 0;
    while (*lx < 5 && (int64_t)1 << *lx < pieces) ++*lx;
    return (pieces + (1 << *lx) - 1) >> *lx;
}

int64_t bias_colblocks(int64_t wide) { return (wide + 15) / 16; }

unsigned bias_threads(int64_t count)
{
    unsigned threads = 64;
    while (threads < 1024 && threads / 16 < count) threads *= 2;
    return threads;
}

}  // namespace

bool gradz_too_large(const GradZ& g)
{
    int32_t lx;
    return (__int128)gradz_chunks(g.rows) * gradz_colblocks(g, &lx) > launch_groups(256);
}

bool bias_grad_too_large(int64_t count, int64_t wide) { return bias_colblocks(wide) > launch_groups(bias_threads(count)); }

hipError_t launch_gradz(const GradZ& g, hipStream_t s)
{
    GradZArgs a{};
    a.g = g;
    a.chunks = gradz_chunks(g.rows);
    a.colblocks = (uint32_t)gradz_colblocks(g, &a.lx);
    const int64_t each = a.chunks * a.colblocks, e = (int64_t)dtype_size(g.dtype), wide = (g.gated ? 2 : 1) * (int64_t)g.out;
    if (each == 0) return hipSuccess;
    const int64_t most = launch_groups(256) / each;
    for (int64_t n = 0; n < g.members; n += most) {
        const int64_t count = std::min(most, g.members - n);
        a.g.dy = static_cast<const char*>(g.dy) + n * g.dy_member * e;
        if (g.pre) a.g.pre = static_cast<const char*>(g.pre) + n * g.pre_member * e;
        if (g.dz) a.g.dz = static_cast<char*>(g.dz) + n * g.rows * g.ldz * e;
        if (g.sums) a.g.sums = g.sums + n * a.chunks * wide;
        if (g.db) a.g.db = static_cast<char*>(g.db) + n * g.db_member * e;
        void (*kernel)(GradZArgs);
        switch (g.dtype) {
        case ES_BF16: kernel = g.gated ? k_gradz<__bf16, true> : k_gradz<__bf16, false>; break;
        case ES_F16: kernel = g.gated ? k_gradz<_Float16, true> : k_gradz<_Float16, false>; break;
        default: kernel = g.gated ? k_gradz<float, true> : k_gradz<float, false>;
        }
        const hipError_t err = launch(kernel, (unsigned)(count * each), 256, 0, s, a);
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

hipError_t launch_bias_grad(int32_t dtype, const float* sums, int64_t groups, int64_t count, int64_t wide, void* db,
                            int64_t db_member, hipStream_t s)
{
    const uint32_t colblocks = (uint32_t)bias_colblocks(wide);
    const unsigned threads = bias_threads(count);
    const int64_t most = launch_groups(threads) / colblocks;
    for (int64_t n = 0; n < groups; n += most) {
        const float* from = sums + n * count * wide;
        const unsigned grid = (unsigned)(std::min(most, groups - n) * colblocks);
        hipError_t err;
        auto go = [&](auto kernel, auto* out) {
            err = launch(kernel, grid, threads, 0, s, from, count, wide, out + n * db_member, db_member, colblocks);
        };
        switch (dtype) {
        case ES_BF16: go(k_bias_grad<__bf16>, static_cast<__bf16*>(db)); break;
        case ES_F16: go(k_bias_grad<_Float16>, static_cast<_Float16*>(db)); break;
        default: go(k_bias_grad<float>, static_cast<float*>(db));
        }
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

}  // namespace esmi
