// es_dense_large.hip -- the matrix products of 16-bit layers at sizes where the
// matrix cores bound them, gfx950.
//
// A workgroup of four waves makes a 256 x 128 tile of C, each wave 128 x 64 of
// it (8 x 4 tiles of v_mfma_f32_16x16x32, 128 accumulators a lane).  Steps of 32
// along k pass through three LDS buffers of 24 KB, filled by loads that go from
// memory to LDS without registers and are two steps ahead; one barrier a step.
// Two workgroups fit a CU (144 KB of LDS, 8 waves): where one waits at its
// barrier, starts up or is in its epilogue, the other's products go on.  A
// wave reads 12 fragments of 1 KB from LDS for 32 products of 16 cycles.
//
// The loads write LDS in lane order, so the spreading over its banks is done by
// which 16 bytes a lane fetches:
//   k-major operand (k contiguous): 64 bytes of k a row; piece c of row r lies at
//     position c ^ f(r), f(r) the two bits of r in which the four groups of
//     rows of a fragment differ (2-3, or 4-5 and 3-4 on the n side): the reads of
//     16 lanes cover all banks;
//   else: a row of m (n) per k, read back transposed by ds_read_b64_tr_b16, which
//     hands lane i of 16 the four k of column i.
// Rows, columns and k beyond the matrices are not fetched: a buffer load out of
// its range writes zeros.
#include <hip/hip_runtime.h>

#include "es_dense.hpp"
#include "es_dense_device.hpp"

namespace esmi {

namespace {

constexpr int BM = 256, BN = 128, BK = 32, STAGES = 3;
constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
constexpr uint32_t OUT = 0x80000000u;  // an offset beyond every buffer's range

typedef __attribute__((address_space(3))) void lds_void;
typedef short shortx4 __attribute__((ext_vector_type(4)));

// One operand's share of a step: EXT rows (k-major) or columns.
// SHIFT: the lower of the two row bits that spread a k-major fragment's rows.
template <bool KMAJOR, bool PERM, int EXT, int SHIFT>
struct Operand {
    static constexpr int LOADS = EXT * BK * 2 / (256 * 16);  // per lane
    static constexpr int ROW = EXT * 2;                      // bytes of a k row (not k-major)
    uint32_t off[LOADS];

    static __device__ __forceinline__ int f(int r) { return (r >> SHIFT) & 3; }

    // row_of(i): the matrix's row (k-major) or first column of the staged piece i, -1 if outside
    template <typename F>
    __device__ __forceinline__ void init(int64_t stride, F row_of)
    {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int p = (int)threadIdx.x + 256 * j;  // 16-byte piece of the stage
            if constexpr (KMAJOR) {
                const int r = p / 4, c = (p % 4) ^ f(r);
                const int64_t row = row_of(r);
                off[j] = row >= 0 ? (uint32_t)((row * stride + 8 * c) * 2) : OUT;
            } else {
                const int k = p / (ROW / 16), c = (p % (ROW / 16)) ^ spread(k);
                const int64_t col = row_of(8 * c);
                off[j] = col >= 0 ? (uint32_t)((k * stride + col) * 2) : OUT;
            }
        }
    }
    // pairs of 16-byte pieces (16 columns) of different k rows on different banks
    static __device__ __forceinline__ int spread(int k) { return 2 * ((k & 3) | ((k >> 1) & 4)); }

    // the step at k0, base: the tile's first row at k0 (k-major) or k row k0
    __device__ __forceinline__ void fetch(const void* base, int64_t stride, int32_t k_left, unsigned char* lds) const
    {
        const int64_t range = KMAJOR ? 0x7FFFFFFF : (k_left < BK ? k_left : BK) * stride * 2;
        auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)range, 0x00020000);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            uint32_t o = off[j];
            if constexpr (KMAJOR) {
                if (k_left < BK) {
                    const int p = (int)threadIdx.x + 256 * j;
                    if (8 * ((p % 4) ^ f(p / 4)) >= k_left) o = OUT;
                }
            }
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(lds + (256 * j + 64 * wave) * 16), 16, (int)o, 0, 0, 0);
        }
    }

    // the fragment of staged rows / columns base + slot(l16) (PERM: tile b of 64)
    __device__ __forceinline__ uintx4 read(const unsigned char* lds, int base, int b, int lane) const
    {
        const int l16 = lane % 16, q = lane / 16;
        if constexpr (KMAJOR) {
            const int r = PERM ? base + 16 * (l16 >> 2) + 4 * b + (l16 & 3) : base + 16 * b + l16;
            return *reinterpret_cast<const uintx4*>(lds + r * 64 + ((q ^ f(r)) * 16));
        } else {
            const int col = base + 16 * b + 4 * (l16 & 3);
            shortx4 v[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = 8 * q + 4 * h + (l16 >> 2);
                const unsigned char* p = lds + k * ROW + (((col / 8) ^ spread(k)) * 16) + (col % 8) * 2;
                v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)p);
            }
            uintx4 out;
            __builtin_memcpy(&out, v, 16);
            return out;
        }
    }
};

// Workgroups are dealt to the 8 XCDs in turn: consecutive tiles go to one XCD, in
// blocks of 4 m tiles, so that the tiles in flight on an XCD share rows in its L2.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t mt, uint32_t nt, int32_t& tm, int32_t& tn)
{
    const uint32_t count = mt * nt, per = count / 8, rest = count % 8, x = id % 8;
    id = x * per + (x < rest ? x : rest) + id / 8;
    constexpr uint32_t G = 4;
    const uint32_t group = id / (G * nt), in = id % (G * nt), first = group * G, rows = mt - first < G ? mt - first : G;
    tm = __builtin_amdgcn_readfirstlane(first + in % rows);
    tn = __builtin_amdgcn_readfirstlane(in / rows);
}

template <typename T, bool AK, bool BKM, bool GATED>
__global__ __launch_bounds__(256, 2) void k_gemm_large(GemmArgs a)
{
    extern __shared__ __align__(1024) unsigned char lds[];
    const Gemm& g = a.g;
    constexpr int OUTS = GATED ? BN / 2 : BN;  // outputs of a tile
    constexpr bool PERM = BKM && !GATED;
    const uint32_t tiles = (uint32_t)a.mt * a.nt, outer = blockIdx.x / tiles;
    int32_t tm, tn;
    tile_of(blockIdx.x % tiles, a.mt, a.nt, tm, tn);
    const int32_t split = __builtin_amdgcn_readfirstlane(outer % a.splits);
    const int64_t batch = (uint32_t)__builtin_amdgcn_readfirstlane(outer / a.splits);
    const int32_t m0 = tm * BM, n0 = tn * OUTS;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), q = lane / 16, l16 = lane % 16;
    const int wm = wave / 2, wn = wave % 2;
    const int32_t steps = (int32_t)g.red * a.kt;  // below 2^31
    const int32_t first = split * a.per, last = steps - first < a.per ? steps : first + a.per;

    // bases at the tile's first row (k-major) or column
    const T* A = static_cast<const T*>(g.a) + batch * g.a_batch + (AK ? m0 * g.a_row : 0);
    const T* B = static_cast<const T*>(g.b) + batch * g.b_batch + (BKM && !GATED ? n0 * g.b_row : 0);
    Operand<AK, false, BM, 2> oa;
    Operand<BKM, PERM, BN, GATED ? 3 : PERM ? 4 : 2> ob;
    oa.init(g.a_row, [&](int i) -> int64_t { return m0 + i < g.M ? (AK ? i : m0 + i) : -1; });
    if constexpr (GATED) {
        // 32 gates, then their 32 others, for each wave's 64
        ob.init(g.b_row, [&](int i) -> int64_t {
            const int32_t n = n0 + 32 * (i / 64) + i % 32;
            return n < g.N ? n + (i / 32 % 2 ? (int64_t)g.N : 0) : -1;
        });
    } else {
        ob.init(g.b_row, [&](int i) -> int64_t { return n0 + i < g.N ? (BKM ? i : n0 + i) : -1; });
    }

    floatx4 acc[8][4];  // [m tile][n tile]
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

    // the next step to fetch, and the buffers of the next fetch and of this step
    int32_t kt = first, to = 0, from = 0;
    const T *pa = A, *pb = B;
    if (a.splits > 1 && g.red > 1) {
        const int32_t r = __builtin_amdgcn_readfirstlane((uint32_t)first / (uint32_t)a.kt);
        kt = first - r * a.kt;
        pa += r * g.a_red;
        pb += r * g.b_red;
    }
    auto fetch = [&](int32_t t) {
        if (t >= last) return;
        const int32_t k0 = kt * BK;
        oa.fetch(pa + (AK ? (int64_t)k0 : k0 * g.a_row), g.a_row, g.K - k0, lds + to);
        ob.fetch(pb + (BKM ? (int64_t)k0 : k0 * g.b_row), g.b_row, g.K - k0, lds + to + A_BYTES);
        to = to == (STAGES - 1) * STAGE_BYTES ? 0 : to + STAGE_BYTES;
        if (++kt == a.kt) {
            kt = 0;
            pa += g.a_red;
            pb += g.b_red;
        }
    };
    static_assert(oa.LOADS + ob.LOADS == 6, "loads per step, counted below");
    fetch(first);
    fetch(first + 1);
    for (int32_t t = first; t < last; ++t) {
        // this step's loads are done once only the next step's are in flight
        if (t + 1 < last) asm volatile("s_waitcnt vmcnt(6) lgkmcnt(0)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // every wave has left the buffer that this fills
        fetch(t + 2);
        const unsigned char* now = lds + from;
        from = from == (STAGES - 1) * STAGE_BYTES ? 0 : from + STAGE_BYTES;
        uintx4 fb[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (GATED) {
                const int row = 64 * wn + 32 * (j >> 1) + 8 * (l16 >> 2) + 4 * (j & 1) + (l16 & 3);
                fb[j] = *reinterpret_cast<const uintx4*>(now + A_BYTES + row * 64 + ((q ^ ob.f(row)) * 16));
            } else {
                fb[j] = ob.read(now + A_BYTES, 64 * wn, j, lane);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uintx4 fa = oa.read(now, 128 * wm, i, lane);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = product<T>(fb[j], fa, acc[i][j]);
        }
    }

    // a lane's outputs of a row: 16 in a row, 8 of a gated layer, or four times 4
    constexpr int W = GATED ? 8 : PERM ? 16 : 4;
#pragma unroll
    for (int p = 0; p < (W == 4 ? 4 : 1); ++p) {
        const int64_t n = GATED ? n0 + 32 * wn + 8 * q : PERM ? n0 + 64 * wn + 16 * q : n0 + 64 * wn + 16 * p + 4 * q;
        float bz[W], bu[W];
        load_bias<T, GATED, W>(g, batch, n, bz, bu);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t m = m0 + 128 * wm + 16 * i + l16;
            if (m >= g.M) continue;
            float z[W], u[W];
#pragma unroll
            for (int e = 0; e < W; ++e) {
                z[e] = acc[i][p + e / 4][e % 4];
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
}

template <typename T>
hipError_t launch_typed(const GemmArgs& a, hipStream_t s)
{
    const Gemm& g = a.g;
    const unsigned grid = (unsigned)(g.batches * a.splits * a.mt * a.nt);
    auto go = [&](void (*kernel)(GemmArgs)) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 STAGES * STAGE_BYTES);
        if (e != hipSuccess) return e;
        kernel<<<grid, 256, STAGES * STAGE_BYTES, s>>>(a);
        return hipGetLastError();
    };
    if (g.gated) return go(k_gemm_large<T, true, true, true>);
    if (g.a_kmajor && g.b_kmajor) return go(k_gemm_large<T, true, true, false>);
    if (g.a_kmajor) return go(k_gemm_large<T, true, false, false>);
    return go(k_gemm_large<T, false, false, false>);
}

bool pieces(const Gemm& g, const void* p, int64_t row, int64_t batch, int64_t red)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && row % 8 == 0 && (g.batches <= 1 || batch % 8 == 0) &&
           (g.red <= 1 || red % 8 == 0);
}

}  // namespace

// 16-bit operands in whole 16-byte pieces (addresses, strides, and the sizes
// along which they are contiguous), offsets within a tile's reach that fit the
// buffer loads' 31 bits, and enough tiles or steps to be worth it.
bool large_fits(const Gemm& g)
{
    if (g.dtype == ES_F32 || g.K == 0 || g.red == 0 || g.red * ((g.K - 1) / BK + 1) > 0x7FFFFFFF) return false;
    if (!pieces(g, g.a, g.a_row, g.a_batch, g.a_red) || !pieces(g, g.b, g.b_row, g.b_batch, g.b_red)) return false;
    if ((g.a_kmajor || g.b_kmajor) && g.K % 8) return false;
    if ((!g.a_kmajor && g.M % 8) || (!g.b_kmajor && g.N % 8)) return false;
    // the buffers' ranges end k rows: these lie behind each other
    if ((!g.a_kmajor && g.a_row < g.M) || (!g.b_kmajor && g.b_row < g.N)) return false;
    const int64_t reach = (int64_t)1 << 30;
    if ((g.a_kmajor ? BM : BK) * g.a_row * 2 + (g.a_kmajor ? 0 : (int64_t)g.M * 2) > reach) return false;
    // a gated layer's two halves lie N rows apart
    if ((g.b_kmajor ? BN + (g.gated ? 2 * (int64_t)g.N : 0) : BK) * g.b_row * 2 + (g.b_kmajor ? 0 : (int64_t)g.N * 2) > reach) return false;
    return g.M >= 64 && g.N >= 64;
}

void large_plan(GemmArgs& a)
{
    const Gemm& g = a.g;
    a.path = PATH_LARGE;
    a.mt = (g.M - 1) / BM + 1;
    a.nt = (g.N - 1) / (g.gated ? BN / 2 : BN) + 1;
    a.kt = (g.K - 1) / BK + 1;
    const int64_t tiles = g.batches * a.mt * a.nt, steps = g.red * a.kt;
    if (tiles < 384 && steps >= 16) {
        const int64_t by_tiles = (512 + tiles - 1) / tiles, by_steps = steps / 8;
        a.splits = (int32_t)(by_tiles < by_steps ? by_tiles : by_steps);
    }
    a.per = (int32_t)((steps + a.splits - 1) / a.splits);
    a.splits = (int32_t)((steps + a.per - 1) / a.per);
}

hipError_t launch_large(const GemmArgs& a, hipStream_t s)
{
    return a.g.dtype == ES_BF16 ? launch_typed<__bf16>(a, s) : launch_typed<_Float16>(a, s);
}

}  // namespace esmi
