// es_dense_large.hip -- the matrix products of 16-bit layers at sizes where the
// matrix cores bound them, gfx950.
//
// k_gemm_wide   256 x 256 tiles of C, for products that fill the chip with them
// k_gemm_mid    128 x 128 tiles
// Steps along k pass through buffers in LDS, filled by loads that go there from
// memory without registers, ahead of their use.
//
// The loads write LDS in lane order, so the spreading over its banks is done by
// which 16 bytes a lane fetches:
//   k-major operand (k contiguous): 128 bytes of k a row; piece c of row r lies at
//     position c ^ f(r).  A 16-byte read serves lanes {0-3, 12-15, 20-27},
//     {4-11, 16-19, 28-31} and those + 32 together (measured), so the rows 4-11 of
//     a fragment meet the other rows' next piece: f spreads each such 16 over all
//     banks (one that spreads 16 lanes in a row costs twice the cycles);
//   else: a row of m (n) per k, read back transposed by ds_read_b64_tr_b16, which
//     hands lane i of 16 the four k of column i.
// Rows, columns and k beyond the matrices are not fetched: a buffer load out of
// its range writes zeros.
#include <hip/hip_runtime.h>

#include "es_dense.hpp"
#include "es_dense_device.hpp"

namespace esmi {

namespace {

constexpr uint32_t OUT = 0x80000000u;  // an offset beyond every buffer's range

typedef __attribute__((address_space(3))) void lds_void;
typedef short shortx4 __attribute__((ext_vector_type(4)));

// One operand's share of a step of STEP k: EXT rows (k-major) or columns,
// fetched by THREADS threads.
template <bool KMAJOR, int EXT, int STEP, int THREADS>
struct Operand {
    static constexpr int LOADS = EXT * STEP * 2 / (THREADS * 16);  // per lane
    static constexpr int ROW = KMAJOR ? STEP * 2 : EXT * 2;        // bytes of a staged row
    static constexpr int PIECES = ROW / 16;
    uint32_t off[LOADS];

    static __device__ __forceinline__ int f(int r)
    {
        const int a = (r >> 2) & 3;
        return (2 * a + ((r >> 1) & 1)) ^ ((a ^ (a >> 1)) & 1);
    }
    // pairs of pieces (16 columns) of different k rows on different banks
    static __device__ __forceinline__ int spread(int k) { return 2 * ((k & 3) | ((k >> 1) & 4)); }

    // row_of(i): the matrix's row (k-major) or first column of the staged piece i, -1 if outside
    template <typename F>
    __device__ __forceinline__ void init(int64_t stride, F row_of)
    {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int p = (int)threadIdx.x + THREADS * j;  // 16-byte piece of the stage
            if constexpr (KMAJOR) {
                const int r = p / PIECES, c = (p % PIECES) ^ f(r);
                const int64_t row = row_of(r);
                off[j] = row >= 0 ? (uint32_t)((row * stride + 8 * c) * 2) : OUT;
            } else {
                const int k = p / PIECES, c = (p % PIECES) ^ spread(k);
                const int64_t col = row_of(8 * c);
                off[j] = col >= 0 ? (uint32_t)((k * stride + col) * 2) : OUT;
            }
        }
    }

    // Piece j of the step at k0, base: the tile's first row at k0 (k-major) or k
    // row k0.  A lane's pieces all lie at the same k of their rows (k-major).
    __device__ __forceinline__ void load(int j, const void* base, int64_t stride, int32_t k_left, unsigned char* lds) const
    {
        static_assert(!KMAJOR || THREADS / PIECES % 16 == 0, "f() is the same for all pieces of a lane");
        const int64_t range = KMAJOR ? 0x7FFFFFFF : (k_left < STEP ? k_left : STEP) * stride * 2;
        auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)range, 0x00020000);
        const int p = (int)threadIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        const bool inside = !KMAJOR || 8 * ((p % PIECES) ^ f(p / PIECES)) < k_left;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(lds + (THREADS * j + 64 * wave) * 16), 16,
                                                 (int)(inside ? off[j] : OUT), 0, 0, 0);
    }
    __device__ __forceinline__ void fetch(const void* base, int64_t stride, int32_t k_left, unsigned char* lds) const
    {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) load(j, base, stride, k_left, lds);
    }

    // the fragment of 32 k, the `ks`th, of staged rows (columns) base + 16 b + l16
    static __device__ __forceinline__ uintx4 read(const unsigned char* lds, int base, int b, int ks, int lane)
    {
        const int l16 = lane % 16, q = lane / 16;
        if constexpr (KMAJOR) {
            const int row = base + 16 * b + l16;
            return *reinterpret_cast<const uintx4*>(lds + row * ROW + ((4 * ks + q) ^ f(row)) * 16);
        } else {
            const int col = base + 16 * b + 4 * (l16 & 3);
            shortx4 v[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = 32 * ks + 8 * q + 4 * h + (l16 >> 2);
                const unsigned char* p = lds + k * ROW + (((col / 8) ^ spread(k)) * 16) + (col % 8) * 2;
                v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)p);
            }
            uintx4 out;
            __builtin_memcpy(&out, v, 16);
            return out;
        }
    }
};

// Workgroups are dealt to the 8 XCDs in turn: consecutive tiles of the `count` go
// to one XCD,
__device__ __forceinline__ uint32_t on_one_xcd(uint32_t id, uint32_t count)
{
    const uint32_t per = count / 8, rest = count % 8, x = id % 8;
    return x * per + (x < rest ? x : rest) + id / 8;
}
// in blocks of 4 m tiles, so that the tiles in flight on an XCD share rows in its L2.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t mt, uint32_t nt, int32_t& tm, int32_t& tn)
{
    constexpr uint32_t G = 4;
    const uint32_t group = id / (G * nt), in = id % (G * nt), first = group * G, rows = mt - first < G ? mt - first : G;
    tm = __builtin_amdgcn_readfirstlane(first + in % rows);
    tn = __builtin_amdgcn_readfirstlane(in / rows);
}

// 128 x 128 tiles.  Four waves, 64 x 64 each; steps of 64 k through a ring of
// STAGES buffers of 32 KB, one barrier a step: the loads are STAGES - 1 steps
// ahead.  With two stages two workgroups share a CU and cover each other's
// barriers and epilogues; a launch of at most one a CU has four stages instead,
// and issues its loads between the products.  2048^3 bf16 29 us, 590 TFLOP/s.
constexpr int MT = 128, MK = 64, M_BYTES = MT * MK * 2;  // of one operand's buffer

template <typename T, bool AK, bool BKM, bool GATED, int STAGES>
__global__ __launch_bounds__(256, 2) void k_gemm_mid(GemmArgs a)
{
    extern __shared__ __align__(1024) unsigned char lds[];
    const Gemm& g = a.g;
    constexpr int OUTS = GATED ? MT / 2 : MT;  // outputs of a tile
    const uint32_t tiles = (uint32_t)a.mt * a.nt, outer = blockIdx.x / tiles;
    int32_t tm, tn;
    tile_of(on_one_xcd(blockIdx.x % tiles, tiles), a.mt, a.nt, tm, tn);
    const int32_t split = __builtin_amdgcn_readfirstlane(outer % a.splits);
    const int64_t batch = (uint32_t)__builtin_amdgcn_readfirstlane(outer / a.splits);
    const int32_t m0 = tm * MT, n0 = tn * OUTS;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wm = wave / 2, wn = wave % 2;
    const int32_t steps = (int32_t)g.red * a.kt;  // below 2^31
    const int32_t per = (int32_t)a.per, first = split * per, count = steps - first < per ? steps - first : per;

    using OA = Operand<AK, MT, MK, 256>;
    using OB = Operand<BKM, MT, MK, 256>;
    OA oa;
    OB ob;
    // bases at the tile's first row (k-major) or column
    const T* pa = static_cast<const T*>(g.a) + batch * g.a_batch + (AK ? m0 * g.a_row : 0);
    const T* pb = static_cast<const T*>(g.b) + batch * g.b_batch + (BKM && !GATED ? n0 * g.b_row : 0);
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
    // the next step to fetch
    int32_t kt = first;
    if (a.splits > 1 && g.red > 1) {
        const int32_t r = __builtin_amdgcn_readfirstlane((uint32_t)first / (uint32_t)a.kt);
        kt = first - r * a.kt;
        pa += r * g.a_red;
        pb += r * g.b_red;
    }
    auto fetch = [&](int32_t t) {  // step t of this workgroup's; behind the last one nothing is fetched
        const int32_t k0 = kt * MK, left = t < count ? g.K - k0 : 0;
        unsigned char* to = lds + (t % STAGES) * 2 * M_BYTES;
        oa.fetch(pa + (AK ? (int64_t)k0 : k0 * g.a_row), g.a_row, left, to);
        ob.fetch(pb + (BKM ? (int64_t)k0 : k0 * g.b_row), g.b_row, left, to + M_BYTES);
        if (++kt == a.kt) {
            kt = 0;
            pa += g.a_red;
            pb += g.b_red;
        }
    };

    floatx4 acc[4][4];  // [m tile][n tile]
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    static_assert(OA::LOADS + OB::LOADS == 8 && (STAGES == 2 || STAGES == 4), "loads per step, counted below");
    for (int s = 0; s + 1 < STAGES; ++s) fetch(s);
    for (int32_t t = 0; t < count; ++t) {
        // this step's loads are done once only the later steps' are in flight
        if constexpr (STAGES == 4) asm volatile("s_waitcnt vmcnt(16) lgkmcnt(0)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // the step to fetch: every wave has left the buffer that it fills
        const int32_t k0 = kt * MK, left = t + STAGES - 1 < count ? g.K - k0 : 0;
        unsigned char* to = lds + ((t + STAGES - 1) % STAGES) * 2 * M_BYTES;
        const T* ba = pa + (AK ? (int64_t)k0 : k0 * g.a_row);
        const T* bb = pb + (BKM ? (int64_t)k0 : k0 * g.b_row);
        if (++kt == a.kt) {
            kt = 0;
            pa += g.a_red;
            pb += g.b_red;
        }
        if constexpr (STAGES == 2) {
            oa.fetch(ba, g.a_row, left, to);
            ob.fetch(bb, g.b_row, left, to + M_BYTES);
        }
        const unsigned char* now = lds + (t % STAGES) * 2 * M_BYTES;
        uintx4 fa[2][4], fb[2][4];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
            for (int j = 0; j < 4; ++j) fb[ks][j] = OB::read(now + M_BYTES, 64 * wn, j, ks, lane);
#pragma unroll
            for (int i = 0; i < 4; ++i) fa[ks][i] = OA::read(now, 64 * wm, i, ks, lane);
        }
        // all reads under way before the first product: left to itself the compiler
        // reads two fragments at a time and waits for each
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (STAGES == 4) {
                    if (ks == 0) oa.load(i, ba, g.a_row, left, to);
                    else ob.load(i, bb, g.b_row, left, to + M_BYTES);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = product<T>(fb[ks][j], fa[ks][i], acc[i][j]);
                if constexpr (STAGES == 4) __builtin_amdgcn_sched_barrier(0);
            }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();  // the buffers serve the epilogue
    epilogue<T, GATED, 4, 4, false>(a, split, batch, m0 + 64 * wm, n0 + (GATED ? 32 : 64) * wn, acc,
                             reinterpret_cast<float*>(lds + wave * EPILOGUE_LDS<4>), lane);
}
static_assert(4 * EPILOGUE_LDS<4> <= 2 * 2 * M_BYTES, "the epilogue's rows fit the buffers");

// 256 x 256 tiles for products that fill the chip with them.  Eight waves, 128 x
// 64 each, in two groups of one wave a SIMD, a phase apart: while one group
// multiplies a step of 64 k (64 products, 1024 cycles, at raised priority), the
// other reads its next fragments; a barrier ends each phase.  A step's rows of a
// k-major operand are whole 128-byte lines.  Two buffers of 64 KB; the loads of
// step t + 1 are issued once both groups have read step t - 1:
//   phase     2t        2t + 1     2t + 2
//   group 0   read t, l multiply t read t + 1
//   group 1   mul., l   read t     multiply t, l
//   (l: loads of t + 1, all there after 2t + 1; in group 1 between the products)
// 8192 x 4096 x 4096 bf16 201 us, 1370 TFLOP/s (phases of 32 k 204, without the
// priority 221); of an earlier form at 209 the products alone took 138, with the
// fragments' reads 155, the loads alone 137: reads and loads share the LDS.
constexpr int WT = 256, WK = 64, W_BYTES = WT * WK * 2;  // of one operand's buffer

template <typename T, bool AK, bool BKM, bool GATED>
__global__ __launch_bounds__(512, 2) void k_gemm_wide(GemmArgs a)
{
    extern __shared__ __align__(1024) unsigned char lds[];
    const Gemm& g = a.g;
    constexpr int OUTS = GATED ? WT / 2 : WT;
    // A launch with a tail starts with half of its parts, so that those CUs are out of
    // step with the others: the epilogues' stores then meet other tiles' products.
    const uint32_t tiles = (uint32_t)a.mt * a.nt, full = tiles - a.tail, ahead = a.tail * (a.tail_splits / 2);
    uint32_t id = blockIdx.x, outer = 0;
    int32_t tm, tn, part = -1;
    if (a.tail == 0) {
        outer = id / tiles;
        id = on_one_xcd(id % tiles, tiles);
    } else if (id >= ahead && id < ahead + full) {
        id = on_one_xcd(id - ahead, full);
    } else {
        part = __builtin_amdgcn_readfirstlane(id < ahead ? id : id - full);
        id = full + part % a.tail;
    }
    tile_of(id, a.mt, a.nt, tm, tn);
    const int32_t split = __builtin_amdgcn_readfirstlane(outer % a.splits);
    const int64_t batch = (uint32_t)__builtin_amdgcn_readfirstlane(outer / a.splits);
    const int32_t m0 = tm * WT, n0 = tn * OUTS;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int group = wave / 4, wm = group, wn = wave % 4;
    const int32_t steps = (int32_t)g.red * a.kt;  // below 2^31
    const int32_t per = part < 0 ? (int32_t)a.per : a.tail_per;
    const int32_t first = (part < 0 ? split : part / a.tail) * per, count = steps - first < per ? steps - first : per;

    using OA = Operand<AK, WT, WK, 512>;
    using OB = Operand<BKM, WT, WK, 512>;
    OA oa;
    OB ob;
    const T* pa = static_cast<const T*>(g.a) + batch * g.a_batch + (AK ? m0 * g.a_row : 0);
    const T* pb = static_cast<const T*>(g.b) + batch * g.b_batch + (BKM && !GATED ? n0 * g.b_row : 0);
    oa.init(g.a_row, [&](int i) -> int64_t { return m0 + i < g.M ? (AK ? i : m0 + i) : -1; });
    if constexpr (GATED) {
        ob.init(g.b_row, [&](int i) -> int64_t {
            const int32_t n = n0 + 32 * (i / 64) + i % 32;
            return n < g.N ? n + (i / 32 % 2 ? (int64_t)g.N : 0) : -1;
        });
    } else {
        ob.init(g.b_row, [&](int i) -> int64_t { return n0 + i < g.N ? (BKM ? i : n0 + i) : -1; });
    }
    int32_t kt = first;
    if (first > 0 && g.red > 1) {
        const int32_t r = __builtin_amdgcn_readfirstlane((uint32_t)first / (uint32_t)a.kt);
        kt = first - r * a.kt;
        pa += r * g.a_red;
        pb += r * g.b_red;
    }
    auto fetch = [&](int32_t t) {  // step t of this workgroup's; behind the last one nothing is fetched
        const int32_t k0 = kt * WK, left = t < count ? g.K - k0 : 0;
        unsigned char* to = lds + (t & 1) * 2 * W_BYTES;
        oa.fetch(pa + (AK ? (int64_t)k0 : k0 * g.a_row), g.a_row, left, to);
        ob.fetch(pb + (BKM ? (int64_t)k0 : k0 * g.b_row), g.b_row, left, to + W_BYTES);
        if (++kt == a.kt) {
            kt = 0;
            pa += g.a_red;
            pb += g.b_red;
        }
    };

    floatx4 acc[8][4];  // [m tile][n tile]
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    uintx4 fa[2][8], fb[2][4];
    auto read = [&](int32_t t) {
        const unsigned char* from = lds + (t & 1) * 2 * W_BYTES;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
            for (int j = 0; j < 4; ++j) fb[ks][j] = OB::read(from + W_BYTES, 64 * wn, j, ks, lane);
#pragma unroll
            for (int i = 0; i < 8; ++i) fa[ks][i] = OA::read(from, 128 * wm, i, ks, lane);
        }
    };
    auto multiply = [&]() {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = product<T>(fb[ks][j], fa[ks][i], acc[i][j]);
        __builtin_amdgcn_s_setprio(0);
    };
    // the same with the loads of step t in between
    auto multiply_fetch = [&](int32_t t) {
        const int32_t k0 = kt * WK, left = t < count ? g.K - k0 : 0;
        unsigned char* to = lds + (t & 1) * 2 * W_BYTES;
        const T* ba = pa + (AK ? (int64_t)k0 : k0 * g.a_row);
        const T* bb = pb + (BKM ? (int64_t)k0 : k0 * g.b_row);
        if (++kt == a.kt) {
            kt = 0;
            pa += g.a_red;
            pb += g.b_red;
        }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i % 4 == 0) oa.load(2 * ks + i / 4, ba, g.a_row, left, to);
                else if (i % 4 == 2) ob.load(2 * ks + i / 4, bb, g.b_row, left, to + W_BYTES);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = product<T>(fb[ks][j], fa[ks][i], acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);
            }
        __builtin_amdgcn_s_setprio(0);
    };
    // ends a phase: what this wave has read is in its registers
    auto phase = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
    };
    auto arrived = [&]() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };

    fetch(0);
    arrived();
    phase();
    if (group == 0) {
        for (int32_t t = 0; t < count; ++t) {
            read(t);
            __builtin_amdgcn_sched_barrier(0);
            fetch(t + 1);
            phase();
            multiply();
            arrived();
            phase();
        }
        phase();
    } else {
        fetch(1);
        phase();
        for (int32_t t = 0; t < count; ++t) {
            read(t);
            arrived();
            phase();
            multiply_fetch(t + 2);
            phase();
        }
    }
    arrived();
    __syncthreads();  // the buffers serve the epilogue
    epilogue<T, GATED, 8, 4, true>(a, split, batch, m0 + 128 * wm, n0 + (GATED ? 32 : 64) * wn, acc,
                             reinterpret_cast<float*>(lds + wave * EPILOGUE_LDS<4>), lane,
                             part < 0 ? nullptr : a.partial + ((int64_t)part * WT + 128 * wm) * WT + (GATED ? 32 : 64) * wn);
}
static_assert(8 * EPILOGUE_LDS<4> <= 4 * W_BYTES, "the epilogue's rows fit the buffers");

// The tail's sums and their epilogue, four outputs a thread.  Bound by memory: 67 MB of
// sums of 64 tiles in 4 parts 12.6 us, 5.3 TB/s
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_tail_join(GemmArgs a)
{
    const Gemm& g = a.g;
    constexpr int OUTS = GATED ? WT / 2 : WT, PER = WT * OUTS / 4 / 256;  // workgroups a tile
    const uint32_t tile = blockIdx.x / PER, at = (blockIdx.x % PER) * 256 + threadIdx.x;
    const int32_t row = at / (OUTS / 4), col = at % (OUTS / 4) * 4;
    int32_t tm, tn;
    tile_of((uint32_t)a.mt * a.nt - a.tail + tile, a.mt, a.nt, tm, tn);
    const int32_t m = tm * WT + row, n = tn * OUTS + col;
    if (m >= g.M || n >= g.N) return;
    float z[4] = {}, u[4] = {}, bz[4], bu[4], r[4];
    load_bias<T, GATED, 4>(g, 0, n, bz, bu);
    load_res<T, 4>(a, 0, m, n, r);
    const float* p = a.partial + ((int64_t)tile * WT + row) * WT + col;
#pragma unroll 2
    for (int32_t s = 0; s < a.tail_splits; ++s, p += (int64_t)a.tail * WT * WT) {
        float v[4];
        load_run<float, 4>(p, 4, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] += v[i];
        if constexpr (GATED) {
            load_run<float, 4>(p + WT / 2, 4, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] += v[i];
        }
    }
    finish<T, GATED, 4>(a, 0, m, n, z, u, bz, bu, r);
}

template <typename T, bool AK, bool BKM, bool GATED>
hipError_t launch_kernel(const GemmArgs& a, hipStream_t s)
{
    const unsigned grid = (unsigned)(a.g.batches * a.splits * a.mt * a.nt + (int64_t)a.tail * (a.tail_splits - 1));
    const bool wide = a.tile == WT, deep = grid <= 256;
    void (*kernel)(GemmArgs) = wide ? k_gemm_wide<T, AK, BKM, GATED>
                               : deep ? k_gemm_mid<T, AK, BKM, GATED, 4> : k_gemm_mid<T, AK, BKM, GATED, 2>;
    const int bytes = wide ? 4 * W_BYTES : (deep ? 4 : 2) * 2 * M_BYTES;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    e = launch(kernel, grid, (unsigned)large_threads(a), (size_t)bytes, s, a);
    if (e == hipSuccess && a.tail) e = launch(k_tail_join<T, GATED>, (unsigned)a.tail * (WT * WT / (GATED ? 2 : 1) / 1024), 256, 0, s, a);
    return e;
}

template <typename T>
hipError_t launch_typed(const GemmArgs& a, hipStream_t s)
{
    const Gemm& g = a.g;
    if (g.gated) return launch_kernel<T, true, true, true>(a, s);
    if (g.a_kmajor && g.b_kmajor) return launch_kernel<T, true, true, false>(a, s);
    if (g.a_kmajor) return launch_kernel<T, true, false, false>(a, s);
    return launch_kernel<T, false, false, false>(a, s);
}

bool pieces(const Gemm& g, const void* p, int64_t row, int64_t batch, int64_t red)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && row % 8 == 0 && (g.batches <= 1 || batch % 8 == 0) &&
           (g.red <= 1 || red % 8 == 0);
}

}  // namespace

// Whether an operand can be fetched in whole 16-byte pieces as it lies: its
// addresses, strides, and the size along which it is contiguous.
bool large_takes(const Gemm& g, bool is_a)
{
    const bool kmajor = is_a ? g.a_kmajor : g.b_kmajor, padded = is_a ? g.a_padded : g.b_padded;
    return (is_a ? pieces(g, g.a, g.a_row, g.a_batch, g.a_red) : pieces(g, g.b, g.b_row, g.b_batch, g.b_red)) &&
           (padded || (kmajor ? g.K : is_a ? g.M : g.N) % 8 == 0);
}

// 16-bit operands in whole pieces, offsets within a tile's reach that fit the
// buffer loads' 31 bits, and at least a quarter of a tile.
bool large_fits(const Gemm& g)
{
    if (g.dtype == ES_F32 || g.K == 0 || g.red == 0 || g.red * ((g.K - 1) / WK + 1) > 0x7FFFFFFF) return false;
    if (!large_takes(g, true) || !large_takes(g, false)) return false;
    // the buffers' ranges end k rows: these lie behind each other
    if ((!g.a_kmajor && g.a_row < g.M) || (!g.b_kmajor && g.b_row < g.N)) return false;
    const int64_t reach = (int64_t)1 << 30;
    if ((g.a_kmajor ? WT : WK) * g.a_row * 2 + (g.a_kmajor ? 0 : (int64_t)g.M * 2) > reach) return false;
    // a gated layer's two halves lie N rows apart
    if ((g.b_kmajor ? WT + (g.gated ? 2 * (int64_t)g.N : 0) : WK) * g.b_row * 2 + (g.b_kmajor ? 0 : (int64_t)g.N * 2) > reach) return false;
    return g.M >= 64 && g.N >= 64;
}

// 256 x 256 tiles from 192 on (three quarters of the CUs: 4096 x 4096 -> 11264 bf16
// 334 us against 390 in smaller ones), and where few of them have long sums (below).  With at most 128 of the smaller ones, a
// long sum is split until the CUs have one each, 8 steps at least: a split's sums
// pass through memory twice (1024^3 in 4 splits of 4 steps 25 us, in 2 of 8 21).
void large_plan(GemmArgs& a)
{
    const Gemm& g = a.g;
    a.path = PATH_LARGE;
    a.tile = WT;
    a.mt = (g.M - 1) / WT + 1;
    a.nt = (g.N - 1) / (g.gated ? WT / 2 : WT) + 1;
    a.kt = (g.K - 1) / WK + 1;
    const int64_t steps = g.red * a.kt;
    const int64_t wides = (int64_t)a.mt * a.nt;
    // no wider than the smaller tiles: half of the larger ones, or more, would be padding
    // (128 rows of 4096 to 49152 bf16 127 us, 99 in smaller tiles; 64 of 2048 to 131072 147, 137)
    const bool thin = g.M <= MT || g.N <= (g.gated ? MT / 2 : MT);
    const bool all_parts = !thin && g.batches == 1 && wides >= 48 && wides <= 128 && steps >= 160;
    if (thin || (g.batches * a.mt * a.nt < 192 && !all_parts)) {
        a.tile = MT;
        a.mt = (g.M - 1) / MT + 1;
        a.nt = (g.N - 1) / (g.gated ? MT / 2 : MT) + 1;
        const int64_t tiles = g.batches * a.mt * a.nt;
        if (tiles <= 128 && steps >= 8) {
            const int64_t by_tiles = 256 / tiles, by_steps = steps / 8;
            a.splits = (int32_t)(by_tiles < by_steps ? by_tiles : by_steps);
        }
    }
    a.per = (steps + a.splits - 1) / a.splits;
    a.splits = (int32_t)((steps + a.per - 1) / a.per);
    // At most half a round of tiles behind full ones: in parts they take a part of a
    // round (1.6 us a step), their sums go through memory once more (bf16, 4096 long:
    // 4352 rows to 4096 outputs, 16 tiles over, 186 -> 131 us; 8192 to 4608, 64 over,
    // 288 -> 257; 8192 to 11264, 128 over, 647 -> 606).  Without full rounds, sums of
    // 160 steps or more are all parts: 2048 to 2048 bf16, 64 tiles, 11264 long 117 us
    // in smaller tiles, 111 in parts, 22528 long 220 and 180, but 8192 long 84 and 86,
    // 4096 long 47 and 55; 2560 to 2048, 80 tiles, 11264 long 148 and 120.
    const int64_t tiles = (int64_t)a.mt * a.nt, rest = tiles % 256;
    if (a.tile == WT && g.batches == 1 && (tiles > 256 || all_parts) && rest > 0 && rest <= 128) {
        int64_t parts = 256 / rest;
        if (parts > steps / 8) parts = steps / 8;
        const double saved = steps * 1.6e-6 * (1.0 - 1.0 / (double)parts);
        const double cost = 2.0 * rest * parts * WT * WT * 4 / 4.5e12 + 5e-6;
        if (parts >= 2 && (saved > cost || all_parts)) {
            a.tail_per = (int32_t)((steps + parts - 1) / parts);
            a.tail_splits = (int32_t)((steps + a.tail_per - 1) / a.tail_per);
            a.tail = (int32_t)rest;
        }
    }
}

int64_t large_threads(const GemmArgs& a) { return a.tile == WT ? 512 : 256; }

hipError_t launch_large(const GemmArgs& a, hipStream_t s)
{
    return a.g.dtype == ES_BF16 ? launch_typed<__bf16>(a, s) : launch_typed<_Float16>(a, s);
}

}  // namespace esmi
