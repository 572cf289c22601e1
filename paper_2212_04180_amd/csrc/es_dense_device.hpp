// es_dense_device.hpp -- device code that the layer kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>

#include "es_dense.hpp"
#include "es_launch.hpp"

namespace esmi {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

// ---- activations ----------------------------------------------------------
// Evaluated in fp32.  FAST: for results that are rounded to 16 bits (or summed
// from 16-bit operands), values within (2 z^2 + 32) 2^-24 relative (the exponent's
// rounding; tanh and silu closer); else the math library's.
constexpr float LOG2E = 1.44269504088896340736f;

template <bool FAST>
__device__ __forceinline__ float act_tanh(float z)
{
    if constexpr (!FAST) return tanhf(z);
    // 1 - 2 / (e^2z + 1) loses its leading digits towards 0; the odd Taylor
    // polynomial to z^7 is within 62/2835 z^8 of tanh z relative: 3e-7 at 1/4
    const float s = z * z;
    const float near = z * fmaf(s, fmaf(s, fmaf(s, -17.f / 315.f, 2.f / 15.f), -1.f / 3.f), 1.f);
    const float far = fmaf(-2.f, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(z * (2.f * LOG2E)) + 1.f), 1.f);
    return s < 0.0625f ? near : far;
}

// Its slope 4 e / (1 + e)^2 with e = e^(-2|z|), which keeps its digits where tanh is
// next to 1 ((1 - t) (1 + t) is off by 6e-2 at 8 and 0 at 10).
template <bool FAST>
__device__ __forceinline__ float tanh_slope(float z)
{
    const float a = __builtin_fabsf(z);
    const float e = FAST ? __builtin_amdgcn_exp2f(a * (-2.f * LOG2E)) : expf(-2.f * a);
    const float r = FAST ? __builtin_amdgcn_rcpf(1.f + e) : 1.f / (1.f + e);
    return 4.f * e * (r * r);
}

// Phi(z), the normal distribution function.  FAST: Phi(-|z|) e^(z^2/2), which falls
// slowly, as a polynomial without constant term in t = 1 / (1 + p |z|) (the form of
// Abramowitz and Stegun 7.1.26), fitted here for the least relative error, 9e-8 for
// |z| up to 13.5, where fp32 ends: 16-bit results keep their half step in the tail
// too (the published coefficients, for absolute errors, are off by 5e-4 at -4 and
// 1e-2 at -8).  With e's exponent rounded, within (2 z^2 + 32) 2^-24 of Phi(-|z|).
template <bool FAST>
__device__ __forceinline__ float normal_cdf(float z, float e /* e^(-z^2/2), FAST only */)
{
    if constexpr (!FAST) return 0.5f * erfcf(-0.70710678118654752440f * z);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.23334524f, __builtin_fabsf(z), 1.f));
    float p = fmaf(t, -0.06796955f, 0.23136756f);
    p = fmaf(t, p, -0.17776404f);
    p = fmaf(t, p, 0.20631662f);
    p = fmaf(t, p, 0.022477893f);
    p = fmaf(t, p, 0.10097145f);
    p = fmaf(t, p, 0.091416836f);
    p = fmaf(t, p, 0.0931832f);
    const float tail = t * p * e;
    return z < 0.f ? tail : 1.f - tail;
}

template <bool FAST>
__device__ __forceinline__ float bell(float z)  // e^(-z^2/2)
{
    if constexpr (!FAST) return expf(-0.5f * z * z);
    return __builtin_amdgcn_exp2f(z * z * (-0.5f * LOG2E));
}

template <bool FAST>
__device__ __forceinline__ float sigmoid(float z)
{
    if constexpr (!FAST) return 1.f / (1.f + expf(-z));
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -LOG2E));
}

// Values, and with SLOPE slopes in d, of W inputs, one branch for all of them.
template <bool FAST, bool SLOPE, int W>
__device__ __forceinline__ void activate(int32_t act, float z[W], float d[W])
{
    switch (act) {
    case ES_ACT_RELU:
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (SLOPE) d[i] = z[i] > 0.f ? 1.f : z[i] != z[i] ? z[i] : 0.f;
            z[i] = z[i] <= 0.f ? 0.f : z[i];  // NaN stays
        }
        break;
    case ES_ACT_TANH:
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (SLOPE) d[i] = tanh_slope<FAST>(z[i]);
            z[i] = act_tanh<FAST>(z[i]);
        }
        break;
    case ES_ACT_GELU:
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float e = FAST || SLOPE ? bell<FAST>(z[i]) : 0.f, phi = normal_cdf<FAST>(z[i], e);
            if constexpr (SLOPE) d[i] = fmaf(z[i] * e, 0.39894228040143267794f, phi);
            z[i] *= phi;
        }
        break;
    case ES_ACT_SILU:
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float s = sigmoid<FAST>(z[i]);
            if constexpr (SLOPE) d[i] = s * fmaf(z[i], 1.f - s, 1.f);
            z[i] *= s;
        }
        break;
    default:
        if constexpr (SLOPE) {
#pragma unroll
            for (int i = 0; i < W; ++i) d[i] = 1.f;
        }
    }
}

template <typename T>
__device__ __forceinline__ float widen(T v) { return (float)v; }

template <typename T>
__device__ __forceinline__ floatx4 product(uintx4 a, uintx4 b, floatx4 c)
{
    if constexpr (sizeof(T) == 4) {
        // four steps of 4: the k index within the 64 bytes is permuted alike on both sides
        const floatx4 x = __builtin_bit_cast(floatx4, a), y = __builtin_bit_cast(floatx4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
        return c;
    } else if constexpr (__is_same(T, __bf16)) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
}

// 16 bytes at an even address: 16-byte loads at odd multiples of 2 run at less
// than half the rate (rows of 4095 bf16 1.9 TB/s, of 4098 4.5), so such 16-bit
// elements are read in the aligned words that hold them, and shifted.  Nothing
// beyond those words is touched.
__device__ __forceinline__ uintx4 load16_odd(const void* p)
{
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    const uint32_t* w = reinterpret_cast<const uint32_t*>(at & ~(uintptr_t)3);
    const uint32_t shift = (uint32_t)(at & 2) * 8;
    uintx4 t, v;
    __builtin_memcpy(&t, w, 16);
    const uint32_t last = w[shift ? 4 : 3];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_alignbit(i < 3 ? t[i + 1] : last, t[i], shift);
    return v;
}

// ---- a product's launch ---------------------------------------------------
enum GemmPath { PATH_STAGED, PATH_LARGE, PATH_ROWS };

struct GemmArgs {
    Gemm g;  // on the packed copies, if any
    int32_t path;
    int32_t splits;        // of the reduction; 1: C is finished here (few rows: among a workgroup's waves)
    int32_t mt, nt, kt;    // tiles
    int32_t tile;          // staged: edge of a tile
    bool odd_a, odd_b;     // 16-bit rows at odd multiples of 2 bytes
    int64_t per;           // steps of a split
    // 256 x 256 tiles only: the last `tail` tiles, which would leave most CUs idle
    // at the end, are split into tail_splits parts of tail_per steps; their sums go
    // to partial as [tail_splits][tail][256][256]
    int32_t tail, tail_splits, tail_per;
    float* partial;        // [splits][batches][M][N or 2 N]
};

// W consecutive elements of a row, `left` > 0 of them in it (the others repeat
// its last).  16-byte accesses at any element's address: the target takes them.
template <typename T, int W>
__device__ __forceinline__ void load_run(const T* p, int32_t left, float out[W])
{
    T t[W];
    // As words: from a copy straight into t the compiler makes W loads (dz of 8192 x
    // 4096 bf16 76 us, so 44; the sums of 4095 columns alone, at odd addresses, 66, so
    // 41).  Not 32-bit ones at other addresses (dz of 96 members' 250 x 253 17.3 us, from W loads 15.6).
    typedef uint32_t words __attribute__((ext_vector_type(W * sizeof(T) / 4), aligned(2)));
    if (left >= W && (sizeof(T) == 2 || reinterpret_cast<uintptr_t>(p) % 16 == 0)) {
        const words q = *reinterpret_cast<const words*>(p);
        __builtin_memcpy(t, &q, W * sizeof(T));
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) t[i] = p[i < left ? i : left - 1];  // no branches: all in flight at once
    }
#pragma unroll
    for (int i = 0; i < W; ++i) out[i] = widen(t[i]);
}

// STREAM: past the caches.  (Chosen at compile time: the compiler joins the two
// stores of a branch into a plain one.)
template <typename T, int W, bool STREAM = false>
__device__ __forceinline__ void store_run(T* p, int32_t left, const float v[W])
{
    T t[W];
#pragma unroll
    for (int i = 0; i < W; ++i) t[i] = (T)v[i];
    if (left >= W) {
        if constexpr (STREAM) {
            typedef uint32_t piece __attribute__((ext_vector_type(4), aligned(2)));
#pragma unroll
            for (int i = 0; i < W * (int)sizeof(T) / 16; ++i) {
                piece q;
                __builtin_memcpy(&q, t + 16 / sizeof(T) * i, 16);
                __builtin_nontemporal_store(q, reinterpret_cast<piece*>(p + 16 / sizeof(T) * i));
            }
        } else {
            __builtin_memcpy(p, t, W * sizeof(T));
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < left) p[i] = t[i];
    }
}

// The residual of W consecutive outputs from column n of row m
template <typename T, int W>
__device__ __forceinline__ void load_res(const GemmArgs& a, int64_t batch, int64_t m, int32_t n, float r[W])
{
    const Gemm& g = a.g;
    if (g.res && n < g.N)
        load_run<T, W>(static_cast<const T*>(g.res) + batch * g.res_batch + m * g.res_row + n, g.N - n, r);
    else
#pragma unroll
        for (int i = 0; i < W; ++i) r[i] = 0.f;
}

// Bias, activation, gate and residual of W consecutive outputs from column n
// of row m, rounded and stored.  bz, bu: their biases, r: the residual.
template <typename T, bool GATED, int W, bool STREAM = false>
__device__ __forceinline__ void finish(const GemmArgs& a, int64_t batch, int64_t m, int32_t n, float z[W], float u[W],
                                       const float bz[W], const float bu[W], const float r[W])
{
    const Gemm& g = a.g;
    constexpr bool FAST = sizeof(T) == 2;
    const int32_t left = g.N - n;
    if (left <= 0) return;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        z[i] += bz[i];
        if constexpr (GATED) u[i] += bu[i];
    }
    if (g.pre) {
        T* pre = static_cast<T*>(g.pre) + batch * g.pre_batch + m * g.pre_row + n;
        store_run<T, W, STREAM>(pre, left, z);
        if constexpr (GATED) store_run<T, W, STREAM>(pre + g.N, left, u);
    }
    activate<FAST, false, W>(g.act, z, nullptr);
    if constexpr (GATED) {
#pragma unroll
        for (int i = 0; i < W; ++i) z[i] *= u[i];
    }
    if (g.res) {
#pragma unroll
        for (int i = 0; i < W; ++i) z[i] += r[i];
    }
    const int64_t at = batch * g.c_batch + m * g.c_row + n;
    if (g.c_dtype == ES_F32) store_run<float, W, STREAM>(static_cast<float*>(g.c) + at, left, z);
    else store_run<T, W, STREAM>(static_cast<T*>(g.c) + at, left, z);
}

template <typename T, bool GATED, int W>
__device__ __forceinline__ void load_bias(const Gemm& g, int64_t batch, int32_t n, float bz[W], float bu[W])
{
#pragma unroll
    for (int i = 0; i < W; ++i) bz[i] = bu[i] = 0.f;
    if (!g.bias || n >= g.N) return;
    const T* b = static_cast<const T*>(g.bias) + batch * g.bias_batch + n;
    load_run<T, W>(b, g.N - n, bz);
    if constexpr (GATED) load_run<T, W>(b + g.N, g.N - n, bu);
}

// Partial sums of W consecutive outputs
template <bool GATED, int W>
__device__ __forceinline__ void store_partial(const GemmArgs& a, int32_t split, int64_t batch, int64_t m, int32_t n,
                                              const float z[W], const float u[W])
{
    const Gemm& g = a.g;
    const int32_t left = g.N - n;
    if (left <= 0) return;
    float* p = a.partial + ((split * g.batches + batch) * g.M + m) * (GATED ? 2 * (int64_t)g.N : g.N) + n;
    store_run<float, W>(p, left, z);
    if constexpr (GATED) store_run<float, W>(p + g.N, left, u);
}

// Bytes of LDS that a wave's epilogue takes: 32 rows of its NB column tiles.
template <int NB>
constexpr int EPILOGUE_LDS = 32 * (16 * NB + 4) * 4;

// Orders a wave's own LDS accesses across its lanes (no instruction: the LDS
// serves a wave in order).
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// What follows a wave's MB x NB tiles of C from row m0 and output n0 (a gated
// layer's columns: the gates, then as many others).  The tiles pass through LDS,
// 32 rows at a time (rows padded by 16 bytes: the writes meet all banks), so that
// a lane finishes 8 outputs side by side and 64-column rows are stored whole;
// straight from the accumulators the same code took 9 times the instructions
// and a seventh of a 4096-long product's time.  lds: this wave's own.
// STREAM: for launches whose outputs are more than the L2s hold (8 of 4 MB): stored
// past them they leave the operands' rows there (8192 x 4096 -> 11264 bf16 with its
// pre 711 -> 640 us).
// part: null, or where the sums of this wave's rows and columns go instead, rows
// of 256, a gated layer's others 128 behind its gates.
template <typename T, bool GATED, int MB, int NB, bool STREAM>
__device__ __forceinline__ void epilogue(const GemmArgs& a, int32_t split, int64_t batch, int32_t m0, int32_t n0,
                                         floatx4 (&acc)[MB][NB], float* lds, int lane, float* part = nullptr)
{
    const Gemm& g = a.g;
    constexpr int COLS = 16 * NB, PITCH = COLS + 4, OUTS = GATED ? COLS / 2 : COLS;
    constexpr int PER_ROW = OUTS / 8, ROWS = 64 / PER_ROW;  // lanes of a row, rows at once
    const int q = lane / 16, l16 = lane % 16, col = lane % PER_ROW * 8;
    const int32_t n = n0 + col;
    float bz[8], bu[8];
    load_bias<T, GATED, 8>(g, batch, n, bz, bu);
#pragma unroll
    for (int p = 0; p < MB / 2; ++p) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
                *reinterpret_cast<floatx4*>(lds + (16 * i + l16) * PITCH + 16 * j + 4 * q) = acc[2 * p + i][j];
        wave_sync();
#pragma unroll 1
        for (int r = lane / PER_ROW; r < 32; r += ROWS) {
            const int32_t m = m0 + 32 * p + r;
            if (m >= g.M || n >= g.N) continue;
            float z[8], u[8], res[8];
            if (a.splits == 1 && !part) load_res<T, 8>(a, batch, m, n, res);
            const float* from = lds + r * PITCH + col;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                z[e] = from[e];
                u[e] = GATED ? from[e + COLS / 2] : 0.f;
            }
            if (part) {
                float* to = part + (32 * p + r) * 256 + col;
                store_run<float, 8>(to, 8, z);
                if constexpr (GATED) store_run<float, 8>(to + 128, 8, u);
            } else if (a.splits > 1) {
                store_partial<GATED, 8>(a, split, batch, m, n, z, u);
            } else {
                finish<T, GATED, 8, STREAM>(a, batch, m, n, z, u, bz, bu, res);
            }
        }
        wave_sync();
    }
}

bool rows_fits(const Gemm& g);
void rows_plan(GemmArgs& a);
hipError_t launch_rows(const GemmArgs& a, hipStream_t s);
bool large_takes(const Gemm& g, bool is_a);
bool large_fits(const Gemm& g);
void large_plan(GemmArgs& a);
int64_t large_threads(const GemmArgs& a);  // of a workgroup
hipError_t launch_large(const GemmArgs& a, hipStream_t s);

}  // namespace esmi
