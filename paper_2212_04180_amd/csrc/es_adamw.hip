// es_adamw.hip -- AdamW on many tensors in one launch, gfx950.
//
// Bound by memory: an element takes 28 bytes with 32-bit states and gradients
// (16 and 1/16 with 8-bit states), against about 70 instructions.  One wave owns
// 256 consecutive elements, four a lane: the loads and stores of p, m, v are
// 16 bytes a lane, and a block of 8-bit states that shares a scale is exactly
// one wave's, so that its new scale is one reduction across the lanes and the
// states are read and written once.
//
// Nothing is read twice, so the arrays go past the caches (nontemporal loads and
// stores): 2.06e8 parameters with 32-bit states, bf16 gradients and copies 1100 -> 989
// us (5.8 TB/s), with 8-bit states and fp32 gradients 631 -> 580 (5.7 TB/s); 2^26 with 32-bit
// states 344 -> 304, 2^22, which the caches hold, 21.1 -> 19.1.
// Only where the last cache just holds a step's arrays (2^23 and 2^24 elements with
// 32-bit states) steps that follow each other at once lose: 36.4 -> 38.8, 69.8 -> 75.3.
#include <hip/hip_runtime.h>
#include <math.h>

#include <cstdio>

#include "es_internal.hpp"
#include "es_launch.hpp"
#include "esmi.h"

// products and sums round by themselves unless written as one fma
#pragma clang fp contract(off)

namespace esmi {

namespace {

constexpr int MAX_TENSORS = 44;   // per launch: their table travels in the kernel's arguments
constexpr int BLOCK = 256;        // elements that share a scale; one wave's work
constexpr int LARGE_SPAN = 4;     // blocks of a wave of large calls
// HIP takes fewer than 2^32 work-items a launch: a tensor's, in one launch
constexpr int64_t MAX_GROUPS = 0xFFFFFFFFll / 256, MAX_N = MAX_GROUPS * 4 * LARGE_SPAN * BLOCK;
constexpr float F8_MAX = 448.f;   // largest e4m3 value
constexpr float F8_MIN = 0x1p-9f; // smallest above zero

struct Tensor {
    float* p;
    const void* g;
    void *m, *v;
    float *ms, *vs;
    void* copy;
    int64_t n;
    float lr, keep;        // keep = 1 - lr weight_decay
    uint32_t first;        // its first workgroup
    uint32_t whole;        // all its arrays take 4 elements a lane at once
};

struct AdamwArgs {
    Tensor t[MAX_TENSORS];
    int32_t count;
    float beta1, omb1, beta2, omb2, bc1, bc2, eps;
    float rbc1, rsbc2;  // 1 / bc1, 1 / sqrt(bc2)
    uint32_t span;  // blocks per wave
};
static_assert(sizeof(AdamwArgs) <= 4096, "the table travels in the kernel's arguments");

template <typename G>
__device__ __forceinline__ void load4(const G* p, bool whole, int left, float out[4])
{
    if (whole && left >= 4) {
        G t[4];
        typedef uint32_t piece __attribute__((ext_vector_type(sizeof(G))));  // 4 elements
        const piece q = __builtin_nontemporal_load(reinterpret_cast<const piece*>(p));
        __builtin_memcpy(t, &q, 4 * sizeof(G));
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = (float)t[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = i < left ? (float)p[i] : 0.f;
    }
}

template <typename G>
__device__ __forceinline__ void store4(G* p, bool whole, int left, const float v[4])
{
    if (whole && left >= 4) {
        G t[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = (G)v[i];
        typedef uint32_t piece __attribute__((ext_vector_type(sizeof(G))));
        piece q;
        __builtin_memcpy(&q, t, 4 * sizeof(G));
        __builtin_nontemporal_store(q, reinterpret_cast<piece*>(p));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) p[i] = (G)v[i];
    }
}

__device__ __forceinline__ uint32_t load4_codes(const uint8_t* p, bool whole, int left)
{
    if (whole && left >= 4) return *reinterpret_cast<const uint32_t*>(p);  // nontemporal: 177 -> 184 us at 2^26
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) c |= (uint32_t)p[i] << (8 * i);
    return c;
}

__device__ __forceinline__ void store4_codes(uint8_t* p, bool whole, int left, uint32_t c)
{
    if (whole && left >= 4) {
        __builtin_nontemporal_store(c, reinterpret_cast<uint32_t*>(p));
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) p[i] = (uint8_t)(c >> (8 * i));
}

__device__ __forceinline__ void decode4(uint32_t c, float scale, float out[4])
{
    typedef float floatx2 __attribute__((ext_vector_type(2)));
    const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    out[0] = lo[0] * scale;
    out[1] = lo[1] * scale;
    out[2] = hi[0] * scale;
    out[3] = hi[1] * scale;
}

// The wave's scale of the finite values, and their nearest codes; a square
// root above zero takes a code above zero: a v of 0 beside an m that is not
// would make the next step divide by eps alone.
template <bool ROOT>
__device__ __forceinline__ uint32_t encode4(const float x[4], float& scale)
{
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = __builtin_fabsf(x[i]);
        top = a < __builtin_inff() ? fmaxf(top, a) : top;  // neither infinities nor NaN
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    scale = fmaxf(top * (1.0f / F8_MAX), 0x1p-126f);
    // x / scale correctly rounded by one residual of x times the correctly rounded
    // reciprocal (Markstein 1990): the wave divides once, not eight times a lane.
    // (The residual is exact for scales above 2^-90; below, a code may be the next one.)
    const float r = 1.0f / scale;
    float q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float q0 = x[i] * r;
        q[i] = __builtin_copysignf(__builtin_fmaf(__builtin_fmaf(-q0, scale, x[i]), r, q0), x[i]);  // -0 stays
        if (ROOT && x[i] > 0.f) q[i] = fmaxf(q[i], F8_MIN);
        // at most 448 but for the division's rounding; infinities become NaN
        q[i] = __builtin_fabsf(x[i]) < __builtin_inff() ? fminf(fmaxf(q[i], -F8_MAX), F8_MAX) : __builtin_nanf("");
    }
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], c, true);
    return (uint32_t)c;
}

// BITS 32: the operation order of es_tell's Adam, so the same bits.  BITS 8:
// every product and sum rounded by itself: a state next to the border of two
// codes then falls on the same side in any fp32 evaluation of the formulas.
template <typename G, typename C, int BITS>
__global__ __launch_bounds__(256) void k_adamw(AdamwArgs a)
{
    // the tensor of this workgroup: the last whose first workgroup is not behind it
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.t[mid].first <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const Tensor& t = a.t[lo];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const bool whole = t.whole;
    const int64_t block0 = ((int64_t)(blockIdx.x - t.first) * 4 + wave) * a.span;
    for (uint32_t k = 0; k < a.span; ++k) {
        const int64_t block = block0 + k, e = block * BLOCK + 4 * lane;
        if (block * BLOCK >= t.n) return;
        const int left = t.n - e >= 4 ? 4 : t.n > e ? (int)(t.n - e) : 0;
        float p[4], g[4], m[4], v[4], q[4];
        load4(t.p + e, whole, left, p);
        load4(static_cast<const G*>(t.g) + e, whole, left, g);
        if constexpr (BITS == 32) {
            float* tm = static_cast<float*>(t.m);
            float* tv = static_cast<float*>(t.v);
            load4(tm + e, whole, left, m);
            load4(tv + e, whole, left, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                m[i] = __builtin_fmaf(a.beta1, m[i], a.omb1 * g[i]);
                v[i] = __builtin_fmaf(a.beta2, v[i], a.omb2 * (g[i] * g[i]));
            }
            store4(tm + e, whole, left, m);
            store4(tv + e, whole, left, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = (m[i] / a.bc1) / (sqrtf(v[i] / a.bc2) + a.eps);
        } else {
            uint8_t* tm = static_cast<uint8_t*>(t.m);
            uint8_t* tv = static_cast<uint8_t*>(t.v);
            float r[4], sm, sv;
            decode4(load4_codes(tm + e, whole, left), t.ms[block], m);
            decode4(load4_codes(tv + e, whole, left), t.vs[block], r);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                m[i] = m[i] * a.beta1 + g[i] * a.omb1;
                v[i] = (r[i] * r[i]) * a.beta2 + (g[i] * g[i]) * a.omb2;
                r[i] = sqrtf(v[i]);
                if (i >= left) m[i] = r[i] = 0.f;
                // the step itself to a few roundings: no code hangs on it
                q[i] = m[i] * a.rbc1 * __builtin_amdgcn_rcpf(__builtin_fmaf(r[i], a.rsbc2, a.eps));
            }
            store4_codes(tm + e, whole, left, encode4<false>(m, sm));
            store4_codes(tv + e, whole, left, encode4<true>(r, sv));
            if (lane == 0) {
                t.ms[block] = sm;
                t.vs[block] = sv;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = __builtin_fmaf(-t.lr, q[i], p[i] * t.keep);
        }
        store4(t.p + e, whole, left, p);
        if (t.copy) store4(static_cast<C*>(t.copy) + e, whole, left, p);
    }
}

template <typename G, typename C>
hipError_t launch_bits(int32_t bits, const AdamwArgs& k, unsigned grid, hipStream_t s)
{
    return launch(bits == 32 ? k_adamw<G, C, 32> : k_adamw<G, C, 8>, grid, 256, 0, s, k);
}

template <typename G>
hipError_t launch_copy(const es_adamw_args& a, const AdamwArgs& k, unsigned grid, hipStream_t s)
{
    return a.copy_dtype == ES_F16 ? launch_bits<G, _Float16>(a.state_bits, k, grid, s)
                                  : launch_bits<G, __bf16>(a.state_bits, k, grid, s);
}

hipError_t launch_types(const es_adamw_args& a, const AdamwArgs& k, unsigned grid, hipStream_t s)
{
    switch (a.g_dtype) {
    case ES_BF16: return launch_copy<__bf16>(a, k, grid, s);
    case ES_F16: return launch_copy<_Float16>(a, k, grid, s);
    default: return launch_copy<float>(a, k, grid, s);
    }
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// What is wrong with a tensor, or null.
const char* tensor_bad(const es_adamw_args& a, const es_adamw_tensor& t)
{
    const size_t ge = a.g_dtype == ES_F32 ? 4 : 2;
    if (t.n < 0 || t.n > MAX_N) return "n is out of range";
    if (!(t.lr >= 0.f) || !(t.lr < __builtin_inff())) return "lr must be finite and >= 0";
    if (!(t.weight_decay >= 0.f) || !(t.weight_decay < __builtin_inff())) return "weight_decay must be finite and >= 0";
    if (t.n == 0) return nullptr;
    if (!t.p || !t.g || !t.m || !t.v) return "null p, g, m or v";
    if (!aligned(t.p, 4) || !aligned(t.g, ge) || (t.copy && !aligned(t.copy, 2))) return "p, g or copy is not aligned to its type";
    if (a.state_bits == 32) {
        if (!aligned(t.m, 4) || !aligned(t.v, 4)) return "m or v is not aligned to its type";
    } else {
        if (!t.m_scale || !t.v_scale) return "null m_scale or v_scale";
        if (!aligned(t.m_scale, 4) || !aligned(t.v_scale, 4)) return "m_scale or v_scale is not aligned to its type";
    }
    return nullptr;
}

}  // namespace

}  // namespace esmi

using namespace esmi;

extern "C" es_status es_adamw(const es_adamw_args* a, const es_adamw_tensor* tensors, void* hip_stream)
{
    static const char* who = "es_adamw";
    if (!a || (a->count > 0 && !tensors)) return init_fail(ES_ERR_ARG, "null argument", who);
    if (a->count < 0) return init_fail(ES_ERR_ARG, "count is negative", who);
    if (a->g_dtype != ES_F32 && a->g_dtype != ES_BF16 && a->g_dtype != ES_F16)
        return init_fail(ES_ERR_ARG, "g_dtype is unknown", who);
    if (a->state_bits != 32 && a->state_bits != 8) return init_fail(ES_ERR_ARG, "state_bits must be 32 or 8", who);
    if (a->reserved) return init_fail(ES_ERR_ARG, "reserved is not 0", who);
    if (a->step < 1) return init_fail(ES_ERR_ARG, "step must be >= 1", who);
    if (!(a->beta1 >= 0.f && a->beta1 < 1.f) || !(a->beta2 >= 0.f && a->beta2 < 1.f))
        return init_fail(ES_ERR_ARG, "betas must be in [0, 1)", who);
    if (!(a->eps >= 0.f) || !(a->eps < __builtin_inff())) return init_fail(ES_ERR_ARG, "eps must be finite and >= 0", who);
    int64_t total = 0;
    for (int32_t i = 0; i < a->count; ++i) {
        const char* why = tensor_bad(*a, tensors[i]);
        if (!why && tensors[i].copy && a->copy_dtype != ES_BF16 && a->copy_dtype != ES_F16)
            why = "copy_dtype must be bf16 or fp16";
        if (why) {
            char msg[128];
            std::snprintf(msg, sizeof(msg), "tensor %d: %s", i, why);
            return init_fail(ES_ERR_ARG, msg, who);
        }
        total += (tensors[i].n + BLOCK - 1) / BLOCK;
    }
    AdamwArgs k{};
    const double t = (double)a->step;
    k.beta1 = a->beta1;
    k.beta2 = a->beta2;
    k.omb1 = (float)(1.0 - (double)a->beta1);
    k.omb2 = (float)(1.0 - (double)a->beta2);
    k.bc1 = (float)(1.0 - std::pow((double)a->beta1, t));
    k.bc2 = (float)(1.0 - std::pow((double)a->beta2, t));
    k.rbc1 = (float)(1.0 / (1.0 - std::pow((double)a->beta1, t)));
    k.rsbc2 = (float)(1.0 / std::sqrt(1.0 - std::pow((double)a->beta2, t)));
    // the 8-bit step multiplies by 1 / (root + eps), which for a root of 0 must be finite
    k.eps = a->state_bits == 8 && a->eps > 0.f ? std::fmax(a->eps, 0x1p-126f) : a->eps;
    k.span = total > (int64_t)1 << 16 ? LARGE_SPAN : 1;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    for (int32_t i = 0; i < a->count;) {
        uint64_t grid = 0;
        k.count = 0;
        for (; i < a->count && k.count < MAX_TENSORS; ++i) {
            const es_adamw_tensor& x = tensors[i];
            if (x.n == 0) continue;
            const uint64_t groups = ((uint64_t)(x.n + BLOCK - 1) / BLOCK + 4 * k.span - 1) / (4 * k.span);
            if (grid + groups > (uint64_t)MAX_GROUPS) break;  // at most MAX_N elements a tensor: never the first one
            const size_t ge = a->g_dtype == ES_F32 ? 16 : 8, se = a->state_bits == 32 ? 16 : 4;
            Tensor& d = k.t[k.count++];
            d = Tensor{x.p, x.g, x.m, x.v, x.m_scale, x.v_scale, x.copy, x.n, x.lr,
                       (float)(1.0 - (double)x.lr * (double)x.weight_decay), (uint32_t)grid,
                       aligned(x.p, 16) && aligned(x.g, ge) && aligned(x.m, se) && aligned(x.v, se) && aligned(x.copy, 8)};
            grid += groups;
        }
        if (k.count == 0) break;
        const hipError_t e = launch_types(*a, k, (unsigned)grid, s);
        if (e != hipSuccess) return init_fail(ES_ERR_HIP, hipGetErrorString(e), who);
    }
    return ES_OK;
}
