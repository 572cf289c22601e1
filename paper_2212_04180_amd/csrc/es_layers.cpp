// es_layers.cpp -- entry points of the layer operators (es_dense, es_gated and
// their gradients): argument checks, the split into matrix products, and the
// workspace's layout.  The kernels are in es_dense.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdio>

#include "es_dense.hpp"
#include "es_internal.hpp"
#include "esmi.h"

using namespace esmi;

namespace {

constexpr int64_t kMaxDim = 0x7FFFFFFF;
// Rows of all members taken as one product: as many as any launch holds (2^23 tiles of 128)
constexpr int64_t kMaxMerged = 1 << 30;
constexpr size_t kAlign = WORKSPACE_ALIGN;

size_t up(size_t n) { return workspace_up(n); }

bool dtype_ok(int32_t t) { return t == ES_F32 || t == ES_BF16 || t == ES_F16; }

// Arguments of one call, both directions, and what is wrong with them.
struct Check {
    const char* who;
    int64_t members, rows;
    char msg[200] = {0};

    bool bad(const char* what, const char* why)
    {
        std::snprintf(msg, sizeof(msg), "%s %s", what, why);
        return true;
    }
    // A matrix of `rows` x `cols` per member; `elem` bytes an element.
    bool matrix(const char* name, const es_matrix& m, int64_t r, int64_t cols, size_t elem, bool needed, bool output,
                bool may_sum = false)
    {
        // a sum over the members is written also where there are none
        const int64_t members = may_sum && m.member == 0 ? 1 : this->members;
        if (members == 0 || r == 0 || cols == 0) return false;  // no element is touched
        if (!m.p) return needed ? bad(name, "is missing") : false;
        if (reinterpret_cast<uintptr_t>(m.p) % elem) return bad(name, "is not aligned to its type");
        if (m.member < 0 || m.row < 0) return bad(name, "has a negative stride");
        const __int128 last = (__int128)(members - 1) * m.member + (__int128)(r - 1) * m.row + cols;
        if (last > ((__int128)1 << 58)) return bad(name, "reaches beyond the address space");
        if (!output) return false;
        if (r > 1 && m.row < cols) return bad(name, "has rows that overlap");
        if (members > 1) {
            // members behind each other, or interleaved within the rows
            const bool apart = (__int128)m.member >= (__int128)(r - 1) * m.row + cols;
            const bool within = m.member >= cols && (r == 1 || (__int128)m.row >= (__int128)(members - 1) * m.member + cols);
            if (!apart && !within) return bad(name, "has members that overlap");
        }
        return false;
    }
    bool dims(int64_t in, int64_t out, int64_t wide)
    {
        if (members < 0 || rows < 0 || in < 0 || out < 0) return bad("a size", "is negative");
        if (members > kMaxDim || rows > kMaxDim || in > kMaxDim || wide > kMaxDim) return bad("a size", "exceeds 2^31 - 1");
        return false;
    }
};

es_status refuse(const Check& c) { return init_fail(ES_ERR_ARG, c.msg, c.who); }

// ---- forward --------------------------------------------------------------
bool forward_bad(const es_dense_args& a, bool gated, Check& c)
{
    const int64_t wide = gated ? 2 * a.out : a.out;
    if (!dtype_ok(a.dtype)) return c.bad("dtype", "is unknown");
    if (a.y_dtype != a.dtype && a.y_dtype != ES_F32) return c.bad("y_dtype", "is neither dtype nor fp32");
    if (a.act < ES_ACT_NONE || a.act > ES_ACT_SILU) return c.bad("act", "is unknown");
    if (a.reserved) return c.bad("reserved", "is not 0");
    if (c.dims(a.in, a.out, wide)) return true;
    const size_t e = dtype_size(a.dtype), ey = dtype_size(a.y_dtype);
    if (gated && a.residual.p) return c.bad("residual", "is not taken by a gated layer");
    if (a.rows > 0 && (c.matrix("w", a.w, wide, a.in, e, true, false) || c.matrix("bias", a.bias, 1, wide, e, false, false)))
        return true;
    return (a.out > 0 && c.matrix("x", a.x, a.rows, a.in, e, true, false)) ||
           c.matrix("residual", a.residual, a.rows, a.out, e, false, false) ||
           c.matrix("y", a.y, a.rows, a.out, ey, true, true) || c.matrix("pre", a.pre, a.rows, wide, e, false, true);
}

Gemm forward_gemm(const es_dense_args& a, bool gated)
{
    Gemm g{};
    g.dtype = a.dtype;
    g.M = (int32_t)a.rows;
    g.N = (int32_t)a.out;
    g.K = (int32_t)a.in;
    g.batches = a.members;
    g.red = 1;
    g.a = a.x.p; g.a_batch = a.x.member; g.a_row = a.x.row; g.a_kmajor = true;
    g.b = a.w.p; g.b_batch = a.w.member; g.b_row = a.w.row; g.b_kmajor = true;
    g.gated = gated;
    g.act = a.act;
    g.bias = a.bias.p; g.bias_batch = a.bias.member;
    g.res = a.residual.p; g.res_batch = a.residual.member; g.res_row = a.residual.row;
    g.pre = a.pre.p; g.pre_batch = a.pre.member; g.pre_row = a.pre.row;
    g.c = a.y.p; g.c_batch = a.y.member; g.c_row = a.y.row; g.c_dtype = a.y_dtype;
    // one network on all members' rows is one product where the rows follow each other
    const int64_t B = a.rows, n = a.members;
    if (n > 1 && B * n <= kMaxMerged && a.w.member == 0 && (!a.bias.p || a.bias.member == 0) && a.x.member == B * a.x.row &&
        a.y.member == B * a.y.row && (!a.residual.p || a.residual.member == B * a.residual.row) &&
        (!a.pre.p || a.pre.member == B * a.pre.row)) {
        g.M = (int32_t)(B * n);
        g.batches = 1;
    }
    return g;
}

es_status forward(const es_dense_args* a, bool gated, const char* who, void* ws, size_t bytes, void* stream, size_t* need)
{
    if (!a || (!need && bytes && !ws)) return init_fail(ES_ERR_ARG, "null argument", who);
    Check c{who, a->members, a->rows};
    if (forward_bad(*a, gated, c)) return refuse(c);
    const Gemm g = forward_gemm(*a, gated);
    const bool empty = g.batches == 0 || g.M == 0 || g.N == 0;
    if (!empty && gemm_too_large(g)) return init_fail(ES_ERR_UNSUPPORTED, "more workgroups than a launch holds", who);
    const size_t want = empty ? 0 : gemm_workspace(g);
    if (need) {
        *need = want;
        return ES_OK;
    }
    if (bytes < want) return init_fail(ES_ERR_ARG, "the workspace is too small", who);
    if (want && reinterpret_cast<uintptr_t>(ws) % kAlign) return init_fail(ES_ERR_ARG, "the workspace is not aligned", who);
    if (empty) return ES_OK;
    const hipError_t e = launch_gemm(g, ws, bytes, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ES_OK : init_fail(ES_ERR_HIP, hipGetErrorString(e), who);
}

// ---- backward -------------------------------------------------------------
bool backward_bad(const es_dense_grad_args& a, bool gated, Check& c)
{
    const int64_t wide = gated ? 2 * a.out : a.out;
    if (!dtype_ok(a.dtype)) return c.bad("dtype", "is unknown");
    if (a.act < ES_ACT_NONE || a.act > ES_ACT_SILU) return c.bad("act", "is unknown");
    if (c.dims(a.in, a.out, wide)) return true;
    const size_t e = dtype_size(a.dtype);
    const bool uses_pre = gated || a.act != ES_ACT_NONE;
    if (a.in > 0 || a.db.p) {
        if (c.matrix("dy", a.dy, a.rows, a.out, e, true, false)) return true;
        if (uses_pre && c.matrix("pre", a.pre, a.rows, wide, e, true, false)) return true;
    }
    return (a.dw.p && a.out > 0 && c.matrix("x", a.x, a.rows, a.in, e, true, false)) ||
           (a.dx.p && a.rows > 0 && c.matrix("w", a.w, wide, a.in, e, true, false)) ||
           c.matrix("dx", a.dx, a.rows, a.in, e, false, true, true) ||
           c.matrix("dw", a.dw, wide, a.in, e, false, true, true) || c.matrix("db", a.db, 1, wide, e, false, true, true);
}

struct BackwardPlan {
    GradZ z;
    Gemm dx, dw;
    bool do_dx, do_dw, do_db, store_dz;
    bool db_there;  // each db is one chunk's sums: no second launch
    int64_t wide, chunks;
    size_t dz_bytes, sums_bytes, partial_bytes;
    size_t total() const { return dz_bytes + sums_bytes + partial_bytes; }
};

BackwardPlan plan_backward(const es_dense_grad_args& a, bool gated)
{
    BackwardPlan p{};
    const size_t e = dtype_size(a.dtype);
    const int64_t B = a.rows, n = a.members, wide = gated ? 2 * a.out : a.out;
    p.wide = wide;
    const bool sum_dx = n != 1 && a.dx.member == 0, sum_dw = n != 1 && a.dw.member == 0, sum_db = n != 1 && a.db.member == 0;
    p.do_dx = a.dx.p && (n || sum_dx) && B && a.in;
    p.do_dw = a.dw.p && (n || sum_dw) && wide && a.in;
    p.do_db = a.db.p && (n || sum_db) && wide;
    p.store_dz = (p.do_dx || p.do_dw) && (gated || a.act != ES_ACT_NONE) && B && wide;
    p.chunks = gradz_chunks(B);
    const int64_t ldz = (wide + 7) / 8 * 8;  // whole 16-byte pieces in every type
    p.dz_bytes = p.store_dz ? up((size_t)n * B * ldz * e) : 0;
    p.db_there = p.do_db && p.chunks == 1 && !sum_db;
    p.sums_bytes = p.do_db && !p.db_there ? up((size_t)n * p.chunks * wide * 4) : 0;
    p.z.dtype = a.dtype; p.z.act = a.act; p.z.gated = gated;
    p.z.members = n; p.z.rows = (int32_t)B; p.z.out = (int32_t)a.out;
    p.z.dy = a.dy.p; p.z.dy_member = a.dy.member; p.z.dy_row = a.dy.row;
    p.z.pre = a.pre.p; p.z.pre_member = a.pre.member; p.z.pre_row = a.pre.row;
    p.z.ldz = ldz;
    const int64_t z_row = p.store_dz ? ldz : a.dy.row, z_member = p.store_dz ? B * ldz : a.dy.member;

    // The plans (and so the workspace) go by addresses: dz will start the workspace.
    const void* z = p.store_dz ? reinterpret_cast<const void*>(kAlign) : a.dy.p;
    Gemm g{};
    g.dtype = g.c_dtype = a.dtype;
    g.act = ES_ACT_NONE;
    // dx[i][k] = sum_o dz[i][o] w[o][k]
    p.dx = g;
    p.dx.M = (int32_t)B; p.dx.N = (int32_t)a.in; p.dx.K = (int32_t)wide;
    p.dx.a = z; p.dx.a_row = z_row; p.dx.a_kmajor = true; p.dx.a_padded = p.store_dz;
    p.dx.b = a.w.p; p.dx.b_row = a.w.row; p.dx.b_kmajor = false;
    p.dx.c = a.dx.p; p.dx.c_row = a.dx.row; p.dx.c_batch = a.dx.member;
    if (sum_dx) {
        p.dx.batches = 1; p.dx.red = n; p.dx.a_red = z_member; p.dx.b_red = a.w.member;
    } else {
        p.dx.batches = n; p.dx.red = 1; p.dx.a_batch = z_member; p.dx.b_batch = a.w.member;
        if (n > 1 && B * n <= kMaxMerged && a.w.member == 0 && z_member == B * z_row && a.dx.member == B * a.dx.row) {
            p.dx.M = (int32_t)(B * n);
            p.dx.batches = 1;
        }
    }
    // dw[o][k] = sum_i dz[i][o] x[i][k]
    p.dw = g;
    p.dw.M = (int32_t)wide; p.dw.N = (int32_t)a.in; p.dw.K = (int32_t)B;
    p.dw.a = z; p.dw.a_row = z_row; p.dw.a_kmajor = false; p.dw.a_padded = p.store_dz;
    p.dw.b = a.x.p; p.dw.b_row = a.x.row; p.dw.b_kmajor = false;
    p.dw.c = a.dw.p; p.dw.c_row = a.dw.row; p.dw.c_batch = a.dw.member;
    if (sum_dw) {
        p.dw.batches = 1; p.dw.red = n; p.dw.a_red = z_member; p.dw.b_red = a.x.member;
        if (B * n <= kMaxDim && z_member == B * z_row && a.x.member == B * a.x.row) {
            p.dw.K = (int32_t)(B * n);
            p.dw.red = 1;
        }
    } else {
        p.dw.batches = n; p.dw.red = 1; p.dw.a_batch = z_member; p.dw.b_batch = a.x.member;
    }
    size_t f = 0;
    if (p.do_dx) f = std::max(f, gemm_workspace(p.dx));
    if (p.do_dw) f = std::max(f, gemm_workspace(p.dw));
    p.partial_bytes = f;
    return p;
}

es_status backward(const es_dense_grad_args* a, bool gated, const char* who, void* ws, size_t bytes, void* stream,
                   size_t* need)
{
    if (!a || (!need && bytes && !ws)) return init_fail(ES_ERR_ARG, "null argument", who);
    Check c{who, a->members, a->rows};
    if (backward_bad(*a, gated, c)) return refuse(c);
    BackwardPlan p = plan_backward(*a, gated);
    const bool sum_db = a->members != 1 && a->db.member == 0;
    const int64_t db_count = sum_db ? a->members * p.chunks : p.chunks;
    if ((p.do_dx && gemm_too_large(p.dx)) || (p.do_dw && gemm_too_large(p.dw)) ||
        ((p.store_dz || p.do_db) && gradz_too_large(p.z)) || (p.do_db && !p.db_there && bias_grad_too_large(db_count, p.wide)))
        return init_fail(ES_ERR_UNSUPPORTED, "more workgroups than a launch holds", who);
    const size_t want = p.total();
    if (need) {
        *need = want;
        return ES_OK;
    }
    if (bytes < want) return init_fail(ES_ERR_ARG, "the workspace is too small", who);
    if (want && reinterpret_cast<uintptr_t>(ws) % kAlign) return init_fail(ES_ERR_ARG, "the workspace is not aligned", who);
    char* at = static_cast<char*>(ws);
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    float* sums = p.do_db && !p.db_there ? reinterpret_cast<float*>(at + p.dz_bytes) : nullptr;
    void* partial = at + p.dz_bytes + p.sums_bytes;
    if (p.store_dz || p.do_db) {
        p.z.dz = p.store_dz ? at : nullptr;
        p.z.sums = sums;
        if (p.db_there) {
            p.z.db = a->db.p;
            p.z.db_member = a->db.member;
        }
        e = launch_gradz(p.z, s);
        if (p.store_dz) p.dx.a = p.dw.a = at;
    }
    if (e == hipSuccess && p.do_db && !p.db_there) {
        e = launch_bias_grad(a->dtype, sums, sum_db ? 1 : a->members, db_count, p.wide, a->db.p, a->db.member, s);
    }
    if (e == hipSuccess && p.do_dx) e = launch_gemm(p.dx, partial, p.partial_bytes, s);
    if (e == hipSuccess && p.do_dw) e = launch_gemm(p.dw, partial, p.partial_bytes, s);
    return e == hipSuccess ? ES_OK : init_fail(ES_ERR_HIP, hipGetErrorString(e), who);
}

}  // namespace

extern "C" {

es_status es_dense_workspace(const es_dense_args* a, size_t* bytes)
{
    if (!bytes) return init_fail(ES_ERR_ARG, "null argument", "es_dense_workspace");
    return forward(a, false, "es_dense_workspace", nullptr, 0, nullptr, bytes);
}

es_status es_dense(const es_dense_args* a, void* workspace, size_t bytes, void* hip_stream)
{
    return forward(a, false, "es_dense", workspace, bytes, hip_stream, nullptr);
}

es_status es_dense_backward_workspace(const es_dense_grad_args* a, size_t* bytes)
{
    if (!bytes) return init_fail(ES_ERR_ARG, "null argument", "es_dense_backward_workspace");
    return backward(a, false, "es_dense_backward_workspace", nullptr, 0, nullptr, bytes);
}

es_status es_dense_backward(const es_dense_grad_args* a, void* workspace, size_t bytes, void* hip_stream)
{
    return backward(a, false, "es_dense_backward", workspace, bytes, hip_stream, nullptr);
}

es_status es_gated_workspace(const es_dense_args* a, size_t* bytes)
{
    if (!bytes) return init_fail(ES_ERR_ARG, "null argument", "es_gated_workspace");
    return forward(a, true, "es_gated_workspace", nullptr, 0, nullptr, bytes);
}

es_status es_gated(const es_dense_args* a, void* workspace, size_t bytes, void* hip_stream)
{
    return forward(a, true, "es_gated", workspace, bytes, hip_stream, nullptr);
}

es_status es_gated_backward_workspace(const es_dense_grad_args* a, size_t* bytes)
{
    if (!bytes) return init_fail(ES_ERR_ARG, "null argument", "es_gated_backward_workspace");
    return backward(a, true, "es_gated_backward_workspace", nullptr, 0, nullptr, bytes);
}

es_status es_gated_backward(const es_dense_grad_args* a, void* workspace, size_t bytes, void* hip_stream)
{
    return backward(a, true, "es_gated_backward", workspace, bytes, hip_stream, nullptr);
}

}  // extern "C"
