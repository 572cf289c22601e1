// es_dense.hpp -- what the layer kernels (es_dense.hip) and their entry points
// (es_layers.cpp) share.  Not part of the C-ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "esmi.h"

namespace esmi {

constexpr size_t WORKSPACE_ALIGN = 256;
constexpr size_t workspace_up(size_t n) { return (n + WORKSPACE_ALIGN - 1) / WORKSPACE_ALIGN * WORKSPACE_ALIGN; }
constexpr size_t dtype_size(int32_t t) { return t == ES_F32 ? 4 : 2; }
// Workgroups of a launch at most: HIP takes fewer than 2^32 work-items.  What has
// more goes in several launches of whole members; one member's work must fit.
constexpr int64_t launch_groups(int64_t threads) { return 0xFFFFFFFFll / threads; }

// One matrix product per batch, C[m][n] = sum over r < red and k < K of
// A(m, k) B(n, k), and what follows it.  An operand is "k-major" where its k
// index is the contiguous one (x and w of the forward), else its m (n) index
// is (w of dx; dz and x of dw).
struct Gemm {
    int32_t dtype;
    int32_t M, N, K;
    int64_t batches, red;
    const void *a, *b;
    int64_t a_batch, a_red, a_row;  // element strides; a_row between rows of the memory's matrix
    int64_t b_batch, b_red, b_row;
    bool a_kmajor, b_kmajor;
    // rows begin at multiples of 16 bytes and zeros follow them up to the next
    // one, readable memory in any case (16-bit types)
    bool a_padded, b_padded;
    // gated: N counts the outputs; B has 2 N rows, the gates' first
    bool gated;
    int32_t act;
    const void* bias;
    int64_t bias_batch;
    const void* res;
    int64_t res_batch, res_row;
    void* pre;
    int64_t pre_batch, pre_row;
    void* c;
    int64_t c_batch, c_row;
    int32_t c_dtype;
};

// Bytes that the product keeps between its launches: copies of operands in whole
// pieces, partial sums where its reduction is split (0: one launch).
size_t gemm_workspace(const Gemm& g);
// hipErrorInvalidValue where `bytes` is less than gemm_workspace gives
hipError_t launch_gemm(const Gemm& g, void* workspace, size_t bytes, hipStream_t s);
bool gemm_too_large(const Gemm& g);  // one member's product has more workgroups than a launch holds

// dz = dy act'(pre) (or both halves of a gated layer) in the type, rows of
// ldz elements, and the column sums of the unrounded dz per chunk of rows.
struct GradZ {
    int32_t dtype, act;
    bool gated;
    int64_t members;
    int32_t rows, out;  // out: columns of dy
    const void *dy, *pre;
    int64_t dy_member, dy_row, pre_member, pre_row;
    void* dz;  // null: not stored
    int64_t ldz;
    float* sums;  // [members][chunks][wide], null: not wanted
    void* db;     // with one chunk of rows a member: where its sums go instead, in the type; null: to sums
    int64_t db_member;
};
int64_t gradz_chunks(int64_t rows);
bool gradz_too_large(const GradZ& g);
hipError_t launch_gradz(const GradZ& g, hipStream_t s);
// db[n][o], n < groups, from [groups][count][wide] sums
bool bias_grad_too_large(int64_t count, int64_t wide);
hipError_t launch_bias_grad(int32_t dtype, const float* sums, int64_t groups, int64_t count, int64_t wide, void* db,
                            int64_t db_member, hipStream_t s);

}  // namespace esmi
