// Dense attention (llsa_dense_*): the host plan and what its kernels are given.
//
// The query heads that share a key head are taken together: row R of a group is query R / G of the group's head R % G (G heads a
// group).  A tile of rows then reads one set of keys whatever G is, the rows of a causal tile belong to neighbouring queries, one
// token of a group is one tile, and the key-major pass sums the heads of a group by walking its rows.
#pragma once
#include "llsa_internal.h"

namespace llsa {

struct DenseStrides { int64_t batch, head, token; };     // bytes

struct DensePlan {
    llsa_dense_desc desc;
    int elt, G;                     // bytes per element, query heads per key head
    int64_t rows;                   // rows of a group: G * Nq
    float scale;
    DenseStrides q, k, v, o;
    bool grads;                     // may gradients be written with the strides of Q, K and V?
    size_t D_off;                   // backward: D = rowsum(dO * O), [batch * kv_heads, rows] fp32, in the order of the rows
    size_t ws_fwd, ws_bwd;
};

struct DenseArgs {
    const char *Q, *K, *V, *O, *dO;
    char *out, *dQ, *dK, *dV;
    DenseStrides q, k, v, o;
    const int32_t *q_lens, *kv_lens;
    float *LSE, *D;
    int64_t Nq, Nkv;
    int32_t kv_heads, G, causal;
    FastDiv div_g;
    float scale, scale2;            // of the scores; times log2 e
};

// one wave a row (dense_row.hip)
hipError_t launch_dense_fwd_rows(const DensePlan &p, const DenseArgs &a, hipStream_t s);
hipError_t launch_dense_dq_rows(const DensePlan &p, const DenseArgs &a, hipStream_t s);      // and D
hipError_t launch_dense_dkv_rows(const DensePlan &p, const DenseArgs &a, hipStream_t s);

}  // namespace llsa
