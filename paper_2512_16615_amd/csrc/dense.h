// Dense attention (llsa_dense_*): the host plan and what its kernels are given.
//
// The query heads that share a key head are taken together: row R of a group is query R / G of the group's head R % G (G heads a
// group).  A tile of rows then reads one set of keys whatever G is, the rows of a causal tile belong to neighbouring queries, one
// token of a group is one tile, and the key-major pass sums the heads of a group by walking its rows.
#pragma once
#include <type_traits>

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
    int fwd_splits, dq_splits, dkv_splits;     // workgroups that share out the other axis of a tile of rows or keys
    int64_t stat_rows;              // rows, rounded up to whole tiles
    size_t nD_off, nlse_off;        // backward: -D = -rowsum(dO * O) and -LSE / scale of the rows of a group, [batch * kv_heads, stat_rows] fp32
    size_t part_off;                // backward: partial sums of split tiles
    size_t ws_fwd, ws_bwd;
};

// A launch over tiles of rows (or keys) x groups x splits
struct DenseGrid {
    FastDiv by_tiles, by_splits, by_rest;      // rest: groups x splits
    uint32_t wgs, groups;
    int32_t splits;
    int64_t rows;                   // rows (or keys) of a group
    float *part, *stat;             // [split][group][row][d] partial sums; [split][group][row][2] their references and sums
};

struct DenseArgs {
    const char *Q, *K, *V, *O, *dO;
    char *out, *dQ, *dK, *dV;
    DenseStrides q, k, v, o;
    const int32_t *q_lens, *kv_lens;
    float *LSE, *nD, *nlse;
    int64_t stat_rows;
    int64_t Nq, Nkv;
    int32_t kv_heads, G, causal;
    FastDiv div_g;
    float scale, scale2;            // of the scores; times log2 e
};

template <class F> auto dense_dispatch(const DensePlan &p, F go) {
    auto by_d = [&](auto t) {
        switch (p.desc.d) {
            case 16: return go(t, std::integral_constant<int, 16>());
            case 32: return go(t, std::integral_constant<int, 32>());
            case 64: return go(t, std::integral_constant<int, 64>());
            default: return go(t, std::integral_constant<int, 128>());
        }
    };
    return p.elt == 4 ? by_d(float()) : by_d(__bf16());
}
DenseGrid dense_grid(const DensePlan &p, int64_t rows, int tile, int splits, int row_floats, float *part);
size_t dense_part_bytes(const DensePlan &p, int64_t rows, int splits, int row_floats);

// tiles on the matrix instructions (dense_fwd.hip, dense_bwd.hip)
int dense_fwd_splits(const DensePlan &p);
hipError_t launch_dense_fwd(const DensePlan &p, const DenseArgs &a, float *ws, hipStream_t s);
int dense_dq_splits(const DensePlan &p);
int dense_dkv_splits(const DensePlan &p);
hipError_t launch_dense_bwd(const DensePlan &p, const DenseArgs &a, float *part, hipStream_t s);

// one wave a row (dense_row.hip)
hipError_t launch_dense_fwd_rows(const DensePlan &p, const DenseArgs &a, hipStream_t s);
hipError_t launch_dense_dq_rows(const DensePlan &p, const DenseArgs &a, hipStream_t s);      // and D
hipError_t launch_dense_dkv_rows(const DensePlan &p, const DenseArgs &a, hipStream_t s);

}  // namespace llsa
