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

// The forms of the tiled kernels: tiles of 128 rows (or keys) whose four waves have 32 each and walk over the other axis together; the same with eight waves, two for each 32, that
// share out every tile of the other axis; tiles of 32 whose four waves share out the other axis itself.
enum DenseForm { kDenseWide, kDensePaired, kDenseNarrow };

// How a launch cuts its axis (rows, or keys) and the other one that each tile of it walks over
struct DenseShape {
    bool narrow;                    // tiles of 32, whose four waves share out the other axis among themselves; else of 128, 32 a wave
    int splits;                     // workgroups that share out the other axis beyond that
    int chunk;                      // .. in pieces of this many of its tiles: a tile that sees less of it has fewer workgroups with something to do
};

struct DensePlan {
    llsa_dense_desc desc;
    int elt, G;                     // bytes per element, query heads per key head
    int64_t rows;                   // rows of a group: G * Nq
    float scale;
    DenseStrides q, k, v, o;
    bool grads;                     // may gradients be written with the strides of Q, K and V?
    DenseShape fwd, dq, dkv;
    int64_t stat_rows;              // rows, rounded up to whole tiles
    size_t nD_off, nlse_off;        // backward: -D = -rowsum(dO * O) and the logsumexp (DenseArgs::nlse) of the rows of a group, [batch * kv_heads, stat_rows] fp32
    size_t part_off;                // backward: partial sums of split tiles
    size_t ws_fwd, ws_bwd;
};

// A launch over tiles of rows (or keys) x groups x splits
struct DenseGrid {
    FastDiv by_tiles, by_splits, by_rest, by_heads;      // rest: groups x splits; heads: key heads x splits
    uint32_t wgs, groups;
    int32_t splits, chunk;
    int64_t rows;                   // rows (or keys) of a group
    float *part, *stat;             // [split][group][row][d] partial sums; [split][group][row][2] their references and sums
};

struct DenseArgs {
    const char *Q, *K, *V, *O, *dO;
    char *out, *dQ, *dK, *dV;
    DenseStrides q, k, v, o;
    const int32_t *q_lens, *kv_lens;
    float *LSE, *nD, *nlse;         // nlse: -LSE / scale (bf16) or -LSE log2 e (fp32)
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
constexpr int dense_tile(bool narrow) { return narrow ? 32 : 128; }                                       // of the launch's axis
constexpr int dense_step(int row_bytes, bool narrow) { return narrow || row_bytes > 256 ? 32 : 64; }      // of the other one
DenseShape dense_shape(const DensePlan &p, int64_t axis, int64_t other);
DenseGrid dense_grid(const DensePlan &p, int64_t rows, const DenseShape &shape, int row_floats, float *part);
size_t dense_part_bytes(const DensePlan &p, int64_t rows, const DenseShape &shape, int row_floats);

// tiles on the matrix instructions (dense_fwd.hip, dense_bwd.hip)
hipError_t launch_dense_fwd(const DensePlan &p, const DenseArgs &a, float *ws, hipStream_t s);
hipError_t launch_dense_bwd(const DensePlan &p, const DenseArgs &a, float *part, hipStream_t s);

// .. with the form that a launch takes
bool dense_paired(const DensePlan &p, const DenseShape &shape, int64_t axis);
template <class F> hipError_t dense_dispatch_form(const DensePlan &p, const DenseShape &shape, int64_t axis, F go) {
    return dense_dispatch(p, [&](auto t, auto d) {
        if (shape.narrow) return go(t, d, std::integral_constant<int, kDenseNarrow>());
        if constexpr (dense_step(decltype(d)::value * (int)sizeof(t), false) == 64)
            if (dense_paired(p, shape, axis)) return go(t, d, std::integral_constant<int, kDensePaired>());
        return go(t, d, std::integral_constant<int, kDenseWide>());
    });
}

// one wave a row (dense_row.hip)
hipError_t launch_dense_fwd_rows(const DensePlan &p, const DenseArgs &a, hipStream_t s);
hipError_t launch_dense_dq_rows(const DensePlan &p, const DenseArgs &a, hipStream_t s);      // and D
hipError_t launch_dense_dkv_rows(const DensePlan &p, const DenseArgs &a, hipStream_t s);

}  // namespace llsa
