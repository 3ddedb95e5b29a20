// Dense attention, one wave a row (dense_row.h): the plain kernels that the tiled ones are checked against.
#include "dense_row.h"

namespace llsa {

// 4 rows a workgroup; row R of a group is query R / G of its head R % G
template <class T, int D> __global__ void __launch_bounds__(256) dense_fwd_rows_kernel(DenseArgs a, int64_t rows) {
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= rows) return;
    const DenseGroup p(a, blockIdx.y);
    const int i = (int)(r / a.G), g = (int)(r - (int64_t)i * a.G);
    dense_row_forward<T, D>(a, p, i, g, lane);
}

template <class T, int D> __global__ void __launch_bounds__(256) dense_dq_rows_kernel(DenseArgs a, int64_t rows) {
    using Row = LaneRow<T, D>;
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= rows) return;
    const DenseGroup p(a, blockIdx.y);
    const int i = (int)(r / a.G), g = (int)(r - (int64_t)i * a.G);
    const int64_t at = g * a.o.head + i * a.o.token;
    float delta = 0.f;
    if (p.seen(a, i) > 0) delta = Row::load(p.dO + at, lane).dot(Row::load(p.O + at, lane));
    if (lane == 0) a.nD[blockIdx.y * a.stat_rows + r] = -delta;
    dense_row_dq<T, D>(a, p, i, g, -delta, lane);
}

template <class T, int D> __global__ void __launch_bounds__(256) dense_dkv_rows_kernel(DenseArgs a, int64_t rows) {
    const int lane = threadIdx.x & 63;
    const int64_t j = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (j >= a.Nkv) return;
    const DenseGroup p(a, blockIdx.y);
    dense_row_dkv<T, D>(a, p, (int)j, a.nD + blockIdx.y * a.stat_rows, lane);
}

#define LLSA_DENSE_ROWS(kernel, count)                                                                             \
    const dim3 grid((unsigned)(((count) + 3) / 4), (unsigned)(p.desc.batch * p.desc.kv_heads));                     \
    return dense_dispatch(p, [&](auto t, auto d) {                                                                  \
        kernel<decltype(t), decltype(d)::value><<<grid, 256, 0, s>>>(a, p.rows);                                    \
        return hipGetLastError();                                                                                   \
    });

hipError_t launch_dense_fwd_rows(const DensePlan &p, const DenseArgs &a, hipStream_t s) { LLSA_DENSE_ROWS(dense_fwd_rows_kernel, p.rows) }
hipError_t launch_dense_dq_rows(const DensePlan &p, const DenseArgs &a, hipStream_t s) { LLSA_DENSE_ROWS(dense_dq_rows_kernel, p.rows) }
hipError_t launch_dense_dkv_rows(const DensePlan &p, const DenseArgs &a, hipStream_t s) { LLSA_DENSE_ROWS(dense_dkv_rows_kernel, p.desc.Nkv) }

}  // namespace llsa
