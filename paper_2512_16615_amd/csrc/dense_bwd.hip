// Dense attention, backward, in two launches that recompute the probabilities from the logsumexp and write each result once (no atomics, so the
// same bits from call to call; S and dP are formed twice, 14 d operations a pair of a query and a key where 10 d would do):
//   query-major: dQ = scale dS K, and D = rowsum(dO O), which the other one needs;   key-major: dV = P^T dO, dK = scale dS^T Q
// with P = exp(S - LSE), dS = P (dO V^T - D).  -LSE / scale and -D are where the first products' sums begin, so P = exp2(scale2 S') and dS = P dP'.
// P and dS enter the second products rounded to the I/O type (bf16: half a step, 2^-8, of each; sums are fp32).
#include "dense_row.h"
#include "dense_tile.h"

namespace llsa {

template <class T, int D> constexpr int bwd_waves() { return D * (int)sizeof(T) <= 256 ? 2 : 1; }

template <class T, int D, int KT>
__global__ void __launch_bounds__(256, (bwd_waves<T, D>())) dense_dq_kernel(DenseArgs a, DenseGrid grid) {
    using Tile = DenseTile<T, D>;
    using Loads = TileLoads<T, D, KT, 4>;
    constexpr int TILEB = KT * Tile::ROWB, SUBS = KT / 32;
    __shared__ __attribute__((aligned(1024))) char lds[2][2][TILEB];      // stage; keys, values
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, col = lane & 31;
    const DenseWork work = dense_work(grid, a.causal, true);
    const DenseGroup p(a, work.group);
    const Tile tile(lane);
    const int64_t row0 = (int64_t)work.tile * 128, wrow0 = row0 + wave * 32, r = wrow0 + col;
    const int end = key_span(a, p, row0, row0 + 127).some;
    const KeySpan mine = key_span(a, p, wrow0, wrow0 + 31);

    const bool in = r < grid.rows;
    const int qi = (int)a.div_g((uint32_t)(in ? r : 0)), qg = (int)((in ? r : 0) - (int64_t)qi * a.G), seen = in ? p.seen(a, qi) : 0;
    const int64_t at_q = qg * a.q.head + (int64_t)qi * a.q.token, at_o = qg * a.o.head + (int64_t)qi * a.o.token;
    Piece<T> q[Tile::KS], g[Tile::KS];
    float delta = 0.f;
#pragma unroll
    for (int ks = 0; ks < Tile::KS; ++ks) {
        const u32x4 zero = {0, 0, 0, 0};
        q[ks].w = seen > 0 ? *reinterpret_cast<const u32x4 *>(p.Q + at_q + 16 * h + 32 * ks) : zero;
        g[ks].w = seen > 0 ? *reinterpret_cast<const u32x4 *>(p.dO + at_o + 16 * h + 32 * ks) : zero;
        const Piece<T> o = {seen > 0 ? *reinterpret_cast<const u32x4 *>(p.O + at_o + 16 * h + 32 * ks) : zero};
        delta = piece_dot(g[ks], o, delta);
    }
    const float nD = -half_sum(delta), nlse = seen > 0 ? -p.LSE[(int64_t)qg * a.Nq + qi] / a.scale : -INFINITY;
    if (work.split == 0 && h == 0) {                         // also for the rows that the last tile has too many
        a.nD[work.group * a.stat_rows + r] = nD;
        a.nlse[work.group * a.stat_rows + r] = nlse;
    }
    f32x16 s_from, dp_from, dq[Tile::NB];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        s_from[e] = nlse;
        dp_from[e] = nD;
#pragma unroll
        for (int n = 0; n < Tile::NB; ++n) dq[n][e] = 0.f;
    }

    const int tiles = (end + KT - 1) / KT, per = (tiles + grid.splits - 1) / grid.splits;
    const int t0 = work.split * per, t1 = min(tiles, t0 + per);
    auto fetch = [&](int t) {
        const int k0 = t * KT, left = min(KT, p.nk - k0);
        const unsigned lds0 = lds_address(&lds[t & 1][0][0]);
        const unsigned kt = (unsigned)a.k.token, vt = (unsigned)a.v.token;
        Loads::keys(buffer_of(p.K + k0 * a.k.token, (left - 1) * kt + Tile::ROWB), kt, lds0, wave, lane);
        Loads::keys(buffer_of(p.V + k0 * a.v.token, (left - 1) * vt + Tile::ROWB), vt, lds0 + TILEB, wave, lane);
    };
    if (t0 < t1) fetch(t0);
    for (int t = t0; t < t1; ++t) {
        vm_wait_barrier<0>();                                // tile t is there, and nobody reads the other stage
        if (t + 1 < t1) fetch(t + 1);
        const int k0 = t * KT;
        if (k0 >= mine.some) continue;
        const char *kt = &lds[t & 1][0][0], *vt = &lds[t & 1][1][0];
#pragma unroll
        for (int u = 0; u < SUBS; ++u) {
            f32x16 s = s_from, dp = dp_from;
#pragma unroll
            for (int ks = 0; ks < Tile::KS; ++ks) s = piece_product(tile.row(kt, u, ks), q[ks], s);
#pragma unroll
            for (int ks = 0; ks < Tile::KS; ++ks) dp = piece_product(tile.row(vt, u, ks), g[ks], dp);
#pragma unroll
            for (int e = 0; e < 16; ++e) dp[e] *= __builtin_amdgcn_exp2f(s[e] * a.scale2);
            if (k0 + 32 * u + 32 > mine.all) {
                const int lim = seen - k0 - 32 * u - 4 * h;
#pragma unroll
                for (int e = 0; e < 16; ++e) dp[e] = 8 * (e >> 2) + (e & 3) < lim ? dp[e] : 0.f;
            }
            Probs<T> ds;
            ds.set(dp);
#pragma unroll
            for (int n = 0; n < Tile::NB; ++n) dq[n] = tile.col_product(kt, u, n, ds, dq[n]);
        }
    }

    if (grid.splits > 1) {
        if (in) store_partial<D>(grid.part + (((int64_t)work.split * grid.groups + work.group) * grid.rows + r) * D, dq, h);
        return;
    }
    keep_rows(dq, seen > 0);
    uint64_t redo = 0;
    if (a.causal) {                                          // a key that some row of the tile does not see may have met it as 0 times an infinity
        redo = not_finite(dq) & __builtin_amdgcn_ballot_w64(seen > 0);
        redo = (redo | redo >> 32) & 0xffffffffu;
    }
    store_rows<T, D>(p.dQ + at_q, dq, a.scale, h, in);
    while (redo) {
        const int i = __builtin_ctzll(redo);
        redo &= redo - 1;
        dense_row_dq<T, D>(a, p, __builtin_amdgcn_readlane(qi, i), __builtin_amdgcn_readlane(qg, i), __int_as_float(__builtin_amdgcn_readlane(__float_as_int(nD), i)), lane);
    }
}

// A wave has 32 keys, theirs and their values' channels in registers, and walks over the rows (of every head that shares them) in tiles of QT.
template <class T, int D, int QT>
__global__ void __launch_bounds__(256, (bwd_waves<T, D>())) dense_dkv_kernel(DenseArgs a, DenseGrid grid) {
    using Tile = DenseTile<T, D>;
    using Loads = TileLoads<T, D, QT, 4>;
    constexpr int TILEB = QT * Tile::ROWB, SUBS = QT / 32;
    __shared__ __attribute__((aligned(1024))) char lds[2][2][TILEB];      // stage; queries, their output's gradients
    __shared__ __attribute__((aligned(1024))) float stat[2][2][64];       // stage; -LSE / scale, -D
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, col = lane & 31;
    const DenseWork work = dense_work(grid, a.causal, false);
    const DenseGroup p(a, work.group);
    const Tile tile(lane);
    const int key0 = work.tile * 128, wkey0 = key0 + wave * 32, j = wkey0 + col;
    const bool valid = j < p.nk;

    Piece<T> k[Tile::KS], v[Tile::KS];
#pragma unroll
    for (int ks = 0; ks < Tile::KS; ++ks) {
        const u32x4 zero = {0, 0, 0, 0};
        k[ks].w = valid ? *reinterpret_cast<const u32x4 *>(p.K + j * a.k.token + 16 * h + 32 * ks) : zero;
        v[ks].w = valid ? *reinterpret_cast<const u32x4 *>(p.V + j * a.v.token + 16 * h + 32 * ks) : zero;
    }
    f32x16 dk[Tile::NB], dv[Tile::NB];
#pragma unroll
    for (int n = 0; n < Tile::NB; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) dk[n][e] = dv[n][e] = 0.f;

    const int rows = p.nq * a.G;                             // rows that see something: of each key, those from its first query's on
    const int from = p.first_query(a, j) * a.G;
    const int wfrom = p.first_query(a, wkey0) * a.G, wto = p.first_query(a, min(wkey0 + 31, max(p.nk - 1, 0))) * a.G;
    const int first = p.first_query(a, key0) * a.G / QT, tiles = max(0, (rows + QT - 1) / QT - first), per = (tiles + grid.splits - 1) / grid.splits;
    const int t0 = first + work.split * per, t1 = min(first + tiles, t0 + per);
    const float *nlse = a.nlse + work.group * a.stat_rows, *nD = a.nD + work.group * a.stat_rows;
    auto fetch = [&](int t) {
        const int r0 = t * QT, q0 = (int)a.div_g(r0);
        const unsigned lds0 = lds_address(&lds[t & 1][0][0]), st0 = lds_address(&stat[t & 1][0][0]);
        Loads::rows(buffer_of(p.Q + (int64_t)q0 * a.q.token, 0xffffff00u), buffer_of(p.dO + (int64_t)q0 * a.o.token, 0xffffff00u), a, r0, q0, rows, lds0, lds0 + TILEB, wave, lane);
        const float *src = wave == 0 ? nlse : nD;
        if (wave < 2) buffer_to_lds_dword(buffer_of(reinterpret_cast<const char *>(src + r0), (unsigned)min((int64_t)64, a.stat_rows - r0) * 4), lane * 4, st0 + wave * 256);
    };
    if (t0 < t1) fetch(t0);
    for (int t = t0; t < t1; ++t) {
        vm_wait_barrier<0>();                                // tile t is there, and nobody reads the other stage
        if (t + 1 < t1) fetch(t + 1);
        const char *qt = &lds[t & 1][0][0], *gt = &lds[t & 1][1][0];
        const float *st = &stat[t & 1][0][0];
#pragma unroll
        for (int u = 0; u < SUBS; ++u) {
            const int r0 = t * QT + 32 * u;
            if (r0 + 31 < wfrom) continue;
            f32x16 s, dp;
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const f32x4 x = *reinterpret_cast<const f32x4 *>(st + 32 * u + 2 * e + 4 * h), y = *reinterpret_cast<const f32x4 *>(st + 64 + 32 * u + 2 * e + 4 * h);
#pragma unroll
                for (int i = 0; i < 4; ++i) { s[e + i] = x[i]; dp[e + i] = y[i]; }
            }
#pragma unroll
            for (int ks = 0; ks < Tile::KS; ++ks) s = piece_product(tile.row(qt, u, ks), k[ks], s);
#pragma unroll
            for (int ks = 0; ks < Tile::KS; ++ks) dp = piece_product(tile.row(gt, u, ks), v[ks], dp);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[e] = __builtin_amdgcn_exp2f(s[e] * a.scale2);
                dp[e] *= s[e];
            }
            if (r0 < wto) {
                const int lim = from - r0 - 4 * h;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const bool sees = 8 * (e >> 2) + (e & 3) >= lim;
                    s[e] = sees ? s[e] : 0.f;
                    dp[e] = sees ? dp[e] : 0.f;
                }
            }
            Probs<T> pr, ds;
            pr.set(s);
            ds.set(dp);
#pragma unroll
            for (int n = 0; n < Tile::NB; ++n) dv[n] = tile.col_product(gt, u, n, pr, dv[n]);
#pragma unroll
            for (int n = 0; n < Tile::NB; ++n) dk[n] = tile.col_product(qt, u, n, ds, dk[n]);
        }
    }

    if (grid.splits > 1) {
        float *to = grid.part + (((int64_t)work.split * grid.groups + work.group) * grid.rows + j) * (2 * D);
        if (j < grid.rows) {
            store_partial<D>(to, dk, h);
            store_partial<D>(to + D, dv, h);
        }
        return;
    }
    uint64_t redo = 0;
    if (a.causal) {                                          // a row that does not see some key of the tile may have met it as 0 times an infinity
        redo = (not_finite(dk) | not_finite(dv)) & __builtin_amdgcn_ballot_w64(valid);
        redo = (redo | redo >> 32) & 0xffffffffu;
    }
    keep_rows(dk, valid);
    keep_rows(dv, valid);
    store_rows<T, D>(p.dK + j * a.k.token, dk, a.scale, h, j < grid.rows);
    store_rows<T, D>(p.dV + j * a.v.token, dv, 1.f, h, j < grid.rows);
    while (redo) {
        const int i = __builtin_ctzll(redo);
        redo &= redo - 1;
        dense_row_dkv<T, D>(a, p, wkey0 + i, nD, lane);
    }
}

// The splits' sums of a row in order, one wave a row.
template <class T, int D> __global__ void __launch_bounds__(256) dense_dq_join_kernel(DenseArgs a, DenseGrid grid) {
    using Row = LaneRow<T, D>;
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= grid.rows) return;
    const DenseGroup p(a, blockIdx.y);
    const int i = (int)a.div_g((uint32_t)r), g = (int)(r - (int64_t)i * a.G);
    Row acc = Row::zero();
    if (p.seen(a, i) > 0)
        for (int s = 0; s < grid.splits; ++s) acc.add_part(grid.part + (((int64_t)s * grid.groups + blockIdx.y) * grid.rows + r) * D, 1.f, lane);
    acc.scale(a.scale);
    if (a.causal && !acc.finite()) dense_row_dq<T, D>(a, p, i, g, a.nD[blockIdx.y * a.stat_rows + r], lane);
    else acc.store(p.dQ + g * a.q.head + i * a.q.token, lane);
}

template <class T, int D> __global__ void __launch_bounds__(256) dense_dkv_join_kernel(DenseArgs a, DenseGrid grid) {
    using Row = LaneRow<T, D>;
    const int lane = threadIdx.x & 63;
    const int64_t j = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (j >= grid.rows) return;
    const DenseGroup p(a, blockIdx.y);
    Row dk = Row::zero(), dv = Row::zero();
    if (j < p.nk) {
        for (int s = 0; s < grid.splits; ++s) {
            const float *at = grid.part + (((int64_t)s * grid.groups + blockIdx.y) * grid.rows + j) * (2 * D);
            dk.add_part(at, 1.f, lane);
            dv.add_part(at + D, 1.f, lane);
        }
        dk.scale(a.scale);
        if (a.causal && !(dk.finite() && dv.finite())) {
            dense_row_dkv<T, D>(a, p, (int)j, a.nD + blockIdx.y * a.stat_rows, lane);
            return;
        }
    }
    dk.store(p.dK + j * a.k.token, lane);
    dv.store(p.dV + j * a.v.token, lane);
}

// Two workgroups a CU's worth of tiles need no splitting; fewer share out the other axis, at least 4 tiles of 64 each.
static int bwd_splits(const DensePlan &p, int64_t axis, int64_t other) {
    const int64_t base = (int64_t)p.desc.batch * p.desc.kv_heads * ((axis + 127) / 128), tiles = (other + 63) / 64;
    if (base >= 256) return 1;
    const int64_t want = (512 + base - 1) / base, most = tiles / 4;
    return (int)(most < 2 ? 1 : want < most ? want : most);
}
int dense_dq_splits(const DensePlan &p) { return bwd_splits(p, p.rows, p.desc.Nkv); }
int dense_dkv_splits(const DensePlan &p) { return bwd_splits(p, p.desc.Nkv, p.rows); }

template <class T, int D> static hipError_t launch_bwd(const DensePlan &p, const DenseArgs &a, float *part, hipStream_t s) {
    constexpr int KT = DenseTile<T, D>::ROWB > 256 ? 32 : 64;
    const DenseGrid gq = dense_grid(p, p.rows, 128, p.dq_splits, D, part);
    dense_dq_kernel<T, D, KT><<<gq.wgs, 256, 0, s>>>(a, gq);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && gq.splits > 1) {
        dense_dq_join_kernel<T, D><<<dim3((unsigned)((gq.rows + 3) / 4), gq.groups), 256, 0, s>>>(a, gq);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    const DenseGrid gk = dense_grid(p, p.desc.Nkv, 128, p.dkv_splits, 2 * D, part);
    dense_dkv_kernel<T, D, KT><<<gk.wgs, 256, 0, s>>>(a, gk);
    e = hipGetLastError();
    if (e == hipSuccess && gk.splits > 1) {
        dense_dkv_join_kernel<T, D><<<dim3((unsigned)((gk.rows + 3) / 4), gk.groups), 256, 0, s>>>(a, gk);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_dense_bwd(const DensePlan &p, const DenseArgs &a, float *part, hipStream_t s) {
    return dense_dispatch(p, [&](auto t, auto d) { return launch_bwd<decltype(t), decltype(d)::value>(p, a, part, s); });
}

}  // namespace llsa
