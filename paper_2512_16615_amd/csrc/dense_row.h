// Dense attention for one row at a time: a wave, its lanes across the channels, fp32 arithmetic, keys one after the other.  Exact for every input
// the interface allows: what a query does not see is not even read.  The tiled kernels fall back on it where a masked place holds an
// infinity or a NaN, which a matrix instruction would multiply by 0 (NaN).
#pragma once
#include "dense.h"
#include "mfma_common.h"

namespace llsa {

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
    return x;
}

template <class T> __device__ __forceinline__ float dense_ld(const char *row, int c);
template <> __device__ __forceinline__ float dense_ld<float>(const char *row, int c) { return reinterpret_cast<const float *>(row)[c]; }
template <> __device__ __forceinline__ float dense_ld<__bf16>(const char *row, int c) { return (float)reinterpret_cast<const __bf16 *>(row)[c]; }
template <class T> __device__ __forceinline__ void dense_st(char *row, int c, float x) { reinterpret_cast<T *>(row)[c] = (T)x; }

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    return x;
}

// A row's channels across the wave: lane l has channel l and, at d = 128, l + 64; the lanes beyond d have zeros.
template <class T, int D> struct LaneRow {
    static constexpr int n = (D + 63) / 64;
    float x[n];
    __device__ __forceinline__ static LaneRow load(const char *row, int lane) {
        LaneRow r;
#pragma unroll
        for (int k = 0; k < n; ++k) r.x[k] = lane + 64 * k < D ? dense_ld<T>(row, lane + 64 * k) : 0.f;
        return r;
    }
    __device__ __forceinline__ static LaneRow zero() {
        LaneRow r;
#pragma unroll
        for (int k = 0; k < n; ++k) r.x[k] = 0.f;
        return r;
    }
    __device__ __forceinline__ void store(char *row, int lane) const {
#pragma unroll
        for (int k = 0; k < n; ++k)
            if (lane + 64 * k < D) dense_st<T>(row, lane + 64 * k, x[k]);
    }
    __device__ __forceinline__ void scale(float f) {
#pragma unroll
        for (int k = 0; k < n; ++k) x[k] *= f;
    }
    __device__ __forceinline__ void add(float f, const LaneRow &o) {
#pragma unroll
        for (int k = 0; k < n; ++k) x[k] = fmaf(f, o.x[k], x[k]);
    }
    // += f[s] times d partial sums, s = 0 .. n - 1 in order, `stride` floats apart; f[s] is lane s's.  Sixteen of them on their way at once, or eight (few rows over a long axis wait
    // for nothing else: 16 x 5 rows over 19042 keys in 32 pieces, d = 128: a step 189 -> 185 us).
    template <int P> __device__ __forceinline__ void add_some(const float *part, int64_t stride, int s, int n, float f, int lane) {
        float v[P][LaneRow::n];
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int k = 0; k < LaneRow::n; ++k) v[i][k] = lane + 64 * k < D ? part[min(s + i, n - 1) * stride + lane + 64 * k] : 0.f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (s + i >= n) break;
            const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), s + i));
#pragma unroll
            for (int k = 0; k < LaneRow::n; ++k) x[k] = fmaf(w, v[i][k], x[k]);
        }
    }
    __device__ __forceinline__ void add_parts(const float *part, int64_t stride, int n, float f, int lane) {
        int s = 0;
        for (; n - s > 8; s += 16) add_some<16>(part, stride, s, n, f, lane);
        if (s < n) add_some<8>(part, stride, s, n, f, lane);
    }
    // in every lane of the wave
    __device__ __forceinline__ bool finite() const {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < n; ++k) s = fmaf(x[k], 0.f, s);
        return __builtin_amdgcn_ballot_w64(s != 0.f) == 0;
    }
    __device__ __forceinline__ float dot(const LaneRow &o) const {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < n; ++k) s = fmaf(x[k], o.x[k], s);
        return wave_sum(s);
    }
};

// one group (batch entry and key head) of the problem
struct DenseGroup {
    const char *Q, *K, *V, *O, *dO;
    char *out, *dQ, *dK, *dV;
    float *LSE;                     // of the group's first head
    int nq, nk;                     // lengths
    __device__ __forceinline__ DenseGroup(const DenseArgs &a, int group) {
        const int b = group / a.kv_heads, h = group - b * a.kv_heads;
        const int64_t oq = b * a.q.batch + (int64_t)h * a.G * a.q.head, oo = b * a.o.batch + (int64_t)h * a.G * a.o.head;
        const int64_t ok = b * a.k.batch + h * a.k.head, ov = b * a.v.batch + h * a.v.head;
        Q = a.Q + oq;
        K = a.K + ok;
        V = a.V + ov;
        O = a.O + oo;
        dO = a.dO + oo;
        out = a.out + oo;
        dQ = a.dQ + oq;
        dK = a.dK + ok;
        dV = a.dV + ov;
        LSE = a.LSE + ((int64_t)b * a.kv_heads + h) * a.G * a.Nq;
        nq = a.q_lens ? max(0, min(a.q_lens[b], (int)a.Nq)) : (int)a.Nq;
        nk = a.kv_lens ? max(0, min(a.kv_lens[b], (int)a.Nkv)) : (int)a.Nkv;
    }
    // keys that query i sees: 0 .. seen(i) - 1
    __device__ __forceinline__ int seen(const DenseArgs &a, int i) const {
        return i >= nq ? 0 : a.causal ? max(0, min(nk, i + nk - nq + 1)) : nk;
    }
    // first query that sees key j (nq: none does)
    __device__ __forceinline__ int first_query(const DenseArgs &a, int j) const { return j >= nk ? nq : a.causal ? min(nq, max(0, j - nk + nq)) : 0; }
};

// Keys of a row seen by the rows first .. last of a group
struct KeySpan { int all, some; };                          // keys that every one of them sees; that one of them sees
__device__ __forceinline__ KeySpan key_span(const DenseArgs &a, const DenseGroup &p, int64_t first, int64_t last) {
    const int i0 = (int)min(first, (int64_t)0x7fffffff), i1 = (int)min(last, (int64_t)0x7fffffff);
    const int q0 = (int)a.div_g(i0), q1 = min((int)a.div_g(i1), p.nq - 1);
    if (q0 >= p.nq) return {0, 0};
    return {p.seen(a, q0), p.seen(a, q1)};
}

// The tiles of the other axis that a workgroup has: piece `split` of its tile's `tiles`, which begin at `first`.  One piece at least: `alone`, its sums are the result.
struct DensePieces {
    int t0, t1;
    bool alone, none;
    __device__ __forceinline__ DensePieces(const DenseGrid &g, int split, int first, int tiles) {
        t0 = first + split * g.chunk;
        t1 = min(first + tiles, t0 + g.chunk);
        alone = tiles <= g.chunk;
        none = split > 0 && t0 >= t1;
    }
};
// .. of a tile of rows, and of a tile of keys
template <int AXIS, int STEP> __device__ __forceinline__ int dense_key_steps(const DenseArgs &a, const DenseGroup &p, int64_t row0) {
    return (key_span(a, p, row0, row0 + AXIS - 1).some + STEP - 1) / STEP;
}
template <int STEP> __device__ __forceinline__ int dense_row_steps(const DenseArgs &a, const DenseGroup &p, int key0, int *first) {
    *first = p.first_query(a, key0) * a.G / STEP;
    return max(0, (p.nq * a.G + STEP - 1) / STEP - *first);
}

// Which rows and keys a workgroup has.  Causal: the tiles with the most work first (the last
// rows, the first keys), of all groups in turn; otherwise the tiles of a group next to each
// other and the groups in stretches, so that the workgroups of one XCD share their keys.
struct DenseWork { int group, split, tile; };
// Causal sequences of different lengths: the tiles by the work they have, which is what they are from their sequence's end (keys) or beginning (rows).  Of tile level l = 1, 2, ..
// every sequence of at least l tiles has one; those behind a length come last.  Where there are three workgroups a CU: below that about all are resident at once, in whatever
// order (2 x 16 heads of 4096 and 1024 tokens, d = 128: forward 116 -> 94 us, backward 371 -> 309; 8 x 16 heads of 50 to 1000, d = 64: backward 68 -> 64; 756 workgroups of 3 x 16 heads, 4 key heads, of
// 1999, 1500 and 700, d = 128: 50.0 -> 50.2 and 197 -> 199).
constexpr int kDenseSorted = 8;                              // sequences that are sorted
template <int AXIS, bool ROWS> __device__ __forceinline__ DenseWork dense_sorted_work(const DenseArgs &a, const DenseGrid &g, int batch) {
    const unsigned heads = g.by_heads.d, tiles = g.by_tiles.d;
    const int32_t *lens = ROWS ? a.q_lens : a.kv_lens;
    const int N = (int)(ROWS ? a.Nq : a.Nkv);
    unsigned n[kDenseSorted], all = 0;
#pragma unroll
    for (int b = 0; b < kDenseSorted; ++b) {
        const int len = b < batch ? max(0, min(lens[min(b, batch - 1)], N)) : 0;
        n[b] = (unsigned)(((int64_t)len * (ROWS ? a.G : 1) + AXIS - 1) / AXIS);
        all += n[b];
    }
    all *= heads;
    const unsigned id = blockIdx.x;
    unsigned rest;
    int batch_entry = 0, tile = 0;
    if (id < all) {
        auto above = [&](unsigned level) {
            unsigned c = 0;
#pragma unroll
            for (int b = 0; b < kDenseSorted; ++b) c += n[b] > level ? n[b] - level : 0;
            return c * heads;
        };
        unsigned lo = 1, hi = tiles;                         // the first level with at most id tiles above it
        while (lo < hi) {
            const unsigned mid = (lo + hi) / 2;
            if (above(mid) <= id) hi = mid;
            else lo = mid + 1;
        }
        rest = id - above(lo);
        unsigned k = g.by_heads(rest);
        rest -= k * heads;
#pragma unroll
        for (int b = 0; b < kDenseSorted; ++b)
            if (n[b] >= lo && k-- == 0) {
                batch_entry = b;
                tile = (int)(ROWS ? lo - 1 : n[b] - lo);
            }
    } else {
        rest = id - all;
        bool found = false;
#pragma unroll
        for (int b = 0; b < kDenseSorted; ++b) {
            const unsigned c = (tiles - n[b]) * heads;
            if (found || b >= batch) continue;
            if (rest < c) {
                const unsigned k = g.by_heads(rest);
                batch_entry = b;
                tile = (int)(n[b] + k);
                rest -= k * heads;
                found = true;
            } else {
                rest -= c;
            }
        }
    }
    const unsigned head = g.by_splits(rest);
    return {__builtin_amdgcn_readfirstlane(batch_entry * a.kv_heads + (int)head), __builtin_amdgcn_readfirstlane((int)(rest - head * g.by_splits.d)),
            __builtin_amdgcn_readfirstlane(tile)};
}
template <int AXIS, bool ROWS> __device__ __forceinline__ DenseWork dense_work(const DenseArgs &a, const DenseGrid &g) {
    if (a.causal) {
        if (gridDim.x >= 768 && (ROWS ? a.q_lens : a.kv_lens)) {
            const int batch = (int)g.groups / a.kv_heads;
            if (batch > 1 && batch <= kDenseSorted) return dense_sorted_work<AXIS, ROWS>(a, g, batch);
        }
        const unsigned t = g.by_rest(blockIdx.x), rest = blockIdx.x - t * g.by_rest.d;
        const unsigned group = g.by_splits(rest);
        return {(int)group, (int)(rest - group * g.by_splits.d), (int)(ROWS ? g.by_tiles.d - 1 - t : t)};
    }
    const unsigned w = xcd_contiguous32(blockIdx.x, gridDim.x), rest = g.by_tiles(w), group = g.by_splits(rest);
    return {(int)group, (int)(rest - group * g.by_splits.d), (int)(w - rest * g.by_tiles.d)};
}

template <class T, int D> __device__ __forceinline__ void dense_row_forward(const DenseArgs &a, const DenseGroup &p, int i, int g, int lane) {
    using Row = LaneRow<T, D>;
    const Row q = Row::load(p.Q + g * a.q.head + i * a.q.token, lane);
    const int n = p.seen(a, i);
    Row acc = Row::zero();
    float m = -INFINITY, l = 0.f;
    for (int j = 0; j < n; ++j) {
        const float s = q.dot(Row::load(p.K + j * a.k.token, lane)) * a.scale;
        const float m2 = fmaxf(m, s);
        if (m2 > m) {                                        // the sums so far, relative to the new maximum
            const float f = __expf(m - m2);
            l *= f;
            acc.scale(f);
            m = m2;
        }
        const float e = s == -INFINITY && m == -INFINITY ? 0.f : __expf(s - m);
        l += e;
        acc.add(e, Row::load(p.V + j * a.v.token, lane));
    }
    if (n > 0) acc.scale(1.f / l);
    acc.store(p.out + g * a.o.head + i * a.o.token, lane);
    if (lane == 0) p.LSE[(int64_t)g * a.Nq + i] = n > 0 ? m + __logf(l) : -INFINITY;
}

// nD: minus D of the row
template <class T, int D> __device__ __forceinline__ void dense_row_dq(const DenseArgs &a, const DenseGroup &p, int i, int g, float nD, int lane) {
    using Row = LaneRow<T, D>;
    Row acc = Row::zero();
    const int n = p.seen(a, i);
    if (n > 0) {
        const Row q = Row::load(p.Q + g * a.q.head + i * a.q.token, lane), go = Row::load(p.dO + g * a.o.head + i * a.o.token, lane);
        const float lse = p.LSE[(int64_t)g * a.Nq + i];
        for (int j = 0; j < n; ++j) {
            const Row k = Row::load(p.K + j * a.k.token, lane);
            const float e = __expf(q.dot(k) * a.scale - lse);
            acc.add(e * (go.dot(Row::load(p.V + j * a.v.token, lane)) + nD), k);
        }
        acc.scale(a.scale);
    }
    acc.store(p.dQ + g * a.q.head + i * a.q.token, lane);
}

// nD: minus D of the group's rows (row i * G + g)
template <class T, int D> __device__ __forceinline__ void dense_row_dkv(const DenseArgs &a, const DenseGroup &p, int j, const float *nD, int lane) {
    using Row = LaneRow<T, D>;
    Row dk = Row::zero(), dv = Row::zero();
    const int first = p.first_query(a, j);
    if (first < p.nq) {
        const Row k = Row::load(p.K + j * a.k.token, lane), v = Row::load(p.V + j * a.v.token, lane);
        for (int i = first; i < p.nq; ++i)
            for (int g = 0; g < a.G; ++g) {
                const Row q = Row::load(p.Q + g * a.q.head + i * a.q.token, lane), go = Row::load(p.dO + g * a.o.head + i * a.o.token, lane);
                const float e = __expf(q.dot(k) * a.scale - p.LSE[(int64_t)g * a.Nq + i]);
                dv.add(e, go);
                dk.add(e * (go.dot(v) + nD[(int64_t)i * a.G + g]), q);
            }
        dk.scale(a.scale);
    }
    dk.store(p.dK + j * a.k.token, lane);
    dv.store(p.dV + j * a.v.token, lane);
}

}  // namespace llsa
