// Dense attention, forward: workgroups of 4 waves, 32 rows each (a row: a query of one of the heads that share a key head), keys and values in
// tiles of KT through LDS, the running maximum and sum of a softmax in registers.  A lane has one row: its scores come out of the first product in the
// registers that the second one takes, O^T = V^T P^T collects channels in the registers of the same lane, so maximum, sum and rescaling are
// the lane's own (and its partner's in the other half of the wave).
//
// 4 d operations a pair of a query and a key: 16 heads x 16384 tokens, d = 64, 1115 to 1190 us (960 TFLOP/s), where the softmax (an exponential a pair and some five other vector instructions) takes the
// issue slots that the matrix unit does not; 4 heads x 32768, d = 128, 1.94 ms (1130 TFLOP/s; a large library product reaches 1336, clocks under that load included).  One token of 32 heads over 8 key
// heads, 8 sequences of 500 to 16384, d = 128: 60 us and 6 for the join, 5.0 TB/s of the keys that are there.
#include "dense_row.h"
#include "dense_tile.h"

#include <type_traits>

namespace llsa {

// Waves a SIMD that the registers are shared out for.  Four at 128 bytes a row (three spilled registers and a wave more: 16 x 16384 tokens, d = 64, 1134 -> 1104 us;
// 16 x 4096, causal, 57.3 -> 58.3).
template <class T, int D, int FORM> constexpr int fwd_waves() { return D * (int)sizeof(T) <= 128 && FORM == kDenseWide ? 4 : D * (int)sizeof(T) <= 256 ? 2 : 1; }

// Narrow: each wave has every fourth tile of keys, in stages of its own.  Paired: the first or second half of every tile.  The waves' sums are added up at the end.
template <class T, int D, int KT, int FORM>
__global__ void __launch_bounds__(FORM == kDensePaired ? 512 : 256, (fwd_waves<T, D, FORM>())) dense_fwd_kernel(DenseArgs a, DenseGrid grid) {
    constexpr bool NARROW = FORM == kDenseNarrow, PAIRED = FORM == kDensePaired;
    using Tile = DenseTile<T, D>;
    using Loads = TileLoads<T, D, KT, NARROW ? 1 : PAIRED ? 8 : 4>;
    constexpr int TILEB = KT * Tile::ROWB, SUBS = PAIRED ? 1 : KT / 32, AXIS = dense_tile(NARROW), WAVES = NARROW ? 4 : 1, KS = Tile::KS, NB = Tile::NB;
    constexpr int ST = dense_stages<T, D, FORM>();
    constexpr int LDSB = WAVES * ST * 2 * TILEB, JOINB = NARROW ? 12288 * NB + 2048 : PAIRED ? 16384 * NB + 4096 : 0;
    __shared__ __attribute__((aligned(1024))) char lds[LDSB > JOINB ? LDSB : JOINB];      // wave; stage; keys, values
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, col = lane & 31;
    const int pair = wave & 3, half = wave >> 2;
    const DenseWork work = dense_work<AXIS, true>(a, grid);
    const DenseGroup p(a, work.group);
    const Tile tile(lane);
    const int64_t row0 = (int64_t)work.tile * AXIS, wrow0 = NARROW ? row0 : row0 + pair * 32, r = wrow0 + col;
    // The wave's rows as operands.  All rows are read, those behind the length too, so that they are on their way before the lengths are there:
    // what such a row holds stays in its own lane.
    const bool in = r < grid.rows;
    const int qi = (int)a.div_g((uint32_t)(in ? r : 0)), qg = (int)((in ? r : 0) - (int64_t)qi * a.G);
    Piece<T> q[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[ks].w = *reinterpret_cast<const u32x4 *>(p.Q + qg * a.q.head + qi * a.q.token + 16 * h + 32 * ks);
    const DensePieces piece(grid, work.split, 0, dense_key_steps<AXIS, KT>(a, p, row0));
    if (piece.none) return;
    const KeySpan mine = key_span(a, p, wrow0, wrow0 + 31);
    const int seen = in ? p.seen(a, qi) : 0;

    f32x16 o[NB];
    float m = -3e38f, l = 0.f;                               // the reference that the exponentials are relative to (log2), their sum in this lane
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[n][e] = 0.f;

    char *const ring = lds + (NARROW ? wave * (ST * 2 * TILEB) : 0);
    const unsigned ring0 = lds_address(ring);
    const int t0 = piece.t0 + (NARROW ? wave : 0);
    auto stage = [&](int t) { return ST == 1 ? 0 : ((t - t0) / WAVES & 1) * 2 * TILEB; };
    auto fetch = [&](int t) {
        const int k0 = t * KT, left = min(KT, p.nk - k0);
        const unsigned kt = (unsigned)a.k.token, vt = (unsigned)a.v.token, to = ring0 + stage(t);
        Loads::keys(buffer_of(p.K + k0 * a.k.token, (left - 1) * kt + Tile::ROWB), kt, to, NARROW ? 0 : wave, lane);
        Loads::keys(buffer_of(p.V + k0 * a.v.token, (left - 1) * vt + Tile::ROWB), vt, to + TILEB, NARROW ? 0 : wave, lane);
    };
    if (ST == 2 && t0 < piece.t1) fetch(t0);
    loads_done();
    for (int t = t0; t < piece.t1; t += WAVES) {
        if (ST == 1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            fetch(t);
        }
        if (NARROW) vm_wait<0>();                            // tile t is there (and nobody else reads the wave's stages),
        else vm_wait_barrier<0>();                           // for all waves, and nobody reads the other stage
        if (ST == 2 && t + WAVES < piece.t1) fetch(t + WAVES);
        const int k0 = t * KT + (PAIRED ? half * 32 : 0);
        if (k0 >= mine.some) continue;
        const char *kt = ring, *vt = ring + TILEB;
        const Tile at = tile.at(stage(t) + (PAIRED ? half * 32 * Tile::ROWB : 0));
        f32x16 s[SUBS];
#pragma unroll
        for (int u = 0; u < SUBS; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[u][e] = 0.f;

        // between the two products
        auto softmax = [&]() {
            if (k0 + 32 * SUBS > mine.all) {                        // a key that some row does not see
                const int lim = seen - k0 - 4 * h;
#pragma unroll
                for (int u = 0; u < SUBS; ++u)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[u][e] = 32 * u + 8 * (e >> 2) + (e & 3) < lim ? s[u][e] : -INFINITY;
            }
            float mx = s[0][0];
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[u][e]);
            mx = half_max(mx) * a.scale2;
            // The reference follows the maximum only once that is 2^8 beyond it (the sums stay far from fp32's range), for all rows of the wave
            // at once: after the first tiles the accumulators are hardly ever rescaled.
            if (__builtin_amdgcn_ballot_w64(mx > m + 8.f)) {
                const float m2 = fmaxf(m, mx), f = __builtin_amdgcn_exp2f(m - m2);
                m = m2;
                l *= f;
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[n][e] *= f;
            }
        };
        auto take_exp = [&](int u, int first, int count) {
#pragma unroll
            for (int e = first; e < first + count; ++e) {
                s[u][e] = __builtin_amdgcn_exp2f(fmaf(s[u][e], a.scale2, -m));
                l += s[u][e];
            }
        };
        if constexpr (sizeof(T) == 2) {
            constexpr int N1 = SUBS * KS, N2 = N1 + SUBS * 2 * NB;
            auto op = operands<N2, 4>([&](auto ic) {
                constexpr int i = decltype(ic)::value, j = i - N1;
                if constexpr (i < N1) return __builtin_bit_cast(bf16x8, at.row(kt, i / KS, i % KS).w);
                else return at.col(vt, j / (2 * NB), j % NB, j / NB % 2);
            });
            constants<N1>([&](auto i) { op.take(i, [&](bf16x8 x) { s[i / KS] = mfma32(x, __builtin_bit_cast(bf16x8, q[i % KS].w), s[i / KS]); }); });
            softmax();
            take_exp(0, 0, 16);
            bf16x8 pr[2] = {round8(s[0], 0), round8(s[0], 1)};
            constants<SUBS * 2 * NB>([&](auto i) {           // the first 32 keys' products while the other ones' exponentials are taken
                constexpr int u = i / (2 * NB), k = i % (2 * NB);
                if constexpr (u > 0 && k == 0) { pr[0] = round8(s[u], 0); pr[1] = round8(s[u], 1); }
                op.take(plus(i, std::integral_constant<int, N1>()), [&](bf16x8 x) { o[k % NB] = mfma32(x, pr[k / NB], o[k % NB]); });
                if constexpr (u + 1 < SUBS) take_exp(u + 1, k * (8 / NB), 8 / NB);
            });
        } else {
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) s[u] = piece_product(at.row(kt, u, ks), q[ks], s[u]);
            softmax();
#pragma unroll
            for (int u = 0; u < SUBS; ++u) {
                take_exp(u, 0, 16);
#pragma unroll
                for (int n = 0; n < NB; ++n) o[n] = at.col_product(vt, u, n, s[u], o[n]);
            }
        }
    }

    if constexpr (FORM != kDenseWide) {                      // each wave's exponentials are relative to its own reference
        constexpr int N = NARROW ? 4 : 2, STEP = NARROW ? 1 : 4, ALL = NARROW ? 4 : 8;     // waves of a row, from one to the next; of the workgroup
        __syncthreads();
        float *ml = reinterpret_cast<float *>(lds + (NARROW ? 12288 : 16384) * NB);
        ml[wave * 64 + lane] = m;
        ml[(ALL + wave) * 64 + lane] = l;
        __syncthreads();
        const int first = NARROW ? 0 : pair;
        float top = m, sum = 0.f;
#pragma unroll
        for (int w = 0; w < N; ++w) top = fmaxf(top, ml[(first + w * STEP) * 64 + lane]);
#pragma unroll
        for (int w = 0; w < N; ++w) sum = fmaf(ml[(ALL + first + w * STEP) * 64 + lane], __builtin_amdgcn_exp2f(ml[(first + w * STEP) * 64 + lane] - top), sum);
        const float f = __builtin_amdgcn_exp2f(m - top);
        if (NARROW) add_waves(o, f, lds, wave, lane);
        else add_halves(o, f, lds, pair, half, lane);
        if (NARROW ? wave > 0 : half > 0) return;
        m = top;
        l = sum;
    }
    const float sum = half_sum(l);
    if (!piece.alone) {
        const int64_t to = ((int64_t)work.split * grid.groups + work.group) * grid.rows + r;
        if (in) {
            store_partial<D>(grid.part + to * D, o, h);
            if (h == 0) *reinterpret_cast<float2 *>(grid.stat + 2 * to) = make_float2(m, sum);
        }
        return;
    }
    const bool any = seen > 0;
    const float f = any ? 1.f / sum : 0.f;
    keep_rows(o, any);
    uint64_t redo = 0;
    if (a.causal) {                                          // a key that some row of the tile does not see may have met it as 0 times an infinity
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[n][e] *= f;
        redo = not_finite(o) & __builtin_amdgcn_ballot_w64(any);
        redo = (redo | redo >> 32) & 0xffffffffu;
    }
    store_rows<T, D>(p.out + qg * a.o.head + qi * a.o.token, o, a.causal ? 1.f : f, h, in);
    if (h == 0 && in) p.LSE[(int64_t)qg * a.Nq + qi] = any ? (m + __log2f(sum)) * kLn2 : -INFINITY;
    while (redo) {
        const int i = __builtin_ctzll(redo);
        redo &= redo - 1;
        dense_row_forward<T, D>(a, p, __builtin_amdgcn_readlane(qi, i), __builtin_amdgcn_readlane(qg, i), lane);
    }
}

// The pieces' partial sums of a row, one wave a row: the exponentials of each are relative to its own reference.
template <class T, int D, int AXIS, int KT> __global__ void __launch_bounds__(256) dense_join_kernel(DenseArgs a, DenseGrid grid) {
    using Row = LaneRow<T, D>;
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= grid.rows) return;
    const DenseGroup p(a, blockIdx.y);
    const int i = (int)a.div_g((uint32_t)r), g = (int)(r - (int64_t)i * a.G);
    char *dst = p.out + g * a.o.head + i * a.o.token;
    const int steps = dense_key_steps<AXIS, KT>(a, p, r / AXIS * AXIS), pieces = (steps + grid.chunk - 1) / grid.chunk;
    if (pieces <= 1) return;                                 // the forward launch's result already
    const bool any = p.seen(a, i) > 0;
    const int64_t at = (int64_t)blockIdx.y * grid.rows + r, step = (int64_t)grid.groups * grid.rows;     // piece 0's sums; from piece to piece
    float m = -3e38f, l = 0.f;
    for (int s = lane; s < pieces; s += 64) m = fmaxf(m, grid.stat[2 * (at + s * step)]);
    m = wave_max(m);
    Row acc = Row::zero();
    for (int s0 = 0; s0 < pieces; s0 += 64) {
        const int s = s0 + lane;
        const float2 st = s < pieces ? *reinterpret_cast<const float2 *>(grid.stat + 2 * (at + s * step)) : make_float2(-3e38f, 0.f);
        const float f = s < pieces ? __builtin_amdgcn_exp2f(st.x - m) : 0.f;
        l += wave_sum(f * st.y);
        acc.add_parts(grid.part + (at + s0 * step) * D, step * D, min(64, pieces - s0), f, lane);
    }
    if (any) acc.scale(1.f / l);
    else acc = Row::zero();
    if (a.causal && any && !acc.finite()) {
        dense_row_forward<T, D>(a, p, i, g, lane);
        return;
    }
    acc.store(dst, lane);
    if (lane == 0) p.LSE[(int64_t)g * a.Nq + i] = any ? (m + __log2f(l)) * kLn2 : -INFINITY;
}

template <class T, int D, int FORM> static hipError_t launch_fwd(const DensePlan &p, const DenseArgs &a, float *ws, hipStream_t s) {
    constexpr bool NARROW = FORM == kDenseNarrow;
    constexpr int KT = dense_step(DenseTile<T, D>::ROWB, NARROW);
    const DenseGrid g = dense_grid(p, p.rows, p.fwd, D, ws);
    dense_fwd_kernel<T, D, KT, FORM><<<g.wgs, FORM == kDensePaired ? 512 : 256, 0, s>>>(a, g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || g.splits == 1) return e;
    dense_join_kernel<T, D, dense_tile(NARROW), KT><<<dim3((unsigned)((p.rows + 3) / 4), g.groups), 256, 0, s>>>(a, g);
    return hipGetLastError();
}

hipError_t launch_dense_fwd(const DensePlan &p, const DenseArgs &a, float *ws, hipStream_t s) {
    return dense_dispatch_form(p, p.fwd, p.rows, [&](auto t, auto d, auto form) { return launch_fwd<decltype(t), decltype(d)::value, decltype(form)::value>(p, a, ws, s); });
}

}  // namespace llsa
