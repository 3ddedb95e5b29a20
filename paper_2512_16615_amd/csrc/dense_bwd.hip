// Dense attention, backward, in two launches that recompute the probabilities from the logsumexp and write each result once (no atomics, so the
// same bits from call to call; S and dP are formed twice, 14 d operations a pair of a query and a key where 10 d would do):
//   query-major: dQ = scale dS K, and D = rowsum(dO O), which the other one needs;   key-major: dV = P^T dO, dK = scale dS^T Q
// with P = exp(S - LSE), dS = P (dO V^T - D).  -LSE / scale and -D are where the first products' sums begin, so P = exp2(scale2 S') and dS = P dP'.  In fp32 S begins
// at 0 and LSE is subtracted where the exponential is taken: LSE / scale is some 100, whose last bit is more than S's own error.
// P and dS enter the second products rounded to the I/O type (bf16: half a step, 2^-8, of each; sums are fp32).
//
// 16 heads x 16384 tokens, d = 64: dQ 1.41 to 1.51 ms, dK and dV 1.96 to 2.0 (1100 TFLOP/s of the 14 d); 16 x 8192, d = 128: 1.67 ms in all (1150).  Bound by the matrix units and, between their
// instructions, by the vector ones of P and dS.
#include "dense_row.h"
#include "dense_tile.h"

namespace llsa {

// Waves a SIMD that the registers are shared out for (the key-major sums of a narrow workgroup take more than half of a CU's LDS at d = 128; three at
// 128 bytes a row: 16 x 16384 tokens, d = 64, backward 3450 -> 3340 us)
template <class T, int D, int FORM> constexpr int dq_waves() { return D * (int)sizeof(T) <= 256 || FORM == kDensePaired ? 2 : 1; }
template <class T, int D, int FORM> constexpr int dkv_waves() {
    return D * (int)sizeof(T) <= 128 && FORM == kDenseWide ? 3 : D * (int)sizeof(T) <= 256 && !(FORM == kDenseNarrow && D == 128) ? 2 : 1;
}

// Narrow: each wave has every fourth tile of keys, in stages of its own.  Paired: the first or second half of every tile.  The waves' sums are added up at the end.
template <class T, int D, int KT, int FORM>
__global__ void __launch_bounds__(FORM == kDensePaired ? 512 : 256, (dq_waves<T, D, FORM>())) dense_dq_kernel(DenseArgs a, DenseGrid grid) {
    constexpr bool NARROW = FORM == kDenseNarrow, PAIRED = FORM == kDensePaired;
    using Tile = DenseTile<T, D>;
    using Loads = TileLoads<T, D, KT, NARROW ? 1 : PAIRED ? 8 : 4>;
    constexpr int TILEB = KT * Tile::ROWB, SUBS = KT / 32, AXIS = dense_tile(NARROW), WAVES = NARROW ? 4 : 1;
    constexpr int ST = dense_stages<T, D, FORM>(), LDSB = WAVES * ST * 2 * TILEB, JOINB = NARROW ? 12288 * Tile::NB : PAIRED ? 16384 * Tile::NB : 0;
    __shared__ __attribute__((aligned(1024))) char lds[LDSB > JOINB ? LDSB : JOINB];      // wave; stage; keys, values
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, col = lane & 31;
    const int pair = wave & 3, half = wave >> 2;
    const DenseWork work = dense_work<AXIS, true>(a, grid);
    const DenseGroup p(a, work.group);
    const Tile tile(lane);
    const int64_t row0 = (int64_t)work.tile * AXIS, wrow0 = NARROW ? row0 : row0 + pair * 32, r = wrow0 + col;
    // All rows are read, those behind the length too, so that they are on their way before the lengths are there: what such a row holds stays in its lane.
    const bool in = r < grid.rows;
    const int qi = (int)a.div_g((uint32_t)(in ? r : 0)), qg = (int)((in ? r : 0) - (int64_t)qi * a.G);
    const int64_t at_q = qg * a.q.head + (int64_t)qi * a.q.token, at_o = qg * a.o.head + (int64_t)qi * a.o.token;
    Piece<T> q[Tile::KS], g[Tile::KS], o[Tile::KS];
#pragma unroll
    for (int ks = 0; ks < Tile::KS; ++ks) {
        q[ks].w = *reinterpret_cast<const u32x4 *>(p.Q + at_q + 16 * h + 32 * ks);
        g[ks].w = *reinterpret_cast<const u32x4 *>(p.dO + at_o + 16 * h + 32 * ks);
        o[ks].w = *reinterpret_cast<const u32x4 *>(p.O + at_o + 16 * h + 32 * ks);
    }
    const float lse = p.LSE[(int64_t)qg * a.Nq + qi];
    const DensePieces piece(grid, work.split, 0, dense_key_steps<AXIS, KT>(a, p, row0));
    if (piece.none) return;
    const KeySpan mine = key_span(a, p, wrow0, wrow0 + 31);
    const int seen = in ? p.seen(a, qi) : 0;
    float delta = 0.f;
#pragma unroll
    for (int ks = 0; ks < Tile::KS; ++ks) delta = piece_dot(g[ks], o[ks], delta);
    float nD = seen > 0 ? -half_sum(delta) : 0.f;
    constexpr bool ROUNDED = sizeof(T) == 2;
    const float nlse = seen > 0 ? (ROUNDED ? -lse / a.scale : -lse * kLog2e) : -INFINITY;
    const bool first = h == 0 && (NARROW ? wave == 0 : half == 0);
    if (work.split == 0 && first) {                          // also for the rows that the last tile has too many
        a.nD[work.group * a.stat_rows + r] = nD;
        a.nlse[work.group * a.stat_rows + r] = nlse;
    }
    f32x16 s_from, dq[Tile::NB];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        s_from[e] = ROUNDED ? nlse : 0.f;
#pragma unroll
        for (int n = 0; n < Tile::NB; ++n) dq[n][e] = 0.f;
    }

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
    // a row's sum over its lanes and waves, in all of them (the ring is free)
    auto row_sum = [&](float x) {
        x = half_sum(x);
        if constexpr (FORM != kDenseWide) {
            float *red = reinterpret_cast<float *>(lds);
            __syncthreads();
            red[wave * 64 + lane] = x;
            __syncthreads();
            x = red[(NARROW ? 0 : pair) * 64 + lane] + red[(NARROW ? 1 : pair + 4) * 64 + lane];
            if (NARROW) x += red[128 + lane] + red[192 + lane];
            __syncthreads();
        }
        return x;
    };
    // D of rowsum(dO O) is off by what O's rounding to bf16 left out: of a row of few keys as much as dS is by its own.  sum_j dS_ij = D - D' for the D' that dS was formed
    // with, so the walk over the keys gives D itself: to the key-major pass always, and where it is short (512 keys: beyond them O is small beside dP) to a second walk that
    // forms dQ.  Error of dQ and dK against 64 bits, causal 3 x 16 heads of up to 1999 tokens, d = 128: 2.5e-3 -> 2.4e-3 (1.7e-3 is the results' own rounding);
    // the sums cost 1.7 % of the backward at 16 x 16384, d = 64, 0.7 % at 16 x 8192, d = 128.
    float sum = 0.f;                                         // of the lane's dS
    const bool two = ROUNDED && piece.alone && (piece.t1 - piece.t0) * KT <= 512;
#pragma unroll 1
    for (int walk = two ? 0 : 1; walk < 2; ++walk) {
        f32x16 dp_from;
#pragma unroll
        for (int e = 0; e < 16; ++e) dp_from[e] = nD;
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
            const int k0 = t * KT;
            if (k0 >= mine.some) continue;
            const char *kt = ring, *vt = ring + TILEB;
#pragma unroll 1
            for (int u = PAIRED ? half : 0; u < SUBS; u += PAIRED ? 2 : 1) {      // (unrolled, the operands of two of them at once do not fit at d = 128)
                const Tile at = tile.at(stage(t) + u * 32 * Tile::ROWB);
                f32x16 s = s_from, dp = dp_from;
                const bool some = k0 + 32 * u + 32 > mine.all;   // a key that some row does not see
                const int lim = seen - k0 - 32 * u - 4 * h;
                auto unseen = [&](f32x16 &x) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] = 8 * (e >> 2) + (e & 3) < lim ? x[e] : 0.f;
                };
                if constexpr (sizeof(T) == 2) {
                    constexpr int KS = Tile::KS, NB = Tile::NB, N1 = KS, N2 = 2 * KS, N3 = N2 + 2 * NB;
                    auto op = operands<N3, 2>([&](auto ic) {
                        constexpr int i = decltype(ic)::value;
                        if constexpr (i < N1) return __builtin_bit_cast(bf16x8, at.row(kt, 0, i).w);
                        else if constexpr (i < N2) return __builtin_bit_cast(bf16x8, at.row(vt, 0, i - N1).w);
                        else return at.col(kt, 0, (i - N2) % NB, (i - N2) / NB);
                    });
                    constants<KS>([&](auto i) { op.take(i, [&](bf16x8 x) { s = mfma32(x, __builtin_bit_cast(bf16x8, q[i].w), s); }); });
                    constants<KS>([&](auto i) {                  // the exponentials while dP is formed
                        op.take(plus(i, std::integral_constant<int, N1>()), [&](bf16x8 x) { dp = mfma32(x, __builtin_bit_cast(bf16x8, g[i].w), dp); });
#pragma unroll
                        for (int e = i * (16 / KS); e < (i + 1) * (16 / KS); ++e) s[e] = __builtin_amdgcn_exp2f(s[e] * a.scale2);
                    });
#pragma unroll
                    for (int e = 0; e < 16; ++e) dp[e] *= s[e];
                    if (some) unseen(dp);
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum += dp[e];
                    if (walk == 0) continue;
                    const bf16x8 ds[2] = {round8(dp, 0), round8(dp, 1)};
                    constants<2 * NB>([&](auto i) { op.take(plus(i, std::integral_constant<int, N2>()), [&](bf16x8 x) { dq[i % NB] = mfma32(x, ds[i / NB], dq[i % NB]); }); });
                } else {
#pragma unroll
                    for (int ks = 0; ks < Tile::KS; ++ks) s = piece_product(at.row(kt, 0, ks), q[ks], s);
#pragma unroll
                    for (int ks = 0; ks < Tile::KS; ++ks) dp = piece_product(at.row(vt, 0, ks), g[ks], dp);
#pragma unroll
                    for (int e = 0; e < 16; ++e) dp[e] *= __builtin_amdgcn_exp2f(fmaf(s[e], a.scale2, nlse));
                    if (some) unseen(dp);
#pragma unroll
                    for (int n = 0; n < Tile::NB; ++n) dq[n] = at.col_product(kt, 0, n, dp, dq[n]);
                }
            }
        }

        if (walk == 0) {
            const float all = row_sum(sum);                      // (barriers: for the waves without rows too)
            nD = seen > 0 ? nD - all : 0.f;
            sum = 0.f;
            if (FORM == kDenseWide) __syncthreads();             // nobody reads the ring that the second walk begins to fill
        }
    }

    if constexpr (ROUNDED) {
        sum = row_sum(sum);
        if (piece.alone) {
            nD = seen > 0 ? nD - sum : 0.f;
            if (in && first) a.nD[work.group * a.stat_rows + r] = nD;
        } else if (in && first) {
            grid.stat[((int64_t)work.split * grid.groups + work.group) * grid.rows + r] = sum;
        }
    }
    if constexpr (FORM != kDenseWide) {
        __syncthreads();
        if (NARROW) add_waves(dq, 1.f, lds, wave, lane);
        else add_halves(dq, 1.f, lds, pair, half, lane);
        if (NARROW ? wave > 0 : half > 0) return;
    }
    if (!piece.alone) {
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
// Narrow: 32 keys, for which each wave has every fourth tile of rows, in stages of its own.  Paired: the first or second half of every tile.
template <class T, int D, int QT, int FORM>
__global__ void __launch_bounds__(FORM == kDensePaired ? 512 : 256, (dkv_waves<T, D, FORM>())) dense_dkv_kernel(DenseArgs a, DenseGrid grid) {
    constexpr bool NARROW = FORM == kDenseNarrow, PAIRED = FORM == kDensePaired;
    using Tile = DenseTile<T, D>;
    using Loads = TileLoads<T, D, QT, NARROW ? 1 : PAIRED ? 8 : 4>;
    constexpr int TILEB = QT * Tile::ROWB, SUBS = QT / 32, AXIS = dense_tile(NARROW), WAVES = NARROW ? 4 : 1;
    constexpr int ST = dense_stages<T, D, FORM>(), STAGEB = 2 * TILEB + 1024;
    // Two of the eight pieces of a lane's key stand in LDS at d = 128: the registers hold 64 of sums for each of dK and dV and 24 of 32 of keys and 32 of values, and a spill to
    // memory in the loop would wait for the ring's newest tile.
    constexpr int SPARE = sizeof(T) == 2 && D == 128 && !NARROW ? 2 : 0, KR = Tile::KS - SPARE;
    constexpr int LDSB = WAVES * ST * STAGEB + 4096 * SPARE, JOINB = NARROW ? 24576 * Tile::NB : PAIRED ? 16384 * Tile::NB : 0;
    // wave; stage; queries, their output's gradients, their -LSE / scale and -D
    __shared__ __attribute__((aligned(1024))) char lds[LDSB > JOINB ? LDSB : JOINB];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, col = lane & 31;
    const int pair = wave & 3, half = wave >> 2;
    const DenseWork work = dense_work<AXIS, false>(a, grid);
    const DenseGroup p(a, work.group);
    const Tile tile(lane);
    const int key0 = work.tile * AXIS, wkey0 = NARROW ? key0 : key0 + pair * 32, j = wkey0 + col;
    // (of all keys, also those behind the length: on their way before the lengths are there, and what such a key holds stays in its lane)
    Piece<T> k[Tile::KS], v[Tile::KS];
    const char *const kj = p.K + min((int64_t)j, a.Nkv - 1) * a.k.token, *const vj = p.V + min((int64_t)j, a.Nkv - 1) * a.v.token;
#pragma unroll
    for (int ks = 0; ks < Tile::KS; ++ks) {
        k[ks].w = *reinterpret_cast<const u32x4 *>(kj + 16 * h + 32 * ks);
        v[ks].w = *reinterpret_cast<const u32x4 *>(vj + 16 * h + 32 * ks);
    }
    int first;
    const int steps = dense_row_steps<QT>(a, p, key0, &first);
    const DensePieces piece(grid, work.split, first, steps);
    if (piece.none) return;
    const bool valid = j < p.nk;
    u32x4 *const spare = reinterpret_cast<u32x4 *>(lds + WAVES * ST * STAGEB + pair * (1024 * SPARE)) + lane;
    f32x16 dk[Tile::NB], dv[Tile::NB];
#pragma unroll
    for (int n = 0; n < Tile::NB; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) dk[n][e] = dv[n][e] = 0.f;

    const int rows = p.nq * a.G;                             // rows that see something: of each key, those from its first query's on
    const int from = p.first_query(a, j) * a.G;
    const int wfrom = p.first_query(a, wkey0) * a.G, wto = p.first_query(a, min(wkey0 + 31, max(p.nk - 1, 0))) * a.G;
    const float *nlse = a.nlse + work.group * a.stat_rows, *nD = a.nD + work.group * a.stat_rows;
    char *const ring = lds + (NARROW ? wave * (ST * STAGEB) : 0);
    const unsigned ring0 = lds_address(ring);
    const int t0 = piece.t0 + (NARROW ? wave : 0);
    auto stage = [&](int t) { return ST == 1 ? 0 : ((t - t0) / WAVES & 1) * STAGEB; };
    auto fetch = [&](int t) {
        const int r0 = t * QT, q0 = (int)a.div_g(r0);
        const unsigned to = ring0 + stage(t), st0 = to + 2 * TILEB, bytes = (unsigned)min((int64_t)64, a.stat_rows - r0) * 4;
        Loads::rows(buffer_of(p.Q + (int64_t)q0 * a.q.token, 0xffffff00u), buffer_of(p.dO + (int64_t)q0 * a.o.token, 0xffffff00u), a, r0, q0, rows, to, to + TILEB, NARROW ? 0 : wave, lane);
        if (NARROW || wave == 0) buffer_to_lds_dword(buffer_of(reinterpret_cast<const char *>(nlse + r0), bytes), lane * 4, st0);
        if (NARROW || wave == 1) buffer_to_lds_dword(buffer_of(reinterpret_cast<const char *>(nD + r0), bytes), lane * 4, st0 + 256);
    };
    if (ST == 2 && t0 < piece.t1) fetch(t0);
    loads_done();
#pragma unroll
    for (int ks = 0; ks < SPARE; ++ks) spare[64 * ks] = k[KR + ks].w;
    for (int t = t0; t < piece.t1; t += WAVES) {
        if (ST == 1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            fetch(t);
        }
        if (NARROW) vm_wait<0>();                            // tile t is there (and nobody else reads the wave's stages),
        else vm_wait_barrier<0>();                           // for all waves, and nobody reads the other stage
        if (ST == 2 && t + WAVES < piece.t1) fetch(t + WAVES);
        const char *qt = ring, *gt = ring + TILEB;
        const float *st = reinterpret_cast<const float *>(ring + stage(t) + 2 * TILEB);
#pragma unroll 1
        for (int u = PAIRED ? half : 0; u < SUBS; u += PAIRED ? 2 : 1) {
            const int r0 = t * QT + 32 * u;
            if (r0 + 31 < wfrom || r0 >= rows) continue;     // (without rows: nobody wrote their -LSE and -D, where the other kernel's tiles are narrow)
            const Tile at = tile.at(stage(t) + u * 32 * Tile::ROWB);
            f32x16 s, dp;
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const f32x4 x = *reinterpret_cast<const f32x4 *>(st + 32 * u + 2 * e + 4 * h), y = *reinterpret_cast<const f32x4 *>(st + 64 + 32 * u + 2 * e + 4 * h);
#pragma unroll
                for (int i = 0; i < 4; ++i) { s[e + i] = x[i]; dp[e + i] = y[i]; }
            }
            const bool some = r0 < wto;                      // a row that does not see some key
            auto unseen = [&](f32x16 &x) {
                int lim = from - r0 - 4 * h;
                asm volatile("" : "+v"(lim));                // (compared anew each time: sixteen pairs of scalar registers would be kept from S to dS)
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = 8 * (e >> 2) + (e & 3) >= lim ? x[e] : 0.f;
            };
            if constexpr (sizeof(T) == 2) {
                constexpr int KS = Tile::KS, NB = Tile::NB, N1 = KS, N2 = 2 * KS, N3 = N2 + 2 * NB, N4 = N3 + 2 * NB;
                auto op = operands<N4, 2>([&](auto ic) {
                    constexpr int i = decltype(ic)::value;
                    if constexpr (i < N1) return __builtin_bit_cast(bf16x8, at.row(qt, 0, i).w);
                    else if constexpr (i < N2) return __builtin_bit_cast(bf16x8, at.row(gt, 0, i - N1).w);
                    else if constexpr (i < N3) return at.col(gt, 0, (i - N2) % NB, (i - N2) / NB);
                    else return at.col(qt, 0, (i - N3) % NB, (i - N3) / NB);
                });
                u32x4 ks[SPARE ? SPARE : 1];
                constants<KS>([&](auto i) {
                    if constexpr (SPARE && i == KR - 2)
#pragma unroll
                        for (int c = 0; c < SPARE; ++c) ks[c] = spare[64 * c];
                    op.take(i, [&](bf16x8 x) {
                        if constexpr (i < KR) s = mfma32(x, __builtin_bit_cast(bf16x8, k[i].w), s);
                        else s = mfma32(x, __builtin_bit_cast(bf16x8, ks[i - KR]), s);
                    });
                });
                constants<KS>([&](auto i) {                  // the exponentials while dP is formed
                    op.take(plus(i, std::integral_constant<int, N1>()), [&](bf16x8 x) { dp = mfma32(x, __builtin_bit_cast(bf16x8, v[i].w), dp); });
#pragma unroll
                    for (int e = i * (16 / KS); e < (i + 1) * (16 / KS); ++e) s[e] = __builtin_amdgcn_exp2f(s[e] * a.scale2);
                });
                if (some) unseen(s);
                bf16x8 x8 = round8(s, 0);
                constants<2 * NB>([&](auto i) {              // dS while P's products are
                    if constexpr (i == NB) x8 = round8(s, 1);
                    op.take(plus(i, std::integral_constant<int, N2>()), [&](bf16x8 x) { dv[i % NB] = mfma32(x, x8, dv[i % NB]); });
#pragma unroll
                    for (int e = i * (8 / NB); e < (i + 1) * (8 / NB); ++e) dp[e] *= s[e];
                });
                if (some) unseen(dp);
                x8 = round8(dp, 0);
                constants<2 * NB>([&](auto i) {
                    if constexpr (i == NB) x8 = round8(dp, 1);
                    op.take(plus(i, std::integral_constant<int, N3>()), [&](bf16x8 x) { dk[i % NB] = mfma32(x, x8, dk[i % NB]); });
                });
            } else {
                const f32x16 nlse16 = s;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
                for (int ks = 0; ks < KR; ++ks) s = piece_product(at.row(qt, 0, ks), k[ks], s);
#pragma unroll
                for (int ks = 0; ks < Tile::KS; ++ks) dp = piece_product(at.row(gt, 0, ks), v[ks], dp);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], a.scale2, nlse16[e]));
                    dp[e] *= s[e];
                }
                if (some) {
                    unseen(s);
                    unseen(dp);
                }
#pragma unroll
                for (int n = 0; n < Tile::NB; ++n) dv[n] = at.col_product(gt, 0, n, s, dv[n]);
#pragma unroll
                for (int n = 0; n < Tile::NB; ++n) dk[n] = at.col_product(qt, 0, n, dp, dk[n]);
            }
        }
    }

    if constexpr (NARROW) {
        __syncthreads();
        add_waves(dk, 1.f, lds, wave, lane);
        add_waves(dv, 1.f, lds + 12288 * Tile::NB, wave, lane);
        if (wave > 0) return;
    } else if constexpr (PAIRED) {
        __syncthreads();
        add_halves(dk, 1.f, lds, pair, half, lane);
        __syncthreads();
        add_halves(dv, 1.f, lds, pair, half, lane);
        if (half > 0) return;
    }
    if (!piece.alone) {
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

// The pieces' sums of a row in order, one wave a row; where there was one piece, its sums are the result already.
template <class T, int D, int AXIS, int KT> __global__ void __launch_bounds__(256) dense_dq_join_kernel(DenseArgs a, DenseGrid grid) {
    using Row = LaneRow<T, D>;
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= grid.rows) return;
    const DenseGroup p(a, blockIdx.y);
    const int i = (int)a.div_g((uint32_t)r), g = (int)(r - (int64_t)i * a.G);
    const int steps = dense_key_steps<AXIS, KT>(a, p, r / AXIS * AXIS), pieces = (steps + grid.chunk - 1) / grid.chunk;
    if (pieces <= 1) return;
    Row acc = Row::zero();
    const int64_t at = (int64_t)blockIdx.y * grid.rows + r, step = (int64_t)grid.groups * grid.rows;      // piece 0's sums; from piece to piece
    float nD = a.nD[blockIdx.y * a.stat_rows + r];
    if (p.seen(a, i) > 0) {
        for (int s = 0; s < pieces; s += 64) acc.add_parts(grid.part + (at + s * step) * D, step * D, min(64, pieces - s), 1.f, lane);
        if constexpr (sizeof(T) == 2) {
            float sum = 0.f;
            for (int s = lane; s < pieces; s += 64) sum += grid.stat[at + s * step];
            nD -= wave_sum(sum);
            if (lane == 0) a.nD[blockIdx.y * a.stat_rows + r] = nD;
        }
    }
    acc.scale(a.scale);
    if (a.causal && !acc.finite()) dense_row_dq<T, D>(a, p, i, g, nD, lane);
    else acc.store(p.dQ + g * a.q.head + i * a.q.token, lane);
}

template <class T, int D, int AXIS, int QT> __global__ void __launch_bounds__(256) dense_dkv_join_kernel(DenseArgs a, DenseGrid grid) {
    using Row = LaneRow<T, D>;
    const int lane = threadIdx.x & 63;
    const int64_t j = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (j >= grid.rows) return;
    const DenseGroup p(a, blockIdx.y);
    int first;
    const int steps = dense_row_steps<QT>(a, p, (int)(j / AXIS * AXIS), &first), pieces = (steps + grid.chunk - 1) / grid.chunk;
    if (pieces <= 1) return;
    Row dk = Row::zero(), dv = Row::zero();
    if (j < p.nk) {
        const int64_t step = (int64_t)grid.groups * grid.rows * (2 * D);
        const float *at = grid.part + ((int64_t)blockIdx.y * grid.rows + j) * (2 * D);
        for (int s = 0; s < pieces; s += 64) {
            dk.add_parts(at + s * step, step, min(64, pieces - s), 1.f, lane);
            dv.add_parts(at + D + s * step, step, min(64, pieces - s), 1.f, lane);
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

template <class T, int D, int FORM> static hipError_t launch_dq(const DensePlan &p, const DenseArgs &a, float *part, hipStream_t s) {
    constexpr bool NARROW = FORM == kDenseNarrow;
    constexpr int KT = dense_step(DenseTile<T, D>::ROWB, NARROW);
    const DenseGrid g = dense_grid(p, p.rows, p.dq, D, part);
    dense_dq_kernel<T, D, KT, FORM><<<g.wgs, FORM == kDensePaired ? 512 : 256, 0, s>>>(a, g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || g.splits == 1) return e;
    dense_dq_join_kernel<T, D, dense_tile(NARROW), KT><<<dim3((unsigned)((g.rows + 3) / 4), g.groups), 256, 0, s>>>(a, g);
    return hipGetLastError();
}

template <class T, int D, int FORM> static hipError_t launch_dkv(const DensePlan &p, const DenseArgs &a, float *part, hipStream_t s) {
    constexpr bool NARROW = FORM == kDenseNarrow;
    constexpr int QT = dense_step(DenseTile<T, D>::ROWB, NARROW);
    const DenseGrid g = dense_grid(p, p.desc.Nkv, p.dkv, 2 * D, part);
    dense_dkv_kernel<T, D, QT, FORM><<<g.wgs, FORM == kDensePaired ? 512 : 256, 0, s>>>(a, g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || g.splits == 1) return e;
    dense_dkv_join_kernel<T, D, dense_tile(NARROW), QT><<<dim3((unsigned)((g.rows + 3) / 4), g.groups), 256, 0, s>>>(a, g);
    return hipGetLastError();
}

hipError_t launch_dense_bwd(const DensePlan &p, const DenseArgs &a, float *part, hipStream_t s) {
    const hipError_t e = dense_dispatch_form(p, p.dq, p.rows, [&](auto t, auto d, auto form) { return launch_dq<decltype(t), decltype(d)::value, decltype(form)::value>(p, a, part, s); });
    if (e != hipSuccess) return e;
    return dense_dispatch_form(p, p.dkv, p.desc.Nkv, [&](auto t, auto d, auto form) { return launch_dkv<decltype(t), decltype(d)::value, decltype(form)::value>(p, a, part, s); });
}

}  // namespace llsa
