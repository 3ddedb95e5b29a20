// The norms between two blocks with gate and residual, forward and backward: one pass over the rows, each held in registers by 4 to 512
// threads (at most 16 channels a thread), so that a row is read once and written once.  What varies by channel only (the gains, and the
// modulation of the batch entry that a workgroup belongs to) stays in registers over all rows of the workgroup, combined:
//   y = n(x') ga + sh, x' = x + gz n(branch)       with ga = gain (1 + scale), sh = shift, gz = alpha gate gain_branch.
// Backward, per row, with h^ = n(x'), u = n(branch) (or the branch itself):
//   p = dy ga;  dh = r (p - h^ mean(p h^) [- mean p]) + dx_out;   w = gz dh;  db = r_b (w - u mean(w u) [- mean w])  (no norm: w)
// and per channel and batch entry three sums over the rows: E = sum dy h^, T = sum dy, F = sum dh u, from which
//   dgain = sum_b (1 + scale) E, dscale = gain E, dshift = T, dgate = alpha gain_branch F, dgain_branch = alpha sum_b gate F.
// A thread keeps its channels' sums over all its rows; the workgroups' sums go to the workspace and a second launch adds them in a fixed order.
// Bytes bound it, cold: 2 x 16384 rows of 1024 in bf16, forward 52 us (268 MB, 5.15 TB/s), backward 84 (403 MB, 4.8 TB/s) and 7.6 for the sums; 3 x 2704 rows of 1001 in fp32 with LayerNorm, whose
// rows begin at any element, backward 54 in all (195 MB, 3.6 TB/s).
#include "lanes.h"
#include "norm.h"

#include <algorithm>
#include <new>
#include <type_traits>

namespace llsa {

// 16 bytes of elements at any element's alignment
template <class T> struct NVec {
    static constexpr int n = 16 / sizeof(T);
    struct __attribute__((packed, aligned(sizeof(T)))) Raw { uint32_t w[4]; };
    Raw r;
};

template <class T> __device__ __forceinline__ float n_get(const T *p);
template <> __device__ __forceinline__ float n_get<float>(const float *p) { return *p; }
template <> __device__ __forceinline__ float n_get<__bf16>(const __bf16 *p) { return (float)*p; }

template <class T> __device__ __forceinline__ void n_unpack(const typename NVec<T>::Raw &r, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            x[i] = __uint_as_float(r.w[i]);
        } else {
            x[2 * i] = __uint_as_float(r.w[i] << 16);
            x[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
        }
    }
}
// Which channels of a row a thread has: NV vectors of n, number k at channel (k TPR + t) n.  The form is a row's:
//   kWhole: the vectors cover it exactly
//   kTail: the last one that is not whole is read n channels from the row's end, and only its last ones are the thread's own; one beyond the row is read at its beginning
//          and has none.  No load needs a branch.
//   kShort: fewer than n channels, element by element
enum NormRow { kWhole, kTail, kShort };
template <class T, int TPR, int NV, int ROW> struct Channels {
    static constexpr int n = NVec<T>::n, E = NV * n;
    static constexpr bool whole = ROW == kWhole, vectors = ROW != kShort;
    int first[NV], own[NV], C;                               // where a vector is read, its first element that is the thread's own
    __device__ __forceinline__ Channels(int t, int C_) : C(C_) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TPR + t) * n;
            first[k] = whole || (c + n <= C || !vectors) ? c : c < C ? C - n : 0;
            own[k] = whole || c + n <= C || (!vectors && c < C) ? 0 : c < C ? c - first[k] : n;
        }
    }
    __device__ __forceinline__ int channel(int i) const { return first[i / n] + i % n; }
    __device__ __forceinline__ bool mine(int i) const { return whole || (i % n >= own[i / n] && (vectors || channel(i) < C)); }
    // a row's channels as they stand in memory, and as numbers; what is not the thread's own is some other channel of the row (kShort: 0)
    struct Raw { typename NVec<T>::Raw r[NV]; };
    __device__ __forceinline__ void ask(const char *base, int64_t at, Raw &x) const {
        const T *row = reinterpret_cast<const T *>(base) + at;
        if constexpr (vectors) {
#pragma unroll
            for (int k = 0; k < NV; ++k) x.r[k] = *reinterpret_cast<const typename NVec<T>::Raw *>(row + first[k]);
        } else {
            union { T v[E]; Raw r; } u;
#pragma unroll
            for (int i = 0; i < E; ++i) u.v[i] = mine(i) ? row[channel(i)] : (T)0.f;
            x = u.r;
        }
    }
    __device__ __forceinline__ void get(const Raw &r, float (&x)[E]) const {
#pragma unroll
        for (int k = 0; k < NV; ++k) n_unpack<T>(r.r[k], x + k * n);
    }
    // .. with zeros for what is not the thread's own
    __device__ __forceinline__ void load(const char *base, int64_t at, float (&x)[E]) const {
        Raw r;
        ask(base, at, r);
        get(r, x);
#pragma unroll
        for (int i = 0; !whole && i < E; ++i) x[i] = mine(i) ? x[i] : 0.f;
    }
    __device__ __forceinline__ void store(char *base, int64_t at, const float (&x)[E]) const {
        T *row = reinterpret_cast<T *>(base) + at;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (whole || (vectors && own[k] == 0)) {
                typename NVec<T>::Raw r;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (sizeof(T) == 4) {
                        r.w[i] = __float_as_uint(x[k * n + i]);
                    } else {
                        union { __bf16 h[2]; uint32_t u; } w;
                        w.h[0] = (__bf16)x[k * n + 2 * i];
                        w.h[1] = (__bf16)x[k * n + 2 * i + 1];
                        r.w[i] = w.u;
                    }
                }
                *reinterpret_cast<typename NVec<T>::Raw *>(row + first[k]) = r;
            }
            if constexpr (!whole) {
                const bool part = !vectors || (own[k] > 0 && own[k] < n);
                if (__builtin_amdgcn_ballot_w64(part)) {     // (in one wave of a row at most)
#pragma unroll
                    for (int e = 0; e < n; ++e)
                        if (part && mine(k * n + e)) row[first[k] + e] = (T)x[k * n + e];
                }
            }
        }
    }
};
// a modulation vector's channel, of either type; `none` where it was not given
__device__ __forceinline__ float n_mod(const char *m, int f32, int64_t at, float none) {
    return !m ? none : f32 ? reinterpret_cast<const float *>(m)[at] : n_get(reinterpret_cast<const __bf16 *>(m) + at);
}
// a thread's channels of a gain or a modulation vector (which may begin at any element)
template <class Ch> __device__ __forceinline__ void channels_of(const Ch &ch, const char *m, int f32, int64_t at, float none, float (&x)[Ch::E]) {
    constexpr int n = Ch::n;
    if (!m) {
#pragma unroll
        for (int i = 0; i < Ch::E; ++i) x[i] = none;
    } else if constexpr (!Ch::vectors) {
#pragma unroll
        for (int i = 0; i < Ch::E; ++i) x[i] = ch.mine(i) ? n_mod(m, f32, at + ch.channel(i), none) : none;
    } else if (f32) {
        struct __attribute__((packed, aligned(4))) Raw { float v[n]; };
#pragma unroll
        for (int k = 0; k < Ch::E / n; ++k) {
            const Raw r = *reinterpret_cast<const Raw *>(reinterpret_cast<const float *>(m) + at + ch.first[k]);
#pragma unroll
            for (int e = 0; e < n; ++e) x[k * n + e] = r.v[e];
        }
    } else {
        struct __attribute__((packed, aligned(2))) Raw { __bf16 v[n]; };
#pragma unroll
        for (int k = 0; k < Ch::E / n; ++k) {
            const Raw r = *reinterpret_cast<const Raw *>(reinterpret_cast<const __bf16 *>(m) + at + ch.first[k]);
#pragma unroll
            for (int e = 0; e < n; ++e) x[k * n + e] = (float)r.v[e];
        }
    }
}
// what the rows of batch entry b are multiplied by (0 for the channels that are not the thread's own): alpha gate gain_branch, gain (1 + scale)
template <class Ch> __device__ __forceinline__ void channel_factors(const NormArgs &a, const Ch &ch, int64_t at, float (&gz)[Ch::E], float (&ga)[Ch::E]) {
    float v[Ch::E], w[Ch::E];
    channels_of(ch, a.gate, a.mod_f32, at, 1.f, v);
    channels_of(ch, reinterpret_cast<const char *>(a.gain_branch), 1, 0, 1.f, w);
#pragma unroll
    for (int i = 0; i < Ch::E; ++i) gz[i] = ch.mine(i) ? a.alpha * v[i] * w[i] : 0.f;
    channels_of(ch, a.scale, a.mod_f32, at, 0.f, v);
    channels_of(ch, reinterpret_cast<const char *>(a.gain), 1, 0, 1.f, w);
#pragma unroll
    for (int i = 0; i < Ch::E; ++i) ga[i] = ch.mine(i) ? w[i] * (1.f + v[i]) : 0.f;
}

// threads of a workgroup: four waves with rows of their own, or one row
constexpr int norm_threads(int tpr) { return tpr <= 64 ? 256 : tpr; }
// which of the workgroup's rows a thread works on (the same for a wave, and known to be, where a row has whole waves)
template <int TPR> __device__ __forceinline__ int norm_row() { return TPR >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TPR) : threadIdx.x / TPR; }

// Sums over the TPR threads of a row, K at once, the result in each of them.  lds: K floats a wave of the workgroup, not read or written by another call
// until a barrier.  The whole workgroup calls.
template <int TPR, int K> __device__ __forceinline__ void row_sums(float (&v)[K], float *lds) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = lanes_sum<(TPR < 64 ? TPR : 64)>(v[k]);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64, ALL = norm_threads(TPR) / 64;
        const int w = threadIdx.x >> 6, w0 = w / W * W;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) lds[k * ALL + w] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) v[k] += lds[k * ALL + w0 + i];
        }
    }
}

// mean and 1 / deviation of a row held as x (zeros beyond C)
template <int TPR, int E, bool LAYER, class Ch>
__device__ __forceinline__ void row_stats(const float (&x)[E], const Ch &ch, float inv_c, float eps, float *lds, float &m, float &r) {
    float s[1] = {0.f};
    m = 0.f;
    if constexpr (LAYER) {
#pragma unroll
        for (int e = 0; e < E; ++e) s[0] += x[e];
        row_sums<TPR, 1>(s, lds);
        m = s[0] * inv_c;
        s[0] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float d = !LAYER || ch.mine(e) ? x[e] - m : 0.f;
        s[0] = fmaf(d, d, s[0]);
    }
    row_sums<TPR, 1>(s, lds + 32);
    r = 1.f / sqrtf(fmaf(s[0], inv_c, eps));
}

template <class T, int TPR, int NV, bool LAYER, int ROW>
__global__ void __launch_bounds__(norm_threads(TPR)) norm_fwd_kernel(NormArgs a) {
    using Ch = Channels<T, TPR, NV, ROW>;
    constexpr int E = Ch::E, GP = norm_threads(TPR) / TPR;
    __shared__ float lds[4][32];
    const int t = threadIdx.x % TPR, b = blockIdx.y;
    const Ch ch(t, a.C);
    float gz[E], ga[E], sh[E];
    channel_factors(a, ch, b * a.mod_stride, gz, ga);
    channels_of(ch, a.shift, a.mod_f32, b * a.mod_stride, 0.f, sh);
    for (int64_t n = (int64_t)blockIdx.x * GP + norm_row<TPR>(); n < a.N; n += (int64_t)gridDim.x * GP) {
        const int64_t row = b * a.N + n;
        float x[E], st[4] = {0.f, 0.f, 0.f, 0.f};
        ch.load(a.x, row * a.C, x);
        if (a.branch) {
            float u[E];
            ch.load(a.branch, row * a.C, u);
            if (a.gain_branch) {
                row_stats<TPR, E, LAYER>(u, ch, a.inv_c, a.eps, lds[0], st[2], st[3]);
#pragma unroll
                for (int e = 0; e < E; ++e) u[e] = (LAYER ? u[e] - st[2] : u[e]) * st[3];
            }
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = (float)(T)fmaf(gz[e], u[e], x[e]);
            ch.store(a.x_out, row * a.C, x);
        }
        if (a.y) {
            row_stats<TPR, E, LAYER>(x, ch, a.inv_c, a.eps, lds[2], st[0], st[1]);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = fmaf((LAYER ? x[e] - st[0] : x[e]) * st[1], ga[e], sh[e]);
            ch.store(a.y, row * a.C, x);
        }
        if (a.stats && t == 0) *reinterpret_cast<float4 *>(a.stats + 4 * row) = make_float4(st[0], st[1], st[2], st[3]);
        if constexpr (TPR > 64) __syncthreads();             // the next row's sums go where this one's are read
    }
}

template <class T, int TPR, int NV, bool LAYER, int ROW>
__global__ void __launch_bounds__(norm_threads(TPR)) norm_bwd_kernel(NormArgs a) {
    using Ch = Channels<T, TPR, NV, ROW>;
    constexpr int E = Ch::E, GP = norm_threads(TPR) / TPR;
    constexpr int SPAN = TPR * E;                            // channels that the threads of a row cover
    __shared__ float lds[2][32];
    __shared__ float sums[GP > 1 ? 3 * SPAN : 1];
    const int t = threadIdx.x % TPR, b = blockIdx.y;
    const Ch ch(t, a.C);
    float gz[E], ga[E], sE[E], sT[E], sF[E];
    channel_factors(a, ch, b * a.mod_stride, gz, ga);
#pragma unroll
    for (int i = 0; i < E; ++i) sE[i] = sT[i] = sF[i] = 0.f;
    // The next two rows (one where a row is 16 registers a thread and tensor) are on their way while this one is worked on.  Their loads are the same whatever the call
    // has: a tensor that it lacks stands for x', a row behind the last one for the last one; between loads that may or may not be there the compiler can only wait
    // for all of them.  For the same reason they are asked for behind this row's stores.
    constexpr int SLOTS = E * (int)sizeof(T) <= 32 ? 2 : 1;
    const int64_t step = (int64_t)gridDim.x * GP;
    int64_t n0 = (int64_t)blockIdx.x * GP + norm_row<TPR>();
    const char *const in_g = a.dy ? a.dy : a.x, *const in_d = a.dx_out ? a.dx_out : a.x, *const in_u = a.branch ? a.branch : a.x;
    struct { typename Ch::Raw x, g, d, u; float4 st; } next[SLOTS];
    auto ask = [&](int64_t n, auto k) {
        const int64_t row = b * a.N + min(n, a.N - 1), at = row * a.C;
        next[k].st = *reinterpret_cast<const float4 *>(a.stats + 4 * row);
        ch.ask(a.x, at, next[k].x);
        ch.ask(in_g, at, next[k].g);
        ch.ask(in_d, at, next[k].d);
        ch.ask(in_u, at, next[k].u);
    };
    auto work = [&](int64_t n, auto k) {
        const int64_t at = (b * a.N + n) * a.C;
        float d[E], u[E], x[E], g[E];                        // gradient of x'; normed branch; x', dy
        const float4 st = next[k].st;
        ch.get(next[k].x, x);
        ch.get(next[k].g, g);
        ch.get(next[k].d, d);
        ch.get(next[k].u, u);
        if (!a.dx_out) {
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] = 0.f;
        }
        if (SLOTS == 1) ask(n + step, k);
        if (a.dy) {
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[e] = (LAYER ? x[e] - st.x : x[e]) * st.y;  // not its own: a value that only meets zeros
                sE[e] = fmaf(g[e], x[e], sE[e]);
                sT[e] += g[e];
                g[e] *= ga[e];
                m[0] = fmaf(g[e], x[e], m[0]);
                if constexpr (LAYER) m[1] += g[e];
            }
            if constexpr (LAYER) {
                row_sums<TPR, 2>(m, lds[0]);
            } else {
                float s[1] = {m[0]};
                row_sums<TPR, 1>(s, lds[0]);
                m[0] = s[0];
            }
            m[0] *= a.inv_c;
            m[1] *= a.inv_c;
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] = fmaf(st.y, LAYER ? fmaf(-x[e], m[0], g[e]) - m[1] : fmaf(-x[e], m[0], g[e]), d[e]);
        }
        ch.store(a.dx, at, d);
        if (a.branch) {
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (a.gain_branch) u[e] = (LAYER ? u[e] - st.z : u[e]) * st.w;
                sF[e] = fmaf(d[e], u[e], sF[e]);
                d[e] *= gz[e];
                m[0] = fmaf(d[e], u[e], m[0]);
                if constexpr (LAYER) m[1] += d[e];
            }
            if (a.gain_branch) {
                if constexpr (LAYER) {
                    row_sums<TPR, 2>(m, lds[1]);
                } else {
                    float s[1] = {m[0]};
                    row_sums<TPR, 1>(s, lds[1]);
                    m[0] = s[0];
                }
                m[0] *= a.inv_c;
                m[1] *= a.inv_c;
#pragma unroll
                for (int e = 0; e < E; ++e) d[e] = (LAYER ? fmaf(-u[e], m[0], d[e]) - m[1] : fmaf(-u[e], m[0], d[e])) * st.w;
            }
            ch.store(a.dbranch, at, d);
        }
        if (SLOTS == 2) ask(n + 2 * step, k);
        if constexpr (TPR > 64) __syncthreads();             // the next row's sums go where this one's are read
    };
    constexpr std::integral_constant<int, 0> k0;
    constexpr std::integral_constant<int, SLOTS - 1> k1;
    ask(n0, k0);
    if (SLOTS == 2) ask(n0 + step, k1);
    if constexpr (SLOTS == 1) {
        for (; n0 < a.N; n0 += step) work(n0, k0);
    } else {                                                 // (two rows a round: one that may leave in between lets the compiler count on no load of the second slot)
        for (; n0 + step < a.N; n0 += 2 * step) {
            work(n0, k0);
            work(n0 + step, k1);
        }
        if (n0 < a.N) work(n0, k0);
    }
    if (!a.part) return;
    // the workgroup's sums: a wave's rows add theirs, then the waves in turn
    if constexpr (TPR < 64) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            sE[e] = rows_sum<TPR>(sE[e]);
            sT[e] = rows_sum<TPR>(sT[e]);
            sF[e] = rows_sum<TPR>(sF[e]);
        }
    }
    if constexpr (GP > 1) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll 1
        for (int w = 0; w < 4; ++w) {
            if (wave == w && lane < TPR)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float *s = sums + e * TPR + t;
                    s[0] = w ? s[0] + sE[e] : sE[e];
                    s[SPAN] = w ? s[SPAN] + sT[e] : sT[e];
                    s[2 * SPAN] = w ? s[2 * SPAN] + sF[e] : sF[e];
                }
            __syncthreads();
        }
        if ((int)threadIdx.x >= TPR) return;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float *s = sums + e * TPR + t;
            sE[e] = s[0];
            sT[e] = s[SPAN];
            sF[e] = s[2 * SPAN];
        }
    }
    float *part = a.part + ((int64_t)b * gridDim.x + blockIdx.x) * 3 * a.C;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int c = ch.channel(i);
        if (ch.mine(i)) {
            part[c] = sE[i];
            part[a.C + c] = sT[i];
            part[2 * a.C + c] = sF[i];
        }
    }
}

// The workgroups' sums added up, E, T and F each by workgroups of their own: 64 slices of 16 channels a workgroup, each slice every 64th workgroup's, then the slices in order.
__global__ void __launch_bounds__(1024) norm_sums_kernel(NormArgs a) {
    __shared__ float lds[64][17];
    const int which = blockIdx.y, col = threadIdx.x & 15, c = blockIdx.x * 16 + col, slice = threadIdx.x >> 4;
    float *const per_batch = which == 0 ? a.dscale : which == 1 ? a.dshift : a.dgate, *const per_channel = which == 0 ? a.dgain : which == 1 ? nullptr : a.dgain_branch;
    if (!per_batch && !per_channel) return;
    const bool in = c < a.C;
    const float *of = which == 0 ? a.gain : which == 1 ? nullptr : a.gain_branch;      // what a batch entry's gradient is multiplied by; the channel's: by its modulation
    const float f = (which == 2 ? a.alpha : 1.f) * (in && of ? of[c] : 1.f);
    float all = 0.f, shared = 0.f;
    for (int b0 = 0; b0 < a.batch; b0 += 2) {                // two batch entries' and eight workgroups' sums on their way at once
        float s[2] = {0.f, 0.f};
        if (in) {
            for (int w0 = slice; w0 < a.blocks; w0 += 512) {
                float v[8][2];
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        v[j][i] = a.part[(((int64_t)min(b0 + i, a.batch - 1) * a.blocks + min(w0 + 64 * j, a.blocks - 1)) * 3 + which) * a.C + c];
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i) s[i] += w0 + 64 * j < a.blocks ? v[j][i] : 0.f;
            }
        }
        for (int i = 0; i < 2 && b0 + i < a.batch; ++i) {
            const int b = b0 + i;
            lds[slice][col] = i == 0 ? s[0] : s[1];
            __syncthreads();
            if (slice < 4) {                                 // 16 slices each, then those four
                float v = 0.f;
#pragma unroll
                for (int q = 0; q < 16; ++q) v += lds[slice * 16 + q][col];
                v += __shfl_xor(v, 16, 64);
                v += __shfl_xor(v, 32, 64);
                if (slice == 0 && in) {
                    const int64_t at = b * a.mod_stride + c;
                    all = fmaf(which == 0 ? 1.f + n_mod(a.scale, a.mod_f32, at, 0.f) : a.alpha * n_mod(a.gate, a.mod_f32, at, 1.f), v, all);
                    shared += v;
                    if (a.mod_stride || b == a.batch - 1) {
                        if (per_batch) per_batch[(a.mod_stride ? (int64_t)b * a.C : 0) + c] = f * shared;
                        shared = 0.f;
                    }
                }
            }
            __syncthreads();
        }
    }
    if (slice == 0 && in && per_channel) per_channel[c] = all;
}

// The fewest threads a row that hold it with at most 16 (backward 8) channels each, 4, 16 or whole waves, up to 512 of them with up to 16 channels.
// Workgroups: what is resident at once, rows dealt out evenly (fp32 backward, 3 x 2704 rows of 1001: 58 -> 54 us against two workgroups in a second round).  Each
// workgroup of the backward pass writes sums that are three rows of fp32, so that as soon as every CU has one they get more rows first, up to 8 (16 x 256 rows of 1024
// 45 -> 37 us, 1 x 2048 24 -> 18, 1 x 1024 22 -> 14; 1 x 256 rows with 8 each 11.3 -> 13.5).
static NormShape norm_shape(const llsa_norm_desc &d, bool backward) {
    const int most = backward ? 8 : 16;
    const int64_t target = backward ? 512 : 1024;            // times 256 threads
    NormShape r;
    const int vn = d.dtype == LLSA_F32 ? 4 : 8, vec = (d.C + vn - 1) / vn;
    r.tpr = vec <= 4 ? 4 : vec <= 16 ? 16 : 64;
    while (r.tpr < 512 && vec > r.tpr * (most / vn)) r.tpr *= 2;
    r.nv = (vec + r.tpr - 1) / r.tpr;
    if (r.nv == 3) r.nv = 4;
    const int64_t rows = norm_threads(r.tpr) / r.tpr, all = (d.N + rows - 1) / rows, share = std::max<int64_t>(1, target * 256 / norm_threads(r.tpr) / d.batch);
    const int64_t least = backward ? std::min<int64_t>(8, (all * d.batch + 255) / 256) : 1, per = std::max(least, (all + share - 1) / share);
    r.blocks = (int)((all + per - 1) / per);
    return r;
}
void norm_layout(NormPlan &p) {
    p.fwd = norm_shape(p.desc, false);
    p.bwd = norm_shape(p.desc, true);
    p.ws = (size_t)p.desc.batch * p.bwd.blocks * 3 * p.desc.C * sizeof(float);
}

// As norm_layout chooses: at most 16 channels a thread, 8 in the backward pass but for 512 threads
template <bool FWD, class F> static void norm_dispatch(const NormPlan &p, const NormShape &sh, F go) {
    using std::integral_constant;
    auto shape = [&](auto t, auto layer) {
        constexpr int vn = 16 / sizeof(t);
        auto with = [&](auto tpr, auto nv) {
            if (p.desc.C == sh.tpr * sh.nv * vn) go(t, tpr, nv, layer, integral_constant<int, kWhole>());
            else if (p.desc.C >= vn) go(t, tpr, nv, layer, integral_constant<int, kTail>());
            else if constexpr (decltype(tpr)::value == 4) go(t, tpr, nv, layer, integral_constant<int, kShort>());
        };
        auto wide = [&](auto tpr) {
            constexpr int most = (FWD || decltype(tpr)::value == 512 ? 16 : 8) / vn;
            if (sh.nv == 1) with(tpr, integral_constant<int, 1>());
            else if constexpr (most >= 2) {
                if (sh.nv == 2) with(tpr, integral_constant<int, 2>());
                else if constexpr (most >= 4) with(tpr, integral_constant<int, 4>());
            }
        };
        switch (sh.tpr) {
            case 4: with(integral_constant<int, 4>(), integral_constant<int, 1>()); break;
            case 16: with(integral_constant<int, 16>(), integral_constant<int, 1>()); break;
            case 64: wide(integral_constant<int, 64>()); break;
            case 128: wide(integral_constant<int, 128>()); break;
            case 256: wide(integral_constant<int, 256>()); break;
            default: wide(integral_constant<int, 512>());
        }
    };
    auto kind = [&](auto t) {
        if (p.desc.kind == LLSA_NORM_LAYER) shape(t, std::true_type());
        else shape(t, std::false_type());
    };
    if (p.desc.dtype == LLSA_F32) kind(float());
    else kind(__bf16());
}

hipError_t launch_norm_forward(const NormPlan &p, NormArgs a, hipStream_t s) {
    const dim3 grid(p.fwd.blocks, p.desc.batch);
    norm_dispatch<true>(p, p.fwd, [&](auto t, auto tpr, auto nv, auto layer, auto row) {
        constexpr int threads = norm_threads(decltype(tpr)::value);
        norm_fwd_kernel<decltype(t), decltype(tpr)::value, decltype(nv)::value, decltype(layer)::value, decltype(row)::value><<<grid, threads, 0, s>>>(a);
    });
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormPlan &p, NormArgs a, hipStream_t s) {
    const dim3 grid(p.bwd.blocks, p.desc.batch);
    a.blocks = p.bwd.blocks;
    norm_dispatch<false>(p, p.bwd, [&](auto t, auto tpr, auto nv, auto layer, auto row) {
        constexpr int threads = norm_threads(decltype(tpr)::value);
        norm_bwd_kernel<decltype(t), decltype(tpr)::value, decltype(nv)::value, decltype(layer)::value, decltype(row)::value><<<grid, threads, 0, s>>>(a);
    });
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.part) return e;
    norm_sums_kernel<<<dim3((a.C + 15) / 16, 3), 1024, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace llsa

using namespace llsa;

struct llsa_norm_plan_s { NormPlan p; };

static bool norm_misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
template <class... P> static bool norm_any_misaligned(P... ptrs) { return (norm_misaligned(ptrs) || ...); }
// gains and modulation vectors: an element's alignment, since they may be pieces of one projection
template <class... P> static bool norm_any_off(size_t a, P... ptrs) { return (((reinterpret_cast<uintptr_t>(ptrs) & (a - 1)) != 0) || ...); }

extern "C" {

llsa_status llsa_norm_plan(const llsa_norm_desc *desc, llsa_norm_plan_t **out) {
    if (!desc || !out) return LLSA_ERR_NULL;
    *out = nullptr;
    const llsa_norm_desc &d = *desc;
    if (d.batch < 1 || d.N < 1 || d.C < 1 || !(d.eps >= 0.f)) return LLSA_ERR_BAD_SHAPE;
    if (d.mod_stride != 0 && d.mod_stride < d.C) return LLSA_ERR_BAD_SHAPE;
    if ((d.dtype != LLSA_F32 && d.dtype != LLSA_BF16) || (d.mod_dtype != LLSA_F32 && d.mod_dtype != LLSA_BF16)) return LLSA_ERR_UNSUPPORTED;
    if (d.kind != LLSA_NORM_RMS && d.kind != LLSA_NORM_LAYER) return LLSA_ERR_UNSUPPORTED;
    if (d.C > 8192 || d.batch > 65535 || d.N > ((int64_t)1 << 40) || d.mod_stride > ((int64_t)1 << 40)) return LLSA_ERR_UNSUPPORTED;
    llsa_norm_plan_s *h = new (std::nothrow) llsa_norm_plan_s;
    if (!h) return LLSA_ERR_RUNTIME;
    h->p = NormPlan{};
    h->p.desc = d;
    norm_layout(h->p);
    *out = h;
    return LLSA_OK;
}

void llsa_norm_plan_destroy(llsa_norm_plan_t *plan) { delete plan; }

size_t llsa_norm_workspace_bytes(const llsa_norm_plan_t *plan) { return plan ? (plan->p.ws + 255) & ~(size_t)255 : 0; }

static NormArgs norm_args(const NormPlan &p) {
    NormArgs a{};
    a.N = p.desc.N;
    a.C = p.desc.C;
    a.batch = p.desc.batch;
    a.mod_stride = p.desc.mod_stride;
    a.mod_f32 = p.desc.mod_dtype == LLSA_F32;
    a.eps = p.desc.eps;
    a.alpha = p.desc.residual_scale;
    a.inv_c = 1.f / (float)p.desc.C;
    return a;
}

llsa_status llsa_norm_forward(const llsa_norm_plan_t *plan, const void *x, const void *branch, const float *gain_branch, const void *gate,
                              const float *gain, const void *scale, const void *shift, void *x_out, void *y, float *stats,
                              void *hip_stream) {
    if (!plan || !x || (branch && !x_out) || (!branch && (gain_branch || gate)) || (!y && (gain || scale || shift)) || (!branch && !y))
        return LLSA_ERR_NULL;
    const size_t mod = plan->p.desc.mod_dtype == LLSA_F32 ? 4 : 2;
    if (norm_any_misaligned(x, branch, x_out, y, stats) || norm_any_off(4, gain_branch, gain) || norm_any_off(mod, gate, scale, shift))
        return LLSA_ERR_BAD_SHAPE;
    NormArgs a = norm_args(plan->p);
    a.x = static_cast<const char *>(x);
    a.branch = static_cast<const char *>(branch);
    a.gain_branch = gain_branch;
    a.gate = static_cast<const char *>(gate);
    a.gain = gain;
    a.scale = static_cast<const char *>(scale);
    a.shift = static_cast<const char *>(shift);
    a.x_out = static_cast<char *>(x_out);
    a.y = static_cast<char *>(y);
    a.stats = stats;
    return launch_norm_forward(plan->p, a, (hipStream_t)hip_stream) == hipSuccess ? LLSA_OK : LLSA_ERR_RUNTIME;
}

llsa_status llsa_norm_backward(const llsa_norm_plan_t *plan, const void *x_out, const void *branch, const float *gain_branch,
                               const void *gate, const float *gain, const void *scale, const float *stats, const void *dy,
                               const void *dx_out, void *dx, void *dbranch, float *dgain_branch, float *dgate, float *dgain,
                               float *dscale, float *dshift, void *workspace, void *hip_stream) {
    if (!plan || !x_out || !stats || !dx || (!dy && !dx_out) || (branch != nullptr) != (dbranch != nullptr)) return LLSA_ERR_NULL;
    if ((!branch && (gain_branch || gate || dgate)) || (!gain_branch && dgain_branch) || (!dy && (gain || scale || dgain || dscale || dshift))) return LLSA_ERR_NULL;
    const bool sums = dgain_branch || dgate || dgain || dscale || dshift;
    if (sums && !workspace) return LLSA_ERR_NULL;
    const size_t mod = plan->p.desc.mod_dtype == LLSA_F32 ? 4 : 2;
    if (norm_any_misaligned(x_out, branch, stats, dy, dx_out, dx, dbranch) || norm_any_off(4, gain_branch, gain, dgain_branch, dgate, dgain, dscale, dshift) ||
        norm_any_off(mod, gate, scale) || norm_any_off(256, workspace))
        return LLSA_ERR_BAD_SHAPE;
    NormArgs a = norm_args(plan->p);
    a.x = static_cast<const char *>(x_out);
    a.branch = static_cast<const char *>(branch);
    a.gain_branch = gain_branch;
    a.gate = static_cast<const char *>(gate);
    a.gain = gain;
    a.scale = static_cast<const char *>(scale);
    a.stats = const_cast<float *>(stats);
    a.dy = static_cast<const char *>(dy);
    a.dx_out = static_cast<const char *>(dx_out);
    a.dx = static_cast<char *>(dx);
    a.dbranch = static_cast<char *>(dbranch);
    a.dgain_branch = dgain_branch;
    a.dgate = dgate;
    a.dgain = dgain;
    a.dscale = dscale;
    a.dshift = dshift;
    a.part = sums ? static_cast<float *>(workspace) : nullptr;
    return launch_norm_backward(plan->p, a, (hipStream_t)hip_stream) == hipSuccess ? LLSA_OK : LLSA_ERR_RUNTIME;
}

}  // extern "C"
