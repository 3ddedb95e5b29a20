// The norms between two blocks with gate and residual, forward and backward: one pass over the rows, each held in registers by 16, 64, 256 or
// 512 threads of a workgroup (at most 16 channels a thread), so that a row is read once and written once.  What varies by channel only (the gains, and the
// modulation of the batch entry that a workgroup belongs to) stays in registers over all rows of the workgroup, combined:
//   y = n(x') ga + sh, x' = x + gz n(branch)       with ga = gain (1 + scale), sh = shift, gz = alpha gate gain_branch.
// Backward, per row, with h^ = n(x'), u = n(branch) (or the branch itself):
//   p = dy ga;  dh = r (p - h^ mean(p h^) [- mean p]) + dx_out;   w = gz dh;  db = r_b (w - u mean(w u) [- mean w])  (no norm: w)
// and per channel and batch entry three sums over the rows: E = sum dy h^, T = sum dy, F = sum dh u, from which
//   dgain = sum_b (1 + scale) E, dscale = gain E, dshift = T, dgate = alpha gain_branch F, dgain_branch = alpha sum_b gate F.
// A thread keeps its channels' sums over all its rows; the workgroups' sums go to the workspace and a second launch adds them in a fixed order.
#include "norm.h"

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
// channels c .. c + n - 1 of a row of C, zeros beyond it
template <class T> __device__ __forceinline__ void n_load(const T *row, int c, int C, float *x) {
    constexpr int n = NVec<T>::n;
    if (c + n <= C) {
        n_unpack<T>(*reinterpret_cast<const typename NVec<T>::Raw *>(row + c), x);
    } else {
#pragma unroll
        for (int e = 0; e < n; ++e) x[e] = c + e < C ? n_get(row + c + e) : 0.f;
    }
}
template <class T> __device__ __forceinline__ void n_store(T *row, int c, int C, const float *x) {
    constexpr int n = NVec<T>::n;
    typename NVec<T>::Raw r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            r.w[i] = __float_as_uint(x[i]);
        } else {
            union { __bf16 h[2]; uint32_t u; } w;
            w.h[0] = (__bf16)x[2 * i];
            w.h[1] = (__bf16)x[2 * i + 1];
            r.w[i] = w.u;
        }
    }
    if (c + n <= C) {
        *reinterpret_cast<typename NVec<T>::Raw *>(row + c) = r;
    } else {
#pragma unroll
        for (int e = 0; e < n; ++e)
            if (c + e < C) row[c + e] = (T)x[e];
    }
}
// a modulation vector's channel, of either type; `none` where it was not given
__device__ __forceinline__ float n_mod(const char *m, int f32, int64_t at, float none) {
    return !m ? none : f32 ? reinterpret_cast<const float *>(m)[at] : n_get(reinterpret_cast<const __bf16 *>(m) + at);
}

// Sums over the TPR threads of a row, K at once, the result in each of them.  lds: K floats a wave, not read or written by another call until
// a barrier (callers take turns with two of them).
template <int TPR, int K> __device__ __forceinline__ void row_sums(float (&v)[K], float *lds) {
#pragma unroll
    for (int o = (TPR < 64 ? TPR : 64) / 2; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], o, 64);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        const int w = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) lds[k * W + w] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) v[k] += lds[k * W + i];
        }
    }
}

// mean and 1 / deviation of a row held as x (zeros beyond C)
template <int TPR, int E, bool LAYER>
__device__ __forceinline__ void row_stats(const float (&x)[E], const bool (&in)[E], float inv_c, float eps, float *lds, float &m, float &r) {
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
        const float d = in[e] ? x[e] - m : 0.f;
        s[0] = fmaf(d, d, s[0]);
    }
    row_sums<TPR, 1>(s, lds + 32);
    r = 1.f / sqrtf(fmaf(s[0], inv_c, eps));
}

template <class T, int TPR, int NV, bool LAYER>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) norm_fwd_kernel(NormArgs a) {
    constexpr int VN = NVec<T>::n, E = NV * VN, GP = TPR > 256 ? 1 : 256 / TPR;
    __shared__ float lds[4][32];
    const int t = threadIdx.x % TPR, b = blockIdx.y;
    int ch[NV];
    bool in[E];
    float gz[E], ga[E], sh[E];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        ch[k] = (k * TPR + t) * VN;
#pragma unroll
        for (int e = 0; e < VN; ++e) {
            const int c = ch[k] + e, i = k * VN + e;
            in[i] = c < a.C;
            const int64_t at = b * a.mod_stride + c;
            gz[i] = in[i] && a.branch ? a.alpha * n_mod(a.gate, a.mod_f32, at, 1.f) * (a.gain_branch ? a.gain_branch[c] : 1.f) : 0.f;
            ga[i] = in[i] && a.y ? (a.gain ? a.gain[c] : 1.f) * (1.f + n_mod(a.scale, a.mod_f32, at, 0.f)) : 0.f;
            sh[i] = in[i] && a.y ? n_mod(a.shift, a.mod_f32, at, 0.f) : 0.f;
        }
    }
    for (int64_t n = (int64_t)blockIdx.x * GP + threadIdx.x / TPR; n < a.N; n += (int64_t)gridDim.x * GP) {
        const int64_t row = b * a.N + n;
        float x[E], st[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NV; ++k) n_load(reinterpret_cast<const T *>(a.x) + row * a.C, ch[k], a.C, x + k * VN);
        if (a.branch) {
            float u[E];
#pragma unroll
            for (int k = 0; k < NV; ++k) n_load(reinterpret_cast<const T *>(a.branch) + row * a.C, ch[k], a.C, u + k * VN);
            if (a.gain_branch) {
                row_stats<TPR, E, LAYER>(u, in, a.inv_c, a.eps, lds[0], st[2], st[3]);
#pragma unroll
                for (int e = 0; e < E; ++e) u[e] = (u[e] - st[2]) * st[3];
            }
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = (float)(T)fmaf(gz[e], u[e], x[e]);
#pragma unroll
            for (int k = 0; k < NV; ++k) n_store(reinterpret_cast<T *>(a.x_out) + row * a.C, ch[k], a.C, x + k * VN);
        }
        if (a.y) {
            row_stats<TPR, E, LAYER>(x, in, a.inv_c, a.eps, lds[2], st[0], st[1]);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = fmaf((x[e] - st[0]) * st[1], ga[e], sh[e]);
#pragma unroll
            for (int k = 0; k < NV; ++k) n_store(reinterpret_cast<T *>(a.y) + row * a.C, ch[k], a.C, x + k * VN);
        }
        if (a.stats && t == 0) *reinterpret_cast<float4 *>(a.stats + 4 * row) = make_float4(st[0], st[1], st[2], st[3]);
        if constexpr (TPR > 64) __syncthreads();             // the next row's sums go where this one's are read
    }
}

template <class T, int TPR, int NV, bool LAYER>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) norm_bwd_kernel(NormArgs a) {
    constexpr int VN = NVec<T>::n, E = NV * VN, GP = TPR > 256 ? 1 : 256 / TPR;
    constexpr int SPAN = TPR * E;                            // channels that the threads of a row cover
    __shared__ float lds[2][32];
    __shared__ float sums[GP > 1 ? 3 * SPAN : 1];
    const int t = threadIdx.x % TPR, b = blockIdx.y;
    int ch[NV];
    float gz[E], ga[E], sE[E], sT[E], sF[E];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        ch[k] = (k * TPR + t) * VN;
#pragma unroll
        for (int e = 0; e < VN; ++e) {
            const int c = ch[k] + e, i = k * VN + e;
            const int64_t at = b * a.mod_stride + c;
            const bool in = c < a.C;
            gz[i] = in && a.branch ? a.alpha * n_mod(a.gate, a.mod_f32, at, 1.f) * (a.gain_branch ? a.gain_branch[c] : 1.f) : 0.f;
            ga[i] = in ? (a.gain ? a.gain[c] : 1.f) * (1.f + n_mod(a.scale, a.mod_f32, at, 0.f)) : 0.f;
            sE[i] = sT[i] = sF[i] = 0.f;
        }
    }
    for (int64_t n = (int64_t)blockIdx.x * GP + threadIdx.x / TPR; n < a.N; n += (int64_t)gridDim.x * GP) {
        const int64_t row = b * a.N + n, at = row * a.C;
        float d[E], u[E];                                    // gradient of x'; normed branch
        const float4 st = *reinterpret_cast<const float4 *>(a.stats + 4 * row);
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] = 0.f;
        if (a.branch)
#pragma unroll
            for (int k = 0; k < NV; ++k) n_load(reinterpret_cast<const T *>(a.branch) + at, ch[k], a.C, u + k * VN);
        if (a.dx_out)
#pragma unroll
            for (int k = 0; k < NV; ++k) n_load(reinterpret_cast<const T *>(a.dx_out) + at, ch[k], a.C, d + k * VN);
        if (a.dy) {
            float x[E], g[E];
#pragma unroll
            for (int k = 0; k < NV; ++k) n_load(reinterpret_cast<const T *>(a.x) + at, ch[k], a.C, x + k * VN);
#pragma unroll
            for (int k = 0; k < NV; ++k) n_load(reinterpret_cast<const T *>(a.dy) + at, ch[k], a.C, g + k * VN);
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[e] = (x[e] - st.x) * st.y;                 // beyond C: a value that only meets zeros
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
            for (int e = 0; e < E; ++e) d[e] = fmaf(st.y, fmaf(-x[e], m[0], g[e]) - m[1], d[e]);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) n_store(reinterpret_cast<T *>(a.dx) + at, ch[k], a.C, d + k * VN);
        if (a.branch) {
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (a.gain_branch) u[e] = (u[e] - st.z) * st.w;
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
                for (int e = 0; e < E; ++e) d[e] = (fmaf(-u[e], m[0], d[e]) - m[1]) * st.w;
            }
#pragma unroll
            for (int k = 0; k < NV; ++k) n_store(reinterpret_cast<T *>(a.dbranch) + at, ch[k], a.C, d + k * VN);
        }
        if constexpr (TPR > 64) __syncthreads();             // the next row's sums go where this one's are read
    }
    if (!a.part) return;
    // the workgroup's sums: its GP rows at a time add theirs in turn
    if constexpr (GP > 1) {
#pragma unroll 1
        for (int w = 0; w < GP; ++w) {
            if ((int)threadIdx.x / TPR == w)
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
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < VN; ++e) {
            const int c = ch[k] + e, i = k * VN + e;
            if (c < a.C) {
                part[c] = sE[i];
                part[a.C + c] = sT[i];
                part[2 * a.C + c] = sF[i];
            }
        }
}

// The workgroups' sums added up: 16 slices of 64 channels a workgroup, each slice every 16th workgroup's, then the slices in order.
__global__ void __launch_bounds__(1024) norm_sums_kernel(NormArgs a) {
    __shared__ float lds[3][16][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
    const bool in = c < a.C;
    float dgain = 0.f, dgb = 0.f, shared[3] = {0.f, 0.f, 0.f};
    const float gain = in && a.gain ? a.gain[c] : 1.f, gb = in && a.gain_branch ? a.gain_branch[c] : 1.f;
    for (int b = 0; b < a.batch; ++b) {
        float s[3] = {0.f, 0.f, 0.f};
        if (in)
            for (int w = slice; w < a.blocks; w += 16) {
                const float *p = a.part + ((int64_t)b * a.blocks + w) * 3 * a.C + c;
#pragma unroll
                for (int k = 0; k < 3; ++k) s[k] += p[k * a.C];
            }
#pragma unroll
        for (int k = 0; k < 3; ++k) lds[k][slice][threadIdx.x & 63] = s[k];
        __syncthreads();
        if (slice == 0 && in) {
            float v[3];
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                v[k] = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) v[k] += lds[k][i][threadIdx.x];
            }
            const int64_t at = b * a.mod_stride + c;
            dgain = fmaf(1.f + n_mod(a.scale, a.mod_f32, at, 0.f), v[0], dgain);
            dgb = fmaf(a.alpha * n_mod(a.gate, a.mod_f32, at, 1.f), v[2], dgb);
#pragma unroll
            for (int k = 0; k < 3; ++k) shared[k] += v[k];
            if (a.mod_stride || b == a.batch - 1) {
                const int64_t to = (a.mod_stride ? (int64_t)b * a.C : 0) + c;
                if (a.dscale) a.dscale[to] = gain * shared[0];
                if (a.dshift) a.dshift[to] = shared[1];
                if (a.dgate) a.dgate[to] = a.alpha * gb * shared[2];
#pragma unroll
                for (int k = 0; k < 3; ++k) shared[k] = 0.f;
            }
        }
        __syncthreads();
    }
    if (slice == 0 && in) {
        if (a.dgain) a.dgain[c] = dgain;
        if (a.dgain_branch) a.dgain_branch[c] = dgb;
    }
}

// The fewest threads a row that hold it with at most 16 channels each.
void norm_layout(NormPlan &p) {
    const llsa_norm_desc &d = p.desc;
    const int vn = d.dtype == LLSA_F32 ? 4 : 8, vec = (d.C + vn - 1) / vn, most = 16 / vn;
    p.tpr = vec <= 16 ? 16 : vec <= 64 * 2 ? 64 : vec <= 256 * most ? 256 : 512;
    p.nv = (vec + p.tpr - 1) / p.tpr;
    if (p.nv == 3) p.nv = 4;
    const int64_t groups = p.tpr >= 256 ? 1 : 256 / p.tpr, all = (d.N + groups - 1) / groups;
    auto blocks = [&](int64_t target) {
        target = (target + d.batch - 1) / d.batch;
        return (int)(all < target ? all : target);
    };
    p.fwd_blocks = blocks(2048);
    p.bwd_blocks = blocks(1024);
    p.ws = (size_t)d.batch * p.bwd_blocks * 3 * d.C * sizeof(float);
}

template <class F> static void norm_dispatch(const NormPlan &p, F go) {
    auto shape = [&](auto t, auto layer) {
        auto with = [&](auto tpr, auto nv) { go(t, tpr, nv, layer); };
        using std::integral_constant;
        auto wide = [&](auto tpr) {
            if (p.nv == 1) with(tpr, integral_constant<int, 1>());
            else if (p.nv == 2 || sizeof(t) == 2) with(tpr, integral_constant<int, 2>());
            else if constexpr (sizeof(t) == 4) with(tpr, integral_constant<int, 4>());
        };
        if (p.tpr == 16) with(integral_constant<int, 16>(), integral_constant<int, 1>());
        else if (p.tpr == 64) wide(integral_constant<int, 64>());
        else if (p.tpr == 256) wide(integral_constant<int, 256>());
        else wide(integral_constant<int, 512>());
    };
    auto kind = [&](auto t) {
        if (p.desc.kind == LLSA_NORM_LAYER) shape(t, std::true_type());
        else shape(t, std::false_type());
    };
    if (p.desc.dtype == LLSA_F32) kind(float());
    else kind(__bf16());
}

hipError_t launch_norm_forward(const NormPlan &p, NormArgs a, hipStream_t s) {
    const dim3 grid(p.fwd_blocks, p.desc.batch);
    norm_dispatch(p, [&](auto t, auto tpr, auto nv, auto layer) {
        constexpr int threads = decltype(tpr)::value > 256 ? decltype(tpr)::value : 256;
        norm_fwd_kernel<decltype(t), decltype(tpr)::value, decltype(nv)::value, decltype(layer)::value><<<grid, threads, 0, s>>>(a);
    });
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormPlan &p, NormArgs a, hipStream_t s) {
    const dim3 grid(p.bwd_blocks, p.desc.batch);
    a.blocks = p.bwd_blocks;
    norm_dispatch(p, [&](auto t, auto tpr, auto nv, auto layer) {
        constexpr int threads = decltype(tpr)::value > 256 ? decltype(tpr)::value : 256;
        norm_bwd_kernel<decltype(t), decltype(tpr)::value, decltype(nv)::value, decltype(layer)::value><<<grid, threads, 0, s>>>(a);
    });
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.part) return e;
    norm_sums_kernel<<<(a.C + 63) / 64, 1024, 0, s>>>(a);
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
