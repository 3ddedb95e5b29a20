// Gradient of the layer glue (QK-Norm and RoPE), Q and K in one pass.  Per row, with x^ = x r, r = 1 / sqrt(mean x^2 + eps):
//   dy[2i] = g[2i] cos + g[2i+1] sin, dy[2i+1] = g[2i+1] cos - g[2i] sin        (the rotation's transpose; g: gradient of Xout)
//   dgamma += dy x^;   p = dy gamma;   dx = r (p - x^ mean(p x^))
// A thread has 16 bytes of channels of one token and walks over the heads, Q and K in turn, so that a token's cosines and sines are read once for
// all of them; the d / (16 / element size) threads of a row are neighbouring lanes.  Bytes bound it, three tensors' worth for each of Q and K:
// 16 heads x 65536 tokens, d = 64, bf16, 153 us (822 MB, 5.4 TB/s) and 5 for the sums; 16 x 4096 12 and 2.7.
// dgamma: a thread's sums over its heads, then over the workgroup's tokens, to the workspace; a second launch adds the workgroups in a fixed order.
#include <algorithm>
#include <type_traits>

#include "lanes.h"
#include "llsa_internal.h"

namespace llsa {

struct GlueBwdArgs {
    const char *x[2], *g[2];
    char *dx[2];
    const float *gamma[2], *cos_t, *sin_t;
    float *part, *dgamma[2];        // part: [workgroup][2][d]
    int64_t N;
    int32_t bh, wgs;
    float eps, inv_d;
};

template <class T> __device__ __forceinline__ void g_unpack(const uint4 &v, float *x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            x[i] = __uint_as_float(w[i]);
        } else {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}
template <class T> __device__ __forceinline__ uint4 g_pack(const float *x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            w[i] = __float_as_uint(x[i]);
        } else {
            union { __bf16 h[2]; uint32_t u; } p;
            p.h[0] = (__bf16)x[2 * i];
            p.h[1] = (__bf16)x[2 * i + 1];
            w[i] = p.u;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// grid: (tokens, slices of the heads)
template <class T, int D> __global__ void __launch_bounds__(256) glue_bwd_kernel(GlueBwdArgs a) {
    constexpr int VN = 16 / sizeof(T), VPR = D / VN, TOK = 256 / VPR;
    __shared__ float lds[2][TOK][D];
    const int cv = threadIdx.x % VPR, tt = threadIdx.x / VPR;
    const int64_t tok = (int64_t)blockIdx.x * TOK + tt;
    const bool in = tok < a.N;
    float cs[VN / 2], sn[VN / 2], gam[2][VN], sum[2][VN];
#pragma unroll
    for (int e = 0; e < VN / 2; ++e) {
        const int64_t at = (in ? tok : 0) * (D / 2) + cv * (VN / 2) + e;
        cs[e] = a.cos_t[at];
        sn[e] = a.sin_t[at];
    }
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int e = 0; e < VN; ++e) {
            gam[y][e] = a.gamma[y][cv * VN + e];
            sum[y][e] = 0.f;
        }
    for (int h = blockIdx.y; h < a.bh; h += gridDim.y) {
        const int64_t at = ((int64_t)h * a.N + (in ? tok : 0)) * (D * sizeof(T)) + cv * 16;
        uint4 xv[2], gv[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            xv[y] = *reinterpret_cast<const uint4 *>(a.x[y] + at);
            gv[y] = *reinterpret_cast<const uint4 *>(a.g[y] + at);
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            float x[VN], g[VN], dy[VN], ss = 0.f, px = 0.f;
            g_unpack<T>(xv[y], x);
            g_unpack<T>(gv[y], g);
#pragma unroll
            for (int e = 0; e < VN / 2; ++e) {
                dy[2 * e] = g[2 * e] * cs[e] + g[2 * e + 1] * sn[e];
                dy[2 * e + 1] = g[2 * e + 1] * cs[e] - g[2 * e] * sn[e];
            }
#pragma unroll
            for (int e = 0; e < VN; ++e) {
                ss = fmaf(x[e], x[e], ss);
                px = fmaf(dy[e] * gam[y][e], x[e], px);
            }
            ss = lanes_sum<VPR>(ss);
            px = lanes_sum<VPR>(px);
            const float r = 1.f / sqrtf(fmaf(ss, a.inv_d, a.eps)), m = px * r * a.inv_d;
#pragma unroll
            for (int e = 0; e < VN; ++e) {
                const float xh = x[e] * r;
                sum[y][e] = fmaf(dy[e], xh, sum[y][e]);
                x[e] = r * fmaf(-xh, m, dy[e] * gam[y][e]);
            }
            if (in) *reinterpret_cast<uint4 *>(a.dx[y] + at) = g_pack<T>(x);
        }
    }
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int e = 0; e < VN; ++e) lds[y][tt][cv * VN + e] = in ? sum[y][e] : 0.f;
    __syncthreads();
    if ((int)threadIdx.x < 2 * D) {
        const int y = threadIdx.x / D, c = threadIdx.x % D;
        float s = 0.f;
        for (int i = 0; i < TOK; ++i) s += lds[y][i][c];
        a.part[((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * D + threadIdx.x] = s;
    }
}

// The workgroups' sums added up: 128 slices of 8 columns a workgroup, each slice every 128th workgroup's, then the slices in order.
template <int D> __global__ void __launch_bounds__(1024) glue_sums_kernel(GlueBwdArgs a) {
    __shared__ float lds[128][9];
    const int col = threadIdx.x & 7, c = blockIdx.x * 8 + col, slice = threadIdx.x >> 3;
    float s = 0.f;
    for (int w0 = slice; w0 < a.wgs; w0 += 1024) {           // eight on their way at once
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = a.part[(int64_t)min(w0 + 128 * j, a.wgs - 1) * 2 * D + c];
#pragma unroll
        for (int j = 0; j < 8; ++j) s += w0 + 128 * j < a.wgs ? v[j] : 0.f;
    }
    lds[slice][col] = s;
    __syncthreads();
    if (slice < 8) {                                         // 16 slices each, then those eight
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += lds[slice * 16 + i][col];
#pragma unroll
        for (int o = 8; o < 64; o <<= 1) s += __shfl_xor(s, o, 64);
        if (slice == 0) a.dgamma[c / D][c % D] = s;
    }
}

// Workgroups over tokens, and into how many slices the heads are cut: 4 workgroups a CU, at least 2 heads a slice
static void glue_bwd_grid(const Plan &p, unsigned *x, unsigned *y) {
    const int tok = 256 / (p.d / (16 / p.elt));
    *x = (unsigned)((p.N + tok - 1) / tok);
    *y = (unsigned)std::max<int64_t>(1, std::min<int64_t>((p.bh + 1) / 2, (1024 + *x - 1) / *x));
}

size_t glue_backward_bytes(const Plan &p) {
    unsigned x, y;
    glue_bwd_grid(p, &x, &y);
    return ((size_t)x * y * 2 * p.d * sizeof(float) + 255) & ~(size_t)255;
}

hipError_t launch_glue_backward(const Plan &p, const void *Qpre, const void *Kpre, const float *gamma_q, const float *gamma_k, const float *cos_t,
                                const float *sin_t, float eps, const void *dQ, const void *dK, void *dQpre, void *dKpre, float *dgamma_q, float *dgamma_k,
                                void *ws, hipStream_t s) {
    unsigned gx, gy;
    glue_bwd_grid(p, &gx, &gy);
    GlueBwdArgs a{};
    a.x[0] = static_cast<const char *>(Qpre);  a.x[1] = static_cast<const char *>(Kpre);
    a.g[0] = static_cast<const char *>(dQ);    a.g[1] = static_cast<const char *>(dK);
    a.dx[0] = static_cast<char *>(dQpre);      a.dx[1] = static_cast<char *>(dKpre);
    a.gamma[0] = gamma_q;                      a.gamma[1] = gamma_k;
    a.dgamma[0] = dgamma_q;                    a.dgamma[1] = dgamma_k;
    a.cos_t = cos_t;
    a.sin_t = sin_t;
    a.part = static_cast<float *>(ws);
    a.N = p.N;
    a.bh = p.bh;
    a.wgs = (int)(gx * gy);
    a.eps = eps;
    a.inv_d = 1.f / (float)p.d;
    auto go = [&](auto d) {
        constexpr int D = decltype(d)::value;
        if (p.elt == 4) glue_bwd_kernel<float, D><<<dim3(gx, gy), 256, 0, s>>>(a);
        else            glue_bwd_kernel<__bf16, D><<<dim3(gx, gy), 256, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        glue_sums_kernel<D><<<2 * D / 8, 1024, 0, s>>>(a);
        return hipGetLastError();
    };
    switch (p.d) {
        case 16: return go(std::integral_constant<int, 16>());
        case 32: return go(std::integral_constant<int, 32>());
        case 64: return go(std::integral_constant<int, 64>());
        default: return go(std::integral_constant<int, 128>());
    }
}

}  // namespace llsa
