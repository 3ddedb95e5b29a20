// C ABI of dense attention: host plan and launch sequences.  Nothing is allocated on the device and the host never waits.
#include <limits.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>

#include "dense.h"

namespace llsa {

static size_t dense_align(size_t x) { return (x + 255) & ~(size_t)255; }

// Strides as the kernels take them (bytes); false: not a layout that they take.
static bool dense_strides(const int64_t (&st)[3], int64_t batch, int64_t heads, int64_t N, int d, int elt, DenseStrides *out) {
    int64_t e[3] = {st[0], st[1], st[2]};
    const int64_t n[3] = {batch, heads, N};
    if (!e[0] && !e[1] && !e[2]) { e[2] = d; e[1] = N * d; e[0] = heads * N * d; }
    for (int i = 0; i < 3; ++i) {
        if (n[i] == 1) e[i] = 0;                             // a stride nobody takes a step with
        if (e[i] < 0 || e[i] > ((int64_t)1 << 40) || (e[i] * elt) % 16) return false;
    }
    *out = {e[0] * elt, e[1] * elt, e[2] * elt};
    return true;
}

// Do rows that are written with these strides lie apart?  (Dimensions in the order of their strides, each past the one before.)
static bool dense_apart(const DenseStrides &st, int64_t batch, int64_t heads, int64_t N, int row_bytes) {
    std::pair<int64_t, int64_t> v[3] = {{st.batch, batch}, {st.head, heads}, {st.token, N}};
    std::sort(v, v + 3);
    int64_t span = row_bytes;
    for (const auto &x : v) {
        if (x.second == 1) continue;
        if (x.first < span) return false;
        span += x.first * (x.second - 1);
    }
    return true;
}

// Tiles of 128 rows (the other axis is brought in once for four waves' 32 each) keep the matrix units busiest; tiles of 32, whose waves share out the other axis, are for what
// leaves half a tile or half the CUs empty otherwise.  The other axis is cut only where there are fewer tiles than CUs, not into pieces of less than 512 rows or
// keys: the partial sums are written and read once more (16 x 2048 tokens, d = 64, 256 tiles: forward 47.8 us in two pieces, 26.3 in one).  Causal tiles differ, and the longest takes
// as long as everything where all are resident at once: long ones are cut up to twice as many tiles (key tiles of 3 x 16 heads, 4 key heads, x 1999 tokens, d = 128, 125 steps:
// backward 261 -> 182 us with lengths of 1999, 1500 and 700, 277 -> 263 without; 32 steps, 16 x 2048: 68.8 uncut, 86 in two).
DenseShape dense_shape(const DensePlan &p, int64_t axis, int64_t other) {
    DenseShape r;
    const int64_t groups = (int64_t)p.desc.batch * p.desc.kv_heads, wide = groups * ((axis + 127) / 128), pieces = std::max<int64_t>(1, other / 512);
    r.narrow = axis <= 64 || wide * pieces < 128;
    const int step = dense_step(p.desc.d * p.elt, r.narrow);
    const int64_t tiles = r.narrow ? groups * ((axis + 31) / 32) : wide, steps = (other + step - 1) / step, least = 512 / step;
    const int64_t target = r.narrow || (p.desc.causal && steps >= 96) ? 512 : 256;
    const int64_t want = r.narrow ? (target + tiles - 1) / tiles : std::max<int64_t>(1, target / tiles);
    r.chunk = (int)std::max((steps + want - 1) / want, least);
    r.splits = (int)((steps + r.chunk - 1) / r.chunk);
    return r;
}

// Eight waves a tile, two for each 32 rows, where a CU has one tile anyway (8 x 4096 tokens, d = 128: forward 89 -> 70 us, backward 252 -> 219; 2 x 16 x 1024, d = 64, 51 -> 48 backward) and walks over
// eight steps at least (8 x 16 heads of 256, four steps: 25 -> 27), or the longest of causal tiles, of 32 steps, decides (16 x 4096, d = 64, 512 tiles: 60 -> 54 and 169 -> 151; 4 x 16384
// 212 -> 191 and 627 -> 513; 512 tiles of 16 steps 64 -> 70, of 4 32 -> 46 backward).  Beyond that two workgroups of four a CU do better: they wait for each other less (756 tiles, d = 128: 58 us,
// paired 66).
bool dense_paired(const DensePlan &p, const DenseShape &shape, int64_t axis) {
    const int64_t tiles = (int64_t)p.desc.batch * p.desc.kv_heads * ((axis + 127) / 128) * shape.splits;
    return shape.chunk >= 8 && tiles <= (p.desc.causal && shape.chunk >= 32 ? 512 : 256);
}

DenseGrid dense_grid(const DensePlan &p, int64_t rows, const DenseShape &shape, int row_floats, float *part) {
    DenseGrid g;
    memset(&g, 0, sizeof(g));
    g.rows = rows;
    g.groups = (uint32_t)(p.desc.batch * p.desc.kv_heads);
    g.splits = shape.splits;
    g.chunk = shape.chunk;
    const int64_t tile = dense_tile(shape.narrow), tiles = (rows + tile - 1) / tile;
    g.by_tiles = FastDiv(tiles);
    g.by_splits = FastDiv(g.splits);
    g.by_rest = FastDiv((int64_t)g.groups * g.splits);
    g.by_heads = FastDiv((int64_t)p.desc.kv_heads * g.splits);
    g.wgs = (uint32_t)(tiles * g.groups * g.splits);
    g.part = part;
    if (g.splits > 1) g.stat = part + (int64_t)g.splits * g.groups * rows * row_floats;
    return g;
}

size_t dense_part_bytes(const DensePlan &p, int64_t rows, const DenseShape &shape, int row_floats) {
    return shape.splits == 1 ? 0 : dense_align((size_t)shape.splits * p.desc.batch * p.desc.kv_heads * rows * row_floats * sizeof(float));
}

static llsa_status build_dense_plan(const llsa_dense_desc &d, DensePlan &p) {
    memset(&p, 0, sizeof(p));
    p.desc = d;
    if (d.batch < 1 || d.heads < 1 || d.kv_heads < 1 || d.Nq < 1 || d.Nkv < 1) return LLSA_ERR_BAD_SHAPE;
    if (d.heads % d.kv_heads) return LLSA_ERR_BAD_SHAPE;
    if (d.dtype != LLSA_F32 && d.dtype != LLSA_BF16) return LLSA_ERR_UNSUPPORTED;
    if (d.d != 16 && d.d != 32 && d.d != 64 && d.d != 128) return LLSA_ERR_UNSUPPORTED;
    if ((d.causal != 0 && d.causal != 1) || (d.kernel_path != 0 && d.kernel_path != 1)) return LLSA_ERR_UNSUPPORTED;
    p.G = d.heads / d.kv_heads;
    // rows and keys are counted in 31 bits, groups are the grid's second dimension
    if (d.Nq > ((int64_t)1 << 30) || d.Nkv > ((int64_t)1 << 30) || d.Nq * p.G > ((int64_t)1 << 30)) return LLSA_ERR_UNSUPPORTED;
    if ((int64_t)d.batch * d.kv_heads > 65535) return LLSA_ERR_UNSUPPORTED;
    // a launch has fewer than 2^32 threads a dimension: 256 for 128 rows or keys of all groups, or 64 for one of a group
    if (d.kernel_path == 0 && (int64_t)d.batch * d.kv_heads * ((d.Nq * p.G + 127) / 128 + (d.Nkv + 127) / 128) >= ((int64_t)1 << 24)) return LLSA_ERR_UNSUPPORTED;
    if (d.kernel_path == 1 && std::max<int64_t>(d.Nq * p.G, d.Nkv) >= ((int64_t)1 << 26)) return LLSA_ERR_UNSUPPORTED;
    p.rows = d.Nq * p.G;
    p.elt = d.dtype == LLSA_F32 ? 4 : 2;
    p.scale = d.sm_scale > 0.f ? d.sm_scale : (float)(1.0 / sqrt((double)d.d));
    if (!isfinite(p.scale)) return LLSA_ERR_UNSUPPORTED;
    if (!dense_strides(d.q_stride, d.batch, d.heads, d.Nq, d.d, p.elt, &p.q) || !dense_strides(d.k_stride, d.batch, d.kv_heads, d.Nkv, d.d, p.elt, &p.k) ||
        !dense_strides(d.v_stride, d.batch, d.kv_heads, d.Nkv, d.d, p.elt, &p.v) || !dense_strides(d.o_stride, d.batch, d.heads, d.Nq, d.d, p.elt, &p.o))
        return LLSA_ERR_BAD_SHAPE;
    const int row = d.d * p.elt;
    if (!dense_apart(p.o, d.batch, d.heads, d.Nq, row)) return LLSA_ERR_BAD_SHAPE;
    p.grads = dense_apart(p.q, d.batch, d.heads, d.Nq, row) && dense_apart(p.k, d.batch, d.kv_heads, d.Nkv, row) &&
              dense_apart(p.v, d.batch, d.kv_heads, d.Nkv, row);
    // offsets inside a tile are 32-bit
    if (d.kernel_path == 0) {
        const int64_t most = ((int64_t)1 << 32) - (1 << 20);
        if (256 * p.k.token > most || 256 * p.v.token > most || (p.G - 1) * p.q.head + 256 * p.q.token > most || (p.G - 1) * p.o.head + 256 * p.o.token > most)
            return LLSA_ERR_UNSUPPORTED;
    }
    if (d.kernel_path == 0) {
        p.fwd = p.dq = dense_shape(p, p.rows, d.Nkv);
        p.dkv = dense_shape(p, d.Nkv, p.rows);
    } else {
        p.fwd.splits = p.dq.splits = p.dkv.splits = 1;
    }
    p.ws_fwd = dense_part_bytes(p, p.rows, p.fwd, d.d + 2);
    p.stat_rows = (p.rows + 127) / 128 * 128;
    const size_t stat = dense_align((size_t)d.batch * d.kv_heads * p.stat_rows * sizeof(float));
    p.nD_off = 0;
    p.nlse_off = stat;
    p.part_off = 2 * stat;
    p.ws_bwd = p.part_off + std::max(dense_part_bytes(p, p.rows, p.dq, d.d + 1), dense_part_bytes(p, d.Nkv, p.dkv, 2 * d.d));
    return LLSA_OK;
}

static DenseArgs dense_args(const DensePlan &p, const void *Q, const void *K, const void *V, const int32_t *q_lens, const int32_t *kv_lens, float *LSE) {
    DenseArgs a;
    memset(&a, 0, sizeof(a));
    a.Q = static_cast<const char *>(Q);
    a.K = static_cast<const char *>(K);
    a.V = static_cast<const char *>(V);
    a.q = p.q; a.k = p.k; a.v = p.v; a.o = p.o;
    a.q_lens = q_lens;
    a.kv_lens = kv_lens;
    a.LSE = LSE;
    a.Nq = p.desc.Nq;
    a.Nkv = p.desc.Nkv;
    a.kv_heads = p.desc.kv_heads;
    a.G = p.G;
    a.div_g = FastDiv(p.G);
    a.causal = p.desc.causal;
    a.stat_rows = p.stat_rows;
    a.scale = p.scale;
    a.scale2 = p.scale * 1.4426950408889634f;
    return a;
}

static bool off_grid(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
template <class... P> static bool any_off_grid(size_t a, P... ptrs) { return (off_grid(ptrs, a) || ...); }

}  // namespace llsa

using namespace llsa;

struct llsa_dense_plan_s { DensePlan p; };

extern "C" {

llsa_status llsa_dense_plan(const llsa_dense_desc *desc, llsa_dense_plan_t **out) {
    if (!desc || !out) return LLSA_ERR_NULL;
    *out = nullptr;
    DensePlan p;
    const llsa_status st = build_dense_plan(*desc, p);
    if (st != LLSA_OK) return st;
    llsa_dense_plan_s *h = new (std::nothrow) llsa_dense_plan_s;
    if (!h) return LLSA_ERR_RUNTIME;
    h->p = p;
    *out = h;
    return LLSA_OK;
}

void llsa_dense_plan_destroy(llsa_dense_plan_t *plan) { delete plan; }

size_t llsa_dense_workspace_bytes(const llsa_dense_plan_t *plan, int for_backward) {
    return !plan ? 0 : for_backward ? plan->p.ws_bwd : plan->p.ws_fwd;
}

llsa_status llsa_dense_forward(const llsa_dense_plan_t *plan, const void *Q, const void *K, const void *V, const int32_t *q_lens,
                               const int32_t *kv_lens, void *O, float *LSE, void *workspace, void *hip_stream) {
    if (!plan || !Q || !K || !V || !O || !LSE || (!workspace && plan->p.ws_fwd)) return LLSA_ERR_NULL;
    if (any_off_grid(16, Q, K, V, O, LSE) || any_off_grid(4, q_lens, kv_lens) || off_grid(workspace, 256)) return LLSA_ERR_BAD_SHAPE;
    DenseArgs a = dense_args(plan->p, Q, K, V, q_lens, kv_lens, LSE);
    a.out = static_cast<char *>(O);
    hipStream_t s = (hipStream_t)hip_stream;
    const hipError_t e = plan->p.desc.kernel_path ? launch_dense_fwd_rows(plan->p, a, s) : launch_dense_fwd(plan->p, a, static_cast<float *>(workspace), s);
    return e == hipSuccess ? LLSA_OK : LLSA_ERR_RUNTIME;
}

llsa_status llsa_dense_backward(const llsa_dense_plan_t *plan, const void *Q, const void *K, const void *V, const int32_t *q_lens,
                                const int32_t *kv_lens, const void *O, const float *LSE, const void *dO, void *dQ, void *dK,
                                void *dV, void *workspace, void *hip_stream) {
    if (!plan || !Q || !K || !V || !O || !LSE || !dO || !dQ || !dK || !dV || !workspace) return LLSA_ERR_NULL;
    if (any_off_grid(16, Q, K, V, O, LSE, dO, dQ, dK, dV) || any_off_grid(4, q_lens, kv_lens) || off_grid(workspace, 256)) return LLSA_ERR_BAD_SHAPE;
    if (!plan->p.grads) return LLSA_ERR_BAD_SHAPE;
    DenseArgs a = dense_args(plan->p, Q, K, V, q_lens, kv_lens, const_cast<float *>(LSE));
    a.O = static_cast<const char *>(O);
    a.dO = static_cast<const char *>(dO);
    a.dQ = static_cast<char *>(dQ);
    a.dK = static_cast<char *>(dK);
    a.dV = static_cast<char *>(dV);
    a.nD = reinterpret_cast<float *>(static_cast<char *>(workspace) + plan->p.nD_off);
    a.nlse = reinterpret_cast<float *>(static_cast<char *>(workspace) + plan->p.nlse_off);
    hipStream_t s = (hipStream_t)hip_stream;
    if (plan->p.desc.kernel_path) {
        if (launch_dense_dq_rows(plan->p, a, s) != hipSuccess || launch_dense_dkv_rows(plan->p, a, s) != hipSuccess) return LLSA_ERR_RUNTIME;
        return LLSA_OK;
    }
    float *part = reinterpret_cast<float *>(static_cast<char *>(workspace) + plan->p.part_off);
    return launch_dense_bwd(plan->p, a, part, s) == hipSuccess ? LLSA_OK : LLSA_ERR_RUNTIME;
}

}  // extern "C"
