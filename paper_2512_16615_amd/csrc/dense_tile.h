// Tiles of rows in LDS and the matrix products of dense attention, for both I/O types.
//
// Every product is a 32 x 32 tile of v_mfma_f32_32x32x16_bf16 or v_mfma_f32_32x32x2_f32 (lane = 32 h + i):
//   A (32 x k): lane holds row i;  B (k x 32): lane holds column i;  contraction slots 8h .. 8h + 7 (bf16) or h (fp32)
//   D (32 x 32): lane holds column i, rows 8 (r / 4) + 4 h + r % 4 in registers r = 0 .. 15
// Scores are formed with what the softmax runs over in the registers and what it is per in the lanes: S^T = K Q^T in the query-major
// kernels (a lane has one query), S = Q K^T in the key-major one (a lane has one key).  The exponentials are then already in place as the B
// operand of the second product: the contraction may go through the rows in any order, so slot 8h + e of step t stands for row
// 16 t + 8 (e / 4) + 4 h + e % 4, which is register 8 t + e (fp32: step r is register r).  The A operand of that product is the tile read across its rows: two
// transposing reads of 4 rows (bf16), single values (fp32).  No score passes through LDS or another lane.
//
// The first product contracts over channels: piece ks of a row is 32 bytes, 16 of them each half of the wave's (16 channels, one
// instruction, or 8 channels, four of them).
#pragma once
#include <utility>

#include "dense.h"
#include "mfma_common.h"

namespace llsa {

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

// Over the two lanes of a column
__device__ __forceinline__ float half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 16 bytes of a row as an operand of a channel product
template <class T> struct Piece { u32x4 w; };
__device__ __forceinline__ f32x16 piece_product(const Piece<__bf16> &a, const Piece<__bf16> &b, f32x16 c) {
    return mfma32(__builtin_bit_cast(bf16x8, a.w), __builtin_bit_cast(bf16x8, b.w), c);
}
__device__ __forceinline__ f32x16 piece_product(const Piece<float> &a, const Piece<float> &b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = mfma32(__uint_as_float(a.w[e]), __uint_as_float(b.w[e]), c);
    return c;
}
// the scalar product of the lane's halves of two rows
__device__ __forceinline__ float piece_dot(const Piece<__bf16> &a, const Piece<__bf16> &b, float s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        s = fmaf(__uint_as_float(a.w[e] << 16), __uint_as_float(b.w[e] << 16), s);
        s = fmaf(__uint_as_float(a.w[e] & 0xffff0000u), __uint_as_float(b.w[e] & 0xffff0000u), s);
    }
    return s;
}
__device__ __forceinline__ float piece_dot(const Piece<float> &a, const Piece<float> &b, float s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) s = fmaf(__uint_as_float(a.w[e]), __uint_as_float(b.w[e]), s);
    return s;
}

// Registers 8 t .. 8 t + 7 of a 32 x 32 tile as the B operand of the second product: rounded to bf16, half a step (2^-8) of each; the sums over
// a row of exponentials are of the unrounded ones.
__device__ __forceinline__ bf16x8 round8(const f32x16 &p, int t) {
    bf16x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (__bf16)p[8 * t + e];
    return r;
}

// f of 0, 1, .. N - 1 as constants
template <class F, int... I> __device__ __forceinline__ void constants(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>()), ...); }
template <int N, class F> __device__ __forceinline__ void constants(F f) { constants(f, std::make_integer_sequence<int, N>()); }

// The LDS operands of a row of N matrix instructions, P of them on their way: the compiler reads each right in front of its instruction and
// waits for it there, some 100 cycles for every 32 of the matrix unit.  take(i, f): f of operand i, then operand i + P is asked for; nothing is moved
// across, so that the vector instructions written between two of them run while the matrix unit is busy.  16 x 8192 tokens, d = 128: forward 520 -> 502 us, backward
// 1604 -> 1560; 16 x 4096, d = 64, causal 63 -> 57 and 175 -> 168; 3 x 16 heads, 4 key heads, x 1999, d = 128 111 -> 107 and 433 -> 392.
template <int N, int P, class Fetch> struct Operands {
    Fetch fetch;
    bf16x8 op[P];
    __device__ __forceinline__ explicit Operands(Fetch f) : fetch(f) {
        constants<P>([&](auto i) { op[i] = fetch(i); });
    }
    template <int I, class F> __device__ __forceinline__ void take(std::integral_constant<int, I>, F f) {
        f(op[I % P]);
        if constexpr (I + P < N) op[I % P] = fetch(std::integral_constant<int, I + P>());
        __builtin_amdgcn_sched_barrier(0);
    }
};
template <int N, int P, class Fetch> __device__ __forceinline__ Operands<N, P, Fetch> operands(Fetch f) { return Operands<N, P, Fetch>(f); }
template <int A, int B> constexpr std::integral_constant<int, A + B> plus(std::integral_constant<int, A>, std::integral_constant<int, B>) { return {}; }

// Rows of D elements in LDS, unpadded; the 16-byte chunk c of row r stands at chunk c ^ key(r).  key permutes bits of r, so that (64 banks, 256 bytes
// a cycle) neither the row-wise 16-byte read, whose 16 lanes at a time are at one chunk of rows that differ in all of r's low four bits, nor
// the transposing read, whose 32 lanes are at 64 bytes of 4 rows that follow each other, meets a bank twice.
template <class T, int D> struct DenseTile {
    static constexpr int ROWB = D * (int)sizeof(T), CH = ROWB / 16, KS = ROWB / 32;
    static constexpr int NB = D >= 32 ? D / 32 : 1;        // 32-channel blocks of a result (d = 16: half of one, the other half a copy)
    static constexpr int NK = D >= 32 ? 4 : 2;             // groups of 4 registers of a block that are channels of their own
    static constexpr int RPI = 1024 / ROWB;                // rows that one load of a wave brings
    static constexpr __device__ __host__ int key(int r) {
        return ROWB >= 256 ? ((r & 3) << 2) | ((r >> 2) & 3) : ROWB == 128 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : ROWB == 64 ? (r >> 2) & 3 : (r >> 3) & 1;
    }
    int lane_row, lane_col;
    __device__ __forceinline__ explicit DenseTile(int lane) {
        const int i = lane & 31, h = lane >> 5;
        lane_row = i * ROWB + ((h ^ key(i)) << 4);
        if constexpr (sizeof(T) == 2) {
            const int lr = lane & 15, q = D >= 32 ? (lane >> 4) & 1 : 0, r = 4 * h + (lr >> 2);
            lane_col = r * ROWB + (((2 * q + ((lr & 3) >> 1)) ^ key(r)) << 4) + ((lr & 1) << 3);
        } else {
            const int c = D >= 32 ? i : i & 15;
            lane_col = 4 * h * ROWB + (((c >> 2) ^ h) << 4) + ((c & 3) << 2);
        }
    }
    // The same for a stage's tiles, `offset` bytes on (a multiple of 1024).  Opaque: the compiler would keep each of the sixteen places that are an exclusive
    // or away from these in a register of its own over the whole loop, and spill others.
    __device__ __forceinline__ DenseTile at(int offset) const {
        DenseTile t = *this;
        t.lane_row += offset;
        t.lane_col += offset;
        asm volatile("" : "+v"(t.lane_row), "+v"(t.lane_col));
        return t;
    }
    // piece ks of row 32 sub + i
    __device__ __forceinline__ Piece<T> row(const char *tile, int sub, int ks) const {
        return {*reinterpret_cast<const u32x4 *>(tile + (lane_row ^ (32 * ks)) + sub * 32 * ROWB)};
    }
    // 32 channels n .. of rows 32 sub + 16 t .. + 15 as an operand of the second product (bf16)
    __device__ __forceinline__ bf16x8 col(const char *tile, int sub, int n, int t) const {
        return lds_tr_pair(tile + (lane_col ^ (64 * n)) + (32 * sub + 16 * t) * ROWB, tile + (lane_col ^ (64 * n) ^ (ROWB >= 64 ? 32 : 16)) + (32 * sub + 16 * t + 8) * ROWB);
    }
    // acc += X^T p, X: rows 32 sub .. + 31 of the tile, channels 32 n .. + 31 (fp32)
    __device__ __forceinline__ f32x16 col_product(const char *tile, int sub, int n, const f32x16 &p, f32x16 acc) const {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = 8 * (r >> 2) + (r & 3);
            acc = mfma32(*reinterpret_cast<const float *>(tile + (lane_col ^ ((key(row) << 4) ^ (128 * n))) + (32 * sub + row) * ROWB), p[r], acc);
        }
        return acc;
    }
};

// Stages of a ring of two tensors' tiles.  A narrow workgroup's four rings have one each from 256 bytes a row: with two workgroups a CU the other one computes meanwhile
// (one token of 32 heads, 8 key heads, d = 128, 8 sequences of 16384: 115 -> 110 us, of 500 to 16384: 69 -> 65).
template <class T, int D, int FORM> constexpr int dense_stages() { return FORM == kDenseNarrow && DenseTile<T, D>::ROWB >= 256 ? 1 : 2; }

// Memory straight into LDS through a buffer descriptor: lane l fetches 16 bytes at its own offset, to 16 l of the 1024 bytes at `lds`; what lies
// outside the descriptor's bytes arrives as zeros.  The asm begins with the wait states that a vector memory instruction needs behind a
// vector instruction that wrote its descriptor (5) and its load follows m0 by one; the compiler inserts neither around asm.
__device__ __forceinline__ u32x4 buffer_of(const char *base, unsigned bytes) {
    const uint64_t b = reinterpret_cast<uint64_t>(base);
    return {(unsigned)__builtin_amdgcn_readfirstlane((int)b), (unsigned)__builtin_amdgcn_readfirstlane((int)(b >> 32)) & 0xffffu,
            (unsigned)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int N> __device__ __forceinline__ void buffer_to_lds(u32x4 buf, const unsigned (&v)[N], unsigned lds) {
    static_assert(N == 1 || N == 2 || N == 4, "");
    lds = __builtin_amdgcn_readfirstlane(lds);
    if constexpr (N == 4)
        asm volatile("s_mov_b32 m0, %5\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %4, 0 offen lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %4, 0 offen lds\n\t"
                     "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %4, 0 offen lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %4, 0 offen lds"
                     ::"v"(v[0]), "v"(v[1]), "v"(v[2]), "v"(v[3]), "s"(buf), "s"(lds) : "memory", "m0", "scc");
    else if constexpr (N == 2)
        asm volatile("s_mov_b32 m0, %3\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     ::"v"(v[0]), "v"(v[1]), "s"(buf), "s"(lds) : "memory", "m0", "scc");
    else
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(v[0]), "s"(buf), "s"(lds) : "memory", "m0");
}
// 4 bytes a lane, to 256 bytes at `lds`
__device__ __forceinline__ void buffer_to_lds_dword(u32x4 buf, unsigned v, unsigned lds) {
    lds = __builtin_amdgcn_readfirstlane(lds);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(v), "s"(buf), "s"(lds) : "memory", "m0");
}
#pragma clang diagnostic pop

// Every load that the compiler knows of is done.  In front of a loop that waits for its ring by itself: the compiler would wait inside it, in each
// round, for what the first one uses, and so for the ring's newest tile (causal, 3 x 16 heads of 1999, 1500 and 700 tokens, d = 128: forward 59.5 -> 53.3 us).
__device__ __forceinline__ void loads_done() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// A wave's share of a tile of ROWS rows: loads first, first + 1, .. of it (1024 bytes each).
template <class T, int D, int ROWS, int WAVES> struct TileLoads {
    using Tile = DenseTile<T, D>;
    static constexpr int ALL = ROWS / Tile::RPI, N = ALL >= WAVES ? ALL / WAVES : 1;      // loads of the tile, of a wave
    static constexpr int STEP = N >= 4 ? 4 : N;
    static_assert(ROWS % Tile::RPI == 0 && (ALL % WAVES == 0 || ALL < WAVES) && N % STEP == 0, "");
    // keys: row r of the tile `token` bytes behind the one before it
    static __device__ __forceinline__ void keys(u32x4 buf, unsigned token, unsigned lds, int wave, int lane) {
        if (ALL < WAVES && wave >= ALL) return;
        const int r0 = lane / Tile::CH, c = lane % Tile::CH;
#pragma unroll
        for (int i = 0; i < N; i += STEP) {
            unsigned v[STEP];
#pragma unroll
            for (int k = 0; k < STEP; ++k) {
                const int row = (wave * N + i + k) * Tile::RPI + r0;
                v[k] = row * token + ((c ^ Tile::key(row)) << 4);
            }
            buffer_to_lds<STEP>(buf, v, lds + (wave * N + i) * 1024);
        }
    }
    // rows r0 + r of a group below `rows`, of two tensors (queries and their output's gradients) whose descriptors begin at query q0 = r0 / G
    static __device__ __forceinline__ void rows(u32x4 qbuf, u32x4 obuf, const DenseArgs &a, int r0, int q0, int rows, unsigned qlds, unsigned olds, int wave, int lane) {
        if (ALL < WAVES && wave >= ALL) return;
        asm volatile("" : "+v"(lane));                       // (offsets formed anew each time: kept over the loop they cost a register each)
        const int rl = lane / Tile::CH, c = lane % Tile::CH;
#pragma unroll
        for (int i = 0; i < N; i += STEP) {
            unsigned vq[STEP], vo[STEP];
#pragma unroll
            for (int k = 0; k < STEP; ++k) {
                const int r = (wave * N + i + k) * Tile::RPI + rl;
                const unsigned q = a.G == 1 ? r0 + r : a.div_g(r0 + r), g = r0 + r - q * a.G, chunk = (c ^ Tile::key(r)) << 4;
                const bool in = r0 + r < rows;
                vq[k] = in ? g * (unsigned)a.q.head + (q - q0) * (unsigned)a.q.token + chunk : 0xffffff00u;
                vo[k] = in ? g * (unsigned)a.o.head + (q - q0) * (unsigned)a.o.token + chunk : 0xffffff00u;
            }
            buffer_to_lds<STEP>(qbuf, vq, qlds + (wave * N + i) * 1024);
            buffer_to_lds<STEP>(obuf, vo, olds + (wave * N + i) * 1024);
        }
    }
};

// The sums of a workgroup's four waves over the same rows, in wave 0 (f: what the lane's own are multiplied by; the waves' in order).  A lane has the
// same rows and channels in each wave, so registers go through LDS as they are.  lds: 12 KB a block, free of everything else.
template <int NB> __device__ __forceinline__ void add_waves(f32x16 (&acc)[NB], float f, char *lds, int wave, int lane) {
    f32x4 *buf = reinterpret_cast<f32x4 *>(lds);
    if (wave > 0) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                buf[(((wave - 1) * NB + n) * 4 + k) * 64 + lane] = f32x4{acc[n][4 * k] * f, acc[n][4 * k + 1] * f, acc[n][4 * k + 2] * f, acc[n][4 * k + 3] * f};
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = acc[n][4 * k + e] * f;
#pragma unroll
                    for (int w = 0; w < 3; ++w) x += buf[((w * NB + n) * 4 + k) * 64 + lane][e];
                    acc[n][4 * k + e] = x;
                }
    }
}

// The sums of two waves over the same rows, `half` 0's and 1's of pair `pair`, in the first.  lds: 16 KB a block.
template <int NB> __device__ __forceinline__ void add_halves(f32x16 (&acc)[NB], float f, char *lds, int pair, int half, int lane) {
    f32x4 *buf = reinterpret_cast<f32x4 *>(lds) + pair * NB * 256 + lane;
    if (half) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                buf[(n * 4 + k) * 64] = f32x4{acc[n][4 * k] * f, acc[n][4 * k + 1] * f, acc[n][4 * k + 2] * f, acc[n][4 * k + 3] * f};
    }
    __syncthreads();
    if (!half) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const f32x4 x = buf[(n * 4 + k) * 64];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[n][4 * k + e] = fmaf(acc[n][4 * k + e], f, x[e]);
            }
    }
}

// 32 rows' results (32-channel blocks, column = row of the tensor) to memory: scaled, rounded once; 16 bytes a lane.
template <class T, int D> __device__ __forceinline__ void store_rows(char *row, const f32x16 (&acc)[DenseTile<T, D>::NB], float f, int h, bool write) {
    using Tile = DenseTile<T, D>;
#pragma unroll
    for (int n = 0; n < Tile::NB; ++n) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int k = 0; k < Tile::NK; ++k) {
                const f32x4 v = {acc[n][4 * k] * f, acc[n][4 * k + 1] * f, acc[n][4 * k + 2] * f, acc[n][4 * k + 3] * f};
                if (write) *reinterpret_cast<f32x4 *>(row + 4 * (32 * n + 8 * k + 4 * h)) = v;
            }
        } else {
            // the upper half of the wave hands its channels 8k + 4 .. 7 down and takes 8k + 8 .. 11, so that each lane has 8 in a row
#pragma unroll
            for (int k = 0; k < Tile::NK; k += 2) {
                u32x4 w;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const auto r = __builtin_amdgcn_permlane32_swap(pack_bf16(acc[n][4 * k + 2 * j] * f, acc[n][4 * k + 2 * j + 1] * f),
                                                                    pack_bf16(acc[n][4 * k + 4 + 2 * j] * f, acc[n][4 * k + 5 + 2 * j] * f), false, false);
                    w[j] = r[0];
                    w[2 + j] = r[1];
                }
                if (write) *reinterpret_cast<u32x4 *>(row + 2 * (32 * n + 8 * (k + h))) = w;
            }
        }
    }
}
// the same in fp32, for partial sums
template <int D, int NB> __device__ __forceinline__ void store_partial(float *row, const f32x16 (&acc)[NB], int h) {
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int k = 0; k < (D >= 32 ? 4 : 2); ++k)
            *reinterpret_cast<f32x4 *>(row + 32 * n + 8 * k + 4 * h) = f32x4{acc[n][4 * k], acc[n][4 * k + 1], acc[n][4 * k + 2], acc[n][4 * k + 3]};
}
// Zeros in the rows that have no result: they had zeros for channels and went along, and 0 times an infinity is none.
template <int NB> __device__ __forceinline__ void keep_rows(f32x16 (&acc)[NB], bool keep) {
    if (__builtin_amdgcn_ballot_w64(!keep) == 0) return;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[n][e] = keep ? acc[n][e] : 0.f;
}
// is one of these not finite in some lane?  (a bit a lane)
template <int NB> __device__ __forceinline__ uint64_t not_finite(const f32x16 (&acc)[NB]) {
    float s = 0.f;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) s = fmaf(acc[n][e], 0.f, s);
    return __builtin_amdgcn_ballot_w64(s != 0.f);           // 0, or a NaN
}

}  // namespace llsa
