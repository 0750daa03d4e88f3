// Gated delta rule: what its kernels share -- operand fragments, rows of a sequence, the workspace of a chunk.
//
//     e_t = v_t - a_t k_t S_{t-1},   u_t = beta_t e_t,   S_t = a_t S_{t-1} + k_t^T u_t,   o_t = q_t S_t,   a_t = exp(g_t)
//
// Over a chunk of 64 tokens, with b_t the sum of its gates up to t, G_ti = exp(b_t - b_i), c_t = exp(b_t), d_t = exp(b_63 - b_t)
// and S the state that enters:
//     e = That (v - c . K S),  That = (1 + N diag(beta))^-1,  N = strictly lower part of G . K K^T
//     o = c . Q S + P (beta . e),  P = lower part of G . Q K^T
//     S_out = c_63 S + K^T (d . beta . e)
// and with D the gradient that arrives at S_out, w the gradient of v:
//     w = That^T (beta . (P^T dO + d . K D)),   D_in = c_63 D + Q^T (c . dO) - K^T (c . w)
//
// The matrices of a chunk (That, P, K^T) do not depend on the state: gd_prepare makes them for all chunks at once.  What is left is a chain of
// three products a chunk, whose columns (values) are independent: a wave takes 16 of them and keeps its part of the state in registers.
//
// v_mfma_f32_16x16x32_bf16, lane (r = l % 16, g = l / 16): A row r and B column r with k = 8g .. 8g + 7; the accumulator holds rows 4g .. 4g + 3 of column
// r.  Rows of a pair of accumulator tiles stand for the indexes 32p + 8g + 4h + i (tile 2p + h, lane group g, register i), so that the eight
// accumulators that a lane holds of a pair are eight consecutive indexes -- the B operand of the next product as it stands, without
// LDS and without a barrier.  v_mfma_f32_16x16x4_f32 takes the same lanes' values one at a time.
#pragma once

#include "vig_common.hpp"

namespace vig {
namespace gd {

constexpr int kC = 64;  // tokens of a chunk

// row r of tile t of a pair-interleaved axis
__device__ __forceinline__ int paired(int tile, int r) { return 32 * (tile >> 1) + 8 * (r >> 2) + 4 * (tile & 1) + (r & 3); }

// ---- fragments -----------------------------------------------------------------------------------
// Eight k-values of a lane: bf16 as stored (Whole), 32-bit values as a sum of N bf16 (Parts: N = 2 keeps 16 bits, N = 3 keeps 24), or as they are (Full).
// Parts: what goes into bf16 results is held to 16 bits, whose error (2^-17) stands 1/256 under the results' own
// rounding; states that are returned in 32 bits take three parts.
struct Whole {
    bf16x8 v;
};
template <int N>
struct Parts {
    bf16x8 p[N];
};
struct Full {
    float v[8];
};

template <typename T, int N>
struct operands;
template <int N>
struct operands<bf16_t, N> {
    using In = Whole;
    using Mid = Parts<N>;
};
template <int N>
struct operands<float, N> {
    using In = Full;
    using Mid = Full;
};

__device__ __forceinline__ void mma(f32x4 &c, const Whole &a, const Whole &b) { c = mfma(a.v, b.v, c); }
template <int N>
__device__ __forceinline__ void mma(f32x4 &c, const Whole &a, const Parts<N> &b)
{
#pragma unroll
    for (int i = N - 1; i >= 0; --i) c = mfma(a.v, b.p[i], c);
}
template <int N>
__device__ __forceinline__ void mma(f32x4 &c, const Parts<N> &a, const Whole &b)
{
#pragma unroll
    for (int i = N - 1; i >= 0; --i) c = mfma(a.p[i], b.v, c);
}
// products of parts below the last one's place are left out; a state's extra part serves products with two as well
template <int N, int M>
__device__ __forceinline__ void mma(f32x4 &c, const Parts<N> &a, const Parts<M> &b)
{
    constexpr int kMost = N < M ? N : M;
#pragma unroll
    for (int s = kMost - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i <= s; ++i) c = mfma(a.p[i], b.p[s - i], c);
}
__device__ __forceinline__ void mma(f32x4 &c, const Full &a, const Full &b)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
}

// eight 32-bit values as an operand
template <int N>
__device__ __forceinline__ void make(Parts<N> &f, const float (&x)[8])
{
    uint32_t w[N][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float lo = x[2 * j], hi = x[2 * j + 1];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            w[n][j] = pack2(lo, hi);
            lo -= bf16_lo_to_f32(w[n][j]);
            hi -= bf16_hi_to_f32(w[n][j]);
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) f.p[n] = __builtin_bit_cast(bf16x8, u32x4{w[n][0], w[n][1], w[n][2], w[n][3]});
}
__device__ __forceinline__ void make(Full &f, const float (&x)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) f.v[j] = x[j];
}
template <typename Frag>
__device__ __forceinline__ Frag from(const f32x4 &lo, const f32x4 &hi)
{
    const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    Frag f;
    make(f, x);
    return f;
}
// eight consecutive 32-bit values in memory
template <typename Frag>
__device__ __forceinline__ Frag from(const float *p)
{
    return from<Frag>(*reinterpret_cast<const f32x4 *>(p), *reinterpret_cast<const f32x4 *>(p + 4));
}
// eight values of an input row, 16-byte aligned
__device__ __forceinline__ void load_row(Whole &f, const bf16_t *p) { f.v = *reinterpret_cast<const bf16x8 *>(p); }
__device__ __forceinline__ void load_row(Full &f, const float *p)
{
    const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) f.v[j] = a[j], f.v[4 + j] = b[j];
}
__device__ __forceinline__ void clear(Whole &f) { f.v = bf16x8{}; }
__device__ __forceinline__ void clear(Full &f)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) f.v[j] = 0.f;
}
// eight single elements
__device__ __forceinline__ void gather(Whole &f, const bf16_t (&x)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = uint32_t(x[2 * j].bits) | uint32_t(x[2 * j + 1].bits) << 16;
    f.v = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
}
__device__ __forceinline__ void gather(Full &f, const float (&x)[8]) { make(f, x); }

// Fragments in the workspace: planes of 16 bytes a lane, a kilobyte each
template <typename Frag>
constexpr int planes = int(sizeof(Frag)) / 16;
template <typename Frag>
constexpr size_t frag_bytes = size_t(planes<Frag>) * 1024;
template <typename Frag>
__device__ __forceinline__ void put(unsigned char *ws, int block, int lane, const Frag &f)
{
    u32x4 w[planes<Frag>];
    __builtin_memcpy(w, &f, sizeof(f));
#pragma unroll
    for (int i = 0; i < planes<Frag>; ++i) *reinterpret_cast<u32x4 *>(ws + (size_t(block) * planes<Frag> + i) * 1024 + 16 * lane) = w[i];
}
template <typename Frag>
__device__ __forceinline__ Frag get(const unsigned char *ws, int block, int lane)
{
    u32x4 w[planes<Frag>];
#pragma unroll
    for (int i = 0; i < planes<Frag>; ++i) w[i] = *reinterpret_cast<const u32x4 *>(ws + (size_t(block) * planes<Frag> + i) * 1024 + 16 * lane);
    Frag f;
    __builtin_memcpy(&f, w, sizeof(f));
    return f;
}

// Blocks of a 64 x 64 triangle in 16-row tiles and 32-wide steps: six of the eight are not zero
__device__ __forceinline__ constexpr int lower_block(int tile, int step) { return tile < 2 ? tile : 2 * tile - 2 + step; }
__device__ __forceinline__ constexpr int upper_block(int tile, int step) { return tile < 2 ? 2 * tile + step : tile + 2; }
constexpr int kTriBlocks = 6;

// ---- problem ---------------------------------------------------------------------------------------
struct Shape {
    int B, H, Hk, L, dk, dv, chunks;
    bool token_major, reverse;
};

// Rows of one head: element (t, c) at p[t * stride + c], t in scan order
template <typename T>
struct Rows {
    T *p;
    long stride;
};
template <typename T>
__device__ __forceinline__ Rows<T> rows_of(T *all, const Shape &s, int b, int head, int heads, int width)
{
    const size_t L = size_t(s.L);
    Rows<T> r;
    r.p = s.token_major ? all + (size_t(b) * L * heads + head) * width : all + (size_t(b) * heads + head) * L * width;
    r.stride = long(s.token_major ? heads : 1) * width;
    if (s.reverse) {
        r.p += (s.L - 1) * r.stride;
        r.stride = -r.stride;
    }
    return r;
}

// A fragment of the tokens' rows: channels 32 step + 8g .. + 7 of one row; channels the head does not have are zero
template <typename T, typename In>
__device__ __forceinline__ void row_frag(In &f, const Rows<const T> &rows, int t, int step, int g, int width)
{
    const int c = 32 * step + 8 * g;
    if (c < width)
        load_row(f, rows.p + t * rows.stride + c);
    else
        clear(f);
}
// A fragment of the transposed rows: one channel, tokens t0 .. t0 + 7 (no further than the last)
template <typename T, typename In>
__device__ __forceinline__ void column_frag(In &f, const Rows<const T> &rows, int t0, int last, int c, int width)
{
    T x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int t = t0 + j < last ? t0 + j : last;
        x[j] = c < width ? rows.p[t * rows.stride + c] : T{};
    }
    gather(f, x);
}

// Gates of a chunk below this (and infinite ones) close it as well: exp(-10000) is 0.  Sums of them are 64-bit, so that what follows a
// closed gate keeps its own decays.
constexpr float kGateFloor = -10000.f;

// Workspace of one chunk of one head, written by gd_prepare: c, beta, d (64 floats each, 64 spare), then fragments
template <typename T, int N, bool kBwd>
struct ChunkWs {
    using Mid = typename operands<T, N>::Mid;
    using Mid2 = typename operands<T, 2>::Mid;
    static constexpr size_t scalars = 0;
    static constexpr size_t inverse = 1024;                                          // That, or its transpose too
    static constexpr size_t scores = inverse + kTriBlocks * frag_bytes<Mid> * (kBwd ? 2 : 1);  // P, or P^T
    static constexpr size_t bytes = scores + kTriBlocks * (kBwd ? frag_bytes<Mid> : frag_bytes<Mid2>);
};
// ... and of one chunk of one key head: K^T, and for the gradient Q^T
template <typename T, int DK, bool kBwd>
struct KeyWs {
    using In = typename operands<T, 2>::In;
    static constexpr int blocks = DK / 16 * 2;
    static constexpr size_t bytes = blocks * frag_bytes<In> * (kBwd ? 2 : 1);
};

inline size_t round256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace gd
}  // namespace vig
