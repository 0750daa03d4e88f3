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
// The matrices of a chunk (That, P diag(beta), K^T) do not depend on the state: gd_prepare makes them for all chunks at once.  What is left is a
// chain of three products a chunk, whose columns (values) are independent: a wave takes 16 of them and keeps its part of the state in registers.
// (e = That v - (That diag(c) K) S, with both factors prepared, is a chain of two products, 0.87 us a chunk instead of 1.1; but what is prepared is then as
// wide as the state.  Matrices + chain of each form, beside each other, us: 8 x 6 heads of 4096 tokens 50 + 56 against 36 + 74, their gradient 65 + 172
// against 44 + 187, 2 x 16 of 8191 with 128 x 128 states 106 + 360 against 55 + 347.  The kept form has become faster since; the other was not made again.)
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

// A product of fragments is a sum of matrix instructions, term by term, the smallest first; terms below the last part's place are left out (a state's
// extra part serves products with two as well).
__device__ __forceinline__ constexpr int terms(const Whole &, const Whole &) { return 1; }
__device__ __forceinline__ void term(f32x4 &c, const Whole &a, const Whole &b, int) { c = mfma(a.v, b.v, c); }
template <int N>
__device__ __forceinline__ constexpr int terms(const Whole &, const Parts<N> &)
{
    return N;
}
template <int N>
__device__ __forceinline__ void term(f32x4 &c, const Whole &a, const Parts<N> &b, int t)
{
    c = mfma(a.v, b.p[N - 1 - t], c);
}
template <int N>
__device__ __forceinline__ constexpr int terms(const Parts<N> &, const Whole &)
{
    return N;
}
template <int N>
__device__ __forceinline__ void term(f32x4 &c, const Parts<N> &a, const Whole &b, int t)
{
    c = mfma(a.p[N - 1 - t], b.v, c);
}
template <int N, int M>
__device__ __forceinline__ constexpr int terms(const Parts<N> &, const Parts<M> &)
{
    constexpr int kMost = N < M ? N : M;
    return kMost * (kMost + 1) / 2;
}
template <int N, int M>
__device__ __forceinline__ void term(f32x4 &c, const Parts<N> &a, const Parts<M> &b, int t)
{
    static_assert(N <= 3 || M <= 3, "");
    const int left = terms(a, b) - t, s = left > 3 ? 2 : left > 1 ? 1 : 0;  // parts whose places add up to s
    const int i = (s + 1) * (s + 2) / 2 - left;
    c = mfma(a.p[i], b.p[s - i], c);
}
__device__ __forceinline__ constexpr int terms(const Full &, const Full &) { return 8; }
__device__ __forceinline__ void term(f32x4 &c, const Full &a, const Full &b, int t)
{
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[t], b.v[t], c, 0, 0, 0);
}
template <typename A, typename B>
__device__ __forceinline__ void mma(f32x4 &c, const A &a, const B &b)
{
#pragma unroll
    for (int t = 0; t < terms(a, b); ++t) term(c, a, b, t);
}
// acc[m] += a(m) b for m of [lo, hi): a term of every tile before the next one's, since an instruction waits for the one before it in its accumulator.
// (32-bit instructions take as long as that wait; a tile at a time they begin before all of a has come.)
template <typename A, typename B>
__device__ __forceinline__ void mma_tiles(f32x4 *acc, int lo, int hi, const A &a, const B &b)
{
    if constexpr (std::is_same<B, Full>::value) {
#pragma unroll
        for (int m = lo; m < hi; ++m) mma(acc[m], a(m), b);
        return;
    }
#pragma unroll
    for (int t = 0; t < terms(a(0), b); ++t)
#pragma unroll
        for (int m = lo; m < hi; ++m) term(acc[m], a(m), b, t);
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
// eight single elements
__device__ __forceinline__ void gather(Whole &f, const bf16_t (&x)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = uint32_t(x[2 * j].bits) | uint32_t(x[2 * j + 1].bits) << 16;
    f.v = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
}
__device__ __forceinline__ void gather(Full &f, const float (&x)[8]) { make(f, x); }

// ---- memory ----------------------------------------------------------------------------------------
// Every access goes through a buffer resource with a 32-bit byte offset that a lane forms once: the resource of a chunk's rows ends with
// the sequence, so rows behind it read as zero and are not written.  kNowhere is behind every resource.
using Rsrc = __amdgpu_buffer_rsrc_t;
constexpr unsigned kNowhere = 0xc0000000u;

__device__ __forceinline__ u32x4 load16(Rsrc r, unsigned at, unsigned base = 0) { return __builtin_amdgcn_raw_buffer_load_b128(r, at, base, 0); }
__device__ __forceinline__ float load4(Rsrc r, unsigned at, unsigned base = 0)
{
    return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, at, base, 0));
}
__device__ __forceinline__ void store4(Rsrc r, unsigned at, float x, unsigned base = 0)
{
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), r, at, base, 0);
}
template <typename T>
__device__ __forceinline__ T load_element(Rsrc r, unsigned at);
template <>
__device__ __forceinline__ float load_element<float>(Rsrc r, unsigned at)
{
    return load4(r, at);
}
template <>
__device__ __forceinline__ bf16_t load_element<bf16_t>(Rsrc r, unsigned at)
{
    return bf16_t{uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r, at, 0, 0))};
}
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(bf16_t x) { return __uint_as_float(uint32_t(x.bits) << 16); }
template <typename T>
__device__ __forceinline__ void store_element(Rsrc r, unsigned at, float x);
template <>
__device__ __forceinline__ void store_element<float>(Rsrc r, unsigned at, float x)
{
    store4(r, at, x);
}
template <>
__device__ __forceinline__ void store_element<bf16_t>(Rsrc r, unsigned at, float x)
{
    __builtin_amdgcn_raw_buffer_store_b16(uint16_t(pack2(x, x)), r, at, 0, 0);
}

// Requests for the next chunk stand between two of these.  Left alone, the compiler moves them to just before their use, where their
// latency is exposed, or above the last use of the registers that they are to reuse: then they get others, and a copy that waits for them.
__device__ __forceinline__ void requests_stay() { __builtin_amdgcn_sched_barrier(0); }

// eight values of an input row, 16-byte aligned
__device__ __forceinline__ void load_row(Whole &f, Rsrc r, unsigned at) { f.v = __builtin_bit_cast(bf16x8, load16(r, at)); }
__device__ __forceinline__ void load_row(Full &f, Rsrc r, unsigned at)
{
    const u32x4 a = load16(r, at), b = load16(r, at + 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) f.v[j] = __uint_as_float(a[j]), f.v[4 + j] = __uint_as_float(b[j]);
}
// eight values of an output row
__device__ __forceinline__ void store_row(Rsrc r, unsigned at, const float (&x)[8], bf16_t)
{
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])}, r, at, 0, 0);
}
__device__ __forceinline__ void store_row(Rsrc r, unsigned at, const float (&x)[8], float)
{
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]}), r, at, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{x[4], x[5], x[6], x[7]}), r, at + 16, 0, 0);
}
// what the wave has put into its own part of LDS is there for its other lanes
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Fragments in the workspace: planes of 16 bytes a lane, a kilobyte each
template <typename Frag>
constexpr int planes = int(sizeof(Frag)) / 16;
template <typename Frag>
constexpr size_t frag_bytes = size_t(planes<Frag>) * 1024;
constexpr int kStream = 2;  // a non-temporal store
template <typename Frag>
__device__ __forceinline__ void put(Rsrc ws, size_t first, int block, int lane, const Frag &f, bool stream)
{
    u32x4 w[planes<Frag>];
    __builtin_memcpy(w, &f, sizeof(f));
#pragma unroll
    for (int i = 0; i < planes<Frag>; ++i) {
        const unsigned at = unsigned(first) + unsigned(block * planes<Frag> + i) * 1024u;
        if (stream)
            __builtin_amdgcn_raw_buffer_store_b128(w[i], ws, 16u * unsigned(lane), at, kStream);
        else
            __builtin_amdgcn_raw_buffer_store_b128(w[i], ws, 16u * unsigned(lane), at, 0);
    }
}
// Matrices of more than half the Infinity Cache's 256 MB are written around the caches: little of them would be there when the chains come to it, and what
// they take would be another's.  (8 x 6 heads of 4096 tokens, gradient, 163 MB: matrices 40 -> 36 us, chains 175 -> 170; 2 x 16 heads of 8191,
// 128 x 128, 160 MB: chains 308 -> 298, inputs from the Infinity Cache.  Below it costs: 8 x 6 of 4096 forward, 101 MB: chains 70 -> 80; 64 x 6 of 196, gradient, 81 MB: 48 -> 66.)
constexpr size_t kStreamedBytes = size_t(128) << 20;
template <typename Frag>
__device__ __forceinline__ Frag get(Rsrc ws, size_t first, int block, int lane)
{
    u32x4 w[planes<Frag>];
#pragma unroll
    for (int i = 0; i < planes<Frag>; ++i) w[i] = load16(ws, 16u * unsigned(lane), unsigned(first) + unsigned(block * planes<Frag> + i) * 1024u);
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

// Chunks are the same in both scan directions, 64 tokens from a multiple of 64 on; a backward scan takes the chunks, and the
// tokens of a chunk, last first.  What is missing of the last chunk then comes before its tokens, with gate 0 and beta 0, which changes
// no state.  Token i of a chunk in scan order:
__device__ __forceinline__ int token_at(const Shape &s, int i) { return s.reverse ? kC - 1 - i : i; }
__device__ __forceinline__ int chunk_at(const Shape &s, int step) { return s.reverse ? s.chunks - 1 - step : step; }

// bytes from one token's row to the next one's
template <typename T>
__device__ __forceinline__ unsigned pitch_of(const Shape &s, int heads, int width)
{
    return unsigned(s.token_major ? heads * width : width) * unsigned(sizeof(T));
}
// the rows of a chunk of one head of [B, heads, L, width] or [B, L, heads, width]
template <typename T>
__device__ __forceinline__ Rsrc chunk_rows(const T *all, const Shape &s, int b, int head, int heads, int width, int chunk)
{
    const size_t L = size_t(s.L), row = size_t(chunk) * kC;
    const size_t first = s.token_major ? (size_t(b) * L + row) * heads + head : (size_t(b) * heads + head) * L + row;
    const unsigned rows = unsigned(s.L - chunk * kC < kC ? s.L - chunk * kC : kC);
    return slab_resource(all + first * width, (rows - 1) * pitch_of<T>(s, heads, width) + unsigned(width) * unsigned(sizeof(T)));
}
// What a chain of chunks reads or writes in turn: a pointer that moves by a constant, so that a step forms a resource with a few scalar
// instructions.  Chunks are full but for the sequence's last one.
struct Walk {
    const unsigned char *p;
    long step;
    unsigned extent, last_extent;
    int chunk, move, last_chunk;

    // `there`: or nothing, what is read is zero and what is written goes nowhere
    __device__ __forceinline__ Rsrc here(bool there = true) const { return slab_resource(p, !there ? 0u : chunk == last_chunk ? last_extent : extent); }
    __device__ __forceinline__ void next() { p += step, chunk += move; }
};
// `first`: the chunk it starts with, `move`: +1 or -1
template <typename T>
__device__ __forceinline__ Walk walk_rows(const T *all, const Shape &s, int b, int head, int heads, int width, int first, int move)
{
    const unsigned pitch = pitch_of<T>(s, heads, width), row = unsigned(width) * unsigned(sizeof(T));
    const size_t L = size_t(s.L), at = s.token_major ? size_t(b) * L * heads + head : (size_t(b) * heads + head) * L;
    Walk w;
    w.p = reinterpret_cast<const unsigned char *>(all + at * width) + long(first) * kC * long(pitch);
    w.step = long(move) * kC * long(pitch);
    w.extent = (kC - 1) * pitch + row;
    w.last_extent = unsigned(s.L - (s.chunks - 1) * kC - 1) * pitch + row;
    w.chunk = first;
    w.move = move;
    w.last_chunk = s.chunks - 1;
    return w;
}
// blocks of `bytes` each, one a chunk
__device__ __forceinline__ Walk walk_blocks(const unsigned char *all, size_t bytes, int first, int move)
{
    return {all + long(first) * long(bytes), long(move) * long(bytes), 0x80000000u, 0x80000000u, first, move, first};
}
// everything from p on
__device__ __forceinline__ Rsrc whole(const void *p) { return slab_resource(p, 0x80000000u); }
// where a lane's part of a fragment's row is: channels 32 step + 8g .. + 7 of a token; channels that the head does not have are nowhere
template <typename T>
__device__ __forceinline__ unsigned row_offset(unsigned pitch, int token, int step, int g, int width)
{
    const int c = 32 * step + 8 * g;
    return c < width ? unsigned(token) * pitch + unsigned(c) * unsigned(sizeof(T)) : kNowhere;
}

// Gates of a chunk below this (and infinite ones) close it as well: exp(-10000) is 0.  Sums of them are 64-bit, so that what follows a
// closed gate keeps its own decays.
constexpr float kGateFloor = -10000.f;

// What stands in for a strength of zero where it is divided by, see beta_divisor
constexpr float kLeastStrength = 1e-20f;

// Workspace of one chunk of one head, written by gd_prepare: c, d . beta and for the gradient d . beta and 1 / beta with the stand-in for a beta of zero
// (64 floats each), then fragments
template <typename T, int N, bool kBwd>
struct ChunkWs {
    using Mid = typename operands<T, N>::Mid;
    using Mid2 = typename operands<T, 2>::Mid;
    static constexpr size_t scalars = 0;
    static constexpr size_t inverse = 1024;                                          // That, or its transpose too
    static constexpr size_t scores = inverse + kTriBlocks * frag_bytes<Mid> * (kBwd ? 2 : 1);  // P diag(beta), or its transpose
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
