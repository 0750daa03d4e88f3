// gd_prepare: the matrices of a chunk that do not depend on the state, one workgroup of four waves per chunk of one head.
//
// K K^T and Q K^T on the matrix cores, a 16-row strip a wave (all four tiles of it: the last wave needs them, and the others lose less
// than by branches); That = (1 + N diag(beta))^-1 in 32-bit arithmetic:
// the four 16 x 16 diagonal blocks by substitution, a wave each (lane: a column), then two joins [[A, 0], [-B C A, B]] of
// blocks twice as large, on v_mfma_f32_16x16x4_f32.  A substitution divides by nothing and a join only multiplies
// inverses, so keys that repeat (N full of ones) lose no more than the recurrence itself does.
//
// Bound by memory where there are many chunks: of 8 x 6 heads of 4096 tokens (bf16, 64 x 64) it reads 50 MB and writes 101 in 35.4 us, 4.3 TB/s; for the
// gradient it writes 163 MB in 43 us.  Of one sequence of 196 tokens it is the latency of its steps, 7.5 us.
#pragma once

#include "gated_delta.hpp"

namespace vig {
namespace gd {

template <typename T>
struct PrepareArgs {
    Shape s;
    const T *q, *k, *g, *beta;
    unsigned char *ws, *key_ws;
    bool stream;  // see kStreamedBytes
};

constexpr int kPitch = 68;  // floats of a row of a 64 x 64 tile in LDS: 16-byte rows, four banks further each

// acc += X Y over 16 indexes; x: 16 bytes of row r of X at 4g, y: the base of Y's column r
__device__ __forceinline__ void mma16(f32x4 &acc, const float *x, const float *y_col, int g)
{
    const f32x4 a = *reinterpret_cast<const f32x4 *>(x + 4 * g);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], y_col[(4 * g + i) * kPitch], acc, 0, 0, 0);
}

// beta as the adjoints' chain takes it: of a beta that is (next to) zero it needs w / beta, the gradient of u, which stays exact however small
// beta is as long as it is not zero.  Everything else takes beta as it is.
__device__ __forceinline__ float beta_divisor(float b) { return fabsf(b) < kLeastStrength ? copysignf(kLeastStrength, b) : b; }

// DPP: a lane's source in its row of 16 or the row before; lanes without one, and rows that are not in the mask, receive 0
template <int CTRL, int kRows>
__device__ __forceinline__ float moved(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, kRows, 0xf, false));
}
template <int CTRL, int kRows>
__device__ __forceinline__ double moved(double x)
{
    const int2 w = __builtin_bit_cast(int2, x);
    return __builtin_bit_cast(double, int2{__builtin_amdgcn_update_dpp(0, w.x, CTRL, kRows, 0xf, false), __builtin_amdgcn_update_dpp(0, w.y, CTRL, kRows, 0xf, false)});
}
// inclusive sums over the 64 lanes
template <typename F>
__device__ __forceinline__ F wave_prefix(F x)
{
    x += moved<0x111, 0xf>(x);  // row_shr:1
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    x += moved<0x142, 0xa>(x);  // row_bcast:15, rows 1 and 3
    x += moved<0x143, 0xc>(x);  // row_bcast:31, rows 2 and 3
    return x;
}
__device__ __forceinline__ double last_lane(double x)
{
    const int2 w = __builtin_bit_cast(int2, x);
    return __builtin_bit_cast(double, int2{__builtin_amdgcn_readlane(w.x, 63), __builtin_amdgcn_readlane(w.y, 63)});
}

// Sums of the gates up to each token, in scan order and in powers of two, and the strengths: every wave its own (a lane a token).  Differences of
// the 64-bit sums are rounded to 32 bits where they are exponentiated.
template <typename T, bool kBwd>
struct Gates {
    T g, beta;
    __device__ __forceinline__ void request(const T *gates, const T *strengths, const Shape &s, int b, int h, int chunk, int lane)
    {
        const unsigned at = unsigned(token_at(s, lane)) * pitch_of<T>(s, s.H, 1);
        g = load_element<T>(chunk_rows(gates, s, b, h, s.H, 1, chunk), at);
        beta = load_element<T>(chunk_rows(strengths, s, b, h, s.H, 1, chunk), at);
    }
    __device__ __forceinline__ double sum() const
    {
        const double kLog2e = 1.4426950408889634074;
        const float x = value(g);
        return wave_prefix(kLog2e * double(x < kGateFloor ? kGateFloor : x));  // (a NaN stays one)
    }
    __device__ __forceinline__ float strength() const { return kBwd ? beta_divisor(value(beta)) : value(beta); }
};

__device__ __forceinline__ float exp2_of(double x) { return fast_exp2(float(x)); }
// decay from token c to token t, both the sums up to them, 1 for pairs that are none (formed for these as well: a branch for each costs more)
__device__ __forceinline__ float decay_of(double t, double c, bool pair)
{
    const float x = float(t - c);
    return fast_exp2(pair ? x : 0.f);
}

// Rows of a chunk in LDS, as they are, for fragments of rows and of columns
template <typename T, int DK>
struct KeyTile {
    static constexpr int pitch = DK + (sizeof(T) == 2 ? 8 : 4), bytes = kC * pitch * int(sizeof(T));
};
template <typename T, int DK, typename In>
__device__ __forceinline__ void key_put(unsigned char *lds, int row, int step, int g, const In &f)
{
    __builtin_memcpy(lds + (row * KeyTile<T, DK>::pitch + 32 * step + 8 * g) * int(sizeof(T)), &f, sizeof(f));
}
template <typename T, int DK, typename In>
__device__ __forceinline__ void key_get(In &f, const unsigned char *lds, int row, int step, int g)
{
    __builtin_memcpy(&f, __builtin_assume_aligned(lds + (row * KeyTile<T, DK>::pitch + 32 * step + 8 * g) * int(sizeof(T)), 16), sizeof(f));
}
// channels paired(tile, r), tokens 32 step + 8g .. + 7
template <int DK>
__device__ __forceinline__ void key_column(Whole &f, const unsigned char *lds, int tile, int step, int r, int g)
{
    const uint16_t *q = reinterpret_cast<const uint16_t *>(lds) + (32 * step + 8 * g + (r >> 2)) * KeyTile<bf16_t, DK>::pitch + paired(tile, 4 * (r & 3));
    f.v = join(lds_read_tr(q), lds_read_tr(q + 4 * KeyTile<bf16_t, DK>::pitch));
}
template <int DK>
__device__ __forceinline__ void key_column(Full &f, const unsigned char *lds, int tile, int step, int r, int g)
{
    const float *q = reinterpret_cast<const float *>(lds) + (32 * step + 8 * g) * KeyTile<float, DK>::pitch + paired(tile, r);
#pragma unroll
    for (int j = 0; j < 8; ++j) f.v[j] = q[j * KeyTile<float, DK>::pitch];
}

template <typename T, int DK, int N, bool kBwd>
__global__ __launch_bounds__(256) void gd_prepare(PrepareArgs<T> a)
{
    using In = typename operands<T, N>::In;
    using Ws = ChunkWs<T, N, kBwd>;
    using Kw = KeyWs<T, DK, kBwd>;
    constexpr int kKs = DK / 32, kTiles = 2 * kC * kPitch * 4, kKeys = KeyTile<T, DK>::bytes * (kBwd ? 2 : 1);
    __shared__ __align__(16) unsigned char shared[kTiles > kKeys ? kTiles : kKeys];  // rows of k (and q), afterwards the two matrices
    __shared__ double sum[4][kC];
    __shared__ float bet[4][kC];
    float *inv = reinterpret_cast<float *>(shared), *sco = inv + kC * kPitch;
    const Shape &s = a.s;
    const int w = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const unsigned unit = blockIdx.x, slab = unit / unsigned(s.chunks);
    const int chunk = int(unit - slab * unsigned(s.chunks));
    const int b = int(slab / unsigned(s.H)), h = int(slab - unsigned(b) * unsigned(s.H)), share = s.H / s.Hk, hk = h / share;
    const Rsrc ws = whole(a.ws + size_t(unit) * Ws::bytes);

    Gates<T, kBwd> gates;
    gates.request(a.g, a.beta, s, b, h, chunk, lane);
    In fq[kKs], fk[kKs];  // a wave's rows
    {
        const Rsrc kr = chunk_rows(a.k, s, b, hk, s.Hk, s.dk, chunk), qr = chunk_rows(a.q, s, b, hk, s.Hk, s.dk, chunk);
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
            const unsigned at = row_offset<T>(pitch_of<T>(s, s.Hk, s.dk), token_at(s, 16 * w + r), ks, g, s.dk);
            load_row(fk[ks], kr, at);
            load_row(fq[ks], qr, at);
        }
    }
    requests_stay();
    {
        const double p = gates.sum(), total = last_lane(p);
        const float beta = gates.strength();
        sum[w][lane] = p;
        bet[w][lane] = beta;
        if (w == 0) {
            const float d = exp2_of(total - p);
            store4(ws, 4u * unsigned(lane), exp2_of(p));
            store4(ws, 4u * unsigned(lane), d * value(gates.beta), 4 * kC);
            if constexpr (kBwd) {
                store4(ws, 4u * unsigned(lane), d * beta, 8 * kC);
                store4(ws, 4u * unsigned(lane), 1.f / beta, 12 * kC);
            }
        }
    }
#pragma unroll
    for (int ks = 0; ks < kKs; ++ks) {
        key_put<T, DK>(shared, 16 * w + r, ks, g, fk[ks]);
        if constexpr (kBwd) key_put<T, DK>(shared + KeyTile<T, DK>::bytes, 16 * w + r, ks, g, fq[ks]);
    }
    __syncthreads();
    if (h == hk * share) {  // K^T and Q^T once per key head
        const Rsrc kw = whole(a.key_ws + ((size_t(b) * s.Hk + hk) * s.chunks + chunk) * Kw::bytes);
#pragma unroll
        for (int o = 0; o < Kw::blocks / 4; ++o) {
            const int block = 4 * o + w;
            In f;
            key_column<DK>(f, shared, block >> 1, block & 1, r, g);
            put(kw, 0, block, lane, f, a.stream);
            if constexpr (kBwd) {
                key_column<DK>(f, shared + KeyTile<T, DK>::bytes, block >> 1, block & 1, r, g);
                put(kw, Kw::blocks * frag_bytes<In>, block, lane, f, a.stream);
            }
        }
    }
    f32x4 kk[4], qk[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        kk[n] = qk[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {  // (the upper tiles too: the last wave has all four, and branches cost the others more)
            In fb;
            key_get<T, DK>(fb, shared, 16 * n + r, ks, g);
            mma(kk[n], fk[ks], fb);
            mma(qk[n], fq[ks], fb);
        }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 16 * w + 4 * g + i, c = 16 * n + r;
            // (factors of 0 and 1 rather than branches)
            const float decay = decay_of(sum[w][t], sum[w][c], c <= t) * bet[w][c];
            inv[t * kPitch + c] = (c < t ? 1.f : 0.f) * decay * kk[n][i];
            sco[t * kPitch + c] = (c <= t ? 1.f : 0.f) * decay * qk[n][i];
        }
    __syncthreads();
    {  // diagonal blocks: column r of the inverse of block w
        float *d = inv + 16 * w * kPitch + 16 * w;
        float x[16];
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            float v = t == r ? 1.f : 0.f;
#pragma unroll
            for (int i = 0; i < t; ++i) v = fmaf(-d[t * kPitch + i], x[i], v);
            x[t] = v;
        }
        if (g == 0)
#pragma unroll
            for (int t = 0; t < 16; ++t) d[t * kPitch + r] = x[t];
    }
    __syncthreads();
    if (w < 2) {  // blocks (1, 0) and (3, 2)
        const int hi = 2 * w + 1, lo = 2 * w;
        f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
        mma16(x, inv + (16 * hi + r) * kPitch + 16 * lo, inv + 16 * lo * kPitch + 16 * lo + r, g);
        const f32x4 left = *reinterpret_cast<const f32x4 *>(inv + (16 * hi + r) * kPitch + 16 * hi + 4 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) y = __builtin_amdgcn_mfma_f32_16x16x4f32(left[i], x[i], y, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) inv[(16 * hi + 4 * g + i) * kPitch + 16 * lo + r] = -y[i];
    }
    __syncthreads();
    f32x4 y[2];
    if (w < 2) {  // rows 32 .. 63, columns 16 w .. 16 w + 15
        f32x4 x[2];
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            x[o] = y[o] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (c >= w) mma16(x[o], inv + (32 + 16 * o + r) * kPitch + 16 * c, inv + 16 * c * kPitch + 16 * w + r, g);
        }
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
            for (int c = 0; c <= o; ++c) {
                const f32x4 left = *reinterpret_cast<const f32x4 *>(inv + (32 + 16 * o + r) * kPitch + 32 + 16 * c + 4 * g);
#pragma unroll
                for (int i = 0; i < 4; ++i) y[o] = __builtin_amdgcn_mfma_f32_16x16x4f32(left[i], x[c][i], y[o], 0, 0, 0);
            }
    }
    __syncthreads();
    if (w < 2)
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
            for (int i = 0; i < 4; ++i) inv[(32 + 16 * o + 4 * g + i) * kPitch + 16 * w + r] = -y[o][i];
    __syncthreads();

    // fragments: a wave the rows of its tile
    using Mid = typename operands<T, N>::Mid;
    using MidP = typename operands<T, kBwd ? N : 2>::Mid;
    const int tr = paired(w, r);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        const int c = 32 * ks + 8 * g;
        if (ks <= (w >> 1)) put(ws, Ws::inverse, lower_block(w, ks), lane, from<Mid>(inv + tr * kPitch + c), a.stream);
        if constexpr (!kBwd) {
            if (ks <= (w >> 1)) put(ws, Ws::scores, lower_block(w, ks), lane, from<MidP>(sco + tr * kPitch + c), a.stream);
        } else if (ks >= (w >> 1)) {
            float x[8], p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = inv[(c + j) * kPitch + tr], p[j] = sco[(c + j) * kPitch + tr];
            Mid f;
            make(f, x);
            put(ws, Ws::inverse + kTriBlocks * frag_bytes<Mid>, upper_block(w, ks), lane, f, a.stream);
            make(f, p);
            put(ws, Ws::scores, upper_block(w, ks), lane, f, a.stream);
        }
    }
}

}  // namespace gd
}  // namespace vig
