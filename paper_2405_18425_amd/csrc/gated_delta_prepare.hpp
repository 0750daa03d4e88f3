// gd_prepare: the matrices of a chunk that do not depend on the state, one workgroup of four waves per chunk of one head.
//
// K K^T and Q K^T on the matrix cores, a 16-row strip a wave, lower triangle only; That = (1 + N diag(beta))^-1 in 32-bit arithmetic:
// the four 16 x 16 diagonal blocks by substitution, a wave each (lane: a column), then two joins [[A, 0], [-B C A, B]] of
// blocks twice as large, on v_mfma_f32_16x16x4_f32.  A substitution divides by nothing and a join only multiplies
// inverses, so keys that repeat (N full of ones) lose no more than the recurrence itself does.
#pragma once

#include "gated_delta.hpp"

namespace vig {
namespace gd {

template <typename T>
struct PrepareArgs {
    Shape s;
    const T *q, *k, *g, *beta;
    unsigned char *ws, *key_ws;
};

constexpr int kPitch = 68;  // floats of a row of a 64 x 64 tile in LDS: 16-byte rows, four banks further each

// acc += X Y over 16 indexes; x: 16 bytes of row r of X at 4g, y: the base of Y's column r
__device__ __forceinline__ void mma16(f32x4 &acc, const float *x, const float *y_col, int g)
{
    const f32x4 a = *reinterpret_cast<const f32x4 *>(x + 4 * g);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], y_col[(4 * g + i) * kPitch], acc, 0, 0, 0);
}

// beta as the gradient takes it: of a beta that is (next to) zero it needs w / beta, the gradient of u, which stays exact however small
// beta is as long as it is not zero
__device__ __forceinline__ float beta_divisor(float b) { return fabsf(b) < 1e-20f ? copysignf(1e-20f, b) : b; }

// inclusive sums over the 64 lanes
__device__ __forceinline__ double wave_prefix(double x, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double y = __shfl_up(x, d);
        x += lane >= d ? y : 0.0;
    }
    return x;
}

template <typename T, int DK, int N, bool kBwd>
__global__ __launch_bounds__(256) void gd_prepare(PrepareArgs<T> a)
{
    using In = typename operands<T, N>::In;
    using Ws = ChunkWs<T, N, kBwd>;
    constexpr int kKs = DK / 32;
    __shared__ __align__(16) float inv[kC * kPitch], sco[kC * kPitch];
    __shared__ double sum[kC];
    __shared__ float bet[kC];
    const Shape &s = a.s;
    const int w = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const unsigned unit = blockIdx.x, slab = unit / unsigned(s.chunks), chunk = unit - slab * unsigned(s.chunks);
    const int b = int(slab / unsigned(s.H)), h = int(slab - unsigned(b) * unsigned(s.H)), share = s.H / s.Hk, hk = h / share;
    const Rsrc kr = chunk_rows(a.k, s, b, hk, s.Hk, s.dk, int(chunk)), qr = chunk_rows(a.q, s, b, hk, s.Hk, s.dk, int(chunk));
    const unsigned pitch = pitch_of<T>(s, s.Hk, s.dk);
    const Rsrc ws = whole(a.ws + size_t(unit) * Ws::bytes);

    // a wave's rows of q and k; columns are the rows of the strips up to its own
    In fq[kKs], fk[kKs];
#pragma unroll
    for (int ks = 0; ks < kKs; ++ks) {
        const unsigned at = row_offset<T>(pitch, token_at(s, 16 * w + r), ks, g, s.dk);
        load_row(fq[ks], qr, at);
        load_row(fk[ks], kr, at);
    }
    if (w == 0) {
        const Rsrc gr = chunk_rows(a.g, s, b, h, s.H, 1, int(chunk)), br = chunk_rows(a.beta, s, b, h, s.H, 1, int(chunk));
        const unsigned at = unsigned(token_at(s, lane)) * pitch_of<T>(s, s.H, 1);
        const float gate = fmaxf(value(load_element<T>(gr, at)), kGateFloor);
        float beta = value(load_element<T>(br, at));
        if constexpr (kBwd) beta = beta_divisor(beta);
        const double p = wave_prefix(double(gate), lane), total = __shfl(p, 63);
        sum[lane] = p;
        bet[lane] = beta;
        store4(ws, 4u * unsigned(lane), expf(float(p)));
        store4(ws, 4u * unsigned(lane), beta, 4 * kC);
        store4(ws, 4u * unsigned(lane), expf(float(total - p)), 8 * kC);
        if constexpr (kBwd) store4(ws, 4u * unsigned(lane), 1.f / beta, 12 * kC);
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        f32x4 kk = {0.f, 0.f, 0.f, 0.f}, qk = kk;
        if (n <= w) {
#pragma unroll
            for (int ks = 0; ks < kKs; ++ks) {
                In fb;
                load_row(fb, kr, row_offset<T>(pitch, token_at(s, 16 * n + r), ks, g, s.dk));
                mma(kk, fk[ks], fb);
                mma(qk, fq[ks], fb);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 16 * w + 4 * g + i, c = 16 * n + r;
            const float decay = c <= t ? expf(float(sum[t] - sum[c])) : 0.f;
            inv[t * kPitch + c] = c < t ? decay * bet[c] * kk[i] : 0.f;
            sco[t * kPitch + c] = c <= t ? decay * qk[i] : 0.f;
        }
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
        if (ks <= (w >> 1)) put(ws, Ws::inverse, lower_block(w, ks), lane, from<Mid>(inv + tr * kPitch + c));
        if constexpr (!kBwd) {
            if (ks <= (w >> 1)) put(ws, Ws::scores, lower_block(w, ks), lane, from<MidP>(sco + tr * kPitch + c));
        } else if (ks >= (w >> 1)) {
            float x[8], p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = inv[(c + j) * kPitch + tr], p[j] = sco[(c + j) * kPitch + tr];
            Mid f;
            make(f, x);
            put(ws, Ws::inverse + kTriBlocks * frag_bytes<Mid>, upper_block(w, ks), lane, f);
            make(f, p);
            put(ws, Ws::scores, upper_block(w, ks), lane, f);
        }
    }
    if (h == hk * share) {  // once per key head
        using Kw = KeyWs<T, DK, kBwd>;
        const Rsrc kw = whole(a.key_ws + ((size_t(b) * s.Hk + hk) * s.chunks + chunk) * Kw::bytes);
#pragma unroll
        for (int o = 0; o < Kw::blocks / 4; ++o) {
            const int block = 4 * o + w, tile = block >> 1, ks = block & 1, c = paired(tile, r);
            T x[8], y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const unsigned at = c < s.dk ? unsigned(token_at(s, 32 * ks + 8 * g + j)) * pitch + unsigned(c) * unsigned(sizeof(T)) : kNowhere;
                x[j] = load_element<T>(kr, at);
                if constexpr (kBwd) y[j] = load_element<T>(qr, at);
            }
            In f;
            gather(f, x);
            put(kw, 0, block, lane, f);
            if constexpr (kBwd) {
                gather(f, y);
                put(kw, Kw::blocks * frag_bytes<In>, block, lane, f);
            }
        }
    }
}

}  // namespace gd
}  // namespace vig
