// states: the chain of a head's chunks, S -> S_out, for 16 value columns, one wave.  See gated_delta.hpp for the formulas.
//
// The wave holds its columns of the state in accumulators (32-bit) and takes a chunk's matrices from the workspace as fragments, 16 bytes
// a lane; each is requested for the next chunk as soon as its last product of this chunk has been issued.  Nothing
// goes through LDS and there is no barrier.  Columns of one head sit on one XCD (blockIdx % 8), whose L2 they read the fragments from.
#pragma once

#include "gated_delta.hpp"

namespace vig {
namespace gd {

template <typename T>
struct ChainArgs {
    Shape s;
    const T *q, *k, *v;
    const float *initial;                 // [B, H, dk, dv] or null
    T *out;                               // forward
    float *final_state;                   // [B, H, dk, dv] or null
    float *states, *wrong;                // gradient: S of every chunk [slab][chunk][dk][dv], e [slab][L][dv]
    const unsigned char *ws, *key_ws;
};

// (slab, first column) of a workgroup: eight consecutive workgroups (one per XCD) take eight slabs, the next eight their next columns
__device__ __forceinline__ bool chain_unit(unsigned block, unsigned slabs, unsigned parts, unsigned &slab, unsigned &part)
{
    const unsigned xcd = block & 7, rest = block >> 3, group = rest / parts;
    part = rest - group * parts;
    slab = group * 8 + xcd;
    return slab < slabs;
}

template <int N, int M>
__device__ __forceinline__ const Parts<M> &first_parts(const Parts<N> &f)
{
    static_assert(M <= N, "");
    return reinterpret_cast<const Parts<M> &>(f);
}
template <int N, int M>
__device__ __forceinline__ const Full &first_parts(const Full &f)
{
    return f;
}

// the three scalars of the tokens 8g .. 8g + 7 of each half chunk
struct Scalars {
    f32x4 c[4], beta[4], d[4];
    float whole;
};
__device__ __forceinline__ Scalars load_scalars(const unsigned char *ws, int g)
{
    const float *p = reinterpret_cast<const float *>(ws);
    Scalars x;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const int t = 32 * (m >> 1) + 8 * g + 4 * (m & 1);
        x.c[m] = *reinterpret_cast<const f32x4 *>(p + t);
        x.beta[m] = *reinterpret_cast<const f32x4 *>(p + kC + t);
        x.d[m] = *reinterpret_cast<const f32x4 *>(p + 2 * kC + t);
    }
    x.whole = p[kC - 1];
    return x;
}

template <typename T, int DK, int N, bool kBwd>
__device__ __forceinline__ void states(const ChainArgs<T> &a)
{
    using In = typename operands<T, N>::In;
    using Mid = typename operands<T, N>::Mid;
    using Mid2 = typename operands<T, 2>::Mid;
    using Ws = ChunkWs<T, N, kBwd>;
    using Kw = KeyWs<T, DK, kBwd>;
    constexpr int kKs = DK / 32, kCt = DK / 16;
    const Shape &s = a.s;
    const int lane = threadIdx.x, r = lane & 15, g = lane >> 4;
    unsigned slab, part;
    if (!chain_unit(blockIdx.x, unsigned(s.B) * unsigned(s.H), unsigned(s.dv) / 16, slab, part)) return;
    const int b = int(slab / unsigned(s.H)), h = int(slab - unsigned(b) * unsigned(s.H)), hk = h / (s.H / s.Hk);
    const int col = 16 * int(part) + r, last = s.L - 1;
    const Rows<const T> kr = rows_of(a.k, s, b, hk, s.Hk, s.dk), qr = rows_of(a.q, s, b, hk, s.Hk, s.dk), vr = rows_of(a.v, s, b, h, s.H, s.dv);
    Rows<T> orow;
    if constexpr (!kBwd) orow = rows_of(a.out, s, b, h, s.H, s.dv);
    const unsigned char *ws = a.ws + size_t(slab) * s.chunks * Ws::bytes;
    const unsigned char *kw = a.key_ws + (size_t(b) * s.Hk + hk) * s.chunks * Kw::bytes;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

    f32x4 S[kCt];
#pragma unroll
    for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = paired(ct, 4 * g + i);
            S[ct][i] = a.initial && c < s.dk ? a.initial[(size_t(slab) * s.dk + c) * s.dv + col] : 0.f;
        }

    In fk[4][kKs], fq[4][kKs], fkt[kCt][2];
    Mid ft[kTriBlocks];
    Mid2 fp[kTriBlocks];
    float v[16];
    Scalars sc;
    auto row = [&](int chunk, int t) __attribute__((always_inline)) {
        t += chunk * kC;
        return t < last ? t : last;
    };
    auto load_keys = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int ks = 0; ks < kKs; ++ks) row_frag<T>(fk[m][ks], kr, row(chunk, paired(m, r)), ks, g, s.dk);
    };
    auto load_queries = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int ks = 0; ks < kKs; ++ks) row_frag<T>(fq[m][ks], qr, row(chunk, paired(m, r)), ks, g, s.dk);
    };
    auto load_values = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = io<T>::load(vr.p + row(chunk, paired(j >> 2, 4 * g + (j & 3))) * vr.stride + col);
    };
    auto load_inverse = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kTriBlocks; ++i) ft[i] = get<Mid>(ws + size_t(chunk) * Ws::bytes + Ws::inverse, i, lane);
    };
    auto load_scores = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kTriBlocks; ++i) fp[i] = get<Mid2>(ws + size_t(chunk) * Ws::bytes + Ws::scores, i, lane);
    };
    auto load_transposed = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) fkt[ct][ks] = get<In>(kw + size_t(chunk) * Kw::bytes, 2 * ct + ks, lane);
    };
    load_keys(0);
    sc = load_scalars(ws, g);
    load_values(0);
    load_inverse(0);
    if constexpr (!kBwd) load_queries(0), load_scores(0);
    load_transposed(0);

    for (int chunk = 0; chunk < s.chunks; ++chunk) {
        const int next = chunk + 1 < s.chunks ? chunk + 1 : chunk;
        if constexpr (kBwd) {
            float *to = a.states + (size_t(slab) * s.chunks + chunk) * s.dk * s.dv + col;
#pragma unroll
            for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = paired(ct, 4 * g + i);
                    if (c < s.dk) to[size_t(c) * s.dv] = S[ct][i];
                }
        }
        Mid fs[kKs];
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) fs[ks] = from<Mid>(S[2 * ks], S[2 * ks + 1]);
        f32x4 e[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            e[m] = zero;
#pragma unroll
            for (int ks = 0; ks < kKs; ++ks) mma(e[m], fk[m][ks], fs[ks]);
#pragma unroll
            for (int i = 0; i < 4; ++i) e[m][i] = fmaf(-sc.c[m][i], e[m][i], v[4 * m + i]);
        }
        load_keys(next);
        load_values(next);
        Mid fe[2] = {from<Mid>(e[0], e[1]), from<Mid>(e[2], e[3])};
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            e[m] = zero;
#pragma unroll
            for (int ks = 0; ks <= (m >> 1); ++ks) mma(e[m], ft[lower_block(m, ks)], fe[ks]);
        }
        load_inverse(next);
        if constexpr (kBwd) {
            float *to = a.wrong + size_t(slab) * s.L * s.dv + col;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int t = chunk * kC + paired(j >> 2, 4 * g + (j & 3));
                if (t <= last) to[size_t(t) * s.dv] = e[j >> 2][j & 3];
            }
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) e[m] *= sc.beta[m];  // u
        if constexpr (!kBwd) {
            const Mid2 fu[2] = {from<Mid2>(e[0], e[1]), from<Mid2>(e[2], e[3])};
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                f32x4 o = zero;
#pragma unroll
                for (int ks = 0; ks < kKs; ++ks) mma(o, fq[m][ks], first_parts<N, 2>(fs[ks]));
                o *= sc.c[m];
#pragma unroll
                for (int ks = 0; ks <= (m >> 1); ++ks) mma(o, fp[lower_block(m, ks)], fu[ks]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = chunk * kC + paired(m, 4 * g + i);
                    if (t <= last) io<T>::store(orow.p + t * orow.stride + col, o[i]);
                }
            }
            load_queries(next);
            load_scores(next);
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) e[m] *= sc.d[m];
        const Mid fd[2] = {from<Mid>(e[0], e[1]), from<Mid>(e[2], e[3])};
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct) {
            S[ct] *= sc.whole;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) mma(S[ct], fkt[ct][ks], fd[ks]);
        }
        load_transposed(next);
        sc = load_scalars(ws + size_t(next) * Ws::bytes, g);
    }
    if (a.final_state)
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = paired(ct, 4 * g + i);
                if (c < s.dk) a.final_state[(size_t(slab) * s.dk + c) * s.dv + col] = S[ct][i];
            }
}

template <typename T, int DK, int N>
__global__ __launch_bounds__(64) void gd_states(ChainArgs<T> a)
{
    states<T, DK, N, false>(a);
}

}  // namespace gd
}  // namespace vig
