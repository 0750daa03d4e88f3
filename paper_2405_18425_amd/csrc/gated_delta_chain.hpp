// states: the chain of a head's chunks, S -> S_out, for 16 value columns, one wave.  See gated_delta.hpp for the formulas.
//
// The wave holds its columns of the state in accumulators (32-bit) and takes a chunk's matrices from the workspace as fragments, 16 bytes
// a lane: what a step needs first (K, That, V) is requested for the next chunk as soon as its last product of this chunk has been issued,
// what it needs later at its start.  Nothing goes through LDS and there is no barrier.  Columns of one head sit on one XCD (blockIdx % 8), whose L2 they read the fragments from.
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
__device__ __forceinline__ f32x4 as_floats(const u32x4 &x) { return __builtin_bit_cast(f32x4, x); }
__device__ __forceinline__ Scalars load_scalars(Rsrc ws, int g)
{
    Scalars x;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const unsigned at = 32u * unsigned(g), base = 128u * unsigned(m >> 1) + 16u * unsigned(m & 1);
        x.c[m] = as_floats(load16(ws, at, base));
        x.beta[m] = as_floats(load16(ws, at, base + 4 * kC));
        x.d[m] = as_floats(load16(ws, at, base + 8 * kC));
    }
    x.whole = load4(ws, 0, 4 * (kC - 1));
    return x;
}

// Rows of a state: element (channel, column) of [dk][dv] floats in the lanes that hold it; channels that the head does not have are nowhere
__device__ __forceinline__ unsigned state_offset(const Shape &s, int ct, int i, int g, int col)
{
    const int c = paired(ct, 4 * g + i);
    return c < s.dk ? 4u * (unsigned(c) * unsigned(s.dv) + unsigned(col)) : kNowhere;
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
    const int col = 16 * int(part) + r;
    const unsigned char *ws_all = a.ws + size_t(slab) * s.chunks * Ws::bytes;
    const unsigned char *kw_all = a.key_ws + (size_t(b) * s.Hk + hk) * s.chunks * Kw::bytes;
    const size_t state_size = size_t(s.dk) * s.dv;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

    // offsets of a lane's rows: of keys and queries, and of its 16 values
    const unsigned key_pitch = pitch_of<T>(s, s.Hk, s.dk), value_pitch = pitch_of<T>(s, s.H, s.dv);
    unsigned key_at[4], value_at[16], e_at[16];
#pragma unroll
    for (int m = 0; m < 4; ++m) key_at[m] = row_offset<T>(key_pitch, token_at(s, paired(m, r)), 0, g, s.dk);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const unsigned t = unsigned(token_at(s, paired(j >> 2, 4 * g + (j & 3))));
        value_at[j] = t * value_pitch + unsigned(col) * unsigned(sizeof(T));
        e_at[j] = 4u * (t * unsigned(s.dv) + unsigned(col));
    }

    f32x4 S[kCt];
#pragma unroll
    for (int ct = 0; ct < kCt; ++ct) S[ct] = zero;
    if (a.initial) {
        const Rsrc from0 = slab_resource(a.initial + slab * state_size, unsigned(state_size * 4));
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) S[ct][i] = load4(from0, state_offset(s, ct, i, g, col));
    }

    In fk[4][kKs];
    Mid ft[kTriBlocks];
    T v[16];
    auto ws_of = [&](int chunk) __attribute__((always_inline)) { return whole(ws_all + size_t(chunk) * Ws::bytes); };
    auto load_keys = [&](int chunk) __attribute__((always_inline)) {
        const Rsrc kr = chunk_rows(a.k, s, b, hk, s.Hk, s.dk, chunk);
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
            for (int m = 0; m < 4; ++m) load_row(fk[m][ks], kr, key_at[m] + 32u * unsigned(ks * sizeof(T)));
    };
    auto load_values = [&](int chunk) __attribute__((always_inline)) {
        const Rsrc vr = chunk_rows(a.v, s, b, h, s.H, s.dv, chunk);
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = load_element<T>(vr, value_at[j]);
    };
    auto load_inverse = [&](int chunk) __attribute__((always_inline)) {
        const Rsrc ws = ws_of(chunk);
#pragma unroll
        for (int i = 0; i < kTriBlocks; ++i) ft[i] = get<Mid>(ws, Ws::inverse, i, lane);
    };
    load_keys(chunk_at(s, 0));
    load_values(chunk_at(s, 0));
    load_inverse(chunk_at(s, 0));
    Scalars sc = load_scalars(ws_of(chunk_at(s, 0)), g);

    for (int step = 0; step < s.chunks; ++step) {
        const int chunk = chunk_at(s, step), next = step + 1 < s.chunks ? chunk_at(s, step + 1) : chunk;
        const Rsrc ws = ws_of(chunk), kw = whole(kw_all + size_t(chunk) * Kw::bytes);
        In fq[4][kKs], fkt[kCt][2];
        Mid2 fp[kTriBlocks];
        if constexpr (!kBwd) {
            const Rsrc qr = chunk_rows(a.q, s, b, hk, s.Hk, s.dk, chunk);
#pragma unroll
            for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
                for (int m = 0; m < 4; ++m) load_row(fq[m][ks], qr, key_at[m] + 32u * unsigned(ks * sizeof(T)));
#pragma unroll
            for (int i = 0; i < kTriBlocks; ++i) fp[i] = get<Mid2>(ws, Ws::scores, i, lane);
        } else {
            const Rsrc to = slab_resource(a.states + (size_t(slab) * s.chunks + chunk) * state_size, unsigned(state_size * 4));
#pragma unroll
            for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
                for (int i = 0; i < 4; ++i) store4(to, state_offset(s, ct, i, g, col), S[ct][i]);
        }
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) fkt[ct][ks] = get<In>(kw, 0, 2 * ct + ks, lane);
        requests_stay();
        Mid fs[kKs];
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) fs[ks] = from<Mid>(S[2 * ks], S[2 * ks + 1]);
        f32x4 e[4], o[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) e[m] = o[m] = zero;
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
            for (int m = 0; m < 4; ++m) mma(e[m], fk[m][ks], fs[ks]);
        load_keys(next);
        requests_stay();
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) e[m][i] = fmaf(-sc.c[m][i], e[m][i], value(v[4 * m + i]));
        load_values(next);
        requests_stay();
        const Mid fe[2] = {from<Mid>(e[0], e[1]), from<Mid>(e[2], e[3])};
#pragma unroll
        for (int m = 0; m < 4; ++m) e[m] = zero;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int m = 2 * ks; m < 4; ++m) mma(e[m], ft[lower_block(m, ks)], fe[ks]);
        load_inverse(next);
        requests_stay();
        if constexpr (kBwd) {
            const Rsrc to = float_rows(a.wrong, s, slab, s.dv, chunk);
#pragma unroll
            for (int j = 0; j < 16; ++j) store4(to, e_at[j], e[j >> 2][j & 3]);
        } else {
#pragma unroll
            for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
                for (int m = 0; m < 4; ++m) mma(o[m], fq[m][ks], first_parts<N, 2>(fs[ks]));
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) e[m] *= sc.beta[m];  // u
        if constexpr (!kBwd) {
            const Mid2 fu[2] = {from<Mid2>(e[0], e[1]), from<Mid2>(e[2], e[3])};
#pragma unroll
            for (int m = 0; m < 4; ++m) o[m] *= sc.c[m];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int m = 2 * ks; m < 4; ++m) mma(o[m], fp[lower_block(m, ks)], fu[ks]);
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) e[m] *= sc.d[m];
        const float whole_decay = sc.whole;
        sc = load_scalars(ws_of(next), g);
        requests_stay();
        const Mid fd[2] = {from<Mid>(e[0], e[1]), from<Mid>(e[2], e[3])};
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct) S[ct] *= whole_decay;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int ct = 0; ct < kCt; ++ct) mma(S[ct], fkt[ct][ks], fd[ks]);
        if constexpr (!kBwd) {
            const Rsrc to = chunk_rows(a.out, s, b, h, s.H, s.dv, chunk);
#pragma unroll
            for (int j = 0; j < 16; ++j) store_element<T>(to, value_at[j], o[j >> 2][j & 3]);
        }
    }
    if (a.final_state) {
        const Rsrc to = slab_resource(a.final_state + slab * state_size, unsigned(state_size * 4));
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) store4(to, state_offset(s, ct, i, g, col), S[ct][i]);
    }
}

template <typename T, int DK, int N>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(1, 1))) void gd_states(ChainArgs<T> a)
{
    states<T, DK, N, false>(a);
}

}  // namespace gd
}  // namespace vig
