// Gated delta rule, gradient (formulas in gated_delta.hpp).  Three launches: gd_prepare; the chains of the states (first chunk to last) and of
// their adjoints (last to first), which do not need each other, side by side; gd_gradients, every chunk on its own.
//
// With r_t the gradient of u_t (w_t = beta_t r_t is that of v_t), per chunk
//     X_ti = G_ti beta_i (dO_t . e_i), i <= t          Y_ti = -G_ti beta_t beta_i (r_t . e_i), i < t     (of q_t . k_i and k_t . k_i)
//     dQ = c . dO S^T + X K                            dK = X^T Q + (Y + Y^T) K + d . beta . e D^T - c . beta . r S^T
//     dbeta_t = r_t . e_t
//     dg_t = sum over everything that decays across t: of the state that enters, what is read after t (a_s), of what is written before t
//            that which leaves (z_i), the pairs i < t <= s, and the state that passes through:
//          = sum_{s >= t} a_s + sum_{i < t} z_i + sum_{s >= t > i} (X_si q_s.k_i + Y_si k_s.k_i) + c_63 <D, S>,
//     a_s = q_s . (c_s dO_s S^T) - k_s . (c_s beta_s r_s S^T),   z_i = k_i . (d_i beta_i e_i D^T)
// (every term carries its own decay; none is the difference of two larger ones).
#include "gated_delta_chain.hpp"
#include "gated_delta_prepare.hpp"
#include "vig_kernels.hpp"
#include "vig_timing.hpp"

namespace vig {

namespace {

using namespace gd;

template <typename T>
struct AdjointArgs {
    Shape s;
    const T *k, *d_out;
    const float *d_final;      // [B, H, dk, dv] or null
    T *dv;
    float *d_initial;          // [B, H, dk, dv] or null
    float *adjoints, *r;       // D of every chunk [slab][chunk][dk][dv], r [slab][L][dv]
    const unsigned char *ws, *key_ws;
};

// The chain of the adjoints for 16 value columns, one wave: the counterpart of gd::states, last chunk first
template <typename T, int DK, int N>
__device__ __forceinline__ void adjoint_chain(const AdjointArgs<T> &a)
{
    using In = typename operands<T, N>::In;
    using Mid = typename operands<T, N>::Mid;
    using Ws = ChunkWs<T, N, true>;
    using Kw = KeyWs<T, DK, true>;
    constexpr int kKs = DK / 32, kCt = DK / 16;
    const Shape &s = a.s;
    const int lane = threadIdx.x, r = lane & 15, g = lane >> 4;
    unsigned slab, part;
    if (!chain_unit(blockIdx.x, unsigned(s.B) * unsigned(s.H), unsigned(s.dv) / 16, slab, part)) return;
    const int b = int(slab / unsigned(s.H)), h = int(slab - unsigned(b) * unsigned(s.H)), hk = h / (s.H / s.Hk);
    const int col = 16 * int(part) + r, last = s.L - 1;
    const Rows<const T> kr = rows_of(a.k, s, b, hk, s.Hk, s.dk), dor = rows_of(a.d_out, s, b, h, s.H, s.dv);
    const Rows<T> dvr = rows_of(a.dv, s, b, h, s.H, s.dv);
    const unsigned char *ws = a.ws + size_t(slab) * s.chunks * Ws::bytes;
    const unsigned char *kw = a.key_ws + (size_t(b) * s.Hk + hk) * s.chunks * Kw::bytes;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

    f32x4 D[kCt];
#pragma unroll
    for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = paired(ct, 4 * g + i);
            D[ct][i] = a.d_final && c < s.dk ? a.d_final[(size_t(slab) * s.dk + c) * s.dv + col] : 0.f;
        }

    In fk[4][kKs], fkt[kCt][2], fqt[kCt][2];
    Mid ft[kTriBlocks], fp[kTriBlocks];
    T dout[16];
    Scalars sc;
    auto load_keys = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int ks = 0; ks < kKs; ++ks) {
                const int t = chunk * kC + paired(m, r);
                row_frag<T>(fk[m][ks], kr, t < last ? t : last, ks, g, s.dk);
            }
    };
    auto load_d_out = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {  // tokens 32 (j / 8) + 8g + j % 8: nothing comes from behind the last
            const int t = chunk * kC + 32 * (j >> 3) + 8 * g + (j & 7);
            dout[j] = t <= last ? dor.p[t * dor.stride + col] : T{};
        }
    };
    auto load_triangles = [&](int chunk) __attribute__((always_inline)) {
        const unsigned char *p = ws + size_t(chunk) * Ws::bytes;
#pragma unroll
        for (int i = 0; i < kTriBlocks; ++i) fp[i] = get<Mid>(p + Ws::scores, i, lane);
#pragma unroll
        for (int i = 0; i < kTriBlocks; ++i) ft[i] = get<Mid>(p + Ws::inverse + kTriBlocks * frag_bytes<Mid>, i, lane);
    };
    auto load_transposed = [&](int chunk) __attribute__((always_inline)) {
        const unsigned char *p = kw + size_t(chunk) * Kw::bytes;
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                fkt[ct][ks] = get<In>(p, 2 * ct + ks, lane);
                fqt[ct][ks] = get<In>(p + Kw::blocks * frag_bytes<In>, 2 * ct + ks, lane);
            }
    };
    load_keys(s.chunks - 1);
    load_d_out(s.chunks - 1);
    load_triangles(s.chunks - 1);
    sc = load_scalars(ws + size_t(s.chunks - 1) * Ws::bytes, g);
    load_transposed(s.chunks - 1);

    for (int chunk = s.chunks - 1; chunk >= 0; --chunk) {
        const int next = chunk > 0 ? chunk - 1 : 0;
        float *to = a.adjoints + (size_t(slab) * s.chunks + chunk) * s.dk * s.dv + col;
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = paired(ct, 4 * g + i);
                if (c < s.dk) to[size_t(c) * s.dv] = D[ct][i];
            }
        Mid fd[kKs];
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) fd[ks] = from<Mid>(D[2 * ks], D[2 * ks + 1]);
        In fo[2];
        f32x4 od[4];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            T x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = dout[8 * p + j];
                od[2 * p + (j >> 2)][j & 3] = io<T>::load(&x[j]) * sc.c[2 * p + (j >> 2)][j & 3];
            }
            gather(fo[p], x);
        }
        load_d_out(next);
        f32x4 u[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            u[m] = zero;
#pragma unroll
            for (int ks = 0; ks < kKs; ++ks) mma(u[m], fk[m][ks], fd[ks]);
            u[m] *= sc.d[m];
#pragma unroll
            for (int ks = m >> 1; ks < 2; ++ks) mma(u[m], fp[upper_block(m, ks)], fo[ks]);
            u[m] *= sc.beta[m];
        }
        load_keys(next);
        const Mid fu[2] = {from<Mid>(u[0], u[1]), from<Mid>(u[2], u[3])};
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            u[m] = zero;
#pragma unroll
            for (int ks = m >> 1; ks < 2; ++ks) mma(u[m], ft[upper_block(m, ks)], fu[ks]);
        }
        load_triangles(next);
        float *rt = a.r + size_t(slab) * s.L * s.dv + col;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = chunk * kC + paired(m, 4 * g + i);
                if (t <= last) {
                    io<T>::store(dvr.p + t * dvr.stride + col, fabsf(sc.beta[m][i]) > 1e-20f ? u[m][i] : 0.f);
                    rt[size_t(t) * s.dv] = u[m][i] / sc.beta[m][i];
                }
                u[m][i] *= -sc.c[m][i];
            }
        const Mid fw[2] = {from<Mid>(u[0], u[1]), from<Mid>(u[2], u[3])}, fod[2] = {from<Mid>(od[0], od[1]), from<Mid>(od[2], od[3])};
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct) {
            D[ct] *= sc.whole;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                mma(D[ct], fqt[ct][ks], fod[ks]);
                mma(D[ct], fkt[ct][ks], fw[ks]);
            }
        }
        load_transposed(next);
        sc = load_scalars(ws + size_t(next) * Ws::bytes, g);
    }
    if (a.d_initial)
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = paired(ct, 4 * g + i);
                if (c < s.dk) a.d_initial[(size_t(slab) * s.dk + c) * s.dv + col] = D[ct][i];
            }
}

template <typename T, int DK, int N>
__global__ __launch_bounds__(64) void gd_both_chains(ChainArgs<T> c, AdjointArgs<T> a)
{
    if (blockIdx.y == 0)
        states<T, DK, N, true>(c);
    else
        adjoint_chain<T, DK, N>(a);
}

template <typename T>
struct GradientArgs {
    Shape s;
    const T *q, *k, *g, *beta, *d_out;
    T *dq, *dk, *dg, *dbeta;
    const float *states, *adjoints, *wrong, *r;
    const unsigned char *key_ws;
};

// eight 32-bit values of a row whose columns from `width` on are zero
__device__ __forceinline__ void row8(float (&x)[8], const float *row, int c, int width)
{
    f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
    if (c < width) lo = *reinterpret_cast<const f32x4 *>(row + c), hi = *reinterpret_cast<const f32x4 *>(row + c + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = lo[j], x[4 + j] = hi[j];
}

// sum over the 16 lanes of a row, in its lane 15
__device__ __forceinline__ float row_sum(float x) { return row_scan<0>(x); }

// One chunk of one key head and all value heads that share it, four waves, 16 tokens each
template <typename T, int DK, int DV>
__global__ __launch_bounds__(256) void gd_gradients(GradientArgs<T> a)
{
    using In = typename operands<T, 2>::In;
    using Mid = typename operands<T, 2>::Mid;
    using Kw = KeyWs<T, DK, true>;
    constexpr int kKs = DK / 32, kCt = DK / 16, kVs = DV / 32;
    __shared__ __align__(16) float X[kC * kPitch], Y[kC * kPitch];
    __shared__ double sum[kC];
    __shared__ float bet[kC], enters[kC], leaves[kC], pairs[4][kC], through[4];
    const Shape &s = a.s;
    const int w = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const unsigned unit = blockIdx.x, key_slab = unit / unsigned(s.chunks), chunk = unit - key_slab * unsigned(s.chunks);
    const int b = int(key_slab / unsigned(s.Hk)), hk = int(key_slab - unsigned(b) * unsigned(s.Hk)), share = s.H / s.Hk;
    const int t0 = int(chunk) * kC, last = s.L - 1;
    const Rows<const T> qr = rows_of(a.q, s, b, hk, s.Hk, s.dk), kr = rows_of(a.k, s, b, hk, s.Hk, s.dk);
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    auto row = [&](int t) __attribute__((always_inline)) { return t0 + t < last ? t0 + t : last; };
    const unsigned char *kw = a.key_ws + size_t(unit) * Kw::bytes;

    f32x4 qk[4], kk[4], dq[kCt], dk[kCt];
    {
        In fq[kKs], fk[kKs];
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) row_frag<T>(fq[ks], qr, row(16 * w + r), ks, g, s.dk), row_frag<T>(fk[ks], kr, row(16 * w + r), ks, g, s.dk);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            qk[n] = kk[n] = zero;
            if (n > w) continue;
#pragma unroll
            for (int ks = 0; ks < kKs; ++ks) {
                In fb;
                row_frag<T>(fb, kr, row(16 * n + r), ks, g, s.dk);
                mma(qk[n], fq[ks], fb);
                mma(kk[n], fk[ks], fb);
            }
        }
    }
#pragma unroll
    for (int ct = 0; ct < kCt; ++ct) dq[ct] = dk[ct] = zero;

    for (int h = hk * share; h < (hk + 1) * share; ++h) {
        const size_t slab = size_t(b) * s.H + h;
        const Rows<const T> dor = rows_of(a.d_out, s, b, h, s.H, s.dv);
        const float *S = a.states + (slab * s.chunks + chunk) * s.dk * s.dv, *D = a.adjoints + (slab * s.chunks + chunk) * s.dk * s.dv;
        const float *e = a.wrong + slab * s.L * s.dv, *rr = a.r + slab * s.L * s.dv;
        if (w == 0) {
            const Rows<const T> gr = rows_of(a.g, s, b, h, s.H, 1), br = rows_of(a.beta, s, b, h, s.H, 1);
            const bool there = t0 + lane <= last;
            sum[lane] = wave_prefix(there ? double(fmaxf(io<T>::load(gr.p + row(lane) * gr.stride), kGateFloor)) : 0.0, lane);
            bet[lane] = there ? beta_divisor(io<T>::load(br.p + row(lane) * br.stride)) : 0.f;
        }
        // operands of the wave's tokens; dbeta
        In fo[kVs];
        Mid fr[kVs], fe[kVs];
        float db = 0.f;
#pragma unroll
        for (int ks = 0; ks < kVs; ++ks) {
            row_frag<T>(fo[ks], dor, row(16 * w + r), ks, g, s.dv);
            float x[8], y[8];
            row8(x, e + size_t(row(16 * w + r)) * s.dv, 32 * ks + 8 * g, s.dv);
            row8(y, rr + size_t(row(16 * w + r)) * s.dv, 32 * ks + 8 * g, s.dv);
            make(fe[ks], x);
            make(fr[ks], y);
#pragma unroll
            for (int j = 0; j < 8; ++j) db = fmaf(x[j], y[j], db);
        }
        db += __shfl_xor(db, 16);
        db += __shfl_xor(db, 32);
        if (g == 0 && t0 + 16 * w + r <= last) {
            const Rows<T> dbr = rows_of(a.dbeta, s, b, h, s.H, 1);
            io<T>::store(dbr.p + (t0 + 16 * w + r) * dbr.stride, db);
        }
        // <D, S>
        float ds = 0.f;
        for (int i = 4 * int(threadIdx.x); i < s.dk * s.dv; i += 1024) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(S + i), y = *reinterpret_cast<const f32x4 *>(D + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) ds = fmaf(x[j], y[j], ds);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) ds += __shfl_xor(ds, d);
        if (lane == 0) through[w] = ds;
        __syncthreads();

        // X, Y and the pairs' part of dg
        float carry[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            f32x4 x = zero, y = zero;
            if (n <= w) {
#pragma unroll
                for (int ks = 0; ks < kVs; ++ks) {
                    float v[8];
                    row8(v, e + size_t(row(16 * n + r)) * s.dv, 32 * ks + 8 * g, s.dv);
                    Mid fn;
                    make(fn, v);
                    mma(x, fo[ks], fn);
                    mma(y, fr[ks], fn);
                }
            }
            float column = 0.f;
            const int c = 16 * n + r;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = 16 * w + 4 * g + i;
                const bool in = c <= t && t0 + t <= last;
                const float decay = in ? expf(float(sum[t] - sum[c])) * bet[c] : 0.f;
                const float xi = in ? decay * x[i] : 0.f, yi = in && c < t ? -decay * bet[t] * y[i] : 0.f;
                X[t * kPitch + c] = xi;
                Y[t * kPitch + c] = yi;
                if (n <= w) {
                    const float z = c < t ? xi * qk[n][i] + yi * kk[n][i] : 0.f, upto = row_scan<0>(z);
                    column += c <= t ? upto - z + carry[i] : 0.f;  // pairs (t, i < c)
                    carry[i] += __shfl(upto, lane | 15);
                }
            }
            column += __shfl_xor(column, 16);
            column += __shfl_xor(column, 32);
            if (g == 0) pairs[w][c] = column;
        }
        __syncthreads();

        Mid fx[2], fxt[2], fy[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const int t = 16 * w + r, c = 32 * ks + 8 * g;
            float x[8], xt[8], y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = X[t * kPitch + c + j];
                xt[j] = X[(c + j) * kPitch + t];
                y[j] = Y[t * kPitch + c + j] + Y[(c + j) * kPitch + t];
            }
            make(fx[ks], x);
            make(fxt[ks], xt);
            make(fy[ks], y);
        }
        f32x4 read, erase, write;  // factors of the three products with the states, by token
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 16 * w + 4 * g + i;
            const float c = expf(float(sum[t])), d = expf(float(sum[kC - 1] - sum[t]));
            const bool in = t0 + t <= last;
            read[i] = in ? c : 0.f;
            erase[i] = in ? -c * bet[t] : 0.f;
            write[i] = in ? d * bet[t] : 0.f;
        }
        f32x4 enter = zero, leave = zero;
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct) {
            const int c = paired(ct, r);
            const bool has = c < s.dk;
            f32x4 x = zero, y = zero, z = zero;
#pragma unroll
            for (int ks = 0; ks < kVs; ++ks) {
                float v[8];
                Mid f;
                row8(v, S + size_t(has ? c : 0) * s.dv, 32 * ks + 8 * g, has ? s.dv : 0);
                make(f, v);
                mma(x, fo[ks], f);
                mma(y, fr[ks], f);
                row8(v, D + size_t(has ? c : 0) * s.dv, 32 * ks + 8 * g, has ? s.dv : 0);
                make(f, v);
                mma(z, fe[ks], f);
            }
            x *= read;
            y *= erase;
            z *= write;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = row(16 * w + 4 * g + i);
                const float qe = has ? io<T>::load(qr.p + t * qr.stride + c) : 0.f, ke = has ? io<T>::load(kr.p + t * kr.stride + c) : 0.f;
                enter[i] = fmaf(qe, x[i], fmaf(ke, y[i], enter[i]));
                leave[i] = fmaf(ke, z[i], leave[i]);
            }
            dq[ct] += x;
            dk[ct] += y + z;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const In fkt = get<In>(kw, 2 * ct + ks, lane), fqt = get<In>(kw + Kw::blocks * frag_bytes<In>, 2 * ct + ks, lane);
                mma(dq[ct], fx[ks], fkt);
                mma(dk[ct], fxt[ks], fqt);
                mma(dk[ct], fy[ks], fkt);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float en = row_sum(enter[i]), le = row_sum(leave[i]);
            if (r == 15) enters[16 * w + 4 * g + i] = en, leaves[16 * w + 4 * g + i] = le;
        }
        __syncthreads();
        if (w == 0) {
            float after = enters[lane], before = leaves[lane];
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const float x = __shfl_down(after, d), y = __shfl_up(before, d);
                after += lane + d < 64 ? x : 0.f;
                before += lane >= d ? y : 0.f;
            }
            const float earlier = __shfl_up(before, 1);
            before = lane > 0 ? earlier : 0.f;
            const float state = expf(float(sum[kC - 1])) * ((through[0] + through[1]) + (through[2] + through[3]));
            const float dg = after + before + ((pairs[0][lane] + pairs[1][lane]) + (pairs[2][lane] + pairs[3][lane])) + state;
            if (t0 + lane <= last) {
                const Rows<T> dgr = rows_of(a.dg, s, b, h, s.H, 1);
                io<T>::store(dgr.p + (t0 + lane) * dgr.stride, dg);
            }
        }
        __syncthreads();
    }
    const Rows<T> dqr = rows_of(a.dq, s, b, hk, s.Hk, s.dk), dkr = rows_of(a.dk, s, b, hk, s.Hk, s.dk);
#pragma unroll
    for (int ct = 0; ct < kCt; ++ct) {
        const int c = paired(ct, r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + 16 * w + 4 * g + i;
            if (t <= last && c < s.dk) {
                io<T>::store(dqr.p + t * dqr.stride + c, dq[ct][i]);
                io<T>::store(dkr.p + t * dkr.stride + c, dk[ct][i]);
            }
        }
    }
}

struct Buffers {
    size_t key_ws, states, adjoints, wrong, r, bytes;
};
template <typename T, int DK, int N>
Buffers buffers(const Shape &s)
{
    const size_t slabs = size_t(s.B) * s.H, units = slabs * s.chunks;
    Buffers at;
    at.key_ws = round256(units * ChunkWs<T, N, true>::bytes);
    at.states = at.key_ws + round256(size_t(s.B) * s.Hk * s.chunks * KeyWs<T, DK, true>::bytes);
    at.adjoints = at.states + round256(units * s.dk * s.dv * 4);
    at.wrong = at.adjoints + round256(units * s.dk * s.dv * 4);
    at.r = at.wrong + round256(slabs * s.L * s.dv * 4);
    at.bytes = at.r + round256(slabs * s.L * s.dv * 4);
    return at;
}

template <typename T, int DK, int N>
hipError_t launch(const Shape &s, const GradientPointers &p, void *workspace, hipStream_t stream)
{
    const unsigned slabs = unsigned(s.B) * unsigned(s.H);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    const Buffers at = buffers<T, DK, N>(s);
    const T *q = static_cast<const T *>(p.q), *k = static_cast<const T *>(p.k), *v = static_cast<const T *>(p.v), *g = static_cast<const T *>(p.g),
            *beta = static_cast<const T *>(p.beta), *d_out = static_cast<const T *>(p.d_out);
    float *S = reinterpret_cast<float *>(ws + at.states), *D = reinterpret_cast<float *>(ws + at.adjoints), *e = reinterpret_cast<float *>(ws + at.wrong),
          *r = reinterpret_cast<float *>(ws + at.r);
    const PrepareArgs<T> prepare = {s, q, k, g, beta, ws, ws + at.key_ws};
    const ChainArgs<T> chain = {s, q, k, v, p.initial, nullptr, nullptr, S, e, ws, ws + at.key_ws};
    const AdjointArgs<T> adjoint = {s, k, d_out, p.d_final, static_cast<T *>(p.dv), p.d_initial, D, r, ws, ws + at.key_ws};
    const GradientArgs<T> gradient = {s, q, k, g, beta, d_out, static_cast<T *>(p.dq), static_cast<T *>(p.dk), static_cast<T *>(p.dg),
                                      static_cast<T *>(p.dbeta), S, D, e, r, ws + at.key_ws};
    const LaunchTimer timer(kKernelGatedDeltaBackward, stream);
    gd_prepare<T, DK, N, true><<<slabs * unsigned(s.chunks), 256, 0, stream>>>(prepare);
    gd_both_chains<T, DK, N><<<dim3((slabs + 7) / 8 * 8 * unsigned(s.dv / 16), 2), 64, 0, stream>>>(chain, adjoint);
    const unsigned key_units = unsigned(s.B) * unsigned(s.Hk) * unsigned(s.chunks);
    if (s.dv <= 32)
        gd_gradients<T, DK, 32><<<key_units, 256, 0, stream>>>(gradient);
    else if (s.dv <= 64)
        gd_gradients<T, DK, 64><<<key_units, 256, 0, stream>>>(gradient);
    else
        gd_gradients<T, DK, 128><<<key_units, 256, 0, stream>>>(gradient);
    return hipGetLastError();
}

// a returned gradient of the initial state takes three parts of 32-bit operands, bf16 gradients two
template <typename T, int DK>
hipError_t launch_parts(const Shape &s, const GradientPointers &p, void *workspace, hipStream_t stream)
{
    if constexpr (sizeof(T) == 2)
        if (p.d_initial) return launch<T, DK, 3>(s, p, workspace, stream);
    return launch<T, DK, 2>(s, p, workspace, stream);
}

template <typename T>
hipError_t launch_width(const Shape &s, const GradientPointers &p, void *workspace, hipStream_t stream)
{
    if (s.dk <= 32) return launch_parts<T, 32>(s, p, workspace, stream);
    if (s.dk <= 64) return launch_parts<T, 64>(s, p, workspace, stream);
    return launch_parts<T, 128>(s, p, workspace, stream);
}

}  // namespace

size_t gated_delta_bwd_workspace_bytes(int B, int H, int Hk, int L, int dk, int dv, bool is_bf16)
{
    const Shape s = {B, H, Hk, L, dk, dv, (L + kC - 1) / kC, false, false};
    const auto of = [&](auto t) {
        using T = decltype(t);
        return (dk <= 32 ? buffers<T, 32, 3>(s) : dk <= 64 ? buffers<T, 64, 3>(s) : buffers<T, 128, 3>(s)).bytes;
    };
    return is_bf16 ? of(bf16_t{}) : of(float{});
}

hipError_t gated_delta_bwd_launch(const GradientPointers &p, int B, int H, int Hk, int L, int dk, int dv, bool is_bf16, bool token_major, bool reverse,
                                  void *workspace, hipStream_t stream)
{
    const Shape s = {B, H, Hk, L, dk, dv, (L + kC - 1) / kC, token_major, reverse};
    return is_bf16 ? launch_width<bf16_t>(s, p, workspace, stream) : launch_width<float>(s, p, workspace, stream);
}

}  // namespace vig
