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

// sums over the four rows of 16 lanes
__device__ __forceinline__ float rows_total(float x)
{
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

template <typename T>
struct AdjointArgs {
    Shape s;
    const T *k, *d_out;
    const float *d_final;         // [B, H, dk, dv] or null
    T *dv;
    float *d_initial;             // [B, H, dk, dv] or null
    unsigned char *adjoints, *r;  // D and r of every chunk as fragments, see gd::Tile
    const unsigned char *ws, *key_ws;
};

// The chain of the adjoints for 16 value columns, last chunk first, the counterpart of gd::states: one wave holds D and takes the three products
// that depend on it; a second one makes what does not, (P diag(beta))^T dO and Q^T (c . dO), a chunk ahead, and takes D, w and r away, a chunk behind.
template <int DK>
struct AdjointLds {
    static constexpr int ahead = 4096 + DK * 64;                     // (P diag(beta))^T dO, Q^T (c . dO): accumulators, 16 bytes a lane
    static constexpr int behind = Tile<DK>::bytes + Tile<kC>::bytes;  // D, w
    static constexpr int bytes = 2 * (ahead + behind);
};

template <typename T, int DK, int N>
__device__ __forceinline__ void adjoint_chain(const AdjointArgs<T> &a, const Columns &at, unsigned char *scal, unsigned char *lds)
{
    using In = typename operands<T, N>::In;
    using Mid = typename operands<T, N>::Mid;
    using Ws = ChunkWs<T, N, true>;
    using Kw = KeyWs<T, DK, true>;
    using Lds = AdjointLds<DK>;
    constexpr int kKs = DK / 32, kCt = DK / 16;
    const Shape &s = a.s;
    const int lane = at.lane, r = at.r, g = at.g, col = at.col;
    const unsigned char *ws_all = a.ws + size_t(at.slab) * s.chunks * Ws::bytes;
    const unsigned char *kw_all = a.key_ws + (size_t(at.b) * s.Hk + at.hk) * s.chunks * Kw::bytes;
    const size_t state_size = size_t(s.dk) * s.dv;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const unsigned key_pitch = pitch_of<T>(s, s.Hk, s.dk);
    unsigned key_at[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) key_at[m] = row_offset<T>(key_pitch, token_at(s, paired(m, r)), 0, g, s.dk);

    f32x4 D[kCt];
#pragma unroll
    for (int ct = 0; ct < kCt; ++ct) D[ct] = zero;
    if (a.d_final) {
        const Rsrc from0 = slab_resource(a.d_final + at.slab * state_size, unsigned(state_size * 4));
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) D[ct][i] = load4(from0, state_offset(s, ct, i, g, col));
    }

    const int first = chunk_at(s, s.chunks - 1), move = s.reverse ? 1 : -1;
    Walk kr = walk_rows(a.k, s, at.b, at.hk, s.Hk, s.dk, first, move), ws = walk_blocks(ws_all, Ws::bytes, first, move),
         kw = walk_blocks(kw_all, Kw::bytes, first, move);
    In fk[4][kKs], fkt[kCt][2];
    Mid ft[kTriBlocks];
    auto load_keys = [&]() __attribute__((always_inline)) {
        const Rsrc from0 = kr.here();
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
            for (int m = 0; m < 4; ++m) load_row(fk[m][ks], from0, key_at[m] + 32u * unsigned(ks * sizeof(T)));
    };
    auto load_inverse = [&]() __attribute__((always_inline)) {
        const Rsrc from0 = ws.here();
#pragma unroll
        for (int i = 0; i < kTriBlocks; ++i) ft[i] = get<Mid>(from0, Ws::inverse + kTriBlocks * frag_bytes<Mid>, i, lane);
    };
    auto load_transposed = [&]() __attribute__((always_inline)) {
        const Rsrc from0 = kw.here();
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int ct = 0; ct < kCt; ++ct) fkt[ct][ks] = get<In>(from0, 0, 2 * ct + ks, lane);
    };
    // (in the order of the loop, see gd::states)
    u32x4 raw = request_scalars(ws.here(), lane);
    requests_stay();
    load_keys();
    requests_stay();
    load_inverse();
    requests_stay();
    load_transposed();
    requests_stay();

    for (int step = s.chunks - 1; step >= 0; --step) {
        if (step > 0) kr.next(), ws.next(), kw.next();  // what is requested from here on
        unsigned char *ahead = lds + (step & 1) * Lds::ahead, *behind = lds + 2 * Lds::ahead + (step & 1) * Lds::behind;
        __syncthreads();
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct) tile_put<DK>(behind, ct, r, g, D[ct]);
        share_scalars(scal, raw, lane);
        requests_stay();
        raw = request_scalars(ws.here(), lane);
        requests_stay();
        Mid fd[kKs];
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) fd[ks] = from<Mid>(D[2 * ks], D[2 * ks + 1]);
        f32x4 u[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) u[m] = zero;
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks)
            mma_tiles(u, 0, 4, [&](int m) -> const In & { return fk[m][ks]; }, fd[ks]);
        requests_stay();
        load_keys();
        requests_stay();
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const f32x4 d = scalars(scal, kRead, m, g), pd = *reinterpret_cast<const f32x4 *>(ahead + 1024 * m + 16 * lane);
#pragma unroll
            for (int i = 0; i < 4; ++i) u[m][i] = fmaf(d[i], u[m][i], pd[i]);
        }
        const Mid fu[2] = {from<Mid>(u[0], u[1]), from<Mid>(u[2], u[3])};
#pragma unroll
        for (int m = 0; m < 4; ++m) u[m] = zero;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
            mma_tiles(u, 0, 2 * ks + 2, [&](int m) -> const Mid & { return ft[upper_block(m, ks)]; }, fu[ks]);
        requests_stay();
        load_inverse();
        requests_stay();
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            tile_put<kC>(behind + Tile<DK>::bytes, m, r, g, u[m]);
            u[m] *= -scalars(scal, kC0, m, g);
        }
        const float all = whole_decay(scal);
        const Mid fw[2] = {from<Mid>(u[0], u[1]), from<Mid>(u[2], u[3])};
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct) {
            const f32x4 qd = *reinterpret_cast<const f32x4 *>(ahead + 4096 + 1024 * ct + 16 * lane);
#pragma unroll
            for (int i = 0; i < 4; ++i) D[ct][i] = fmaf(all, D[ct][i], qd[i]);
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
            mma_tiles(D, 0, kCt, [&](int ct) -> const In & { return fkt[ct][ks]; }, fw[ks]);
        requests_stay();
        load_transposed();
        requests_stay();
    }
    __syncthreads();
    if (a.d_initial) {
        const Rsrc to = slab_resource(a.d_initial + at.slab * state_size, unsigned(state_size * 4));
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) store4(to, state_offset(s, ct, i, g, col), D[ct][i]);
    }
}

template <typename T, int DK, int N>
__device__ __forceinline__ void adjoint_sides(const AdjointArgs<T> &a, const Columns &at, unsigned char *own /* the wave's: two chunks' scalars, then a strip */,
                                              unsigned char *lds)
{
    using In = typename operands<T, N>::In;
    using Mid = typename operands<T, N>::Mid;
    using Mid2 = typename operands<T, 2>::Mid;
    using Ws = ChunkWs<T, N, true>;
    using Kw = KeyWs<T, DK, true>;
    using Lds = AdjointLds<DK>;
    constexpr int kCt = DK / 16;
    const Shape &s = a.s;
    const int lane = at.lane, g = at.g, part = at.col >> 4;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const unsigned value_pitch = pitch_of<T>(s, s.H, s.dv);
    unsigned value_at[Strip<T>::loads];
#pragma unroll
    for (int l = 0; l < Strip<T>::loads; ++l) value_at[l] = strip_offset<T>(s, value_pitch, part, lane, l);
    const size_t state_bytes = emitted_bytes<T>(DK / 16, s.dv), token_bytes = emitted_bytes<T>(4, s.dv), units = size_t(at.slab) * s.chunks;

    const int first = chunk_at(s, s.chunks - 1), move = s.reverse ? 1 : -1;
    // (what is taken away starts a chunk late)
    Walk dor = walk_rows(a.d_out, s, at.b, at.h, s.H, s.dv, first, move),
         dvr = walk_rows(static_cast<const T *>(a.dv), s, at.b, at.h, s.H, s.dv, first - move, move),
         ws = walk_blocks(a.ws + units * Ws::bytes, Ws::bytes, first, move),
         kw = walk_blocks(a.key_ws + (size_t(at.b) * s.Hk + at.hk) * s.chunks * Kw::bytes, Kw::bytes, first, move),
         to_d = walk_blocks(a.adjoints + units * state_bytes, state_bytes, first - move, move),
         to_r = walk_blocks(a.r + units * token_bytes, token_bytes, first - move, move);
    In fqt[kCt][2];
    Mid fp[kTriBlocks];
    Strip<T> dout;
    u32x4 raw;
    int left = s.chunks;  // chunks from the one requested on
    auto request_rows = [&]() __attribute__((always_inline)) {
        const Rsrc from0 = dor.here();
        raw = request_scalars(ws.here(), lane);
#pragma unroll
        for (int l = 0; l < Strip<T>::loads; ++l) dout.w[l] = load16(from0, value_at[l]);
    };
    auto request_scores = [&]() __attribute__((always_inline)) {
        const Rsrc from0 = ws.here();
#pragma unroll
        for (int i = 0; i < kTriBlocks; ++i) fp[i] = get<Mid>(from0, Ws::scores, i, lane);
    };
    auto request_queries = [&]() __attribute__((always_inline)) {
        const Rsrc from0 = kw.here();
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int ct = 0; ct < kCt; ++ct) fqt[ct][ks] = get<In>(from0, Kw::blocks * frag_bytes<In>, 2 * ct + ks, lane);
    };
    // a chunk's part without D, and the requests of the next one as registers become free (what is made ahead of the last step is never read)
    auto make_ahead = [&](int step) __attribute__((always_inline)) {
        unsigned char *to = lds + (step & 1) * Lds::ahead, *scal = own + (step & 1) * kScalarBytes, *strip = own + 2 * kScalarBytes;
        if (--left > 0) ws.next(), kw.next(), dor.next();
        In fo[2];
        Mid fod[2];
        strip_put(strip, dout, lane);
        share_scalars(scal, raw, lane);
        requests_stay();
        request_rows();
        requests_stay();
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            T x[8];
            float y[8];
            strip_column(x, strip, p, at.r, g);
            const f32x4 c[2] = {scalars(scal, kC0, 2 * p, g), scalars(scal, kC0, 2 * p + 1, g)};
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = value(x[j]) * c[j >> 2][j & 3];
            gather(fo[p], x);
            make(fod[p], y);
        }
        f32x4 w[4], qd[kCt];
#pragma unroll
        for (int m = 0; m < 4; ++m) w[m] = zero;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
            mma_tiles(w, 0, 2 * ks + 2, [&](int m) -> const Mid & { return fp[upper_block(m, ks)]; }, fo[ks]);
        requests_stay();
        request_scores();
        requests_stay();
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct) qd[ct] = zero;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
            mma_tiles(qd, 0, kCt, [&](int ct) -> const In & { return fqt[ct][ks]; }, fod[ks]);
        requests_stay();
        request_queries();
        requests_stay();
#pragma unroll
        for (int m = 0; m < 4; ++m) *reinterpret_cast<f32x4 *>(to + 1024 * m + 16 * lane) = w[m];
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct) *reinterpret_cast<f32x4 *>(to + 4096 + 1024 * ct + 16 * lane) = qd[ct];
    };
    // takes chunk `step` away; one that is not there goes nowhere
    auto take = [&](int step) __attribute__((always_inline)) {
        const unsigned char *behind = lds + 2 * Lds::ahead + (step & 1) * Lds::behind, *scal = own + (step & 1) * kScalarBytes;
        const bool there = step < s.chunks;
        const Rsrc to = to_d.here(there), tr = to_r.here(there), dv0 = dvr.here(there);
        to_d.next(), to_r.next(), dvr.next();
        float x[8];
#pragma unroll
        for (int i = 0; i < DK / 32; ++i) {
            const int item = 64 * i + lane;
            tile_row<DK>(x, behind, item >> 1, item & 1);
            emit<Mid2>(to, unpaired(item >> 1), part, item & 1, s.dv, x);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int item = 64 * i + lane, t = item >> 1;
            tile_row<kC>(x, behind + Tile<DK>::bytes, t, item & 1);
            const float inverse = *reinterpret_cast<const float *>(scal + kInverseBeta + 4 * t);
            const bool written = fabsf(inverse) < 0.99f / kLeastStrength;  // beta is not the stand-in for zero
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                y[j] = written ? x[j] : 0.f;
                x[j] *= inverse;
            }
            store_row(dv0, unsigned(token_at(s, t)) * value_pitch + unsigned(16 * part + 8 * (item & 1)) * unsigned(sizeof(T)), y, T{});
            emit<Mid2>(tr, natural(t), part, item & 1, s.dv, x);
        }
    };
    // (no branches around requests and stores: a wait counts what was asked for behind what it is for, and where paths with different counts
    // meet, that is everything)
    request_rows();
    requests_stay();
    request_scores();
    requests_stay();
    request_queries();
    requests_stay();
    make_ahead(s.chunks - 1);
    for (int step = s.chunks - 1; step >= 0; --step) {
        __syncthreads();
        take(step + 1);
        requests_stay();
        make_ahead(step - 1);
    }
    __syncthreads();
    take(0);
}

// Two waves per 16 columns of the states' chain (blockIdx.y = 0) and of the adjoints'.  8 x 6 heads of 4096 tokens (bf16, 64 x 64): 167 us for 160 MB in and
// 222 MB out; one chain after the other 87 + 129 us.  A load a line two chunks ahead, to have them in L2, costs more (197 us) than it saves.
template <typename T, int DK, int N>
__global__ __launch_bounds__(128) __attribute__((amdgpu_waves_per_eu(chain_waves<T, DK, 1>, chain_waves<T, DK, 1>))) void gd_both_chains(ChainArgs<T> c, AdjointArgs<T> a)
{
    __shared__ __align__(16) unsigned char lds[AdjointLds<DK>::bytes], scal[kScalarBytes + Strip<T>::bytes], own[2 * kScalarBytes + Strip<T>::bytes];
    Columns at;
    if (!columns_of(a.s, at)) return;
    if (blockIdx.y == 0) {
        if (threadIdx.x < 64)
            states<T, DK, N, true, 1>(c, at, 0, scal, lds, nullptr);
        else
            emit_states<T, DK>(c, at, lds);
    } else {
        if (threadIdx.x < 64)
            adjoint_chain<T, DK, N>(a, at, scal, lds);
        else
            adjoint_sides<T, DK, N>(a, at, own, lds);
    }
}

template <typename T>
struct GradientArgs {
    Shape s;
    const T *q, *k, *g, *beta, *d_out;
    T *dq, *dk, *dg, *dbeta;
    const unsigned char *states, *adjoints, *wrong, *r;  // fragments, see gd::Tile
};

// the tokens 16 w + 4g .. + 3 of channel paired(tile, r) of rows in LDS
template <int DK>
__device__ __forceinline__ f32x4 four_tokens(const Whole &, const unsigned char *lds, int tile, int w, int r, int g)
{
    const uint16_t *q = reinterpret_cast<const uint16_t *>(lds) + (16 * w + 4 * g + (r >> 2)) * KeyTile<bf16_t, DK>::pitch + paired(tile, 4 * (r & 3));
    return unpack4(__builtin_bit_cast(uint2, lds_read_tr(q)));
}
template <int DK>
__device__ __forceinline__ f32x4 four_tokens(const Full &, const unsigned char *lds, int tile, int w, int r, int g)
{
    const float *q = reinterpret_cast<const float *>(lds) + (16 * w + 4 * g) * KeyTile<float, DK>::pitch + paired(tile, r);
    return f32x4{q[0], q[KeyTile<float, DK>::pitch], q[2 * KeyTile<float, DK>::pitch], q[3 * KeyTile<float, DK>::pitch]};
}

__device__ __forceinline__ void lds_element(bf16_t *p, float x) { p->bits = uint16_t(pack2(x, x)); }
__device__ __forceinline__ void lds_element(float *p, float x) { *p = x; }

// a fragment at a lane's offset (0, or nowhere for one that is not there)
template <typename Frag>
__device__ __forceinline__ Frag get_at(Rsrc ws, unsigned at, int block, int lane)
{
    u32x4 w[planes<Frag>];
#pragma unroll
    for (int i = 0; i < planes<Frag>; ++i) w[i] = load16(ws, at | (unsigned(block * planes<Frag> + i) * 1024u + 16u * unsigned(lane)));
    Frag f;
    __builtin_memcpy(&f, w, sizeof(f));
    return f;
}
// The sum of products of the rows of two tiles, in parts: the matrix cores' products of every row with every row, of which the diagonal is wanted (two
// instructions a part where unpacking and adding up takes eighty); 32-bit values one by one.
__device__ __forceinline__ void inner(f32x4 &acc, const Parts<2> &a, const Parts<2> &b) { mma(acc, a, b); }
__device__ __forceinline__ void inner(f32x4 &acc, const Full &a, const Full &b)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[0] = fmaf(a.v[j], b.v[j], acc[0]);
}
template <typename Frag>
__device__ __forceinline__ float of_lane(const f32x4 &acc, int r, int g)
{
    if constexpr (std::is_same<Frag, Full>::value) return acc[0];
    const float x = (r & 2) ? ((r & 1) ? acc[3] : acc[2]) : ((r & 1) ? acc[1] : acc[0]);
    return (r >> 2) == g ? x : 0.f;
}

// One chunk of one key head and all value heads that share it, four waves, 16 tokens each.  What more than one wave needs -- rows of k and q, e, the rows
// of S and D -- each requests a quarter of and all read from LDS; every request of a turn stands before its first wait: one trip to memory
// a turn.  The contractions over value columns take kSlice of them at a time.  Bound by the phases of two waves a SIMD (64 x 64, bf16: 1200 vector and 180 matrix
// instructions each, ten phases between barriers): 8 x 6 heads of 4096 tokens take 77 us, and 90 in
// workgroups that go on to another chunk with its requests under way.
// kOne: the values are one slice; two workgroups then fit a compute unit's registers (without it the accumulators are live across the
// requests of the next slice, and what spills costs more than the second workgroup brings).
template <typename T, int DK, bool kOne>
__global__ __launch_bounds__(256, kOne && DK <= 64 && sizeof(T) == 2 ? 2 : 1) void gd_gradients(GradientArgs<T> a)
{
    using In = typename operands<T, 2>::In;
    using Mid = typename operands<T, 2>::Mid;
    constexpr int kKs = DK / 32, kCt = DK / 16, kSlice = DK <= 64 ? 64 : 32, kVs = kSlice / 32;
    constexpr int kStates = 2 * kCt * kVs * int(frag_bytes<Mid>), kTiles = 2 * kC * kPitch * 4, kOwn = (kCt * kVs + 3) / 4;
    extern __shared__ __align__(16) unsigned char shared[];  // the rows of S and D, afterwards X and Y; then what is below
    unsigned char *wrong = shared + (kStates > kTiles ? kStates : kTiles), *keys = wrong + 4 * kVs * frag_bytes<Mid>,
                  *queries = keys + KeyTile<T, DK>::bytes;
    __shared__ double sum[4][kC];
    __shared__ float bet[4][kC], enters[kC], leaves[kC], pairs[4][kC], through[4];
    float *X = reinterpret_cast<float *>(shared), *Y = X + kC * kPitch;
    unsigned char *fS = shared, *fD = shared + kStates / 2;
    const Shape &s = a.s;
    const int w = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6));
    int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const unsigned unit = blockIdx.x, key_slab = unit / unsigned(s.chunks);
    const int chunk = int(unit - key_slab * unsigned(s.chunks));
    const int b = int(key_slab / unsigned(s.Hk)), hk = int(key_slab - unsigned(b) * unsigned(s.Hk)), share = s.H / s.Hk;
    const unsigned key_pitch = pitch_of<T>(s, s.Hk, s.dk), value_pitch = pitch_of<T>(s, s.H, s.dv);
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const int blocks = value_blocks(s.dv);
    const size_t state_bytes = emitted_bytes<T>(kCt, s.dv), token_bytes = emitted_bytes<T>(4, s.dv);

    Gates<T, false> gates;
    In fo[kVs];
    Mid fr[kVs], fe[kVs], fs[kOwn], fd[kOwn];
    auto request_gates = [&](int h) __attribute__((always_inline)) { gates.request(a.g, a.beta, s, b, h, chunk, lane); };
    auto request_slice = [&](int h, int v0) __attribute__((always_inline)) {
        const size_t value_unit = (size_t(b) * s.H + h) * s.chunks + unsigned(chunk);
        const Rsrc dor = chunk_rows(a.d_out, s, b, h, s.H, s.dv, chunk), er = whole(a.wrong + value_unit * token_bytes),
                   rr = whole(a.r + value_unit * token_bytes), Sr = whole(a.states + value_unit * state_bytes),
                   Dr = whole(a.adjoints + value_unit * state_bytes);
#pragma unroll
        for (int ks = 0; ks < kVs; ++ks) {
            const unsigned nowhere = 32 * (v0 + ks) + 8 * g < s.dv ? 0u : kNowhere;
            load_row(fo[ks], dor, row_offset<T>(value_pitch, token_at(s, 16 * w + r), v0 + ks, g, s.dv));
            fe[ks] = get_at<Mid>(er, nowhere, w * blocks + v0 + ks, lane);
            fr[ks] = get_at<Mid>(rr, nowhere, w * blocks + v0 + ks, lane);
        }
#pragma unroll
        for (int o = 0; o < kOwn; ++o) {
            const int block = 4 * o + w, ct = block / kVs, ks = block % kVs;
            const unsigned nowhere = block < kCt * kVs && 32 * (v0 + ks) + 8 * g < s.dv ? 0u : kNowhere;
            fs[o] = get_at<Mid>(Sr, nowhere, ct * blocks + v0 + ks, lane);
            fd[o] = get_at<Mid>(Dr, nowhere, ct * blocks + v0 + ks, lane);
        }
    };

    auto put_gates = [&]() __attribute__((always_inline)) {
        sum[w][lane] = gates.sum();
        bet[w][lane] = gates.strength();
    };

    f32x4 dq[kCt], dk[kCt];
    In fq[kKs], fk[kKs];  // the wave's rows
    {
        const Rsrc qr = chunk_rows(a.q, s, b, hk, s.Hk, s.dk, chunk), kr = chunk_rows(a.k, s, b, hk, s.Hk, s.dk, chunk);
        request_gates(hk * share);
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
            const unsigned at = row_offset<T>(key_pitch, token_at(s, 16 * w + r), ks, g, s.dk);
            load_row(fq[ks], qr, at);
            load_row(fk[ks], kr, at);
        }
        request_slice(hk * share, 0);
        requests_stay();
    }
    put_gates();
#pragma unroll
    for (int ks = 0; ks < kKs; ++ks) {
        key_put<T, DK>(keys, 16 * w + r, ks, g, fk[ks]);
        key_put<T, DK>(queries, 16 * w + r, ks, g, fq[ks]);
    }
#pragma unroll
    for (int ct = 0; ct < kCt; ++ct) dq[ct] = dk[ct] = zero;

    for (int h = hk * share; h < (hk + 1) * share; ++h) {
        // (addresses are formed from here on in every turn: formed once for all, they would be more than the registers hold)
        asm volatile("" : "+v"(lane));
        r = lane & 15, g = lane >> 4;
        if (h > hk * share) {
            request_gates(h);
            request_slice(h, 0);
            requests_stay();
            put_gates();
        }
        f32x4 x[4], y[4], read[kCt], erase[kCt], write[kCt];
#pragma unroll
        for (int n = 0; n < 4; ++n) x[n] = y[n] = zero;
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct) read[ct] = erase[ct] = write[ct] = zero;
        f32x4 inners = zero;  // <D, S>
        for (int v0 = 0; v0 < (kOne ? 1 : blocks); v0 += kVs) {
            if (!kOne && v0 > 0) {
                request_slice(h, v0);
                requests_stay();
            }
#pragma unroll
            for (int ks = 0; ks < kVs; ++ks) lds_put(wrong, w * kVs + ks, lane, fe[ks]);
#pragma unroll
            for (int o = 0; o < kOwn; ++o)
                if (kCt * kVs % 4 == 0 || 4 * o + w < kCt * kVs) {
                    inner(inners, fd[o], fs[o]);
                    lds_put(fS, 4 * o + w, lane, fs[o]);
                    lds_put(fD, 4 * o + w, lane, fd[o]);
                }
            __syncthreads();
#pragma unroll
            for (int ks = 0; ks < kVs; ++ks) {
#pragma unroll
                for (int n = 0; n < 4; ++n) {  // (the upper tiles too: the last wave has all four, and branches cost the others more)
                    const Mid f = lds_get<Mid>(wrong, n * kVs + ks, lane);
                    mma(x[n], fo[ks], f);
                    mma(y[n], fr[ks], f);
                }
#pragma unroll
                for (int ct = 0; ct < kCt; ++ct) {
                    if (ct % 2 == 0) requests_stay();  // (fragments from LDS: two tiles' ahead, not all)
                    const Mid f = lds_get<Mid>(fS, ct * kVs + ks, lane);
                    mma(read[ct], fo[ks], f);
                    mma(erase[ct], fr[ks], f);
                    mma(write[ct], fe[ks], lds_get<Mid>(fD, ct * kVs + ks, lane));
                }
            }
            __syncthreads();
        }
        const float ds = wave_prefix(of_lane<Mid>(inners, r, g));
        if (lane == 63) through[w] = ds;

        // X, Y and the pairs' part of dg
        {  // r_t . e_t stands on the diagonal of y
            const f32x4 d = w < 2 ? (w == 0 ? y[0] : y[1]) : (w == 2 ? y[2] : y[3]);
            const float db = (r & 2) ? ((r & 1) ? d[3] : d[2]) : ((r & 1) ? d[1] : d[0]);
            store_element<T>(chunk_rows(a.dbeta, s, b, h, s.H, 1, chunk), (r >> 2) == g ? unsigned(token_at(s, 16 * w + r)) * pitch_of<T>(s, s.H, 1) : kNowhere, db);
        }
        float carry[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
            key_get<T, DK>(fk[ks], keys, 16 * w + r, ks, g);
            key_get<T, DK>(fq[ks], queries, 16 * w + r, ks, g);
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            float column = 0.f;
            const int c = 16 * n + r;
            f32x4 qk = zero, kk = zero;
            requests_stay();
#pragma unroll
            for (int ks = 0; ks < kKs; ++ks) {
                In f;
                key_get<T, DK>(f, keys, 16 * n + r, ks, g);
                mma(qk, fq[ks], f);
                mma(kk, fk[ks], f);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = 16 * w + 4 * g + i;
                // (factors of 0 and 1 rather than branches)
                const float upto_t = c <= t ? 1.f : 0.f, before_t = c < t ? 1.f : 0.f;
                const float decay = decay_of(sum[w][t], sum[w][c], c <= t) * bet[w][c];
                const float xi = upto_t * decay * x[n][i], yi = before_t * -decay * bet[w][t] * y[n][i];
                X[t * kPitch + c] = xi;
                Y[t * kPitch + c] = yi;
                const float z = before_t * xi * qk[i] + yi * kk[i], upto = row_scan<0>(z);
                column += upto_t * (upto - z + carry[i]);  // pairs (t, i < c)
                carry[i] += moved<0x15f, 0xf>(upto);  // row_newbcast:15
            }
            column = rows_total(column);
            if (g == 0) pairs[w][c] = column;
        }
        f32x4 enter = zero, leave = zero;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 16 * w + 4 * g + i;
            const float c = exp2_of(sum[w][t]), d = exp2_of(sum[w][kC - 1] - sum[w][t]) * bet[w][t];
#pragma unroll
            for (int ct = 0; ct < kCt; ++ct) {
                read[ct][i] *= c;
                erase[ct][i] *= -c * bet[w][t];
                write[ct][i] *= d;
            }
        }
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct) {
            if (ct % 2 == 0) requests_stay();
            const f32x4 qe = four_tokens<DK>(In{}, queries, ct, w, r, g), ke = four_tokens<DK>(In{}, keys, ct, w, r, g);
            enter += qe * read[ct] + ke * erase[ct];
            leave += ke * write[ct];
            dq[ct] += read[ct];
            dk[ct] += erase[ct] + write[ct];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float en = row_scan<0>(enter[i]), le = row_scan<0>(leave[i]);  // sums in lane 15
            if (r == 15) enters[16 * w + 4 * g + i] = en, leaves[16 * w + 4 * g + i] = le;
        }
        __syncthreads();

#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const int t = 16 * w + r, c = 32 * ks + 8 * g;
            float x8[8], t8[8], y8[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x8[j] = X[t * kPitch + c + j];
                t8[j] = X[(c + j) * kPitch + t];
                y8[j] = Y[t * kPitch + c + j] + Y[(c + j) * kPitch + t];
            }
            Mid fx, ft, fy;
            make(fx, x8);
            make(ft, t8);
            make(fy, y8);
#pragma unroll
            for (int ct = 0; ct < kCt; ++ct) {
                if (ct % 2 == 0) requests_stay();
                In fkt, fqt;
                key_column<DK>(fkt, keys, ct, ks, r, g);
                key_column<DK>(fqt, queries, ct, ks, r, g);
                mma(dq[ct], fx, fkt);
                mma(dk[ct], ft, fqt);
                mma(dk[ct], fy, fkt);
            }
        }
        if (w == 0) {
            const float suffix = wave_prefix(enters[kC - 1 - lane]), before = moved<0x138, 0xf>(wave_prefix(leaves[lane]));  // wave_shr:1
            enters[kC - 1 - lane] = suffix;
            wave_fence();
            const float after = enters[lane];
            const float state = exp2_of(sum[w][kC - 1]) * ((through[0] + through[1]) + (through[2] + through[3]));
            const float dg = after + before + ((pairs[0][lane] + pairs[1][lane]) + (pairs[2][lane] + pairs[3][lane])) + state;
            store_element<T>(chunk_rows(a.dg, s, b, h, s.H, 1, chunk), unsigned(token_at(s, lane)) * pitch_of<T>(s, s.H, 1), dg);
        }
        __syncthreads();
    }
    // rows of dq and dk through the wave's own part of LDS: 16 bytes a lane
    constexpr int kRowPitch = DK + 8;
    T *rows = reinterpret_cast<T *>(shared) + 16 * w * kRowPitch;
    const Rsrc dqr = chunk_rows(a.dq, s, b, hk, s.Hk, s.dk, chunk), dkr = chunk_rows(a.dk, s, b, hk, s.Hk, s.dk, chunk);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) lds_element(rows + (4 * g + i) * kRowPitch + paired(ct, r), which == 0 ? dq[ct][i] : dk[ct][i]);
        wave_fence();
        constexpr int kPiece = 16 / int(sizeof(T)), kPieces = DK / kPiece;
#pragma unroll
        for (int o = 0; o < 16 * kPieces / 64; ++o) {
            const int item = 64 * o + lane, t = item / kPieces, c = (item % kPieces) * kPiece;
            const unsigned to = c < s.dk ? unsigned(token_at(s, 16 * w + t)) * key_pitch + unsigned(c) * unsigned(sizeof(T)) : kNowhere;
            __builtin_amdgcn_raw_buffer_store_b128(*reinterpret_cast<const u32x4 *>(rows + t * kRowPitch + c), which == 0 ? dqr : dkr, to, 0, 0);
        }
        wave_fence();
    }
}

template <typename T, int DK>
constexpr size_t gradient_lds()
{
    constexpr int vs = DK <= 64 ? 2 : 1;
    using In = typename operands<T, 2>::In;
    using Mid = typename operands<T, 2>::Mid;
    constexpr size_t states = 2 * DK / 16 * vs * frag_bytes<Mid>, tiles = 2 * kC * kPitch * 4;
    return (states > tiles ? states : tiles) + 4 * vs * frag_bytes<Mid> + 2 * KeyTile<T, DK>::bytes;
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
    at.adjoints = at.states + units * emitted_bytes<T>(DK / 16, s.dv);
    at.wrong = at.adjoints + units * emitted_bytes<T>(DK / 16, s.dv);
    at.r = at.wrong + units * emitted_bytes<T>(4, s.dv);
    at.bytes = at.r + units * emitted_bytes<T>(4, s.dv);
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
    unsigned char *S = ws + at.states, *D = ws + at.adjoints, *e = ws + at.wrong, *r = ws + at.r;
    const PrepareArgs<T> prepare = {s, q, k, g, beta, ws, ws + at.key_ws, at.states > kStreamedBytes};
    const ChainArgs<T> chain = {s, q, k, v, p.initial, nullptr, nullptr, S, e, ws, ws + at.key_ws};
    const AdjointArgs<T> adjoint = {s, k, d_out, p.d_final, static_cast<T *>(p.dv), p.d_initial, D, r, ws, ws + at.key_ws};
    const GradientArgs<T> gradient = {s, q, k, g, beta, d_out, static_cast<T *>(p.dq), static_cast<T *>(p.dk), static_cast<T *>(p.dg),
                                      static_cast<T *>(p.dbeta), S, D, e, r};
    const LaunchTimer timer(kKernelGatedDeltaBackward, stream);
    gd_prepare<T, DK, N, true><<<slabs * unsigned(s.chunks), 256, 0, stream>>>(prepare);
    gd_both_chains<T, DK, N><<<dim3((slabs + 7) / 8 * 8 * unsigned(s.dv / 16), 2), 128, 0, stream>>>(chain, adjoint);
    const unsigned key_units = unsigned(s.B) * unsigned(s.Hk) * unsigned(s.chunks);
    constexpr size_t lds = gradient_lds<T, DK>();
    if (s.dv <= (DK <= 64 ? 64 : 32))
        gd_gradients<T, DK, true><<<key_units, 256, lds, stream>>>(gradient);
    else
        gd_gradients<T, DK, false><<<key_units, 256, lds, stream>>>(gradient);
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
