// The chain of a head's chunks, S -> S_out, for 16 value columns, one wave, and a second wave for their outputs.  Formulas: gated_delta.hpp.
//
// The chain's wave holds its columns of the state in accumulators (32-bit) and takes a chunk's matrices from the workspace as fragments, 16 bytes
// a lane, each requested for the next chunk as soon as its last product of this chunk has been issued.  The three products of a step
// follow each other in registers; only what the outputs need goes through LDS, with one barrier a chunk.  Columns of one head sit on one
// XCD (blockIdx % 8), whose L2 they read the fragments from.
//
// What bounds it (64 x 64, bf16): where every workgroup has a compute unit, its own instructions, 50 matrix and 225 vector ones a chunk in one wave, 1.1 us
// (8 x 6 heads of 4096 tokens: 70 us with inputs in the Infinity Cache, 66 without a request in the loop, 63 without the outputs' either; 85 us with inputs from
// memory).  With several workgroups on a compute unit, what
// comes through its first-level cache, 50 KB a chunk and 16 columns: 16 x 16 heads of 1024 tokens take 79 us, 35 without requests.  Two groups of columns
// in a wave take twice as long a step; two in a workgroup read the same lines at different times (115 us instead of 74).
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
    unsigned char *states, *wrong;        // gradient: S and e of every chunk as fragments, see Emitted
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

__device__ __forceinline__ f32x4 as_floats(const u32x4 &x) { return __builtin_bit_cast(f32x4, x); }

// A chunk's scalars: a lane requests 16 bytes of the kilobyte, the wave shares them through its own LDS when the chunk's turn comes (as
// registers of the lanes that use them they would be 37 for a whole step), and reads what it needs when it needs it.
constexpr int kScalarBytes = 1024;
__device__ __forceinline__ u32x4 request_scalars(Rsrc ws, int lane) { return load16(ws, 16u * unsigned(lane)); }
__device__ __forceinline__ void share_scalars(unsigned char *lds, const u32x4 &x, int lane)
{
    *reinterpret_cast<u32x4 *>(lds + 16 * lane) = x;
    wave_fence();
}
// of the tokens that accumulators of tile m stand for
enum Scalar { kC0 = 0, kWritten = 256 /* d . beta */, kRead = 512, kInverseBeta = 768 };
__device__ __forceinline__ f32x4 scalars(const unsigned char *lds, Scalar which, int m, int g)
{
    return *reinterpret_cast<const f32x4 *>(lds + which + 128 * (m >> 1) + 16 * (m & 1) + 32 * g);
}
__device__ __forceinline__ float whole_decay(const unsigned char *lds) { return *reinterpret_cast<const float *>(lds + 4 * (kC - 1)); }

// Rows of a state: element (channel, column) of [dk][dv] floats in the lanes that hold it; channels that the head does not have are nowhere
__device__ __forceinline__ unsigned state_offset(const Shape &s, int ct, int i, int g, int col)
{
    const int c = paired(ct, 4 * g + i);
    return c < s.dk ? 4u * (unsigned(c) * unsigned(s.dv) + unsigned(col)) : kNowhere;
}

// What the chain of a chunk leaves for its outputs, in LDS: the state as fragments (two parts) and e as it is
template <typename T, int DK>
struct HandOver {
    using Mid2 = typename operands<T, 2>::Mid;
    static constexpr int e = DK / 32 * int(frag_bytes<Mid2>);
    static constexpr int bytes = e + 4096;
};
template <typename Frag>
__device__ __forceinline__ void lds_put(unsigned char *lds, int block, int lane, const Frag &f)
{
    u32x4 w[planes<Frag>];
    __builtin_memcpy(w, &f, sizeof(f));
#pragma unroll
    for (int i = 0; i < planes<Frag>; ++i) *reinterpret_cast<u32x4 *>(lds + (block * planes<Frag> + i) * 1024 + 16 * lane) = w[i];
}
template <typename Frag>
__device__ __forceinline__ Frag lds_get(const unsigned char *lds, int block, int lane)
{
    u32x4 w[planes<Frag>];
#pragma unroll
    for (int i = 0; i < planes<Frag>; ++i) w[i] = *reinterpret_cast<const u32x4 *>(lds + (block * planes<Frag> + i) * 1024 + 16 * lane);
    Frag f;
    __builtin_memcpy(&f, w, sizeof(f));
    return f;
}

// a wave's 16 columns of one head
struct Columns {
    unsigned slab;
    int b, h, hk, col, lane, r, g;
};
__device__ __forceinline__ bool columns_of(const Shape &s, Columns &c)
{
    unsigned part;
    if (!chain_unit(blockIdx.x, unsigned(s.B) * unsigned(s.H), unsigned(s.dv) / 16, c.slab, part)) return false;
    c.b = int(c.slab / unsigned(s.H));
    c.h = int(c.slab - unsigned(c.b) * unsigned(s.H));
    c.hk = c.h / (s.H / s.Hk);
    c.lane = threadIdx.x & 63;
    c.r = c.lane & 15;
    c.g = c.lane >> 4;
    c.col = 16 * int(part) + c.r;
    return true;
}

// The 16 columns of a chunk's 64 rows of values: requested as rows, 16 bytes a lane, and read back from LDS by column, tokens 32p + 8g .. + 7 of
// column r.  (One element a lane would be 16 requests instead of 2, each as long in the address unit as one of 16 bytes.)
template <typename T>
struct Strip {
    static constexpr int pieces = 16 * int(sizeof(T)) / 16, loads = pieces;  // 16-byte pieces of a row; a load takes 64 / pieces rows
    static constexpr int pitch = sizeof(T) == 2 ? 16 : 17, bytes = kC * pitch * int(sizeof(T));
    u32x4 w[loads];
};
template <typename T>
__device__ __forceinline__ unsigned strip_offset(const Shape &s, unsigned pitch, int part, int lane, int load)
{
    constexpr int kPieces = Strip<T>::pieces;
    const int t = load * (64 / kPieces) + lane / kPieces, piece = lane % kPieces;
    return unsigned(token_at(s, t)) * pitch + unsigned(16 * part) * unsigned(sizeof(T)) + 16u * unsigned(piece);
}
template <typename T>
__device__ __forceinline__ void strip_put(unsigned char *lds, const Strip<T> &x, int lane)
{
    constexpr int kPieces = Strip<T>::pieces;
#pragma unroll
    for (int l = 0; l < Strip<T>::loads; ++l) {
        const int t = l * (64 / kPieces) + lane / kPieces, piece = lane % kPieces;
        if constexpr (sizeof(T) == 2)
            *reinterpret_cast<u32x4 *>(lds + t * 32 + 16 * piece) = x.w[l];
        else  // rows of 17 floats: columns are read without bank conflicts
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<unsigned *>(lds + 4 * (t * 17 + 4 * piece + i)) = x.w[l][i];
    }
}
// tokens 32 p + 8g .. + 7 of column r
__device__ __forceinline__ void strip_column(bf16_t (&x)[8], const unsigned char *lds, int p, int r, int g)
{
    const uint16_t *q = reinterpret_cast<const uint16_t *>(lds) + (32 * p + 8 * g + (r >> 2)) * 16 + 4 * (r & 3);
    const bf16x8 v = join(lds_read_tr(q), lds_read_tr(q + 4 * 16));
    __builtin_memcpy(x, &v, sizeof(v));
}
__device__ __forceinline__ void strip_column(float (&x)[8], const unsigned char *lds, int p, int r, int g)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = *reinterpret_cast<const float *>(lds + 4 * ((32 * p + 8 * g + j) * 17 + r));
}

// What the chains of the gradient leave: a state (DK rows) or 64 tokens' rows, 16 columns a wave, first in LDS as [column][row] tiles of floats, which a
// second wave takes to the workspace as fragments of two parts: rows by 16 in tiles, columns along the products.  By non-temporal stores: read by the
// next launch only, they leave the L2 to the fragments that the columns of a head share (chains of 8 x 6 heads of 4096 tokens 185 -> 173 us, 64 x 6 of 196
// 54.5 -> 48, inputs in the Infinity Cache).
template <int kRows>
struct Tile {
    static constexpr int pitch = kRows + 4, bytes = 16 * pitch * 4;
};
template <int kRows>
__device__ __forceinline__ void tile_put(unsigned char *lds, int tile, int r, int g, const f32x4 &x)  // rows paired(tile, 4g) .. + 3 of column r
{
    *reinterpret_cast<f32x4 *>(lds + 4 * (r * Tile<kRows>::pitch + paired(tile, 4 * g))) = x;
}
inline __host__ __device__ int value_blocks(int dv) { return (dv + 31) / 32; }
template <typename T>
constexpr size_t row_block_bytes = frag_bytes<typename operands<T, 2>::Mid>;
// bytes of `tiles` tiles of 16 rows
template <typename T>
__host__ __device__ __forceinline__ size_t emitted_bytes(int tiles, int dv)
{
    return size_t(tiles) * value_blocks(dv) * row_block_bytes<T>;
}
// row -> its tile and its place in it
struct Place {
    int tile, r;
};
__device__ __forceinline__ Place natural(int row) { return {row >> 4, row & 15}; }
__device__ __forceinline__ Place unpaired(int row) { return {2 * (row >> 5) + ((row >> 2) & 1), 4 * ((row >> 3) & 3) + (row & 3)}; }

// eight columns of a row as a fragment's lane (of a head whose last block has 16 columns, the other half is not written: who reads it leaves it out)
template <typename Mid2>
__device__ __forceinline__ void emit(Rsrc to, Place at, int part, int group, int dv, const float (&x)[8])
{
    Mid2 f;
    make(f, x);
    u32x4 w[planes<Mid2>];
    __builtin_memcpy(w, &f, sizeof(f));
    const unsigned block = unsigned(at.tile * value_blocks(dv) + (part >> 1)) * unsigned(frag_bytes<Mid2>);
    const unsigned off = block + 16u * unsigned(at.r + 16 * (2 * (part & 1) + group));
#pragma unroll
    for (int p = 0; p < planes<Mid2>; ++p) __builtin_amdgcn_raw_buffer_store_b128(w[p], to, off + 1024u * unsigned(p), 0, kStream);
}
template <int kRows>
__device__ __forceinline__ void tile_row(float (&x)[8], const unsigned char *lds, int row, int group)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = *reinterpret_cast<const float *>(lds + 4 * ((8 * group + j) * Tile<kRows>::pitch + row));
}

// kWaves waves share the chain of 16 columns, each with its channels of the state: one exchange a chunk, of the sums over channels; e is formed by each
template <typename T, int DK, int N, bool kBwd, int kWaves>
__device__ __forceinline__ void states(const ChainArgs<T> &a, const Columns &at, int wave, unsigned char *scal /* the wave's: scalars, then a strip */,
                                       unsigned char *lds /* two HandOvers, or two state and two token tiles */, unsigned char *sums /* of two chunks */)
{
    using In = typename operands<T, N>::In;
    using Mid = typename operands<T, N>::Mid;
    using Ws = ChunkWs<T, N, kBwd>;
    using Kw = KeyWs<T, DK, kBwd>;
    using Hand = HandOver<T, DK>;
    constexpr int kKs = DK / 32 / kWaves, kCt = DK / 16 / kWaves;
    const int ks0 = wave * kKs, ct0 = wave * kCt;
    const Shape &s = a.s;
    const int lane = at.lane, r = at.r, g = at.g, col = at.col;
    const unsigned slab = at.slab;
    const unsigned char *ws_all = a.ws + size_t(slab) * s.chunks * Ws::bytes;
    const unsigned char *kw_all = a.key_ws + (size_t(at.b) * s.Hk + at.hk) * s.chunks * Kw::bytes;
    const size_t state_size = size_t(s.dk) * s.dv;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

    // offsets of a lane's rows of keys, and of its pieces of values
    const unsigned key_pitch = pitch_of<T>(s, s.Hk, s.dk);
    unsigned key_at[4], value_at[Strip<T>::loads];
#pragma unroll
    for (int m = 0; m < 4; ++m) key_at[m] = row_offset<T>(key_pitch, token_at(s, paired(m, r)), ks0, g, s.dk);
#pragma unroll
    for (int l = 0; l < Strip<T>::loads; ++l) value_at[l] = strip_offset<T>(s, pitch_of<T>(s, s.H, s.dv), col >> 4, lane, l);

    f32x4 S[kCt];
#pragma unroll
    for (int ct = 0; ct < kCt; ++ct) S[ct] = zero;
    if (a.initial) {
        const Rsrc from0 = slab_resource(a.initial + slab * state_size, unsigned(state_size * 4));
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) S[ct][i] = load4(from0, state_offset(s, ct0 + ct, i, g, col));
    }

    const int first = chunk_at(s, 0), move = s.reverse ? -1 : 1;
    Walk kr = walk_rows(a.k, s, at.b, at.hk, s.Hk, s.dk, first, move), vr = walk_rows(a.v, s, at.b, at.h, s.H, s.dv, first, move),
         ws = walk_blocks(ws_all, Ws::bytes, first, move), kw = walk_blocks(kw_all, Kw::bytes, first, move);
    In fk[4][kKs], fkt[kCt][2];
    Mid ft[kTriBlocks];
    Strip<T> v;
    u32x4 raw;
    auto load_keys = [&]() __attribute__((always_inline)) {
        const Rsrc from0 = kr.here();
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
            for (int m = 0; m < 4; ++m) load_row(fk[m][ks], from0, key_at[m] + 32u * unsigned(ks * sizeof(T)));
    };
    auto load_first = [&]() __attribute__((always_inline)) {
        raw = request_scalars(ws.here(), lane);
        const Rsrc from0 = vr.here();
#pragma unroll
        for (int l = 0; l < Strip<T>::loads; ++l) v.w[l] = load16(from0, value_at[l]);
    };
    auto load_inverse = [&]() __attribute__((always_inline)) {
        const Rsrc from0 = ws.here();
#pragma unroll
        for (int i = 0; i < kTriBlocks; ++i) ft[i] = get<Mid>(from0, Ws::inverse, i, lane);
    };
    auto load_transposed = [&]() __attribute__((always_inline)) {
        const Rsrc from0 = kw.here();
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int ct = 0; ct < kCt; ++ct) fkt[ct][ks] = get<In>(from0, 0, 2 * (ct0 + ct) + ks, lane);
    };
    // (in the order of the loop: its waits count the requests behind the one they are for, and hold for the way into the loop as well)
    load_first();
    requests_stay();
    load_keys();
    requests_stay();
    load_inverse();
    requests_stay();
    load_transposed();
    requests_stay();

    for (int step = 0; step < s.chunks; ++step) {
        if (step + 1 < s.chunks) kr.next(), vr.next(), ws.next(), kw.next();  // what is requested from here on
        unsigned char *hand = lds + (step & 1) * (kBwd ? Tile<DK>::bytes + Tile<kC>::bytes : Hand::bytes);
        if constexpr (kBwd) {
            __syncthreads();
#pragma unroll
            for (int ct = 0; ct < kCt; ++ct) tile_put<DK>(hand, ct0 + ct, r, g, S[ct]);
        }
        strip_put(scal + kScalarBytes, v, lane);
        share_scalars(scal, raw, lane);
        requests_stay();
        load_first();
        requests_stay();
        Mid fs[kKs];
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
            fs[ks] = from<Mid>(S[2 * ks], S[2 * ks + 1]);
            if constexpr (!kBwd) lds_put(hand, ks0 + ks, lane, first_parts<N, 2>(fs[ks]));
        }
        f32x4 e[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) e[m] = zero;
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks)
            mma_tiles(e, 0, 4, [&](int m) -> const In & { return fk[m][ks]; }, fs[ks]);
        requests_stay();
        load_keys();
        requests_stay();
        if constexpr (kWaves == 2) {
            unsigned char *mine = sums + 4096 * (2 * (step & 1) + wave), *other = sums + 4096 * (2 * (step & 1) + 1 - wave);
#pragma unroll
            for (int m = 0; m < 4; ++m) *reinterpret_cast<f32x4 *>(mine + 1024 * m + 16 * lane) = e[m];
            __syncthreads();
#pragma unroll
            for (int m = 0; m < 4; ++m) e[m] += *reinterpret_cast<const f32x4 *>(other + 1024 * m + 16 * lane);
        }
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            T x[8];
            strip_column(x, scal + kScalarBytes, p, r, g);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const f32x4 c = scalars(scal, kC0, 2 * p + j, g);
#pragma unroll
                for (int i = 0; i < 4; ++i) e[2 * p + j][i] = fmaf(-c[i], e[2 * p + j][i], value(x[4 * j + i]));
            }
        }
        const Mid fe[2] = {from<Mid>(e[0], e[1]), from<Mid>(e[2], e[3])};
#pragma unroll
        for (int m = 0; m < 4; ++m) e[m] = zero;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
            mma_tiles(e, 2 * ks, 4, [&](int m) -> const Mid & { return ft[lower_block(m, ks)]; }, fe[ks]);
        requests_stay();
        load_inverse();
        requests_stay();
        const float whole = whole_decay(scal);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            if (wave > 0)
                ;
            else if constexpr (kBwd)
                tile_put<kC>(hand + Tile<DK>::bytes, m, r, g, e[m]);
            else
                *reinterpret_cast<f32x4 *>(hand + Hand::e + 1024 * m + 16 * lane) = e[m];
            e[m] *= scalars(scal, kWritten, m, g);
        }
        const Mid fd[2] = {from<Mid>(e[0], e[1]), from<Mid>(e[2], e[3])};
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct) S[ct] *= whole;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
            mma_tiles(S, 0, kCt, [&](int ct) -> const In & { return fkt[ct][ks]; }, fd[ks]);
        requests_stay();
        load_transposed();
        requests_stay();
        if constexpr (!kBwd) __syncthreads();
    }
    if constexpr (kBwd) __syncthreads();
    if (!kBwd && a.final_state) {
        const Rsrc to = slab_resource(a.final_state + slab * state_size, unsigned(state_size * 4));
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) store4(to, state_offset(s, ct0 + ct, i, g, col), S[ct][i]);
    }
}

// S and e of the gradient's chain to the workspace, one chunk behind it
template <typename T, int DK>
__device__ __forceinline__ void emit_states(const ChainArgs<T> &a, const Columns &at, const unsigned char *lds)
{
    using Mid2 = typename operands<T, 2>::Mid;
    const Shape &s = a.s;
    const int part = at.col >> 4;
    const size_t state_bytes = emitted_bytes<T>(DK / 16, s.dv), token_bytes = emitted_bytes<T>(4, s.dv);
    const int first = chunk_at(s, 0), move = s.reverse ? -1 : 1;
    const size_t units = size_t(at.slab) * s.chunks;
    Walk ws = walk_blocks(a.states + units * state_bytes, state_bytes, first, move), we = walk_blocks(a.wrong + units * token_bytes, token_bytes, first, move);
    for (int step = 0; step <= s.chunks; ++step) {
        __syncthreads();
        if (step == 0) continue;
        const unsigned char *hand = lds + ((step - 1) & 1) * (Tile<DK>::bytes + Tile<kC>::bytes);
        const Rsrc to = ws.here(), te = we.here();
        ws.next();
        we.next();
        float x[8];
#pragma unroll
        for (int i = 0; i < DK / 32; ++i) {
            const int item = 64 * i + at.lane;
            tile_row<DK>(x, hand, item >> 1, item & 1);
            emit<Mid2>(to, unpaired(item >> 1), part, item & 1, s.dv, x);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int item = 64 * i + at.lane;
            tile_row<kC>(x, hand + Tile<DK>::bytes, item >> 1, item & 1);
            emit<Mid2>(te, natural(item >> 1), part, item & 1, s.dv, x);
        }
    }
}

// The outputs of a wave's columns, one chunk behind the chain
template <typename T, int DK, int N, int kWaves>
__device__ __forceinline__ void outputs(const ChainArgs<T> &a, const Columns &at, unsigned char *own /* the wave's: scalars, then a tile */, const unsigned char *lds)
{
    using In = typename operands<T, N>::In;
    using Mid2 = typename operands<T, 2>::Mid;
    using Ws = ChunkWs<T, N, false>;
    using Hand = HandOver<T, DK>;
    constexpr int kKs = DK / 32;
    const Shape &s = a.s;
    const int lane = at.lane, r = at.r, g = at.g;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const unsigned key_pitch = pitch_of<T>(s, s.Hk, s.dk), value_pitch = pitch_of<T>(s, s.H, s.dv);
    unsigned key_at[4], out_at[2];
#pragma unroll
    for (int m = 0; m < 4; ++m) key_at[m] = row_offset<T>(key_pitch, token_at(s, paired(m, r)), 0, g, s.dk);
#pragma unroll
    for (int i = 0; i < 2; ++i)  // the rows that a lane writes, eight columns each
        out_at[i] = unsigned(token_at(s, 32 * i + (lane >> 1))) * value_pitch + unsigned((at.col & ~15) + 8 * (lane & 1)) * unsigned(sizeof(T));

    const int first = chunk_at(s, 0), move = s.reverse ? -1 : 1;
    Walk qr = walk_rows(a.q, s, at.b, at.hk, s.Hk, s.dk, first, move), to = walk_rows(static_cast<const T *>(a.out), s, at.b, at.h, s.H, s.dv, first, move),
         ws = walk_blocks(a.ws + size_t(at.slab) * s.chunks * Ws::bytes, Ws::bytes, first, move);
    In fq[4][kKs];
    Mid2 fp[kTriBlocks];
    u32x4 raw;
    auto load_queries = [&]() __attribute__((always_inline)) {
        const Rsrc from0 = qr.here();
        raw = request_scalars(ws.here(), lane);
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
            for (int m = 0; m < 4; ++m) load_row(fq[m][ks], from0, key_at[m] + 32u * unsigned(ks * sizeof(T)));
    };
    auto load_scores = [&]() __attribute__((always_inline)) {
        const Rsrc from0 = ws.here();
#pragma unroll
        for (int i = 0; i < kTriBlocks; ++i) fp[i] = get<Mid2>(from0, Ws::scores, i, lane);
    };
    load_queries();
    requests_stay();
    load_scores();
    requests_stay();
    if (kWaves == 2) __syncthreads();
    for (int step = 0; step < s.chunks; ++step) {
        const Rsrc out = to.here();
        to.next();
        if (step + 1 < s.chunks) qr.next(), ws.next();
        const unsigned char *hand = lds + (step & 1) * Hand::bytes;
        share_scalars(own, raw, lane);
        __syncthreads();  // the chain has left this chunk's state and e; it writes the other half until the next one
        f32x4 o[4], e[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            o[m] = zero;
            e[m] = *reinterpret_cast<const f32x4 *>(hand + Hand::e + 1024 * m + 16 * lane);
        }
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
            const Mid2 fs = lds_get<Mid2>(hand, ks, lane);
            mma_tiles(o, 0, 4, [&](int m) -> const In & { return fq[m][ks]; }, fs);
        }
        requests_stay();
        load_queries();
        requests_stay();
        if (kWaves == 2 && step + 1 < s.chunks) __syncthreads();  // (the chain's waves exchange the next chunk's sums)
        const Mid2 fe[2] = {from<Mid2>(e[0], e[1]), from<Mid2>(e[2], e[3])};
#pragma unroll
        for (int m = 0; m < 4; ++m) o[m] *= scalars(own, kC0, m, g);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
            mma_tiles(o, 2 * ks, 4, [&](int m) -> const Mid2 & { return fp[lower_block(m, ks)]; }, fe[ks]);
        requests_stay();
        load_scores();
        requests_stay();
#pragma unroll
        for (int m = 0; m < 4; ++m) tile_put<kC>(own + kScalarBytes, m, r, g, o[m]);
        wave_fence();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float x[8];
            tile_row<kC>(x, own + kScalarBytes, 32 * i + (lane >> 1), lane & 1);
            store_row(out, out_at[i], x, T{});
        }
    }
}

// Waves on a SIMD: two where their registers fit
template <typename T, int DK, int kWaves>
constexpr int chain_waves = DK / kWaves * int(sizeof(T)) <= 128 ? 2 : 1;

// The waves of a chain, and one for the outputs, a chunk behind
template <typename T, int DK, int N, int kWaves>
__global__ __launch_bounds__(64 * (kWaves + 1)) __attribute__((amdgpu_waves_per_eu(chain_waves<T, DK, kWaves>, chain_waves<T, DK, kWaves>))) void gd_states(ChainArgs<T> a)
{
    __shared__ __align__(16) unsigned char lds[2 * HandOver<T, DK>::bytes], scal[kWaves][kScalarBytes + Strip<T>::bytes], own[kScalarBytes + Tile<kC>::bytes],
        sums[kWaves == 2 ? 4 * 4096 : 16];
    Columns at;
    if (!columns_of(a.s, at)) return;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6));
    if (wave < kWaves)
        states<T, DK, N, false, kWaves>(a, at, wave, scal[wave], lds, sums);
    else
        outputs<T, DK, N, kWaves>(a, at, own, lds);
}

}  // namespace gd
}  // namespace vig
