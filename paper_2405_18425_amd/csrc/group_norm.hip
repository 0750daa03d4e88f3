// Channels-last group norm with an activation, and its gradient.  x is [B, L, C]; group j of element b holds the channels jC/G .. and all L
// positions, N = L C / G values:
//     xn = (x - mean) rstd,  z = xn w + b,  y = act(z),   mean, rstd = (var + eps)^-1/2 per (b, j)
//     da = dy act'(z),  dw = sum da xn,  db = sum da  (over b and L),   dx = rstd (da w - m1 - xn m2),
//     m1 = mean of da w, m2 = mean of da w xn over the group.
//
// Bound by memory: x in, y out (x, dy in, dx out).  A group of few values is held in the registers of one workgroup: one launch, x is
// read once.  Otherwise two launches: partial sums of strips of rows over all channels, then the result, whose workgroups join the strips' sums of their
// element themselves (the same order in each, so results do not depend on the launch); the second reading of x comes from
// the Infinity Cache up to its size.  A thread owns 16 bytes of channels of every RG-th row, so a wave reads whole rows whatever the group width.
//
// Measured (bf16, inputs from memory, medians): 8 x 4096 x 384 in 6 groups 10.4 + 11.2 us, 25 MB in, 25 MB in again and 25 MB out: 2.4 and 4.5 TB/s;
// 16 x 3136 x 128 in 2 groups, gradient, 10.8 + 9.3 us; 64 x 49 x 1024 in 16 groups, one launch, 7.1 us for 13 MB, mostly the latency of one trip in, the sums and
// one trip out.  Far from the data's time: the gradient of few elements with many groups, whose workgroups each read all strips' sums at a stride
// (1 x 4096 x 2048 in 32 groups: 83 us for 50 MB; the forward, whose pairs lie by group, 37), and groups of few values, a workgroup of 256 threads each
// (16384 x 1 x 1024 in 16 groups: 269 us, gradient 165).
//
// Variances are sums of terms that are not negative, never a difference: runs of four rows, a strip's channels and threads and the strips are
// joined by the squared distances of their means from the mean of all, which a pass before has.  (From the first of those means, as one pass would have
// to, an outlier there is in all terms: with one channel of 8192 at 3.3 and the others 0, 1 / sqrt(var) was off by 1.4 %.)
#include "vig_common.hpp"
#include "vig_kernels.hpp"
#include "vig_timing.hpp"

namespace vig {

namespace {

constexpr int kThreads = 256;

template <typename T>
constexpr int kVec = 16 / int(sizeof(T));

template <typename T>
struct Values {
    float v[kVec<T>];
};
__device__ __forceinline__ void load(Values<bf16_t> &x, const bf16_t *p)
{
    const u32x4 u = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) x.v[2 * j] = bf16_lo_to_f32(u[j]), x.v[2 * j + 1] = bf16_hi_to_f32(u[j]);
}
__device__ __forceinline__ void load(Values<float> &x, const float *p)
{
    const f32x4 u = *reinterpret_cast<const f32x4 *>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) x.v[j] = u[j];
}
__device__ __forceinline__ void store(bf16_t *p, const Values<bf16_t> &x)
{
    u32x4 u;
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = pack2(x.v[2 * j], x.v[2 * j + 1]);
    *reinterpret_cast<u32x4 *>(p) = u;
}
__device__ __forceinline__ void store(float *p, const Values<float> &x) { *reinterpret_cast<f32x4 *>(p) = f32x4{x.v[0], x.v[1], x.v[2], x.v[3]}; }

// 1 / (1 + exp(-z)): the exponential overflows to infinity where the result is 0
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + fast_exp2(-1.4426950408889634f * z)); }
template <bool kSilu>
__device__ __forceinline__ float act(float z)
{
    return kSilu ? z * sigmoid(z) : z;
}
template <bool kSilu>
__device__ __forceinline__ float act_slope(float z)
{
    if (!kSilu) return 1.f;
    const float s = sigmoid(z);
    return s * fmaf(z, 1.f - s, 1.f);
}

// the sum over the 64 lanes, in each of them
__device__ __forceinline__ float wave_sum(float x)
{
    x = row_scan<0>(x);
    x += dpp_or_zero<0x142>(x);  // row_bcast:15
    x += dpp_or_zero<0x143>(x);  // row_bcast:31, the whole sum in lane 63
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

constexpr int kWorkgroups = 1024;  // of a launch over strips, four a compute unit; no element has more strips

struct Plan {
    int B, L, C, G, strips, rows;  // rows of a strip
    int vecs, row_groups;          // 16-byte pieces of a row; rows that a workgroup takes at a time
};

template <typename T>
struct NormArgs {
    Plan p;
    const T *x, *weight, *bias;  // weight and bias may be null
    T *out;
    float *stats;                // [B, G, 2] mean, rstd
    float eps;
    unsigned first_block;        // of the launch
    float2 *partial;             // [B][G][strips] mean, squared distances from it; of the gradient [B][strips][G], sums
    // gradient
    const float *in_stats;
    const T *d_out;
    T *d_weight, *d_bias;
    float2 *channel;             // [B][strips][C] sums of da, da xn
};

template <typename T>
__device__ __forceinline__ Values<T> vector_or(const T *p, int c, float value)
{
    Values<T> x;
    if (p)
        load(x, p + c);
    else
#pragma unroll
        for (int j = 0; j < kVec<T>; ++j) x.v[j] = value;
    return x;
}

// a group's pair for each of a thread's channels: one, where groups are whole pieces
template <typename T>
__device__ __forceinline__ void by_group(const float2 *pair, int c, int width, float (&x)[kVec<T>], float (&y)[kVec<T>])
{
    if (width % kVec<T> == 0) {
        const float2 v = pair[c / width];
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) x[e] = v.x, y[e] = v.y;
    } else {
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) {
            const float2 v = pair[(c + e) / width];
            x[e] = v.x;
            y[e] = v.y;
        }
    }
}

// a power of two of values, two by two
template <int N>
__device__ __forceinline__ float sum_of(const float (&x)[N])
{
    float s[N];
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = x[i];
#pragma unroll
    for (int n = N / 2; n > 0; n /= 2)
#pragma unroll
        for (int i = 0; i < n; ++i) s[i] += s[i + n];
    return s[0];
}

// ---- a group per workgroup -------------------------------------------------------------------------

template <typename T, int R /* pieces of a thread */, bool kSilu>
__global__ __launch_bounds__(kThreads) void norm_group_kernel(NormArgs<T> a)
{
    constexpr int V = kVec<T>, kWaves = kThreads / 64;
    __shared__ float part[2][kWaves];
    const Plan &p = a.p;
    const unsigned block = a.first_block + blockIdx.x, b = block / unsigned(p.G), j = block - b * unsigned(p.G);
    const int width = p.C / p.G, pieces = width / V, all = p.L * pieces;
    const size_t base = size_t(b) * p.L * p.C + size_t(j) * width;
    const int w = threadIdx.x >> 6;
    // Distances from the group's first value, then from their mean: of values that are next to each other they keep their bits, and of values that are
    // all the same nothing is left.  Where the first value is an outlier, their sums, joined two by two, are off by a rounding or two of it.
    const float first = io<T>::load(a.x + base);
    Values<T> x[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int at = int(threadIdx.x) + i * kThreads, row = at / pieces, c = (at - row * pieces) * V;
        if (at < all)
            load(x[i], a.x + base + size_t(row) * p.C + c);
        else
#pragma unroll
            for (int e = 0; e < V; ++e) x[i].v[e] = first;
    }
    float sums[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
        for (int e = 0; e < V; ++e) x[i].v[e] -= first;
        sums[i] = sum_of(x[i].v);
    }
    const float sum = wave_sum(sum_of(sums)), inv = 1.f / (float(p.L) * float(width));
    if ((threadIdx.x & 63) == 0) part[0][w] = sum;
    __syncthreads();
    const float mean = ((part[0][0] + part[0][1]) + (part[0][2] + part[0][3])) * inv;
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const bool there = int(threadIdx.x) + i * kThreads < all;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            x[i].v[e] -= mean;
            sq = there ? fmaf(x[i].v[e], x[i].v[e], sq) : sq;
        }
    }
    sq = wave_sum(sq);
    if ((threadIdx.x & 63) == 0) part[1][w] = sq;
    __syncthreads();
    const float var = ((part[1][0] + part[1][1]) + (part[1][2] + part[1][3])) * inv, rstd = 1.f / sqrtf(var + a.eps);
    if (threadIdx.x == 0) *reinterpret_cast<float2 *>(a.stats + 2 * size_t(block)) = make_float2(first + mean, rstd);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int at = int(threadIdx.x) + i * kThreads, row = at / pieces, c = (at - row * pieces) * V;
        if (at >= all) continue;
        const Values<T> wt = vector_or(a.weight, int(j) * width + c, 1.f), bi = vector_or(a.bias, int(j) * width + c, 0.f);
        Values<T> y;
#pragma unroll
        for (int e = 0; e < V; ++e) y.v[e] = act<kSilu>(fmaf(x[i].v[e], rstd * wt.v[e], bi.v[e]));
        store(a.out + base + size_t(row) * p.C + c, y);
    }
}

// ---- strips of rows --------------------------------------------------------------------------------

__device__ __forceinline__ int rows_at(const Plan &p, int strip, int &first)
{
    first = strip * p.rows;
    const int n = p.L - first;
    return n < p.rows ? n : p.rows;
}
__device__ __forceinline__ int rows_of_group(int rows, int group, int groups) { return group < rows ? (rows - group + groups - 1) / groups : 0; }

// Rows that a thread takes at a time for its channels' means and squared distances
constexpr int kRun = 4;

// Of n values with mean v.x and squared distances v.y from it: what they add to the squared distances from `mean`, which is next to the whole's
// mean, and to what it is off by.  (Off by a few roundings, `mean` adds their square to a variance: nothing.)
__device__ __forceinline__ void join(float2 v, float n, float mean, float &rest, float &sq)
{
    const float d = v.x - mean;
    rest = fmaf(n, d, rest);
    sq += fmaf(n * d, d, v.y);
}

// Mean and squared distances of every group over the rows of a strip
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_strip_kernel(NormArgs<T> a)
{
    constexpr int V = kVec<T>;
    extern __shared__ __align__(16) float2 entry[];  // [row_groups][C] mean, squared distances
    const Plan &p = a.p;
    const unsigned block = a.first_block + blockIdx.x, b = block / unsigned(p.strips), strip = block - b * unsigned(p.strips);
    int first;
    const int rows = rows_at(p, int(strip), first);
    const T *x = a.x + (size_t(b) * p.L + first) * p.C;
    const int rg = p.row_groups > 1 ? int(threadIdx.x) / p.vecs : 0;
    if (rg < p.row_groups)
        for (int vec = p.row_groups > 1 ? int(threadIdx.x) - rg * p.vecs : int(threadIdx.x); vec < p.vecs; vec += kThreads) {
            const int n = rows_of_group(rows, rg, p.row_groups);
            // Of distances from the first row: of a channel far from zero they keep their bits.  Runs of kRun rows; the first one, from the first row on, has
            // what is left (rows that it does not have are read as its last one, and count nothing).
            float mean[V], sq[V];
            Values<T> base, y[kRun];
            const T *q = x + size_t(rg) * p.C + vec * V;
            const size_t step = size_t(p.row_groups) * p.C;
            const int head = n > 0 ? (n - 1) % kRun + 1 : 0;
#pragma unroll
            for (int e = 0; e < V; ++e) mean[e] = sq[e] = base.v[e] = 0.f;
            if (n > 0) {
                load(base, q);
#pragma unroll
                for (int o = 1; o < kRun; ++o) load(y[o], q + (o < head ? o : head - 1) * step);
                const float inv = 1.f / float(head);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float sum = 0.f;
#pragma unroll
                    for (int o = 1; o < kRun; ++o) sum += y[o].v[e] = o < head ? y[o].v[e] - base.v[e] : 0.f;
                    mean[e] = sum * inv;
                    sq[e] = mean[e] * mean[e];
#pragma unroll
                    for (int o = 1; o < kRun; ++o) {
                        const float d = o < head ? y[o].v[e] - mean[e] : 0.f;
                        sq[e] = fmaf(d, d, sq[e]);
                    }
                }
            }
            for (int i = head; i < n; i += kRun) {
#pragma unroll
                for (int o = 0; o < kRun; ++o) load(y[o], q + (i + o) * step);
                const float share = float(kRun) / float(i + kRun), weight = float(i) * share;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float sum = 0.f, own = 0.f;
#pragma unroll
                    for (int o = 0; o < kRun; ++o) sum += y[o].v[e] -= base.v[e];
                    const float run = sum * (1.f / kRun), d = run - mean[e];
#pragma unroll
                    for (int o = 0; o < kRun; ++o) own = fmaf(y[o].v[e] - run, y[o].v[e] - run, own);
                    sq[e] += fmaf(weight * d, d, own);
                    mean[e] = fmaf(share, d, mean[e]);
                }
            }
#pragma unroll
            for (int e = 0; e < V; ++e) entry[rg * p.C + vec * V + e] = make_float2(base.v[e] + mean[e], sq[e]);
        }
    __syncthreads();
    const int lane = threadIdx.x & 63, width = p.C / p.G;
    const int least = rows / p.row_groups, more = rows - least * p.row_groups, there = least > 0 ? p.row_groups : more;  // (rows of a row group, see rows_of_group)
    for (int j = threadIdx.x >> 6; j < p.G; j += kThreads / 64) {
        const float2 *own = entry + j * width;
        const auto entries = [&](auto take) {
            for (int g = 0; g < there; ++g) {
                const float n = float(g < more ? least + 1 : least);
                for (int c = lane; c < width; c += 64) take(n, own[g * p.C + c]);
            }
        };
        const float inv = 1.f / (float(rows) * float(width)), first = own[0].x;
        float s = 0.f, rest = 0.f, sq = 0.f;
        entries([&](float n, float2 v) { s = fmaf(n, v.x - first, s); });
        const float mean = fmaf(wave_sum(s), inv, first);
        entries([&](float n, float2 v) { join(v, n, mean, rest, sq); });
        rest = wave_sum(rest);
        sq = wave_sum(sq);
        if (lane == 0) a.partial[(size_t(b) * p.G + j) * p.strips + strip] = make_float2(fmaf(rest, inv, mean), sq);
    }
}

// Mean and variance of a group from its strips' means and squared distances, in every lane.  The pairs are read once, all requests on their way together.
template <int kMine /* pairs of a lane */>
__device__ __forceinline__ float2 join_strips(const Plan &p, const float2 *part, int lane, int width)
{
    asm volatile("" : "+v"(lane));  // (what depends on the lane is formed here, not ahead of the loop over groups for every form of this)
    float2 v[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int at = 64 * i + lane;
        v[i] = part[at < p.strips ? at : 0];
    }
    const float inv = 1.f / (float(p.L) * float(width)), whole = float(p.rows) * float(width),
                last = float(p.L - (p.strips - 1) * p.rows) * float(width), first = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v[0].x)));
    const auto values = [&](int i) {
        const int left = p.strips - 1 - (64 * i + lane);
        return left > 0 ? whole : left == 0 ? last : 0.f;
    };
    float s = 0.f, rest = 0.f, sq = 0.f;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        if (64 * i + lane >= p.strips) v[i].y = 0.f;
        s = fmaf(values(i), v[i].x - first, s);
    }
    const float mean = fmaf(wave_sum(s), inv, first);
#pragma unroll
    for (int i = 0; i < kMine; ++i) join(v[i], values(i), mean, rest, sq);
    return make_float2(fmaf(wave_sum(rest), inv, mean), wave_sum(sq) * inv);
}

template <typename T, bool kSilu>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(NormArgs<T> a)
{
    constexpr int V = kVec<T>;
    extern __shared__ __align__(16) float2 stat[];  // [G] mean, rstd
    const Plan &p = a.p;
    const unsigned block = a.first_block + blockIdx.x, b = block / unsigned(p.strips), strip = block - b * unsigned(p.strips);
    const int lane = threadIdx.x & 63, width = p.C / p.G;
    for (int j = threadIdx.x >> 6; j < p.G; j += kThreads / 64) {  // the strips' sums of the element
        const float2 *part = a.partial + (size_t(b) * p.G + j) * p.strips;
        const float2 s = p.strips <= 64 ? join_strips<1>(p, part, lane, width) : p.strips <= 256 ? join_strips<4>(p, part, lane, width)
                                                                                              : join_strips<kWorkgroups / 64>(p, part, lane, width);
        const float mean = s.x, rstd = 1.f / sqrtf(s.y + a.eps);
        if (lane == 0) {
            stat[j] = make_float2(mean, rstd);
            if (strip == 0) *reinterpret_cast<float2 *>(a.stats + 2 * (size_t(b) * p.G + j)) = make_float2(mean, rstd);
        }
    }
    __syncthreads();
    int first;
    const int rows = rows_at(p, int(strip), first);
    const size_t at = (size_t(b) * p.L + first) * p.C;
    const int rg = p.row_groups > 1 ? int(threadIdx.x) / p.vecs : 0;
    if (rg >= p.row_groups) return;
    for (int vec = p.row_groups > 1 ? int(threadIdx.x) - rg * p.vecs : int(threadIdx.x); vec < p.vecs; vec += kThreads) {
        const int n = rows_of_group(rows, rg, p.row_groups);
        Values<T> scale = vector_or(a.weight, vec * V, 1.f), bi = vector_or(a.bias, vec * V, 0.f);
        float mean[V], rstd[V];
        by_group<T>(stat, vec * V, width, mean, rstd);
#pragma unroll
        for (int e = 0; e < V; ++e) scale.v[e] *= rstd[e];
        const size_t from = at + size_t(rg) * p.C + vec * V, step = size_t(p.row_groups) * p.C;
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
            Values<T> y;
            load(y, a.x + from + i * step);
#pragma unroll
            for (int e = 0; e < V; ++e) y.v[e] = act<kSilu>(fmaf(y.v[e] - mean[e], scale.v[e], bi.v[e]));
            store(a.out + from + i * step, y);
        }
    }
}

// ---- gradient --------------------------------------------------------------------------------------

template <typename T>
struct Channels {  // what a thread needs of its channels
    float mean[kVec<T>], rstd[kVec<T>], w[kVec<T>], b[kVec<T>];
};
template <typename T>
__device__ __forceinline__ Channels<T> channels_at(const NormArgs<T> &a, unsigned b, int c)
{
    const Values<T> w = vector_or(a.weight, c, 1.f), bi = vector_or(a.bias, c, 0.f);
    const int width = a.p.C / a.p.G;
    Channels<T> ch;
    const float2 *stats = reinterpret_cast<const float2 *>(a.in_stats) + size_t(b) * a.p.G;
    by_group<T>(stats, c, width, ch.mean, ch.rstd);
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) {
        ch.w[e] = w.v[e];
        ch.b[e] = bi.v[e];
    }
    return ch;
}

// Sums of da and da xn over the rows of a strip: by channel, and weighted by group
template <typename T, bool kSilu>
__global__ __launch_bounds__(kThreads) void norm_sums_kernel(NormArgs<T> a)
{
    constexpr int V = kVec<T>;
    extern __shared__ __align__(16) float2 entry[];  // [row_groups][C]
    const Plan &p = a.p;
    const unsigned block = a.first_block + blockIdx.x, b = block / unsigned(p.strips), strip = block - b * unsigned(p.strips);
    int first;
    const int rows = rows_at(p, int(strip), first);
    const size_t at = (size_t(b) * p.L + first) * p.C;
    const int rg = p.row_groups > 1 ? int(threadIdx.x) / p.vecs : 0;
    if (rg < p.row_groups)
        for (int vec = p.row_groups > 1 ? int(threadIdx.x) - rg * p.vecs : int(threadIdx.x); vec < p.vecs; vec += kThreads) {
            const int n = rows_of_group(rows, rg, p.row_groups);
            const Channels<T> ch = channels_at(a, b, vec * V);
            float s1[V], s2[V];
#pragma unroll
            for (int e = 0; e < V; ++e) s1[e] = s2[e] = 0.f;
            const size_t from = at + size_t(rg) * p.C + vec * V, step = size_t(p.row_groups) * p.C;
#pragma unroll 4
            for (int i = 0; i < n; ++i) {
                Values<T> x, d;
                load(x, a.x + from + i * step);
                load(d, a.d_out + from + i * step);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float xn = (x.v[e] - ch.mean[e]) * ch.rstd[e], da = d.v[e] * act_slope<kSilu>(fmaf(xn, ch.w[e], ch.b[e]));
                    s1[e] += da;
                    s2[e] = fmaf(da, xn, s2[e]);
                }
            }
#pragma unroll
            for (int e = 0; e < V; ++e) entry[rg * p.C + vec * V + e] = make_float2(s1[e], s2[e]);
        }
    __syncthreads();
    for (int c = threadIdx.x; c < p.C; c += kThreads) {
        float2 s = entry[c];
        for (int g = 1; g < p.row_groups; ++g) s.x += entry[g * p.C + c].x, s.y += entry[g * p.C + c].y;
        a.channel[size_t(block) * p.C + c] = s;
        const float w = a.weight ? io<T>::load(a.weight + c) : 1.f;
        entry[c] = make_float2(s.x * w, s.y * w);  // (a thread's own channel: no other reads it before the barrier)
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, width = p.C / p.G;
    for (int j = threadIdx.x >> 6; j < p.G; j += kThreads / 64) {
        float s1 = 0.f, s2 = 0.f;
        for (int c = lane; c < width; c += 64) s1 += entry[j * width + c].x, s2 += entry[j * width + c].y;
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        if (lane == 0) a.partial[size_t(block) * p.G + j] = make_float2(s1, s2);
    }
}

// The first workgroups join the strips' channel sums (kJoined channels each: few, for their chain of additions is what a launch of long strips
// waits for), the others write dx
constexpr int kJoined = 16;
template <typename T, bool kSilu>
__global__ __launch_bounds__(kThreads) void norm_grad_kernel(NormArgs<T> a, unsigned joins)
{
    constexpr int V = kVec<T>;
    extern __shared__ __align__(16) float2 stat[];  // [G] m1, m2; or [kThreads]
    const Plan &p = a.p;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const unsigned item = a.first_block + blockIdx.x;
    if (item < joins) {
        const int c = int(item) * kJoined + int(threadIdx.x) % kJoined, row = int(threadIdx.x) / kJoined;
        float s1 = 0.f, s2 = 0.f;
        if (c < p.C)
#pragma unroll 8
            for (int i = row; i < p.B * p.strips; i += kThreads / kJoined) {
                const float2 v = a.channel[size_t(i) * p.C + c];
                s1 += v.x;
                s2 += v.y;
            }
        stat[threadIdx.x] = make_float2(s1, s2);
        __syncthreads();
        if (threadIdx.x < kJoined && c < p.C) {
            s1 = s2 = 0.f;
#pragma unroll
            for (int i = 0; i < kThreads / kJoined; ++i) s1 += stat[i * kJoined + threadIdx.x].x, s2 += stat[i * kJoined + threadIdx.x].y;
            io<T>::store(a.d_bias + c, s1);
            io<T>::store(a.d_weight + c, s2);
        }
        return;
    }
    const unsigned block = item - joins, b = block / unsigned(p.strips), strip = block - b * unsigned(p.strips);
    const int width = p.C / p.G;
    for (int j = w; j < p.G; j += kThreads / 64) {
        const float2 *part = a.partial + size_t(b) * p.strips * p.G + j;
        float s1 = 0.f, s2 = 0.f;
        for (int i = lane; i < p.strips; i += 64) s1 += part[size_t(i) * p.G].x, s2 += part[size_t(i) * p.G].y;
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        const float inv = 1.f / (float(p.L) * float(width));
        if (lane == 0) stat[j] = make_float2(s1 * inv, s2 * inv);
    }
    __syncthreads();
    int first;
    const int rows = rows_at(p, int(strip), first);
    const size_t at = (size_t(b) * p.L + first) * p.C;
    const int rg = p.row_groups > 1 ? int(threadIdx.x) / p.vecs : 0;
    if (rg >= p.row_groups) return;
    for (int vec = p.row_groups > 1 ? int(threadIdx.x) - rg * p.vecs : int(threadIdx.x); vec < p.vecs; vec += kThreads) {
        const int n = rows_of_group(rows, rg, p.row_groups);
        const Channels<T> ch = channels_at(a, b, vec * V);
        float m1[V], m2[V];
        by_group<T>(stat, vec * V, width, m1, m2);
        const size_t from = at + size_t(rg) * p.C + vec * V, step = size_t(p.row_groups) * p.C;
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
            Values<T> x, d;
            load(x, a.x + from + i * step);
            load(d, a.d_out + from + i * step);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xn = (x.v[e] - ch.mean[e]) * ch.rstd[e], da = d.v[e] * act_slope<kSilu>(fmaf(xn, ch.w[e], ch.b[e]));
                d.v[e] = ch.rstd[e] * (fmaf(da, ch.w[e], -m1[e]) - xn * m2[e]);
            }
            store(a.out + from + i * step, d);
        }
    }
}

// ---- plans -----------------------------------------------------------------------------------------

Plan plan_of(int B, int L, int C, int G, int vec)
{
    Plan p = {B, L, C, G, 1, L, C / vec, 1};
    if (p.vecs < kThreads) p.row_groups = kThreads / p.vecs;
    // strips until the chip is full, of no fewer than four rows a thread
    const int most = (L + 4 * p.row_groups - 1) / (4 * p.row_groups), want = (kWorkgroups + B - 1) / B;
    p.strips = want < most ? want : most;
    p.rows = (L + p.strips - 1) / p.strips;
    p.strips = (L + p.rows - 1) / p.rows;
    return p;
}
Plan plan_of(int B, int L, int C, int G, bool is_bf16) { return plan_of(B, L, C, G, is_bf16 ? 8 : 4); }

constexpr int kMostPieces = 8;  // of a thread of norm_group_kernel

bool group_in_registers(const Plan &p, int vec)
{
    const int width = p.C / p.G;
    return width % vec == 0 && long(p.L) * (width / vec) <= long(kMostPieces) * kThreads;
}

template <typename T, bool kSilu>
hipError_t forward(NormArgs<T> a, hipStream_t stream)
{
    const Plan &p = a.p;
    const LaunchTimer timer(kKernelGroupNorm, stream);
    if (group_in_registers(p, kVec<T>)) {
        const int pieces = p.L * (p.C / p.G / kVec<T>), each = (pieces + kThreads - 1) / kThreads;
        return in_launches(size_t(p.B) * p.G, kThreads, [&](unsigned first, unsigned grid) {
            a.first_block = first;
            if (each <= 1)
                norm_group_kernel<T, 1, kSilu><<<grid, kThreads, 0, stream>>>(a);
            else if (each <= 2)
                norm_group_kernel<T, 2, kSilu><<<grid, kThreads, 0, stream>>>(a);
            else if (each <= 4)
                norm_group_kernel<T, 4, kSilu><<<grid, kThreads, 0, stream>>>(a);
            else
                norm_group_kernel<T, 8, kSilu><<<grid, kThreads, 0, stream>>>(a);
        });
    }
    const size_t blocks = size_t(p.B) * p.strips;
    const hipError_t e = in_launches(blocks, kThreads, [&](unsigned first, unsigned grid) {
        a.first_block = first;
        norm_strip_kernel<T><<<grid, kThreads, size_t(p.row_groups) * p.C * sizeof(float2), stream>>>(a);
    });
    if (e != hipSuccess) return e;
    return in_launches(blocks, kThreads, [&](unsigned first, unsigned grid) {
        a.first_block = first;
        norm_apply_kernel<T, kSilu><<<grid, kThreads, size_t(p.G) * sizeof(float2), stream>>>(a);
    });
}

template <typename T, bool kSilu>
hipError_t backward(NormArgs<T> a, hipStream_t stream)
{
    const Plan &p = a.p;
    const LaunchTimer timer(kKernelGroupNormBackward, stream);
    const size_t blocks = size_t(p.B) * p.strips;
    const unsigned joins = a.d_weight ? unsigned(p.C + kJoined - 1) / kJoined : 0;
    const size_t stat = size_t(p.G > 256 ? p.G : 256) * sizeof(float2);
    const hipError_t e = in_launches(blocks, kThreads, [&](unsigned first, unsigned grid) {
        a.first_block = first;
        norm_sums_kernel<T, kSilu><<<grid, kThreads, size_t(p.row_groups) * p.C * sizeof(float2), stream>>>(a);
    });
    if (e != hipSuccess) return e;
    return in_launches(blocks + joins, kThreads, [&](unsigned first, unsigned grid) {
        a.first_block = first;
        norm_grad_kernel<T, kSilu><<<grid, kThreads, stat, stream>>>(a, joins);
    });
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

template <typename T>
hipError_t forward_of(const void *x, const void *weight, const void *bias, void *out, float *stats, const Plan &p, float eps, bool silu, void *workspace,
                      hipStream_t stream)
{
    NormArgs<T> a = {};
    a.p = p;
    a.x = static_cast<const T *>(x);
    a.weight = static_cast<const T *>(weight);
    a.bias = static_cast<const T *>(bias);
    a.out = static_cast<T *>(out);
    a.stats = stats;
    a.eps = eps;
    a.partial = static_cast<float2 *>(workspace);
    return silu ? forward<T, true>(a, stream) : forward<T, false>(a, stream);
}

template <typename T>
hipError_t backward_of(const void *x, const void *weight, const void *bias, const float *stats, const void *d_out, void *dx, void *d_weight, void *d_bias,
                       const Plan &p, bool silu, void *workspace, hipStream_t stream)
{
    NormArgs<T> a = {};
    a.p = p;
    a.x = static_cast<const T *>(x);
    a.weight = static_cast<const T *>(weight);
    a.bias = static_cast<const T *>(bias);
    a.in_stats = stats;
    a.d_out = static_cast<const T *>(d_out);
    a.out = static_cast<T *>(dx);
    a.d_weight = static_cast<T *>(d_weight);
    a.d_bias = static_cast<T *>(d_bias);
    a.partial = static_cast<float2 *>(workspace);
    a.channel = a.partial + round256(size_t(p.B) * p.strips * p.G * sizeof(float2)) / sizeof(float2);
    return silu ? backward<T, true>(a, stream) : backward<T, false>(a, stream);
}

}  // namespace

size_t group_norm_workspace_bytes(int B, int L, int C, int groups, bool is_bf16)
{
    const Plan p = plan_of(B, L, C, groups, is_bf16);
    if (group_in_registers(p, is_bf16 ? 8 : 4)) return 0;
    return round256(size_t(B) * p.strips * groups * sizeof(float2));
}

size_t group_norm_bwd_workspace_bytes(int B, int L, int C, int groups, bool is_bf16)
{
    const Plan p = plan_of(B, L, C, groups, is_bf16);
    return round256(size_t(B) * p.strips * groups * sizeof(float2)) + round256(size_t(B) * p.strips * C * sizeof(float2));
}

hipError_t group_norm_launch(const void *x, const void *weight, const void *bias, void *out, float *stats, int B, int L, int C, int groups, float eps,
                             bool silu, bool is_bf16, void *workspace, hipStream_t stream)
{
    const Plan p = plan_of(B, L, C, groups, is_bf16);
    return is_bf16 ? forward_of<bf16_t>(x, weight, bias, out, stats, p, eps, silu, workspace, stream)
                   : forward_of<float>(x, weight, bias, out, stats, p, eps, silu, workspace, stream);
}

hipError_t group_norm_bwd_launch(const void *x, const void *weight, const void *bias, const float *stats, const void *d_out, void *dx, void *d_weight,
                                 void *d_bias, int B, int L, int C, int groups, bool silu, bool is_bf16, void *workspace, hipStream_t stream)
{
    const Plan p = plan_of(B, L, C, groups, is_bf16);
    return is_bf16 ? backward_of<bf16_t>(x, weight, bias, stats, d_out, dx, d_weight, d_bias, p, silu, workspace, stream)
                   : backward_of<float>(x, weight, bias, stats, d_out, dx, d_weight, d_bias, p, silu, workspace, stream);
}

}  // namespace vig
