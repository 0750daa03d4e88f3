// Gated delta rule, one token per sequence (S_t and o_t of gated_delta.hpp with the state in memory), one workgroup per (sequence, head).
//
// Bound by the state: dk x dv floats read and written once.  A thread owns four neighbouring columns of every kRows-th row, so a wave reads whole
// rows, and keeps them in registers from the read to the write.  Both products with the old state, k S and q S, are summed in one
// pass and joined once through LDS: with the written correction u, o = a q S + (q . k) u.
// 117 sequences of 16 heads with 128 x 128 states: 246 MB in 55 us from memory, 4.5 TB/s (a large copy reaches 4.8), 38 us where the Infinity Cache holds
// part of the pool from the call before.  One sequence: what a launch costs.
#include "vig_common.hpp"
#include "vig_kernels.hpp"
#include "vig_timing.hpp"

namespace vig {

namespace {

template <typename T>
struct StepArgs {
    int H, Hk, slots_n;
    unsigned first_block;  // of the launch
    const T *q, *k, *v, *g, *beta;
    float *state;
    const int *slots;
    T *out;
};

template <typename T, int DK, int DV>
__global__ __launch_bounds__(256) void gated_delta_step_kernel(StepArgs<T> a)
{
    constexpr int kQuads = DV / 4;                                       // column groups of a row
    constexpr int kThreads = DK * kQuads < 256 ? DK * kQuads : 256;      // small states need fewer
    constexpr int kRows = kThreads / kQuads, kMine = DK / kRows;         // rows of a pass, of a thread
    constexpr int kWaves = (kThreads + 63) / 64, kLane = kThreads < 64 ? kThreads : 64;
    const int tid = threadIdx.x, quad = tid % kQuads, r0 = tid / kQuads;
    const unsigned block = a.first_block + blockIdx.x, b = block / unsigned(a.H), h = block - b * unsigned(a.H), hk = h / unsigned(a.H / a.Hk);
    const size_t row = size_t(b) * a.H + h;
    T *out = a.out + row * DV;
    static_assert(kThreads >= DV, "");
    const int slot = a.slots ? a.slots[b] : int(b);
    if (slot < 0 || slot >= a.slots_n) {  // a padded row of the batch
        if (tid < DV) io<T>::store(out + tid, 0.f);
        return;
    }
    float *state = a.state + (size_t(slot) * a.H + h) * (DK * DV) + 4 * quad;
    const T *q = a.q + (size_t(b) * a.Hk + hk) * DK, *k = a.k + (size_t(b) * a.Hk + hk) * DK;
    f32x4 S[kMine], ks = {0.f, 0.f, 0.f, 0.f}, qs = ks, v;
    float kv[kMine], qv[kMine], qk = 0.f;
#pragma unroll
    for (int i = 0; i < kMine; ++i) S[i] = *reinterpret_cast<const f32x4 *>(state + size_t(r0 + i * kRows) * DV);
#pragma unroll
    for (int i = 0; i < kMine; ++i) kv[i] = io<T>::load(k + r0 + i * kRows), qv[i] = io<T>::load(q + r0 + i * kRows);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = io<T>::load(a.v + row * DV + 4 * quad + i);
    const float alpha = expf(io<T>::load(a.g + row)), beta = io<T>::load(a.beta + row);
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        S[i] *= alpha;
        ks += kv[i] * S[i];
        qs += qv[i] * S[i];
        qk = fmaf(qv[i], kv[i], qk);
    }
    // rows of the wave's other threads with the same columns
#pragma unroll
    for (int d = kQuads; d < kLane; d *= 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) ks[i] += __shfl_xor(ks[i], d), qs[i] += __shfl_xor(qs[i], d);
        qk += __shfl_xor(qk, d);
    }
    if constexpr (kWaves > 1) {
        __shared__ f32x4 part[kWaves][kQuads][2];
        __shared__ float part_qk[kWaves];
        const int w = tid >> 6;
        if ((tid & 63) < kQuads) part[w][quad][0] = ks, part[w][quad][1] = qs;
        if ((tid & 63) == 0) part_qk[w] = qk;
        __syncthreads();
        ks = qs = f32x4{0.f, 0.f, 0.f, 0.f};
        qk = 0.f;
#pragma unroll
        for (int o = 0; o < kWaves; ++o) ks += part[o][quad][0], qs += part[o][quad][1], qk += part_qk[o];
    }
    const f32x4 u = beta * (v - ks);
#pragma unroll
    for (int i = 0; i < kMine; ++i) *reinterpret_cast<f32x4 *>(state + size_t(r0 + i * kRows) * DV) = S[i] + kv[i] * u;
    if (r0 == 0) {
        const f32x4 o = qs + qk * u;
#pragma unroll
        for (int i = 0; i < 4; ++i) io<T>::store(out + 4 * quad + i, o[i]);
    }
}

template <typename T, int DK>
hipError_t launch_dv(int dv, int B, StepArgs<T> a, hipStream_t stream)
{
    const LaunchTimer timer(kKernelGatedDeltaStep, stream);
    const unsigned threads = unsigned(DK * dv / 4 < 256 ? DK * dv / 4 : 256);
    return in_launches(size_t(B) * a.H, threads, [&](unsigned first, unsigned grid) {
        a.first_block = first;
        switch (dv) {
            case 16: gated_delta_step_kernel<T, DK, 16><<<grid, threads, 0, stream>>>(a); break;
            case 32: gated_delta_step_kernel<T, DK, 32><<<grid, threads, 0, stream>>>(a); break;
            case 64: gated_delta_step_kernel<T, DK, 64><<<grid, threads, 0, stream>>>(a); break;
            default: gated_delta_step_kernel<T, DK, 128><<<grid, threads, 0, stream>>>(a); break;
        }
    });
}

template <typename T>
hipError_t launch(const void *q, const void *k, const void *v, const void *g, const void *beta, float *state, const int *slots, void *out, int B, int H,
                  int Hk, int slots_n, int dk, int dv, hipStream_t stream)
{
    const StepArgs<T> a = {H, Hk, slots_n, 0, static_cast<const T *>(q), static_cast<const T *>(k), static_cast<const T *>(v), static_cast<const T *>(g),
                           static_cast<const T *>(beta), state, slots, static_cast<T *>(out)};
    switch (dk) {
        case 16: return launch_dv<T, 16>(dv, B, a, stream);
        case 32: return launch_dv<T, 32>(dv, B, a, stream);
        case 64: return launch_dv<T, 64>(dv, B, a, stream);
        default: return launch_dv<T, 128>(dv, B, a, stream);
    }
}

}  // namespace

hipError_t gated_delta_step_launch(const void *q, const void *k, const void *v, const void *g, const void *beta, float *state, const int *slots,
                                   void *out, int B, int H, int Hk, int slots_n, int dk, int dv, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? launch<bf16_t>(q, k, v, g, beta, state, slots, out, B, H, Hk, slots_n, dk, dv, stream)
                   : launch<float>(q, k, v, g, beta, state, slots, out, B, H, Hk, slots_n, dk, dv, stream);
}

}  // namespace vig
