// Gated delta rule, forward: gd_prepare for the chunks' matrices, gd_states for the chain.
#include "gated_delta_chain.hpp"
#include "gated_delta_prepare.hpp"
#include "vig_kernels.hpp"
#include "vig_timing.hpp"

namespace vig {

namespace {

using namespace gd;

constexpr unsigned kComputeUnits = 256;

// Parts of a 32-bit operand: a returned state takes three, bf16 results two
template <typename T, int DK, int N>
size_t matrix_bytes(const Shape &s)
{
    const size_t units = size_t(s.B) * s.H * s.chunks, key_units = size_t(s.B) * s.Hk * s.chunks;
    return round256(units * ChunkWs<T, N, false>::bytes) + round256(key_units * KeyWs<T, DK, false>::bytes);
}

template <typename T, int DK, int N>
hipError_t launch(const Shape &s, const void *q, const void *k, const void *v, const void *g, const void *beta, const float *initial, void *out,
                  float *final_state, void *workspace, hipStream_t stream)
{
    const unsigned slabs = unsigned(s.B) * unsigned(s.H), units = slabs * unsigned(s.chunks);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    unsigned char *key_ws = ws + round256(size_t(units) * ChunkWs<T, N, false>::bytes);
    const PrepareArgs<T> p = {s, static_cast<const T *>(q), static_cast<const T *>(k), static_cast<const T *>(g), static_cast<const T *>(beta), ws, key_ws,
                               matrix_bytes<T, DK, N>(s) > kStreamedBytes};
    const ChainArgs<T> c = {s, p.q, p.k, static_cast<const T *>(v), initial, static_cast<T *>(out), final_state, nullptr, nullptr, ws, key_ws};
    const LaunchTimer timer(kKernelGatedDelta, stream);
    gd_prepare<T, DK, N, false><<<units, 256, 0, stream>>>(p);
    // 128 channels are two waves' while every workgroup has a compute unit to itself (2 x 16 heads of 8191 tokens, bf16: 340 -> 312 us; 2 x 4 of
    // 2048, fp32: 192 -> 150), and one wave's behind that (8 x 16 heads, 2048 tokens in bf16: 289 -> 282; 1024 in fp32: 330 -> 294)
    const unsigned blocks = (slabs + 7) / 8 * 8 * unsigned(s.dv / 16);
    if (DK == 128 && slabs * unsigned(s.dv / 16) <= kComputeUnits)
        gd_states<T, DK, N, DK == 128 ? 2 : 1><<<blocks, 192, 0, stream>>>(c);
    else
        gd_states<T, DK, N, 1><<<blocks, 128, 0, stream>>>(c);
    return hipGetLastError();
}

template <typename T, int DK, typename... A>
hipError_t launch_parts(bool states, const Shape &s, A... rest)
{
    if constexpr (sizeof(T) == 2)
        if (states) return launch<T, DK, 3>(s, rest...);
    return launch<T, DK, 2>(s, rest...);
}

template <typename T, typename... A>
hipError_t launch_width(bool states, const Shape &s, A... rest)
{
    if (s.dk <= 32) return launch_parts<T, 32>(states, s, rest...);
    if (s.dk <= 64) return launch_parts<T, 64>(states, s, rest...);
    return launch_parts<T, 128>(states, s, rest...);
}

}  // namespace

size_t gated_delta_workspace_bytes(int B, int H, int Hk, int L, int dk, int dv, bool is_bf16)
{
    const Shape s = {B, H, Hk, L, dk, dv, (L + kC - 1) / kC, false, false};
    const auto of = [&](auto t) {
        using T = decltype(t);
        return dk <= 32 ? matrix_bytes<T, 32, 3>(s) : dk <= 64 ? matrix_bytes<T, 64, 3>(s) : matrix_bytes<T, 128, 3>(s);
    };
    return is_bf16 ? of(bf16_t{}) : of(float{});
}

hipError_t gated_delta_launch(const void *q, const void *k, const void *v, const void *g, const void *beta, const float *initial, void *out,
                              float *final_state, int B, int H, int Hk, int L, int dk, int dv, bool is_bf16, bool token_major, bool reverse,
                              void *workspace, hipStream_t stream)
{
    const Shape s = {B, H, Hk, L, dk, dv, (L + kC - 1) / kC, token_major, reverse};
    const bool states = final_state != nullptr;
    if (is_bf16) return launch_width<bf16_t>(states, s, q, k, v, g, beta, initial, out, final_state, workspace, stream);
    return launch_width<float>(states, s, q, k, v, g, beta, initial, out, final_state, workspace, stream);
}

}  // namespace vig
