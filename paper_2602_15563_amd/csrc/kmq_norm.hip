// The norms around a block, with its gate and the residual sum, in one pass over the row:
//
//     n_i = x_i * post_gain_i / sqrt( (1/H) sum_j x_j^2 + eps )       (or n = x)
//     s_i = residual_scale * residual_i + scale * g_i * n_i            g: 1, the gate, or its sigmoid
//     out_i = s_i,   normed_i = s_i * pre_gain_i / sqrt( (1/H) sum_j s_j^2 + eps )
//
// Computed in 64 bits, rounded to 32 and then to bf16: what comes out goes into a router, where scores next to each other decide, so
// a norm that is the definition's own makes the choice the definition's own.
#include "kmq_kv.h"

namespace kmq {

namespace {

// The sum over a workgroup's threads, in all of them; `part` has an entry a wave, used by this sum alone.
__device__ __forceinline__ double sum_over_workgroup(double v, double* part) {
    const int waves = static_cast<int>(blockDim.x) >> 6;
    v = sum_over<64>(v);
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < waves; ++w) v += part[w];
    return v;
}

__device__ __forceinline__ uint32_t round2(double a, double b) {
    float y[2] = {static_cast<float>(a), static_cast<float>(b)};
    asm("" : "+v"(y[0]));                                 // (else the compiler makes one rounding of the two, which are specified)
    asm("" : "+v"(y[1]));
    return kv_pack2(y[0], y[1]);
}

// A workgroup a row, V times eight elements a thread.
template <int V>
__global__ __launch_bounds__(1024) void block_norm_kernel(BlockNormArgs a) {
    __shared__ double part[2][16];
    const int pieces = static_cast<int>(a.width >> 3);
    const int64_t row = blockIdx.x;
    const double mean = 1.0 / static_cast<double>(a.width), eps = a.eps;
    u32x4_t x[V], res[V], gate[V];
    const u32x4_t ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u}, zeros = {0, 0, 0, 0};
    const auto read = [&](const uint16_t* p, int64_t stride, int i) { return *reinterpret_cast<const u32x4_t*>(p + row * stride + 8 * i); };
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = static_cast<int>(threadIdx.x) + v * static_cast<int>(blockDim.x);
        const bool live = i < pieces;
        x[v] = live ? read(a.x, a.x_stride, i) : zeros;
        res[v] = live && a.residual ? read(a.residual, a.residual_stride, i) : zeros;
        gate[v] = live && a.gate ? read(a.gate, a.gate_stride, i) : ones;
    }
    double r = 1.0;
    if (a.post_norm) {
        double sum = 0.0;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double t = kv_half(x[v][e / 2], e % 2);
                sum = fma(t, t, sum);
            }
        r = inverse_root(fma(sum_over_workgroup(sum, part[0]), mean, eps));
    }
    r *= a.scale;
    double s[V][8], sum = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = static_cast<int>(threadIdx.x) + v * static_cast<int>(blockDim.x);
        const u32x4_t gain = a.post_norm && a.post_gain && i < pieces ? *reinterpret_cast<const u32x4_t*>(a.post_gain + 8 * i) : ones;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            double n = kv_half(x[v][e / 2], e % 2) * r, g = kv_half(gate[v][e / 2], e % 2);
            if (a.sigmoid) g = 1.0 / (1.0 + exp(-g));
            n *= kv_half(gain[e / 2], e % 2);
            n *= g;
            if (a.residual) n = fma(static_cast<double>(a.residual_scale), static_cast<double>(kv_half(res[v][e / 2], e % 2)), n);
            s[v][e] = n;
            if (i < pieces) sum = fma(n, n, sum);
        }
        if (a.out && i < pieces) {
            u32x4_t y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = round2(s[v][2 * e], s[v][2 * e + 1]);
            *reinterpret_cast<u32x4_t*>(a.out + row * a.out_stride + 8 * i) = y;
        }
    }
    if (!a.normed) return;
    r = inverse_root(fma(sum_over_workgroup(sum, part[1]), mean, eps));
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = static_cast<int>(threadIdx.x) + v * static_cast<int>(blockDim.x);
        if (i >= pieces) continue;
        const u32x4_t gain = a.pre_gain ? *reinterpret_cast<const u32x4_t*>(a.pre_gain + 8 * i) : ones;
        u32x4_t y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = round2(s[v][2 * e] * r * kv_half(gain[e], 0), s[v][2 * e + 1] * r * kv_half(gain[e], 1));
        *reinterpret_cast<u32x4_t*>(a.normed + row * a.normed_stride + 8 * i) = y;
    }
}

}  // namespace

hipError_t launch_block_norm(const BlockNormArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    const int64_t pieces = a.width / 8;
    const int v = static_cast<int>((pieces + 1023) / 1024);
    const unsigned threads = static_cast<unsigned>(((pieces + v - 1) / v + 63) / 64 * 64);
    const dim3 grid(static_cast<unsigned>(a.rows));
    switch (v) {
        case 1: block_norm_kernel<1><<<grid, threads, 0, s>>>(a); break;
        case 2: block_norm_kernel<2><<<grid, threads, 0, s>>>(a); break;
        case 3: block_norm_kernel<3><<<grid, threads, 0, s>>>(a); break;
        default: block_norm_kernel<4><<<grid, threads, 0, s>>>(a); break;
    }
    return hipGetLastError();
}

}  // namespace kmq
