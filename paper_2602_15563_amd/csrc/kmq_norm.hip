// The norms around a block, with its gate and the residual sum, in one pass over the row:
//
//     n_i = x_i * post_gain_i / sqrt( (1/H) sum_j x_j^2 + eps )       (or n = x)
//     s_i = residual_scale * residual_i + scale * g_i * n_i            g: 1, the gate, or its sigmoid
//     out_i = s_i,   normed_i = s_i * pre_gain_i / sqrt( (1/H) sum_j s_j^2 + eps )
//
// Computed in 64 bits, rounded to 32 and then to bf16: what comes out goes into a router, where scores next to each other decide, so
// a norm that is the definition's own makes the choice the definition's own.
//
// 4001 rows of 5120 take 41 us with all of it (164 MB at 4.0 TB/s; a copy of them 32): 64-bit conversions and products, some 40 clocks an element and lane, fill
// most of vector issue; without the first norm, gate and their gains 34 us, 4.8 TB/s.
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

// 1 / (1 + exp(-g)) of a gate: 2^(k + f) with |f| <= 1/2, the power series of 2^f to the eleventh power (6e-15 of it), the unit's reciprocal and
// two Newton steps.  (With the library's exponential and a division 16 rows of 7168 take 6.9 us, with this 6.3; 4001 of 4096 50 and 46.)
__device__ __forceinline__ double sigmoid(double g) {
    const double t = fmin(fmax(-g, -745.0), 709.0), k = rint(t * 1.4426950408889634), f = fma(t, 1.4426950408889634, -k);
    constexpr double c[] = {1.0, 0.6931471805599453, 0.24022650695910072, 0.05550410866482158, 0.009618129107628477, 0.0013333558146428443, 0.0001540353039338161, 1.5252733804059841e-05, 1.321548679014431e-06, 1.01780860092397e-07, 7.054911620801123e-09, 4.4455382718708116e-10};
    double p = c[11];
#pragma unroll
    for (int i = 10; i >= 0; --i) p = fma(p, f, c[i]);
    const double d = 1.0 + ldexp(p, static_cast<int>(k));
    double y = __builtin_amdgcn_rcp(d);
    y = fma(fma(-d, y, 1.0), y, y);
    y = fma(fma(-d, y, 1.0), y, y);
    return g != g ? g : g < -709.7 ? 0.0 : y;             // (behind that the exponential is an infinity)
}

// A workgroup a row, V times eight elements a thread; what is read is asked for at once, ahead of the first sum (but gains for V = 4: they
// would be spilled).
template <int V>
__global__ __launch_bounds__(1024) void block_norm_kernel(BlockNormArgs a) {
    __shared__ double part[2][16];
    const int pieces = static_cast<int>(a.width >> 3);
    const int64_t row = blockIdx.x;
    const double mean = 1.0 / static_cast<double>(a.width), eps = a.eps, residual_scale = a.residual_scale;
    const u32x4_t zeros = {0, 0, 0, 0};
    u32x4_t x[V], res[V], gate[V], post[V], pre[V];
    const auto read = [&](const uint16_t* p, int64_t at, bool live) { return live && p ? *reinterpret_cast<const u32x4_t*>(p + at) : zeros; };
    const auto piece = [&](int v) { return static_cast<int>(threadIdx.x) + v * static_cast<int>(blockDim.x); };
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = 8 * piece(v);
        const bool live = piece(v) < pieces;
        x[v] = read(a.x, row * a.x_stride + i, live);
        res[v] = read(a.residual, row * a.residual_stride + i, live);
        gate[v] = read(a.gate, row * a.gate_stride + i, live);
        if constexpr (V < 4) {
            post[v] = read(a.post_gain, i, live);
            pre[v] = read(a.pre_gain, i, live);
        }
    }
    double s[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[v][e] = kv_half(x[v][e / 2], e % 2);
    double r = 1.0;
    if (a.post_norm) {
        double sum = 0.0;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fma(s[v][e], s[v][e], sum);
        r = inverse_root(fma(sum_over_workgroup(sum, part[0]), mean, eps));
    }
    r *= a.scale;
    double sum = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[v][e] *= r;
        if (a.post_gain) {
            if constexpr (V == 4) post[v] = read(a.post_gain, 8 * piece(v), piece(v) < pieces);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[v][e] *= kv_half(post[v][e / 2], e % 2);
        }
        if (a.gate) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double g = kv_half(gate[v][e / 2], e % 2);
                s[v][e] *= a.sigmoid ? sigmoid(g) : g;
            }
        }
        if (a.residual) {
#pragma unroll
            for (int e = 0; e < 8; ++e) s[v][e] = fma(residual_scale, static_cast<double>(kv_half(res[v][e / 2], e % 2)), s[v][e]);
        }
        if (piece(v) >= pieces) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fma(s[v][e], s[v][e], sum);
        if (a.out) {
            u32x4_t y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = round2(s[v][2 * e], s[v][2 * e + 1]);
            *reinterpret_cast<u32x4_t*>(a.out + row * a.out_stride + 8 * piece(v)) = y;
        }
    }
    if (!a.normed) return;
    r = inverse_root(fma(sum_over_workgroup(sum, part[1]), mean, eps));
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (piece(v) >= pieces) continue;
        if constexpr (V == 4) pre[v] = read(a.pre_gain, 8 * piece(v), true);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[v][e] *= r;
            if (a.pre_gain) s[v][e] *= kv_half(pre[v][e / 2], e % 2);
        }
        u32x4_t y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = round2(s[v][2 * e], s[v][2 * e + 1]);
        *reinterpret_cast<u32x4_t*>(a.normed + row * a.normed_stride + 8 * piece(v)) = y;
    }
}

template <int V>
void start(const BlockNormArgs& a, hipStream_t s) {
    const int64_t pieces = a.width / 8;
    block_norm_kernel<V><<<dim3(static_cast<unsigned>(a.rows)), static_cast<unsigned>(((pieces + V - 1) / V + 63) / 64 * 64), 0, s>>>(a);
}

}  // namespace

// Pieces a thread, us: 4001 rows of 5120 with one / two / three 50 / 43 / 44, 2500 of 8192 43 / 39 / 46, 8192 of 1024 16.2 / 15.8 / 15.9; 16 rows of 7168 6.9 / 7.6 / 9.3.
// Not kept: two rows a workgroup, which read the gains once (4001 x 5120: 60 against 45), rows in turn with the gains in registers and
// the next row asked for ahead (90: 64-bit elements of two rows leave no registers).
hipError_t launch_block_norm(const BlockNormArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    const int64_t pieces = a.width / 8;
    if (pieces > 2048 || (a.rows >= 512 && pieces > 1024)) start<4>(a, s);
    else if (pieces > 1024 || (a.rows >= 512 && pieces >= 128)) start<2>(a, s);
    else start<1>(a, s);
    return hipGetLastError();
}

}  // namespace kmq
