// The router of a mixture of experts: products with the experts' rows, scores, choice of the experts and their weights.
//
//     l_e = sum_k X_k W_ek,   s = softmax(l) or sigmoid(l),   c = s + bias
//     the top_k largest c (of the best groups, where there are groups), ties to the lowest index;  weight s_e [/ sum] * scale
//
// In 64 bits, sums and scores: the choice is a comparison, and with them it is the definition's own.  Products are
// v_mfma_f64_16x16x4_f64: lane (n, q) holds column q of row n of both operands, and in D tokens q, q + 4, q + 8, q + 12 of expert n.
// As the four columns of a step may be any, a lane's eight consecutive bf16 are the operands of eight steps.  The row
// length is cut into slices; a workgroup multiplies 16 experts with up to 64 tokens over a slice, its waves take chunks of 64
// columns in turn, and what comes out goes to the workspace.  A second kernel, a wave a token, adds the slices in their order and chooses.
//
// One token, 128 experts of 4096: 3.4 + 4.3 us, both chains of memory round trips (reading slices one by one took the second kernel 8.8); 16
// tokens, 256 experts of 7168 in groups 4.6 + 7.9, of which the products' own time is about 1 and the choice's twelve rounds of a maximum over the wave
// half; 128 tokens, 64 experts of 2048 6.5 + 4.1: at four tiles a workgroup these are 64 workgroups, a quarter of the units, and of a wave's 5.7 us its 64 matrix
// instructions of 64 clocks are 1.7 and waiting for memory 46 %.  Prompts: the 64-bit matrix instructions; 4001 rows, 128 experts of 4096 89 + 9 us, a unit's
// busy for 54 of the 89 (7 us for the bytes).
#include "kmq_kv.h"

namespace kmq {

namespace {

typedef __attribute__((ext_vector_type(4))) double f64x4_t;

constexpr int kRouteWaves = 4, kRouteChunk = 64;          // columns a wave takes at a time

template <int TILES>
__global__ __launch_bounds__(kRouteWaves * kWave) void route_product_kernel(RouteArgs a, int slices) {
    __shared__ double part[kRouteWaves][TILES * 256];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    const int first_row = static_cast<int>(blockIdx.z) * (16 * TILES);
    const int expert = static_cast<int>(blockIdx.x) * 16 + n;
    const uint16_t* w = a.router + static_cast<int64_t>(expert < a.experts ? expert : a.experts - 1) * a.width;
    const uint16_t* x[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const int row = first_row + 16 * t + n;
        x[t] = a.x + static_cast<int64_t>(row < a.rows ? row : a.rows - 1) * a.x_stride;
    }
    f64x4_t acc[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) acc[t] = f64x4_t{0.0, 0.0, 0.0, 0.0};
    for (int64_t at = (static_cast<int64_t>(blockIdx.y) * kRouteWaves + wave) * kRouteChunk; at < a.width;
         at += static_cast<int64_t>(slices) * (kRouteWaves * kRouteChunk)) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int64_t k = at + 32 * half + 8 * q;
            const bool live = k < a.width;                // (the width is a multiple of 8)
            const u32x4_t none = {0, 0, 0, 0}, wv = live ? *reinterpret_cast<const u32x4_t*>(w + k) : none;
            u32x4_t xv[TILES];
#pragma unroll
            for (int t = 0; t < TILES; ++t) xv[t] = live ? *reinterpret_cast<const u32x4_t*>(x[t] + k) : none;
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int t = 0; t < TILES; ++t)
                    acc[t] = __builtin_amdgcn_mfma_f64_16x16x4f64(kv_half(xv[t][e / 2], e % 2), kv_half(wv[e / 2], e % 2), acc[t], 0, 0, 0);
        }
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) part[wave][t * 256 + (q + 4 * r) * 16 + n] = acc[t][r];
    __syncthreads();
    double* out = static_cast<double*>(a.workspace) + static_cast<int64_t>(blockIdx.y) * a.rows * a.experts;
    for (int o = threadIdx.x; o < TILES * 256; o += kRouteWaves * kWave) {
        const int row = first_row + o / 16, e = static_cast<int>(blockIdx.x) * 16 + o % 16;
        double s = part[0][o];
#pragma unroll
        for (int i = 1; i < kRouteWaves; ++i) s += part[i][o];
        if (row < a.rows && e < a.experts) out[static_cast<int64_t>(row) * a.experts + e] = s;
    }
}

__device__ __forceinline__ uint32_t max_over_wave(uint32_t v) {
    const auto other = [](uint32_t x, auto ctrl) { return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), decltype(ctrl)::value, 0xF, 0xF, true)); };
    v = max(v, other(v, std::integral_constant<int, 0xB1>{}));          // quad_perm [1,0,3,2]
    v = max(v, other(v, std::integral_constant<int, 0x4E>{}));          // quad_perm [2,3,0,1]
    v = max(v, other(v, std::integral_constant<int, 0x141>{}));         // row_half_mirror
    v = max(v, other(v, std::integral_constant<int, 0x140>{}));         // row_mirror
    u32x2_t r = across_rows<false>(v);
    r = across_rows<true>(max(r[0], r[1]));
    return max(r[0], r[1]);
}
__device__ __forceinline__ uint64_t max_over_wave(uint64_t v) {
    const uint32_t hi = max_over_wave(static_cast<uint32_t>(v >> 32));
    return static_cast<uint64_t>(hi) << 32 | max_over_wave(static_cast<uint32_t>(v >> 32) == hi ? static_cast<uint32_t>(v) : 0u);
}

// A number that orders as the value does; a NaN comes behind all of them, and 0 is left for what may not be chosen.
__device__ __forceinline__ uint64_t order_of(double v) {
    if (v != v) return 1;
    const uint64_t u = __builtin_bit_cast(uint64_t, v + 0.0);
    return u >> 63 ? ~u : u | (uint64_t(1) << 63);
}
// The value that such a number stands for (not of a NaN or of 0).
__device__ __forceinline__ double value_of(uint64_t order) { return __builtin_bit_cast(double, order >> 63 ? order & ~(uint64_t(1) << 63) : ~order); }
// The lowest lane that holds the largest of the wave's numbers.
__device__ __forceinline__ int lane_of_largest(uint64_t v) { return __ffsll(__ballot(v == max_over_wave(v))) - 1; }

// A wave a token; lane l holds experts l * PER .. l * PER + PER - 1.
template <int PER>
__global__ __launch_bounds__(kWave) void route_choose_kernel(RouteArgs a, int slices) {
    constexpr int kAtOnce = PER <= 2 ? 16 : PER <= 4 ? 8 : 2;
    __shared__ double choice[kWave * PER];
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    const double* logits = static_cast<const double*>(a.workspace) + row * a.experts;
    const int64_t slice = static_cast<int64_t>(a.rows) * a.experts;
    double s[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) s[i] = 0.0;
    for (int k0 = 0; k0 < slices; k0 += kAtOnce) {        // (several slices at once: a memory round trip each would be most of the call)
        double v[kAtOnce][PER];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = lane * PER + i;
                v[k][i] = k0 + k < slices && e < a.experts ? logits[(k0 + k) * slice + e] : 0.0;
            }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
            for (int i = 0; i < PER; ++i) s[i] += v[k][i];
    }
    if (a.sigmoid) {
#pragma unroll
        for (int i = 0; i < PER; ++i) s[i] = 1.0 / (1.0 + exp(-s[i]));
    } else {
        uint64_t largest = 0;                             // (a NaN is the least of them)
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (lane * PER + i < a.experts) largest = max(largest, order_of(s[i]));
        largest = max_over_wave(largest);
        const double most = largest == 1 ? __builtin_nan("") : value_of(largest);
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            s[i] = exp(s[i] - most);
            if (lane * PER + i < a.experts) sum += s[i];
        }
        sum = sum_over<64>(sum);
#pragma unroll
        for (int i = 0; i < PER; ++i) s[i] /= sum;
    }
    uint64_t order[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = lane * PER + i;
        const double c = s[i] + (a.bias && e < a.experts ? static_cast<double>(a.bias[e]) : 0.0);
        order[i] = e < a.experts ? order_of(c) : 0;
        choice[e] = c != c ? -__builtin_inf() : c;
    }
    if (a.groups > 1) {
        __syncthreads();
        const int size = a.experts / a.groups;
        uint64_t mine = 0;
        if (lane < a.groups) {
            double best = -__builtin_inf(), next = -__builtin_inf();
#pragma unroll 8
            for (int i = 0; i < size; ++i) {
                const double c = choice[lane * size + i];
                next = fmax(next, fmin(best, c));
                best = fmax(best, c);
            }
            mine = order_of(size > 1 ? best + next : best);
        }
        uint64_t kept = 0;
        for (int g = 0; g < a.top_groups; ++g) {
            const int at = lane_of_largest(mine);
            kept |= uint64_t(1) << at;
            if (lane == at) mine = 0;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = lane * PER + i;
            if (e < a.experts && !(kept >> (e / size) & 1)) order[i] = 0;
        }
    }
    int id = 0;
    double weight = 0.0;
    for (int j = 0; j < a.top_k; ++j) {
        uint64_t best = 0;
        int at = 0;
        double score = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (order[i] > best) { best = order[i]; at = i; score = s[i]; }
        const int from = lane_of_largest(best);
        const int e = from * PER + __builtin_amdgcn_readlane(at, from);
        const uint64_t bits = __builtin_bit_cast(uint64_t, score);
        score = __builtin_bit_cast(double, static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(bits >> 32), from))) << 32 |
                                               static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(bits), from)));
        if (lane == j) { id = e; weight = score; }
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (lane * PER + i == e) order[i] = 0;
    }
    if (a.normalise) {
        const double sum = sum_over<64>(weight);
        weight = sum == 0.0 ? 0.0 : weight / sum;
    }
    if (lane < a.top_k) {
        a.ids[row * a.top_k + lane] = id;
        a.gates[row * a.top_k + lane] = static_cast<float>(weight * static_cast<double>(a.scale));
    }
}

}  // namespace

static int route_tiles(int64_t rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }

// Slices of the row length: workgroups for every compute unit, and at least one chunk for each of their waves.
int route_slices(int64_t rows, int64_t experts, int64_t width) {
    const int64_t blocks = (experts + 15) / 16 * ((rows + 16 * route_tiles(rows) - 1) / (16 * route_tiles(rows)));
    const int64_t most = (width + kRouteWaves * kRouteChunk - 1) / (kRouteWaves * kRouteChunk), want = (256 + blocks - 1) / blocks;
    return static_cast<int>(want < most ? want : most);
}

hipError_t launch_route(const RouteArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    const int slices = route_slices(a.rows, a.experts, a.width), tiles = route_tiles(a.rows);
    const dim3 grid(static_cast<unsigned>((a.experts + 15) / 16), static_cast<unsigned>(slices), static_cast<unsigned>((a.rows + 16 * tiles - 1) / (16 * tiles)));
    switch (tiles) {
        case 1: route_product_kernel<1><<<grid, kRouteWaves * kWave, 0, s>>>(a, slices); break;
        case 2: route_product_kernel<2><<<grid, kRouteWaves * kWave, 0, s>>>(a, slices); break;
        default: route_product_kernel<4><<<grid, kRouteWaves * kWave, 0, s>>>(a, slices); break;
    }
    const dim3 rows(static_cast<unsigned>(a.rows));
    if (a.experts <= kWave) route_choose_kernel<1><<<rows, kWave, 0, s>>>(a, slices);
    else if (a.experts <= 2 * kWave) route_choose_kernel<2><<<rows, kWave, 0, s>>>(a, slices);
    else if (a.experts <= 4 * kWave) route_choose_kernel<4><<<rows, kWave, 0, s>>>(a, slices);
    else if (a.experts <= 8 * kWave) route_choose_kernel<8><<<rows, kWave, 0, s>>>(a, slices);
    else route_choose_kernel<16><<<rows, kWave, 0, s>>>(a, slices);
    return hipGetLastError();
}

}  // namespace kmq
