// Rows of heads between the QKV product and the attention: RMSNorm of every query and key head, the rotation by
// position, and the quantised write of keys and values into the 4-bit cache, in one pass over the row.
//
//     n_i = x_i * gain_i / sqrt( (1/D) sum_j x_j^2 + eps )
//     split pairs (i, i + R/2), i < R/2; interleaved pairs (2i, 2i + 1); a_i = position * inv_freq_i
//     y_left = n_left cos a_i - n_right sin a_i,   y_right = n_right cos a_i + n_left sin a_i
//     cache:  scale = max |y| over 64 elements,  index = number of boundaries b_j with y > b_j * scale
//
// All of it is computed in 64 bits, rounded to 32 and then to bf16: a far position times a frequency needs them, and the
// index of a key is decided by a comparison, so that with them it is the definition's own and the oracle's.
// (The vector units multiply and add 64-bit floats at the rate of 32-bit ones.)
#include "kmq_kv.h"

namespace kmq {

constexpr int kHeadThreads = 256;
constexpr int kMaxRotaryPairs = 256;

// The boundary between two centroids, in 32 bits.
__device__ __forceinline__ double kv_boundary(const uint16_t* codebook, int i) {
    return static_cast<double>((bf16_to_f32(codebook[i]) + bf16_to_f32(codebook[i + 1])) * 0.5f);
}

// Index of x (bf16): boundaries that lie below it once they are scaled.  A boundary of at most 24 bits times a scale of 8
// is exact in 64 bits.  Four comparisons: the boundaries ascend.
__device__ __forceinline__ uint32_t kv_index(const double* boundary, double scale, double x) {
    uint32_t i = 0;
#pragma unroll
    for (int half = 8; half > 0; half >>= 1) i += x > boundary[i + half - 1] * scale ? half : 0;
    return i;
}

// LANES lanes hold a head, 8 elements each; a head never crosses a wave.
template <int LANES>
__global__ void __launch_bounds__(kHeadThreads) heads_kernel(HeadsArgs a, KvCacheArgs c, KvBatchArgs b, bool cached, int heads_per_group) {
    __shared__ double turn[2][kMaxRotaryPairs];
    __shared__ double boundary[2][kKvCentroids - 1];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x;
    const KvRow at = cached ? kv_find_row(b, row) : KvRow{0, 0};
    if (at.seq < 0) return;                               // (the same for all waves of the workgroup)
    if (a.rotary_dim) {
        const double pos = a.positions ? static_cast<double>(a.positions[row]) : static_cast<double>(at.pos);
        for (int i = tid; i < a.rotary_dim / 2; i += kHeadThreads) sincos(pos * static_cast<double>(a.inv_freq[i]), &turn[1][i], &turn[0][i]);
    }
    if (cached && tid < 2 * (kKvCentroids - 1)) {
        const int kv = tid / (kKvCentroids - 1), i = tid % (kKvCentroids - 1);
        boundary[kv][i] = kv_boundary(c.codebooks + kv * kKvCentroids, i);
    }
    __syncthreads();

    const int sub = tid % LANES, d0 = sub * 8;
    const int D = a.head_dim, half = a.rotary_dim / 2;
    const int total = a.q_heads + a.k_heads + a.v_heads;
    const int first = blockIdx.y * heads_per_group;
    const int last = first + heads_per_group < total ? first + heads_per_group : total;
    for (int base = first; base < last; base += kHeadThreads / LANES) {
        const int h = base + tid / LANES;
        const bool live = h < last && d0 < D;
        const int kind = h < a.q_heads ? 0 : h < a.q_heads + a.k_heads ? 1 : 2;
        const int hh = h - (kind == 0 ? 0 : kind == 1 ? a.q_heads : a.q_heads + a.k_heads);
        const uint16_t* src = kind == 0 ? a.q + row * a.q_stride : kind == 1 ? a.k + row * a.k_stride : a.v + row * a.v_stride;
        src += static_cast<int64_t>(hh) * D;
        const bool turned = live && kind < 2 && d0 < a.rotary_dim;
        const int other = a.interleaved ? d0 : d0 < half ? d0 + half : d0 - half;
        u32x4_t own = {0, 0, 0, 0}, far = {0, 0, 0, 0};
        if (live) own = *reinterpret_cast<const u32x4_t*>(src + d0);
        if (turned && !a.interleaved) far = *reinterpret_cast<const u32x4_t*>(src + other);

        if (kind < 2 && (a.norm || a.rotary_dim)) {
            double x[8], r = 1.0;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = bf16_to_f32(own[e / 2] >> (e % 2 * 16) & 0xFFFFu);
            if (a.norm) {
                double ss = 0.0;
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fma(x[e], x[e], ss);
#pragma unroll
                for (int m = 1; m < LANES; m <<= 1) ss += __shfl_xor(ss, m);
                r = 1.0 / sqrt(ss / D + static_cast<double>(a.eps));
            }
            const uint16_t* gain = !a.norm ? nullptr : kind == 0 ? a.q_gain : a.k_gain;
            u32x4_t gown = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u}, gfar = gown;
            if (gain && live) gown = *reinterpret_cast<const u32x4_t*>(gain + d0);
            if (gain && turned && !a.interleaved) gfar = *reinterpret_cast<const u32x4_t*>(gain + other);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= r * static_cast<double>(bf16_to_f32(gown[e / 2] >> (e % 2 * 16) & 0xFFFFu));
            if (turned) {
                if (a.interleaved) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const double co = turn[0][(d0 + e) / 2], si = turn[1][(d0 + e) / 2], l = x[e], t = x[e + 1];
                        x[e] = l * co - t * si;
                        x[e + 1] = t * co + l * si;
                    }
                } else {
                    const int i0 = d0 < half ? d0 : d0 - half;
                    const double sign = d0 < half ? -1.0 : 1.0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const double f = static_cast<double>(bf16_to_f32(far[e / 2] >> (e % 2 * 16) & 0xFFFFu)) *
                                         (r * static_cast<double>(bf16_to_f32(gfar[e / 2] >> (e % 2 * 16) & 0xFFFFu)));
                        x[e] = x[e] * turn[0][i0 + e] + sign * (f * turn[1][i0 + e]);
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 8; e += 2)
                own[e / 2] = f32_to_bf16(static_cast<float>(x[e])) | static_cast<uint32_t>(f32_to_bf16(static_cast<float>(x[e + 1]))) << 16;
        }

        if (kind == 0 || (kind == 1 && a.k_out)) {
            uint16_t* dst = kind == 0 ? a.q_out + row * a.q_out_stride : a.k_out + row * a.k_out_stride;
            if (live) *reinterpret_cast<u32x4_t*>(dst + static_cast<int64_t>(hh) * D + d0) = own;
            continue;
        }
        // keys and values of the cache: 8 lanes hold a block of 64 elements (D is a multiple of it here)
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t m = own[e / 2] >> (e % 2 * 16) & 0x7FFFu;
            top = m > top ? m : top;
        }
#pragma unroll
        for (int m = 1; m < 8; m <<= 1) {
            const uint32_t o = __shfl_xor(top, m);
            top = o > top ? o : top;
        }
        const double scale = top ? static_cast<double>(bf16_to_f32(top)) : 1.0;
        uint32_t word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            word |= kv_index(boundary[kind - 1], scale, bf16_to_f32(own[e / 2] >> (e % 2 * 16) & 0xFFFFu)) << (4 * e);
        const uint32_t pair = __shfl_xor(word, 2);        // the elements 16 further on, or back
        uint8_t* tile = live ? kv_tile(c, b, D, at, hh) : nullptr;
        if (!tile) continue;
        const int t = static_cast<int>(at.pos % kKvTile);
        if (kind == 1) {
            *reinterpret_cast<uint32_t*>(tile + kv_k_dword(D, t, d0)) = word;
        } else {
            const bool upper = d0 & 16;                   // this lane stores bytes 4..7 of the pair's eight
            const uint32_t lo = (upper ? pair >> 16 : word), hi = (upper ? word >> 16 : pair);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                tile[kv_v_byte(D, t, (d0 & ~16) + (upper ? 4 : 0) + e)] = static_cast<uint8_t>((lo >> (4 * e) & 15u) | (hi >> (4 * e) & 15u) << 4);
        }
        if (sub % 8 == 0) *reinterpret_cast<uint16_t*>(tile + kv_scale(D, t, kind - 1, d0)) = static_cast<uint16_t>(top);
    }
}

// Rows of the cache as bf16: one rounding of centroid * scale; zeros where the page table has no page.
__global__ void __launch_bounds__(kHeadThreads) kv_read_kernel(KvCacheArgs c, KvBatchArgs b, uint16_t* k, int64_t k_stride, uint16_t* v, int64_t v_stride) {
    __shared__ float centroid[2 * kKvCentroids];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, D = c.head_dim;
    if (tid < 2 * kKvCentroids) centroid[tid] = bf16_to_f32(c.codebooks[tid]);
    const KvRow at = kv_find_row(b, row);
    if (at.seq < 0) return;
    __syncthreads();
    const int per_head = D / 8, t = static_cast<int>(((at.pos % kKvTile) + kKvTile) % kKvTile);
    for (int i = tid; i < 2 * c.kv_heads * per_head; i += kHeadThreads) {
        const int kv = i / (c.kv_heads * per_head), rest = i % (c.kv_heads * per_head), h = rest / per_head, d0 = rest % per_head * 8;
        const uint8_t* tile = kv_tile(c, b, D, at, h);
        u32x4_t out = {0, 0, 0, 0};
        if (tile) {
            uint32_t word = 0;
            if (kv == 0) {
                word = *reinterpret_cast<const uint32_t*>(tile + kv_k_dword(D, t, d0));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    word |= (static_cast<uint32_t>(tile[kv_v_byte(D, t, (d0 & ~16) + e)]) >> (d0 & 16 ? 4 : 0) & 15u) << (4 * e);
            }
            const float scale = bf16_to_f32(*reinterpret_cast<const uint16_t*>(tile + kv_scale(D, t, kv, d0)));
#pragma unroll
            for (int e = 0; e < 8; e += 2)
                out[e / 2] = f32_to_bf16(centroid[kv * kKvCentroids + (word >> (4 * e) & 15u)] * scale) |
                             static_cast<uint32_t>(f32_to_bf16(centroid[kv * kKvCentroids + (word >> (4 * e + 4) & 15u)] * scale)) << 16;
        }
        uint16_t* dst = kv ? v + row * v_stride : k + row * k_stride;
        *reinterpret_cast<u32x4_t*>(dst + static_cast<int64_t>(h) * D + d0) = out;
    }
}

hipError_t launch_heads(const HeadsArgs& a, const KvCacheArgs* cache, const KvBatchArgs* batch, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    const KvCacheArgs c = cache ? *cache : KvCacheArgs{};
    const KvBatchArgs b = batch ? *batch : KvBatchArgs{};
    const int lanes = a.head_dim <= 64 ? 8 : a.head_dim <= 128 ? 16 : a.head_dim <= 256 ? 32 : 64;
    const int total = a.q_heads + a.k_heads + a.v_heads, per = kHeadThreads / lanes;
    const int group = a.rows >= 1024 ? total : per;        // few rows: a workgroup a pass; many: the angles of a row are computed once
    const dim3 grid(static_cast<unsigned>(a.rows), static_cast<unsigned>((total + group - 1) / group));
    switch (lanes) {
        case 8: heads_kernel<8><<<grid, kHeadThreads, 0, s>>>(a, c, b, cache != nullptr, group); break;
        case 16: heads_kernel<16><<<grid, kHeadThreads, 0, s>>>(a, c, b, cache != nullptr, group); break;
        case 32: heads_kernel<32><<<grid, kHeadThreads, 0, s>>>(a, c, b, cache != nullptr, group); break;
        default: heads_kernel<64><<<grid, kHeadThreads, 0, s>>>(a, c, b, cache != nullptr, group); break;
    }
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvCacheArgs& c, const KvBatchArgs& b, uint16_t* k, int64_t k_stride, uint16_t* v, int64_t v_stride, hipStream_t s) {
    if (b.rows == 0) return hipSuccess;
    kv_read_kernel<<<dim3(static_cast<unsigned>(b.rows)), kHeadThreads, 0, s>>>(c, b, k, k_stride, v, v_stride);
    return hipGetLastError();
}

}  // namespace kmq
