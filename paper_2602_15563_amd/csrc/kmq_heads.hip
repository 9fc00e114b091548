// Rows of heads between the QKV product and the attention: RMSNorm of every query and key head, the rotation by
// position, and the quantised write of keys and values into the 4-bit cache, in one pass over the row.
//
//     n_i = x_i * gain_i / sqrt( (1/D) sum_j x_j^2 + eps )
//     split pairs (i, i + R/2), i < R/2; interleaved pairs (2i, 2i + 1); a_i = position * inv_freq_i
//     y_left = n_left cos a_i - n_right sin a_i,   y_right = n_right cos a_i + n_left sin a_i
//     cache:  scale = max |y| over 64 elements,  index = number of boundaries b_j with y > b_j * scale
//
// The turning is computed in 64 bits, rounded to 32 and then to bf16: a far position times a frequency needs them, and the
// index of a key is decided by a comparison, so that with them it is the definition's own and the oracle's.  (The vector units
// multiply and add 64-bit floats at the rate of 32-bit ones.)  With r = 1 / sqrt(..) an element is
//     y_e = r * (x_e A_e + x_partner B_e),   A_e = gain_e cos,  B_e = +-gain_partner sin,
// and A and B are the same for all query heads of a row, and for all its key heads: three operations an element.
//
// 4001 rows of 64 query and 8 key heads take 39 us, 3.8 TB/s read and written (a copy of them 31).  A write of keys and values alone is
// bound by vector issue: 10004 rows of 8 + 8 heads 23.5 us, 74 % of it issuing the 17 operations that an element takes.
#include <type_traits>

#include "kmq_kv.h"

namespace kmq {

constexpr int kHeadThreads = 256, kHeadWaves = kHeadThreads / kWave;

__device__ __forceinline__ u32x4_t swap_halves(u32x4_t v) {
    return u32x4_t{v[0] >> 16 | v[0] << 16, v[1] >> 16 | v[1] << 16, v[2] >> 16 | v[2] << 16, v[3] >> 16 | v[3] << 16};
}
// The largest of 8 neighbouring lanes' patterns, in all of them.
__device__ __forceinline__ uint32_t max_over_8(uint32_t v) {
    const auto other = [](uint32_t x, auto ctrl) { return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), decltype(ctrl)::value, 0xF, 0xF, true)); };
    const uint32_t a = other(v, std::integral_constant<int, 0xB1>{});   // quad_perm [1,0,3,2]
    v = a > v ? a : v;
    const uint32_t b = other(v, std::integral_constant<int, 0x4E>{});   // quad_perm [2,3,0,1]
    v = b > v ? b : v;
    const uint32_t c = other(v, std::integral_constant<int, 0x141>{});  // row_half_mirror
    return c > v ? c : v;
}

// What turns the elements of a lane, the same for every head of a kind: y = r * (x * own + partner * far).
struct Factors {
    double own[8], far[8];
};
// `angles`: cosine and sine of every pair, and (1, 0) behind the last for the elements that are not turned.
__device__ __forceinline__ Factors make_factors(const HeadsArgs& a, const uint16_t* gain, const double2* angles, int d0, bool live) {
    Factors f;
    const int half = a.rotary_dim / 2;
    const bool turned = live && d0 < a.rotary_dim, left = d0 < half;
    u32x4_t g = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u}, go = g;
    if (gain && live) g = go = *reinterpret_cast<const u32x4_t*>(gain + d0);
    if (a.interleaved) {
        go = swap_halves(go);
#pragma unroll
        for (int e = 0; e < 4; ++e) go[e] ^= 0x00008000u;                     // the even element takes its partner's sine with a minus
    } else {
        if (gain && turned) go = *reinterpret_cast<const u32x4_t*>(gain + (left ? d0 + half : d0 - half));
#pragma unroll
        for (int e = 0; e < 4; ++e) go[e] ^= left ? 0x80008000u : 0u;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double2 t = angles[!turned ? half : a.interleaved ? d0 / 2 + e / 2 : (left ? d0 : d0 - half) + e];
        f.own[e] = static_cast<double>(kv_half(g[e / 2], e % 2)) * t.x;
        f.far[e] = turned ? static_cast<double>(kv_half(go[e / 2], e % 2)) * t.y : -0.0;      // (partners of zero are added: less zero, so that -0 stays -0)
    }
    return f;
}

// One head's elements of a lane, turned.  `far` are its partners in the split form; `mean` is 1 / D.
template <int LANES>
__device__ __forceinline__ u32x4_t turn_head(const HeadsArgs& a, const Factors& f, u32x4_t own, u32x4_t far, bool turned, double mean) {
    if (a.interleaved && turned) far = swap_halves(own);
    double r = 1.0;
    if (a.norm) {
        double ss = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double x = kv_half(own[e / 2], e % 2);
            ss = fma(x, x, ss);
        }
        r = inverse_root(fma(sum_over<LANES>(ss), mean, static_cast<double>(a.eps)));
    }
    u32x4_t out;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        float y[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const double x = kv_half(own[e / 2], k), p = kv_half(far[e / 2], k);
            y[k] = static_cast<float>(r * fma(x, f.own[e + k], p * f.far[e + k]));
            asm("" : "+v"(y[k]));                         // (else the compiler makes one rounding of the two, which are specified)
        }
        out[e / 2] = kv_pack2(y[0], y[1]);
    }
    return out;
}

// The scale below which 32 bits may not hold what the rounding of boundary * scale takes away.  That is a multiple of 2^-30 of the product (24 and 8
// bits), so they do from 2^-119 on: with boundaries of 2^-40 and more (or zero) for scales of 2^-60 and more, with a smaller boundary for none.
__device__ __forceinline__ float small_scale(const float* boundary) {
    const float edge = fabsf(boundary[threadIdx.x & (kKvCentroids - 1)]);
    return __ballot(edge != 0.f && edge < 0x1p-40f) ? __builtin_inff() : 0x1p-60f;
}

// Eight elements of a block of 64 (8 neighbouring lanes) -> their indices in the nibbles of a dword, and the block's scale.
// `boundary`: the boundaries as a binary tree, node n's children 2 n and 2 n + 1, root 1.  `place`: this wave's thresholds in
// shared memory, a tree for each of its 8 blocks.  A threshold is b * s rounded down: then x > threshold exactly where x > b * s.
// An element walks down the tree, and where it arrives is 16 + its index.  Below a scale of `small` (small_scale) the product is made in
// 64 bits: what its rounding takes away may be too small for 32.
__device__ __forceinline__ uint32_t quantise8(u32x4_t x, const float* boundary, float small, float* place, uint32_t& scale) {
    typedef __attribute__((ext_vector_type(2))) uint16_t u16x2_t;
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1), sub = lane & 7;
    const auto size = [](uint32_t v) { return __builtin_bit_cast(u16x2_t, v & 0x7FFF7FFFu); };
    const u16x2_t m = __builtin_elementwise_max(__builtin_elementwise_max(size(x[0]), size(x[1])), __builtin_elementwise_max(size(x[2]), size(x[3])));
    const uint32_t top = max_over_8(m[0] > m[1] ? m[0] : m[1]);
    scale = top;
    const float s = top ? bf16_to_f32(top) : 1.f;
    float* const tree = place + lane / 8 * 16;
    float t[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float edge = boundary[2 * sub + k];
        t[k] = edge * s;
        if (fmaf(edge, s, -t[k]) < 0.f) t[k] = __uint_as_float(__float_as_uint(t[k]) + (t[k] > 0.f ? -1 : 1));
    }
    if (__ballot(s < small)) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const double exact = static_cast<double>(boundary[2 * sub + k]) * static_cast<double>(s);             // 24 and 8 bits
            t[k] = static_cast<float>(exact);
            if (static_cast<double>(t[k]) > exact)
                t[k] = t[k] == 0.f ? -__uint_as_float(1u) : __uint_as_float(__float_as_uint(t[k]) + (t[k] > 0.f ? -1 : 1));
        }
    }
    tree[2 * sub] = t[0];                                 // (entry 0 is not looked at)
    tree[2 * sub + 1] = t[1];
    __builtin_amdgcn_wave_barrier();
    const float t1 = tree[1], t2 = tree[2], t3 = tree[3];
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float v = kv_half(x[e / 2], e % 2);
        const bool first = v > t1;
        uint32_t n = (first ? 6u : 4u) + (v > (first ? t3 : t2) ? 1u : 0u);
        n = 2 * n + (v > tree[n] ? 1u : 0u);
        n = 2 * n + (v > tree[n] ? 1u : 0u);
        word += n << (4 * e);
    }
    __builtin_amdgcn_wave_barrier();
    return word - 0x11111110u;                            // less the sixteens
}

// Where a row's token goes: the first tile of its page's heads, and its place in the tile.
struct Target {
    uint8_t* page_tile;    // tile of head 0; nullptr: not in the cache
    int token;
};
__device__ __forceinline__ Target target_of(const KvCacheArgs& c, const KvBatchArgs& b, int D, KvRow r) {
    return {kv_tile(c, b, D, r, 0), static_cast<int>(r.pos & (kKvTile - 1))};
}

__device__ __forceinline__ void store_k(uint8_t* tile, int D, int t, int d0, uint32_t word, uint32_t scale) {
    *reinterpret_cast<uint32_t*>(tile + kv_k_dword(D, t, d0)) = word;
    if (d0 % KMQ_BLOCK == 0) *reinterpret_cast<uint16_t*>(tile + kv_scale(D, t, 0, d0)) = static_cast<uint16_t>(scale);
}
// The four bytes of V that a lane stores for a token: elements d and d + 16 for four d, from its own dword and that of the lane which
// holds the other 16.  Returned with byte e for the e-th of the four d.
__device__ __forceinline__ uint32_t v_bytes(uint32_t word, int d0) {
    const uint32_t pair = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(word), 0x4E, 0xF, 0xF, true));   // two lanes on, or back
    const bool upper = d0 & 16;                           // this lane stores the later four of the pair's eight
    const uint32_t lo = upper ? pair >> 16 : word & 0xFFFFu, hi = upper ? word >> 16 : pair & 0xFFFFu;
    // nibbles spread to bytes: 0x4321 -> 0x04030201
    const auto spread = [](uint32_t n) {
        n = (n | n << 8) & 0x00FF00FFu;
        return (n | n << 4) & 0x0F0F0F0Fu;
    };
    return spread(lo) | spread(hi) << 4;
}
__device__ __forceinline__ int v_first(int d0) { return (d0 & ~16) + (d0 & 16 ? 4 : 0); }

// LANES lanes hold a head, 8 elements each; a head never crosses a wave.  ROWS = 1: a workgroup takes a row, or with few rows a
// part of its heads.  ROWS = 4: four rows, cached those of four tokens that share V's dwords, of one sequence; with few of them a part
// of their heads.
template <int LANES, int ROWS, bool TURNS>
__global__ void __launch_bounds__(kHeadThreads, 4) heads_kernel(HeadsArgs a, KvCacheArgs c, KvBatchArgs b, bool cached, int units_per_group) {
    constexpr int kHeads = kWave / LANES;                 // heads of a unit: what a wave takes at once
    __shared__ double2 angles[ROWS][LANES * 4 + 1];        // a head has LANES * 8 elements at most
    __shared__ float boundary[2][kKvCentroids], threshold[kHeadWaves][8 * 16];
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int D = a.head_dim;

    // the rows of this workgroup: first .. first + 3, those in `have`
    int64_t first;
    uint32_t have = 1;
    KvRow at = {0, 0};                                    // of row `first` (which need not be a row: a group starts at a multiple of four tokens)
    if constexpr (ROWS == 1) {
        first = blockIdx.x;
        if (cached) at = kv_find_row(b, first);
        if (at.seq < 0) return;                           // (the same for the whole workgroup)
    } else if (cached) {
        const KvGroup g = kv_find_group(b, static_cast<int>(blockIdx.x));
        if (g.seq < 0) return;
        first = g.row;
        have = g.have;
        at = {g.seq, g.pos};
    } else {
        first = static_cast<int64_t>(blockIdx.x) * ROWS;
        have = a.rows - first >= ROWS ? 15u : (1u << (a.rows - first)) - 1u;
    }
    const int sub = lane % LANES, d0 = sub * 8;
    const bool inside = d0 < D;
    const int pairs = a.rotary_dim / 2, half = pairs;
    const bool turned = inside && d0 < a.rotary_dim;
    const int partner = (lane + (turned ? (d0 < half ? half : -half) / 8 : 0)) * 4;      // the lane of the split form's partners, as a byte address

    // units: what a wave takes at once.  Query and key heads of a row: ROWS = 4: a wave takes the units of its row one after the other,
    // ROWS = 1: they are dealt to the waves in turn.  Then values, of all rows at once.
    const int nq = (a.q_heads + kHeads - 1) / kHeads, nk = (a.k_heads + kHeads - 1) / kHeads, nv = (a.v_heads + kHeads - 1) / kHeads;
    const int units = nq + nk + nv, stride = ROWS == 1 ? kHeadWaves : 1;
    const int begin = static_cast<int>(blockIdx.y) * units_per_group, end = begin + units_per_group < units ? begin + units_per_group : units;
    const int r = ROWS == 1 ? 0 : wave;                   // this wave's row of queries and keys
    const bool mine = have >> r & 1u;
    const int qk_end = !mine ? 0 : end < nq + nk ? end : nq + nk;
    const int64_t row = first + r;
    const auto head_of = [&](int u) __attribute__((always_inline)) { return (u < nq ? u : u - nq) * kHeads + lane / LANES; };
    const auto read = [&](int u) __attribute__((always_inline)) {
        const int h = head_of(u);
        u32x4_t v = {0, 0, 0, 0};
        if (u < qk_end && inside && h < (u < nq ? a.q_heads : a.k_heads))
            v = *reinterpret_cast<const u32x4_t*>((u < nq ? a.q + row * a.q_stride : a.k + row * a.k_stride) + static_cast<int64_t>(h) * D + d0);
        return v;
    };
    int u = begin + (ROWS == 1 ? wave : 0);
    u32x4_t own = read(u);                                // asked for before the angles are computed

    if (TURNS && pairs) {
        const auto angle = [&](int of, int p) __attribute__((always_inline)) {
            const double pos = a.positions ? static_cast<double>(a.positions[first + of]) : static_cast<double>(at.pos + of);
            double2 t;
            sincos(pos * static_cast<double>(a.inv_freq[p]), &t.y, &t.x);
            angles[of][p] = t;
        };
        if constexpr (ROWS == 1) {
            for (int p = tid; p < pairs; p += kHeadThreads) angle(0, p);
        } else if (mine) {
            for (int p = lane; p < pairs; p += kWave) angle(r, p);
        }
    }
    if (TURNS && tid < ROWS) angles[tid][pairs] = double2{1.0, 0.0};
    if (cached && tid < 2 * kKvCentroids) {
        const int kv = tid / kKvCentroids, i = tid % kKvCentroids;
        const uint16_t* book = c.codebooks + kv * kKvCentroids;
        const int level = 31 - __clz(i | 1), j = (2 * (i - (1 << level)) + 1) * (8 >> level) - 1;      // node i of the tree is boundary j
        boundary[kv][i] = i ? (bf16_to_f32(book[j]) + bf16_to_f32(book[j + 1])) * 0.5f : 0.f;
    }
    Target to = {nullptr, 0};
    if (cached) to = target_of(c, b, D, at);
    const int64_t head_bytes = cached ? static_cast<int64_t>(c.page_size / kKvTile) * kv_tile_bytes(D) : 0;
    const double mean = 1.0 / D;
    __syncthreads();
    const float small_k = cached ? small_scale(boundary[0]) : 0.f, small_v = cached ? small_scale(boundary[1]) : 0.f;

    Factors f;
    int factors_of = -1;                                  // the kind that f belongs to
#pragma unroll 1
    for (; u < qk_end; u += stride) {
        const u32x4_t coming = read(u + stride);
        const int kind = u < nq ? 0 : 1, h = head_of(u);
        const bool live = inside && h < (kind ? a.k_heads : a.q_heads);
        if constexpr (TURNS) {
            u32x4_t far = {0, 0, 0, 0};
            if (!a.interleaved && pairs) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t v = static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute(partner, static_cast<int>(own[e])));
                    far[e] = turned ? v : 0u;
                }
            }
            if (factors_of != kind) {
                factors_of = kind;
                f = make_factors(a, !a.norm ? nullptr : kind ? a.k_gain : a.q_gain, angles[r], d0, inside);
            }
            own = turn_head<LANES>(a, f, own, far, turned, mean);
        }
        uint16_t* out = kind ? a.k_out : a.q_out;
        if (out) {
            if (live) *reinterpret_cast<u32x4_t*>(out + row * (kind ? a.k_out_stride : a.q_out_stride) + static_cast<int64_t>(h) * D + d0) = own;
        } else {
            uint32_t scale;
            const uint32_t word = quantise8(own, boundary[0], small_k, threshold[wave], scale);
            if (live && to.page_tile) store_k(to.page_tile + h * head_bytes, D, to.token + r, d0, word, scale);
        }
        own = coming;
    }
    {
        const int lo = begin > nq + nk ? begin : nq + nk;
        for (int v = lo + ((wave - (lo - begin)) & (kHeadWaves - 1)); v < end; v += kHeadWaves) {
            const int h = (v - nq - nk) * kHeads + lane / LANES;
            const bool live = inside && h < a.v_heads;
            uint32_t bytes[ROWS], scale[ROWS];
            u32x4_t x[ROWS];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                x[r] = u32x4_t{0, 0, 0, 0};
                if (live && (have >> r & 1u)) x[r] = *reinterpret_cast<const u32x4_t*>(a.v + (first + r) * a.v_stride + static_cast<int64_t>(h) * D + d0);
            }
#pragma unroll
            for (int r = 0; r < ROWS; ++r) bytes[r] = v_bytes(quantise8(x[r], boundary[1], small_v, threshold[wave], scale[r]), d0);
            if (!live || !to.page_tile) continue;
            uint8_t* tile = to.page_tile + h * head_bytes;
            const int v0 = kv_v_byte(D, to.token, v_first(d0)), step = D / 8;
            bool whole = false;
            if constexpr (ROWS == 4) {                    // whole dwords: bytes of four tokens, for each of four elements
                whole = have == 15u;
                if (whole) {
                    const uint32_t t01 = __builtin_amdgcn_perm(bytes[1], bytes[0], 0x05010400u), t01h = __builtin_amdgcn_perm(bytes[1], bytes[0], 0x07030602u);
                    const uint32_t t23 = __builtin_amdgcn_perm(bytes[3], bytes[2], 0x05010400u), t23h = __builtin_amdgcn_perm(bytes[3], bytes[2], 0x07030602u);
                    *reinterpret_cast<uint32_t*>(tile + v0) = __builtin_amdgcn_perm(t23, t01, 0x05040100u);
                    *reinterpret_cast<uint32_t*>(tile + v0 + step) = __builtin_amdgcn_perm(t23, t01, 0x07060302u);
                    *reinterpret_cast<uint32_t*>(tile + v0 + 2 * step) = __builtin_amdgcn_perm(t23h, t01h, 0x05040100u);
                    *reinterpret_cast<uint32_t*>(tile + v0 + 3 * step) = __builtin_amdgcn_perm(t23h, t01h, 0x07060302u);
                }
            }
            if (!whole) {
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
                    if (have >> r & 1u) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) tile[v0 + e * step + r] = static_cast<uint8_t>(bytes[r] >> (8 * e));
                    }
            }
            if (d0 % KMQ_BLOCK == 0) {
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
                    if (have >> r & 1u) *reinterpret_cast<uint16_t*>(tile + kv_scale(D, to.token + r, 1, d0)) = static_cast<uint16_t>(scale[r]);
            }
        }
    }
}

// Rows of the cache as bf16: one rounding of centroid * scale; zeros where the page table has no page.
// A thread takes eight elements of a head, of one row or of four tokens that share V's dwords.
template <int ROWS>
__global__ void __launch_bounds__(kHeadThreads) kv_read_kernel(KvCacheArgs c, KvBatchArgs b, uint16_t* k, int64_t k_stride, uint16_t* v, int64_t v_stride) {
    __shared__ float centroid[2 * kKvCentroids];
    const int tid = static_cast<int>(threadIdx.x), D = c.head_dim;
    if (tid < 2 * kKvCentroids) centroid[tid] = bf16_to_f32(c.codebooks[tid]);
    int64_t first;
    uint32_t have = 1;
    KvRow at;
    if constexpr (ROWS == 1) {
        first = blockIdx.x;
        at = kv_find_row(b, first);
    } else {
        const KvGroup g = kv_find_group(b, static_cast<int>(blockIdx.x));
        first = g.row;
        have = g.have;
        at = {g.seq, g.pos};
    }
    if (at.seq < 0) return;
    __syncthreads();
    const Target from = target_of(c, b, D, at);
    const int64_t head_bytes = static_cast<int64_t>(c.page_size / kKvTile) * kv_tile_bytes(D);
    const int per_head = D / 8, all = c.kv_heads * per_head;
    for (int i = tid + static_cast<int>(blockIdx.y) * kHeadThreads; i < 2 * all; i += kHeadThreads * static_cast<int>(gridDim.y)) {
        const int kv = i >= all, rest = i - kv * all, h = rest / per_head, d0 = (rest - h * per_head) * 8;
        const uint8_t* tile = from.page_tile + h * head_bytes;
        uint32_t word[ROWS] = {}, scale[ROWS] = {};
        if (from.page_tile) {
            if (kv) {
                const uint8_t* at_v = tile + kv_v_byte(D, from.token, d0 & ~16);
                const int shift = d0 & 16 ? 4 : 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (ROWS == 1) {
                        word[0] |= (static_cast<uint32_t>(at_v[e * (D / 8)]) >> shift & 15u) << (4 * e);
                    } else {
                        const uint32_t w = *reinterpret_cast<const uint32_t*>(at_v + e * (D / 8)) >> shift;
#pragma unroll
                        for (int r = 0; r < ROWS; ++r) word[r] |= (w >> (8 * r) & 15u) << (4 * e);
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                if (!kv) word[r] = *reinterpret_cast<const uint32_t*>(tile + kv_k_dword(D, from.token + r, d0));
                scale[r] = *reinterpret_cast<const uint16_t*>(tile + kv_scale(D, from.token + r, kv, d0));
            }
        }
        uint16_t* out = (kv ? v + first * v_stride : k + first * k_stride) + static_cast<int64_t>(h) * D + d0;
        const float* book = centroid + kv * kKvCentroids;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (!(have >> r & 1u)) continue;
            const float s = bf16_to_f32(scale[r]);
            u32x4_t y = {0, 0, 0, 0};
            if (from.page_tile) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) y[e / 2] = kv_pack2(book[word[r] >> (4 * e) & 15u] * s, book[word[r] >> (4 * e + 4) & 15u] * s);
            }
            *reinterpret_cast<u32x4_t*>(out + r * (kv ? v_stride : k_stride)) = y;
        }
    }
}

// Rows in groups of four tokens where sequences have several rows; the groups there can be at most.
static bool by_groups(const KvBatchArgs& b) { return b.row_starts && b.rows >= 4 * static_cast<int64_t>(b.sequences) && b.rows >= 64; }
static int64_t most_groups(const KvBatchArgs& b) { return kv_pieces(b.rows, b.sequences, 4, 1, kKvGroupSlack); }

// Units of a group's heads that a workgroup takes: where groups are fewer than 512 workgroups a part of them, `least` at least.  Append
// and read back, us, whole groups / parts: 37 sequences of 9 rows (192 + 24 + 24 heads) 60 / 27, a piece of 300 rows (32 + 8 + 8)
// 18.7 / 14.0, of 1024 rows 22 / 19.7; parts up to 1024 workgroups 25, 14.3 and 18.7, but 41.9 for 37 where a piece has 4000 rows.
constexpr int64_t kFewGroups = 512;
static int part_of(int units, int64_t groups, int least) {
    const int64_t parts = groups < kFewGroups ? (kFewGroups + groups - 1) / groups : 1, part = (units + parts - 1) / parts;
    return static_cast<int>(part > least ? part : least < units ? least : units > 0 ? units : 1);
}

template <int LANES, int ROWS>
static void start(bool turns, dim3 grid, hipStream_t s, const HeadsArgs& a, const KvCacheArgs& c, const KvBatchArgs& b, bool cached, int units) {
    if (turns) heads_kernel<LANES, ROWS, true><<<grid, kHeadThreads, 0, s>>>(a, c, b, cached, units);
    else heads_kernel<LANES, ROWS, false><<<grid, kHeadThreads, 0, s>>>(a, c, b, cached, units);
}

hipError_t launch_heads(const HeadsArgs& a, const KvCacheArgs* cache, const KvBatchArgs* batch, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    const KvCacheArgs c = cache ? *cache : KvCacheArgs{};
    const KvBatchArgs b = batch ? *batch : KvBatchArgs{};
    const int lanes = a.head_dim <= 64 ? 8 : a.head_dim <= 128 ? 16 : a.head_dim <= 256 ? 32 : 64, heads = kWave / lanes;
    const int units = (a.q_heads + heads - 1) / heads + (a.k_heads + heads - 1) / heads + (a.v_heads + heads - 1) / heads;
    const bool turns = a.norm || a.rotary_dim;
    if (cache ? by_groups(b) : a.rows >= 1024) {
        const int64_t groups = cache ? most_groups(b) : (a.rows + 3) / 4;
        const int group = part_of(units, groups, 4);
        const dim3 grid(static_cast<unsigned>(groups), static_cast<unsigned>((units + group - 1) / group));
        switch (lanes) {
            case 8: start<8, 4>(turns, grid, s, a, c, b, cache != nullptr, group); break;
            case 16: start<16, 4>(turns, grid, s, a, c, b, cache != nullptr, group); break;
            case 32: start<32, 4>(turns, grid, s, a, c, b, cache != nullptr, group); break;
            default: start<64, 4>(turns, grid, s, a, c, b, cache != nullptr, group); break;
        }
        return hipGetLastError();
    }
    const int group = a.rows >= 1024 ? units : kHeadWaves;         // few rows: a workgroup for four units; many: the angles of a row are computed once
    const dim3 grid(static_cast<unsigned>(a.rows), static_cast<unsigned>((units + group - 1) / group));
    switch (lanes) {
        case 8: start<8, 1>(turns, grid, s, a, c, b, cache != nullptr, group); break;
        case 16: start<16, 1>(turns, grid, s, a, c, b, cache != nullptr, group); break;
        case 32: start<32, 1>(turns, grid, s, a, c, b, cache != nullptr, group); break;
        default: start<64, 1>(turns, grid, s, a, c, b, cache != nullptr, group); break;
    }
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvCacheArgs& c, const KvBatchArgs& b, uint16_t* k, int64_t k_stride, uint16_t* v, int64_t v_stride, hipStream_t s) {
    if (b.rows == 0) return hipSuccess;
    if (by_groups(b)) {
        const int units = (2 * c.kv_heads * (c.head_dim / 8) + kHeadThreads - 1) / kHeadThreads;
        const int64_t groups = most_groups(b);
        const int group = part_of(units, groups, 1);
        const dim3 grid(static_cast<unsigned>(groups), static_cast<unsigned>((units + group - 1) / group));
        kv_read_kernel<4><<<grid, kHeadThreads, 0, s>>>(c, b, k, k_stride, v, v_stride);
    } else {
        const int work = 2 * c.kv_heads * (c.head_dim / 8), wide = b.rows >= 1024 ? 1 : (work + kHeadThreads - 1) / kHeadThreads;
        kv_read_kernel<1><<<dim3(static_cast<unsigned>(b.rows), static_cast<unsigned>(wide)), kHeadThreads, 0, s>>>(c, b, k, k_stride, v, v_stride);
    }
    return hipGetLastError();
}

}  // namespace kmq
