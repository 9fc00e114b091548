// Attention of new rows over the 4-bit key / value cache.
//
//     S_j = scale * sum_blocks sK[j, block] * sum_{d in block} cK[idx(j, d)] * q_d
//     out = sum_j exp(S_j - max S) * sV[j, block] * cV[idx(j, d)]  /  sum_j exp(S_j - max S)
//
// Both products run on the matrix cores as (tokens x elements) * (elements x columns): a column is a (row, query head) pair of
// one key head, so the query heads that share keys share every decoded index.  S^T has its tokens in a lane's four
// registers and in the four quarters of a wave; a 32-token step takes two such results as the second product's operand
// as they are, because V is stored in that order of tokens (kmq_kv.h): no probability crosses a lane.
// Maxima, sums and products are kept in 32 bits; queries and centroids are bf16 as they come, and p * sV is rounded to
// bf16 for the second product (off by 2^-8 of itself at most, to either side; the sum of p that divides it is not rounded).
#include "kmq_kv.h"

namespace kmq {

constexpr int kAttnWaves = 4, kAttnThreads = kAttnWaves * kWave;
constexpr int kAttnColumns = 16;              // columns of a workgroup: one matrix-core tile
constexpr int kAttnMinSteps = 2 * kAttnWaves; // steps of a part at least: fewer are not worth the joining
constexpr float kLowest = -3.402823466e38f;   // start of a running maximum: finite, so that differences from it are no NaN
constexpr float kSlack = 8.f;                 // scores (base 2) may pass the running maximum by this before everything is rescaled
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// 16 centroids as two byte planes (low bytes, high bytes), four entries a register.
struct Centroids {
    uint32_t lo[4], hi[4];
};
__device__ __forceinline__ Centroids load_centroids(const uint16_t* codebook) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(codebook);
    Centroids c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        c.lo[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x06040200u);
        c.hi[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07050301u);
    }
    return c;
}
// Four indices in the low nibbles of a dword's bytes (bits 3 of them moved to `which`, as byte selectors) -> two registers of bf16.
__device__ __forceinline__ void decode4(const Centroids& c, uint32_t idx, uint32_t which, uint32_t& first, uint32_t& second) {
    const uint32_t l = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c.lo[3], c.lo[2], idx), __builtin_amdgcn_perm(c.lo[1], c.lo[0], idx), which);
    const uint32_t h = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c.hi[3], c.hi[2], idx), __builtin_amdgcn_perm(c.hi[1], c.hi[0], idx), which);
    first = __builtin_amdgcn_perm(h, l, 0x05010400u);
    second = __builtin_amdgcn_perm(h, l, 0x07030602u);
}
// A dword of eight indices: the low nibbles of its bytes, then the high ones.  The selector of the last choice takes byte i
// from the upper eight centroids where bit 3 of index i is set (4 + i), else from the lower ones (i).
__device__ __forceinline__ u32x4_t decode8(const Centroids& c, uint32_t w) {
    uint32_t r[4];
    decode4(c, w & 0x07070707u, (w >> 1 & 0x04040404u) | 0x03020100u, r[0], r[1]);
    decode4(c, w >> 4 & 0x07070707u, (w >> 5 & 0x04040404u) | 0x03020100u, r[2], r[3]);
    return u32x4_t{r[0], r[1], r[2], r[3]};
}

// The same from a table of all pairs in shared memory: a byte's two indices are a register's two bf16, in their order.
__device__ __forceinline__ u32x4_t decode8_table(const uint32_t* table, uint32_t w) {
    return u32x4_t{table[w & 0xFFu], table[w >> 8 & 0xFFu], table[w >> 16 & 0xFFu], table[w >> 24]};
}
// Eight bf16 in the order in which decode8 leaves a dword's indices: even ones, then odd ones.
__device__ __forceinline__ u32x4_t even_odd(u32x4_t v) {
    return u32x4_t{__builtin_amdgcn_perm(v[1], v[0], 0x05040100u), __builtin_amdgcn_perm(v[3], v[2], 0x05040100u),
                   __builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u)};
}
__device__ __forceinline__ float half_of(uint32_t v, int upper) { return __uint_as_float(upper ? v & 0xFFFF0000u : v << 16); }

// N dwords (N * 4 a power of two, or a multiple of 16 bytes) from an address aligned to their size, at most 16 bytes a load.
template <int N>
__device__ __forceinline__ void load_words(uint32_t* to, const uint8_t* from) {
    if constexpr (N >= 4) {
#pragma unroll
        for (int i = 0; i < N; i += 4) *reinterpret_cast<u32x4_t*>(to + i) = *reinterpret_cast<const u32x4_t*>(from + 4 * i);
    } else {
        static_assert(N == 2, "two or a multiple of four");
        *reinterpret_cast<u32x2_t*>(to) = *reinterpret_cast<const u32x2_t*>(from);
    }
}
// A step's indices of K and all its scales: of a lane's token in every tile, and of the four tokens of its quarter.
template <int D>
struct KWords {
    uint32_t k[2][D / 32], sc[2][D / 16];
    __device__ __forceinline__ void load(const uint8_t* base, int lane, int quarter) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            load_words<D / 32>(k[t], base + t * 17 * D + lane * (D / 8));
            load_words<D / 16>(sc[t], base + t * 17 * D + 16 * D + quarter * (D / 4));
        }
    }
};
struct Place {
    const uint8_t* base;   // of a step's two tiles
    bool there;
};

__device__ __forceinline__ f32x4_t mfma(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const bf16x2_t v = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
    return __builtin_bit_cast(uint32_t, v);
}
// (the maximum of two, a NaN carried by neither: it reaches the output through exp)
__device__ __forceinline__ float max_over_quarters(float v) {
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float sum_over_quarters(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// The columns a workgroup takes: a tile of the (row, query head) pairs of one sequence and one key head.
struct Tile {
    int seq, index;        // sequence (-1: none), tile in it
    int start, count;      // rows of the sequence
};
__device__ __forceinline__ int clamped_start(const KvBatchArgs& b, int i) {
    const int v = b.row_starts[i], most = static_cast<int>(b.rows);
    return v < 0 ? 0 : v > most ? most : v;
}
__device__ __forceinline__ Tile find_tile(const KvBatchArgs& b, int group, int columns, int at) {
    if (!b.row_starts) {
        const int per = (group + columns - 1) / columns;
        return {at / per, at % per, at / per, 1};
    }
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1);
    int64_t before = 0;                                        // tiles of the sequences of earlier rounds
    for (int i = 0; i < b.sequences; i += kWave) {
        const int s = i + lane;
        int first = 0, n = 0;
        if (s < b.sequences) {
            first = clamped_start(b, s);
            n = clamped_start(b, s + 1) - first;
            n = n < 0 ? 0 : n;
        }
        const int64_t mine = (static_cast<int64_t>(n) * group + columns - 1) / columns;
        int64_t upto = mine;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int64_t o = __shfl_up(upto, d);
            upto += lane >= d ? o : 0;
        }
        const uint64_t past = __ballot(before + upto > at);
        if (past) {
            const int l = __ffsll(static_cast<unsigned long long>(past)) - 1;
            return {i + l, static_cast<int>(at - before - __shfl(upto - mine, l)), __shfl(first, l), __shfl(n, l)};
        }
        before += __shfl(upto, kWave - 1);
    }
    return {-1, 0, 0, 0};
}

struct AttnArgs {
    AttentionArgs a;
    int splits;
    float* part_o;         // splits x rows x heads x D
    float* part_ml;        // splits x rows x heads x 2
};

#ifdef KMQ_ATTN_PERM
constexpr bool LUT_K = false;
#else
constexpr bool LUT_K = true;
#endif
template <int D>
__global__ void __launch_bounds__(kAttnThreads) attn_kernel(AttnArgs A) {
    constexpr int NB = D / KMQ_BLOCK, DT = D / 16;
    constexpr int kTile = 17 * D;
    const AttentionArgs& a = A.a;
    const KvBatchArgs& b = a.batch;
    constexpr int DC = D < 128 ? D : 128;            // elements joined at a time
    __shared__ float part[kAttnWaves][kAttnColumns][DC + 4];
    __shared__ uint32_t table[256];
    __shared__ float stat[2][kAttnWaves][kAttnColumns];

    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
    const int col = lane & 15, quarter = lane >> 4;
    const int head = static_cast<int>(blockIdx.x) % a.cache.kv_heads;
    const int group = a.q_heads / a.cache.kv_heads;
    const Tile tile = find_tile(b, group, kAttnColumns, static_cast<int>(blockIdx.x) / a.cache.kv_heads);
    if (tile.seq < 0) return;

    // this lane's column, and the tokens it may see
    const int64_t column = static_cast<int64_t>(tile.index) * kAttnColumns + col;
    const bool live = column < static_cast<int64_t>(tile.count) * group;
    const int i = live ? static_cast<int>(column / group) : 0;
    const int64_t row = tile.start + i;
    const int qh = head * group + (live ? static_cast<int>(column % group) : 0);
    const int64_t capacity = static_cast<int64_t>(b.table_width) * a.cache.page_size;
    const int64_t length = b.lengths[tile.seq];
    const int64_t inside = length < 0 ? 0 : length < capacity ? length : capacity;
    const int64_t first_pos = length - (b.row_starts ? b.row_starts[tile.seq + 1] - b.row_starts[tile.seq] : 1);
    const int64_t pos = first_pos + i;
    const int64_t see_end = a.causal && pos + 1 < inside ? (pos + 1 > 0 ? pos + 1 : 0) : inside;
    const int64_t see_begin = a.window && pos - a.window + 1 > 0 ? pos - a.window + 1 : 0;
    // the workgroup's range: from its first row's begin to its last row's end
    const int64_t i_lo = static_cast<int64_t>(tile.index) * kAttnColumns / group;
    int64_t i_hi = (static_cast<int64_t>(tile.index) * kAttnColumns + kAttnColumns - 1) / group;
    if (i_hi > tile.count - 1) i_hi = tile.count - 1;
    const int64_t p_lo = first_pos + i_lo, p_hi = first_pos + i_hi;
    const int64_t end = a.causal && p_hi + 1 < inside ? (p_hi + 1 > 0 ? p_hi + 1 : 0) : inside;
    const int64_t begin = a.window && p_lo - a.window + 1 > 0 ? p_lo - a.window + 1 : 0;
    const int step0 = static_cast<int>(begin / kKvStep), step1 = static_cast<int>((end + kKvStep - 1) / kKvStep);
    const int steps = step1 > step0 ? step1 - step0 : 0;
    int per = (steps + A.splits - 1) / A.splits;
    per = per > kAttnMinSteps ? per : kAttnMinSteps;
    const int64_t from64 = step0 + static_cast<int64_t>(blockIdx.y) * per;
    const int from = static_cast<int>(from64 < step1 ? from64 : step1), to = step1 - from < per ? step1 : from + per;

    if (A.splits > 1 && from >= to) {                              // a part without tokens
        if (wave == 0 && quarter == 0 && live) {
            float* ml = A.part_ml + ((static_cast<int64_t>(blockIdx.y) * b.rows + row) * a.q_heads + qh) * 2;
            ml[0] = kLowest;
            ml[1] = 0.f;
        }
        return;
    }

    // queries as the first product's second operand: lane (column, quarter) holds elements 64 b + 16 quarter + 8 j + e, in the
    // order in which a dword's indices are decoded
    u32x4_t q[2 * NB];
#pragma unroll
    for (int s = 0; s < 2 * NB; ++s) {
        u32x4_t v = {0, 0, 0, 0};
        if (live) v = *reinterpret_cast<const u32x4_t*>(a.q + row * a.q_stride + static_cast<int64_t>(qh) * D + s / 2 * 64 + quarter * 16 + s % 2 * 8);
        q[s] = LUT_K ? v : even_odd(v);
    }
    Centroids ck;
    if (LUT_K) {
        const uint32_t at = threadIdx.x;
        table[at] = a.cache.codebooks[at & 15] | static_cast<uint32_t>(a.cache.codebooks[at >> 4]) << 16;
        __syncthreads();
    } else {
        ck = load_centroids(a.cache.codebooks);
    }
    const Centroids cv = load_centroids(a.cache.codebooks + kKvCentroids);
    const float scale = a.scale * kLog2e;

    f32x4_t o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = kLowest, l = 0.f;

    // steps that every live column sees whole need no mask
    const int64_t last_begin = a.window && p_hi - a.window + 1 > 0 ? p_hi - a.window + 1 : 0;
    const int64_t first_end = a.causal && p_lo + 1 < inside ? (p_lo + 1 > 0 ? p_lo + 1 : 0) : inside;
    const int whole_from = static_cast<int>((last_begin + kKvStep - 1) / kKvStep), whole_to = static_cast<int>(first_end / kKvStep);
    const int see_from = static_cast<int>(see_begin), see_to = static_cast<int>(see_end);

    const int32_t* const table_row = b.page_table + static_cast<int64_t>(tile.seq) * b.table_width;
    const int64_t page_stride = static_cast<int64_t>(a.cache.kv_heads) * (a.cache.page_size / kKvTile) * kTile;
    const uint8_t* const head_base = a.cache.pages + static_cast<int64_t>(head) * (a.cache.page_size / kKvTile) * kTile;
    const int steps_per_page = a.cache.page_size / kKvStep;
    int step = from + wave;
    int slot = step / steps_per_page, within = step - slot * steps_per_page;      // of the step whose page is looked up next
    const auto look_up = [&](int s) {                     // page of step s, whose place is (slot, within); then on to the wave's next step
        const int page = s < to ? table_row[slot] : 0;
        const bool there = page >= 0 && page < a.cache.num_pages;
        const uint8_t* base = head_base + (there ? page : 0) * page_stride + within * (2 * kTile);
        within += kAttnWaves;
        while (within >= steps_per_page) {
            within -= steps_per_page;
            ++slot;
        }
        return Place{base, there};
    };
    Place at = look_up(step), next = look_up(step + kAttnWaves);
    KWords<D> kw;
    if (step < to) kw.load(at.base, lane, quarter);
    for (; step < to; step += kAttnWaves) {
        uint32_t vw[2][D / 32];
#pragma unroll
        for (int t = 0; t < 2; ++t) load_words<D / 32>(vw[t], at.base + t * kTile + 8 * D + lane * (D / 8));
        const KWords<D> now = kw;
        if (step + kAttnWaves < to) kw.load(next.base, lane, quarter);
        const Place after = look_up(step + 2 * kAttnWaves);

        float s[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t w = now.k[t][2 * n + j];
                    acc = mfma(LUT_K ? decode8_table(table, w) : decode8(ck, w), q[2 * n + j], acc);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] = fmaf(acc[e], half_of(now.sc[t][n * 2 + e / 2], e % 2), sum[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * t + e] = sum[e] * scale;
        }
        float sv[NB][8];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) sv[n][e] = half_of(now.sc[e / 4][(NB + n) * 2 + e % 4 / 2], e % 2);
        if (step < whole_from || step >= whole_to || !at.there) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int j = step * kKvStep + e / 4 * kKvTile + quarter * 4 + e % 4;
                const bool seen = at.there && j >= see_from && j < see_to;
                s[e] = seen ? s[e] : -INFINITY;
#pragma unroll
                for (int n = 0; n < NB; ++n) sv[n][e] = seen ? sv[n][e] : 0.f;       // (what lies behind a sequence may be anything)
            }
        }
        float top = s[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e]);
        if (__ballot(top > m + kSlack)) {
            top = fmaxf(m, max_over_quarters(top));
            const float shrink = __builtin_amdgcn_exp2f(m - top);
            m = top;
            l *= shrink;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[d][e] *= shrink;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[e] = __builtin_amdgcn_exp2f(s[e] - m);
            l += s[e];
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            u32x4_t p;
#pragma unroll
            for (int e = 0; e < 8; e += 2) p[e / 2] = pack_bf16(s[e] * sv[n][e], s[e + 1] * sv[n][e + 1]);
#pragma unroll
            for (int j = 2 * n; j < 2 * n + 2; ++j) {
                const u32x4_t x = decode8(cv, vw[0][j]), y = decode8(cv, vw[1][j]);
                o[2 * j] = mfma(u32x4_t{x[0], x[1], y[0], y[1]}, p, o[2 * j]);
                o[2 * j + 1] = mfma(u32x4_t{x[2], x[3], y[2], y[3]}, p, o[2 * j + 1]);
            }
        }
        at = next;
        next = after;
    }

    // the waves' results joined: every wave's on the scale of the largest maximum
    l = sum_over_quarters(l);
    if (quarter == 0) {
        stat[0][wave][col] = m;
        stat[1][wave][col] = l;
    }
    __syncthreads();
    float most = stat[0][0][col], all = 0.f;
#pragma unroll
    for (int w = 1; w < kAttnWaves; ++w) most = fmaxf(most, stat[0][w][col]);
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) all += stat[1][w][col] * __builtin_amdgcn_exp2f(stat[0][w][col] - most);
    const int64_t pair = row * a.q_heads + qh;                       // (this lane's column; every wave's lanes have the same ones)
    const bool whole = A.splits == 1;
    const bool none = !(all > 0.f) && !(all != all);                 // nothing seen (a NaN sum stays one)
    if (wave == 0 && quarter == 0 && live) {
        if (!whole) {
            float* ml = A.part_ml + (static_cast<int64_t>(blockIdx.y) * b.rows * a.q_heads + pair) * 2;
            ml[0] = most;
            ml[1] = all;
        } else if (a.lse) {
            a.lse[pair] = none ? -INFINITY : (most + __builtin_amdgcn_logf(all)) * kLn2;
        }
    }
    const float weight = __builtin_amdgcn_exp2f(m - most), norm = none ? 0.f : 1.f / all;
#pragma unroll
    for (int c0 = 0; c0 < D; c0 += DC) {
        if (c0) __syncthreads();
#pragma unroll
        for (int d = 0; d < DC / 16; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[wave][col][16 * d + 4 * quarter + e] = o[c0 / 16 + d][e] * weight;
        __syncthreads();
        // a wave's lane writes its column's elements 4 x (wave * 4 + quarter) + 64 x n
#pragma unroll
        for (int n = 0; n < DC / 64; ++n) {
            const int d = n * 64 + (wave * 4 + quarter) * 4;
            f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kAttnWaves; ++w)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += part[w][col][d + e];
            if (!live) continue;
            if (whole) {
                const u32x2_t r = {pack_bf16(none ? 0.f : sum[0] * norm, none ? 0.f : sum[1] * norm),
                                   pack_bf16(none ? 0.f : sum[2] * norm, none ? 0.f : sum[3] * norm)};
                *reinterpret_cast<u32x2_t*>(a.out + row * a.out_stride + static_cast<int64_t>(qh) * D + c0 + d) = r;
            } else {
                *reinterpret_cast<f32x4_t*>(A.part_o + (static_cast<int64_t>(blockIdx.y) * b.rows * a.q_heads + pair) * D + c0 + d) = sum;
            }
        }
    }
}

// The parts of a (row, query head) pair joined, a wave a pair.  Parts without tokens wrote a sum of zero and are passed over.
template <int D>
__global__ void __launch_bounds__(kAttnThreads) attn_join_kernel(AttnArgs A) {
    const AttentionArgs& a = A.a;
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1);
    const int64_t pairs = a.batch.rows * a.q_heads;
    const int64_t pair = static_cast<int64_t>(blockIdx.x) * kAttnWaves + threadIdx.x / kWave;
    if (pair >= pairs) return;
    const int64_t row = pair / a.q_heads;
    if (kv_find_row(a.batch, row).seq < 0) return;                 // rows of no sequence stay as they were
    float most = kLowest;
    for (int s = 0; s < A.splits; ++s) most = fmaxf(most, A.part_ml[(s * pairs + pair) * 2]);
    float all = 0.f, sum[D / 64];
#pragma unroll
    for (int n = 0; n < D / 64; ++n) sum[n] = 0.f;
    for (int s = 0; s < A.splits; ++s) {
        const float l = A.part_ml[(s * pairs + pair) * 2 + 1];
        if (l == 0.f) continue;
        const float w = __builtin_amdgcn_exp2f(A.part_ml[(s * pairs + pair) * 2] - most);
        all += l * w;
#pragma unroll
        for (int n = 0; n < D / 64; ++n) sum[n] = fmaf(A.part_o[(s * pairs + pair) * D + n * 64 + lane], w, sum[n]);
    }
    const bool none = all == 0.f;
    uint16_t* out = a.out + row * a.out_stride + (pair - row * a.q_heads) * D;
#pragma unroll
    for (int n = 0; n < D / 64; ++n) out[n * 64 + lane] = none ? 0 : f32_to_bf16(sum[n] / all);
    if (a.lse && lane == 0) a.lse[pair] = none ? -INFINITY : (most + __builtin_amdgcn_logf(all)) * kLn2;
}

static int64_t column_tiles(const KvBatchArgs& b, int group, int columns) {
    if (!b.row_starts) return b.rows * ((group + columns - 1) / columns);
    const int64_t used = b.rows < b.sequences ? b.rows : b.sequences;       // sequences that have rows, at most
    return (b.rows * group + (columns - 1) * used) / columns;
}

AttentionPlan attention_plan(const KvCacheArgs& c, const KvBatchArgs& b, int q_heads) {
    AttentionPlan p{"kv_attention", kAttnColumns, 1, 0};
    const int64_t items = column_tiles(b, q_heads / c.kv_heads, kAttnColumns) * c.kv_heads;
    const int64_t steps = static_cast<int64_t>(b.table_width) * (c.page_size / kKvStep);
    int64_t splits = (1024 + items - 1) / (items > 0 ? items : 1);
    const int64_t most = (steps + kAttnMinSteps - 1) / kAttnMinSteps;
    if (splits > most) splits = most;
    if (splits > 256) splits = 256;
    if (splits > 1) {
        p.splits = static_cast<int>(splits);
        p.workspace_bytes = static_cast<size_t>(splits) * b.rows * q_heads * (c.head_dim + 2) * sizeof(float);
    }
    return p;
}

template <int D>
static hipError_t launch_attn(const AttnArgs& A, int64_t items, hipStream_t s) {
    attn_kernel<D><<<dim3(static_cast<unsigned>(items), static_cast<unsigned>(A.splits)), kAttnThreads, 0, s>>>(A);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || A.splits == 1) return e;
    const int64_t pairs = A.a.batch.rows * A.a.q_heads;
    attn_join_kernel<D><<<dim3(static_cast<unsigned>((pairs + kAttnWaves - 1) / kAttnWaves)), kAttnThreads, 0, s>>>(A);
    return hipGetLastError();
}

hipError_t launch_attention(const AttentionArgs& a, hipStream_t s) {
    if (a.batch.rows == 0) return hipSuccess;
    const AttentionPlan p = attention_plan(a.cache, a.batch, a.q_heads);
    AttnArgs A{a, p.splits, static_cast<float*>(a.workspace), nullptr};
    if (p.splits > 1) A.part_ml = A.part_o + static_cast<int64_t>(p.splits) * a.batch.rows * a.q_heads * a.cache.head_dim;
    const int64_t items = column_tiles(a.batch, a.q_heads / a.cache.kv_heads, p.columns) * a.cache.kv_heads;
    switch (a.cache.head_dim) {
        case 64: return launch_attn<64>(A, items, s);
        case 128: return launch_attn<128>(A, items, s);
        default: return launch_attn<256>(A, items, s);
    }
}

}  // namespace kmq
