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
// Steps of a part at least (us with 8 / 16: one sequence of 4096 tokens, 8 key heads 10.9 / 14.5; one of 16000 16.7 / 14.9).
constexpr int kAttnMinSteps = 2 * kAttnWaves;
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
// Of V, whose bytes hold elements d and d + 16 of a token: tokens side by side, as decode8 leaves them.
__device__ __forceinline__ u32x4_t decode8_table_of_v(const uint32_t* table, uint32_t w) {
    const u32x4_t r = decode8_table(table, w);
    return u32x4_t{__builtin_amdgcn_perm(r[1], r[0], 0x05040100u), __builtin_amdgcn_perm(r[3], r[2], 0x05040100u),
                   __builtin_amdgcn_perm(r[1], r[0], 0x07060302u), __builtin_amdgcn_perm(r[3], r[2], 0x07060302u)};
}
// Eight bf16 in the order in which decode8 leaves a dword's indices: even ones, then odd ones.
__device__ __forceinline__ u32x4_t even_odd(u32x4_t v) {
    return u32x4_t{__builtin_amdgcn_perm(v[1], v[0], 0x05040100u), __builtin_amdgcn_perm(v[3], v[2], 0x05040100u),
                   __builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u)};
}
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
    // Whether a scale of K, of any of the step's tokens, is an infinity or a NaN (or has a sign, which none has that is written here).
    __device__ __forceinline__ bool not_finite() const {
        typedef __attribute__((ext_vector_type(2))) uint16_t u16x2_t;
        u16x2_t most = {0, 0};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < D / 32; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2_t, sc[t][i]));
        return __ballot(most[0] > 0x7F7F || most[1] > 0x7F7F) != 0;
    }
};
__device__ __forceinline__ f32x4_t mfma(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
// A column of queries with an infinity becomes one with a NaN.  Every score of such a row is an infinity or a NaN, and exp(S) / sum exp(S) is NaN
// whichever they are; but where all of them are minus infinity, they would pass for tokens that are not seen.  The products with
// zeros find the column: 0, or NaN.  (While the first step is on its way; a comparison of every element took 0.1 to 0.3 us longer.)
template <int N>
__device__ __forceinline__ void infinity_to_nan(u32x4_t (&q)[N]) {
    f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < N; ++s) zero = mfma(u32x4_t{0, 0, 0, 0}, q[s], zero);
    q[0][0] |= zero[0] == 0.f ? 0u : 0x00007FC0u;
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
__device__ __forceinline__ KvPiece find_tile(const KvBatchArgs& b, int group, int columns, int at) {
    if (!b.row_starts) {
        const int per = (group + columns - 1) / columns, seq = at / per;
        return {seq, at - seq * per, seq, 1};
    }
    KvPiece p = kv_find_piece(b, at, columns, group, columns - 1);
    if (p.index * static_cast<int64_t>(columns) >= static_cast<int64_t>(p.count) * group) p.seq = -1;
    return p;
}

struct AttnArgs {
    AttentionArgs a;
    int splits;
    float* part_o;         // splits x rows x heads x D
    float* part_ml;        // splits x rows x heads x 2
};

// The positions that a row sees: causal up to its own, a window back from it.
struct Sight {
    int64_t first_pos;     // of the sequence's first row: may be negative
    int64_t inside;        // tokens that the cache can hold
    int window;
    bool causal;
    __device__ __forceinline__ int64_t begin(int64_t row) const {
        const int64_t v = first_pos + row - window + 1;
        return window && v > 0 ? v : 0;
    }
    __device__ __forceinline__ int64_t end(int64_t row) const {
        const int64_t v = first_pos + row + 1;
        return causal && v < inside ? (v > 0 ? v : 0) : inside;
    }
};
__device__ __forceinline__ Sight sight_of(const AttentionArgs& a, int seq) {
    const KvBatchArgs& b = a.batch;
    const int64_t length = b.lengths[seq], capacity = static_cast<int64_t>(b.table_width) * a.cache.page_size;
    const int64_t rows = b.row_starts ? static_cast<int64_t>(b.row_starts[seq + 1]) - b.row_starts[seq] : 1;
    return {length - rows, length < 0 ? 0 : length < capacity ? length : capacity, a.window, a.causal};
}
// Steps of 32 tokens: those that any of the rows lo..hi sees, and those that every one of them sees whole (they need no mask).
struct Steps {
    int from, to, whole_from, whole_to;
};
__device__ __forceinline__ Steps steps_of(const Sight& g, int64_t lo, int64_t hi) {
    Steps s;
    s.from = static_cast<int>(g.begin(lo) / kKvStep);
    s.to = static_cast<int>((g.end(hi) + kKvStep - 1) / kKvStep);
    s.to = s.to > s.from ? s.to : s.from;
    s.whole_from = static_cast<int>((g.begin(hi) + kKvStep - 1) / kKvStep);
    s.whole_to = static_cast<int>(g.end(lo) / kKvStep);
    return s;
}
// This workgroup's part of them.
__device__ __forceinline__ void take_part(Steps& s, int splits, int part) {
    int per = (s.to - s.from + splits - 1) / splits;
    per = per > kAttnMinSteps ? per : kAttnMinSteps;
    const int64_t from = s.from + static_cast<int64_t>(part) * per;
    s.from = static_cast<int>(from < s.to ? from : s.to);
    s.to = s.to - s.from < per ? s.to : s.from + per;
}

// Walks the page table along steps.  64 page numbers are read at once, one a lane: a number read by itself for every step would be waited
// for, and read as a scalar it would make every wait for shared memory a wait for all of it.
struct Place {
    const uint8_t* base;   // of a step's two tiles
    bool there;
};
template <int D>
struct Walk {
    const int32_t* table;
    const uint8_t* head_base;
    int64_t page_stride;
    int width, num_pages, steps_per_page;
    int slot, within;      // of the step that the walk stands at
    int first_slot, pages; // of lane 0, and this lane's number
    __device__ __forceinline__ Walk(const AttentionArgs& a, int seq, int head, int step) {
        const int tiles = a.cache.page_size / kKvTile;
        table = a.batch.page_table + static_cast<int64_t>(seq) * a.batch.table_width;
        width = a.batch.table_width;
        num_pages = static_cast<int>(a.cache.num_pages);
        page_stride = static_cast<int64_t>(a.cache.kv_heads) * tiles * (17 * D);
        head_base = a.cache.pages + static_cast<int64_t>(head) * tiles * (17 * D);
        steps_per_page = tiles / 2;
        slot = step / steps_per_page;
        within = step - slot * steps_per_page;
        pages = read();
    }
    __device__ __forceinline__ int read() {
        const int at = slot + (static_cast<int>(threadIdx.x) & (kWave - 1));
        first_slot = slot;
        return at < width ? table[at] : -1;
    }
    // The place of the step that the walk stands at (one that is not there reads the first page, and nothing of it is used).
    __device__ __forceinline__ Place place(bool inside) {
        if (slot - first_slot >= kWave) {
            int v = read();
            asm volatile("" : "+v"(v));                   // (waited for here, and not wherever the number is used)
            pages = v;
        }
        const int page = __builtin_amdgcn_readlane(pages, slot - first_slot);
        const bool there = inside && page >= 0 && page < num_pages;
        return {head_base + (there ? page : 0) * page_stride + static_cast<int64_t>(within) * (2 * 17 * D), there};
    }
    __device__ __forceinline__ void on(int stride) {
        within += stride;
        while (within >= steps_per_page) {
            within -= steps_per_page;
            ++slot;
        }
    }
};

// Probabilities times the scales of V, as bf16.
__device__ __forceinline__ u32x4_t weigh(const float (&p)[8], const float (&sv)[8]) {
    u32x4_t r;
#pragma unroll
    for (int e = 0; e < 8; e += 2) r[e / 2] = kv_pack2(p[e] * sv[e], p[e + 1] * sv[e + 1]);
    return r;
}
// Zeros for the tokens that are not seen, whatever their scales are.  (Not for every probability of zero: that of a token which is seen may
// round to it, and an infinity or a NaN in its values reaches the row.)
template <typename F>
__device__ __forceinline__ void clear_unseen(u32x4_t& w, const F& seen) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) w[e / 2] &= (seen(e) ? 0x0000FFFFu : 0u) | (seen(e + 1) ? 0xFFFF0000u : 0u);
}

// CT columns' running maxima, sums, and how far a score (base 2, less the maximum) may be up before everything is brought to a new
// maximum: kSlack, and before the first token anything that is a number.
template <int CT>
struct Running {
    float m[CT], l[CT], limit[CT];
    __device__ __forceinline__ Running() {
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            m[c] = l[c] = 0.f;
            limit[c] = kLowest;
        }
    }
    __device__ __forceinline__ float maximum(int c) const { return limit[c] == kLowest ? kLowest : m[c]; }
    // The maxima follow the scores of a step: this lane's four tokens of each of its tiles.
    template <int DT>
    __device__ __forceinline__ void follow(float (&s)[CT][8], f32x4_t (&o)[CT][DT]) {
        float top[CT];
        bool past = false;
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            top[c] = s[c][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) top[c] = fmaxf(top[c], s[c][e]);
            past |= top[c] > limit[c];
        }
        if (__ballot(past)) {
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const bool first = limit[c] == kLowest;           // (nothing is accumulated yet, and the maximum may be far below 0)
                const float to = max_over_quarters(top[c]), up = to > (first ? kLowest : 0.f) ? to : 0.f;
                const float shrink = first ? 1.f : __builtin_amdgcn_exp2f(-up);
                limit[c] = to > kLowest ? kSlack : limit[c];
                m[c] += up;
                l[c] *= shrink;
#pragma unroll
                for (int e = 0; e < 8; ++e) s[c][e] -= up;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[c][d][e] *= shrink;
            }
        }
    }
    // Scores become probabilities, and are added up.
    __device__ __forceinline__ void soften(float (&s)[CT][8]) {
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s[c][e] = __builtin_amdgcn_exp2f(s[c][e]);
                l[c] += s[c][e];
            }
    }
};

// Few columns a sequence (single tokens, drafts): a workgroup takes 16 x CT columns, and its waves take the steps in turn.  A wave reads
// and decodes for itself, K and half of V by tables of index pairs in shared memory, the other half of V by byte permutes from
// registers: any more of one alone keeps its unit busier than the memory (16 contexts of 17408 to 32768 tokens, when each was tried: 112 us so,
// 121 with K alone by the table, 118 with all of V too; nothing by it 151, when K alone took 134).  They take 102 us now, 4.3 TB/s of cache (a
// copy takes 91): vector issue is busy for 73 % of that and the tables for 69 % (48 % lanes that want the same bank).
// Two column tiles take 228 registers at 128 elements (two waves a unit, not three) and decode half as often.
template <int D, int CT>
__global__ void __launch_bounds__(kAttnThreads, 2) attn_kernel(AttnArgs A) {
    constexpr int NB = D / KMQ_BLOCK, DT = D / 16;
    constexpr int kTile = 17 * D, kColumns = kAttnColumns * CT;
    const AttentionArgs& a = A.a;
    const KvBatchArgs& b = a.batch;
    constexpr int DC = D < 128 ? D : 128;            // elements joined at a time
    __shared__ float part[kAttnWaves][kAttnColumns][DC + 4];
    __shared__ uint32_t table[2][256];                // pairs of centroids of K, and of V
    __shared__ float stat[2][kAttnWaves][kColumns];

    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
    const int col = lane & 15, quarter = lane >> 4;
    const int head = static_cast<int>(blockIdx.x) % a.cache.kv_heads;
    const int group = a.q_heads / a.cache.kv_heads;
    const KvPiece tile = find_tile(b, group, kColumns, static_cast<int>(blockIdx.x) / a.cache.kv_heads);
    if (tile.seq < 0) return;

    // this lane's columns, and the tokens they may see
    const int first_column = tile.index * kColumns, columns = tile.count * group;      // (fewer than 2^30: kmq_kv_attention sees to it)
    const Sight sight = sight_of(a, tile.seq);
    bool live[CT];
    int64_t row[CT];
    int qh[CT], see_from[CT], see_to[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        live[c] = first_column + 16 * c + col < columns;
        const int column = live[c] ? first_column + 16 * c + col : first_column, i = column / group;
        row[c] = tile.start + i;
        qh[c] = head * group + column - i * group;
        see_from[c] = static_cast<int>(sight.begin(i));
        see_to[c] = static_cast<int>(sight.end(i));
    }
    const int last_column = first_column + kColumns < columns ? first_column + kColumns - 1 : columns - 1;
    Steps steps = steps_of(sight, first_column / group, last_column / group);
    take_part(steps, A.splits, static_cast<int>(blockIdx.y));

    if (A.splits > 1 && steps.from >= steps.to) {                              // a part without tokens
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            if (wave || quarter || !live[c]) continue;
            float* ml = A.part_ml + ((static_cast<int64_t>(blockIdx.y) * b.rows + row[c]) * a.q_heads + qh[c]) * 2;
            ml[0] = kLowest;
            ml[1] = 0.f;
        }
        return;
    }

    // what is read first is asked for together: page numbers, queries, codebooks, and then the first step
    int step = steps.from + wave;
    Walk<D> walk(a, tile.seq, head, step);
    // queries as the first product's second operand: lane (column, quarter) holds elements 64 b + 16 quarter + 8 j + e
    u32x4_t q[CT][2 * NB];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int s = 0; s < 2 * NB; ++s) {
            u32x4_t v = {0, 0, 0, 0};
            if (live[c]) v = *reinterpret_cast<const u32x4_t*>(a.q + row[c] * a.q_stride + static_cast<int64_t>(qh[c]) * D + s / 2 * 64 + quarter * 16 + s % 2 * 8);
            q[c][s] = v;
        }
    uint32_t pairs[2];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        const uint16_t* book = a.cache.codebooks + kv * kKvCentroids;
        pairs[kv] = book[threadIdx.x & 15] | static_cast<uint32_t>(book[threadIdx.x >> 4]) << 16;
    }
    const Centroids cv = load_centroids(a.cache.codebooks + kKvCentroids);
    Place at = walk.place(step < steps.to);
    KWords<D> kw;
    if (step < steps.to) kw.load(at.base, lane, quarter);
    table[0][threadIdx.x] = pairs[0];
    table[1][threadIdx.x] = pairs[1];
#pragma unroll
    for (int c = 0; c < CT; ++c) infinity_to_nan(q[c]);
    __syncthreads();
    const float scale = a.scale * kLog2e;

    f32x4_t o[CT][DT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int d = 0; d < DT; ++d) o[c][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    Running<CT> run;

    for (; step < steps.to; step += kAttnWaves) {
        uint32_t vw[2][D / 32];
#pragma unroll
        for (int t = 0; t < 2; ++t) load_words<D / 32>(vw[t], at.base + t * kTile + 8 * D + lane * (D / 8));
        const KWords<D> now = kw;
        walk.on(kAttnWaves);
        const Place next = walk.place(step + kAttnWaves < steps.to);
        if (step + kAttnWaves < steps.to) kw.load(next.base, lane, quarter);

        // a key whose scale is an infinity scores NaN: its product with the sum over the block would be one of either sign, and minus infinity no score
        const bool odd = now.not_finite();
        float s[CT][8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4_t sum[CT];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                f32x4_t acc[CT];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const u32x4_t w = decode8_table(table[0], now.k[t][2 * n + j]);
#pragma unroll
                    for (int c = 0; c < CT; ++c) acc[c] = mfma(w, q[c][2 * n + j], j ? acc[c] : f32x4_t{0.f, 0.f, 0.f, 0.f});
                }
#pragma unroll
                for (int c = 0; c < CT; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[c][e] = fmaf(acc[c][e], kv_half(now.sc[t][n * 2 + e / 2], e % 2), n ? sum[c][e] : 0.f);
            }
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[c][4 * t + e] = fmaf(sum[c][e], scale, -run.m[c]);
        }
        const bool masked = step < steps.whole_from || step >= steps.whole_to || !at.there || odd;
        const auto seen = [&](int first, int c, int e) __attribute__((always_inline)) {
            const int j = first + e / 4 * kKvTile + e % 4;
            return at.there && j >= see_from[c] && j < see_to[c];
        };
        if (masked) {
            const int first = step * kKvStep + quarter * 4;
            if (odd) {                                               // (read again: held until here, the scales would take registers in every step)
                const uint8_t* scales = at.base + 16 * D + quarter * (D / 4);
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        uint32_t w = *reinterpret_cast<const uint32_t*>(scales + e / 4 * kTile + n * 8 + e % 4 * 2);
                        asm volatile("" : "+v"(w));
#pragma unroll
                        for (int c = 0; c < CT; ++c) {
                            s[c][e] += kv_half(w, 0) * 0.f;
                            s[c][e + 1] += kv_half(w, 1) * 0.f;
                        }
                    }
            }
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) s[c][e] = seen(first, c, e) ? s[c][e] : -INFINITY;
        }
        run.template follow<DT>(s, o);
        run.soften(s);
        u32x4_t p[NB][CT];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            float sv[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) sv[e] = kv_half(now.sc[e / 4][(NB + n) * 2 + e % 4 / 2], e % 2);
#pragma unroll
            for (int c = 0; c < CT; ++c) p[n][c] = weigh(s[c], sv);
        }
        if (masked) {
            int first = step * kKvStep + quarter * 4;
            asm volatile("" : "+v"(first));                          // (worked out again: what the mask found would be held through every step)
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int c = 0; c < CT; ++c) clear_unseen(p[n][c], [&](int e) { return seen(first, c, e); });
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) {
#pragma unroll
            for (int j = 2 * n; j < 2 * n + 2; ++j) {
                const u32x4_t x = decode8_table_of_v(table[1], vw[0][j]), y = decode8(cv, vw[1][j]);
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    o[c][2 * j] = mfma(u32x4_t{x[0], x[1], y[0], y[1]}, p[n][c], o[c][2 * j]);
                    o[c][2 * j + 1] = mfma(u32x4_t{x[2], x[3], y[2], y[3]}, p[n][c], o[c][2 * j + 1]);
                }
            }
        }
        at = next;
    }

    // the waves' results joined: every wave's on the scale of the largest maximum
    float m[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const float sum_l = sum_over_quarters(run.l[c]);
        m[c] = run.maximum(c);
        if (quarter == 0) {
            stat[0][wave][16 * c + col] = m[c];
            stat[1][wave][16 * c + col] = sum_l;
        }
    }
    __syncthreads();
    const bool whole = A.splits == 1;
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int place = 16 * c + col;
        float most = stat[0][0][place], all = 0.f;
#pragma unroll
        for (int w = 1; w < kAttnWaves; ++w) most = fmaxf(most, stat[0][w][place]);
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) all += stat[1][w][place] * __builtin_amdgcn_exp2f(stat[0][w][place] - most);
        const int64_t pair = row[c] * a.q_heads + qh[c];             // (this lane's column; every wave's lanes have the same ones)
        const bool none = !(all > 0.f) && !(all != all);             // nothing seen (a NaN sum stays one)
        if (wave == 0 && quarter == 0 && live[c]) {
            if (!whole) {
                float* ml = A.part_ml + (static_cast<int64_t>(blockIdx.y) * b.rows * a.q_heads + pair) * 2;
                ml[0] = most;
                ml[1] = all;
            } else if (a.lse) {
                a.lse[pair] = none ? -INFINITY : (most + __builtin_amdgcn_logf(all)) * kLn2;
            }
        }
        const float weight = __builtin_amdgcn_exp2f(m[c] - most), norm = none ? 0.f : 1.f / all;
#pragma unroll
        for (int c0 = 0; c0 < D; c0 += DC) {
            if (c || c0) __syncthreads();
#pragma unroll
            for (int d = 0; d < DC / 16; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) part[wave][col][16 * d + 4 * quarter + e] = o[c][c0 / 16 + d][e] * weight;
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
                if (!live[c]) continue;
                if (whole) {
                    const u32x2_t r = {kv_pack2(none ? 0.f : sum[0] * norm, none ? 0.f : sum[1] * norm),
                                       kv_pack2(none ? 0.f : sum[2] * norm, none ? 0.f : sum[3] * norm)};
                    *reinterpret_cast<u32x2_t*>(a.out + row[c] * a.out_stride + static_cast<int64_t>(qh[c]) * D + c0 + d) = r;
                } else {
                    *reinterpret_cast<f32x4_t*>(A.part_o + (static_cast<int64_t>(blockIdx.y) * b.rows * a.q_heads + pair) * D + c0 + d) = sum;
                }
            }
        }
    }
}

// Many columns a sequence (prompts, long drafts): a workgroup takes 16 x CT columns a wave, and its waves decode every step
// together, an equal share of it each, into shared memory in the order of the first product's and the second product's first operand.
// Two such buffers: the next step is decoded into one while the products read the other.  A prompt of 4096 tokens (32 query heads of
// 128 elements) takes 210 us, 653 TFLOP/s: vector issue (exponentials, scales, roundings, decode) is busy for 57 % of it and the
// matrix cores for 28 %, and two waves a unit, which is what the registers allow, seldom overlap them.
template <int D, int CT, int WAVES>
__global__ void __launch_bounds__(WAVES * kWave, 2) attn_tile_kernel(AttnArgs A) {
    constexpr int NB = D / KMQ_BLOCK, DT = D / 16, KF = D / 32;
    constexpr int kTile = 17 * D, kColumns = WAVES * 16 * CT;
    // a wave's dwords a lane: of K in one tile (a share of it), of V in both tiles (where waves are more than those: half of the nibbles of one)
    constexpr int kShares = WAVES / 2, KD = KF / kShares;
    constexpr bool kHalves = KF < WAVES;
    static_assert(KD >= 1 && (kHalves ? WAVES == 2 * KF : WAVES == KF), "an equal share");
    __shared__ u32x4_t kf[2][2 * KF][kWave], vf[2][DT][kWave];
    __shared__ float scales[2][D];                                   // in the tiles' order, K's times the scale of the scores
    const AttentionArgs& a = A.a;
    const KvBatchArgs& b = a.batch;
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int col = lane & 15, quarter = lane >> 4;
    const int head = static_cast<int>(blockIdx.x) % a.cache.kv_heads;
    const int group = a.q_heads / a.cache.kv_heads;
    // the last tiles first: they see most
    const KvPiece tile = find_tile(b, group, kColumns, static_cast<int>(gridDim.x / a.cache.kv_heads - 1 - blockIdx.x / a.cache.kv_heads));
    if (tile.seq < 0) return;

    const int columns = tile.count * group;
    const int first_column = tile.index * kColumns, mine = first_column + wave * 16 * CT;
    const int last_column = first_column + kColumns < columns ? first_column + kColumns - 1 : columns - 1;
    const int my_last = mine + 16 * CT < columns ? mine + 16 * CT - 1 : columns - 1;
    const bool busy = mine < columns;                                // a wave without columns works all the same, and stores nothing
    const Sight sight = sight_of(a, tile.seq);
    Steps steps = steps_of(sight, first_column / group, last_column / group);
    Steps own = steps_of(sight, (busy ? mine : first_column) / group, (busy ? my_last : first_column) / group);
    take_part(steps, A.splits, static_cast<int>(blockIdx.y));

    u32x4_t q[CT][2 * NB];
    f32x4_t o[CT][DT];
    Running<CT> run;
    int see_from[CT], see_to[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int column = mine + 16 * c + col;
        const bool live = column < columns;
        const int at_column = live ? column : columns - 1, i = at_column / group;
        see_from[c] = static_cast<int>(sight.begin(i));
        see_to[c] = static_cast<int>(sight.end(i));
        const uint16_t* from = a.q + static_cast<int64_t>(tile.start + i) * a.q_stride + (head * group + at_column - i * group) * D;
#pragma unroll
        for (int s = 0; s < 2 * NB; ++s) {
            u32x4_t v = {0, 0, 0, 0};
            if (live) v = *reinterpret_cast<const u32x4_t*>(from + s / 2 * 64 + quarter * 16 + s % 2 * 8);
            q[c][s] = even_odd(v);
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) o[c][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const Centroids ck = load_centroids(a.cache.codebooks), cv = load_centroids(a.cache.codebooks + kKvCentroids);

    // this wave's share of a step
    const int kt = wave / kShares, k0 = wave % kShares * KD;
    const int v0 = kHalves ? wave >> 1 : wave, v_shift = (wave & 1) * 4;
    const bool of_k = !(tid / (2 * NB) & 1);                         // (dword tid of a step's scales: a quarter's K, then its V)
    const float sf = a.scale * kLog2e;
    uint32_t kw[KD], vw[2], sw = 0;
    const auto load = [&](const uint8_t* base) __attribute__((always_inline)) {
        const uint8_t* k = base + kt * kTile + lane * (D / 8) + 4 * k0;
        if constexpr (KD == 1) kw[0] = *reinterpret_cast<const uint32_t*>(k);
        else load_words<KD>(kw, k);
#pragma unroll
        for (int t = 0; t < 2; ++t) vw[t] = *reinterpret_cast<const uint32_t*>(base + t * kTile + 8 * D + lane * (D / 8) + 4 * v0);
        if (tid < D / 2) sw = *reinterpret_cast<const uint32_t*>(base + tid / (D / 4) * kTile + 16 * D + tid % (D / 4) * 4);
    };
    const auto decode = [&](int buffer) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < KD; ++i) kf[buffer][kt * KF + k0 + i][lane] = decode8(ck, kw[i]);
        if constexpr (!kHalves) {
            const u32x4_t x = decode8(cv, vw[0]), y = decode8(cv, vw[1]);
            vf[buffer][2 * v0][lane] = u32x4_t{x[0], x[1], y[0], y[1]};
            vf[buffer][2 * v0 + 1][lane] = u32x4_t{x[2], x[3], y[2], y[3]};
        } else {
            uint32_t r[4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint32_t w = vw[t] >> v_shift;
                decode4(cv, w & 0x07070707u, (w >> 1 & 0x04040404u) | 0x03020100u, r[2 * t], r[2 * t + 1]);
            }
            vf[buffer][wave][lane] = u32x4_t{r[0], r[1], r[2], r[3]};
        }
        if (tid < D / 2) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float x = kv_half(sw, i);
                scales[buffer][2 * tid + i] = of_k ? fmaf(x, 0.f, x * sf) : x;     // (of K an infinity becomes a NaN)
            }
        }
    };
    const auto multiply = [&](int step, int buffer, bool there) __attribute__((always_inline)) {
        float s[CT][8];
        __builtin_amdgcn_s_setprio(1);                               // the waves of a unit out of step: one multiplies while another computes exponentials
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const u32x4_t a0 = kf[buffer][t * KF + 2 * n][lane], a1 = kf[buffer][t * KF + 2 * n + 1][lane];
                const f32x4_t sk = *reinterpret_cast<const f32x4_t*>(&scales[buffer][t * (D / 2) + quarter * (D / 8) + 4 * n]);
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
                    acc = mfma(a0, q[c][2 * n], acc);
                    acc = mfma(a1, q[c][2 * n + 1], acc);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[c][4 * t + e] = fmaf(acc[e], sk[e], n ? s[c][4 * t + e] : -run.m[c]);
                }
            }
        __builtin_amdgcn_s_setprio(0);
        const bool masked = step < own.whole_from || step >= own.whole_to || !there;
        const auto seen = [&](int first, int c, int e) __attribute__((always_inline)) {
            const int j = first + e / 4 * kKvTile + e % 4;
            return there && j >= see_from[c] && j < see_to[c];
        };
        if (masked) {
            const int first = step * kKvStep + quarter * 4;
            asm volatile("");                                        // (kept a branch: few steps are masked)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) s[c][e] = seen(first, c, e) ? s[c][e] : -INFINITY;
        }
        run.template follow<DT>(s, o);
        run.soften(s);
        u32x4_t p[NB][CT];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            float sv[8];
#pragma unroll
            for (int t = 0; t < 2; ++t)
                *reinterpret_cast<f32x4_t*>(sv + 4 * t) = *reinterpret_cast<const f32x4_t*>(&scales[buffer][t * (D / 2) + quarter * (D / 8) + 4 * (NB + n)]);
#pragma unroll
            for (int c = 0; c < CT; ++c) p[n][c] = weigh(s[c], sv);
        }
        if (masked) {
            int first = step * kKvStep + quarter * 4;
            asm volatile("" : "+v"(first));
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int c = 0; c < CT; ++c) clear_unseen(p[n][c], [&](int e) { return seen(first, c, e); });
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const u32x4_t v = vf[buffer][d][lane];
#pragma unroll
            for (int c = 0; c < CT; ++c) o[c][d] = mfma(v, p[d / 4][c], o[c][d]);
        }
    };

    const int last = steps.to - 1;
    if (steps.from <= last) {
        Walk<D> walk(a, tile.seq, head, steps.from);
        Place place = walk.place(true);
        bool there = place.there;                                    // whether the step in the buffer, and the one in registers, is in the cache
        load(place.base);
#pragma unroll
        for (int c = 0; c < CT; ++c) infinity_to_nan(q[c]);
        walk.on(1);
        place = walk.place(steps.from < last);
        decode(0);
        load(place.base);
        bool coming = place.there;
        __syncthreads();
#pragma unroll 1
        for (int step = steps.from, buffer = 0; step <= last; ++step, buffer ^= 1) {
            decode(buffer ^ 1);                                      // the next step's
            walk.on(1);
            place = walk.place(step + 2 <= last);
            load(place.base);
            if (busy && step >= own.from && step < own.to) multiply(step, buffer, there);
            there = coming;
            coming = place.there;
            __syncthreads();
        }
    }

    const bool whole = A.splits == 1;
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int column = mine + 16 * c + col;
        const float all = sum_over_quarters(run.l[c]), most = run.maximum(c);
        if (column >= columns) continue;
        const bool none = all == 0.f;
        const float norm = none ? 0.f : 1.f / all;
        const int i = column / group, qh = head * group + column - i * group;
        const int64_t row = tile.start + i;
        const int64_t pair = row * a.q_heads + qh;
        if (quarter == 0) {
            if (!whole) {
                float* ml = A.part_ml + (static_cast<int64_t>(blockIdx.y) * b.rows * a.q_heads + pair) * 2;
                ml[0] = most;
                ml[1] = all;
            } else if (a.lse) {
                a.lse[pair] = none ? -INFINITY : (most + __builtin_amdgcn_logf(all)) * kLn2;
            }
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const f32x4_t v = o[c][d];
            const int at_d = 16 * d + 4 * quarter;
            if (whole) {
                const u32x2_t r = {kv_pack2(none ? 0.f : v[0] * norm, none ? 0.f : v[1] * norm), kv_pack2(none ? 0.f : v[2] * norm, none ? 0.f : v[3] * norm)};
                *reinterpret_cast<u32x2_t*>(a.out + row * a.out_stride + static_cast<int64_t>(qh) * D + at_d) = r;
            } else if (!none) {
                *reinterpret_cast<f32x4_t*>(A.part_o + (static_cast<int64_t>(blockIdx.y) * b.rows * a.q_heads + pair) * D + at_d) = v;
            }
        }
    }
}

template <int D>
__device__ __forceinline__ void join_store(const AttentionArgs& a, int64_t pair, int64_t row, int d, f32x4_t sum, float all, float most) {
    const bool none = all == 0.f;
    const float norm = none ? 0.f : 1.f / all;
    const u32x2_t r = {kv_pack2(sum[0] * norm, sum[1] * norm), kv_pack2(sum[2] * norm, sum[3] * norm)};     // (nothing seen: every sum is zero)
    *reinterpret_cast<u32x2_t*>(a.out + row * a.out_stride + (pair - row * a.q_heads) * D + 4 * d) = r;
    if (a.lse && d == 0) a.lse[pair] = none ? -INFINITY : (most + __builtin_amdgcn_logf(all)) * kLn2;
}

// The parts of a (row, query head) pair joined, a workgroup a pair: a thread a part for the weights, then D / 4 threads a part and
// several parts at once for the sums, which are added in a fixed order.  Parts without tokens (l is zero) have no sums and are passed over;
// every other one counts whatever its weight, since a NaN in l or in the sums stays one where the weight rounds to zero, or where
// a part has no maximum but the lowest number because all of its scores are NaN.
template <int D>
__global__ void __launch_bounds__(kAttnThreads) attn_join_kernel(AttnArgs A) {
    constexpr int kLanes = D / 4, kAtOnce = kAttnThreads / kLanes;
    __shared__ float weight[kAttnThreads], scratch[2][kAttnWaves];
    __shared__ f32x4_t sums[kAtOnce][kLanes];
    const AttentionArgs& a = A.a;
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kWave - 1), wave = tid / kWave;
    const int64_t pairs = a.batch.rows * a.q_heads, pair = blockIdx.x;
    const int64_t row = pair / a.q_heads;
    if (kv_find_row(a.batch, row).seq < 0) return;                 // rows of no sequence stay as they were
    float m = kLowest, l = 0.f;
    if (tid < A.splits) {
        const float* ml = A.part_ml + (tid * pairs + pair) * 2;
        m = ml[0];
        l = ml[1];
    }
    float most = m;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
    if (lane == 0) scratch[0][wave] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) most = fmaxf(most, scratch[0][w]);
    const float mine = __builtin_amdgcn_exp2f(m - most);
    weight[tid] = l == 0.f ? -1.f : mine;                          // (no weight is negative: nothing to add)
    float all = l == 0.f ? 0.f : l * mine;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) all += __shfl_xor(all, d);
    if (lane == 0) scratch[1][wave] = all;
    __syncthreads();
    all = 0.f;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) all += scratch[1][w];

    const int part = tid / kLanes, d = tid % kLanes;
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = part; s < A.splits; s += kAtOnce) {
        const float w = weight[s];
        if (w < 0.f) continue;
        const f32x4_t o = *reinterpret_cast<const f32x4_t*>(A.part_o + (s * pairs + pair) * D + 4 * d);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmaf(o[e], w, sum[e]);
    }
    sums[part][d] = sum;
    __syncthreads();
    if (part) return;
#pragma unroll
    for (int p = 1; p < kAtOnce; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += sums[p][d][e];
    join_store<D>(a, pair, row, d, sum, all, most);
}

// The same for few parts: D / 4 threads a pair, and each passes over all of them.
constexpr int kFewParts = 8;
template <int D>
__global__ void __launch_bounds__(kAttnThreads) attn_join_few_kernel(AttnArgs A) {
    constexpr int kLanes = D / 4;
    const AttentionArgs& a = A.a;
    const int64_t pairs = a.batch.rows * a.q_heads;
    const int64_t pair = static_cast<int64_t>(blockIdx.x) * (kAttnThreads / kLanes) + threadIdx.x / kLanes;
    const int d = static_cast<int>(threadIdx.x) % kLanes;
    const int row = static_cast<int>((pair < pairs ? pair : pairs - 1) / a.q_heads);
    bool mine = false;                                             // (a wave looks for a row together, so for its pairs' rows one after the other)
#pragma unroll
    for (int i = 0; i < kWave / kLanes; ++i) {
        const bool found = kv_find_row(a.batch, __builtin_amdgcn_readlane(row, i * kLanes)).seq >= 0;
        mine |= found && static_cast<int>(threadIdx.x) % kWave / kLanes == i;
    }
    if (!mine || pair >= pairs) return;
    float m[kFewParts], l[kFewParts], most = kLowest;
#pragma unroll
    for (int s = 0; s < kFewParts; ++s) {
        m[s] = kLowest;
        l[s] = 0.f;
        if (s < A.splits) {
            const float* ml = A.part_ml + (s * pairs + pair) * 2;
            m[s] = ml[0];
            l[s] = ml[1];
        }
        most = fmaxf(most, m[s]);
    }
    float all = 0.f;
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < kFewParts; ++s) {
        if (s >= A.splits || l[s] == 0.f) continue;
        const float w = __builtin_amdgcn_exp2f(m[s] - most);
        all += l[s] * w;
        const f32x4_t o = *reinterpret_cast<const f32x4_t*>(A.part_o + (s * pairs + pair) * D + 4 * d);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmaf(o[e], w, sum[e]);
    }
    join_store<D>(a, pair, row, d, sum, all, most);
}

static int64_t column_tiles(const KvBatchArgs& b, int group, int columns) {
    if (!b.row_starts) return b.rows * ((group + columns - 1) / columns);
    return kv_pieces(b.rows, b.sequences, columns, group, columns - 1);
}

template <int D> constexpr int kTileWaves = D == 64 ? 4 : 8;
template <int D> constexpr int kColumnTiles = D == 256 ? 1 : 2;        // of 16 columns a wave: what its registers hold
template <int D> constexpr int kTileColumns = kTileWaves<D> * 16 * kColumnTiles<D>;
static int tile_columns(int D) { return D == 64 ? kTileColumns<64> : D == 128 ? kTileColumns<128> : kTileColumns<256>; }

// Which kernel, and into how many parts the tokens go.  Both go by the structures' numbers alone, so that a captured call can be replayed with other
// lengths: columns a sequence are an average, and the table's width stands for the tokens.  What that costs, us (8 key heads, 32 query heads of
// 128 elements): one token after 200 in a table of 256 tokens 7.0, of 4096 10.5, of 131072 11.0 (96 parts, 95 of them empty); 16 tokens of 2000 in a
// table of 2048 17.9, of 131072 18.6; a piece of 2048 rows beside 15 single tokens, 8000 tokens each, 470, and one after the other 354 + 37.
// Turns of waves with two column tiles decode half as often, but leave half as many
// workgroups and fewer waves a unit: from 2048 tokens on, where there are more columns than one tile, at up to 128 elements.  The tiles
// decode a step once for all of their columns and are worth it where they are full and few.  Measured, us, one column tile / two / the
// tiles (8 key heads, 128 elements, 8000 tokens; of several sequences the first, the others down to half of its columns and tokens):
//     one sequence: 256 columns 38 / 31 / 33, 1600 columns 192 / 140 / 108, a prompt of 16384 columns 399 / 296 / 210
//     two: 160 columns 45 / 43 / 51, 256 columns 58 / 49 / 55, 320 columns 67 / 57 / 63, 2048 columns 291 / 211 / 195
//     four, 320 columns 102 / 85 / 106; eight: 192 columns 112 / 93 / 176, 256 columns 138 / 111 / 160, 384 columns 195 / 157 / 193,
//     512 columns 252 / 193 / 251, 640 columns - / 241 / 264
//     beyond the line: four, 1024 columns - / 195 / 191; eight, 1024 columns - / 347 / 353, 2048 columns - / 642 / 607
//     eight drafts of 8 tokens (32 columns) on 4000 tokens 28 / 25 / -; of 1000 tokens: four, 256 columns 26 / 27 / 28, eight, 64 elements, 256 columns 16 / 24 / 26
//     256 elements: one, 100 columns 48 / - / 33; two, 200 columns 94 / - / 70; four, 120 columns 102 / - / 97; eight, 256 columns 272 / - / 281,
//     512 columns 501 / - / 408
// The lines below were drawn at 128 elements and serve 256 too, where they are not the best: the first three of its points go to the turns of waves,
// though the tiles are faster there.
// Parts of the waves' turns: as many workgroups as the compute units hold at once (three a unit, two where the head or the tile is wide); more would
// begin when the first end (131071 tokens, 8 key heads: 96 parts 42, 192 parts 50).  But sequences of
// different lengths end at different times: where their parts are long, twice as many (16 x 32768 tokens, when it was tried: 6 parts 115, 12 parts 107).
// Parts of the tiles: a unit holds one workgroup (three at 64 elements), and what counts is how many turns of them there are and how long
// each is: turns * (steps of a part + 4 to begin with), and a step for a million elements of the parts' results, written and read.  One
// more workgroup than the units hold makes it two turns.  us at 8000 tokens and 8 key heads: one sequence of 1600 columns, 4 parts (224
// workgroups) 108, 5 (280) 149; of 4000 columns 1 / 2 / 4 parts 359 / 196 / 207; two of 2048 and 1536 columns 2 / 3 / 5 parts 195 / 230 /
// 223; 256 elements, 1500 columns 2 / 3 / 5 / 6 parts 219 / 282 / 192 / 237; 64 elements, 1600 columns 5 / 7 / 8 parts 81 / 65 / 79.
static int64_t tile_splits(const KvCacheArgs& c, const KvBatchArgs& b, int group, int64_t steps, int64_t most) {
    const int64_t columns = tile_columns(c.head_dim), at_once = 256 * (c.head_dim == 64 ? 3 : 1);
    int64_t tiles = (b.rows * group + columns - 1) / columns + b.sequences / 2;     // (half a tile of every sequence without columns)
    if (tiles > column_tiles(b, group, columns)) tiles = column_tiles(b, group, columns);
    const int64_t items = tiles * c.kv_heads;
    int64_t best = 1;
    double least = 0;
    for (int64_t parts = 1; parts <= most && (parts == 1 || items * parts <= 4 * at_once); ++parts) {
        const int64_t turns = (items * parts + at_once - 1) / at_once, own = (steps + parts - 1) / parts;
        const double cost = static_cast<double>(turns) * (own + 4) + (parts > 1 ? parts * static_cast<double>(b.rows) * group * c.kv_heads * c.head_dim * 1e-6 : 0);
        if (parts == 1 || cost < least) {
            least = cost;
            best = parts;
        }
    }
    return best;
}

AttentionPlan attention_plan(const KvCacheArgs& c, const KvBatchArgs& b, int q_heads) {
    const int group = q_heads / c.kv_heads;
    const int64_t columns = b.rows * group;
    const int64_t steps = static_cast<int64_t>(b.table_width) * (c.page_size / kKvStep);
    const bool longer = c.head_dim <= 128 && steps >= 64;
    const bool two = longer && columns > static_cast<int64_t>(b.sequences) * kAttnColumns;
    const int least = (b.sequences == 1 ? 128 : b.sequences == 2 ? 256 : 384) * (longer ? 2 : 1);
    const bool wide = columns > static_cast<int64_t>(b.sequences) * least;
    AttentionPlan p{"kv_attention", kAttnColumns, 1, 0, 0};
    if (wide) p = {"kv_attention_tile", tile_columns(c.head_dim), 1, 0, 0};
    else if (two) p = {"kv_attention_two", 2 * kAttnColumns, 1, 0, 0};
    const int64_t items = p.workgroups = column_tiles(b, group, p.columns) * c.kv_heads;
    int64_t most = (steps + kAttnMinSteps - 1) / kAttnMinSteps;
    if (most > kAttnThreads) most = kAttnThreads;                  // (the joining kernel has a thread a part)
    int64_t splits;
    if (wide) {
        splits = tile_splits(c, b, group, steps, most);
    } else {
        const int64_t at_once = 256 * (c.head_dim == 256 || two ? 2 : 3);
        splits = (at_once + items - 1) / (items > 0 ? items : 1);
        if (b.sequences > 1 && steps >= 96 * splits) splits *= 2;
        if (splits > most) splits = most;
    }
    if (b.rows * q_heads * (c.head_dim / 4) > (int64_t(1) << 32) - kAttnThreads) splits = 1;     // (the joining launch's threads are counted in 32 bits)
    if (splits > 1) {
        p.splits = static_cast<int>(splits);
        p.workspace_bytes = static_cast<size_t>(splits) * b.rows * q_heads * (c.head_dim + 2) * sizeof(float);
    }
    return p;
}

template <int D>
static hipError_t launch_attn(const AttnArgs& A, const AttentionPlan& p, hipStream_t s) {
    const KvBatchArgs& b = A.a.batch;
    const dim3 grid(static_cast<unsigned>(p.workgroups), static_cast<unsigned>(A.splits));
    if (p.columns == kAttnColumns) {
        attn_kernel<D, 1><<<grid, kAttnThreads, 0, s>>>(A);
    } else if (p.columns == 2 * kAttnColumns) {
        if constexpr (D <= 128) attn_kernel<D, 2><<<grid, kAttnThreads, 0, s>>>(A);
    }
    else attn_tile_kernel<D, kColumnTiles<D>, kTileWaves<D>><<<grid, kTileWaves<D> * kWave, 0, s>>>(A);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || A.splits == 1) return e;
    const int64_t pairs = b.rows * A.a.q_heads, at_once = kAttnThreads / (D / 4);
    if (A.splits <= kFewParts) attn_join_few_kernel<D><<<dim3(static_cast<unsigned>((pairs + at_once - 1) / at_once)), kAttnThreads, 0, s>>>(A);
    else attn_join_kernel<D><<<dim3(static_cast<unsigned>(pairs)), kAttnThreads, 0, s>>>(A);
    return hipGetLastError();
}

hipError_t launch_attention(const AttentionArgs& a, hipStream_t s) {
    if (a.batch.rows == 0) return hipSuccess;
    const AttentionPlan p = attention_plan(a.cache, a.batch, a.q_heads);
    AttnArgs A{a, p.splits, static_cast<float*>(a.workspace), nullptr};
    if (p.splits > 1) A.part_ml = A.part_o + static_cast<int64_t>(p.splits) * a.batch.rows * a.q_heads * a.cache.head_dim;
    switch (a.cache.head_dim) {
        case 64: return launch_attn<64>(A, p, s);
        case 128: return launch_attn<128>(A, p, s);
        default: return launch_attn<256>(A, p, s);
    }
}

}  // namespace kmq
