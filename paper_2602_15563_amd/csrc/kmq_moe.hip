// Experts of a mixture of experts for a few tokens, weights in the block-scaled format on the tiled layout:
//
//     h_p = silu(G_e x) * (U_e x),   y = residual + sum_j gate_j * D_e h_p            pair p = (token, j), e = its expert
//
// Every expert that some token chose is read once.  Both kernels build the list of these experts from the choices themselves (so the
// launches do not depend on them, and a captured call may be replayed with others) and gather the tokens of an expert as the
// columns of matrix steps: v_mfma_f32_16x16x32_bf16 with the tokens first, so that what belongs to a row of the
// matrix (its scales) is needed by the lane that holds it.  Columns do not mix: what one token holds reaches no other.
//   gate_up   a workgroup takes 16 rows of both matrices of an expert at a time; its waves split the row, their sums are added in
//             shared memory, and SwiGLU of the two goes to the workspace, a row a pair, rounded to bf16;
//   down      a workgroup owns 16 rows of the output for all experts; its waves share the experts' super-blocks evenly, each
//             adds what it has of an expert, times the pair's weight, to its own sums in shared memory; these are added in the waves' order.
// Block scales: two matrix steps are a block of 64 columns; their sum from zero is multiplied by the block's scale.
#include <type_traits>

#include "kmq_kv.h"
#include "kmq_mfma_any.h"

namespace kmq {

namespace {

// Bundles a wave has asked for, by their registers.
#ifndef KMQ_RING
#define KMQ_RING 60
#endif
constexpr int depth(int words) { return words * 4 <= KMQ_RING ? 4 : words * 3 <= KMQ_RING ? 3 : 2; }
// Waves a SIMD that the registers have to leave room for: as many as an instance needs no spilling for.
constexpr int gate_up_waves(int bits, int t) { return t > 16 ? 2 : t == 16 && bits <= 2 ? 3 : t == 8 && bits == 1 ? 3 : 4; }
constexpr int down_waves(int bits, int t) { return t > 16 ? bits == 2 ? 2 : 3 : 4; }

typedef __amdgpu_buffer_rsrc_t Rows;
// Rows read by byte offset; kNoRow gives zeros.
constexpr uint32_t kNoRow = 0x80000000u;
__device__ __forceinline__ Rows rows_at(const void* p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7FFFFFFF, 0x00027000); }
__device__ __forceinline__ u32x4_t load_row16(Rows r, uint32_t lane_offset, uint32_t offset) {
    return __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, lane_offset, offset, 0));
}

template <int BITS> struct Granule {
    static constexpr int STEPS = BITS == 1 ? 16 : BITS == 2 ? 8 : 4;      // matrix steps of 32 columns
    static constexpr int WORDS = STEPS * BITS / 4, COLUMNS = 32 * STEPS, BLOCKS = STEPS / 2;
    uint32_t w[WORDS];
    uint32_t scale[BLOCKS / 2];                           // of the lane's row, two a word
};

// 16 rows of one expert's matrix from some unit (super-block) on, as a lane sees them: granules, and the scales of its row.
// (Rows come in whole blocks: their number is a multiple of 128.)
struct Matrix {
    const uint32_t* words;                                // the same in all lanes
    const uint16_t* scales;
};
template <int BITS>
__device__ __forceinline__ Matrix matrix_of(const MoeMatrix& m, int expert, int block, int units, int unit) {
    using G = Granule<BITS>;
    const int64_t at = expert * (m.rows >> 4) + block;
    return {m.words + (at * units + unit) * (64 * G::WORDS), m.scales + (at * 16 * units + unit) * G::BLOCKS};
}
template <int BITS>
__device__ __forceinline__ void load_granule(const Matrix& m, int units, int unit, int lane, Granule<BITS>& g) {
    using G = Granule<BITS>;
    const uint32_t* p = m.words + unit * (64 * G::WORDS) + lane * G::WORDS;
    if constexpr (G::WORDS == 3) {
        typedef u32x3_t __attribute__((aligned(4))) u32x3_a4_t;
        const u32x3_t t = __builtin_nontemporal_load(reinterpret_cast<const u32x3_a4_t*>(p));
        g.w[0] = t[0]; g.w[1] = t[1]; g.w[2] = t[2];
    } else {
        const u32x4_t t = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
        g.w[0] = t[0]; g.w[1] = t[1]; g.w[2] = t[2]; g.w[3] = t[3];
    }
    const uint16_t* s = m.scales + unit * G::BLOCKS + (lane & 15) * (units * G::BLOCKS);
    if constexpr (BITS >= 3) {
        g.scale[0] = *reinterpret_cast<const uint32_t*>(s);
    } else if constexpr (BITS == 2) {
        const u32x2_t t = *reinterpret_cast<const u32x2_t*>(s);
        g.scale[0] = t[0]; g.scale[1] = t[1];
    } else {
        const u32x4_t t = *reinterpret_cast<const u32x4_t*>(s);
        g.scale[0] = t[0]; g.scale[1] = t[1]; g.scale[2] = t[2]; g.scale[3] = t[3];
    }
}

// An expert's centroids, ready to be looked up: 1 bit both in registers, 2 and 3 bits their bytes as v_perm_b32 pools, 4 bits a table
// [centroid][lane] in shared memory (a lane reads its own bank), the centroid in both halves.
template <int BITS> struct Centroids {
    uint32_t a, b, c, d;
};
typedef uint32_t Table[16][64];
template <int BITS>
__device__ __forceinline__ Centroids<BITS> centroids_of(const uint16_t* book) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(book);
    Centroids<BITS> c = {0, 0, 0, 0};
    if constexpr (BITS == 1) {
        c.a = __builtin_amdgcn_perm(w[0], w[0], 0x01000100u);
        c.b = __builtin_amdgcn_perm(w[0], w[0], 0x03020302u);
    } else if constexpr (BITS <= 3) {
        c.a = __builtin_amdgcn_perm(w[1], w[0], 0x06040200u);
        c.c = __builtin_amdgcn_perm(w[1], w[0], 0x07050301u);
        c.b = c.a;
        c.d = c.c;
        if constexpr (BITS == 3) {
            c.b = __builtin_amdgcn_perm(w[3], w[2], 0x06040200u);
            c.d = __builtin_amdgcn_perm(w[3], w[2], 0x07050301u);
        }
    }
    return c;
}
// Pairs of entries first, first + step, .. of a 4-bit table.
__device__ __forceinline__ void fill_table(Table& table, const uint16_t* book, int first, int step, int lane) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(book);
    for (int e = first; e < 8; e += step) {
        const uint32_t two = w[e];
        table[2 * e][lane] = __builtin_amdgcn_perm(two, two, 0x01000100u);
        table[2 * e + 1][lane] = __builtin_amdgcn_perm(two, two, 0x03020302u);
    }
}

// Eight weights of step j.  4 bits: `at` are look-up addresses, byte 0 = lane * 4; byte 1 is the index, with `which` above it (the number of
// the table behind the one at `table`, in all bytes' upper halves).
struct LookUp {
    uint32_t at[8];
    uint32_t which;
};
template <int BITS>
__device__ __forceinline__ u32x4_t decode(const Granule<BITS>& g, const Centroids<BITS>& c, LookUp& l, uint32_t table, const u32x2_t* masks, int j) {
    if constexpr (BITS == 1) {
        const uint32_t b = g.w[j >> 2] >> (8 * (j & 3));
        const u32x2_t lo = masks[b & 15u], hi = masks[(b >> 4) & 15u];
        const auto choose = [&](uint32_t m) { return (m & c.b) | (~m & c.a); };
        return u32x4_t{choose(lo[0]), choose(lo[1]), choose(hi[0]), choose(hi[1])};
    } else if constexpr (BITS <= 3) {
        u32x4_t a;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t sel;
            if constexpr (BITS == 2) {
                const int i = 2 * j + h;
                sel = (g.w[i >> 2] >> (2 * (i & 3))) & 0x03030303u;
            } else {
                if (j < 3) sel = (h == 0 ? g.w[j] : g.w[j] >> 3) & 0x07070707u;
                else if (h == 0) sel = ((g.w[0] >> 6) & 0x03030303u) | ((g.w[1] >> 4) & 0x04040404u);
                else sel = ((g.w[1] >> 7) & 0x01010101u) | ((g.w[2] >> 5) & 0x06060606u);
            }
            const uint32_t lo = __builtin_amdgcn_perm(c.b, c.a, sel), hi = __builtin_amdgcn_perm(c.d, c.c, sel);
            a[2 * h] = __builtin_amdgcn_perm(hi, lo, 0x05010400u);
            a[2 * h + 1] = __builtin_amdgcn_perm(hi, lo, 0x07030602u);
        }
        return a;
    } else {
        const uint32_t even = (g.w[j] & 0x0F0F0F0Fu) | l.which, odd = ((g.w[j] >> 4) & 0x0F0F0F0Fu) | l.which;
        uint32_t v[8];
        const auto look = [&](auto bc) {
            constexpr int b = decltype(bc)::value;
            canon_index_to_byte1<b>(l.at[2 * b], even, 0xFFu);
            v[2 * b] = *reinterpret_cast<clds_cu32_t*>(static_cast<size_t>(l.at[2 * b] + table));
            canon_index_to_byte1<b>(l.at[2 * b + 1], odd, 0xFFu);
            v[2 * b + 1] = *reinterpret_cast<clds_cu32_t*>(static_cast<size_t>(l.at[2 * b + 1] + table));
        };
        look(std::integral_constant<int, 0>{});
        look(std::integral_constant<int, 1>{});
        look(std::integral_constant<int, 2>{});
        look(std::integral_constant<int, 3>{});
        return u32x4_t{__builtin_amdgcn_perm(v[1], v[0], 0x07060100u), __builtin_amdgcn_perm(v[3], v[2], 0x07060100u),
                       __builtin_amdgcn_perm(v[5], v[4], 0x07060100u), __builtin_amdgcn_perm(v[7], v[6], 0x07060100u)};
    }
}

__device__ __forceinline__ f32x4_t step(u32x4_t tokens, u32x4_t weights, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, tokens), __builtin_bit_cast(bf16x8_t, weights), c, 0, 0, 0);
}

// Which experts were chosen: a bit each, in shared memory; the pairs' ids as they are, their experts (-1: none, or an earlier pair of the
// token has the same) and, where they are asked for, their weights: of all the token's pairs with that expert.
template <int ROWS, bool WEIGHTS>
struct Choices {
    static constexpr int PAIRS = ROWS * KMQ_MOE_MAX_TOP_K;
    uint32_t has[KMQ_MOE_MAX_EXPERTS / 32];
    int16_t id[PAIRS + KMQ_MOE_MAX_TOP_K], expert[PAIRS];
    float gate[WEIGHTS ? PAIRS + KMQ_MOE_MAX_TOP_K : 1], weight[WEIGHTS ? PAIRS : 1];
};
// What a lane knows of them: its 32 experts' bits, and how many experts were chosen up to them.
struct Chosen {
    uint32_t mine;
    int upto, all;
    // The a-th chosen expert.
    __device__ __forceinline__ int expert(int a) const {
        const int word = __ffsll(__ballot(upto > a)) - 1;
        uint32_t bits = __builtin_amdgcn_readlane(mine, word);
        for (int skip = a - (__builtin_amdgcn_readlane(upto, word) - __popc(bits)); skip > 0; --skip) bits &= bits - 1;
        return __builtin_amdgcn_readfirstlane(word * 32 + __ffs(bits) - 1);
    }
};
template <int ROWS, bool WEIGHTS>
__device__ __forceinline__ Chosen find_choices(const MoeArgs& a, Choices<ROWS, WEIGHTS>& p) {
    static_assert(KMQ_MOE_MAX_EXPERTS / 32 <= kWave, "a word a lane");
    const int pairs = a.rows * a.top_k, tid = threadIdx.x, lane = tid & 63;
    for (int i = tid; i < pairs; i += blockDim.x) {
        const int e = a.ids[i];
        p.id[i] = static_cast<int16_t>(e >= 0 && e < a.experts ? e : -1);
        if constexpr (WEIGHTS) p.gate[i] = a.gates[i];
    }
    if (tid < KMQ_MOE_MAX_EXPERTS / 32) p.has[tid] = 0;
    __syncthreads();
    for (int i = tid; i < pairs; i += blockDim.x) {
        const int e = p.id[i], slot = i % a.top_k, first = i - slot;
        bool counts = e >= 0;
        [[maybe_unused]] float w = 0.f;
#pragma unroll
        for (int j = 0; j < KMQ_MOE_MAX_TOP_K; ++j) {     // (behind the last pair there is room for reading on)
            const bool same = j < a.top_k && p.id[first + j] == e;
            counts = counts && !(same && j < slot);
            if constexpr (WEIGHTS) w += same ? p.gate[first + j] : 0.f;
        }
        p.expert[i] = static_cast<int16_t>(counts ? e : -1);
        if constexpr (WEIGHTS) p.weight[i] = w;
        if (counts) atomicOr(&p.has[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
    Chosen c;
    c.mine = lane < KMQ_MOE_MAX_EXPERTS / 32 ? p.has[lane] : 0u;
    c.upto = __popc(c.mine);
    for (int d = 1; d < KMQ_MOE_MAX_EXPERTS / 32; d *= 2) {
        const int o = __shfl_up(c.upto, d);
        if (lane >= d) c.upto += o;
    }
    c.all = __builtin_amdgcn_readlane(c.upto, KMQ_MOE_MAX_EXPERTS / 32 - 1);
    return c;
}

// The pairs of an expert, into `list` (this wave's own): token << 16 | pair.  How many.
template <int ROWS, bool WEIGHTS>
__device__ __forceinline__ int pairs_of(const Choices<ROWS, WEIGHTS>& p, int pairs, int top_k, int expert, uint32_t* list) {
    const int lane = threadIdx.x & 63;
    int count = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int i = lane; i < (pairs + 63) / 64 * 64; i += 64) {
        const bool mine = i < pairs && p.expert[i] == expert;
        const uint64_t all = __ballot(mine);
        if (mine) list[count + __popcll(all & ((uint64_t(1) << lane) - 1))] = static_cast<uint32_t>(i / top_k) << 16 | static_cast<uint32_t>(i);
        count += __popcll(all);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return __builtin_amdgcn_readfirstlane(count);
}

__device__ __forceinline__ void fill_masks(u32x2_t (&masks)[16]) {
    if (threadIdx.x < 16) {
        const uint32_t e = threadIdx.x;
        masks[e] = u32x2_t{((e & 1u) ? 0xFFFFu : 0u) | ((e & 2u) ? 0xFFFF0000u : 0u), ((e & 4u) ? 0xFFFFu : 0u) | ((e & 8u) ? 0xFFFF0000u : 0u)};
    }
}

// What a wave asks for at a time: a super-block of N matrices, and the elements under it of T tokens of the expert.  Fewer than 16 tokens
// leave most lanes of the operand without one, so 16 / T steps' operands come with one load: lane n takes token n % T at step n / T, and a
// rotation inside 16 lanes brings it to where the step wants it.  (What the other lanes hold then are columns that nobody reads.)
// T = 16 at 1 bit would take 64 registers: there the elements are read when they are needed.
template <int BITS, int T, int N>
struct Bundle {
    static constexpr int TILES = T > 16 ? T / 16 : 1, LOADS = T > 16 ? 4 : T / 4;      // column tiles; loads a tile and four steps
    static constexpr bool TOKENS = BITS > 1 || T < 16;
    static constexpr int WORDS = N * (Granule<BITS>::WORDS + Granule<BITS>::BLOCKS / 2) + (TOKENS ? TILES * LOADS * Granule<BITS>::STEPS : 0);
    Granule<BITS> g[N];
    u32x4_t x[TILES][TOKENS ? Granule<BITS>::STEPS / 4 : 1][LOADS];
};
template <int T>
struct Tokens {
    static constexpr int TILES = T > 16 ? T / 16 : 1;
    Rows rows;
    uint32_t at[TILES];                                   // the lane's token of every column tile
};
template <int T>
__device__ __forceinline__ void load_tokens(const Tokens<T>& tokens, int tile, uint32_t column, u32x4_t (&x)[T > 16 ? 4 : T / 4]) {
#pragma unroll
    for (int l = 0; l < (T > 16 ? 4 : T / 4); ++l) x[l] = load_row16(tokens.rows, tokens.at[tile] + l * (T < 16 ? 1024 / T : 64), column * 2);
}
template <int BITS, int T, int N>
__device__ __forceinline__ void load_bundle(const Matrix (&m)[N], int units, int unit, const Tokens<T>& tokens, int first_column, int lane, Bundle<BITS, T, N>& b) {
    using G = Granule<BITS>;
    using B = Bundle<BITS, T, N>;
#pragma unroll
    for (int i = 0; i < N; ++i) load_granule<BITS>(m[i], units, unit, lane, b.g[i]);
    if constexpr (B::TOKENS) {
#pragma unroll
        for (int t = 0; t < B::TILES; ++t)
#pragma unroll
            for (int k = 0; k < G::STEPS / 4; ++k) load_tokens<T>(tokens, t, first_column + unit * G::COLUMNS + 128 * k, b.x[t][k]);
    }
}
// The operand of step j of four.
template <int T>
__device__ __forceinline__ u32x4_t operand(const u32x4_t (&x)[T > 16 ? 4 : T / 4], int j) {
    if constexpr (T >= 16) return x[j];
    u32x4_t v;
    const auto turn = [&](auto ctrl) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x[j * T / 16][i]), decltype(ctrl)::value, 0xF, 0xF, true));
        return v;
    };
    switch (j % (16 / T) * T) {                           // row_ror: lane i takes what lane i + 4, 8, 12 (of 16) has
        case 4: return turn(std::integral_constant<int, 0x12C>{});
        case 8: return turn(std::integral_constant<int, 0x128>{});
        case 12: return turn(std::integral_constant<int, 0x124>{});
        default: return x[j * T / 16];
    }
}
template <int BITS, int T, int N>
__device__ __forceinline__ void multiply_bundle(const Bundle<BITS, T, N>& b, const Centroids<BITS> (&c)[N], LookUp& l, uint32_t tables, const u32x2_t* masks,
                                                const Tokens<T>& tokens, int column, f32x4_t (&acc)[N][Tokens<T>::TILES]) {
    using G = Granule<BITS>;
    using B = Bundle<BITS, T, N>;
#pragma unroll
    for (int k = 0; k < G::STEPS / 4; ++k) {
        u32x4_t x[B::TILES][B::LOADS];
#pragma unroll
        for (int t = 0; t < B::TILES; ++t) {
            if constexpr (B::TOKENS) {
#pragma unroll
                for (int i = 0; i < B::LOADS; ++i) x[t][i] = b.x[t][k][i];
            } else {
                load_tokens<T>(tokens, t, column + 128 * k, x[t]);
            }
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int block = 2 * k + half;
            u32x4_t x0[B::TILES], x1[B::TILES];
#pragma unroll
            for (int t = 0; t < B::TILES; ++t) {
                x0[t] = operand<T>(x[t], 2 * half);
                x1[t] = operand<T>(x[t], 2 * half + 1);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const u32x4_t w0 = decode<BITS>(b.g[i], c[i], l, tables + i * sizeof(Table), masks, 2 * block), w1 = decode<BITS>(b.g[i], c[i], l, tables + i * sizeof(Table), masks, 2 * block + 1);
                const float s = kv_half(b.g[i].scale[block / 2], block % 2);
#pragma unroll
                for (int t = 0; t < B::TILES; ++t) {
                    f32x4_t d = step(x0[t], w0, f32x4_t{0.f, 0.f, 0.f, 0.f});
                    d = step(x1[t], w1, d);
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][t][r] = fmaf(s, d[r], acc[i][t][r]);
                }
            }
        }
        if constexpr (!B::TOKENS) __builtin_amdgcn_sched_barrier(0);      // (else the elements of all steps are asked for at once, and spilled)
    }
}
// The sums over `count` super-blocks; the first D bundles have been asked for.  The loop's loads are unconditional, the last
// super-blocks a copy of the code of their own: a branch around a load would make every wait assume the fewest of them.
template <int BITS, int T, int N, int D>
__device__ __forceinline__ void run_units(Bundle<BITS, T, N> (&b)[D], const Matrix (&m)[N], int units, int count, const Centroids<BITS> (&c)[N], LookUp& l, uint32_t tables,
                                          const u32x2_t* masks, const Tokens<T>& tokens, int first_column, int lane, f32x4_t (&acc)[N][Tokens<T>::TILES]) {
    constexpr int COLUMNS = Granule<BITS>::COLUMNS;
    int u = 0;
    const auto multiply_at = [&](int slot, int unit) { multiply_bundle<BITS, T, N>(b[slot], c, l, tables, masks, tokens, first_column + unit * COLUMNS, acc); };
    for (; u + 2 * D <= count; u += D) {
#pragma unroll
        for (int p = 0; p < D; ++p) {
            multiply_at(p, u + p);
            load_bundle<BITS, T, N>(m, units, u + p + D, tokens, first_column, lane, b[p]);
        }
    }
#pragma unroll
    for (int p = 0; p < D; ++p) {
        if (u + p >= count) return;
        multiply_at(p, u + p);
        if (u + p + D < count) load_bundle<BITS, T, N>(m, units, u + p + D, tokens, first_column, lane, b[p]);
    }
#pragma unroll
    for (int p = 0; p < D - 1; ++p) {
        if (u + D + p >= count) return;
        multiply_at(p, u + D + p);
    }
}
template <int BITS, int T, int N, int D>
__device__ __forceinline__ void first_bundles(Bundle<BITS, T, N> (&b)[D], const Matrix (&m)[N], int units, int count, const Tokens<T>& tokens, int first_column, int lane) {
#pragma unroll
    for (int p = 0; p < D; ++p)
        if (p < count) load_bundle<BITS, T, N>(m, units, p, tokens, first_column, lane, b[p]);
}
// Where the lane's tokens begin, of those from `first` on in the list: rows of `stride` bytes; PAIR: a row a pair, else a row a token.
template <int T, bool PAIR>
__device__ __forceinline__ void find_tokens(Tokens<T>& tokens, const uint32_t* list, int first, int count, uint32_t stride, int lane) {
    const int n = lane & 15, q = lane >> 4;
#pragma unroll
    for (int t = 0; t < Tokens<T>::TILES; ++t) {
        const int i = first + 16 * t + (T < 16 ? n % T : n);
        tokens.at[t] = kNoRow;
        if (i < count) tokens.at[t] = (PAIR ? list[i] & 0xFFFFu : list[i] >> 16) * stride + 16u * q + (T < 16 ? n / T * 64u : 0u);
    }
}
__device__ __forceinline__ uint32_t shared_offset(const void* p) { return static_cast<uint32_t>(reinterpret_cast<size_t>((clds_cu32_t*)(p))); }
__device__ __forceinline__ LookUp look_up(uint32_t which, int lane) {
    LookUp l;
#pragma unroll
    for (int e = 0; e < 8; ++e) l.at[e] = static_cast<uint32_t>(lane) * 4u;
    l.which = which * 0x10101010u;
    return l;
}

template <int BITS, int T, int ROWS, int NW>
__global__ __launch_bounds__(NW * kWave) __attribute__((amdgpu_waves_per_eu(gate_up_waves(BITS, T)))) void moe_gate_up_kernel(MoeArgs a) {
    using G = Granule<BITS>;
    constexpr int TILES = Tokens<T>::TILES, D = depth(Bundle<BITS, T, 2>::WORDS);
    struct alignas(256) Smem {
        Table tables[BITS == 4 ? 2 : 1];
        Choices<ROWS, false> choices;
        float part[2][NW][2][16][17];
        uint32_t lists[NW][2][ROWS];
        u32x2_t masks[16];
    };
    __shared__ Smem sm;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    if constexpr (BITS == 1) fill_masks(sm.masks);
    const Chosen chosen = find_choices(a, sm.choices);
    const int blocks = static_cast<int>(a.width >> 4), units = static_cast<int>(a.hidden / G::COLUMNS), pairs = a.rows * a.top_k;
    const int u0 = units * wave / NW, mine = units * (wave + 1) / NW - u0, column = u0 * G::COLUMNS;
    const int64_t items = static_cast<int64_t>(chosen.all) * blocks;
    const int from = static_cast<int>(items * blockIdx.x / gridDim.x), to = static_cast<int>(items * (blockIdx.x + 1) / gridDim.x);
    if (from >= to) return;
    uint16_t* const h = static_cast<uint16_t*>(a.workspace);
    Tokens<T> tokens;
    tokens.rows = rows_at(a.x);
    Bundle<BITS, T, 2> b[D];
    Matrix m[2];
    Centroids<BITS> c[2] = {};
    LookUp l = look_up(0, lane);
    const uint32_t tables = shared_offset(&sm.tables[0]);
    // where the wave is: rows `block` of the `which`-th expert, its pairs first ..
    int which = from / blocks, block = from - which * blocks, e = chosen.expert(which), turn = 0;
    uint32_t* list = sm.lists[wave][0];
    int count = pairs_of(sm.choices, pairs, a.top_k, e, list), first = 0;
    const auto ask = [&] {
        m[0] = matrix_of<BITS>(a.gate, e, block, units, u0);
        m[1] = matrix_of<BITS>(a.up, e, block, units, u0);
        find_tokens<T, false>(tokens, list, first, count, static_cast<uint32_t>(a.x_stride * 2), lane);
        first_bundles<BITS, T, 2, D>(b, m, units, mine, tokens, column, lane);
    };
    const auto look_at = [&] {                            // an expert's centroids
        const uint16_t *bg = a.gate.books + (e << BITS), *bu = a.up.books + (e << BITS);
        c[0] = centroids_of<BITS>(bg);
        c[1] = centroids_of<BITS>(bu);
        if constexpr (BITS == 4) {
            fill_table(sm.tables[0], bg, wave, NW, lane);
            fill_table(sm.tables[1], bu, wave, NW, lane);
            __syncthreads();
        }
    };
    ask();
    look_at();
    for (int item = from;;) {
        f32x4_t acc[2][TILES];
#pragma unroll
        for (int t = 0; t < TILES; ++t) acc[0][t] = acc[1][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        run_units<BITS, T, 2, D>(b, m, units, mine, c, l, tables, sm.masks, tokens, column, lane, acc);
        // what comes next is asked for before the sums are joined
        const int left = count - first < T ? count - first : T, done = first, row = block * 16, last = e;
        const uint32_t* const now = list;
        bool more = true;
        if (first + T < count) {
            first += T;
        } else {
            first = 0;
            if (++item == to) more = false;
            else if (++block == blocks) {
                block = 0;
                e = chosen.expert(++which);
                list = sm.lists[wave][which & 1];
                if (list == now) list = sm.lists[wave][(which & 1) ^ 1];
                count = pairs_of(sm.choices, pairs, a.top_k, e, list);
            }
        }
        if (more) ask();
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            if (16 * t >= left) break;
            float (&part)[NW][2][16][17] = sm.part[turn];
            turn ^= 1;
            if (16 * t + 4 * q < left) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    part[wave][0][4 * q + i][n] = acc[0][t][i];
                    part[wave][1][4 * q + i][n] = acc[1][t][i];
                }
            }
            __syncthreads();
            const int column = threadIdx.x >> 4, r = threadIdx.x & 15;
            if (column < 16 && 16 * t + column < left) {
                float g = part[0][0][column][r], u = part[0][1][column][r];
#pragma unroll
                for (int w = 1; w < NW; ++w) {
                    g += part[w][0][column][r];
                    u += part[w][1][column][r];
                }
                h[(now[done + 16 * t + column] & 0xFFFFu) * a.width + row + r] = f32_to_bf16(g / (1.f + expf(-g)) * u);
            }
        }
        if (!more) break;
        if (e != last) look_at();
    }
}

template <int BITS, int T, int ROWS, int NW>
__global__ __launch_bounds__(NW * kWave) __attribute__((amdgpu_waves_per_eu(down_waves(BITS, T)))) void moe_down_kernel(MoeArgs a) {
    using G = Granule<BITS>;
    constexpr int TILES = Tokens<T>::TILES, D = depth(Bundle<BITS, T, 1>::WORDS);
    struct alignas(256) Smem {
        Table tables[BITS == 4 ? NW : 1];
        Choices<ROWS, true> choices;
        uint32_t lists[NW][2][ROWS];
        u32x2_t masks[16];
    };
    __shared__ Smem sm;
    extern __shared__ float sums[];                       // [wave][token][16 rows]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    if constexpr (BITS == 1) fill_masks(sm.masks);
    for (int i = threadIdx.x; i < NW * a.rows * 16; i += NW * kWave) sums[i] = 0.f;
    const Chosen chosen = find_choices(a, sm.choices);
    const int block = blockIdx.x, units = static_cast<int>(a.width / G::COLUMNS), pairs = a.rows * a.top_k;
    const int64_t all = static_cast<int64_t>(chosen.all) * units;
    const int from = static_cast<int>(all * wave / NW), to = static_cast<int>(all * (wave + 1) / NW);
    float* const mine = sums + wave * a.rows * 16;
    if (from < to) {
        Tokens<T> tokens;
        tokens.rows = rows_at(a.workspace);
        Bundle<BITS, T, 1> b[D];
        Matrix m[1];
        Centroids<BITS> c[1];
        LookUp l = look_up(wave, lane);
        const uint32_t tables = shared_offset(&sm.tables[0]);
        int which = from / units, u0 = from - which * units, some = units < u0 + to - from ? units - u0 : to - from, done = from + some;
        int e = chosen.expert(which), first = 0;
        uint32_t* list = sm.lists[wave][0];
        int count = pairs_of(sm.choices, pairs, a.top_k, e, list);
        const auto ask = [&] {
            m[0] = matrix_of<BITS>(a.down, e, block, units, u0);
            find_tokens<T, true>(tokens, list, first, count, static_cast<uint32_t>(a.width * 2), lane);
            first_bundles<BITS, T, 1, D>(b, m, units, some, tokens, u0 * G::COLUMNS, lane);
        };
        const auto look_at = [&] {
            const uint16_t* book = a.down.books + (e << BITS);
            c[0] = centroids_of<BITS>(book);
            if constexpr (BITS == 4) {
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                fill_table(sm.tables[wave], book, 0, 1, lane);
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
        };
        ask();
        look_at();
        for (;;) {
            f32x4_t acc[1][TILES];
#pragma unroll
            for (int t = 0; t < TILES; ++t) acc[0][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            run_units<BITS, T, 1, D>(b, m, units, some, c, l, tables, sm.masks, tokens, u0 * G::COLUMNS, lane, acc);
            const int start = first, had = count < first + T ? count : first + T, last = e;
            const uint32_t* const now = list;
            bool more = true;
            if (first + T < count) {
                first += T;
            } else {
                first = 0;
                if (done == to) more = false;
                else {
                    ++which;
                    u0 = 0;
                    some = units < to - done ? units : to - done;
                    done += some;
                    e = chosen.expert(which);
                    list = now == sm.lists[wave][0] ? sm.lists[wave][1] : sm.lists[wave][0];
                    count = pairs_of(sm.choices, pairs, a.top_k, e, list);
                }
            }
            if (more) ask();
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = start + 16 * t + 4 * q + i;
                    if (at < had) {
                        const uint32_t p = now[at];
                        float* s = mine + (p >> 16) * 16 + n;
                        *s = fmaf(sm.choices.weight[p & 0xFFFFu], acc[0][t][i], *s);
                    }
                }
            if (!more) break;
            if (e != last) look_at();
        }
    }
    __syncthreads();
    for (int o = threadIdx.x; o < a.rows * 16; o += NW * kWave) {
        const int64_t token = o >> 4, row = static_cast<int64_t>(block) * 16 + (o & 15);
        float s = a.residual ? bf16_to_f32(a.residual[token * a.residual_stride + row]) : 0.f;
        for (int w = 0; w < NW; ++w) s += sums[w * a.rows * 16 + o];
        a.y[token * a.y_stride + row] = f32_to_bf16(s);
    }
}

}  // namespace

size_t moe_workspace_bytes(int64_t rows, int64_t top_k, int64_t width) { return static_cast<size_t>(rows * top_k * width * 2); }

#ifndef KMQ_NWG
#define KMQ_NWG 4
#define KMQ_GRID 1024
#endif
template <int BITS, int T, int ROWS, int NWD>
static void launch_moe_one(const MoeArgs& a, hipStream_t s) {
    const int64_t pairs = static_cast<int64_t>(a.rows) * a.top_k, most = (pairs < a.experts ? pairs : a.experts) * (a.width / 16);
    moe_gate_up_kernel<BITS, T, ROWS, KMQ_NWG><<<dim3(static_cast<unsigned>(most < KMQ_GRID ? most : KMQ_GRID)), KMQ_NWG * kWave, 0, s>>>(a);
    moe_down_kernel<BITS, T, ROWS, NWD><<<dim3(static_cast<unsigned>(a.hidden / 16)), NWD * kWave, NWD * a.rows * 16 * sizeof(float), s>>>(a);
}
#ifndef KMQ_TM
#define KMQ_TM 32
#endif
template <int BITS>
static void launch_moe_bits(const MoeArgs& a, hipStream_t s) {
    const int64_t pairs = static_cast<int64_t>(a.rows) * a.top_k;
    const bool thin = pairs <= 2 * static_cast<int64_t>(a.experts);       // about two tokens an expert
    if (a.rows <= 4) launch_moe_one<BITS, 4, 16, 16>(a, s);
    else if (a.rows <= 8 || (a.rows <= 16 && thin)) launch_moe_one<BITS, 8, 16, 16>(a, s);
    else if (a.rows <= 16) launch_moe_one<BITS, 16, 16, 16>(a, s);
    else launch_moe_one<BITS, KMQ_TM, KMQ_MOE_MAX_ROWS, 8>(a, s);
}

hipError_t launch_moe(const MoeArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    switch (a.bits) {
        case 1: launch_moe_bits<1>(a, s); break;
        case 2: launch_moe_bits<2>(a, s); break;
        case 3: launch_moe_bits<3>(a, s); break;
        default: launch_moe_bits<4>(a, s); break;
    }
    return hipGetLastError();
}

}  // namespace kmq
