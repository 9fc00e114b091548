// Experts of a mixture of experts for a few tokens, weights in the block-scaled format on the tiled layout:
//
//     h_p = silu(G_e x) * (U_e x),   y = residual + sum_j gate_j * D_e h_p            pair p = (token, j), e = its expert
//
// An expert that some token chose is read once for every T (4, 8 or 16) of its tokens, the repeats mostly from the L2; the others are not
// read.  The kernels build the list of these experts from the choices themselves (so the launches do not depend on them, and a captured call
// may be replayed with others) and gather the tokens of an expert as the columns of matrix steps: v_mfma_f32_16x16x32_bf16 with the tokens
// first, so that what belongs to a row of the matrix (its scales) is needed by the lane that holds it.  Columns do not mix: what one token
// holds reaches no other.
//
// Three launches: the rows of G and U (SwiGLU of both goes to the workspace, a row a pair, rounded to bf16: the matrix instruction takes no
// more, and two parts of it would double the second product's steps; of an output without a residual the r.m.s. error is 0.0024 with it,
// 0.0017, the output's own rounding, without), the rows of D (a row a pair again, in fp32), and the sum of a token's pairs.  The first two
// are one kernel: a wave multiplies 16 rows of two matrices with the same tokens, the gate's and the up projection's, or two blocks of the
// down projection.  NW waves (a team) split the rows' length, their sums are added in shared memory; the teams of a workgroup share the
// table of the expert's centroids.  A workgroup takes neighbouring rows of the list of all experts' rows, as many as any other; the first
// super-blocks of what comes next are asked for before the sums are joined.  Above 16 rows the 16 tokens of an item stand in shared memory
// as operands, for all of the workgroup's waves.
//
// What bounds it: 4 bits, 16 tokens of 128 experts of 4096 x 1536, the memory (90 + 57 us, 4.9 TB/s); 2 bits, five tokens of 8 experts of 4096 x 14336, the decode
// (62 + 37 us, of which vector issue 32 + 15, look-ups as much); one token, 6 to 8 experts, latencies (15 + 10 us, 6 before the first products in each).
//
// Block scales: two matrix steps are a block of 64 columns; their sum from zero is multiplied by the block's scale.
//
// Decode: tables in shared memory whose entries are ready operand registers, a column a lane modulo 32, so that look-ups never collide
// whatever the indices are.  2 to 4 bits: a pair of indices (4, 6, 8 bits of a byte of the granule) is an entry of two centroids; at 2 and 3
// bits it is elements k and k + 4 of a step, and the tokens' elements are brought into that order.  1 bit: four indices, eight bytes.  The
// index goes into byte 1 of the address by one instruction.  (2 bits with four indices too, half the instructions for the same bytes: 109 us and 110, five tokens, 2 of 8
// experts of 4096 x 14336; what a token's sums cost behind the next item's barrier instead of ahead of it: no difference.)
#include <cstddef>
#include <type_traits>

#include "kmq_kv.h"
#include "kmq_mfma_any.h"

namespace kmq {

namespace {

// Bundles a wave has asked for, by their registers: what fits beside the rest.  (Three instead of two, 16 tokens, 8 of 128 experts of 4096 x 1536: 2 bits 132 ->
// 149 us, 4 bits 166 both; one token, 4 bits 30 -> 31.5.)  With tokens in shared memory two: sixteen waves a unit ask for enough (three, four: 128 tokens, 6 of 64
// experts of 2048 x 1408, 3 bits 100 -> 105, 105; 64 tokens of them, 4 bits 97 -> 101, 107).
constexpr int depth(int words) { return words <= 10 ? 3 : 2; }
// Waves a SIMD that the registers have to leave room for.  (1 bit, few tokens: what is kept over an item and does not fit, 5 to 7 words, is spilled outside the
// loop; two waves instead 113 -> 129 us, 16 tokens, 8 of 128 experts of 4096 x 1536.)
constexpr int waves_for(int bits, int t, bool staged) { return staged ? (bits == 1 ? 2 : 4) : (t == 16 && (bits == 2 || bits == 4)) ? 2 : bits == 1 || (bits == 2 && t == 8) || t == 16 ? 3 : 4; }

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
};

// 16 rows of one expert's matrix: granules, and the scales, two blocks a word.  The same in all lanes.
// (Rows come in whole blocks: their number is a multiple of 128.)
struct Matrix {
    const uint32_t* words;
    const uint32_t* scales;
};
template <int BITS>
__device__ __forceinline__ Matrix matrix_of(const MoeMatrix& m, int expert, int block, int units) {
    using G = Granule<BITS>;
    const int64_t at = (expert * (m.rows >> 4) + block) * units;
    return {m.words + at * (64 * G::WORDS), reinterpret_cast<const uint32_t*>(m.scales) + at * (16 * G::BLOCKS / 2)};
}
template <int BITS>
__device__ __forceinline__ void load_granule(const Matrix& m, int unit, int lane, Granule<BITS>& g) {
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
}

// A row's length goes by pieces of kPiece columns, whose scales a team keeps in shared memory, [matrix][row][word], rows an odd number of
// words apart.  They are asked for as they lie, row after row: granule by granule, 4 to 16 bytes of each of 16 rows an instruction, the same
// lines are asked for from the L2 again and again (a layer of 16 tokens, 128 experts of 4096 x 1536, 4 bits: 218 us, and 204).
template <int PIECE> using PieceScales = uint32_t[2][16 * (PIECE / 128 + 1)];
template <int PIECE, int LANES>
struct Scales {
    static constexpr int EACH = (16 * (PIECE / 128) + LANES - 1) / LANES;
    uint32_t raw[2][EACH];
    // Words first .. first + words - 1 of 16 rows of `row_words`; `lane` of the team's.
    __device__ __forceinline__ void load(const Matrix (&m)[2], int row_words, int first, int words, int lane) {
        const uint32_t inverse = 65536u / words + 1;      // (exact below 512 = 16 rows of 32 words)
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const uint32_t d = lane + k * LANES;
            if (k * LANES >= 16 * words) break;
            const uint32_t row = min(d * inverse >> 16, 15u), at = min(d - row * words, static_cast<uint32_t>(words - 1));
#pragma unroll
            for (int i = 0; i < 2; ++i) raw[i][k] = m[i].scales[row * row_words + first + at];
        }
    }
    __device__ __forceinline__ void keep(PieceScales<PIECE>& to, int words, int lane) const {
        const uint32_t inverse = 65536u / words + 1, odd = words | 1;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const uint32_t d = lane + k * LANES;
            if (k * LANES >= 16 * words) break;
            const uint32_t row = d * inverse >> 16;
            if (row < 16) {
#pragma unroll
                for (int i = 0; i < 2; ++i) to[i][row * odd + d - row * words] = raw[i][k];
            }
        }
    }
};

// The tables of two matrices' centroids: entries of 256 bytes, the first matrix's columns, then the second's; 1 bit: one after the other,
// columns of eight bytes.
template <int BITS> struct alignas(256) Tables {
    static constexpr int ENTRIES = BITS == 1 ? 32 : 1 << (2 * BITS);
    uint32_t word[ENTRIES][64];
};
// `centroids`: lane l < 16 holds the first matrix's l-th, lane 16 + l the second's.  Filled by all waves of a workgroup, 1 KB a write.
template <int BITS>
__device__ __forceinline__ void fill_tables(Tables<BITS>& tables, uint32_t centroids, int wave, int waves, int lane) {
    const auto centroid = [&](int matrix, int index) { return static_cast<uint32_t>(__shfl(static_cast<int>(centroids), matrix * 16 + index)); };
    for (int i = wave; i < Tables<BITS>::ENTRIES / 4; i += waves) {
        const int e = 4 * i + (lane >> 4);
        u32x4_t v;
        if constexpr (BITS == 1) {
            const uint32_t c0 = centroid(i >> 2, 0), c1 = centroid(i >> 2, 1);
            v[0] = v[2] = (e & 1 ? c1 : c0) | (e & 2 ? c1 : c0) << 16;
            v[1] = v[3] = (e & 4 ? c1 : c0) | (e & 8 ? c1 : c0) << 16;
        } else {
            const int matrix = (lane >> 3) & 1;
            v[0] = v[1] = v[2] = v[3] = centroid(matrix, e & ((1 << BITS) - 1)) | centroid(matrix, e >> BITS) << 16;
        }
        *reinterpret_cast<u32x4_t*>(&tables.word[e][4 * (lane & 15)]) = v;
    }
}

// Look-up addresses: byte 0 is the lane's column, byte 1 the entry.
template <int BITS>
struct LookUp {
    static constexpr int EACH = BITS == 1 ? 2 : 4;
    uint32_t at[2][EACH];
    uint32_t table;
    __device__ __forceinline__ LookUp(const Tables<BITS>& t, int lane) {
        table = static_cast<uint32_t>(reinterpret_cast<size_t>((clds_cu32_t*)(&t.word[0][0])));
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < EACH; ++i) at[m][i] = BITS == 1 ? (lane & 31) * 8u : m * 128u + (lane & 31) * 4u;
    }
};
typedef __attribute__((address_space(3))) const u32x2_t lds_u32x2_t;

// Eight weights of step j of one granule.
template <int BITS>
__device__ __forceinline__ u32x4_t decode(const Granule<BITS>& g, LookUp<BITS>& l, int m, int j) {
    u32x4_t v;
    if constexpr (BITS == 1) {
        const uint32_t even = g.w[j >> 2], odd = even >> 4, base = l.table + m * 4096u;
        const auto look = [&](auto bc) {
            constexpr int b = decltype(bc)::value;
            canon_index_to_byte1<b>(l.at[m][0], even, 0x0Fu);
            canon_index_to_byte1<b>(l.at[m][1], odd, 0x0Fu);
        };
        switch (j & 3) {
            case 0: look(std::integral_constant<int, 0>{}); break;
            case 1: look(std::integral_constant<int, 1>{}); break;
            case 2: look(std::integral_constant<int, 2>{}); break;
            default: look(std::integral_constant<int, 3>{}); break;
        }
        const u32x2_t lo = *reinterpret_cast<lds_u32x2_t*>(static_cast<size_t>(l.at[m][0] + base)), hi = *reinterpret_cast<lds_u32x2_t*>(static_cast<size_t>(l.at[m][1] + base));
        v = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
    } else {
        uint32_t x;
        if constexpr (BITS == 4) x = g.w[j];
        else if constexpr (BITS == 2) x = g.w[j >> 1] >> (4 * (j & 1));
        else x = j < 3 ? g.w[j] : ((g.w[0] >> 6) & 0x03030303u) | ((g.w[1] >> 4) & 0x0C0C0C0Cu) | ((g.w[2] >> 2) & 0x30303030u);
        const auto look = [&](auto bc) {
            constexpr int b = decltype(bc)::value;
            canon_index_to_byte1<b>(l.at[m][b], x, (1u << (2 * BITS)) - 1u);
            v[b] = *reinterpret_cast<clds_cu32_t*>(static_cast<size_t>(l.at[m][b] + l.table));
        };
        look(std::integral_constant<int, 0>{});
        look(std::integral_constant<int, 1>{});
        look(std::integral_constant<int, 2>{});
        look(std::integral_constant<int, 3>{});
    }
    return v;
}

__device__ __forceinline__ f32x4_t step(u32x4_t tokens, u32x4_t weights, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, tokens), __builtin_bit_cast(bf16x8_t, weights), c, 0, 0, 0);
}

// What a workgroup finds out about the choices: the pairs by their experts, those without one and those whose token has the same expert in an earlier
// pair left out, and the list of what there is to do: T tokens at most of an expert, as often as its tokens need, experts ascending.
template <int ROWS, int T>
struct Choices {
    static constexpr int PAIRS = ROWS * KMQ_MOE_MAX_TOP_K;
    static constexpr int MOST = (PAIRS < KMQ_MOE_MAX_EXPERTS ? PAIRS : KMQ_MOE_MAX_EXPERTS) + PAIRS / T;
    static_assert(PAIRS <= 2048 && ROWS <= 128 && ROWS / T <= 8 && KMQ_MOE_MAX_EXPERTS <= 1024, "bits of an entry");
    union {
        int16_t expert[PAIRS + KMQ_MOE_MAX_TOP_K];        // of a pair, -1: none
        uint16_t pairs[PAIRS];                            // an expert's one after the other, ascending: all workgroups cut them alike
    };
    uint32_t list[MOST];                                  // expert << 21 | where its pairs begin << 10 | their number less one << 3 | how many times T came before
    int all;                                              // entries of the list
};
// The sum over this lane and those below it.
__device__ __forceinline__ int sum_upto(int v) {
    const auto add = [&](auto ctrl, auto rows) { v += __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xF, true); };
    add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xF>{});      // row_shr 1, 2, 4, 8
    add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xF>{});
    add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xF>{});
    add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xF>{});
    add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});      // row_bcast15 into rows 1 and 3
    add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});      // row_bcast31 into rows 2 and 3
    return v;
}
// Which tokens an expert has, a bit each, gives their number and every pair's place.  (Counted and ranked by ballots over all pairs, expert by expert, when one was
// needed: 6 us more for 128 tokens, 6 of 64 experts.)  The bits stand in memory that is not used yet, with them
// where the expert's pairs begin.
template <int ROWS>
struct Bits {
    static constexpr int WORDS = (ROWS + 31) / 32, STRIDE = ROWS <= 16 ? 1 : WORDS + 1;
    static constexpr uint32_t MASK = ROWS <= 16 ? 0xFFFFu : ~0u;
    uint32_t* word;
    __device__ __forceinline__ void set(int expert, int token) { atomicOr(&word[expert * STRIDE + (token >> 5)], 1u << (token & 31)); }
    __device__ __forceinline__ int count(int expert) const {
        int n = 0;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) n += __popc(word[expert * STRIDE + i]);
        return n;
    }
    __device__ __forceinline__ void begin(int expert, int at) {
        if constexpr (ROWS <= 16) word[expert] |= static_cast<uint32_t>(at) << 16;
        else word[expert * STRIDE + WORDS] = at;
    }
    __device__ __forceinline__ int place(int expert, int token) const {
        int n = ROWS <= 16 ? word[expert] >> 16 : word[expert * STRIDE + STRIDE - 1];
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const int below = token - 32 * i;             // bits of this word that count
            n += __popc(word[expert * STRIDE + i] & MASK & (below >= 32 ? ~0u : below > 0 ? (1u << below) - 1u : 0u));
        }
        return n;
    }
};
template <int ROWS, int T, int THREADS>
__device__ __forceinline__ void find_choices(const MoeArgs& a, Choices<ROWS, T>& p, Bits<ROWS> bits) {
    constexpr int EACH = (Choices<ROWS, T>::PAIRS + THREADS - 1) / THREADS;
    const int pairs = a.rows * a.top_k, tid = threadIdx.x;
    int e[EACH], token[EACH];
#pragma unroll
    for (int t = 0; t < EACH; ++t) {
        const int i = tid + t * THREADS;
        e[t] = i < pairs ? a.ids[i] : -1;
        if (e[t] < 0 || e[t] >= a.experts) e[t] = -1;
        if (i < pairs) p.expert[i] = static_cast<int16_t>(e[t]);
    }
    for (int i = tid; i < a.experts * Bits<ROWS>::STRIDE; i += THREADS) bits.word[i] = 0;
    __syncthreads();
#pragma unroll
    for (int t = 0; t < EACH; ++t) {
        const int i = tid + t * THREADS;
        if (i >= pairs) continue;
        token[t] = i / a.top_k;
        const int slot = i - token[t] * a.top_k;
        bool again = false;
#pragma unroll
        for (int j = 0; j < KMQ_MOE_MAX_TOP_K - 1; ++j) again |= (j < slot) & (p.expert[i - slot + j] == e[t]);      // (there is room behind the last pair)
        if (again) e[t] = -1;
        if (e[t] >= 0) bits.set(e[t], token[t]);
    }
    __syncthreads();
    if (tid < kWave) {                                    // experts lane * some .. lane * some + some - 1
        const int some = (a.experts + kWave - 1) / kWave, first = tid * some, end = min(first + some, a.experts);
        int sum = 0;                                      // pairs << 16 | times
        for (int i = first; i < end; ++i) sum += bits.count(i) << 16 | (bits.count(i) + T - 1) / T;
        const int upto = sum_upto(sum);
        if (tid == kWave - 1) p.all = upto & 0xFFFF;
        int at = (upto - sum) & 0xFFFF, begin = (upto - sum) >> 16;
        for (int i = first; i < end; ++i) {
            const int count = bits.count(i);
            for (int k = 0; k * T < count; ++k) p.list[at++] = static_cast<uint32_t>(i << 21 | begin << 10 | (count - 1) << 3 | k);
            bits.begin(i, begin);
            begin += count;
        }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < EACH; ++t)
        if (e[t] >= 0) p.pairs[bits.place(e[t], token[t])] = static_cast<uint16_t>(tid + t * THREADS);
    __syncthreads();
}

// What a wave asks for at a time: a super-block of two matrices, and the elements under it of T tokens of the expert.  Fewer than 16 tokens
// leave most lanes of the operand without one, so 16 / T steps' operands come with one load: lane n takes token n % T at step n / T, and a
// rotation inside 16 lanes brings it to where the step wants it.  (What the other lanes hold then are columns that nobody reads.)
// T = 16 at 1 bit would take 64 registers: there the elements are read when they are needed.
template <int BITS, int T, bool STAGED>
struct Bundle {
    static constexpr int LOADS = T / 4;                   // of tokens, for four steps
    static constexpr bool TOKENS = !STAGED && (BITS > 1 || T < 16);
    static constexpr int WORDS = 2 * Granule<BITS>::WORDS + (TOKENS ? LOADS * Granule<BITS>::STEPS : 0);
    Granule<BITS> g[2];
    u32x4_t x[TOKENS ? Granule<BITS>::STEPS / 4 : 1][LOADS];
};
struct Tokens {
    Rows rows;
    uint32_t at;                                          // where the lane's token begins
    const u32x4_t* staged;                                // operands in shared memory, 64 lanes a step
};
template <int T>
__device__ __forceinline__ void load_tokens(const Tokens& tokens, uint32_t column, u32x4_t (&x)[T / 4]) {
#pragma unroll
    for (int l = 0; l < T / 4; ++l) x[l] = load_row16(tokens.rows, tokens.at + l * (1024 / T), column * 2);
}
template <int BITS, int T, bool STAGED>
__device__ __forceinline__ void load_bundle(const Matrix (&m)[2], int unit, const Tokens& tokens, int lane, Bundle<BITS, T, STAGED>& b) {
    using G = Granule<BITS>;
#pragma unroll
    for (int i = 0; i < 2; ++i) load_granule<BITS>(m[i], unit, lane, b.g[i]);
    if constexpr (Bundle<BITS, T, STAGED>::TOKENS) {
#pragma unroll
        for (int k = 0; k < G::STEPS / 4; ++k) load_tokens<T>(tokens, unit * G::COLUMNS + 128 * k, b.x[k]);
    }
}
// Elements 0 .. 7 as (0, 4), (1, 5), (2, 6), (3, 7).
__device__ __forceinline__ u32x4_t pairs_apart(u32x4_t x) {
    return u32x4_t{__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u),
                   __builtin_amdgcn_perm(x[3], x[1], 0x05040100u), __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
}
// The operand of step j of four.
template <int T>
__device__ __forceinline__ u32x4_t operand(const u32x4_t (&x)[T / 4], int j) {
    if constexpr (T == 16) return x[j];
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
// One bundle's products, added to acc; `scales`: the lane's row from the super-block on, `staged`: the operands from it on.
template <int BITS, int T, bool STAGED, int PIECE>
__device__ __forceinline__ void multiply_bundle(const Bundle<BITS, T, STAGED>& b, LookUp<BITS>& l, const uint32_t* scales, const u32x4_t* staged, const Tokens& tokens,
                                                int unit, int lane, f32x4_t (&acc)[2]) {
    using G = Granule<BITS>;
    using B = Bundle<BITS, T, STAGED>;
#pragma unroll
    for (int k = 0; k < G::STEPS / 4; ++k) {
        u32x4_t x[B::LOADS];
        if constexpr (STAGED) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = staged[(4 * k + i) * kWave + lane];
        } else if constexpr (B::TOKENS) {
#pragma unroll
            for (int i = 0; i < B::LOADS; ++i) x[i] = b.x[k][i];
        } else {
            load_tokens<T>(tokens, unit * G::COLUMNS + 128 * k, x);
        }
        if constexpr (!STAGED && (BITS == 2 || BITS == 3)) {
#pragma unroll
            for (int i = 0; i < B::LOADS; ++i) x[i] = pairs_apart(x[i]);
        }
        uint32_t both[2];                                 // the scales of two blocks
#pragma unroll
        for (int i = 0; i < 2; ++i) both[i] = scales[i * sizeof(PieceScales<PIECE>) / 8 + k];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int block = 2 * k + half;
            const u32x4_t x0 = operand<T>(x, 2 * half), x1 = operand<T>(x, 2 * half + 1);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32x4_t w0 = decode<BITS>(b.g[i], l, i, 2 * block), w1 = decode<BITS>(b.g[i], l, i, 2 * block + 1);
                const float s = kv_half(both[i], half);
                f32x4_t d = step(x0, w0, f32x4_t{0.f, 0.f, 0.f, 0.f});
                d = step(x1, w1, d);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][r] = fmaf(s, d[r], acc[i][r]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);                // (else what later steps need is looked up and turned early, and spilled)
    }
}
// The sums over super-blocks u .. end - 1; the first D bundles have been asked for.  `scales`: the lane's row from super-block `start` on.  The
// loop's loads are unconditional, the last super-blocks a copy of the code of their own: a branch around a load would make every wait
// assume the fewest of them.
template <int BITS, int T, bool STAGED, int PIECE, int D>
__device__ __forceinline__ void run_units(Bundle<BITS, T, STAGED> (&b)[D], const Matrix (&m)[2], int u, int end, LookUp<BITS>& l, const uint32_t* scales, int start,
                                          const Tokens& tokens, int lane, f32x4_t (&acc)[2]) {
    using G = Granule<BITS>;
    const auto multiply_at = [&](int slot, int unit) {
        multiply_bundle<BITS, T, STAGED, PIECE>(b[slot], l, scales + (unit - start) * (G::BLOCKS / 2), tokens.staged + (unit - start) * (G::STEPS * kWave), tokens, unit, lane, acc);
    };
    for (; u + 2 * D <= end; u += D) {
#pragma unroll
        for (int p = 0; p < D; ++p) {
            multiply_at(p, u + p);
            load_bundle<BITS, T, STAGED>(m, u + p + D, tokens, lane, b[p]);
        }
    }
#pragma unroll
    for (int p = 0; p < D; ++p) {
        if (u + p >= end) return;
        multiply_at(p, u + p);
        if (u + p + D < end) load_bundle<BITS, T, STAGED>(m, u + p + D, tokens, lane, b[p]);
    }
#pragma unroll
    for (int p = 0; p < D - 1; ++p) {
        if (u + D + p >= end) return;
        multiply_at(p, u + D + p);
    }
}
// A value that the compiler does not know to be the same in every round of a loop: what is worked out from it is worked out there again,
// where kept for later it would take a register for as long.
__device__ __forceinline__ int anew(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// More tokens than a wave's 16 at once stand as operands in shared memory, a piece of the columns at a time.
constexpr bool staged(int rows) { return rows > 16; }
constexpr int piece_columns(int bits, int rows) { return !staged(rows) ? 4096 : bits == 4 ? 1024 : 2048; }

template <int BITS, int T, int ROWS, int NW, int TEAMS>
struct Shared {
    static constexpr bool STAGED = staged(ROWS);
    static constexpr int PIECE = piece_columns(BITS, ROWS);
    Tables<BITS> tables;
    u32x4_t tokens[STAGED ? PIECE / 32 * kWave : 1];
    f32x4_t part[TEAMS][NW > 1 ? NW - 1 : 1][2][NW > 1 ? 4 * T : 1];      // sums of a team's waves but the first
    PieceScales<PIECE> scales[TEAMS];
    Choices<ROWS, T> choices;
};
// The operands of a piece on their way into shared memory, step by step, the workgroup's waves in turn.
template <int BITS, int PIECE, int WAVES>
struct Stage {
    static constexpr int EACH = PIECE ? PIECE / 32 / WAVES : 1;
    u32x4_t raw[EACH];
    __device__ __forceinline__ void load(const Tokens& tokens, int first, int steps, int wave) {
#pragma unroll
        for (int k = 0; k < EACH; ++k)
            if (wave + k * WAVES < steps) raw[k] = load_row16(tokens.rows, tokens.at, (first + wave + k * WAVES) * 64);
    }
    __device__ __forceinline__ void keep(u32x4_t* to, int steps, int wave, int lane) const {
#pragma unroll
        for (int k = 0; k < EACH; ++k)
            if (wave + k * WAVES < steps) to[(wave + k * WAVES) * kWave + lane] = BITS == 2 || BITS == 3 ? pairs_apart(raw[k]) : raw[k];
    }
};

// A workgroup of TEAMS teams of NW waves; T tokens at a time.  GATED: rows of gate and up, else pairs of row blocks of down.
template <int BITS, int T, int ROWS, int NW, int TEAMS, bool GATED>
__global__ __launch_bounds__(NW * TEAMS * kWave) __attribute__((amdgpu_waves_per_eu(waves_for(BITS, T, staged(ROWS))))) void moe_rows_kernel(MoeArgs a) {
    using G = Granule<BITS>;
    using Sm = Shared<BITS, T, ROWS, NW, TEAMS>;
    constexpr bool STAGED = Sm::STAGED;
    constexpr int PIECE = Sm::PIECE, D = STAGED ? 2 : depth(Bundle<BITS, T, STAGED>::WORDS), LANES = 4 * T;
    __shared__ Sm sm;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = wave / NW, member = wave % NW;
    const auto lane_anew = [] { return anew(static_cast<int>(threadIdx.x)) & 63; };
    const int kept = threadIdx.x & 63;
    // (at 1 bit there is no register to keep it in: 118 -> 113 us, 16 tokens, 8 of 128 experts of 4096 x 1536; at 2 to 4 bits it would cost 4 to 6 % there)
    const auto lane_kept = [&] { return BITS == 1 ? lane_anew() : kept; };
    const auto place = [&] { return member * kWave + lane_anew(); };        // in the team
    static_assert(offsetof(Sm, choices) >= sizeof(uint32_t) * Bits<ROWS>::STRIDE * KMQ_MOE_MAX_EXPERTS, "bits");      // (what lies before is filled later)
    find_choices<ROWS, T, NW * TEAMS * kWave>(a, sm.choices, Bits<ROWS>{reinterpret_cast<uint32_t*>(&sm)});
    const int columns = static_cast<int>(GATED ? a.hidden : a.width), units = columns / G::COLUMNS, pairs = a.rows * a.top_k;
    const int per_expert = static_cast<int>(GATED ? a.width >> 4 : a.hidden >> 5) / TEAMS;
    const unsigned items = static_cast<unsigned>(sm.choices.all) * per_expert, each = items / gridDim.x, over = items - each * gridDim.x;
    const int from = static_cast<int>(each * blockIdx.x + min(blockIdx.x, over)), to = from + static_cast<int>(each + (blockIdx.x < over));
    if (from >= to) return;
    uint16_t* const h = static_cast<uint16_t*>(a.workspace);
    float* const out = reinterpret_cast<float*>(h + static_cast<int64_t>(pairs) * a.width);
    const uint32_t stride = static_cast<uint32_t>(GATED ? a.x_stride : a.width) * 2u;
    Tokens tokens;
    tokens.rows = rows_at(GATED ? static_cast<const void*>(a.x) : h);
    tokens.staged = sm.tokens;
    Bundle<BITS, T, STAGED> b[D];
    Scales<PIECE, NW * kWave> scales;
    Stage<BITS, STAGED ? PIECE : 0, NW * TEAMS> stage;
    Matrix m[2];
    LookUp<BITS> l(sm.tables, lane_kept());
    // where the workgroup is: the `group`-th row blocks of expert e, of whose `count` pairs (from `begin` on) those from `time` * T on (`times` in all), a piece
    // of the columns, of which super-blocks u .. end - 1 are this wave's; this lane's pair.  An expert's items lie by row blocks first, so that
    // all its tokens meet these while they are in the L2; `entry` is the list's first of the next expert.
    int entry = from / per_expert, group, e, time, times, count, begin, piece = 0, u, end, words, pair;
    const auto find_expert = [&](int at) {
        const uint32_t found = __builtin_amdgcn_readfirstlane(sm.choices.list[at]);
        e = found >> 21;
        begin = found >> 10 & 0x7FF;
        count = (found >> 3 & 0x7F) + 1;
        times = (count + T - 1) / T;
        entry = at - (found & 7) + times;
    };
    find_expert(entry);
    {
        const int within = from - (entry - times) * per_expert;
        group = within / times;
        time = within - group * times;
    }
    uint32_t centroids = 0;
    int steps = 0;                                        // to be staged
    const auto ask_piece = [&](bool tokens_too) {
        constexpr int MOST = PIECE / G::COLUMNS;
        const int start = piece * MOST, some = units - start < MOST ? units - start : MOST;
        words = some * (G::BLOCKS / 2);
        u = start + some * member / NW;
        end = start + some * (member + 1) / NW;
        scales.load(m, columns / 128, piece * (PIECE / 128), words, place());
        if constexpr (STAGED) {
            steps = tokens_too ? some * G::STEPS : 0;
            stage.load(tokens, start * G::STEPS, steps, wave);
        }
#pragma unroll
        for (int p = 0; p < D; ++p)
            if (u + p < end) load_bundle<BITS, T, STAGED>(m, u + p, tokens, lane_kept(), b[p]);
    };
    const auto ask = [&](bool other, bool tokens_too) {
        if (other) {                                      // (before the bundles: what is waited for first is asked for first)
            const int lane = lane_anew();
            const uint16_t* book = (!GATED ? a.down.books : lane & 16 ? a.up.books : a.gate.books) + (e << BITS);
            centroids = book[lane & ((1 << BITS) - 1)];
        }
        const int block = group * TEAMS + team;
        m[0] = matrix_of<BITS>(GATED ? a.gate : a.down, e, GATED ? block : 2 * block, units);
        m[1] = matrix_of<BITS>(GATED ? a.up : a.down, e, GATED ? block : 2 * block + 1, units);
        if (tokens_too) {
            const int lane = lane_anew(), n = lane & 15, q = lane >> 4;
            const int i = n % T, from = begin + time * T;
            pair = n < count - time * T ? sm.choices.pairs[from + n] : 0;
            const int p = __shfl(pair, i);
            tokens.at = kNoRow;
            if (time * T + i < count) tokens.at = static_cast<uint32_t>(GATED ? p / a.top_k : p) * stride + 16u * q + n / T * 64u;
        }
        piece = 0;
        ask_piece(tokens_too || columns > PIECE);
    };
    const auto keep = [&] {
        scales.keep(sm.scales[team], words, place());
        if constexpr (STAGED) stage.keep(sm.tokens, steps, wave, lane_anew());
    };
    ask(true, true);
    keep();
    fill_tables<BITS>(sm.tables, centroids, wave, NW * TEAMS, lane_anew());
    __syncthreads();
    for (int item = from;;) {
        f32x4_t acc[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
        for (;;) {
            const int lane = lane_kept();
            run_units<BITS, T, STAGED, PIECE, D>(b, m, u, end, l, &sm.scales[team][0][(lane & 15) * (words | 1)], piece * (PIECE / G::COLUMNS), tokens, lane, acc);
            if ((piece + 1) * PIECE >= columns) break;
            ++piece;
            ask_piece(true);
            __syncthreads();
            keep();
            __syncthreads();
        }
        // what comes next is asked for before the sums are joined
        const int left = count - time * T < T ? count - time * T : T, block = group * TEAMS + team, now = pair;
        const bool more = ++item < to, several = times > 1;
        bool other = false;
        if (more && ++time == times) {
            time = 0;
            if (++group == per_expert) {
                group = 0;
                find_expert(entry);
                other = true;
            }
        }
        if (more) ask(other, other || several);
        {
            const int lane = lane_anew(), n = lane & 15, q = lane >> 4;
            if (member > 0 && lane < LANES) {
                sm.part[team][member - 1][0][lane] = acc[0];
                sm.part[team][member - 1][1][lane] = acc[1];
            }
            __syncthreads();
            if (member == 0) {
                if (lane < LANES) {
#pragma unroll
                    for (int w = 0; w < NW - 1; ++w) {
                        acc[0] += sm.part[team][w][0][lane];
                        acc[1] += sm.part[team][w][1][lane];
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = 4 * q + i;
                    const int64_t p = __shfl(now, at);
                    if (at >= left) continue;
                    if constexpr (GATED) {
                        const float g = acc[0][i], v = acc[1][i];
                        h[p * a.width + block * 16 + n] = f32_to_bf16(g / (1.f + expf(-g)) * v);
                    } else {
                        out[p * a.hidden + block * 32 + n] = acc[0][i];
                        out[p * a.hidden + block * 32 + 16 + n] = acc[1][i];
                    }
                }
            }
        }
        if (!more) break;
        keep();                                           // (every wave has been past a barrier since it read the last ones)
        if (other) fill_tables<BITS>(sm.tables, centroids, wave, NW * TEAMS, lane_anew());
        __syncthreads();
    }
}

// y = residual + the sum of a token's pairs, in their order.  A thread four elements.  (Pairs asked for before the ids have come, as they may: no faster.)
__global__ __launch_bounds__(256) void moe_join_kernel(MoeArgs a) {
    const int token = blockIdx.y, column = (static_cast<int>(blockIdx.x) * 256 + static_cast<int>(threadIdx.x)) * 4;
    if (column >= a.hidden) return;
    const float* out = reinterpret_cast<const float*>(static_cast<const uint16_t*>(a.workspace) + static_cast<int64_t>(a.rows) * a.top_k * a.width);
    const int32_t* ids = a.ids + token * a.top_k;
    const float* gates = a.gates + token * a.top_k;
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
    if (a.residual) {
        const u32x2_t r = *reinterpret_cast<const u32x2_t*>(a.residual + token * a.residual_stride + column);
        s = f32x4_t{kv_half(r[0], 0), kv_half(r[0], 1), kv_half(r[1], 0), kv_half(r[1], 1)};
    }
    int id[KMQ_MOE_MAX_TOP_K];
#pragma unroll
    for (int j = 0; j < KMQ_MOE_MAX_TOP_K; ++j) id[j] = j < a.top_k ? ids[j] : -1;
    f32x4_t v[KMQ_MOE_MAX_TOP_K];
    float w[KMQ_MOE_MAX_TOP_K];
#pragma unroll
    for (int j = 0; j < KMQ_MOE_MAX_TOP_K; ++j) {
        int from = j;                                     // the first of the token's pairs with this expert
#pragma unroll
        for (int i = j - 1; i >= 0; --i) from = id[i] == id[j] ? i : from;
        const bool counts = id[j] >= 0 && id[j] < a.experts;
        w[j] = counts ? gates[j] : 0.f;
        v[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (counts) v[j] = *reinterpret_cast<const f32x4_t*>(out + (static_cast<int64_t>(token) * a.top_k + from) * a.hidden + column);
    }
#pragma unroll
    for (int j = 0; j < KMQ_MOE_MAX_TOP_K; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = fmaf(w[j], v[j][i], s[i]);
    }
    *reinterpret_cast<u32x2_t*>(a.y + token * a.y_stride + column) = u32x2_t{kv_pack2(s[0], s[1]), kv_pack2(s[2], s[3])};
}

}  // namespace

size_t moe_workspace_bytes(int64_t rows, int64_t top_k, int64_t width, int64_t hidden) { return static_cast<size_t>(rows * top_k * (width * 2 + hidden * 4)); }

template <int BITS, int T, int ROWS, int NW, int WAVES, bool GATED>
static void launch_rows(const MoeArgs& a, hipStream_t s) {
    constexpr int TEAMS = WAVES / NW, BY_WAVES = 4 * waves_for(BITS, T, staged(ROWS)) / WAVES, BY_MEMORY = 160 * 1024 / sizeof(Shared<BITS, T, ROWS, NW, TEAMS>);
    static_assert(8 % TEAMS == 0, "row blocks come in eights");
    constexpr int64_t MOST = 256 * (BY_WAVES < BY_MEMORY ? BY_WAVES : BY_MEMORY);          // as many as run at once
    const int64_t pairs = static_cast<int64_t>(a.rows) * a.top_k, experts = pairs < a.experts ? pairs : a.experts;
    const int64_t items = (experts + pairs / T) * ((GATED ? a.width / 16 : a.hidden / 32) / TEAMS);
    moe_rows_kernel<BITS, T, ROWS, NW, TEAMS, GATED><<<dim3(static_cast<unsigned>(items < MOST ? items : MOST)), WAVES * kWave, 0, s>>>(a);
}

// Waves that split a row (us, `rows` tokens, top_k of experts, hidden x width): four, or two where rows are short (fewer than 16 super-blocks) and there are enough of
// them (16, 8 of 128, 4096 x 1536: 1 bit 112 with two, 122 with four; 2 bits 125, 136; 3 bits 144, 149).  At 4 bits eight waves share the table, 64 KB, and two of
// them a row are slower (the same 164 with four, 197 with two; 2048 x 768 62 and 74).  Eight where few long rows would leave units without work (one token, 1
// expert of 2176 x 15744, 3 bits 35.8, with four 42.7; 2 of 4096 x 14336, 4 bits 52, 60.5; 2 of 7040 x 8576, 4 bits 56, 58.5; 4 of 3840 x 8704, 3 bits 49, 51).  Up to 1024
// items instead of 512 it no longer pays (one token, 8 of 4096 x 1536: 2 bits 24.3 -> 24.9, 3 bits 26.4 -> 26.9, 4 bits 30.7 -> 30.1; 4 of 4096 x 3584, 4 bits 32.1 -> 32.7; two
// tokens, 8 of 64, 2048 x 1024, 4 bits 24.4 -> 25.1).
template <int BITS, int T, bool GATED>
static void launch_few(const MoeArgs& a, hipStream_t s) {
    const int64_t pairs = static_cast<int64_t>(a.rows) * a.top_k, experts = pairs < a.experts ? pairs : a.experts;
    const int64_t units = (GATED ? a.hidden : a.width) / Granule<BITS>::COLUMNS, items = experts * (GATED ? a.width / 16 : a.hidden / 32);
    if constexpr (T == 4) {
        if (items <= 512 && units >= 16) {
            launch_rows<BITS, T, 16, 8, 8, GATED>(a, s);
            return;
        }
    }
    if constexpr (BITS == 4) launch_rows<BITS, T, 16, 4, 8, GATED>(a, s);
    else if (units < 16 && items >= 2048) launch_rows<BITS, T, 16, 2, 4, GATED>(a, s);
    else launch_rows<BITS, T, 16, 4, 4, GATED>(a, s);
}

// Tokens at a time (us, as above): where more of them choose an expert its rows are read again (from the L2, mostly), and every four more cost registers and loads.  With
// 4 / 8 / 16 at a time: 16 tokens, 8 of 128, 4096 x 1536, 2 bits 129 / 140 / 168, 3 bits 147 / 143, 4 bits 164 / 163 / 184; 5 tokens, 2 of 8, 4096 x 14336, 2 bits 102 / 113 /
// 125; but 16 tokens, 8 of 64, 4096 x 1536, 3 bits 119 / 113 / 120, and 2 of 8, 4096 x 14336, 4 bits 197 with 4, 166 with 16, 1 bit 131 and 127.
// More than 16 tokens take 16 at a time (32: 128 tokens, 6 of 64, 2048 x 1408, 3 bits 137 -> 171 before tokens were shared), which eight teams of two waves share in shared
// memory (every wave for itself from the caches: these 122 -> 105; 64 of them, 4 bits 130 -> 98; 100, 2048 x 1536, 2 bits 131 -> 86).  Four teams of four: 98 -> 112, 97 -> 108, 86 ->
// 103.  1 bit needs the registers of eight waves (40 tokens, 8 of 128, 4096 x 1536: 180; sixteen, spilled, 250; four teams of two 232).
// Eight waves a row where eight teams would leave half of the units without work (53 tokens, 1 of 4, 2048 x 7168, 4 bits 59, without 78; 60 tokens, 1 of 4, 2048 x 8192, 1 bit 35,
// 55); at twice that many items no longer (20 tokens, 1 of 16, 3328 x 5120, 4 bits 107 -> 122; 40, 2 of 8, 4096 x 14336, 2 bits 174 -> 189).  For 16 rows and fewer sharing tokens
// does not pay (16 tokens, 2 of 8, 4096 x 14336, 4 bits 166 -> 191, 1 bit 127 -> 142; 8 of 64, 4096 x 1536, 3 bits 112 -> 111).
template <int BITS, bool GATED>
static void launch_product(const MoeArgs& a, hipStream_t s) {
    const int64_t pairs = static_cast<int64_t>(a.rows) * a.top_k, experts = a.experts, items = ((pairs < experts ? pairs : experts) + pairs / 16) * (GATED ? a.width / 128 : a.hidden / 256);
    if (a.rows <= 4 || (a.rows <= 16 && 2 * pairs <= (BITS == 1 ? 6 : 3) * experts)) {
        launch_few<BITS, 4, GATED>(a, s);
        return;
    }
    if constexpr (BITS > 1) {
        if (a.rows <= 8 || (a.rows <= 16 && pairs <= 3 * experts)) {
            launch_few<BITS, 8, GATED>(a, s);
            return;
        }
    }
    if (a.rows <= 16) {
        launch_rows<BITS, 16, 16, 2, 4, GATED>(a, s);
        return;
    }
    constexpr int WAVES = BITS == 1 ? 8 : 16;
    if (items <= 128) {
        launch_rows<BITS, 16, KMQ_MOE_MAX_ROWS, 8, WAVES, GATED>(a, s);
        return;
    }
    // (eight teams need row blocks in sixteens: the down projection's pairs of them come in fours at 3 and 4 bits)
    if constexpr (!GATED && BITS >= 3) {
        if (a.hidden % 256 != 0) {
            launch_rows<BITS, 16, KMQ_MOE_MAX_ROWS, WAVES / 4, WAVES, GATED>(a, s);
            return;
        }
    }
    launch_rows<BITS, 16, KMQ_MOE_MAX_ROWS, WAVES / 8, WAVES, GATED>(a, s);
}

template <int BITS>
static void launch_moe_bits(const MoeArgs& a, hipStream_t s) {
    launch_product<BITS, true>(a, s);
    launch_product<BITS, false>(a, s);
    moe_join_kernel<<<dim3(static_cast<unsigned>((a.hidden + 1023) / 1024), static_cast<unsigned>(a.rows)), 256, 0, s>>>(a);
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
