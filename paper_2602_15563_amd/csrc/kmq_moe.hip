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

constexpr int kMoeWaves = 8, kMoeThreads = kMoeWaves * kWave;
constexpr int kMoePairs = KMQ_MOE_MAX_ROWS * KMQ_MOE_MAX_TOP_K;

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

// One matrix of one expert, as a lane sees it: its granules, and the scales of its row.
struct Matrix {
    const uint32_t* words;
    const uint16_t* scales;
};
template <int BITS>
__device__ __forceinline__ Matrix matrix_of(const MoeMatrix& m, int expert, int row_block, int units, int lane) {
    using G = Granule<BITS>;
    const int64_t blocks = (m.rows + 15) >> 4;
    int64_t row = static_cast<int64_t>(row_block) * 16 + (lane & 15);
    row = row < m.rows ? row : m.rows - 1;
    return {m.words + ((expert * blocks + row_block) * units * 64 + lane) * G::WORDS, m.scales + (expert * m.rows + row) * (units * G::BLOCKS)};
}
template <int BITS>
__device__ __forceinline__ void load_granule(const Matrix& m, int unit, Granule<BITS>& g) {
    using G = Granule<BITS>;
    const uint32_t* p = m.words + static_cast<int64_t>(unit) * (64 * G::WORDS);
    if constexpr (G::WORDS == 3) {
        typedef u32x3_t __attribute__((aligned(4))) u32x3_a4_t;
        const u32x3_t t = __builtin_nontemporal_load(reinterpret_cast<const u32x3_a4_t*>(p));
        g.w[0] = t[0]; g.w[1] = t[1]; g.w[2] = t[2];
    } else {
        const u32x4_t t = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
        g.w[0] = t[0]; g.w[1] = t[1]; g.w[2] = t[2]; g.w[3] = t[3];
    }
    const uint16_t* s = m.scales + unit * G::BLOCKS;
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
// Entries first, first + step, .. of the pairs of a 4-bit table.
__device__ __forceinline__ void fill_table(Table& table, const uint16_t* book, int first, int step, int lane) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(book);
    for (int e = first; e < 8; e += step) {
        const uint32_t two = w[e];
        table[2 * e][lane] = __builtin_amdgcn_perm(two, two, 0x01000100u);
        table[2 * e + 1][lane] = __builtin_amdgcn_perm(two, two, 0x03020302u);
    }
}

// Eight weights of step j.
template <int BITS>
__device__ __forceinline__ u32x4_t decode(const Granule<BITS>& g, const Centroids<BITS>& c, const uint32_t* table, const u32x2_t* masks, int j) {
    if constexpr (BITS == 1) {
        const uint32_t b = g.w[j >> 2] >> (8 * (j & 3));
        const u32x2_t l = masks[b & 15u], h = masks[(b >> 4) & 15u];
        const auto choose = [&](uint32_t m) { return (m & c.b) | (~m & c.a); };
        return u32x4_t{choose(l[0]), choose(l[1]), choose(h[0]), choose(h[1])};
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
        // `table` is the lane's column
        const uint32_t x = g.w[j];
        uint32_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = table[((x >> (4 * e)) & 15u) * 64];
        return u32x4_t{__builtin_amdgcn_perm(v[1], v[0], 0x07060100u), __builtin_amdgcn_perm(v[3], v[2], 0x07060100u),
                       __builtin_amdgcn_perm(v[5], v[4], 0x07060100u), __builtin_amdgcn_perm(v[7], v[6], 0x07060100u)};
    }
}

__device__ __forceinline__ f32x4_t step(u32x4_t tokens, u32x4_t weights, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, tokens), __builtin_bit_cast(bf16x8_t, weights), c, 0, 0, 0);
}

// What both kernels find out about the choices: which pairs count, their weights, which experts have any.
struct Plan {
    uint32_t has[KMQ_MOE_MAX_EXPERTS / 32];               // a bit an expert
    int16_t expert[kMoePairs];                            // of a pair; -1: none, or the same as an earlier one's of the token
    float weight[kMoePairs];                              // the sum over the token's pairs with this expert
    uint16_t list[KMQ_MOE_MAX_EXPERTS];                   // experts that have pairs, ascending
    int experts;
};
__device__ void make_plan(const MoeArgs& a, Plan& p) {
    const int pairs = a.rows * a.top_k, tid = threadIdx.x, lane = tid & 63;
    for (int i = tid; i < KMQ_MOE_MAX_EXPERTS / 32; i += kMoeThreads) p.has[i] = 0;
    for (int i = tid; i < pairs; i += kMoeThreads) {
        const int e = a.ids[i];
        p.expert[i] = static_cast<int16_t>(e >= 0 && e < a.experts ? e : -1);
    }
    __syncthreads();
    bool first[(kMoePairs + kMoeThreads - 1) / kMoeThreads];
    for (int i = tid, t = 0; i < pairs; i += kMoeThreads, ++t) {
        const int e = p.expert[i], token = i / a.top_k;
        first[t] = e >= 0;
        float w = a.gates[i];
        for (int j = token * a.top_k; j < i; ++j) first[t] = first[t] && p.expert[j] != e;
        for (int j = i + 1; j < (token + 1) * a.top_k; ++j)
            if (p.expert[j] == e) w += a.gates[j];
        p.weight[i] = w;
        if (first[t]) atomicOr(&p.has[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
    for (int i = tid, t = 0; i < pairs; i += kMoeThreads, ++t)
        if (!first[t]) p.expert[i] = -1;
    if (tid < kWave) {
        uint32_t mine = lane < KMQ_MOE_MAX_EXPERTS / 32 ? p.has[lane] : 0u;
        int before = __popc(mine);
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(before, d);
            if (lane >= d) before += o;
        }
        if (lane == 63) p.experts = before;
        before -= __popc(mine);
        for (; mine; mine &= mine - 1) p.list[before++] = static_cast<uint16_t>(lane * 32 + __ffs(mine) - 1);
    }
    __syncthreads();
}

// The pairs of an expert, into `list` (this wave's own); how many.
__device__ int pairs_of(const Plan& p, int pairs, int expert, uint16_t* list) {
    const int lane = threadIdx.x & 63;
    int count = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int i = lane; i < (pairs + 63) / 64 * 64; i += 64) {
        const bool mine = i < pairs && p.expert[i] == expert;
        const uint64_t all = __ballot(mine);
        if (mine) list[count + __popcll(all & ((uint64_t(1) << lane) - 1))] = static_cast<uint16_t>(i);
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

// One granule times the tokens of CT column tiles, added to acc.
template <int BITS, int CT>
__device__ __forceinline__ void multiply(const Granule<BITS>& g, const Centroids<BITS>& c, const uint32_t* table, const u32x2_t* masks,
                                         const u32x4_t (&x)[CT][4], int quarter, f32x4_t (&acc)[CT]) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int block = 2 * quarter + b;
        const u32x4_t w0 = decode<BITS>(g, c, table, masks, 2 * block), w1 = decode<BITS>(g, c, table, masks, 2 * block + 1);
        const float s = kv_half(g.scale[block / 2], block % 2);
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            f32x4_t d = step(x[t][2 * b], w0, f32x4_t{0.f, 0.f, 0.f, 0.f});
            d = step(x[t][2 * b + 1], w1, d);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][i] = fmaf(s, d[i], acc[t][i]);
        }
    }
}

template <int BITS, int CT>
__global__ __launch_bounds__(kMoeThreads) void moe_gate_up_kernel(MoeArgs a) {
    using G = Granule<BITS>;
    __shared__ Plan plan;
    __shared__ uint16_t lists[kMoeWaves][KMQ_MOE_MAX_ROWS];
    __shared__ u32x2_t masks[BITS == 1 ? 16 : 1];
    __shared__ Table tables[BITS == 4 ? 2 : 1];
    __shared__ float part[kMoeWaves][2][16][17];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    if constexpr (BITS == 1) fill_masks(masks);
    make_plan(a, plan);
    const int blocks = static_cast<int>((a.gate.rows + 15) >> 4), units = static_cast<int>(a.hidden / G::COLUMNS);
    const int u0 = units * wave / kMoeWaves, u1 = units * (wave + 1) / kMoeWaves;
    const Rows xr = rows_at(a.x);
    uint16_t* h = static_cast<uint16_t*>(a.workspace);
    int seen = -1, count = 0;
    Centroids<BITS> cg = {}, cu = {};
    for (int item = blockIdx.x; item < plan.experts * blocks; item += gridDim.x) {
        const int e = __builtin_amdgcn_readfirstlane(plan.list[item / blocks]), block = item % blocks;
        const Matrix mg = matrix_of<BITS>(a.gate, e, block, units, lane), mu = matrix_of<BITS>(a.up, e, block, units, lane);
        if (e != seen) {
            seen = e;
            count = pairs_of(plan, a.rows * a.top_k, e, lists[wave]);
            const uint16_t *bg = a.gate.books + (e << BITS), *bu = a.up.books + (e << BITS);
            cg = centroids_of<BITS>(bg);
            cu = centroids_of<BITS>(bu);
            if constexpr (BITS == 4) {
                __syncthreads();
                fill_table(tables[0], bg, wave, kMoeWaves, lane);
                fill_table(tables[1], bu, wave, kMoeWaves, lane);
                __syncthreads();
            }
        }
        const uint32_t *tg = &tables[0][0][lane], *tu = &tables[BITS == 4 ? 1 : 0][0][lane];
        for (int first = 0; first < count; first += 16 * CT) {
            uint32_t at[CT];
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                const int i = first + 16 * t + n;
                at[t] = i < count ? static_cast<uint32_t>(lists[wave][i] / a.top_k) * static_cast<uint32_t>(a.x_stride * 2) + 16u * q : kNoRow;
            }
            f32x4_t ag[CT], au[CT];
#pragma unroll
            for (int t = 0; t < CT; ++t) ag[t] = au[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            Granule<BITS> gg, gu;
            if (u0 < u1) {
                load_granule<BITS>(mg, u0, gg);
                load_granule<BITS>(mu, u0, gu);
            }
            for (int u = u0; u < u1; ++u) {
                Granule<BITS> ng = gg, nu = gu;
#pragma unroll
                for (int k = 0; k < G::STEPS / 4; ++k) {
                    u32x4_t x[CT][4];
#pragma unroll
                    for (int t = 0; t < CT; ++t)
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[t][j] = load_row16(xr, at[t] + 64 * j, (u * G::COLUMNS + 128 * k) * 2);
                    if (k == 0) {
                        const int next = u + 1 < u1 ? u + 1 : u;
                        load_granule<BITS>(mg, next, ng);
                        load_granule<BITS>(mu, next, nu);
                    }
                    multiply<BITS, CT>(gg, cg, tg, masks, x, k, ag);
                    multiply<BITS, CT>(gu, cu, tu, masks, x, k, au);
                }
                gg = ng;
                gu = nu;
            }
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                if (first + 16 * t >= count) break;
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    part[wave][0][4 * q + i][n] = ag[t][i];
                    part[wave][1][4 * q + i][n] = au[t][i];
                }
                __syncthreads();
                if (threadIdx.x < 256) {
                    const int m = threadIdx.x >> 4, r = threadIdx.x & 15, i = first + 16 * t + m;
                    const int64_t row = static_cast<int64_t>(block) * 16 + r;
                    float g = part[0][0][m][r], u = part[0][1][m][r];
#pragma unroll
                    for (int w = 1; w < kMoeWaves; ++w) {
                        g += part[w][0][m][r];
                        u += part[w][1][m][r];
                    }
                    if (i < count && row < a.gate.rows) h[lists[wave][i] * a.width + row] = f32_to_bf16(g / (1.f + expf(-g)) * u);
                }
            }
        }
    }
}

template <int BITS, int CT>
__global__ __launch_bounds__(kMoeThreads) void moe_down_kernel(MoeArgs a) {
    using G = Granule<BITS>;
    __shared__ Plan plan;
    __shared__ uint16_t lists[kMoeWaves][KMQ_MOE_MAX_ROWS];
    __shared__ u32x2_t masks[BITS == 1 ? 16 : 1];
    __shared__ Table tables[BITS == 4 ? kMoeWaves : 1];
    extern __shared__ float sums[];                       // [wave][token][16 rows]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    if constexpr (BITS == 1) fill_masks(masks);
    for (int i = threadIdx.x; i < kMoeWaves * a.rows * 16; i += kMoeThreads) sums[i] = 0.f;
    make_plan(a, plan);
    const int block = blockIdx.x, units = static_cast<int>(a.width / G::COLUMNS);
    const int all = plan.experts * units;
    const int from = static_cast<int>(static_cast<int64_t>(all) * wave / kMoeWaves), to = static_cast<int>(static_cast<int64_t>(all) * (wave + 1) / kMoeWaves);
    const Rows hr = rows_at(a.workspace);
    float* mine = sums + wave * a.rows * 16;
    Table& table = tables[BITS == 4 ? wave : 0];
    for (int done = from; done < to;) {
        const int which = done / units, u0 = done - which * units, u1 = units < u0 + to - done ? units : u0 + to - done;
        done += u1 - u0;
        const int e = __builtin_amdgcn_readfirstlane(plan.list[which]);
        const Matrix m = matrix_of<BITS>(a.down, e, block, units, lane);
        const int count = pairs_of(plan, a.rows * a.top_k, e, lists[wave]);
        const uint16_t* book = a.down.books + (e << BITS);
        const Centroids<BITS> c = centroids_of<BITS>(book);
        if constexpr (BITS == 4) {
            fill_table(table, book, 0, 1, lane);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        for (int first = 0; first < count; first += 16 * CT) {
            uint32_t at[CT];
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                const int i = first + 16 * t + n;
                at[t] = i < count ? static_cast<uint32_t>(lists[wave][i]) * static_cast<uint32_t>(a.width * 2) + 16u * q : kNoRow;
            }
            f32x4_t acc[CT];
#pragma unroll
            for (int t = 0; t < CT; ++t) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            Granule<BITS> g;
            load_granule<BITS>(m, u0, g);
            for (int u = u0; u < u1; ++u) {
                Granule<BITS> next = g;
#pragma unroll
                for (int k = 0; k < G::STEPS / 4; ++k) {
                    u32x4_t x[CT][4];
#pragma unroll
                    for (int t = 0; t < CT; ++t)
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[t][j] = load_row16(hr, at[t] + 64 * j, (u * G::COLUMNS + 128 * k) * 2);
                    if (k == 0) load_granule<BITS>(m, u + 1 < u1 ? u + 1 : u, next);
                    multiply<BITS, CT>(g, c, &table[0][lane], masks, x, k, acc);
                }
                g = next;
            }
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int column = first + 16 * t + 4 * q + i;
                    if (column < count) {
                        const int p = lists[wave][column];
                        float* s = mine + (p / a.top_k) * 16 + n;
                        *s = fmaf(plan.weight[p], acc[t][i], *s);
                    }
                }
        }
    }
    __syncthreads();
    for (int o = threadIdx.x; o < a.rows * 16; o += kMoeThreads) {
        const int64_t m = o >> 4, row = static_cast<int64_t>(block) * 16 + (o & 15);
        if (row >= a.hidden) continue;
        float s = a.residual ? bf16_to_f32(a.residual[m * a.residual_stride + row]) : 0.f;
        for (int w = 0; w < kMoeWaves; ++w) s += sums[w * a.rows * 16 + o];
        a.y[m * a.y_stride + row] = f32_to_bf16(s);
    }
}

}  // namespace

size_t moe_workspace_bytes(int64_t rows, int64_t top_k, int64_t width) { return static_cast<size_t>(rows * top_k * width * 2); }

template <int BITS, int CT>
static void launch_moe_bits(const MoeArgs& a, hipStream_t s) {
    const int64_t pairs = static_cast<int64_t>(a.rows) * a.top_k, most = (pairs < a.experts ? pairs : a.experts) * ((a.gate.rows + 15) / 16);
    moe_gate_up_kernel<BITS, CT><<<dim3(static_cast<unsigned>(most < 1024 ? most : 1024)), kMoeThreads, 0, s>>>(a);
    moe_down_kernel<BITS, CT><<<dim3(static_cast<unsigned>((a.hidden + 15) / 16)), kMoeThreads, kMoeWaves * a.rows * 16 * sizeof(float), s>>>(a);
}

hipError_t launch_moe(const MoeArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    const bool few = a.rows <= 16;
    switch (a.bits) {
        case 1: few ? launch_moe_bits<1, 1>(a, s) : launch_moe_bits<1, 4>(a, s); break;
        case 2: few ? launch_moe_bits<2, 1>(a, s) : launch_moe_bits<2, 4>(a, s); break;
        case 3: few ? launch_moe_bits<3, 1>(a, s) : launch_moe_bits<3, 4>(a, s); break;
        default: few ? launch_moe_bits<4, 1>(a, s) : launch_moe_bits<4, 4>(a, s); break;
    }
    return hipGetLastError();
}

}  // namespace kmq
