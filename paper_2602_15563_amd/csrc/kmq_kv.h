// Layout of the paged 4-bit key / value cache and of a batch over it, for the kernels that write, read and
// attend to it.  The format is specified in include/kmq.h ("The key / value cache").
#ifndef KMQ_KV_H
#define KMQ_KV_H

#include "kmq_device.h"
#include "kmq_launch.h"

namespace kmq {

constexpr int kKvTile = 16;       // tokens per tile of a page
constexpr int kKvStep = 32;       // tokens per step of the attention kernels: two tiles of one page
constexpr int kKvCentroids = 16;

// Bytes of a tile of one head: 16 tokens of K and V at half a byte an element, and their scales.
KMQ_HD inline int kv_tile_bytes(int head_dim) { return 17 * head_dim; }

// The bf16 in a half of a register as fp32, and two fp32 as bf16 (to nearest even, NaN stays NaN).
__device__ __forceinline__ float kv_half(uint32_t v, int upper) { return __uint_as_float(upper ? v & 0xFFFF0000u : v << 16); }
__device__ __forceinline__ uint32_t kv_pack2(float a, float b) {
    const bf16x2_t v = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
    return __builtin_bit_cast(uint32_t, v);
}

// Where the row's token belongs: the sequence (-1: the row belongs to none) and the position in it, which may lie outside the cache.
struct KvRow {
    int seq;
    int64_t pos;
};

// The sequence of a row, found by all lanes of a wave together: 64 starts are read at once.
__device__ __forceinline__ KvRow kv_find_row(const KvBatchArgs& b, int64_t row) {
    if (!b.row_starts) return {static_cast<int>(row), static_cast<int64_t>(b.lengths[row]) - 1};
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1);
    int seq = 0;                                       // starts[1..] that are at most `row`
    for (int i = 0; i < b.sequences; i += kWave) {
        const int at = i + lane + 1;
        seq += __popcll(__ballot(at <= b.sequences && b.row_starts[at <= b.sequences ? at : 0] <= row));
    }
    if (seq >= b.sequences || b.row_starts[seq] > row) return {-1, 0};
    return {seq, static_cast<int64_t>(b.lengths[seq]) - b.row_starts[seq + 1] + row};
}

// Workgroups that take `size` rows-times-`each` of one sequence at a time, without a sum over the sequences before theirs: sequence b has
// the places from (row_starts[b] * each + slack * b) / size on.  With slack >= size - 1 + what may stand before a sequence's first
// row that is room for all of its pieces, and a place behind them belongs to nobody.  Found by all lanes of a wave together.
struct KvPiece {
    int seq, index;        // sequence (-1: none), piece in it (there may be no such piece)
    int start, count;      // rows of the sequence, inside the batch's
};
KMQ_HD inline int64_t kv_pieces(int64_t rows, int64_t sequences, int size, int each, int slack) { return (rows * each + slack * sequences) / size; }
__device__ __forceinline__ KvPiece kv_find_piece(const KvBatchArgs& b, int at, int size, int each, int slack) {
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1), most = static_cast<int>(b.rows);
    const int64_t reach = static_cast<int64_t>(at) * size + size - 1;
    int seq = -1;
    for (int i = 0; i < b.sequences; i += kWave) {
        const int s = i + lane;
        const int64_t first = s < b.sequences ? static_cast<int64_t>(b.row_starts[s]) * each + static_cast<int64_t>(slack) * s : reach + 1;
        seq += __popcll(__ballot(first <= reach));
    }
    if (seq < 0) return {-1, 0, 0, 0};
    const int v = b.row_starts[seq], w = b.row_starts[seq + 1];
    const int start = v < 0 ? 0 : v > most ? most : v, end = w < start ? start : w > most ? most : w;
    return {seq, at - static_cast<int>((static_cast<int64_t>(v) * each + static_cast<int64_t>(slack) * seq) / size), start, end - start};
}

// Four tokens at positions 4 i .. 4 i + 3 of a sequence, as many of them as have rows.
constexpr int kKvGroupSlack = 6;
struct KvGroup {
    int seq;               // -1: none
    int64_t row, pos;      // of the group's first token, which need not have a row
    uint32_t have;         // a bit a token
};
__device__ __forceinline__ KvGroup kv_find_group(const KvBatchArgs& b, int at) {
    const KvPiece p = kv_find_piece(b, at, 4, 1, kKvGroupSlack);
    if (p.seq < 0) return {-1, 0, 0, 0};
    const int64_t pos = static_cast<int64_t>(b.lengths[p.seq]) - b.row_starts[p.seq + 1] + p.start;
    const int64_t skip = 4 * static_cast<int64_t>(p.index) - (pos & 3);           // rows before the group's first token
    uint32_t have = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) have |= skip + r >= 0 && skip + r < p.count ? 1u << r : 0u;
    return {have ? p.seq : -1, p.start + skip, pos + skip, have};
}

// The tile of head `head` that holds position `pos` of sequence `seq`; nullptr where the page table has no page for it.
__device__ __forceinline__ uint8_t* kv_tile(const KvCacheArgs& c, const KvBatchArgs& b, int head_dim, KvRow r, int head) {
    if (r.seq < 0 || r.pos < 0 || r.pos > 0x7FFFFFFF) return nullptr;
    const int pos = static_cast<int>(r.pos), slot = pos / c.page_size;
    if (slot >= b.table_width) return nullptr;
    const int64_t page = b.page_table[static_cast<int64_t>(r.seq) * b.table_width + slot];
    if (page < 0 || page >= c.num_pages) return nullptr;
    const int64_t tile = (page * c.kv_heads + head) * (c.page_size / kKvTile) + (pos - slot * c.page_size) / kKvTile;
    return c.pages + tile * kv_tile_bytes(head_dim);
}

// Offsets in a tile, token t = 0..15.
// K: the dword of elements d..d+7 (d a multiple of 8), element d + e in nibble e.
__device__ __forceinline__ int kv_k_dword(int head_dim, int t, int d) {
    return ((d >> 4 & 3) * 16 + t) * (head_dim / 8) + (d >> 6) * 8 + (d >> 3 & 1) * 4;
}
// V: the byte of elements d (low nibble) and d + 16 (high nibble), d % 32 < 16.
__device__ __forceinline__ int kv_v_byte(int head_dim, int t, int d) {
    return 8 * head_dim + ((t >> 2) * 16 + (d & 15)) * (head_dim / 8) + (d >> 5) * 4 + (t & 3);
}
// The bf16 scale of block d / 64 of K (kv = 0) or V (kv = 1).
__device__ __forceinline__ int kv_scale(int head_dim, int t, int kv, int d) {
    return 16 * head_dim + (((t >> 2) * 2 + kv) * (head_dim / KMQ_BLOCK) + (d >> 6)) * 8 + (t & 3) * 2;
}

}  // namespace kmq

#endif
