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

// The tile of head `head` that holds position `pos` of sequence `seq`; nullptr where the page table has no page for it.
__device__ __forceinline__ uint8_t* kv_tile(const KvCacheArgs& c, const KvBatchArgs& b, int head_dim, KvRow r, int head) {
    if (r.seq < 0 || r.pos < 0) return nullptr;
    const int64_t slot = r.pos / c.page_size;
    if (slot >= b.table_width) return nullptr;
    const int64_t page = b.page_table[static_cast<int64_t>(r.seq) * b.table_width + slot];
    if (page < 0 || page >= c.num_pages) return nullptr;
    const int64_t tile = (page * c.kv_heads + head) * (c.page_size / kKvTile) + r.pos % c.page_size / kKvTile;
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
