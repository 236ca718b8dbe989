// Sizes and schedules of the paged-cache calls: plain arithmetic without a word of HIP but for the qualifiers of what a kernel calls too, so
// that a program without a GPU can evaluate them.
#pragma once
#include <stddef.h>
#include <stdint.h>

// The attention of a step is cut into items, one workgroup for each of them and each kv head.  An item is a tile of query rows (row = token
// of the request * group + query head of the group) and a range of 32-key blocks.
//   Streamed: up to PAGE_STREAM_ROWS rows, the whole request in one tile.  The cache is read once and bounds the time, so the waves of a
//     workgroup take different blocks.
//   Tiled: more rows, tiles of PAGE_TILE_ROWS.  The matrix units bound the time, so the waves take different rows and share the blocks in LDS.
constexpr int PAGE_STREAM_ROWS = 64;
constexpr int PAGE_TILE_ROWS = 128;
// Workgroups that the key ranges are cut for (fewer rows and requests than that are split over the keys), and the shortest ranges.  Streamed requests
// of more than 16 rows at most: 512 and 4, since their partial results are what a range costs (16 x 33 rows of 32 heads: 80 us, 92 with 1024; 4 x 7 rows
// * 4 behind 300 to 2000 keys: 15 us, 20 with ranges of 8 blocks or more, 29 with 16); of fewer: 1024 and 8 (8 requests behind 1500 keys: 14 us, 17 with
// ranges of 4, 19 with 32; 8 x 1 row of 32 heads behind 1000 to 4000: 52, 61 with 512).
// A batch whose requests have room for `whole` blocks at most is not cut, since a second launch joins ranges.  Uncut against cut, replayed graphs, us:
//   up to 16 rows, 9 rows of 32 heads behind 100, 512, 750, 1000 and 2000 keys: 5.3 7.9 9.8 12.4 21.0 against 7.0 9.9 10.0 10.4 12.0; 8 requests of
//   one row, 32 heads over 8: 5.2 8.9 10.3 13.4 23.3 against 7.2 9.6 10.0 10.4 15.5: they cross at about 24 blocks;
//   more rows, 33 of 32 heads behind 100, 200, 300 and 512: 10.9 14.4 17.6 25.1 against 11.3 13.2 13.1 14.3; 17 of 12 heads of 64: 5.9 7.4 8.2 11.3
//   against 7.5 9.2 9.2 10.5: between 4 and 12 blocks.
// (Steps whose workgroups fill the card uncut do not need ranges at any length: 8 x 9 rows of 32 heads behind 2000 keys 43 against 49.)
// Short requests in a table with room for more are cut all the same: the joining launch is there anyway, and what it costs them is the difference
// above (2 us at 512 keys).  With it, ranges are the faster form (30 x 1 row behind 100 to 1000 keys: 14 us, 20 in whole ranges).
struct PageCut {
    int target, least, whole;
};
__host__ __device__ __forceinline__ PageCut page_stream_cut(int max_new, int group) {
    return (long long)max_new * group <= 16 ? PageCut{1024, 8, 24} : PageCut{512, 4, 8};
}
// Tiled: one workgroup a compute unit, though two fit there at heads of 128 and three at 64, since a partial result of 128 rows is 67 or 35 KB to
// write and to read again.  With 256, 512 and 128, replayed graphs: 24 streams beside three chunks of 400 to 1000 rows, heads of 64: 37, 42, 36 us;
// 128 rows of 32 heads behind 30000 keys: 27, 37, 31; 512 rows of 32 heads behind 3000: 28.5, 30.5, 29.4; 64 decoding requests beside a chunk of 512
// rows: 135, 149, 122 (there the streams want the card).
constexpr int PAGE_TILE_TARGET = 256, PAGE_TILE_MIN_BLOCKS = 16;

// Limits that keep every sum of a plan inside 32 bits: 4096 requests of 2^18 rows, 2^18 pages or 2^18 blocks each.
constexpr int PAGE_MAX_REQUESTS = 4096, PAGE_MAX_ROWS = 1 << 18, PAGE_MAX_SLOTS = 1 << 23;

struct PageWork {       // what a request asks of the attention, and how it is cut
    int blocks;         // 32-key blocks of all its slots
    int tiles;          // tiles of query rows; 0: nothing to do
    bool streamed;
};
__host__ __device__ __forceinline__ PageWork page_work(int cached, int rows_new, int group) {
    PageWork w;
    w.blocks = (cached + rows_new + 31) / 32;
    w.streamed = rows_new * group <= PAGE_STREAM_ROWS;
    w.tiles = rows_new == 0 ? 0 : w.streamed ? 1 : (rows_new * group + PAGE_TILE_ROWS - 1) / PAGE_TILE_ROWS;
    return w;
}
// Longest key range, in blocks, for `work` = sum of tiles * blocks over the requests of a kind: work / range is then at most target / heads.
__host__ __device__ __forceinline__ int page_range(long long work, int heads, int target, int least) {
    const long long r = (work * heads + target - 1) / target;
    return r < least ? least : (int)r;
}
__host__ __device__ __forceinline__ int page_stream_range(long long work, int heads, const PageCut& cut, int max_blocks) {
    return max_blocks <= cut.whole ? cut.whole : page_range(work, heads, cut.target, cut.least);
}
__host__ __device__ __forceinline__ int page_chunks(int blocks, int range) { return (blocks + range - 1) / range; }
// A tile that sees `blocks` blocks is cut into at most `chunks` ranges of this length.
__host__ __device__ __forceinline__ int page_chunk_blocks(int blocks, int chunks) { return (blocks + chunks - 1) / chunks; }
// Joining the ranges of a tile: a workgroup and head takes this many rows, fewer where a row has many ranges.
constexpr int PAGE_MERGE_RANGES = 8;
__host__ __device__ __forceinline__ int page_merge_rows(int chunks) { return chunks > PAGE_MERGE_RANGES ? 1 : 16; }
__host__ __device__ __forceinline__ int page_merge_entries(int pairs, int chunks) { return (pairs + page_merge_rows(chunks) - 1) / page_merge_rows(chunks); }
static_assert(PAGE_TILE_ROWS % 16 == 0 && PAGE_STREAM_ROWS % 16 == 0, "an entry's rows are of one tile");
// Blocks that the rows [first, first + count) of a request see.
__host__ __device__ __forceinline__ int page_tile_blocks(int cached, int first, int count, int group) { return (cached + (first + count - 1) / group) / 32 + 1; }

// Where things lie in the workspace, and how many of each there can be whatever the lengths are.
//   items of a kind: sum of tiles * ceil(blocks / range) <= work / range + sum of tiles <= target / heads + tiles
//   ranges of requests that are cut: ceil(blocks / range) <= 2 blocks / range there, so at most 2 target / heads of them
struct PageLayout {
    int stream_items, tile_items, stream_parts, tile_parts, merges;
    int stream_rows;  // rows kept per streamed partial result
    size_t info, released, stream, tile, merge, part_stream, part_tile, total;
};
constexpr int PAGE_HEADER_INTS = 64, PAGE_INFO_INTS = 16, PAGE_ITEM_INTS = 16, PAGE_MERGE_INTS = 8;

inline PageLayout page_layout(int requests, int max_rows, int max_new, int max_blocks, int hq, int hkv, int D) {
    const int group = hq / hkv;
    const bool tiles_possible = (long long)max_new * group > PAGE_STREAM_ROWS;
    PageLayout l;
    const PageCut cut = page_stream_cut(max_new, group);
    l.stream_items = cut.target / hkv + requests;
    l.stream_parts = max_blocks > cut.whole ? 2 * cut.target / hkv : 0;
    // a tiled request has more than PAGE_STREAM_ROWS rows
    const long long all = (long long)max_rows * group;
    const long long tiled_requests = all / (PAGE_STREAM_ROWS + 1) < requests ? all / (PAGE_STREAM_ROWS + 1) : requests;
    l.tile_items = tiles_possible ? (int)(PAGE_TILE_TARGET / hkv + all / PAGE_TILE_ROWS + tiled_requests) : 0;
    l.tile_parts = tiles_possible && max_blocks > PAGE_TILE_MIN_BLOCKS ? 2 * PAGE_TILE_TARGET / hkv : 0;
    const long long rows = (long long)max_new * group;
    l.stream_rows = rows >= PAGE_STREAM_ROWS ? PAGE_STREAM_ROWS : (int)((rows + 15) / 16 * 16);
    // a tile of up to R rows has 2 ranges or more and R / 16 entries at most, or 9 ranges or more and R entries: R / 8 entries a range at most
    l.merges = (l.stream_parts * PAGE_STREAM_ROWS + l.tile_parts * PAGE_TILE_ROWS) / 8;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off += (bytes + 255) / 256 * 256;
        return at;
    };
    take(PAGE_HEADER_INTS * 4);
    l.info = take((size_t)requests * PAGE_INFO_INTS * 4);
    l.released = take((size_t)requests * 4);
    l.stream = take((size_t)l.stream_items * PAGE_ITEM_INTS * 4);
    l.tile = take((size_t)l.tile_items * PAGE_ITEM_INTS * 4);
    l.merge = take((size_t)l.merges * PAGE_MERGE_INTS * 4);
    l.part_stream = take((size_t)l.stream_parts * hkv * l.stream_rows * (D + 4) * 4);
    l.part_tile = take((size_t)l.tile_parts * hkv * PAGE_TILE_ROWS * (D + 4) * 4);
    l.total = off;
    return l;
}
