// The paged-cache calls' sizes and cuts (plain arithmetic) for the tests to call.
#define __host__
#define __device__
#define __forceinline__ inline
#include "../paper_2503_00784_amd/csrc/duo_page_rules.h"

extern "C" {

void layout(int requests, int max_rows, int max_new, int max_blocks, int hq, int hkv, int D, long long* out) {
    const PageLayout l = page_layout(requests, max_rows, max_new, max_blocks, hq, hkv, D);
    const long long v[] = {l.stream_items, l.tile_items, l.stream_parts, l.tile_parts, l.merges, l.stream_rows, (long long)l.info, (long long)l.stream,
                           (long long)l.tile, (long long)l.merge, (long long)l.part_stream, (long long)l.part_tile, (long long)l.total};
    for (int i = 0; i < 13; ++i) out[i] = v[i];
}

// What a plan of these requests (cached, new rows) makes of the attention: items, partial results and merges as the planning kernels count them.
void cut(int count, const int* cached, const int* rows, int max_new, int max_blocks, int hq, int hkv, int* out) {
    const int group = hq / hkv;
    long long work[2] = {0, 0};
    for (int r = 0; r < count; ++r) {
        const PageWork w = page_work(cached[r], rows[r], group);
        work[w.streamed ? 0 : 1] += (long long)w.tiles * w.blocks;
    }
    const int range[2] = {page_stream_range(work[0], hkv, page_stream_cut(max_new, group), max_blocks),
                          page_range(work[1], hkv, PAGE_TILE_TARGET, PAGE_TILE_MIN_BLOCKS)};
    int items[2] = {0, 0}, parts[2] = {0, 0}, merges = 0, covered = 1;
    for (int r = 0; r < count; ++r) {
        const PageWork w = page_work(cached[r], rows[r], group);
        if (w.tiles == 0) continue;
        const int kind = w.streamed ? 0 : 1, chunks = page_chunks(w.blocks, range[kind]);
        items[kind] += w.tiles * chunks;
        if (chunks > 1) parts[kind] += w.tiles * chunks, merges += page_merge_entries(rows[r] * group, chunks);
        for (int t = 0; t < w.tiles; ++t) {  // the ranges of a tile cover what its rows see, once
            const int first = t * PAGE_TILE_ROWS, pairs = rows[r] * group;
            const int n = w.streamed ? pairs : (pairs - first < PAGE_TILE_ROWS ? pairs - first : PAGE_TILE_ROWS);
            const int blocks = page_tile_blocks(cached[r], first, n, group), length = page_chunk_blocks(blocks, chunks);
            if (length * chunks < blocks || blocks > w.blocks || length < 1) covered = 0;
        }
    }
    const int v[] = {items[0], items[1], parts[0], parts[1], merges, covered};
    for (int i = 0; i < 6; ++i) out[i] = v[i];
}
}
