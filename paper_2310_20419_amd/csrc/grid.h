// Grids of calls of any size, as plain host arithmetic.  A launch holds fewer than 2^32 threads.  Of a larger grid the runtime
// starts what the low 32 bits of its threads say and reports nothing (186 million rows looked up, 16.9 million blocks of 256: 0.8 % of
// them written, status success); it refuses the grid only where those bits are all zero.
#pragma once
#include <stdint.h>

static inline uint64_t most_blocks(uint32_t threads) { return 0xFFFFFFFFull / threads; }

// Items of one block: `wanted`, or more where `items` would need more than `room` blocks.
static inline uint64_t items_per_block(uint64_t items, uint64_t wanted, uint64_t room)
{
    const uint64_t need = (items + room - 1) / room;
    return need > wanted ? need : wanted;
}

// launch(first, blocks) for runs of blocks that are `total` together; runs start at multiples of 8, one per XCD.
template <typename F> void in_launches(uint64_t total, uint32_t threads, F launch)
{
    const uint64_t most = most_blocks(threads) / 8 * 8;
    for (uint64_t first = 0; first < total; first += most) launch(first, total - first < most ? total - first : most);
}

// Cuts `count` lists of length(i) elements into tiles, and the tiles into launches of at most `room` tiles of at most `parts` lists or parts
// of lists: part(i, first, n, tile) adds the n elements of list i from `first` on (a multiple of a tile) to the launch, whose tiles up to
// `tile` are taken; launch(tiles) sends it off.
template <typename L, typename P, typename F>
void cut_into_launches(int32_t count, uint64_t tile, uint64_t room, uint32_t parts, L length, P part, F launch)
{
    uint64_t first = 0;
    for (int32_t i = 0; i < count;) {
        uint64_t tiles = 0;
        for (uint32_t k = 0; i < count && k < parts && tiles < room;) {
            const uint64_t left = length(i) - first;
            if (left) {
                uint64_t n = (room - tiles) * tile;
                if (n > left) n = left;
                part(i, first, n, tiles);
                tiles += (n + tile - 1) / tile;
                first += n;
                ++k;
                if (n < left) break;        // (the launch is full)
            }
            first = 0;
            ++i;
        }
        if (tiles) launch(tiles);
    }
}
