// Rows looked up by id, and the gradient of the table they come from.
//
//   out[t] = scale * table[ids[t]]                               (zero where ids[t] is no row of the table)
//   grad[v] (+)= scale * sum of dout[t] over the t with ids[t] = v, in ascending t
//
// Both only move rows: a lookup reads and writes n of them, a gradient reads n and writes V (added to what is there:
// reads and writes the rows that are named).  The gradient's sums are in float32 and in an order that types, sizes and ids decide, and
// not where the rows lie: up to SMALL_TOKENS tokens a block finds those of an id by itself, in one launch; more are sorted by id (stable),
// and every sum runs over neighbours in that order.  Tokens of one id that several groups of lanes share are summed by each group and the groups' sums
// added one after the other; how many groups there are goes by the accesses that aligned rows allow, also where rows are not aligned and
// are moved in shorter ones.
#include "rows.h"

// ------------------------------------------------------------------------------------------------ lookup
#define EMBED_ITEMS 4

// A block takes rows_per_block rows; a thread one piece of VEC coordinates of EMBED_ITEMS rows at a time: their ids,
// then their pieces, are on the way together.  Bound by memory: 65,536 of 300,000 rows x 768 bfloat16 33 us, 500,003 of 1,000,000 x 96
// float32 to bfloat16 38 us (4.1 and 3.9 TB/s of the bytes that a call cannot do without; a large copy makes 5.2); one row 8 us, of
// which the kernel is 1.5.
template <int DT, int OT, int VEC>
__global__ __launch_bounds__(256) void k_embed(const void *__restrict__ table, u32 V, u32 pieces, const int *__restrict__ ids,
                                               u64 n, float scale, void *__restrict__ out, u32 rows_per_block)
{
    const u64 row0 = (u64)blockIdx.x * rows_per_block;
    const u32 rows = (u32)(n - row0 < rows_per_block ? n - row0 : rows_per_block);
    const u32 total = rows * pieces;
    for (u32 base = threadIdx.x; base < total; base += 256 * EMBED_ITEMS) {
        int id[EMBED_ITEMS];
        u32 row[EMBED_ITEMS], piece[EMBED_ITEMS];
        Pack<DT, VEC> p[EMBED_ITEMS];
#pragma unroll
        for (int i = 0; i < EMBED_ITEMS; ++i) {
            const u32 at = base + 256 * i;
            row[i] = at / pieces;
            piece[i] = at - row[i] * pieces;
            id[i] = at < total ? ids[row0 + row[i]] : -1;
        }
#pragma unroll
        for (int i = 0; i < EMBED_ITEMS; ++i)
            if ((u32)id[i] < V) p[i] = load_pack<DT, VEC>(table, ((u64)(u32)id[i] * pieces + piece[i]) * VEC);
#pragma unroll
        for (int i = 0; i < EMBED_ITEMS; ++i) {
            if (base + 256 * i >= total) break;
            float x[VEC];
            unpack<DT, VEC>(p[i], x);
#pragma unroll
            for (int k = 0; k < VEC; ++k) x[k] = (u32)id[i] < V ? x[k] * scale : 0.0f;
            store_pack<OT, VEC>(out, ((row0 + row[i]) * pieces + piece[i]) * VEC, x);
        }
    }
}

template <int DT, int OT>
static void launch_embed(const void *table, int64_t V, int d, const int32_t *ids, int64_t n, float scale, void *out, hipStream_t st)
{
    const int vec = row_vec(d, table, dt_size(DT), out, dt_size(OT));
    const u32 pieces = d / vec;
    // one trip per block; small calls: one row per block at least
    const u64 rows = items_per_block(n, (256 * EMBED_ITEMS + pieces - 1) / pieces, most_blocks(256));
    const dim3 grid((u32)((n + rows - 1) / rows));
#define RNND_EMBED(VEC) hipLaunchKernelGGL((k_embed<DT, OT, VEC>), grid, dim3(256), 0, st, table, (u32)V, pieces, ids, (u64)n, scale, out, (u32)rows)
    switch (vec) {
    case 8: RNND_EMBED(8); break;
    case 4: RNND_EMBED(4); break;
    case 2: RNND_EMBED(2); break;
    default: RNND_EMBED(1);
    }
#undef RNND_EMBED
}

#define RNND_FOR_TYPES(A, B, F)                                   \
    switch ((A) * 4 + (B)) {                                      \
    case RNND_F32 * 4 + RNND_F32: F(DT_F32, DT_F32); break;       \
    case RNND_F32 * 4 + RNND_F16: F(DT_F32, DT_F16); break;       \
    case RNND_F32 * 4 + RNND_BF16: F(DT_F32, DT_BF16); break;     \
    case RNND_F16 * 4 + RNND_F32: F(DT_F16, DT_F32); break;       \
    case RNND_F16 * 4 + RNND_F16: F(DT_F16, DT_F16); break;       \
    case RNND_F16 * 4 + RNND_BF16: F(DT_F16, DT_BF16); break;     \
    case RNND_BF16 * 4 + RNND_F32: F(DT_BF16, DT_F32); break;     \
    case RNND_BF16 * 4 + RNND_F16: F(DT_BF16, DT_F16); break;     \
    default: F(DT_BF16, DT_BF16);                                 \
    }

static int check_rows(int64_t V, int32_t d, int64_t n, int type_a, int type_b)
{
    if (!row_type(type_a) || !row_type(type_b)) return RNND_ERR_UNSUPPORTED;
    if (V < 1 || V > 2147483646LL || d < 1 || d > RNND_MAX_ROW || n < 0 || n > 2147483646LL) return RNND_ERR_BAD_SHAPE;
    return RNND_OK;
}

extern "C" int rnnd_embed(const void *table, int64_t V, int32_t d, int dtype, const int32_t *ids, int64_t n, float scale,
                          void *out, int out_dtype, void *stream)
{
    const int rc = check_rows(V, d, n, dtype, out_dtype);
    if (rc) return rc;
    if (!table || (n && (!ids || !out))) return RNND_ERR_NULL;
    if ((uintptr_t)table % dt_size(dtype) || (uintptr_t)ids % 4 || (uintptr_t)out % dt_size(out_dtype)) return RNND_ERR_BAD_PARAM;
    if (!n) return RNND_OK;
#define RNND_F(A, B) launch_embed<A, B>(table, V, d, ids, n, scale, out, (hipStream_t)stream)
    RNND_FOR_TYPES(dtype, out_dtype, RNND_F)
#undef RNND_F
    return launched("rnnd_embed");
}

// ------------------------------------------------------------------------------------------------ tokens sorted by id
// Pairs (id, token), least significant digit first, up to SORT_BITS bits a pass, three launches each: every block counts its
// digits, the counts become sums over the blocks before, every block places its tokens.  A block's order
// is kept (stable) because its wavefronts number equal digits lane by lane, with a ballot per bit.  An id that is no row
// sorts as V, behind all rows.
#define SORT_BITS 10
#define SORT_DIGITS (1 << SORT_BITS)
#define SORT_THREADS 512
#define SORT_WAVES (SORT_THREADS / 64)
#define SORT_ITEMS 4
#define SORT_TILE (SORT_THREADS * SORT_ITEMS)
#define SORT_DIRECT 64          // blocks up to which each sums the counts of all by itself, instead of a launch that does it once

struct SortPass {
    const int *ids;             // first pass: the caller's ids; else null
    const uint2 *in;            // (key, token)
    uint2 *out;
    u32 *hist;                  // [blocks][digits]: a block's own lie together, so that it writes and reads whole lines
    u32 *totals;                // [digits]
    unsigned char *named;       // first pass: set to 1 for every row that an id names (may be null)
    u32 *clear;                 // first pass: `clear_words` words that are set to zero beside the count, by the blocks behind it
    u32 clear_words;
    u32 n, V, blocks;
    int shift, bits, direct;    // direct: k_sort_place sums the counts itself
};

__device__ __forceinline__ u32 id_key(int id, u32 V) { return (u32)id < V ? (u32)id : V; }

// the lanes of `on` that hold the same digit
__device__ __forceinline__ u64 same_digit(u32 digit, int bits, bool on)
{
    u64 same = __ballot(on);
    for (int b = 0; b < bits; ++b) {
        const bool bit = digit >> b & 1;
        const u64 set = __ballot(bit);
        same &= bit ? set : ~set;
    }
    return same;
}

// One addition for the lanes of a digit: ids are popular or not, and of the high digits a few take most tokens; 64 additions to one
// word one after the other took twice the time of the ballots.
__global__ __launch_bounds__(SORT_THREADS) void k_sort_count(SortPass s)
{
    __shared__ u32 count[SORT_DIGITS];
    if (blockIdx.x >= s.blocks) {
        for (size_t i = (size_t)(blockIdx.x - s.blocks) * SORT_THREADS + threadIdx.x; i < s.clear_words; i += (size_t)(gridDim.x - s.blocks) * SORT_THREADS)
            s.clear[i] = 0;
        return;
    }
    const u32 digits = 1u << s.bits;
    for (u32 i = threadIdx.x; i < digits; i += SORT_THREADS) count[i] = 0;
    __syncthreads();
    const u32 base = blockIdx.x * SORT_TILE;
    u32 key[SORT_ITEMS];
#pragma unroll
    for (int i = 0; i < SORT_ITEMS; ++i) {
        const u32 t = base + i * SORT_THREADS + threadIdx.x;
        key[i] = t < s.n ? s.ids ? id_key(s.ids[t], s.V) : s.in[t].x : 0;
    }
#pragma unroll
    for (int i = 0; i < SORT_ITEMS; ++i) {
        const bool on = base + i * SORT_THREADS + threadIdx.x < s.n;
        const u32 digit = (key[i] >> s.shift) & (digits - 1);
        const u64 same = same_digit(digit, s.bits, on);
        if (on && (same & lanes_below(threadIdx.x & 63)) == 0) atomicAdd(&count[digit], (u32)__popcll(same));
    }
    __syncthreads();
    for (u32 i = threadIdx.x; i < digits; i += SORT_THREADS) s.hist[((size_t)blockIdx.x << s.bits) + i] = count[i];
}

__device__ __forceinline__ u32 wave_inclusive(u32 v, int lane)
{
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const u32 o = __shfl_up(v, k);
        if (lane >= k) v += o;
    }
    return v;
}

// Exclusive sums of every digit's counts over the blocks: 64 digits (two lines of each block's counts) for a workgroup,
// whose wavefronts take a run of blocks each.
#define OFFSET_WAVES 16
__global__ __launch_bounds__(64 * OFFSET_WAVES) void k_sort_offsets(SortPass s)
{
    __shared__ u32 sums[OFFSET_WAVES][64];
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6, digit = blockIdx.x * 64 + lane;
    const bool on = digit < 1u << s.bits;
    const u32 each = (s.blocks + OFFSET_WAVES - 1) / OFFSET_WAVES;
    const u32 begin = wave * each < s.blocks ? wave * each : s.blocks, end = s.blocks - begin < each ? s.blocks : begin + each;
    u32 *const h = s.hist + digit;
    u32 sum = 0;
    if (on)
#pragma unroll 8
        for (u32 b = begin; b < end; ++b) sum += h[(size_t)b << s.bits];
    sums[wave][lane] = sum;
    __syncthreads();
    u32 at = 0, all = 0;
#pragma unroll
    for (u32 w = 0; w < OFFSET_WAVES; ++w) {
        if (w == wave) at = all;
        all += sums[w][lane];
    }
    if (!on) return;
    if (wave == 0) s.totals[digit] = all;
    for (u32 b = begin; b < end; b += 8) {
        u32 v[8];
#pragma unroll
        for (u32 i = 0; i < 8; ++i) v[i] = b + i < end ? h[(size_t)(b + i) << s.bits] : 0;
#pragma unroll
        for (u32 i = 0; i < 8; ++i) {
            if (b + i < end) h[(size_t)(b + i) << s.bits] = at;
            at += v[i];
        }
    }
}

__global__ __launch_bounds__(SORT_THREADS) void k_sort_place(SortPass s)
{
    constexpr int PER = SORT_DIGITS / SORT_THREADS;     // digits of a thread
    __shared__ u32 count[SORT_WAVES][SORT_DIGITS];
    __shared__ u32 wave_total[SORT_WAVES];
    const u32 digits = 1u << s.bits;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (u32 i = threadIdx.x; i < SORT_WAVES * SORT_DIGITS; i += SORT_THREADS) (&count[0][0])[i] = 0;
    // a wavefront owns SORT_ITEMS * 64 neighbouring tokens, so that its order is the order of the input
    const u32 base = blockIdx.x * SORT_TILE + wave * (64 * SORT_ITEMS);
    uint2 item[SORT_ITEMS];
    u32 rank[SORT_ITEMS];
#pragma unroll
    for (int i = 0; i < SORT_ITEMS; ++i) {
        const u32 t = base + i * 64 + lane;
        item[i] = make_uint2(0, 0);
        if (t < s.n) item[i] = s.ids ? make_uint2(id_key(s.ids[t], s.V), t) : s.in[t];
        if (s.named && t < s.n && item[i].x < s.V) s.named[item[i].x] = 1;
    }
    // where each digit starts: exclusive sums of the totals, and of this block's counts
    u32 first[PER], ahead_of[PER] = {}, total[PER] = {}, mine = 0;
    if (s.direct) {     // (2^bits counts of a block, bits > 0: a thread's digits are all there or none)
        typedef u32 Counts __attribute__((ext_vector_type(PER)));
        const u32 digit = threadIdx.x * PER;
        for (u32 b0 = 0; b0 < s.blocks; b0 += 16) {
            Counts v[16];
#pragma unroll
            for (u32 i = 0; i < 16; ++i)
                if (b0 + i < s.blocks && digit < digits) v[i] = *(const Counts *)&s.hist[((size_t)(b0 + i) << s.bits) + digit];
                else v[i] = Counts{};
#pragma unroll
            for (u32 i = 0; i < 16; ++i)
#pragma unroll
                for (int k = 0; k < PER; ++k) {
                    total[k] += v[i][k];
                    ahead_of[k] += b0 + i < blockIdx.x ? v[i][k] : 0;
                }
        }
    } else
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const u32 digit = threadIdx.x * PER + k;
            if (digit >= digits) continue;
            total[k] = s.totals[digit];
            ahead_of[k] = s.hist[((size_t)blockIdx.x << s.bits) + digit];
        }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        first[k] = mine;
        mine += total[k];
    }
    const u32 inc = wave_inclusive(mine, lane);
    if (lane == 63) wave_total[wave] = inc;
    __syncthreads();
    u32 before_waves = inc - mine;
    for (int w = 0; w < wave; ++w) before_waves += wave_total[w];
#pragma unroll
    for (int k = 0; k < PER; ++k) first[k] += before_waves + ahead_of[k];
#pragma unroll
    for (int i = 0; i < SORT_ITEMS; ++i) {
        const bool on = base + i * 64 + lane < s.n;
        const u32 digit = (item[i].x >> s.shift) & (digits - 1);
        const u64 same = same_digit(digit, s.bits, on);
        const u32 ahead = __popcll(same & lanes_below(lane));
        u32 before = 0;
        if (on) before = count[wave][digit];
        wave_sync();
        if (on && ahead == 0) count[wave][digit] = before + __popcll(same);
        wave_sync();
        rank[i] = before + ahead;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        u32 at = first[k];
        for (int w = 0; w < SORT_WAVES; ++w) {
            const u32 n = count[w][threadIdx.x * PER + k];
            count[w][threadIdx.x * PER + k] = at;
            at += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SORT_ITEMS; ++i)
        if (base + i * 64 + lane < s.n) s.out[count[wave][(item[i].x >> s.shift) & (digits - 1)] + rank[i]] = item[i];
}

// ------------------------------------------------------------------------------------------------ gradient
// The sorted tokens are cut into chunks.  A lane takes VEC coordinates of a chunk (no lane needs another, so they are counted
// through, whatever the length of a row), and sums the rows of one id after the other.  An id whose tokens end at most one chunk behind the chunk they start in is summed by
// that chunk's lanes alone (they read on, and the next chunk's leave them out).  A longer one -- words as frequent as "the" --
// leaves one partial sum per chunk, which k_grad_join adds in order, a whole block for each such id and slab.
// Bound by memory, but for the sort before it (two passes for 300,000 or 1,000,000 rows): 1,000,000 x 96 float32 235 us, of which the sums
// are 168 (768 MB, 4.6 TB/s) and the sort 63; 100,003 x 768 bfloat16 added to 300,000 float32 rows 145 us, sums 83, sort 33.
#define GRAD_UNROLL 8       // divides every chunk
#define GRAD_SLOTS 2        // partial sums of a chunk: 0 = of an id that started before it, 1 = of the id that goes on after it
#define JOIN_THREADS 512

struct GradPar {
    const void *dout;
    const uint2 *item;          // sorted (key, token)
    void *grad;
    float *partial;             // [chunks][GRAD_SLOTS][d]
    u32 *hot;                   // [0] how many, [1 ..] chunks in which a long id starts
    const unsigned char *named; // [V] whether a row is named (the others are cleared here)
    u32 n, V, chunk, chunks, pieces, slabs, reduce_blocks, clear_rows;
    int accumulate;
    float scale;
};

template <int GT, int VEC>
__device__ __forceinline__ void grad_write(const GradPar &g, u32 id, u32 piece, float (&acc)[VEC])
{
    const u64 at = ((u64)id * g.pieces + piece) * VEC;
#pragma unroll
    for (int k = 0; k < VEC; ++k) acc[k] *= g.scale;
    if (g.accumulate) {
        float old[VEC];
        unpack<GT, VEC>(load_pack<GT, VEC>(g.grad, at), old);
#pragma unroll
        for (int k = 0; k < VEC; ++k) acc[k] += old[k];
    }
    store_pack<GT, VEC>(g.grad, at, acc);
}

template <int DT, int GT, int VEC>
__global__ __launch_bounds__(256) void k_grad_reduce(GradPar g)
{
    if (blockIdx.x >= g.reduce_blocks) {        // the other blocks clear the rows that no token names, clear_rows each
        const float zero[VEC] = {};
        const u64 v0 = (u64)(blockIdx.x - g.reduce_blocks) * g.clear_rows;
        const u32 rows = (u32)(g.V - v0 < g.clear_rows ? g.V - v0 : g.clear_rows);
        for (u32 i = threadIdx.x; i < rows * g.pieces; i += 256) {
            const u32 r = i / g.pieces;
            if (!g.named[v0 + r]) store_pack<GT, VEC>(g.grad, (v0 * g.pieces + i) * VEC, zero);
        }
        return;
    }
    const u64 flat = (u64)blockIdx.x * 256 + threadIdx.x;
    const u32 c = (u32)(flat / g.pieces), piece = (u32)(flat - (u64)c * g.pieces);
    if (c >= g.chunks) return;
    const u64 begin64 = (u64)c * g.chunk;
    const u32 begin = (u32)begin64, end = g.n - begin < g.chunk ? g.n : begin + g.chunk, C = g.chunk;
    u32 id = g.item[begin].x;
    if (id >= g.V) return;
    const bool incoming = begin > 0 && g.item[begin - 1].x == id;
    // (sorted: the tokens of `id` end at or before position x if x is the end or holds another key)
    const bool skip = incoming && (begin - C == 0 || g.item[begin - C - 1].x != id) && ((u64)begin + C >= g.n || g.item[begin + C].x != id);
    bool first = incoming;          // still in the id that started before the chunk
    const u32 last = g.item[end - 1].x;
    const bool goes_on = end < g.n && g.item[end].x == last && last < g.V && !(incoming && last == id);
    const bool hot = goes_on && (u64)end + C < g.n && g.item[end + C].x == last;
    const u32 stop = goes_on && !hot ? (g.n - end < C ? g.n : end + C) : end;      // and no further than the key `last`

    float acc[VEC] = {};
    bool some = false;
    // the next tokens' names are fetched behind this trip's rows: a trip waits for one latency, not for two (1,000,000 x 96: 189 -> 168 us)
    uint2 ahead[GRAD_UNROLL];
#pragma unroll
    for (int i = 0; i < GRAD_UNROLL; ++i) ahead[i] = g.item[begin + i < stop ? begin + i : stop - 1];
    for (u32 t = begin; t < stop; t += GRAD_UNROLL) {
        uint2 it[GRAD_UNROLL];
        Pack<DT, VEC> row[GRAD_UNROLL];
#pragma unroll
        for (int i = 0; i < GRAD_UNROLL; ++i) it[i] = ahead[i];
#pragma unroll
        for (int i = 0; i < GRAD_UNROLL; ++i) {
            const u32 at = t + i;
            if (at >= stop || (at >= end && it[i].x != last)) it[i].x = 0xFFFFFFFFu;      // nothing there for this chunk
            if (it[i].x < g.V && !(skip && first && it[i].x == id)) row[i] = load_pack<DT, VEC>(g.dout, ((u64)it[i].y * g.pieces + piece) * VEC);
        }
#pragma unroll
        for (int i = 0; i < GRAD_UNROLL; ++i) {
            const u32 at = t + GRAD_UNROLL + i;
            ahead[i] = g.item[at < stop ? at : stop - 1];
        }
        bool done = false;
#pragma unroll
        for (int i = 0; i < GRAD_UNROLL; ++i) {
            if (done) break;
            if (it[i].x != id) {
                if (some) {
                    if (first) store_pack<DT_F32, VEC>(g.partial, ((u64)c * GRAD_SLOTS * g.pieces + piece) * VEC, acc);
                    else grad_write<GT, VEC>(g, id, piece, acc);
                }
#pragma unroll
                for (int k = 0; k < VEC; ++k) acc[k] = 0.0f;
                some = false;
                first = false;
                id = it[i].x;
                if (id >= g.V) { done = true; break; }
            }
            if (skip && first) continue;
            float x[VEC];
            unpack<DT, VEC>(row[i], x);
#pragma unroll
            for (int k = 0; k < VEC; ++k) acc[k] += x[k];
            some = true;
        }
        if (done) break;
    }
    if (!some) return;
    if (first || hot) {
        store_pack<DT_F32, VEC>(g.partial, (((u64)c * GRAD_SLOTS + (first ? 0 : 1)) * g.pieces + piece) * VEC, acc);
        if (!first && piece == 0) g.hot[1 + atomicAdd(&g.hot[0], 1u)] = c;
    } else
        grad_write<GT, VEC>(g, id, piece, acc);
}

// One block per long id and slab: its groups take every (JOIN_THREADS / G)-th partial sum, four at a time, and their sums are added
// in the groups' order.
template <int GT, int VEC, int G>
__global__ __launch_bounds__(JOIN_THREADS) void k_grad_join(GradPar g)
{
    constexpr u32 groups = JOIN_THREADS / G;
    __shared__ float part[groups][G * VEC];
    const u32 lane = threadIdx.x % G, group = threadIdx.x / G;
    const u32 work = g.hot[0] * g.slabs;
    for (u32 at = blockIdx.x; at < work; at += gridDim.x) {
        const u32 c = g.hot[1 + at / g.slabs], piece = at % g.slabs * G + lane;
        const u32 id = g.item[(u64)(c + 1) * g.chunk - 1].x;
        u32 lo = c + 1, hi = (g.n - 1) / g.chunk;      // the last chunk whose first token is of `id`: a long id fills c + 1
        while (lo < hi) {       // 64 places at a time: a wait for memory each
            const u32 step = (hi - lo + 63) / 64, left = (hi - lo) / step, ahead = (threadIdx.x & 63) + 1;
            const bool same = ahead <= left && g.item[(u64)(lo + ahead * step) * g.chunk].x == id;
            const u32 found = __popcll(__ballot(same));
            lo += found * step;
            if (found < left) hi = lo + step - 1;
        }
        const u32 chunks = lo - c + 1;
        float acc[VEC] = {};
        if (piece < g.pieces)
            for (u32 j0 = group; j0 < chunks; j0 += 4 * groups) {
                Pack<DT_F32, VEC> p[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const u32 j = j0 + u * groups;
                    if (j < chunks) p[u] = load_pack<DT_F32, VEC>(g.partial, (((u64)(c + j) * GRAD_SLOTS + (j == 0 ? 1 : 0)) * g.pieces + piece) * VEC);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (j0 + u * groups < chunks)
#pragma unroll
                        for (int k = 0; k < VEC; ++k) acc[k] += p[u].v[k];
            }
#pragma unroll
        for (int k = 0; k < VEC; ++k) part[group][lane * VEC + k] = acc[k];
        __syncthreads();
        if (group == 0 && piece < g.pieces) {
            const u32 most = groups < chunks ? groups : chunks;
            for (u32 j = 1; j < most; ++j)
#pragma unroll
                for (int k = 0; k < VEC; ++k) acc[k] += part[j][lane * VEC + k];
            grad_write<GT, VEC>(g, id, piece, acc);
        }
        __syncthreads();
    }
}

// Few tokens: one launch, without a sort.  A block for each token looks through all ids and lists the tokens of its own in order.  The blocks of
// the tokens of one id share its row: the k-th takes every slab of it whose number is k modulo how many they are, and has nothing to do if there is none.  A slab
// is what a group of lanes takes of a row; the groups of a block sum pieces of the list, and their sums are added in the groups' order.  An id of more than
// SMALL_MANY tokens has groups of 8 lanes, the more of them.  (With one block for an id and always as many lanes as a row has pieces, up to 64, 4,096 tokens of
// one id took 335 us with 768 coordinates and 3,328 with 8,192, sorted 47 and 40; now 26 and 27.)  The ids are a few KB that every block finds in its L2 -- 4,096 blocks read 64 MB of
// them -- where a sort and its joins are four launches at least that wait for each other: 1,000 x 32 10.5 us (18 sorted), 4,096 x 32 10.4
// (36), 4,096 x 768 f32 into 30,000 rows 32 (44).  The looking grows with the square of the tokens: 8,192 x 32 took 30 us, 8,192 x 768
// 94, sorted 32 and 44.  Blocks behind the first reduce_blocks clear clear_rows rows each, but for those that an id names.
#define SMALL_TOKENS 4096
#define SMALL_MANY 256
#define SMALL_SLABS 4           // blocks of a token, at most (more than 1,024 tokens fill the GPU with one each).  With 1 / 2 / 4 / 16, us: 100 tokens x 4,096 added
                                // 12.2 / 8.5 / 8.2 / 7.9, 1,000 x 4,096 17.0 / 13.3 / 14.9 / 30.2; 1,000 x 768 into 30,000 rows, written whole, 16.1 / 18.5 / 19.7 / 19.8
#define SMALL_CLEAR 8192        // rows of a block that clears, at most

template <int DT, int GT, int VEC>
__global__ __launch_bounds__(256) void k_grad_small(GradPar g, const int *__restrict__ ids, u32 log_lanes, u32 token_blocks)
{
    constexpr int ITEMS = SMALL_TOKENS / 256;
    __shared__ u64 mask[SMALL_TOKENS / 64];
    __shared__ alignas(16) unsigned short list[SMALL_TOKENS];
    __shared__ float part[256 * VEC];
    const u32 tid = threadIdx.x, lane = tid & 63;
    int id[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) id[i] = i * 256 + tid < g.n ? ids[i * 256 + tid] : -1;
    if (blockIdx.x >= g.reduce_blocks) {
        u32 *const named = (u32 *)list;         // a bit for each row: SMALL_CLEAR bits
        static_assert(SMALL_CLEAR / 8 <= sizeof list, "bits");
        const u64 v0 = (u64)(blockIdx.x - g.reduce_blocks) * g.clear_rows;
        const u32 rows = (u32)(g.V - v0 < g.clear_rows ? g.V - v0 : g.clear_rows);
        for (u32 i = tid; i < SMALL_CLEAR / 32; i += 256) named[i] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const u64 r = (u64)(u32)id[i] - v0;
            if ((u32)id[i] < g.V && r < rows) atomicOr(&named[r >> 5], 1u << (r & 31));
        }
        __syncthreads();
        const float zero[VEC] = {};
        for (u32 i = tid; i < rows * g.pieces; i += 256) {
            const u32 r = i / g.pieces;
            if (!(named[r >> 5] >> (r & 31) & 1)) store_pack<GT, VEC>(g.grad, (v0 * g.pieces + i) * VEC, zero);
        }
        return;
    }
    const u32 t = blockIdx.x / token_blocks;
    const int key = ids[t];
    if ((u32)key >= g.V) return;        // a whole block
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const bool same = id[i] == key;     // (no token: -1, which is no key)
        const u64 all = __ballot(same);
        if (lane == 0) mask[i * 4 + (tid >> 6)] = all;
    }
    __syncthreads();
    // a word's tokens follow those of the words before it: sums over the lanes, a word each
    static_assert(SMALL_TOKENS <= 64 * 64, "a word for each lane");
    const u32 mine = lane < (g.n + 63) / 64 ? __popcll(mask[lane]) : 0, upto = wave_inclusive(mine, lane);
    const u32 count = __builtin_amdgcn_readlane(upto, 63);
    // this block's number among those of its id, and its first slab
    const u32 rank = __builtin_amdgcn_readlane(upto - mine, __builtin_amdgcn_readfirstlane(t >> 6)) + __popcll(mask[t >> 6] & lanes_below(t & 63));
    if (count > SMALL_MANY) log_lanes = 3;
    const u32 lanes = 1u << log_lanes, groups = 256 >> log_lanes, slabs = (g.pieces + lanes - 1) >> log_lanes;
    const u32 first = rank * token_blocks + blockIdx.x % token_blocks;
    if (first >= slabs) return;         // a whole block
    if (count > 1) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const u32 word = i * 4 + (tid >> 6);
            const u64 all = __ballot(id[i] == key);
            const u32 before = __builtin_amdgcn_readlane(upto - mine, __builtin_amdgcn_readfirstlane(word));
            if (id[i] == key) list[before + __popcll(all & lanes_below(lane))] = (unsigned short)(i * 256 + tid);
        }
        __syncthreads();
    }
    const u32 group = tid >> log_lanes, at = tid & (lanes - 1);
    u32 each = (count + groups - 1) / groups;
    if (each < GRAD_UNROLL) each = GRAD_UNROLL;
    const u32 begin = group * each < count ? group * each : count, end = begin + each < count ? begin + each : count;
    const u32 used = (count + each - 1) / each;
    for (u32 slab = first; slab < slabs; slab += count * token_blocks) {
        const u32 piece = slab * lanes + at;
        float acc[VEC] = {};
        if (piece < g.pieces)
            for (u32 j = begin; j < end; j += GRAD_UNROLL) {
                Pack<DT, VEC> row[GRAD_UNROLL];
#pragma unroll
                for (int i = 0; i < GRAD_UNROLL; ++i)
                    if (j + i < end) row[i] = load_pack<DT, VEC>(g.dout, ((u64)(count > 1 ? list[j + i] : t) * g.pieces + piece) * VEC);
#pragma unroll
                for (int i = 0; i < GRAD_UNROLL; ++i)
                    if (j + i < end) {
                        float x[VEC];
                        unpack<DT, VEC>(row[i], x);
#pragma unroll
                        for (int k = 0; k < VEC; ++k) acc[k] += x[k];
                    }
            }
        if (used > 1) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) part[(group * lanes + at) * VEC + k] = acc[k];
            __syncthreads();
            if (group == 0)
                for (u32 o = 1; o < used; ++o)
#pragma unroll
                    for (int k = 0; k < VEC; ++k) acc[k] += part[(o * lanes + at) * VEC + k];
            __syncthreads();
        }
        if (group == 0 && piece < g.pieces) grad_write<GT, VEC>(g, (u32)key, piece, acc);
    }
}

struct GradPlan {
    u32 chunk, chunks, blocks;
    int passes, bits;
    size_t o_item[2], o_hist, o_totals, o_partial, o_hot, o_named, bytes;
};

static GradPlan grad_plan(int64_t n, int d, int64_t V)
{
    GradPlan p = {};
    if (n <= SMALL_TOKENS) {
        p.bytes = 256;          // (none of it is used)
        return p;
    }
    // Long chunks leave fewer partial sums; short calls need chunks short enough to occupy the GPU: three wavefronts per SIMD, of about
    // 256 coordinates each.
    p.chunk = 128;
    while (p.chunk > 8 && n / p.chunk * ((d + 255) / 256) < 6144) p.chunk >>= 1;
    p.chunks = (u32)((n + p.chunk - 1) / p.chunk);
    p.blocks = (u32)((n + SORT_TILE - 1) / SORT_TILE);
    int bits = 1;
    while ((V >> bits) != 0) ++bits;          // keys 0 .. V
    p.passes = (bits + SORT_BITS - 1) / SORT_BITS;
    p.bits = (bits + p.passes - 1) / p.passes;
    size_t off = 0;
    auto take = [&](size_t b) { const size_t o = off; off += ws_align(b); return o; };
    for (int i = 0; i < 2; ++i) p.o_item[i] = take((size_t)n * 8);
    p.o_hist = take((size_t)SORT_DIGITS * p.blocks * 4);
    p.o_totals = take(SORT_DIGITS * 4);
    p.o_partial = take((size_t)p.chunks * GRAD_SLOTS * d * 4);
    p.o_named = take((size_t)V);
    p.o_hot = take((size_t)(p.chunks + 1) * 4);       // (right behind `named`: its first word is cleared with it)
    p.bytes = off;
    return p;
}

extern "C" int rnnd_embed_grad_workspace(int64_t n, int32_t d, int64_t V, size_t *bytes)
{
    const int rc = check_rows(V, d, n, RNND_F32, RNND_F32);
    if (rc) return rc;
    if (!bytes) return RNND_ERR_NULL;
    *bytes = grad_plan(n, d, V).bytes;
    return RNND_OK;
}

template <int GT, int VEC, int G>
static void launch_join(GradPar &g, hipStream_t st)
{
    g.slabs = (g.pieces + G - 1) / G;
    const u64 units = (u64)g.chunks * g.slabs;
    hipLaunchKernelGGL((k_grad_join<GT, VEC, G>), dim3((u32)(units < 1024 ? units : 1024)), dim3(JOIN_THREADS), 0, st, g);
}
// aligned_pieces: pieces of a row whose address allows the longest accesses that d does; decides the order of the sums
template <int DT, int GT, int VEC>
static void launch_grad_vec(GradPar &g, int d, u32 aligned_pieces, const int32_t *small_ids, hipStream_t st)
{
    g.pieces = d / VEC;
    const bool clear = !g.accumulate;
    if (small_ids || !g.n) {
        u32 log_lanes = 3;
        while (log_lanes < 6 && (1u << log_lanes) < aligned_pieces) ++log_lanes;
        const u32 slabs = (g.pieces + (1u << log_lanes) - 1) >> log_lanes;
        const u32 token_blocks = g.n > 1024 ? 1 : slabs < SMALL_SLABS ? slabs : SMALL_SLABS;
        g.reduce_blocks = g.n * token_blocks;
        // 512 to 8,192 pieces for a block that clears: enough blocks, and each writes more than it reads of ids.  Always 512 / by this rule / always 8,192, us:
        // 1,000 x 768 into 30,000 rows 28.8 / 19.7 / 19.7, 4,096 x 768 33.2 / 22.6 / 22.6, 4,096 x 32 into 5,000 rows 10.2 / 10.1 / 12.4
        u32 pieces = 512;
        while (pieces < 8192 && (u64)g.V * g.pieces / pieces > 1024) pieces <<= 1;
        g.clear_rows = (u32)items_per_block(g.V, pieces / g.pieces > 1 ? pieces / g.pieces : 1, most_blocks(256) - g.reduce_blocks);
        const u32 clear_blocks = clear ? (g.V + g.clear_rows - 1) / g.clear_rows : 0;
        hipLaunchKernelGGL((k_grad_small<DT, GT, VEC>), dim3(g.reduce_blocks + clear_blocks), dim3(256), 0, st, g, small_ids, log_lanes, token_blocks);
        return;
    }
    // (at most 2^23 blocks of sums, see rnnd_embed_grad(): 2^23 at least are left for the others)
    g.reduce_blocks = (u32)(((u64)g.chunks * g.pieces + 255) / 256);
    g.clear_rows = (u32)items_per_block(g.V, 2048 / g.pieces > 1 ? 2048 / g.pieces : 1, most_blocks(256) - g.reduce_blocks);
    const u32 clear_blocks = clear ? (g.V + g.clear_rows - 1) / g.clear_rows : 0;
    hipLaunchKernelGGL((k_grad_reduce<DT, GT, VEC>), dim3(g.reduce_blocks + clear_blocks), dim3(256), 0, st, g);
    if (aligned_pieces <= 8) launch_join<GT, VEC, 8>(g, st);
    else if (aligned_pieces <= 16) launch_join<GT, VEC, 16>(g, st);
    else if (aligned_pieces <= 32) launch_join<GT, VEC, 32>(g, st);
    else launch_join<GT, VEC, 64>(g, st);
}
template <int DT, int GT>
static void launch_grad(GradPar &g, int d, const int32_t *small_ids, hipStream_t st)
{
    constexpr int MOST = DT == DT_F32 ? 4 : 8;
    const int aligned = row_vec(d, nullptr, dt_size(DT), nullptr, dt_size(GT)), vec = row_vec(d, g.dout, dt_size(DT), g.grad, dt_size(GT));
    const u32 pieces = d / (aligned < MOST ? aligned : MOST);
    if (vec >= MOST) launch_grad_vec<DT, GT, MOST>(g, d, pieces, small_ids, st);
    else if (vec == 4) launch_grad_vec<DT, GT, 4>(g, d, pieces, small_ids, st);
    else if (vec == 2) launch_grad_vec<DT, GT, 2>(g, d, pieces, small_ids, st);
    else launch_grad_vec<DT, GT, 1>(g, d, pieces, small_ids, st);
}

extern "C" int rnnd_embed_grad(const void *dout, int dtype, const int32_t *ids, int64_t n, int32_t d, float scale, int64_t V,
                               void *grad, int grad_dtype, int accumulate, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = check_rows(V, d, n, dtype, grad_dtype);
    if (rc) return rc;
    if (!grad || (n && (!dout || !ids))) return RNND_ERR_NULL;
    if (accumulate != 0 && accumulate != 1) return RNND_ERR_BAD_PARAM;
    if ((uintptr_t)dout % dt_size(dtype) || (uintptr_t)ids % 4 || (uintptr_t)grad % dt_size(grad_dtype)) return RNND_ERR_BAD_PARAM;
    if (!n && accumulate) return RNND_OK;
    const GradPlan p = grad_plan(n, d, V);
    if ((u64)p.chunks * d > (u64)256 << 23) return RNND_ERR_BAD_SHAPE;      // rows of 500 GB, which no device holds
    if (!workspace) return RNND_ERR_NULL;
    if ((uintptr_t)workspace % 16) return RNND_ERR_BAD_PARAM;
    if (workspace_bytes < p.bytes) return RNND_ERR_SCRATCH;
    hipStream_t st = (hipStream_t)stream;
    GradPar g = {};
    g.dout = dout;
    g.grad = grad;
    g.n = (u32)n;
    g.V = (u32)V;
    g.accumulate = accumulate;
    g.scale = scale;
    if (p.passes) {
        char *w = (char *)workspace;
        uint2 *item[2] = {(uint2 *)(w + p.o_item[0]), (uint2 *)(w + p.o_item[1])};
        unsigned char *named = (unsigned char *)(w + p.o_named);
        // the number of long ids, and (all rows written) which rows are named
        const size_t from = accumulate ? p.o_hot : p.o_named, words = (p.o_hot + 4 - from) / 4;
        int at = 0;
        for (int i = 0; i < p.passes; ++i) {
            SortPass s = {};
            s.ids = i ? nullptr : ids;
            s.in = item[at];
            at ^= 1;
            s.out = item[at];
            s.hist = (u32 *)(w + p.o_hist);
            s.totals = (u32 *)(w + p.o_totals);
            s.named = i || accumulate ? nullptr : named;
            s.clear = (u32 *)(w + from);
            s.clear_words = i ? 0 : (u32)words;
            s.n = (u32)n;
            s.V = (u32)V;
            s.blocks = p.blocks;
            s.shift = i * p.bits;
            s.bits = p.bits;
            s.direct = p.blocks <= SORT_DIRECT;
            const u32 clear_blocks = (s.clear_words + 2047) / 2048;
            hipLaunchKernelGGL(k_sort_count, dim3(p.blocks + (clear_blocks < 1024 ? clear_blocks : 1024)), dim3(SORT_THREADS), 0, st, s);
            if (!s.direct) hipLaunchKernelGGL(k_sort_offsets, dim3(((1u << p.bits) + 63) / 64), dim3(64 * OFFSET_WAVES), 0, st, s);
            hipLaunchKernelGGL(k_sort_place, dim3(p.blocks), dim3(SORT_THREADS), 0, st, s);
        }
        g.item = item[at];
        g.partial = (float *)(w + p.o_partial);
        g.hot = (u32 *)(w + p.o_hot);
        g.named = named;
        g.chunk = p.chunk;
        g.chunks = p.chunks;
    }
#define RNND_F(A, B) launch_grad<A, B>(g, d, p.passes ? nullptr : ids, st)
    RNND_FOR_TYPES(dtype, grad_dtype, RNND_F)
#undef RNND_F
    return launched("rnnd_embed_grad");
}
