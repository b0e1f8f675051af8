// Shared-prefix attention's plan: blocks of 128 rows and a range of keys, as plain functions of
// sizes.  (Apart from the other launch rules, whose text the recorded traffic of the indexer is tied to.)
#pragma once

#include <stdint.h>

namespace janus {

constexpr int PA_ROWS = 128;  // (token, head) rows of a block
constexpr int PA_XCD = 8;
constexpr int PA_CUS = 256;
// Keys of a range at most.  A block's O is rounded to fp32 once for 16 keys: over n of them that score alike it
// may be off by n / 16 * 2^-25 of sum p |v|, 2^-10 here (measured in one range: 2^-9 at 2^20 keys, 3% at 2^24).
constexpr int PA_LONGEST = 1 << 19;
constexpr int64_t PA_MAX_BLOCKS = (1 << 24) - 1;  // a launch takes fewer than 2^32 threads

// First tile of session s's own rows, whose tokens start at q_start: each session has as
// many tiles as its rows fill, or one more, and none needs the sessions before
// its own.  (With 128 heads every token is a tile.)
constexpr int prefix_tile_first(int q_start, int heads, int s)
{
    return (int)((int64_t)q_start * heads / PA_ROWS) + (heads % PA_ROWS != 0 ? s : 0);
}

struct PrefixPlan {
    int prefix;        // ids that rows of different sessions meet together
    int chunk;         // keys of a block
    int shared_tiles, shared_chunks;  // over the prefix
    int own_tiles, own_chunks;        // over the ids behind it
    int one;           // no session has more than a tile: tile s is session s
    int whole;         // own tiles, the first ones, that are one block each over all their keys
    int alike;         // own chunks that read the same pages in every session
    int slots;         // ranges of a row whose keys are split (1: none is)
    int64_t part_rows;  // rows of each slot in the workspace
    int64_t blocks;
};

constexpr PrefixPlan prefix_plan(int num_seqs, int total_q, int max_q, int max_ctx, int64_t total_ctx, int prefix_len,
                                 int heads, bool mla)
{
    PrefixPlan p = {};
    const int64_t rows = (int64_t)total_q * heads;
    const int full = (int)((rows + PA_ROWS - 1) / PA_ROWS);  // tiles of all rows together
    // tiles of the sessions apart, at the mean length
    const int64_t each = (rows / num_seqs + PA_ROWS - 1) / PA_ROWS;
    const int64_t apart = num_seqs * (each > 1 ? each : 1);
    const bool share = prefix_len > 0 && (int64_t)full * 8 <= apart * 7;
    const int tile = 32, resident = PA_CUS * (mla ? 1 : 2);
    p.prefix = share ? prefix_len : 0;
    p.shared_tiles = share ? full : 0;
    // Tiles by session where none has more than one: with tiles that may be empty, either some CUs have
    // no block or more blocks than the chip takes at once do have rows (64 sessions of 64 MLA heads
    // on a prefix of 16384 201 us, by session 167; 32 of 32 heads on 65536 170 and 162).
    p.one = heads % PA_ROWS != 0 && (int64_t)max_q * heads <= PA_ROWS;
    p.own_tiles = p.one ? num_seqs : prefix_tile_first(total_q, heads, num_seqs);
    // Whole rounds of blocks need no split; the last tiles are split over the round that is left.
    const int own = max_ctx - p.prefix;
    const int64_t rounds = share || own > PA_LONGEST ? 0 : apart / resident;
    p.whole = (int)(rounds * resident * p.own_tiles / apart);
    const int64_t rest = apart - rounds * resident, ids = p.own_tiles - p.whole;
    const int mean = total_ctx / num_seqs > p.prefix ? (int)(total_ctx / num_seqs) - p.prefix : 0;
    const int span = own > p.prefix ? own : p.prefix;
    // Time of a split, in keys of a block.  Blocks that all run at once take as long as the
    // longest; more of them share the chip and leave half a block at the end.  (Where
    // tiles may be empty, MLA blocks run at once up to 94% of the chip: the places of
    // empty ones are not all taken again.  Without them counted, up to 4/5.)  An MQA
    // block beside another on its CU adds a third of its time.  Each block starts for 64 keys,
    // and a range of a row costs a hundredth of a key to write and read again.  Fitted
    // to 35 batches of 1 to 100 sessions.  Of 39 batches, each timed with 27 chunk lengths too, the
    // plan's time is 2.7% off the shortest in the mean for MLA and 3.7% for MQA, 15% at most (three
    // MQA batches and one of MLA by 9% and more); the shortest of 27 times is itself low by their scatter.  (Whole
    // rounds of blocks, a start of 128 or 256 keys and a join of 0.02 or 0.01: 6 and 13% in the mean of 18.)
    const double start = 64, join = 0.01, tail = 0.5, slack = 0.8, beside = mla ? 0.0 : 0.35;
    const double room = (mla && heads % PA_ROWS != 0 && !p.one ? 0.94 : 1.0) * resident;
    double best = -1.0;
    auto attempt = [&](int n) {  // n chunks over the longer part; whether more would be too many
        const int chunk = (span > n ? (span + n - 1) / n + tile - 1 : tile) / tile * tile;
        const int sc = share ? (prefix_len + chunk - 1) / chunk : 0, oc = own > 0 ? (own + chunk - 1) / chunk : 1;
        const int mine = mean > 0 ? (mean + chunk - 1) / chunk : 1;
        const double together = (double)p.shared_tiles * sc, work = together + (double)rest * mine;
        const double longest = chunk + start;
        double cost = longest;
        if (mla || work > PA_CUS)
            cost *= 1.0 + beside;
        if (together + (double)ids * oc > room && work > slack * resident) {
            const double all = (double)p.shared_tiles * (p.prefix + sc * start) + (double)rest * (mean + mine * start);
            const double spread = all * (1.0 + beside) / resident + tail * longest;
            cost = spread > cost ? spread : cost;
        }
        if (sc + oc > 1)
            cost += join * (sc + oc) * (double)(share ? rows : rest * PA_ROWS);
        if (best < 0.0 || cost < best) {
            best = cost;
            p.chunk = chunk;
            p.shared_chunks = sc;
            p.own_chunks = oc;
        }
        return chunk == tile || work > 8.0 * resident;
    };
    const int least = span / PA_LONGEST + (span % PA_LONGEST != 0);
    const int first = least > 1 ? least : 1;
    for (int n = first; (n == first || n <= 256) && !attempt(n); n += 1 + n / 16)
        ;
    // and as many as fill the chip once, with the own chunks as they are
    const double fill = share ? (room - (double)ids * p.own_chunks) / p.shared_tiles : room / (double)(ids > 0 ? ids : 1);
    if (fill > 1.0 && fill >= least)
        attempt((int)fill);
    p.slots = p.shared_chunks + p.own_chunks;
    if (p.slots == 1 || rest == 0) {
        p.whole = p.own_tiles;
        p.own_chunks = p.slots = 1;
    }
    p.alike = share || p.whole ? 0 : prefix_len / p.chunk;
    p.part_rows = p.slots == 1 ? 0 : share ? rows : (int64_t)(p.own_tiles - p.whole) * PA_ROWS;
    p.blocks = (int64_t)p.shared_tiles * p.shared_chunks + p.whole + (int64_t)(p.own_tiles - p.whole) * p.own_chunks;
    return p;
}

// Block blk of a plan.  Blocks that read the same keys are neighbours in the numbering,
// and blocks of one XCD (blk % 8) have consecutive numbers: the keys come into one L2.
struct PrefixBlock {
    bool shared;
    int tile, chunk;
    int slot;  // -1: the tile's keys are not split
};
constexpr int prefix_xcd(int blk, int n)
{
    const int x = blk % PA_XCD, per = n / PA_XCD, more = n % PA_XCD;
    return x * per + (x < more ? x : more) + blk / PA_XCD;
}
constexpr PrefixBlock prefix_block(const PrefixPlan &p, int blk)
{
    const int together = p.shared_tiles * p.shared_chunks;
    if (blk < together) {
        const int id = prefix_xcd(blk, together), c = id / p.shared_tiles;
        return {true, id - c * p.shared_tiles, c, c};
    }
    blk -= together;
    if (blk < p.whole)
        return {false, blk, 0, -1};
    blk -= p.whole;
    const int tiles = p.own_tiles - p.whole, alike = tiles * p.alike;
    const int id = blk < alike ? prefix_xcd(blk, alike) : blk, c = id / tiles;
    return {false, p.whole + id - c * tiles, c, p.shared_chunks + c};
}

} // namespace janus
