// Rules by which the C ABI picks a kernel or the shape of a launch, as plain
// functions of sizes: they can be evaluated without a GPU.
#pragma once

#include <stdint.h>

namespace janus {

// ---- page demand: one block for all of it, or three launches -----------------

constexpr int PD_ROWS = 4;          // rows in flight per block
constexpr int RUN_THREADS = 1024;   // the one block, and the list and run kernel's
constexpr int PD_SMALL_STEPS = 2;

// Steps that one block takes over the ids, one after another: PD_ROWS rows at
// a time, four ids of each row per thread.
constexpr int64_t pd_steps(int64_t total_q, int64_t k)
{
    return ((total_q + PD_ROWS - 1) / PD_ROWS) * ((k + 4 * RUN_THREADS - 1) / (4 * RUN_THREADS));
}

// A step is a chain of dependent loads, about 2 us however few ids it has, and
// many rows would be walked by one block alone.  Measured, one block against
// three launches: 8 rows of 2048 ids 12.9 against 13 us (and two launches
// less for the host), 12 of 1024 14.9 against 12.9, 64 of 256 46 against 14,
// 256 of 64 162 against 18.  (The one block has a word of the bitmap per thread.)
constexpr bool pd_one_block(int64_t total_q, int64_t k, int nwords)
{
    return total_q > 0 && nwords > 0 && nwords <= RUN_THREADS && pd_steps(total_q, k) <= PD_SMALL_STEPS;
}

// ---- prefill indexer: key chunks of a session -----------------------------------

constexpr int IDX_XCD = 8;            // L2 domains (XCDs) of the chip
constexpr int IDX_STAGE = 128;        // keys per LDS stage
constexpr int IDX_KEY_CHUNK = 16384;  // target keys per block: long blocks spread each block's query and weight loads over more keys

// Chunks per XCD of every session: the longest session's are at most
// IDX_KEY_CHUNK keys long.  Contexts up to 2^24: at most 128.
constexpr int prefill_per_xcd(int max_ctx)
{
    const int per = ((max_ctx + IDX_XCD - 1) / IDX_XCD + IDX_KEY_CHUNK - 1) / IDX_KEY_CHUNK;
    return per > 1 ? per : 1;
}
// ceil(2^31 / n): the division by n that session_chunk makes, as a multiplication
constexpr unsigned prefill_recip(int n) { return ((1u << 31) + (unsigned)n - 1) / (unsigned)n; }

// Keys of one chunk of a session: its context over the launch's chunk count
// (IDX_XCD * n), in whole stages.  Every session has chunks on every XCD that
// way; with the chunk length of the longest session, a shorter one had only the
// first chunks, so that the last XCDs idled (eight sessions of 10K to 51K
// tokens, MXFP4 keys: 3995 -> 2998 us; sixteen of 0.5K to 131K, fp8 keys: 2948
// -> 950).  x = ceil(ctx / 8) + n - 1 is below 2^22 and the reciprocal's error
// below n <= 2^7 in 2^31, so that x * recip >> 31 is the exact quotient: a
// block's first loads wait for it, and with a division appends of 5 to 200
// tokens took 1% longer (fp8 keys, 16K tokens: 47.9 against 47.4 us).  About half
// of that is where the main loop then lay: its place against 32 bytes moves the
// three prefill kernels by up to 0.8%, and MXFP4's lies 0.7% better with the
// division (131K + 64 tokens: 172.5 and 173.5 us).
constexpr int session_chunk(int ctx, int n, unsigned recip)
{
    const unsigned x = (unsigned)((ctx + IDX_XCD - 1) / IDX_XCD + n - 1);
    const int keys = (int)((unsigned long long)x * recip >> 31);
    return (keys + IDX_STAGE - 1) / IDX_STAGE * IDX_STAGE;
}

// ---- decode indexer: blocks of a batch ----------------------------------------

// First block of session s, whose keys start at ctx_start, in chunks of 2^shift
// keys: each session has as many blocks as chunks, or one more, and no block
// needs the sessions before its own.
constexpr int rows_first(int ctx_start, int s, int shift) { return (ctx_start >> shift) + s; }

// Keys per block of a decode batch, and how its blocks are numbered.
struct RowsPlan {
    int chunk;       // keys per block, 4096 down to 256 (one 64-key group per wave)
    int per_seq;     // blocks of every session, or 0: numbered by rows_first
    int64_t blocks;
};
constexpr int ROWS_CHUNK_MIN = 256;
constexpr int64_t ROWS_MAX_BLOCKS = (1 << 24) - 1;  // a launch takes fewer than 2^32 threads

// The chunk with the shortest time estimated, in keys of one block alone on its
// CU, by the blocks that the fullest CU takes (a session of C keys makes about
// C / chunk + 1/2; one block more than the CUs is left out: the last key of a
// power of two and one).  The first block costs its start and its keys.  Each
// next one that is resident beside it (with one token per session 3 blocks a CU,
// 4 with FP4 keys, else 2) runs mostly under it, but for what the memory takes for its keys; with
// the CU full, the next one costs like the first.  The constants are fitted to
// 1071 batches of 1 to 4096 sessions of 500 to 1M keys, even and ragged, with 1,
// 2 and 4 tokens and both key types: the chunk taken is 0.9% off the best one in
// the mean with keys from HBM and 1.3% with keys in the cache.  The chunk that
// fills rounds of resident blocks best was 7.3% and 10% off, whole chunks per CU
// with a fixed cost per block 3.3% and 4.2% (us, the three in turn, fp8 keys: 16
// sessions of 15K to 60K 19.4, 19.4, 25.8; 48 of 8192 with 2 tokens 19.1, 18.8,
// 23.8; 256 of 4000 32.0, 40.6, 32.0; one of 1M with 63 of 1K and 2 tokens 42, 51,
// 42; 64 of 32K to 164K 151, 151, 150).
// Blocks are numbered by rows_first unless the grid of the longest session's
// chunks for each session needs no more of them, or has each on a CU of its own:
// it saves the search, 0.2 us.
constexpr RowsPlan rows_plan(int num_seqs, int max_ctx, int64_t total_ctx, int max_q, int cus, bool fp4)
{
    const bool one = max_q <= 1;
    const int resident = one ? fp4 ? 4 : 3 : 2;
    const int start = fp4 ? one ? 512 : 384 : 128, beside = fp4 ? one ? 384 : 256 : one ? 448 : 1024;
    RowsPlan best = {0, 0, 0};
    double best_cost = -1.0;
    for (int c = one ? 2048 : 4096; c >= ROWS_CHUNK_MIN; c /= 2) {
        const int per_seq = (max_ctx + c - 1) / c;
        const int64_t grid = (int64_t)num_seqs * per_seq, numbered = total_ctx / c + num_seqs;
        const bool even = grid <= numbered || grid <= cus;
        const int64_t blocks = even ? grid : numbered;
        if (best.chunk && blocks > ROWS_MAX_BLOCKS)
            break;
        const double about = (double)total_ctx / c + 0.5 * num_seqs;
        const double useful = about < (double)grid ? about : (double)grid;
        const double first = c + start, memory = 0.6 * c, under = 0.2 * c + beside;
        const double next = under > memory ? under : memory;
        int64_t n = (int64_t)((useful - 1.0) / cus);  // blocks after the fullest CU's first
        if (n > 0 && (double)n * cus >= useful - 1.0)
            --n;
        const int64_t refills = n / resident;
        const double cost = first + (double)(n - refills) * next + (double)refills * (first > next ? first : next);
        if (best_cost < 0.0 || cost < best_cost) {
            best_cost = cost;
            best = RowsPlan{c, even ? per_seq : 0, blocks};
        }
    }
    return best;
}

// ---- top-k: the sample that seeds a row's threshold ----------------------------

constexpr int TK_SAMPLE_GROUPS = 512;  // ~1/32 of a 128K row, in 8-element groups

// Group of a row of ngroups groups that is the sample's g-th, over the whole
// row.  A whole stride (ngroups / TK_SAMPLE_GROUPS) left out up to half of a
// short row, its end, and a row with its high scores ahead of that was streamed
// again: 512 rows of 8184 descending scores (k = 512) 31.3 us, now 10.9.
// (ngroups <= 2^16 by the launcher's bound on contexts: the product fits.)
constexpr int tk_sample_group(int g, int ngroups)
{
    return ngroups <= TK_SAMPLE_GROUPS ? g : (int)((unsigned)g * (unsigned)ngroups / TK_SAMPLE_GROUPS);
}

// ---- MQA attention: one token per wave, or the block's waves on one token ------

constexpr int MQA_WAVES = 4;  // waves per block

// Whether a block's four waves share one token.  A batch takes rounds of one
// block per CU, of which the whole chip has 256 (asking the device took 0.4 of
// the 12 us of a small call, and a part of a chip only gets the slower form).
// One round's time in ns, fitted to 270 batches of 8 to 6000 rows of 32 to 1024
// ids with 1, 8 and 16 heads (which differ by 5%): 3400 + 12 k for a shared
// token, 3800 + 49 k for four.  The rule takes the faster form of all of them to
// within 2% (256 ids: 500 rows 13.8 us shared, 18.6 else, 768 rows 19.5 and 19.1;
// 512 ids: 1024 rows 39 and 31, 1100 rows 46 and 58).  Up to 100 ids, three or
// four tiles for four waves, the forms take as long as each other in one round,
// and longer batches keep a token per wave.
constexpr bool mqa_shared(int64_t total_q, int64_t k)
{
    const int64_t one = (total_q + 255) / 256;
    const int64_t four = (total_q + 256 * MQA_WAVES - 1) / (256 * MQA_WAVES);
    return k > 100 && one * (3400 + 12 * k) < four * (3800 + 49 * k);
}

// ---- shared-prefix attention: blocks of 128 rows and a range of keys ------------

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
    // to 35 batches of 1 to 100 sessions; of 39 batches on the kernels as they are, each with 27
    // chunk lengths, the chunk taken is 0.5% off the best one in the mean for MLA and
    // 2.6% for MQA, 10% at most (whole rounds of blocks, a start of 128 or 256 keys and a
    // join of 0.02 or 0.01: 6 and 13% in the mean of the first 18).
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
