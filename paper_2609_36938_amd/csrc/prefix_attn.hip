// Dense causal attention over the paged cache, for a batch whose sessions
// begin with a common prefix.
//
// A row is one (token, head): o = sum_j 2^(x_j - m) v_j / sum_j 2^(x_j - m), with
// x_j = (q . k_j) scale log2 e over the keys before the row's limit.  A block takes
// 128 rows and a range of keys and goes over them once, in tiles of 32:
//   * The tiles come straight into LDS (global_load_lds), into a ring of buffers two or
//     three tiles ahead.  Within a row the 16-byte chunks are exchanged by the row's
//     number (swz16, swz8): neither the row-wise reads of K nor the transposing
//     reads of V meet in a bank (0 conflict cycles counted).
//   * A wave has 32 of the rows and scores them: their queries in registers, S^T = K Q^T
//     on 32x32x16 MFMA, so that a lane's results are logits of one row and
//     its exponentials, as they lie, are the operand of O^T = V^T P^T.
//   * Rows of different sessions share the blocks over the prefix: its keys are
//     read once for 128 rows instead of once for each session's heads.
//   * Ranges of one row are joined by their maxima and sums (prefix_combine): few rows
//     have too few blocks for 256 CUs otherwise.
// Logits, maxima, sums and O are fp32.  Probabilities are rounded to bf16, the type of
// the V that they multiply (in two parts they would take twice the MFMAs), also where the output
// is fp32; their sums are taken before that.  The error is 2^-8 of the
// values at most for each key, and mostly averages out (2.2e-3 of the result
// with 4096 keys, 1.7e-3 of it the rounding of the result to bf16).
//
// Two kernels, by what a row costs in registers.  prefix_mqa: 128 dims, O of a wave's own rows
// in its registers, two blocks a CU.  prefix_mla: O of 128 rows of 512 dims is all
// the accumulators of a CU, so a wave has a quarter of the dims of all rows, and the
// probabilities go through LDS.
#include "attn_device.hpp"
#include "janus_device.hpp"
#include "janus_host.hpp"
#include "launch_rules.hpp"

#include <type_traits>

namespace janus {

constexpr int PA_WAVES = 4;
constexpr int PA_THREADS = 64 * PA_WAVES;
static_assert(PA_ROWS == 32 * PA_WAVES, "a wave has 32 rows");
typedef float v16f __attribute__((ext_vector_type(16)));

struct PrefixArgs {
    const int32_t *q_start, *hist_len;
    int num_seqs, es;
    const uint16_t *q;
    int heads;
    const uint8_t *k, *v;
    int64_t k_rb, v_rb;  // row bytes
    const int32_t *table;
    int pt_ld, page_shift;
    float scale_log2;
    void *out;
    int out_f32;
    float *lse;
    float *part;  // O of the ranges, then their maxima and sums
    PrefixPlan plan;
};

// Session of an own tile, and the tile's rows (row0 >= row1: none).  WAVE: every lane of
// the wave asks for the same tile, 64 sessions are looked at in one load.
template <bool WAVE>
JANUS_DEV int tile_rows(const PrefixArgs &g, int tile, int &row0, int &row1)
{
    if (g.plan.one) {
        row0 = g.q_start[tile] * g.heads;
        row1 = min(row0 + PA_ROWS, g.q_start[tile + 1] * g.heads);
        return tile;
    }
    int lo = 0, hi = g.num_seqs;  // the session is in [lo, hi)
    while (hi - lo > 1) {
        if constexpr (WAVE) {
            const int step = (hi - lo + kWave - 1) / kWave, s = lo + (int)(threadIdx.x & 63) * step;
            const uint64_t below = __ballot(s < hi && prefix_tile_first(g.q_start[s], g.heads, s) <= tile);
            lo += max((int)__popcll(below) - 1, 0) * step;
            hi = min(hi, lo + step);
        } else {
            const int mid = (lo + hi) >> 1;
            (prefix_tile_first(g.q_start[mid], g.heads, mid) <= tile ? lo : hi) = mid;
        }
    }
    const int q0 = g.q_start[lo];
    row0 = q0 * g.heads + (tile - prefix_tile_first(q0, g.heads, lo)) * PA_ROWS;
    row1 = min(row0 + PA_ROWS, g.q_start[lo + 1] * g.heads);
    return lo;
}

// The block's rows, keys and table, and where its results go: to row `part` of the
// workspace on, or (part < 0) to out.
struct PrefixRange {
    int row0, row1, kbeg, kend, sess;
    int64_t part;
    bool shared;
    bool whole;  // every row has all of the keys
};
JANUS_DEV PrefixRange prefix_range(const PrefixArgs &g, int blk)
{
    const PrefixBlock bk = prefix_block(g.plan, blk);
    PrefixRange r;
    r.shared = bk.shared;
    r.sess = 0;
    r.whole = false;
    if (bk.shared) {
        r.row0 = bk.tile * PA_ROWS;
        r.kbeg = bk.chunk * g.plan.chunk;
        r.kend = min(r.kbeg + g.plan.chunk, g.plan.prefix);
        const int tokens = g.q_start[g.num_seqs];
        if (g.num_seqs <= 4 * kWave) {
            // mostly all sessions reach behind the prefix: one load, where the search for each
            // row's own is a chain of them
            bool all = true;
            for (int s = threadIdx.x & 63; s < g.num_seqs; s += kWave)
                all = all && last_cand(g.hist_len[s], 0, g.es) + 1 >= r.kend;
            r.whole = __ballot(!all) == 0;
        }
        r.row1 = min(r.row0 + PA_ROWS, tokens * g.heads);
        r.part = bk.slot * g.plan.part_rows + r.row0;
        return r;
    }
    r.sess = tile_rows<true>(g, bk.tile, r.row0, r.row1);
    r.kbeg = g.plan.prefix + bk.chunk * g.plan.chunk;
    r.kend = r.kbeg;
    if (r.row0 < r.row1) {
        r.kend = last_cand(g.hist_len[r.sess], (r.row1 - 1) / g.heads - g.q_start[r.sess], g.es) + 1;
        if (bk.slot >= 0)
            r.kend = min(r.kend, r.kbeg + g.plan.chunk);
    }
    r.part = bk.slot < 0           ? -1
             : g.plan.prefix > 0 ? bk.slot * g.plan.part_rows + r.row0
                                 : bk.slot * g.plan.part_rows + (int64_t)(bk.tile - g.plan.whole) * PA_ROWS;
    return r;
}
// First key that the row's token does not attend to.
JANUS_DEV int row_limit(const PrefixArgs &g, const PrefixRange &r, int row)
{
    if (r.whole)
        return r.kend;
    const int token = row / g.heads;
    const int s = r.shared ? session_of_row(g.q_start, g.num_seqs, token) : r.sess;
    return min(r.kend, last_cand(g.hist_len[s], token - g.q_start[s], g.es) + 1);
}

// Keys before it are every row's of the block, whose limits are in LDS.  One session's grow with its
// rows; only where sessions end inside the prefix are all of them looked at.
JANUS_DEV int block_limit(const PrefixRange &r, const int *lim)
{
    if (r.whole)
        return r.kend;
    if (!r.shared)
        return __builtin_amdgcn_readfirstlane(lim[0]);
    const int lane = threadIdx.x & 63;
    int least = min(r.row0 + lane < r.row1 ? lim[lane] : 0x7fffffff,
                    r.row0 + 64 + lane < r.row1 ? lim[64 + lane] : 0x7fffffff);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1)
        least = min(least, __shfl_xor(least, o));
    return __builtin_amdgcn_readfirstlane(least);
}

// A row's sum of probabilities, over a range of any length: a tile's are added pairwise, and the
// tiles' sums with what each addition rounds off carried to the next (Kahan, CACM 8, 1965).  One
// after the other in fp32, half a million equal terms are off by 2e-3.
struct Total {
    float sum, off;
    JANUS_DEV void add(float x)
    {
        const float y = x - off, t = sum + y;
        off = (t - sum) - y;
        sum = t;
    }
    JANUS_DEV void scale(float f)
    {
        sum *= f;
        off *= f;
    }
};
JANUS_DEV float sum8(v8f p) { return ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])); }

// Values of V that are not finite, where rows end: a probability of 0 does not undo them for the rows
// without the key, so the tiles in which rows end are searched for them, and the products take 0 in
// their place.  What they give the rows that have the key is known without a product: any sum with them
// is infinite or NaN.  (A block that was done again key by key for their sake, all 128 rows of it, took
// minutes over long contexts: one overflowed row of the cache held up a batch.)
JANUS_DEV bool not_finite(int x) { return ((x & 0x7f80) == 0x7f80) | ((x & 0x7f800000) == 0x7f800000); }
JANUS_DEV bool not_finite(v4i x) { return not_finite(x[0]) | not_finite(x[1]) | not_finite(x[2]) | not_finite(x[3]); }
JANUS_DEV v4i finite_or_0(v4i x)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] &= (x[e] & 0x7f80) == 0x7f80 ? (int)0xffff0000 : -1;
        x[e] &= (x[e] & 0x7f800000) == 0x7f800000 ? 0xffff : -1;
    }
    return x;
}
constexpr int NEVER = 0x7fffffff;  // no tile, no key

// Adds the values that are not finite of V's keys from `from` on, dims dim0 .. dim0 + 127, to rows
// rbeg .. rend - 1 of O, which this wave has written; sixteen lanes a key, then a row.  ONE_POOL: V's rows are
// K's, so the key's logit is infinite too, and its probability NaN, or 0, or makes all others 0: NaN in
// every case.  With pools apart that is so where the key's row of K is not finite either.
template <int DV, bool ONE_POOL>
JANUS_DEV void add_not_finite(const PrefixArgs &g, const PrefixRange &r, const int *lim, int from, int dim0, int rbeg,
                              int rend)
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");  // (other lanes' stores)
    const int lane = threadIdx.x & 63, in = lane & 15, group = lane >> 4;
    const int32_t *pt = g.table + (int64_t)r.sess * g.pt_ld;
    int plus[8], minus[8];  // the first keys with +inf and -inf, or NaN, of eight dims
#pragma unroll
    for (int e = 0; e < 8; ++e)
        plus[e] = minus[e] = NEVER;
    constexpr int AHEAD = 4;
    for (int k0 = max(from, r.kbeg); k0 < r.kend; k0 += 4 * AHEAD) {
        int64_t slot[AHEAD];
        v4i x[AHEAD];
        bool hit = false;
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int key = min(k0 + 4 * a + group, r.kend - 1);
            slot[a] = ((int64_t)pt[key >> g.page_shift] << g.page_shift) + (key & ((1 << g.page_shift) - 1));
            x[a] = *(const v4i *)(g.v + slot[a] * g.v_rb + 2 * dim0 + 16 * in);
            hit |= not_finite(x[a]);
        }
        if (__ballot(hit) == 0)
            continue;
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int key = min(k0 + 4 * a + group, r.kend - 1);
            bool both = ONE_POOL;
            if (!ONE_POOL)
                both = (__ballot(not_finite(*(const v4i *)(g.k + slot[a] * g.k_rb + 16 * in))) >> (16 * group) & 0xffff) != 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t v = (uint32_t)x[a][e / 2] >> (16 * (e % 2)) & 0xffff;
                if ((v & 0x7f80) != 0x7f80)
                    continue;
                const bool nan = both || (v & 0x7f) != 0;
                if (nan || v < 0x8000)
                    plus[e] = min(plus[e], key);
                if (nan || v >= 0x8000)
                    minus[e] = min(minus[e], key);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int o = 16; o < 64; o <<= 1) {
            plus[e] = min(plus[e], __shfl_xor(plus[e], o));
            minus[e] = min(minus[e], __shfl_xor(minus[e], o));
        }
    for (int row = rbeg + group; row < rend; row += 4) {
        const int end = lim[row - r.row0];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool up = plus[e] < end, down = minus[e] < end;
            if (!up && !down)
                continue;
            const float x = up && down ? NAN : up ? INFINITY : -INFINITY;
            const int dim = dim0 + 8 * in + e;
            const int64_t o = (int64_t)row * DV + dim;
            if (r.part >= 0)
                g.part[(r.part + (row - r.row0)) * DV + dim] += x;
            else if (g.out_f32)
                ((float *)g.out)[o] += x;
            else
                ((__bf16 *)g.out)[o] = (__bf16)((float)((__bf16 *)g.out)[o] + x);
        }
    }
}

// Within a row in LDS, chunk c (16 bytes) of row r lies at c ^ swz16(r), in rows of 16
// chunks and more, and at c ^ swz8(r) in rows of eight.  Sixteen rows of one chunk (a K
// read), and four rows of four neighbouring ones (a transposing read), then lie in
// banks of their own.
JANUS_DEV int swz16(int r) { return ((r & 1) << 3) | ((r & 2) << 1) | ((r & 4) >> 1) | ((r & 8) >> 3); }
JANUS_DEV int swz8(int r) { return ((r & 2) << 1) | ((r & 4) >> 1) | ((r & 8) >> 3); }

constexpr int PQ_KT = 32;  // keys of a tile

// MQA, 128 dims.  A tile is 8 MFMAs for S^T and 8 for O^T in each wave, 512 cycles, and
// 16 exponentials a lane: those go under the MFMAs that score the next tile.  What bounds
// it: long contexts, LDS, from which every wave reads the whole tile, 16 KB for its 16 MFMAs: eight waves
// of a CU 128 KB in the 1024 cycles that their MFMAs take, all that LDS gives beside the gathers' writes
// (2 sessions of 1000 to 2000 tokens x 16 heads on 31000 ids: 790 to 835 us, card by card, 1.0 PFLOP/s;
// scores and exponentials one after the other 10% more); few rows, the chain of loads before the first
// tile (2.4 us), a loop of few tiles, and the launch of the join (16 sessions x 8 heads on 4096 ids: 10 us).  32
// keys a tile and 66 KB of LDS let two blocks share a CU, so that one's waits are the
// other's work: the first form took 1740 us for the long case with 64 keys and one block a
// CU, 1190 with this.  Four buffers, and a turn for each of them, keep LDS offsets constant.
__global__ __launch_bounds__(PA_THREADS, 2) void prefix_mqa(PrefixArgs g)
{
    constexpr int RB = 256;                              // bytes of a row
    constexpr int KBUF = PQ_KT * RB, BUF = 2 * KBUF;     // K rows, then V rows
    constexpr int STEPS = 8, NB = 4;                     // K-steps, blocks of 32 dims
    constexpr int GATHERS = KBUF / (1024 * PA_WAVES);    // a wave's, of each pool
    __shared__ __attribute__((aligned(16))) uint8_t ring[4 * BUF];
    __shared__ int sLim[PA_ROWS];
    __shared__ __attribute__((aligned(16))) int sBad[PA_WAVES];  // a wave's `bad`

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c32 = lane & 31, hf = lane >> 5;
    const PrefixRange r = prefix_range(g, blockIdx.x);
    if (r.row0 >= r.row1)
        return;
    typedef const __attribute__((address_space(4))) int32_t *scalar_i32;  // read through the scalar cache
    const scalar_i32 pt = (scalar_i32)(g.table + (int64_t)r.sess * g.pt_ld);
    const int kbeg = r.kbeg, kend = r.kend;
    const int row = r.row0 + 32 * wave + c32;
    const bool live = row < r.row1;
    const int lim = row_limit(g, r, live ? row : r.row1 - 1);
    if (hf == 0)
        sLim[32 * wave + c32] = lim;
    v8bf qf[STEPS];
    {
        const uint16_t *qr = g.q + (int64_t)(live ? row : r.row1 - 1) * 128 + 8 * hf;
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
            qf[st] = as_v8bf(*(const v4i *)(qr + 16 * st));
    }
    v16f o[NB];
#pragma unroll
    for (int d = 0; d < NB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            o[d][i] = 0.f;
    float m = M_INIT;
    Total lsum = {0.f, 0.f};
    int bad = NEVER;  // the first tile where rows end whose V is not finite, in this wave's share of it
    int bmin = 0;     // keys before it are every row's

    // Tiles begin at multiples of their length: a tile of longer pages lies in one.
    // A wave gathers four rows at a time, rows 16 j + 4 wave .. of K and of V.
    const int base0 = kbeg & ~(PQ_KT - 1);
    const int nt = kend > kbeg ? (kend - base0 + PQ_KT - 1) / PQ_KT : 0;
    const int ps = (1 << g.page_shift) - 1;
    const int gr = lane >> 4;
    const uint32_t gc = 16 * ((lane & 15) ^ swz16(4 * wave + gr));
    const uint32_t koff = gr * (uint32_t)g.k_rb + gc, voff = gr * (uint32_t)g.v_rb + gc;
    auto entry = [&](int t) { return pt[min(base0 + t * PQ_KT, kend - 1) >> g.page_shift]; };
    auto issue = [&](int t, int page) {
        uint8_t *dst = ring + (t & 3) * BUF + 1024 * wave;
        const int base = base0 + t * PQ_KT;
        if (ps >= PQ_KT - 1 && base >= kbeg && base + PQ_KT <= kend) {
            const int64_t slot = ((int64_t)page << g.page_shift) + (base & ps) + 4 * wave;
#pragma unroll
            for (int j = 0; j < GATHERS; ++j) {
                gather16(g.k + (slot + 16 * j) * g.k_rb, koff, dst + 4096 * j);
                gather16(g.v + (slot + 16 * j) * g.v_rb, voff, dst + KBUF + 4096 * j);
            }
        } else {
            // keys outside [kbeg, kend) load the nearest one inside
#pragma unroll
            for (int j = 0; j < GATHERS; ++j) {
                const int key = min(max(base + 16 * j + 4 * wave + gr, kbeg), kend - 1);
                const int64_t slot = ((int64_t)pt[key >> g.page_shift] << g.page_shift) + (key & ps);
                gather16(g.k + slot * g.k_rb + gc, dst + 4096 * j);
                gather16(g.v + slot * g.v_rb + gc, dst + KBUF + 4096 * j);
            }
        }
    };
#pragma unroll
    for (int st = 0; st < STEPS; ++st)
        asm volatile("" ::"v"(qf[st]));  // waited for here: a wait in the loop would be for the gathers too
    if (nt > 0) {
        issue(0, entry(0));
        issue(1, entry(1));
        issue(2, entry(2));
    }
    int page = nt > 0 ? entry(3) : 0;

    // LDS offsets in a tile.  K: chunk 2 st + hf of key c32.  V: keys 8 u + 4 hf + (lane / 4) % 4
    // (and 16 more) and dims 32 d + 16 (lane / 16 % 2) + 4 (lane % 4)
    int kat[STEPS], vat[NB][2];
#pragma unroll
    for (int st = 0; st < STEPS; ++st)
        kat[st] = c32 * RB + 16 * ((2 * st + hf) ^ swz16(c32));
#pragma unroll
    for (int d = 0; d < NB; ++d)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int k = 8 * u + 4 * hf + ((lane >> 2) & 3);
            vat[d][u] = k * RB + 16 * ((4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swz16(k)) + 8 * (lane & 1);
        }
    auto logits = [&](const uint8_t *tile) {
        v16f x;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            x[i] = 0.f;
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_v8bf(*(const v4i *)(tile + kat[st])), qf[st], x, 0, 0, 0);
        return x;
    };
    // A turn scores tile t + 1 while it takes the exponentials of tile t, then multiplies
    // them with tile t's V.  (Behind the last tile it scores what the ring holds, for nothing.)
    auto turn = [&](auto slot, int t, v16f &s, v16f &ahead) {
        constexpr int SLOT = decltype(slot)::value;
        // tile t + 1 has landed, the next one's gathers may be on their way (behind the last
        // tile they read its last key again)
        __builtin_amdgcn_s_waitcnt(vmcnt_only(2 * GATHERS));
        lds_barrier();
        const int next = entry(t + 4);
        issue(t + 3, page);
        page = next;
        const uint8_t *vt = ring + SLOT * BUF + KBUF;
        const int base = base0 + t * PQ_KT;
        float mult = g.scale_log2;
        const bool ragged = base < kbeg || base + PQ_KT > bmin;
        if (ragged || mult <= 0.f) {
            // keys 8 (i / 4) + 4 hf + i % 4 of this lane's row
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = base + 8 * (i / 4) + 4 * hf + i % 4;
                s[i] = key >= kbeg && key < lim ? s[i] * mult : -INFINITY;
            }
            mult = 1.f;
        }
        if (ragged) {  // (every wave comes here, with a share of the tile)
            uint8_t *share = ring + SLOT * BUF + KBUF + 1024 * wave + 16 * lane;
            static_assert(KBUF == 2 * 1024 * PA_WAVES, "two pieces a wave");
            const v4i x = *(const v4i *)share, y = *(const v4i *)(share + 1024 * PA_WAVES);
            if (__ballot(not_finite(x) | not_finite(y)) != 0) {
                *(v4i *)share = finite_or_0(x);
                *(v4i *)(share + 1024 * PA_WAVES) = finite_or_0(y);
                bad = min(bad, t);
            }
            lds_barrier();
        }
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i)
            mx = fmaxf(mx, s[i]);
        mx *= mult;
        if (__ballot(mx > m + RESCALE_SLACK) != 0) {
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float mnew = mx > m + RESCALE_SLACK ? mx : m;
            const float alpha = __builtin_amdgcn_exp2f(m - mnew);
            lsum.scale(alpha);
            m = mnew;
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    o[d][i] *= alpha;
        }
        ahead = logits(ring + (SLOT + 1) % 4 * BUF);
        v8bf pb[2];
        float sums[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v8f p;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                p[e] = __builtin_amdgcn_exp2f(s[8 * h + e] * mult - m);
            sums[h] = sum8(p);
            pb[h] = __builtin_convertvector(p, v8bf);
        }
        lsum.add(sums[0] + sums[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int d = 0; d < NB; ++d) {
                v4s16 part[2];
                v8bf a;
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    part[u] = lds_read_tr16(vt, vat[d][u] + 16 * RB * h);
                __builtin_memcpy(&a, part, 16);
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[h], o[d], 0, 0, 0);
            }
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int x = 0; x < STEPS; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a matrix instruction
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // an operand read
            __builtin_amdgcn_sched_group_barrier(0x002, 7, 0);  // under it, seven others
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int x = 0; x < 2 * NB; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
    };
    if (nt > 0) {
        using std::integral_constant;
        __builtin_amdgcn_s_waitcnt(vmcnt_only(4 * GATHERS));
        lds_barrier();
        bmin = block_limit(r, sLim);
        v16f sa = logits(ring), sb;
#pragma unroll 1
        for (int t = 0;; t += 4) {
            turn(integral_constant<int, 0>{}, t, sa, sb);
            if (t + 1 >= nt)
                break;
            turn(integral_constant<int, 1>{}, t + 1, sb, sa);
            if (t + 2 >= nt)
                break;
            turn(integral_constant<int, 2>{}, t + 2, sa, sb);
            if (t + 3 >= nt)
                break;
            turn(integral_constant<int, 3>{}, t + 3, sb, sa);
            if (t + 4 >= nt)
                break;
        }
    }

    if (lane == 0)
        sBad[wave] = bad;
    const float l = lsum.sum + __shfl_xor(lsum.sum, 32);
    lds_barrier();
    const v4i any = *(const v4i *)sBad;
    const int first = __builtin_amdgcn_readfirstlane(min(min(any[0], any[1]), min(any[2], any[3])));
    if (live && r.part >= 0) {
        const int64_t at = r.part + (row - r.row0);
        if (hf == 0)
            *(float2 *)(g.part + g.plan.slots * g.plan.part_rows * 128 + 2 * at) = float2{m, l};
        if (nt > 0) {
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *(v4f *)(g.part + at * 128 + 32 * d + 2 * i + 4 * hf) =
                        v4f{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
        }
    } else if (live) {
        const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
        for (int d = 0; d < NB; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                store_out4(g.out, g.out_f32, (int64_t)row * 128 + 32 * d + 2 * i + 4 * hf,
                           v4f{o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv});
        if (g.lse && hf == 0)
            g.lse[row] = l != 0.f ? (m + log2f(l)) * LN2 : -INFINITY;
    }
    // the gathers behind the last tile still write LDS: a wave waits for its own before it ends
    __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
    if (first != NEVER) {
        const int r0 = r.row0 + 32 * wave;
        add_not_finite<128, false>(g, r, sLim, base0 + first * PQ_KT, 0, r0, min(r0 + 32, r.row1));
    }
}

constexpr int PM_KT = 32, PM_STEPS = 576 / 16;
constexpr int PM_MAIN = PM_KT * 1024, PM_TAIL = PM_KT * 128;  // bytes of dims 0..511 of a tile, and of 512..575
// A row's maximum is that of its first tile, and probabilities may exceed 1 by this
// much (log2): nothing is lost, their exponents have room.  Rows that outgrow it
// are done again from their maxima, so that O is never rescaled.
constexpr float PM_HEADROOM = 32.f;
constexpr int PM_WITH = 16;  // steps of P V among those of K Q^T

// S^T on registers that are not accumulators: O fills all 256 of those, and the
// compiler would put S among them.  It inserts no wait states for assembly: two
// before an MFMA whose sources the VALU may have written, and what reads S
// waits by itself (settled).
JANUS_DEV void mfma_first(v16f &s, v4i a, v8bf b)
{
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(a), "v"(b));
}
JANUS_DEV void mfma_next(v16f &s, v4i a, v8bf b)
{
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(a), "v"(b));
}
JANUS_DEV void settled(v16f &s) { asm volatile("s_nop 15\n\ts_nop 7" : "+v"(s)); }

// MLA, 576 dims scored and 512 of them multiplied again as V.  A wave scores its 32 rows (36 MFMAs,
// a chain), writes their probabilities to LDS, and multiplies all 128 rows' by its 128
// dims of V (32 MFMAs): V is read from LDS once a block instead of once a wave, and O^T takes 256
// accumulators, which leaves 256 registers for 144 of queries and the operands.
// While tile t is scored, tile t - 1 is multiplied: PM_WITH of its steps stand among the chain's, the
// others under the exponentials (the longest case below 7.77 ms with 8 steps, 7.40 with 16, 7.43 with
// 24, on one card).  1.10 to 1.24 PFLOP/s on long ranges (8 sessions of 100 to 300 tokens x 128 heads on
// 17000 ids, 6.5 to 7.3 ms, card by card), where a library product of 8192^3 reaches 1.22 and of 16384^3
// 1.40.  The MFMAs are busy in 54% of the cycles; between them lie the scoring chain's dependences, the
// exchange of probabilities and a barrier a tile.  Few rows pay 5 to 8 us before the first tile (queries
// and tiles from HBM), as much behind the last, and the join: 32 sessions x 16 heads on 131072 ids take
// 163 to 185 us where the product's rate would take 105.  47 registers are spilled, 30 dwords a lane in all: in the
// loop one is read back a tile; the others are written before the loop and in the epilogue, which takes O
// out of the accumulators.  The first form, with each wave's O^T rescaled
// as maxima grow, spilled O itself and took 95 ms for the longest case; gathers left out behind the last
// tile, by a branch, cost 7%.  A block whose logits outgrow its first tile's by 2^32 is done again, 2.5 to 2.7 times
// the work: logits of a standard deviation of 4 nats do not (6.53 ms), of 16 nats do (17.5).
// SMALL: pages of fewer than eight ids, where a wave's eight rows lie in different ones.
template <bool SMALL>
__global__ __launch_bounds__(PA_THREADS, 1) void prefix_mla(PrefixArgs g)
{
    // Tile t is scored while tile t - 1 meets its probabilities and two more are on
    // their way; the last dims are done with a tile earlier.
    __shared__ __attribute__((aligned(16))) uint8_t main_ring[4 * PM_MAIN], tail_ring[3 * PM_TAIL];
    __shared__ v4i sP[2][PA_WAVES][2][64];       // probabilities of the waves' rows, as operands
    __shared__ v4i sOver;                        // a wave's rows outgrew their maxima
    __shared__ int sBad[PA_WAVES];               // the first tile that a wave has cleaned
    __shared__ int sLim[PA_ROWS];
    __shared__ float sM[PA_ROWS], sL[PA_ROWS];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c32 = lane & 31, hf = lane >> 5;
    const PrefixRange r = prefix_range(g, blockIdx.x);
    if (r.row0 >= r.row1)
        return;
    typedef const __attribute__((address_space(4))) int32_t *scalar_i32;  // read through the scalar cache
    const scalar_i32 pt = (scalar_i32)(g.table + (int64_t)r.sess * g.pt_ld);
    const int kbeg = r.kbeg, kend = r.kend;
    const int row = r.row0 + 32 * wave + c32;
    const bool live = row < r.row1;
    const int lim = row_limit(g, r, live ? row : r.row1 - 1);
    if (hf == 0)
        sLim[32 * wave + c32] = lim;
    if (lane == 0)
        sBad[wave] = NEVER;

    v8bf qf[PM_STEPS];
    {
        const uint16_t *qr = g.q + (int64_t)(live ? row : r.row1 - 1) * 576 + 8 * hf;
#pragma unroll
        for (int st = 0; st < PM_STEPS; ++st)
            qf[st] = as_v8bf(*(const v4i *)(qr + 16 * st));
    }
    // O^T of dims 128 wave + 32 d .. and rows 32 rb ..
    v16f o[4][PA_WAVES];
    float m = M_INIT;
    Total lsum = {0.f, 0.f};

    const int base0 = kbeg & ~(PM_KT - 1);
    const int nt = kend > kbeg ? (kend - base0 + PM_KT - 1) / PM_KT : 0;
    const int ps = (1 << g.page_shift) - 1;
    const uint32_t rb32 = (uint32_t)g.k_rb;
    auto key_row = [&](int key) {  // (uniform)
        return g.k + (((int64_t)pt[key >> g.page_shift] << g.page_shift) + (key & ps)) * (int64_t)rb32;
    };
    // Wave w gathers rows 8 w .. 8 w + 7: dims 0..511 a row at a time (64 lanes of 16
    // bytes), the last 64 dims of the eight together.  Keys outside [kbeg, kend) load the nearest
    // one inside.
    const int tr = lane >> 3;
    auto entry = [&](int t) {  // table entry of the wave's rows of tile t, pages of eight ids and more
        return pt[min(max(base0 + t * PM_KT + 8 * wave, kbeg), kend - 1) >> g.page_shift];
    };
    auto fire = [&](int t, int page, int i) {
        const int key0 = base0 + t * PM_KT + 8 * wave;
        const uint8_t *first = g.k + ((int64_t)page << g.page_shift) * rb32;
        int ln = lane;
        asm volatile("" : "+v"(ln));  // the lane's chunk is worked out here, not kept for the whole loop
        if (i < 8) {
            const int key = min(max(key0 + i, kbeg), kend - 1) & ps;
            gather16(first + (int64_t)key * rb32, 16u * (ln ^ swz16(8 * (wave & 1) + i)),
                     main_ring + (t & 3) * PM_MAIN + 1024 * (8 * wave + i));
        } else {
            const int from = min(max(key0, kbeg), kend - 1), key = min(max(key0 + (ln >> 3), kbeg), kend - 1);
            gather16(first + (int64_t)(from & ps) * rb32,
                     (key - from) * rb32 + 1024u + 16u * ((ln & 7) ^ swz8(8 * (wave & 1) + (ln >> 3))),
                     tail_ring + t % 3 * PM_TAIL + 1024 * wave);
        }
    };
    auto issue = [&](int t) {
        if constexpr (!SMALL) {
            const int page = entry(t);
#pragma unroll
            for (int i = 0; i < 9; ++i)
                fire(t, page, i);
        } else {
            const int key0 = base0 + t * PM_KT + 8 * wave;
            const uint8_t *mine = g.k;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint8_t *src = key_row(min(max(key0 + i, kbeg), kend - 1));
                gather16(src, 16u * (lane ^ swz16(8 * (wave & 1) + i)),
                         main_ring + (t & 3) * PM_MAIN + 1024 * (8 * wave + i));
                mine = tr == i ? src : mine;
            }
            gather16(mine + 1024 + 16 * ((lane & 7) ^ swz8(8 * (wave & 1) + tr)),
                     tail_ring + t % 3 * PM_TAIL + 1024 * wave);
        }
    };
    // The wave's gathers have landed but for the newest tile's nine.
    auto landed = [&]() { __builtin_amdgcn_s_waitcnt(vmcnt_only(9)); };
    if (nt > 0) {
        issue(0);
        issue(1);
        issue(2);
    }

    const int kcol = (hf ^ swz16(c32)) * 16, tcol = (hf ^ swz8(c32)) * 16;
    const int vkey = 4 * hf + ((lane >> 2) & 3);
    const int vch = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    v16f s;
    v8bf pb[2];
    __builtin_amdgcn_s_waitcnt(vmcnt_only(18));
    lds_barrier();
    const int bmin = block_limit(r, sLim);
    int bad = 0;  // a tile where rows end holds values of V that are not finite

    // O += P V of a tile, this wave's dims, as 32 steps: keys 16 h + .., dims 128 wave +
    // 32 d + .., rows 32 rb + .., with j = 16 h + 4 d + rb.  The operands of step j are read
    // four steps before it.
    v4i p[PA_WAVES];
    v8bf va[2];
    auto read_v = [&](int t, int h, int d) {
        const uint8_t *vt = main_ring + (t & 3) * PM_MAIN + 256 * wave;
        v4s16 part[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int k = 16 * h + 8 * u + vkey;
            part[u] = lds_read_tr16(vt, k * 1024 + 16 * ((4 * d + vch) ^ swz16(8 * u + vkey)) + 8 * (lane & 1));
        }
        __builtin_memcpy(&va[d & 1], part, 16);
    };
    auto product_begin = [&](int t) {
#pragma unroll
        for (int rb = 0; rb < PA_WAVES; ++rb)
            p[rb] = sP[t & 1][rb][0][lane];
        read_v(t, 0, 0);
    };
    auto product_step = [&](int t, int j) {
        const int h = j / 16, d = j / 4 % 4, rb = j % 4;
        if (rb == 0 && j + 4 < 32)
            read_v(t, (j + 4) / 16, (j + 4) / 4 % 4);
        o[d][rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[d & 1], as_v8bf(p[rb]), o[d][rb], 0, 0, 0);
        if (h == 0 && d == 3)
            p[rb] = sP[t & 1][rb][1][lane];
    };
    // S^T of tile t, with the first `with` steps of the tile before it between its own:
    // its MFMAs wait for each other.  K operands are read AHEAD steps ahead.
    auto logits = [&](int t, auto with, int page) {
        constexpr int WITH = decltype(with)::value;
        const uint8_t *tile = main_ring + (t & 3) * PM_MAIN, *tail = tail_ring + t % 3 * PM_TAIL;
        constexpr int AHEAD = 4;
        auto kop = [&](int st) {
            return st < 32 ? *(const v4i *)(tile + c32 * 1024 + (kcol ^ (32 * (st & 7))) + 256 * (st >> 3))
                           : *(const v4i *)(tail + c32 * 128 + (tcol ^ (32 * (st & 3))));
        };
        v4i ahead[AHEAD];
        if (WITH)
            product_begin(t - 1);
#pragma unroll
        for (int x = 0; x < AHEAD; ++x)
            ahead[x] = kop(x);
#pragma unroll
        for (int st = 0; st < PM_STEPS; ++st) {
            if (st == 0)
                mfma_first(s, ahead[0], qf[0]);
            else
                mfma_next(s, ahead[st % AHEAD], qf[st]);
            if (st + AHEAD < PM_STEPS)
                ahead[st % AHEAD] = kop(st + AHEAD);
            if (st < WITH)
                product_step(t - 1, st);
            if (!SMALL && WITH && st < 9)
                fire(t + 2, page, st);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Four keys of the wave's dims of a tile (the other waves score them, and do not multiply them).
    auto own_dims = [&](int t, int w) {
        return (v4i *)(main_ring + (t & 3) * PM_MAIN + 1024 * (4 * w + (lane >> 4)) + 256 * wave + 16 * (lane & 15));
    };
    // The logits of tile t scaled, those of keys that a row does not have -inf;
    // returns the factor that is left to apply.
    auto mask = [&](int t) {
        settled(s);
        const int base = base0 + t * PM_KT;
        const bool inside = base >= kbeg && base + PM_KT <= bmin;
        if (inside && g.scale_log2 > 0.f)
            return g.scale_log2;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int key = base + 8 * (i / 4) + 4 * hf + i % 4;
            s[i] = key >= kbeg && key < lim ? s[i] * g.scale_log2 : -INFINITY;
        }
        if (!inside) {
#pragma unroll 2
            for (int w = 0; w < 8; ++w)
                bad |= not_finite(*own_dims(t, w));
        }
        return 1.f;
    };
    // Once a wave has found such values, it takes them out of its dims of every tile that it multiplies,
    // when the tile has been scored.
    auto clean = [&](int t) {
        if (__ballot(bad) == 0)
            return;
#pragma unroll 1
        for (int w = 0; w < 8; ++w)
            *own_dims(t, w) = finite_or_0(*own_dims(t, w));
        if (lane == 0)
            sBad[wave] = min(sBad[wave], t);
    };
    // Probabilities of s * mult (mult > 0), relative to the maximum of the first
    // tile that has keys of the row.
    bool over = false;
    auto probabilities = [&](float mult) {
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i)
            mx = fmaxf(mx, s[i]);
        mx *= mult;
        if (__ballot(mx > m + PM_HEADROOM) != 0) {
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            over |= m != M_INIT && mx > m + PM_HEADROOM;
            m = m == M_INIT ? fmaxf(mx, M_INIT) : m;
        }
        float sums[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v8f p;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                p[e] = __builtin_amdgcn_exp2f(s[8 * h + e] * mult - m);
            sums[h] = sum8(p);
            pb[h] = __builtin_convertvector(p, v8bf);
        }
        lsum.add(sums[0] + sums[1]);
    };
    auto give = [&](int t) {
        sP[t & 1][wave][0][lane] = __builtin_bit_cast(v4i, pb[0]);
        sP[t & 1][wave][1][lane] = __builtin_bit_cast(v4i, pb[1]);
        landed();
        lds_barrier();
    };
    if (nt > 0) {
        // The second time round, the rows' maxima over all their keys are known.
#pragma unroll 1
        for (int round = 0; round < 2; ++round) {
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int rb = 0; rb < PA_WAVES; ++rb)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        o[d][rb][i] = 0.f;
            lsum = {0.f, 0.f};
            logits(0, std::integral_constant<int, 0>{}, 0);
            probabilities(mask(0));
            give(0);
            int page = SMALL ? 0 : entry(3);
#pragma unroll 1
            for (int t = 1; t < nt; ++t) {
                // (behind the last tile the gathers read its last key again)
                const int next = SMALL ? 0 : entry(t + 3);
                clean(t - 1);
                if (SMALL)
                    issue(t + 2);
                logits(t, std::integral_constant<int, PM_WITH>{}, page);
                page = next;
#pragma unroll
                for (int j = PM_WITH; j < PM_WITH + 4; ++j)
                    product_step(t - 1, j);
                __builtin_amdgcn_sched_barrier(0);
                probabilities(mask(t));
#pragma unroll
                for (int j = PM_WITH + 4; j < 32; ++j)
                    product_step(t - 1, j);
#pragma unroll
                for (int j = PM_WITH + 4; j < 32; ++j) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a matrix instruction
                    __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);  // under it, six others
                }
                give(t);
            }
            clean(nt - 1);
            product_begin(nt - 1);
#pragma unroll
            for (int j = 0; j < 32; ++j)
                product_step(nt - 1, j);
            if (lane == 0)
                ((int *)&sOver)[wave] = 0;
            if (__ballot(over) != 0 && lane == 0)
                ((int *)&sOver)[wave] = 1;
            lds_barrier();
            const v4i any = sOver;
            if (round || !__builtin_amdgcn_readfirstlane(any[0] | any[1] | any[2] | any[3]))
                break;
            over = false;
            __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
            lds_barrier();
            issue(0);
            issue(1);
#pragma unroll 1
            for (int t = 0; t < nt; ++t) {
                landed();
                lds_barrier();
                issue(t + 2);
                logits(t, std::integral_constant<int, 0>{}, 0);
                const float mult = mask(t);
                float mx = s[0];
#pragma unroll
                for (int i = 1; i < 16; ++i)
                    mx = fmaxf(mx, s[i]);
                m = fmaxf(m, mx * mult);
            }
            m = fmaxf(m, __shfl_xor(m, 32));
            __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
            lds_barrier();
            issue(0);
            issue(1);
            issue(2);
            __builtin_amdgcn_s_waitcnt(vmcnt_only(18));
            lds_barrier();
        }
        __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
    }

    const float l = lsum.sum + __shfl_xor(lsum.sum, 32);
    if (hf == 0) {
        sM[32 * wave + c32] = m;
        sL[32 * wave + c32] = l;
    }
    __syncthreads();
#pragma unroll
    for (int rb = 0; rb < PA_WAVES; ++rb) {
        const int at = 32 * rb + c32, to = r.row0 + at;
        if (to >= r.row1)
            continue;
        const float mm = sM[at], ll = sL[at];
        if (r.part >= 0) {
            const int64_t slot = r.part + at;
            if (hf == 0 && wave == 0)
                *(float2 *)(g.part + g.plan.slots * g.plan.part_rows * 512 + 2 * slot) = float2{mm, ll};
            if (nt > 0) {
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        *(v4f *)(g.part + slot * 512 + 128 * wave + 32 * d + 2 * i + 4 * hf) =
                            v4f{o[d][rb][i], o[d][rb][i + 1], o[d][rb][i + 2], o[d][rb][i + 3]};
            }
            continue;
        }
        const float inv = ll != 0.f ? 1.f / ll : 0.f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                v4f x = {0.f, 0.f, 0.f, 0.f};
                if (nt > 0)  // (without keys O has not been begun)
                    x = v4f{o[d][rb][i] * inv, o[d][rb][i + 1] * inv, o[d][rb][i + 2] * inv, o[d][rb][i + 3] * inv};
                store_out4(g.out, g.out_f32, (int64_t)to * 512 + 128 * wave + 32 * d + 2 * i + 4 * hf, x);
            }
        if (g.lse && hf == 0 && wave == 0)
            g.lse[to] = ll != 0.f ? (mm + log2f(ll)) * LN2 : -INFINITY;
    }
    if (__ballot(bad) != 0)
        add_not_finite<512, true>(g, r, sLim, base0 + sBad[wave] * PM_KT, 128 * wave, r.row0, r.row1);
}

// Joins the ranges of a row: with maxima m_s and sums l_s, M = max m_s and w_s =
// 2^(m_s - M), O = sum w_s O_s / sum w_s l_s and lse = (M + log2 sum w_s l_s) ln 2.
// A range without keys (l = 0) wrote no O.  Bound by bytes where rows are many (22528 rows
// of six ranges of 512 dims, 305 MB: 50 us, 6.1 TB/s), by latency where they are few (128 rows of
// 72 ranges of 128 dims: 4.2 us; with the maxima of all ranges first, which O's loads waited
// for, 6.3).  A worker is LANES lanes of eight dims, and WPR of them share a piece of a
// row, each with a maximum of its own until the end, so that few rows of many ranges are
// not a chain of loads (with one worker a row, 69 ranges took 55 us).
template <int DV, int LANES, int WPR>
__global__ __launch_bounds__(256) void prefix_combine(PrefixArgs g)
{
    constexpr int PIECES = DV / (8 * LANES), WORKERS = 256 / LANES;
    static_assert(WORKERS % WPR == 0, "whole pieces in a block");
    // Few rows: what was not written is read as well, and not used, since a load of O that waits for
    // its sum is another memory latency.  Many rows: that would be bytes.
    constexpr bool FEW = WPR == 16;
    __shared__ v4f sO[WPR > 1 ? 2 * 256 : 1];
    __shared__ float2 sML[WPR > 1 ? WORKERS : 1];
    const int worker = threadIdx.x / LANES, in = threadIdx.x % LANES, w = worker % WPR;
    const int slots = g.plan.slots;
    const int64_t rows = g.plan.part_rows, id = (int64_t)blockIdx.x * (WORKERS / WPR) + worker / WPR;
    const int64_t at = min(id / PIECES, rows - 1);  // row of the workspace
    const int dim = 8 * (LANES * (int)(id % PIECES) + in);
    const float2 *ml = (const float2 *)(g.part + slots * rows * DV) + at;
    const float *po = g.part + at * DV + dim;
    const int64_t step = rows * DV;
    float2 x[4];
    v4f u[4], v[4];
    auto load = [&](int s0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int s = s0 + k * WPR;
            x[k] = s < slots ? ml[s * rows] : float2{0.f, 0.f};
            if (FEW) {
                const v4f *src = (const v4f *)(po + min(s, slots - 1) * step);
                u[k] = src[0];
                v[k] = src[1];
            }
        }
        if (!FEW) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                u[k] = v[k] = v4f{0.f, 0.f, 0.f, 0.f};
                if (x[k].y != 0.f) {
                    const v4f *src = (const v4f *)(po + (s0 + k * WPR) * step);
                    u[k] = src[0];
                    v[k] = src[1];
                }
            }
        }
    };
    load(w);
    // the row of out that it is
    int row = (int)at;
    bool live = id / PIECES < rows;
    if (g.plan.prefix > 0) {
        live = live && row < g.q_start[g.num_seqs] * g.heads;
    } else {
        int row0, row1;
        tile_rows<false>(g, g.plan.whole + row / PA_ROWS, row0, row1);
        row = row0 + row % PA_ROWS;
        live = live && row < row1;
    }
    float M = M_INIT, L = 0.f;
    v4f a = {0.f, 0.f, 0.f, 0.f}, b = a;
    for (int s0 = w;;) {
        float top = M;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            top = x[k].y != 0.f ? fmaxf(top, x[k].x) : top;
        const float old = __builtin_amdgcn_exp2f(M - top);
        M = top;
        L *= old;
        a *= old;
        b *= old;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (x[k].y != 0.f) {
                const float f = __builtin_amdgcn_exp2f(x[k].x - M);
                L += f * x[k].y;
                a += f * u[k];
                b += f * v[k];
            }
        s0 += 4 * WPR;
        if (s0 >= slots)
            break;
        load(s0);
    }
    if constexpr (WPR > 1) {
        sO[2 * threadIdx.x] = a;
        sO[2 * threadIdx.x + 1] = b;
        if (in == 0)
            sML[worker] = float2{M, L};
        __syncthreads();
        if (w != 0)
            return;
        float2 y[WPR];
#pragma unroll
        for (int k = 0; k < WPR; ++k)
            y[k] = sML[worker + k];
#pragma unroll
        for (int k = 1; k < WPR; ++k)
            M = fmaxf(M, y[k].x);
        L = 0.f;
        a = b = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < WPR; ++k) {  // (a worker without keys: sums of 0)
            const float f = __builtin_amdgcn_exp2f(y[k].x - M);
            L += f * y[k].y;
            a += f * sO[2 * (threadIdx.x + k * LANES)];
            b += f * sO[2 * (threadIdx.x + k * LANES) + 1];
        }
    }
    if (!live)
        return;
    const float inv = L != 0.f ? 1.f / L : 0.f;
    store_out4(g.out, g.out_f32, (int64_t)row * DV + dim, a * inv);
    store_out4(g.out, g.out_f32, (int64_t)row * DV + dim + 4, b * inv);
    if (g.lse && dim == 0)
        g.lse[row] = L != 0.f ? (M + log2f(L)) * LN2 : -INFINITY;
}

template <int DV>
static void launch_combine(const PrefixArgs &g, hipStream_t st)
{
    auto go = [&](auto lanes, auto wpr) {
        constexpr int LANES = decltype(lanes)::value, WPR = decltype(wpr)::value;
        hipLaunchKernelGGL((prefix_combine<DV, LANES, WPR>),
                           dim3(ceil_div(g.plan.part_rows * (DV / (8 * LANES)) * WPR, 256 / LANES)), dim3(256), 0, st, g);
    };
    using std::integral_constant;
    constexpr int ALL = DV / 8;  // lanes of a whole row
    // A worker a row keeps four ranges in flight.  Few rows: sixteen workers and a block each, or to each
    // quarter of one.  Calls with four workers against these two: 8192 rows of 4 ranges of 512 dims 579 us
    // and 570, of 7.5 ranges of 128 dims 62.1 and 58.7, 1024 rows of 24 ranges of 128 dims 24.7 and 27.2;
    // 128 rows of 228 ranges of 512 dims 60.3 and 52.9, of 72 ranges of 128 dims 17.1 and 14.0,
    // 512 rows of 61 ranges of 512 dims 66.9 and 68.7, 2048 rows of 24 ranges of 128 dims 47.4 and 50.7.
    const bool few = g.plan.part_rows * DV < 1 << 17;
    if (g.plan.slots <= (few ? 4 : 16))
        go(integral_constant<int, ALL>{}, integral_constant<int, 1>{});
    else if (few)
        go(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    else
        go(integral_constant<int, ALL>{}, integral_constant<int, 4>{});
}

}  // namespace janus

using namespace janus;

extern "C" int janus_prefix_attn(const janus_batch *bt, const void *q, int Hq, int dqk, int dv, const void *k_pool,
                                 const void *v_pool, int64_t k_row_stride, int64_t v_row_stride,
                                 const int32_t *page_table, int pt_ld, int page_size, int prefix_len,
                                 float softmax_scale, void *out, janus_dtype out_dt, float *lse, void *workspace,
                                 size_t *workspace_bytes, void *stream)
{
    if (!batch_ok(bt) || !q || !k_pool || !v_pool || !page_table || !out || !workspace_bytes || Hq < 1 || dqk < 1 ||
        dv < 1 || !pow2(page_size) || !table_covers(bt, pt_ld, page_size) || k_row_stride < dqk ||
        v_row_stride < dv || prefix_len < 0 || prefix_len > bt->max_ctx)
        return JANUS_ERR_INVALID_ARG;
    auto at = [](const void *p, int a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; };
    const bool mla = dqk == 576 && dv == 512 && v_pool == k_pool && k_row_stride == v_row_stride;
    const bool mqa = dqk == 128 && dv == 128;
    if ((out_dt != JANUS_BF16 && out_dt != JANUS_F32) || (!mla && !mqa) || Hq > 128 || k_row_stride % 8 != 0 ||
        v_row_stride % 8 != 0 || k_row_stride > (1 << 24) || v_row_stride > (1 << 24) || !at(q, 16) ||
        !at(k_pool, 16) || !at(v_pool, 16) || !at(out, 4) || bt->max_ctx > (1 << 30) ||
        (int64_t)bt->total_q * Hq + (int64_t)bt->num_seqs * PA_ROWS >= (int64_t)1 << 31)
        return JANUS_ERR_UNSUPPORTED;
    const PrefixPlan plan =
        prefix_plan(bt->num_seqs, bt->total_q, bt->max_q, bt->max_ctx, bt->total_ctx, prefix_len, Hq, mla);
    if (plan.blocks > PA_MAX_BLOCKS)
        return JANUS_ERR_UNSUPPORTED;
    const size_t need = plan.slots > 1 ? (size_t)plan.slots * plan.part_rows * (dv + 2) * sizeof(float) : 0;
    if (!workspace) {
        *workspace_bytes = need;
        return JANUS_OK;
    }
    if (*workspace_bytes < need)
        return JANUS_ERR_WORKSPACE;
    if (need > 0 && !at(workspace, 16))
        return JANUS_ERR_UNSUPPORTED;
    if (bt->total_q == 0)
        return JANUS_OK;
    PrefixArgs g;
    g.q_start = bt->q_start;
    g.hist_len = bt->hist_len;
    g.num_seqs = bt->num_seqs;
    g.es = bt->entry_shift;
    g.q = (const uint16_t *)q;
    g.heads = Hq;
    g.k = (const uint8_t *)k_pool;
    g.v = (const uint8_t *)v_pool;
    g.k_rb = 2 * k_row_stride;
    g.v_rb = 2 * v_row_stride;
    g.table = page_table;
    g.pt_ld = pt_ld;
    g.page_shift = __builtin_ctz((unsigned)page_size);
    g.scale_log2 = softmax_scale * LOG2E;
    g.out = out;
    g.out_f32 = out_dt == JANUS_F32;
    g.lse = lse;
    g.part = (float *)workspace;
    g.plan = plan;
    hipStream_t st = as_stream(stream);
    if (mla)
        hipLaunchKernelGGL(page_size < 8 ? prefix_mla<true> : prefix_mla<false>, dim3(plan.blocks), dim3(PA_THREADS), 0, st, g);
    else
        hipLaunchKernelGGL(prefix_mqa, dim3(plan.blocks), dim3(PA_THREADS), 0, st, g);
    if (plan.slots == 1)
        return launch_status();
    if (hipGetLastError() != hipSuccess)
        return JANUS_ERR_DEVICE;
    if (mla)
        launch_combine<512>(g, st);
    else
        launch_combine<128>(g, st);
    return launch_status();
}
