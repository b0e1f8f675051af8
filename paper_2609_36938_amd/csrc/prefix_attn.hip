// Dense causal attention over the paged cache, for a batch whose sessions
// begin with a common prefix.
//
// A row is one (token, head).  A block takes 128 rows and a range of keys and
// goes over them once with a running maximum and sum (exp2 domain):
//   * 32 or 64 keys at a time come straight into LDS (global_load_lds), into a
//     ring of tile buffers.  Within a row the 16-byte chunks are exchanged by the
//     row's number (swz), so that neither the row-wise reads of K nor the
//     transposing reads of V meet in a bank.
//   * A wave has 32 of the rows: their queries in registers, S^T = K Q^T on
//     32x32x16 MFMA.  A lane's results then are one row's logits, and the
//     exponentials, as they lie, the operand of O^T = V^T P^T: probabilities
//     never leave the lane, and rescaling O needs no exchange.
//   * Rows of different sessions share the blocks over the prefix: its keys are
//     read once for 128 rows instead of once for each session's heads.
// Ranges of one row are joined by their maxima and sums (prefix_combine).
#include "attn_device.hpp"
#include "janus_device.hpp"
#include "janus_host.hpp"
#include "launch_rules.hpp"

#include <algorithm>

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
    float *part;  // null: one range a row, written to out
    PrefixPlan plan;
};

// Exchange of a row's 16-byte chunks: chunk c of row r lies at c ^ swz(r).
// Eight rows of four neighbouring chunks (a transposing read) and sixteen rows
// of one (a K read) then spread over the banks evenly.  Rows of 256 bytes begin in
// the same bank; MLA rows (4.5 x 256) alternate between two halves.
template <int RB>
JANUS_DEV int swz(int r)
{
    if constexpr (RB % 256 == 0)
        return ((r & 1) << 3) | ((r & 2) << 1) | ((r & 4) >> 1) | ((r & 8) >> 3);
    else
        return ((r & 2) << 1) | ((r & 4) >> 1) | ((r & 8) >> 3);
}

template <int DQK, int DV, bool ONE, int KT, int NBUF>
__global__ __launch_bounds__(PA_THREADS, 1) void prefix_attn(PrefixArgs g)
{
    constexpr int KRB = DQK * 2, VRB = ONE ? KRB : DV * 2;  // bytes of a row in LDS
    constexpr int KBUF = KT * KRB, BUF = KBUF + (ONE ? 0 : KT * VRB);
    constexpr int KI = KBUF / (1024 * PA_WAVES), VI = ONE ? 0 : KT * VRB / (1024 * PA_WAVES);
    constexpr int STEPS = DQK / 16, NB = DV / 32, NK = KT / 32;
    static_assert(KI * 1024 * PA_WAVES == KBUF, "whole gathers");
    __shared__ __attribute__((aligned(16))) uint8_t ring[NBUF * BUF];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c32 = lane & 31, hf = lane >> 5;
    const PrefixBlock bk = prefix_block(g.plan, blockIdx.x);
    // the block's rows, keys [kbeg, kend) and table
    int row0, row1, kbeg, kend, sess = 0;
    if (bk.shared) {
        row0 = bk.tile * PA_ROWS;
        row1 = min(row0 + PA_ROWS, g.q_start[g.num_seqs] * g.heads);
        kbeg = bk.chunk * g.plan.chunk;
        kend = min(kbeg + g.plan.chunk, g.plan.prefix);
    } else {
        int lo = 0, hi = g.num_seqs - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (prefix_tile_first(g.q_start[mid], g.heads, mid) <= bk.tile)
                lo = mid;
            else
                hi = mid - 1;
        }
        sess = lo;
        const int q0 = g.q_start[sess], q1 = g.q_start[sess + 1];
        row0 = q0 * g.heads + (bk.tile - prefix_tile_first(q0, g.heads, sess)) * PA_ROWS;
        row1 = min(row0 + PA_ROWS, q1 * g.heads);
        if (row0 >= row1)
            return;
        kbeg = g.plan.prefix + bk.chunk * g.plan.chunk;
        kend = min(kbeg + g.plan.chunk, last_cand(g.hist_len[sess], (row1 - 1) / g.heads - q0, g.es) + 1);
    }
    if (row0 >= row1)
        return;
    const int32_t *pt = g.table + (int64_t)sess * g.pt_ld;
    // this lane's row and the end of its keys
    const int row = row0 + 32 * wave + c32;
    const bool live = row < row1;
    const int token = (live ? row : row1 - 1) / g.heads;
    const int mine = bk.shared ? session_of_row(g.q_start, g.num_seqs, token) : sess;
    const int lim = min(kend, last_cand(g.hist_len[mine], token - g.q_start[mine], g.es) + 1);
    int wmin = live ? lim : 0x7fffffff;  // keys before it are every row's of the wave
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
        wmin = min(wmin, __shfl_xor(wmin, o));
    wmin = __builtin_amdgcn_readfirstlane(wmin);

    v8bf qf[STEPS];
    {
        const uint16_t *qr = g.q + (int64_t)(live ? row : row1 - 1) * DQK + 8 * hf;
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
    float m = M_INIT, lsum = 0.f;

    // Tiles begin at multiples of KT: a tile of a page of at least KT ids lies
    // in one page.  Keys outside [kbeg, kend) load the nearest one inside.
    const int base0 = kbeg & ~(KT - 1);
    const int nt = kend > kbeg ? (kend - base0 + KT - 1) / KT : 0;
    const bool one_page = (1 << g.page_shift) >= KT;
    auto slot_of = [&](int key) {
        return ((int64_t)pt[key >> g.page_shift] << g.page_shift) + (key & ((1 << g.page_shift) - 1));
    };
    auto issue = [&](int t) {
        uint8_t *dst = ring + (t % NBUF) * BUF;
        const int base = base0 + t * KT;
        const int first = max(kbeg - base, 0), last = min(kend - base, KT) - 1;
        const int64_t slot0 = one_page ? slot_of(base) : 0;
#pragma unroll
        for (int j = 0; j < KI + VI; ++j) {
            const bool isv = j >= KI;
            const int rb16 = (isv ? VRB : KRB) / 16;
            const int at = 64 * (wave + PA_WAVES * (isv ? j - KI : j));
            const int p = at + lane, r = p / rb16, c = p - r * rb16;
            const int rr = min(max(r, first), last);
            const int64_t slot = one_page ? slot0 + rr : slot_of(base + rr);
            const uint8_t *src = (isv ? g.v : g.k) + slot * (isv ? g.v_rb : g.k_rb) +
                                 16 * (isv ? c ^ swz<VRB>(r) : c ^ swz<KRB>(r));
            gather16(src, dst + (isv ? KBUF : 0) + 16 * at);
        }
    };
#pragma unroll
    for (int t = 0; t < NBUF - 1; ++t)
        if (t < nt)
            issue(t);

    const int kcol = (hf ^ swz<KRB>(c32)) * 16;  // K: chunk 2 st + hf of key c32
    // V: this lane addresses key 16 s + 8 u + 4 hf + (lane / 4) % 4 and dims 32 d + 16 (lane / 16 % 2) + 4 (lane % 4)
    const int vkey = 4 * hf + ((lane >> 2) & 3);
    const int vch = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    for (int t = 0; t < nt; ++t) {
        if (NBUF > 2 && t + 1 < nt)
            __builtin_amdgcn_s_waitcnt(vmcnt_only(KI + VI));
        else
            __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
        lds_barrier();
        if (t + NBUF - 1 < nt)
            issue(t + NBUF - 1);
        const uint8_t *tile = ring + (t % NBUF) * BUF;
        const uint8_t *vt = ONE ? tile : tile + KBUF;
        const int base = base0 + t * KT;

        // K operands are read AHEAD steps before their MFMA, with a scheduling
        // fence a step: the compiler alone hoists as many reads as it finds, and spills.
        v16f s[NK];
        {
            constexpr int AHEAD = 4, ALL = NK * STEPS;
            auto kop = [&](int x) {
                // step x / NK of keys 32 (x % NK) + c32; chunk 2 st + hf, exchanged: the low bits
                // by xor, the others as they are
                constexpr int LOW = KRB % 256 == 0 ? 8 : 4;  // steps whose chunks the exchange mixes
                const int st = x / NK;
                return *(const v4i *)(tile + (32 * (x % NK) + c32) * KRB + (kcol ^ (32 * (st % LOW))) +
                                      32 * (st - st % LOW));
            };
            v4i ahead[AHEAD];
#pragma unroll
            for (int x = 0; x < AHEAD; ++x)
                ahead[x] = kop(x);
#pragma unroll
            for (int kb = 0; kb < NK; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[kb][i] = 0.f;
#pragma unroll
            for (int x = 0; x < ALL; ++x) {
                const v4i a = ahead[x % AHEAD];
                s[x % NK] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_v8bf(a), qf[x / NK], s[x % NK], 0, 0, 0);
                if (x + AHEAD < ALL)
                    ahead[x % AHEAD] = kop(x + AHEAD);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        // keys 32 kb + 8 (i / 4) + 4 hf + i % 4 of this lane's row
        const bool whole = base >= kbeg && base + KT <= wmin && g.scale_log2 > 0.f;
        float mx = -INFINITY, mult = g.scale_log2;
        if (whole) {
#pragma unroll
            for (int kb = 0; kb < NK; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    mx = fmaxf(mx, s[kb][i]);
            mx *= mult;
        } else {
#pragma unroll
            for (int kb = 0; kb < NK; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = base + 32 * kb + 8 * (i / 4) + 4 * hf + i % 4;
                    s[kb][i] = key >= kbeg && key < lim ? s[kb][i] * mult : -INFINITY;
                    mx = fmaxf(mx, s[kb][i]);
                }
            mult = 1.f;
        }
        if (__ballot(mx > m + RESCALE_SLACK) != 0) {
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float mnew = mx > m + RESCALE_SLACK ? mx : m;
            const float alpha = __builtin_amdgcn_exp2f(m - mnew);
            lsum *= alpha;
            m = mnew;
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    o[d][i] *= alpha;
        }
        v8bf pb[2 * NK];
#pragma unroll
        for (int kb = 0; kb < NK; ++kb)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v8f p;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(s[kb][8 * h + e] * mult - m);
                    lsum += p[e];
                }
                pb[2 * kb + h] = __builtin_convertvector(p, v8bf);
            }
        auto vop = [&](int h, int d) {
            v8bf a;
            v4s16 part[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int r = 16 * h + 8 * u + vkey;
                part[u] = lds_read_tr16(vt, r * VRB + 16 * ((4 * d + vch) ^ swz<VRB>(8 * u + vkey)) + 8 * (lane & 1));
            }
            __builtin_memcpy(&a, part, 16);
            return a;
        };
        // V^T P^T, its V operands read ahead likewise.
        constexpr int VALL = 2 * NK * NB, VAHEAD = 4;
        // Where rows of the tile end at different keys, a probability of 0 does not undo an
        // infinity or NaN that a row of V holds for another token.  With any of
        // them in the tile, they are left out of the product, and come back as the
        // overflow of products of large finite numbers, which are 0 for rows without the key.
        bool odd = false;
        if (!whole) {
            int bad = 0;
#pragma unroll 4
            for (int w = 0; w < KT * VRB / 1024; ++w) {
                const v4i x = *(const v4i *)(vt + 1024 * w + 16 * lane);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    bad |= (x[e] & 0x7f80) == 0x7f80 || (x[e] & 0x7f800000) == 0x7f800000;
            }
            odd = __ballot(bad) != 0;
        }
        if (!odd) {
            v8bf ahead[VAHEAD];
#pragma unroll
            for (int x = 0; x < VAHEAD; ++x)
                ahead[x] = vop(x / NB, x % NB);
#pragma unroll
            for (int x = 0; x < VALL; ++x) {
                o[x % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ahead[x % VAHEAD], pb[x / NB], o[x % NB], 0, 0, 0);
                if (x + VAHEAD < VALL)
                    ahead[x % VAHEAD] = vop((x + VAHEAD) / NB, (x + VAHEAD) % NB);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2 * NK; ++h) {
                v4i has;  // the largest bf16 for keys that the row has
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int key = base + 16 * h + 8 * (w / 2) + 4 * hf + 2 * (w % 2);
                    has[w] = (key >= kbeg && key < lim ? 0x7f7f : 0) |
                             (key + 1 >= kbeg && key + 1 < lim ? 0x7f7f0000 : 0);
                }
#pragma unroll
                for (int d = 0; d < NB; ++d) {
                    const v4i a = __builtin_bit_cast(v4i, vop(h, d));
                    v4i fin, up, down;  // finite values; +inf or NaN; -inf or NaN
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        fin[w] = up[w] = down[w] = 0;
#pragma unroll
                        for (int z = 0; z < 32; z += 16) {
                            const int x = a[w] >> z & 0xffff;
                            const bool bad = (x & 0x7f80) == 0x7f80;
                            fin[w] |= bad ? 0 : x << z;
                            up[w] |= bad && x != 0xff80 ? 0x7f7f << z : 0;
                            down[w] |= bad && x != 0x7f80 ? 0xff7f << z : 0;
                        }
                    }
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_v8bf(fin), pb[h], o[d], 0, 0, 0);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_v8bf(up), as_v8bf(has), o[d], 0, 0, 0);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_v8bf(down), as_v8bf(has), o[d], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    }

    float l = lsum + __shfl_xor(lsum, 32);
    if (!live)
        return;
    if (g.part) {
        const int64_t at = (int64_t)bk.slot * g.plan.rows + row;
        if (hf == 0)
            *(float2 *)(g.part + (int64_t)g.plan.slots * g.plan.rows * DV + 2 * at) = float2{m, l};
        if (nt > 0) {
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *(v4f *)(g.part + at * DV + 32 * d + 2 * i + 4 * hf) =
                        v4f{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
        }
        return;
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int d = 0; d < NB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            store_out4(g.out, g.out_f32, (int64_t)row * DV + 32 * d + 2 * i + 4 * hf,
                       v4f{o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv});
    if (g.lse && hf == 0)
        g.lse[row] = l != 0.f ? (m + log2f(l)) * LN2 : -INFINITY;
}

// Joins the ranges of a row: with maxima m_s and sums l_s, M = max m_s and w_s =
// 2^(m_s - M), O = sum w_s O_s / sum w_s l_s and lse = (M + log2 sum w_s l_s) ln 2.
// Eight dims a lane; a range without keys (l = 0) wrote no O.
template <int DV>
__global__ __launch_bounds__(256) void prefix_combine(const float *__restrict__ part, int slots, int rows,
                                                      const int32_t *__restrict__ q_start, int num_seqs, int heads,
                                                      void *__restrict__ out, int out_f32, float *__restrict__ lse)
{
    constexpr int LANES = DV / 8;
    const int row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, in = threadIdx.x % LANES;
    if (row >= q_start[num_seqs] * heads || row >= rows)
        return;
    const float2 *ml = (const float2 *)(part + (int64_t)slots * rows * DV) + row;
    float M = M_INIT;
    for (int s = 0; s < slots; ++s) {
        const float2 x = ml[(int64_t)s * rows];
        if (x.y != 0.f)
            M = fmaxf(M, x.x);
    }
    float L = 0.f;
    v4f a = {0.f, 0.f, 0.f, 0.f}, b = a;
    for (int s = 0; s < slots; ++s) {
        const float2 x = ml[(int64_t)s * rows];
        if (x.y == 0.f)
            continue;
        const float w = __builtin_amdgcn_exp2f(x.x - M);
        const v4f *src = (const v4f *)(part + ((int64_t)s * rows + row) * DV) + 2 * in;
        L += w * x.y;
        a += w * src[0];
        b += w * src[1];
    }
    const float inv = L != 0.f ? 1.f / L : 0.f;
    store_out4(out, out_f32, (int64_t)row * DV + 8 * in, a * inv);
    store_out4(out, out_f32, (int64_t)row * DV + 8 * in + 4, b * inv);
    if (lse && in == 0)
        lse[row] = L != 0.f ? (M + log2f(L)) * LN2 : -INFINITY;
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
        v_row_stride % 8 != 0 || k_row_stride > (1 << 30) || v_row_stride > (1 << 30) || !at(q, 16) ||
        !at(k_pool, 16) || !at(v_pool, 16) || !at(out, 4) || (int64_t)bt->total_q * Hq >= (int64_t)1 << 31)
        return JANUS_ERR_UNSUPPORTED;
    const PrefixPlan plan = prefix_plan(bt->num_seqs, bt->total_q, bt->max_q, bt->max_ctx, bt->total_ctx, prefix_len,
                                        Hq, mla);
    const size_t need = plan.slots > 1 ? (size_t)plan.slots * plan.rows * (dv + 2) * sizeof(float) : 0;
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
    g.part = plan.slots > 1 ? (float *)workspace : nullptr;
    g.plan = plan;
    hipStream_t st = as_stream(stream);
    if (mla)
        hipLaunchKernelGGL((prefix_attn<576, 512, true, 32, 3>), dim3(plan.blocks), dim3(PA_THREADS), 0, st, g);
    else
        hipLaunchKernelGGL((prefix_attn<128, 128, false, 64, 2>), dim3(plan.blocks), dim3(PA_THREADS), 0, st, g);
    if (!g.part)
        return launch_status();
    if (hipGetLastError() != hipSuccess)
        return JANUS_ERR_DEVICE;
    const int lanes = dv / 8;
    hipLaunchKernelGGL(mla ? prefix_combine<512> : prefix_combine<128>, dim3(ceil_div(plan.rows, 256 / lanes)),
                       dim3(256), 0, st, g.part, plan.slots, plan.rows, bt->q_start, bt->num_seqs, Hq, out, g.out_f32,
                       lse);
    return launch_status();
}
