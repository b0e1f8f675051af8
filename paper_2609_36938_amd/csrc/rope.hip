// Rotary positions, and the rows of the caches.
//
// A rotated head takes its pairs (x_a, x_b) to
//
//   (m (x_a cos t - x_b sin t), m (x_b cos t + x_a sin t)),  t = position * inv_freq[pair]
//
// (t negated for the transpose).  t is reduced to a fraction of a turn in 64
// bits, where far positions lose nothing.  Sine and cosine are taken of that fraction
// rounded to 32, and turned on by the angle d that the rounding lost (under 1e-7, so
// sin(a + d) = sin a + d cos a and cos(a + d) = cos a - d sin a to fp32's last bit):
// without that a sine near 0 keeps none of its bits.  They are worked out once per
// token and pair, into LDS, and used by all heads.
//
// One kernel does queries (many heads a token, written in place or apart) and
// cache rows (one head a token, scattered through a slot map), to fp32, bf16 or
// fp8 with one scale per token.  A token is LPR lanes (16, 64 or 256, by the
// length of its row): an fp8 row's largest value is then a reduction over
// those lanes, and short rows share a block.  A lane's unit is two groups of V
// elements, 16 bytes each (8 bf16, 4 fp32; 1 where an address or a size is odd).  Loads go out before the
// angles are worked out.
//
// Bound by the bytes read and written where there are many (8192 tokens x 128 heads x 64 rotated
// dims of bf16, 268 MB: 58 us, 4.6 TB/s; 2048 tokens x 64 heads x 128 dims to fp8, 50 MB: 12.0 us, of
// which 0.5 are the corrections of the quotients), by one chain of loads (the session, its length, the
// frequencies' angles, the slot) where there are few (16 decode queries 3.7 us, 64 cache rows to fp8
// 4.2; an empty kernel takes 2.5).  Loads behind branches, which wait for each other: 71 us for the first of these.
#include "janus_device.hpp"
#include "janus_host.hpp"

#include <math.h>
#include <type_traits>
#include <utility>

namespace janus {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_MAX_DIM = 1024;   // sines and cosines of a block fit in LDS
constexpr int ROPE_MAX_ROWS = 1 << 24;  // a launch takes fewer than 2^32 threads, 256 for the longest rows
constexpr float FP8_LARGEST = 448.f;
constexpr float AMAX_FLOOR = 1e-12f;  // an all-zero row's scale stays positive

struct RopeArgs {
    const int32_t *q_start, *ctx_start, *hist_len;
    int num_seqs, es, total_q;
    const void *x;               // plain elements (all of them where xr == nullptr)
    const void *xr;              // rotated elements, or nullptr
    int64_t x_rs, x_hs, xr_rs;   // strides in elements
    int heads, size, off, dim;   // a head's elements, and the rotated ones among them
    int halves, inverse;         // pairs (j, j + dim/2); transpose
    float mag;
    const double *inv_freq;
    const int32_t *positions;
    uint8_t *out;
    int64_t o_rs, o_hs;          // bytes
    int plain_units;             // units a head of the elements that are only copied (0: in place)
    int turn_shift, plain_shift; // log2 of a head's units of both kinds, or -1
    int pair_shift;              // log2 of a pair's elements that are neighbours
    int plain_step, plain_gap;   // elements between units (log2), and between a unit's groups
    int scatter;                 // cache rows: to `rows`, or by context where it is null
    const int64_t *rows;
    int64_t num_rows;
    float *scale;                // fp8: one per output row; null: in the row, behind its elements
};

// Session of `row`, found by LPR lanes together (64 at most).
template <int LPR>
JANUS_DEV int session_of_row_lanes(const int32_t *q_start, int num_seqs, int row)
{
    constexpr int K = LPR < kWave ? LPR : kWave;
    const int lane = threadIdx.x & 63, in = lane & (K - 1);
    int lo = 0, hi = num_seqs;  // the session is in [lo, hi)
    while (__ballot(hi - lo > 1) != 0) {
        const int step = max(1, (hi - lo + K - 1) / K);
        const int s = lo + in * step;
        uint64_t below = __ballot(s < hi && q_start[s] <= row);
        if constexpr (K < kWave)
            below = (below >> (lane & ~(K - 1))) & ((1ull << K) - 1);
        lo += max((int)__popcll(below) - 1, 0) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

// V elements as they are loaded, and as fp32.
template <class T, int V>
struct Raw {
    using Word = typename std::conditional<V == 1, T, v4i>::type;
    static constexpr int N = V * sizeof(T) / sizeof(Word);
    Word w[N];
    JANUS_DEV void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
            w[i] = ((const Word *)p)[i];
    }
    JANUS_DEV void unpack(float (&v)[V]) const
    {
        if constexpr (V == 1) {
            if constexpr (sizeof(T) == 4)
                v[0] = w[0];
            else
                v[0] = bf16_to_f32(w[0]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (sizeof(T) == 4) {
                        v[4 * i + e] = __int_as_float(w[i][e]);
                    } else {
                        v[2 * e] = __uint_as_float((uint32_t)w[i][e] << 16);
                        v[2 * e + 1] = __uint_as_float((uint32_t)w[i][e] & 0xffff0000u);
                    }
                }
        }
    }
};

// To the nearest bf16, ties to even (NaN stays NaN).
JANUS_DEV uint32_t bf16_pair(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v2f{a, b}, v2bf));
}
// To the nearest e4m3, ties to even (NaN stays NaN); the values are in its range.
JANUS_DEV uint32_t fp8_quad(float a, float b, float c, float d)
{
    v2s w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, 1.0f, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, 1.0f, true);
    return __builtin_bit_cast(uint32_t, w);
}

// An fp8 row's scale, and its reciprocal rounded to nearest.
struct Scale {
    float step, inv;
    // v / step rounded to nearest: the product with the reciprocal, corrected once by its remainder, which
    // an fma gives exactly (Markstein, IBM J. Res. Dev. 34, 1990).  The product alone is off by up to an ulp and
    // a half, which takes values next to a border of e4m3 to its other side.  (A zero keeps its sign.)
    JANUS_DEV float of(float v) const
    {
        const float q = v * inv;
        return copysignf(fmaf(fmaf(-q, step, v), inv, q), v);
    }
};

template <int DT, int V>
JANUS_DEV void store_group(uint8_t *p, const float (&v)[V], Scale s)
{
    if constexpr (DT == JANUS_F32) {
        if constexpr (V == 1) {
            *(float *)p = v[0];
        } else {
#pragma unroll
            for (int e = 0; e < V; e += 4)
                *(v4f *)(p + 4 * e) = v4f{v[e], v[e + 1], v[e + 2], v[e + 3]};
        }
    } else if constexpr (DT == JANUS_BF16) {
        if constexpr (V == 1)
            *(uint16_t *)p = (uint16_t)bf16_pair(v[0], 0.f);
        else if constexpr (V == 4)
            *(v2i *)p = v2i{(int)bf16_pair(v[0], v[1]), (int)bf16_pair(v[2], v[3])};
        else
            *(v4i *)p = v4i{(int)bf16_pair(v[0], v[1]), (int)bf16_pair(v[2], v[3]), (int)bf16_pair(v[4], v[5]),
                            (int)bf16_pair(v[6], v[7])};
    } else {
        if constexpr (V == 1)
            *p = (uint8_t)fp8_quad(s.of(v[0]), 0.f, 0.f, 0.f);
        else if constexpr (V == 4)
            *(uint32_t *)p = fp8_quad(s.of(v[0]), s.of(v[1]), s.of(v[2]), s.of(v[3]));
        else
            *(v2i *)p = v2i{(int)fp8_quad(s.of(v[0]), s.of(v[1]), s.of(v[2]), s.of(v[3])),
                            (int)fp8_quad(s.of(v[4]), s.of(v[5]), s.of(v[6]), s.of(v[7]))};
    }
}

// Where a unit lies: its head, the first elements of its two groups in the
// head (b < 0: one group), and its first pair (-1: not rotated).  The groups are half of
// the rotated, or of many plain, elements apart, so that neighbouring lanes' are neighbours
// (8192 cache rows 6.9 us with groups side by side, 6.2 so; 1000 tokens x 128 heads x 128 fp32 in
// interleaved pairs, with groups of eight, 30.5, and 21.5).
struct Unit {
    int head, a, b, pair;
};
// All heads' rotated units come first: a wave's lanes then mostly do the same.
template <int V>
JANUS_DEV Unit unit_at(const RopeArgs &g, int u)
{
    auto over = [](int x, int n, int shift) { return shift >= 0 ? x >> shift : x / n; };
    const int turned = g.dim / (2 * V), first = g.heads * turned;
    Unit at;
    if (u < first) {
        at.head = g.heads == 1 ? 0 : over(u, turned, g.turn_shift);
        const int j = (u - at.head * turned) * V;
        if constexpr (V > 1) {  // (a group of neighbours is whole pairs)
            at.pair = j >> g.pair_shift;
            at.a = g.off + j;
            at.b = at.a + g.dim / 2;
        } else {
            at.pair = j;
            at.a = g.off + (j << g.pair_shift);
            at.b = at.a + (g.halves ? g.dim / 2 : 1);
        }
    } else {
        u -= first;
        at.head = g.heads == 1 ? 0 : over(u, g.plain_units, g.plain_shift);
        const int e = (u - at.head * g.plain_units) << g.plain_step, f = e + g.plain_gap;  // among the plain elements
        at.pair = -1;
        at.a = e < g.off ? e : e + g.dim;
        at.b = f < g.off ? f : f + g.dim;
        if (at.b >= g.size)
            at.b = -1;
    }
    return at;
}

template <class T, int DT, int V, int LPR, int UPT>
__global__ __launch_bounds__(ROPE_THREADS) void rope_rows(RopeArgs g)
{
    extern __shared__ float2 turn[];  // [rows of the block][dim / 2]: cosine, sine
    __shared__ float red[ROPE_THREADS / kWave];
    constexpr int ROWS = ROPE_THREADS / LPR;
    constexpr bool FP8 = DT == JANUS_FP8_E4M3;
    const int tid = threadIdx.x, lane = tid % LPR, mine = tid / LPR;
    const bool live = (int64_t)blockIdx.x * ROWS + mine < g.total_q;
    const int row = live ? blockIdx.x * ROWS + mine : g.total_q - 1;
    const int pairs = g.dim / 2;
    const int units = g.heads * (g.dim / (2 * V) + g.plain_units);
    // fp8 rows: all units of the token, LPR * UPT at a time; others: the block's share of them
    const int u0 = FP8 ? 0 : blockIdx.y * LPR * UPT;

    // Loads without a branch, so that all of them are under way at once: lanes
    // behind the last unit take it again, units of one group take that twice.
    Unit at[UPT];
    Raw<T, V> ra[UPT], rb[UPT];
    auto load = [&](int first) {
        const T *x = (const T *)g.x + (int64_t)row * g.x_rs;
        const T *xr = g.xr ? (const T *)g.xr + (int64_t)row * g.xr_rs - g.off : nullptr;
        const int skip = g.xr ? g.dim : 0;  // the rotated elements are elsewhere
#pragma unroll
        for (int k = 0; k < UPT; ++k) {
            at[k] = unit_at<V>(g, min(first + k * LPR + lane, units - 1));
            const int a = at[k].a, b = at[k].b < 0 ? a : at[k].b;
            const bool other = at[k].pair >= 0 && g.xr;
            const T *p = other ? xr : x + (int64_t)at[k].head * g.x_hs;
            ra[k].load(p + (other || a < g.off ? a : a - skip));
            rb[k].load(p + (other || b < g.off ? b : b - skip));
        }
    };
    load(u0);
    const double freq = pairs > 0 ? g.inv_freq[min(lane, pairs - 1)] : 0.0;

    // the token's session, position and output row
    int64_t to = row;
    bool store = live && row < g.q_start[g.num_seqs];
    int pos;
    {
        const int b = session_of_row_lanes<LPR>(g.q_start, g.num_seqs, row);
        const int tokens = g.hist_len[b] + row - g.q_start[b] + 1;
        pos = g.positions ? g.positions[row] : tokens - 1;
        if (g.scatter) {
            if (g.rows) {
                to = g.rows[row];
            } else {
                to = (int64_t)g.ctx_start[b] + entries_of(tokens, g.es) - 1;
                store = store && (tokens & ((1 << g.es) - 1)) == 0;
            }
            store = store && to >= 0 && to < g.num_rows;
        }
    }
    for (int p = lane; p < pairs; p += LPR) {
        double t = (double)pos * (p < LPR ? freq : g.inv_freq[p]) * 0.15915494309189533577;  // turns
        t -= rint(t);
        const float hi = (float)t, lo = (float)(t - (double)hi) * 6.2831853071795865f;
        float s0, c0;
        sincospif(2.f * hi, &s0, &c0);
        const float s = fmaf(lo, c0, s0), c = fmaf(-lo, s0, c0);
        turn[mine * pairs + p] = float2{c * g.mag, (g.inverse ? -s : s) * g.mag};
    }
    if constexpr (LPR > kWave)
        __syncthreads();
    else
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (a token is one wave's or less)

    float va[UPT][V], vb[UPT][V];
    auto rotate = [&]() {
#pragma unroll
        for (int k = 0; k < UPT; ++k) {
            ra[k].unpack(va[k]);
            rb[k].unpack(vb[k]);
            if (at[k].pair < 0)
                continue;
            const float2 *t = turn + mine * pairs + at[k].pair;
            if (g.halves || V == 1) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float a = va[k][e], b = vb[k][e];
                    va[k][e] = a * t[e].x - b * t[e].y;
                    vb[k][e] = b * t[e].x + a * t[e].y;
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const float a = va[k][e], b = va[k][e + 1], c = vb[k][e], d = vb[k][e + 1];
                    const float2 ta = t[e / 2], tb = t[g.dim / 4 + e / 2];
                    va[k][e] = a * ta.x - b * ta.y;
                    va[k][e + 1] = b * ta.x + a * ta.y;
                    vb[k][e] = c * tb.x - d * tb.y;
                    vb[k][e + 1] = d * tb.x + c * tb.y;
                }
            }
        }
    };
    constexpr int BYTES = FP8 ? 1 : DT == JANUS_BF16 ? 2 : 4;
    auto put = [&](int first, Scale scale) {
#pragma unroll
        for (int k = 0; k < UPT; ++k) {
            if (first + k * LPR + lane >= units || !store)
                continue;
            uint8_t *p = g.out + to * g.o_rs + (int64_t)at[k].head * g.o_hs;
            store_group<DT, V>(p + (int64_t)at[k].a * BYTES, va[k], scale);
            if (at[k].b >= 0)
                store_group<DT, V>(p + (int64_t)at[k].b * BYTES, vb[k], scale);
        }
    };
    rotate();
    if constexpr (!FP8) {
        put(u0, Scale{1.f, 1.f});
    } else {
        // Largest magnitude of the token (fmaxf passes over NaN), and if that is
        // infinite, the largest finite one: infinities are then written as the largest e4m3.
        const bool again = units > LPR * UPT;
        float top = 0.f;
        bool finite = false;  // only finite ones
        auto tops = [&]() {
#pragma unroll
            for (int k = 0; k < UPT; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float a = fabsf(va[k][e]), b = fabsf(vb[k][e]);
                    top = fmaxf(top, finite && !(a < INFINITY) ? 0.f : a);
                    top = fmaxf(top, finite && !(b < INFINITY) ? 0.f : b);
                }
        };
        auto largest = [&]() {
            top = 0.f;
            tops();
            for (int u = LPR * UPT; u < units; u += LPR * UPT) {
                load(u);
                rotate();
                tops();
            }
#pragma unroll
            for (int o = 1; o < (LPR < kWave ? LPR : kWave); o <<= 1)
                top = fmaxf(top, __shfl_xor(top, o));
            if constexpr (LPR > kWave) {
                if ((tid & 63) == 0)
                    red[tid >> 6] = top;
                __syncthreads();
                top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
            }
        };
        auto fit = [&]() {
#pragma unroll
            for (int k = 0; k < UPT; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    va[k][e] = fabsf(va[k][e]) == INFINITY ? copysignf(top, va[k][e]) : va[k][e];
                    vb[k][e] = fabsf(vb[k][e]) == INFINITY ? copysignf(top, vb[k][e]) : vb[k][e];
                }
        };
        largest();
        // (by blocks where a token is one: the second pass has a barrier)
        const bool odd = LPR > kWave ? top == INFINITY : __ballot(top == INFINITY) != 0;
        if (odd) {
            if constexpr (LPR > kWave)
                __syncthreads();
            if (again) {
                load(0);
                rotate();
            }
            finite = true;
            largest();
            top = fmaxf(top, AMAX_FLOOR);
            if (!again)
                fit();
        }
        const float step = fmaxf(top, AMAX_FLOOR) / FP8_LARGEST;
        const Scale scale = {step, 1.f / step};
        if (again) {
            // a row longer than the lanes' registers is read again
            for (int u = 0; u < units; u += LPR * UPT) {
                load(u);
                rotate();
                if (odd)
                    fit();
                put(u, scale);
            }
        } else {
            put(0, scale);
        }
        if (lane == 0 && store) {
            if (g.scale)
                g.scale[to] = step;
            else
                *(float *)(g.out + to * g.o_rs + g.size) = step;
        }
    }
}

template <class T, int DT, int V>
static void launch_rope_rows(RopeArgs g, hipStream_t st)
{
    const int turned = g.dim / (2 * V), units = g.heads * (turned + g.plain_units);
    g.turn_shift = pow2(turned) ? __builtin_ctz((unsigned)turned) : -1;
    g.plain_shift = pow2(g.plain_units) ? __builtin_ctz((unsigned)g.plain_units) : -1;
    g.pair_shift = g.halves ? 0 : 1;
    // Few plain elements of a head are one line of memory either way.
    const bool many = g.plain_units >= 16;
    g.plain_step = (V == 8 ? 3 : V == 4 ? 2 : 0) + !many;
    g.plain_gap = many ? V * g.plain_units : V;
    auto go = [&](auto lanes, auto regs) {
        constexpr int LPR = decltype(lanes)::value, UPT = decltype(regs)::value;
        const int rows = ROPE_THREADS / LPR;
        hipLaunchKernelGGL((rope_rows<T, DT, V, LPR, UPT>),
                           dim3(ceil_div(g.total_q, rows), DT == JANUS_FP8_E4M3 ? 1 : ceil_div(units, LPR * UPT)),
                           dim3(ROPE_THREADS), (size_t)rows * (g.dim / 2) * sizeof(float2), st, g);
    };
    // Many rows: the fewest lanes whose registers hold one, since a lane takes as many
    // instructions whether or not it has a unit (8192 MLA rows, 36 units of 16 elements, with
    // groups side by side 6.5 us on 16 lanes of three units, 7.3 on 64 lanes of two).  Few rows: one unit a lane (64 of them 4.2 us, 4.6 with two).
    using std::integral_constant;
    constexpr int S = V == 4 ? 2 : 1;  // units of 16 elements in two
    if (V > 1 && units <= 16 * S)
        go(integral_constant<int, 16>{}, integral_constant<int, S>{});
    else if (units <= 48 * S && (V == 1 || g.total_q >= 4096))
        go(integral_constant<int, 16>{}, integral_constant<int, 3 * S>{});
    else if (V > 1 && units <= 64 * S)
        go(integral_constant<int, 64>{}, integral_constant<int, S>{});
    else if (units <= 128 * S)
        go(integral_constant<int, 64>{}, integral_constant<int, 2 * S>{});
    else
        go(integral_constant<int, 256>{}, integral_constant<int, 2 * S>{});
}

template <class T>
static int launch_rope(RopeArgs g, int x_dt, int out_dt, bool in_place, hipStream_t st)
{
    // Groups of 16 bytes of x where every one of them lies at an address of that alignment
    // (in fp8 rows 8), else single elements.
    const int64_t in = x_dt == JANUS_F32 ? 4 : 8, align = out_dt == JANUS_FP8_E4M3 ? 8 : 16;
    auto at = [](const void *p, int64_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; };
    const bool wide = g.dim % 16 == 0 && g.off % 8 == 0 && g.size % 8 == 0 && at(g.x, 16) && at(g.xr, 16) &&
                      at(g.out, align) && g.x_rs % in == 0 && g.x_hs % in == 0 && g.xr_rs % in == 0 &&
                      g.o_rs % align == 0 && g.o_hs % align == 0;
    constexpr int V = 16 / sizeof(T);
    const int plain = in_place ? 0 : g.size - g.dim;
    auto go = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (wide) {
            g.plain_units = (plain + 2 * V - 1) / (2 * V);
            launch_rope_rows<T, DT, V>(g, st);
        } else {
            g.plain_units = (plain + 1) / 2;
            launch_rope_rows<T, DT, 1>(g, st);
        }
    };
    if (out_dt == JANUS_F32)
        go(std::integral_constant<int, JANUS_F32>{});
    else if (out_dt == JANUS_BF16)
        go(std::integral_constant<int, JANUS_BF16>{});
    else
        go(std::integral_constant<int, JANUS_FP8_E4M3>{});
    return launch_status();
}

static bool rotary_ok(const janus_rotary *r, int size)
{
    return r && r->dim >= 2 && r->dim % 2 == 0 && r->offset >= 0 && r->offset <= size - r->dim && r->inv_freq &&
           (r->layout == JANUS_ROTARY_HALVES || r->layout == JANUS_ROTARY_INTERLEAVED);
}

// Rows of `size` elements at these strides share none: the smaller stride holds a row,
// the larger one all rows of the smaller.
static bool apart(int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t size)
{
    if (n1 <= 1 || (n2 > 1 && s2 < s1)) {
        std::swap(n1, n2);
        std::swap(s1, s2);
    }
    return n1 <= 1 || (s1 >= size && (n2 <= 1 || s2 >= s1 * (n1 - 1) + size));
}

static RopeArgs rope_args(const janus_batch *b, const janus_rotary *r)
{
    RopeArgs g = {};
    g.q_start = b->q_start;
    g.ctx_start = b->ctx_start;
    g.hist_len = b->hist_len;
    g.num_seqs = b->num_seqs;
    g.es = b->entry_shift;
    g.total_q = b->total_q;
    if (r) {
        g.off = r->offset;
        g.dim = r->dim;
        g.halves = r->layout == JANUS_ROTARY_HALVES;
        g.inverse = r->inverse != 0;
        g.mag = r->magnitude;
        g.inv_freq = r->inv_freq;
        g.positions = r->positions;
    }
    return g;
}

}  // namespace janus

using namespace janus;

extern "C" int janus_rope(const janus_batch *b, const janus_rotary *r, const void *x, janus_dtype x_dt,
                          int64_t x_row_stride, int64_t x_head_stride, int heads, int size, void *out,
                          janus_dtype out_dt, int64_t out_row_stride, int64_t out_head_stride, float *out_scale,
                          void *stream)
{
    if (!batch_ok(b) || !x || !out || heads < 1 || size < 1 || !rotary_ok(r, size) || !dtype_ok(x_dt) ||
        !dtype_ok(out_dt) || x_row_stride < 0 || x_head_stride < 0 || out_row_stride < 0 || out_head_stride < 0)
        return JANUS_ERR_INVALID_ARG;
    if (!apart(b->total_q, out_row_stride, heads, out_head_stride, size))
        return JANUS_ERR_INVALID_ARG;
    const bool fp8 = out_dt == JANUS_FP8_E4M3;
    if (fp8 != (out_scale != nullptr))
        return JANUS_ERR_INVALID_ARG;
    const bool in_place = out == x;
    if (in_place && (x_dt != out_dt || x_row_stride != out_row_stride || x_head_stride != out_head_stride))
        return JANUS_ERR_INVALID_ARG;
    if (x_dt == JANUS_FP8_E4M3 || r->dim > ROPE_MAX_DIM || (int64_t)heads * size > (1 << 24) ||
        b->total_q >= ROPE_MAX_ROWS)
        return JANUS_ERR_UNSUPPORTED;
    if (b->total_q == 0)
        return JANUS_OK;
    const int64_t ob = out_dt == JANUS_F32 ? 4 : out_dt == JANUS_BF16 ? 2 : 1;
    RopeArgs g = rope_args(b, r);
    g.x = x;
    g.x_rs = x_row_stride;
    g.x_hs = x_head_stride;
    g.heads = heads;
    g.size = size;
    g.out = (uint8_t *)out;
    g.o_rs = out_row_stride * ob;
    g.o_hs = out_head_stride * ob;
    g.scale = out_scale;
    return x_dt == JANUS_F32 ? launch_rope<float>(g, x_dt, out_dt, in_place, as_stream(stream))
                             : launch_rope<uint16_t>(g, x_dt, out_dt, in_place, as_stream(stream));
}

extern "C" int janus_kv_append(const janus_batch *b, const janus_rotary *r, const void *x, janus_dtype x_dt,
                               int64_t x_row_stride, const void *x_rot, int64_t x_rot_stride, int size,
                               const int64_t *rows, int64_t num_rows, void *out, janus_dtype out_dt,
                               int64_t out_row_bytes, float *out_scale, void *stream)
{
    if (!batch_ok(b) || !out || size < 1 || num_rows < 0 || !dtype_ok(x_dt) || !dtype_ok(out_dt) ||
        x_row_stride < 0 || x_rot_stride < 0 || (r && !rotary_ok(r, size)) || (x_rot && !r) ||
        (!x && !(x_rot && r->dim == size)) || (!rows && !b->ctx_start))
        return JANUS_ERR_INVALID_ARG;
    const int64_t ob = out_dt == JANUS_F32 ? 4 : out_dt == JANUS_BF16 ? 2 : 1;
    const bool fp8 = out_dt == JANUS_FP8_E4M3, inlined = fp8 && !out_scale;
    if (out_row_bytes < size * ob + (inlined ? 4 : 0) || out_row_bytes % ob != 0 || (out_scale && !fp8))
        return JANUS_ERR_INVALID_ARG;
    if (x_dt == JANUS_FP8_E4M3 || (r && r->dim > ROPE_MAX_DIM) || size > (1 << 24) ||
        b->total_q >= ROPE_MAX_ROWS)
        return JANUS_ERR_UNSUPPORTED;
    // the scale in the row is one aligned word
    if (inlined && (size % 4 != 0 || out_row_bytes % 4 != 0 || (reinterpret_cast<uintptr_t>(out) & 3) != 0))
        return JANUS_ERR_UNSUPPORTED;
    if (b->total_q == 0 || num_rows == 0)
        return JANUS_OK;
    RopeArgs g = rope_args(b, r);
    g.x = x;
    g.xr = x_rot;
    g.x_rs = x_row_stride;
    g.xr_rs = x_rot_stride;
    g.heads = 1;
    g.size = size;
    g.out = (uint8_t *)out;
    g.o_rs = out_row_bytes;
    g.scatter = 1;
    g.rows = rows;
    g.num_rows = num_rows;
    g.scale = out_scale;
    return x_dt == JANUS_F32 ? launch_rope<float>(g, x_dt, out_dt, false, as_stream(stream))
                             : launch_rope<uint16_t>(g, x_dt, out_dt, false, as_stream(stream));
}

extern "C" int janus_rotary_frequencies(int dim, double base, double factor, int scaling, int original_ctx,
                                        double beta_fast, double beta_slow, double *inv_freq, float *magnitude)
{
    if (dim < 2 || dim % 2 != 0 || !(base > 1.0) || !inv_freq || !magnitude || !(factor >= 1.0) ||
        scaling < JANUS_SCALING_NONE || scaling > JANUS_SCALING_YARN ||
        (scaling == JANUS_SCALING_YARN && (original_ctx < 1 || !(beta_slow > 0.0) || !(beta_fast > beta_slow))))
        return JANUS_ERR_INVALID_ARG;
    // the pair whose wave makes `turns` turns over the original context
    auto pair_of = [&](double turns) { return dim * log(original_ctx / (2.0 * M_PI * turns)) / (2.0 * log(base)); };
    double low = 0.0, high = 0.0;
    if (scaling == JANUS_SCALING_YARN) {
        low = fmax(floor(pair_of(beta_fast)), 0.0);
        high = fmin(ceil(pair_of(beta_slow)), dim - 1.0);
    }
    for (int j = 0; j < dim / 2; ++j) {
        const double f = pow(base, -2.0 * j / dim);
        double stretched = 0.0;  // share of the stretched frequency
        if (scaling == JANUS_SCALING_LINEAR)
            stretched = 1.0;
        else if (scaling == JANUS_SCALING_YARN)
            stretched = fmin(fmax((j - low) / fmax(high - low, 1e-3), 0.0), 1.0);
        inv_freq[j] = f * (1.0 - stretched) + f / factor * stretched;
    }
    *magnitude = scaling == JANUS_SCALING_YARN ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
    return JANUS_OK;
}
