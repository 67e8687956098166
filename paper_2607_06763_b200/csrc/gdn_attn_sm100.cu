// Attention over a paged cache for units of more than 64 rows (trees and prompt chunks of the query heads that share a key/value
// head): bf16, heads of 64 or 128 components, both products on the tensor cores with their sums in tensor memory.  The formulas stand
// in gdn_attn_general.cu.
//
// A unit has 256 rows, two streams of 128 that share every tile of 128 keys and values: at the tensor cores' rate a tile for one
// stream alone would ask L2 for 64 bytes per clock and SM, for two for half of that.  Per tile a stream goes through
//     S = Q K^T  ->  weights P of its rows (one thread each)  ->  O += P V
// and its next S stands behind its P V in the tensor cores' queue; while one stream forms weights the other multiplies.  P
// overwrites S in tensor memory (128 columns of S and D of O per stream).  Maxima that rise by less than 2^8 do not move the sums:
// weights up to 256 are as exact in bf16, and O is multiplied only where a row's maximum has risen by more.
//
// Roles: warps 0-3 and 4-7 the rows of the streams, warp 8 the tiles of keys and warp 9 those of values, which warp 11 looks at where
// not all rows see them, warp 10 the products.  Two or more stages of keys and of values, each with its own barriers.  Pages whose size
// is a multiple of 8 come by tensor copies, a page or a part of one each, straight into the swizzled layout of the products' operands;
// others by cp.async, row by row, which one warp cannot issue as fast as the products go (trees of 32 sequences: 294 us with pages of 7
// tokens, 183 with pages of 16).
// A row's 128 scores stay in its thread's registers (the warps of the rows take over what the others leave).
// Every wait is bounded; one that expires raises a flag that ends the others.
#include "gdn_attn.cuh"

namespace gdn {

namespace {

constexpr int AS_THREADS = 384;
constexpr int AS_M = 256, AS_TN = 128, AS_MOST = 4;
constexpr float AS_SLACK = 8.f;   // a maximum may rise by this many powers of two before the sums follow

template <int D> __host__ __device__ constexpr int as_tile_bytes() { return AS_TN * D * 2; }
// Tiles of keys, and of values, on their way or at work: what shared memory holds beside the queries.  (Trees of 32 sequences: with two tiles
// of values 187 us on pages of 16 tokens and 196 on pages of 24, with three 183 and 193.)
template <int D> __host__ __device__ constexpr int as_k_stages() { return D == 128 ? 2 : 4; }
template <int D> __host__ __device__ constexpr int as_v_stages() { return D == 128 ? 3 : 4; }
template <int D> __host__ __device__ constexpr size_t as_smem() { return (size_t)as_tile_bytes<D>() * (2 + as_k_stages<D>() + as_v_stages<D>()) + 1024; }

struct UnitShared {
    unsigned long long anc[AT_SMALL_ROWS];
    int anc_up[AT_SMALL_ROWS];
    unsigned long long q_full, k_full[AS_MOST], v_full[AS_MOST], v_landed[AS_MOST], k_empty[AS_MOST], v_empty[AS_MOST], s_full[2], p_full[2][2], o_full[2];   // p_full: [half of the tile][stream]
    uint32_t tmem;
    int odd, dead;
};

// Byte offset of 16-byte piece c of row r of a [128][D] operand tile: [D / 64][128 rows][128 bytes], swizzled.
__device__ __forceinline__ uint32_t as_at(int r, int c) { return (uint32_t)((c >> 3) * (AS_TN * 128)) + sw128_row_offset(r, c & 7); }

// The same tile seen with its rows along the product's K (values): 64 components contiguous, blocks of 64 AS_TN * 128 bytes
// apart, eight rows 1024.
__device__ __forceinline__ uint64_t desc_rows_along_k(uint32_t addr)
{
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)((AS_TN * 128) >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void umma_bf16_ts_into(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
#define GDN_TMEM_ST16(taddr, r)                                                                              \
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"    \
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),       \
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])              \
                 : "memory")

// One arrival for a whole warp.  (An arrival per thread has the 128 of a stream one behind the other: 500 clocks.)
__device__ __forceinline__ void mbar_arrive_warp(uint32_t bar, int lane)
{
    __syncwarp();
    if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

// Bit j: row node `node` sees token t0 + j.
__device__ __forceinline__ uint32_t seen_word(const AttnParams &p, AttnMaskKind kind, const unsigned long long *anc, const AttnSeq &s, int node, int t0)
{
    if (!p.row_offsets) return low_bits(s.len - t0);
    if (kind == AT_CHAIN) return low_bits(s.len + node + 1 - t0);
    const int first = t0 - s.len;   // the node whose bit comes first, negative: that many committed tokens in front
    if (first <= -32) return ~0u;
    if (kind == AT_WORDS64) {
        const unsigned long long a = anc[node];
        return first >= 64 ? 0u : first >= 0 ? (uint32_t)(a >> first) : (uint32_t)(a << -first) | low_bits(-first);
    }
    const uint32_t *row = p.mask + (size_t)(s.row0 + node) * p.mask_words;   // (words behind the node's own are not written)
    const int last = node >> 5;
    if (first < 0) return row[0] << -first | low_bits(-first);
    const int w = first >> 5;
    const uint32_t lo = w <= last ? row[w] : 0u, hi = w + 1 <= last ? row[w + 1] : 0u;
    return __funnelshift_r(lo, hi, first & 31);
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *tm, int x, int y, int z, int w, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(tm), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

struct CacheMaps {
    CUtensorMap k, v;   // [page][head][token][component], boxes of 64 components of `box` tokens
    int box;
};

// Makes what is infinite or no number in eight bf16 values zero; whether there was any.
__device__ __forceinline__ bool zero_odd(uint4 &u)
{
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint32_t &y = (&u.x)[e];
        if ((y & 0x7F80u) == 0x7F80u) { y &= 0xFFFF0000u; odd = true; }
        if ((y & 0x7F800000u) == 0x7F800000u) { y &= 0xFFFFu; odd = true; }
    }
    return odd;
}

// Two fp32 operations at once.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 d, a, b, c;\n\t"
        "mov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
// 2^x of two numbers of at most 2^7 without the special function unit, which forms 16 per clock and SM where a tile pair's products
// leave time for 32768 / 2048: x = n + r, |r| <= 1/2, 2^r by the polynomial of degree 3 with p(0) = 1 that is off by the least
// relative error there, 1.0e-4 (fitted to 2^r; a twentieth of the step of the bf16 weights), and n into the exponent.  Below
// 2^-126 the result stays there, and so it does for what is no number: not for scores that are hidden, and not for a tile of a row whose
// largest score is infinite or among whose scores one is no number.
__device__ __forceinline__ float2 power_of_two_by_products(float2 x)
{
    x.x = fmaxf(x.x, -126.f);
    x.y = fmaxf(x.y, -126.f);
    const float2 big = make_float2(12582912.f, 12582912.f);   // 1.5 * 2^23: rounds to whole numbers, which stand in the low bits
    const float2 n = add2(x, big);
    const float2 r = add2(x, fma2(n, make_float2(-1.f, -1.f), big));
    float2 y = fma2(r, make_float2(0.05500893294811249f, 0.05500893294811249f), make_float2(0.2422109693288803f, 0.2422109693288803f));
    y = fma2(r, y, make_float2(0.6932829022407532f, 0.6932829022407532f));
    y = fma2(r, y, make_float2(1.f, 1.f));
    return make_float2(__int_as_float(__float_as_int(y.x) + (__float_as_int(n.x) << 23)), __int_as_float(__float_as_int(y.y) + (__float_as_int(n.y) << 23)));
}

// The largest of three; no number where one of them is none.
__device__ __forceinline__ float max3_nan(float a, float b, float c)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// What all warps know of the unit at hand.
struct Unit {
    AttnSegment g;
    int row_first, rows, upto, tile1, n_tiles, streams;
    int common;   // tokens that all its rows see: what lies behind them is hidden from some
};

template <int D, bool TMA> __global__ void __launch_bounds__(AS_THREADS, 1)
attn_sm100_kernel(const AttnParams p, const __grid_constant__ CacheMaps maps)
{
    constexpr int TILE = as_tile_bytes<D>(), KS = D / 16, PIECES = D / 8, K_STAGES = as_k_stages<D>(), V_STAGES = as_v_stages<D>();
    extern __shared__ __align__(16) unsigned char as_raw[];
    __shared__ UnitShared sh;
    unsigned char *const data = as_raw + ((1024u - (smem_u32(as_raw) & 1023u)) & 1023u);   // swizzled tiles begin on 1024 bytes
    const uint32_t q_s = smem_u32(data), k_s = q_s + 2 * TILE, v_s = k_s + K_STAGES * TILE;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = (int)blockIdx.x;
    const AttnMaskKind kind = attn_mask_kind(p);
    const __nv_bfloat16 *k_cache = static_cast<const __nv_bfloat16 *>(p.k_cache), *v_cache = static_cast<const __nv_bfloat16 *>(p.v_cache);

    if (tid == 0) {
        mbar_init(smem_u32(&sh.q_full), 8);
        for (int i = 0; i < AS_MOST; ++i) {
            mbar_init(smem_u32(&sh.k_full[i]), 1);
            mbar_init(smem_u32(&sh.v_full[i]), 1);
            mbar_init(smem_u32(&sh.v_landed[i]), 1);
            mbar_init(smem_u32(&sh.k_empty[i]), 1);
            mbar_init(smem_u32(&sh.v_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh.s_full[i]), 1);
            mbar_init(smem_u32(&sh.p_full[0][i]), 4);
            mbar_init(smem_u32(&sh.p_full[1][i]), 4);
            mbar_init(smem_u32(&sh.o_full[i]), 1);
        }
        sh.dead = 0;
    }
    wait_for_previous_kernel();
    if (warp == 10) tmem_alloc(smem_u32(&sh.tmem), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;   // stream s: S (and P over it) at columns s * 256, O at s * 256 + 128
    volatile int *dead = &sh.dead;

    auto wait_alone = [&](unsigned long long *bar, uint32_t parity) {   // false: expired here or elsewhere
        const uint32_t at = smem_u32(bar);
        bool there = mbar_try_wait(at, parity);
        if (!there) {
            const long long t0 = clock64();
            while (!(there = mbar_try_wait(at, parity)) && !*dead)
                if (clock64() - t0 > 400000000LL) {
                    *dead = 1;
                    report_status(p.status_dev, GDN_ERR_TIMEOUT);
                }
        }
        return there;
    };
    auto wait = [&](unsigned long long *bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_alone(bar, parity)) != 0; };   // by a whole warp

    // what has gone through the barriers before this unit: tiles, and tiles of the second stream; units
    uint32_t done = 0, done1 = 0, units = 0, units1 = 0;
    AttnWalk walk;
    walk.begin(p, cta, AS_M, AS_TN);
    auto next_unit = [&](Unit &t) {   // by all threads together
        for (;;) {
            if (!walk.next(p, cta, AS_M, AS_TN, t.g)) return false;
            __syncthreads();   // the unit before is through
            if (*dead) return false;
            if (p.row_offsets && kind == AT_WORDS64 && !attn_ancestors(p, t.g.s, sh.anc, sh.anc_up)) {
                if (tid == 0) report_status(p.status_dev, GDN_ERR_TREE);
                continue;
            }
            if (p.row_offsets && kind == AT_WORDS && !p.tree_ok[t.g.b]) continue;
            t.row_first = t.g.m_tile * AS_M;
            t.rows = min(AS_M, t.g.s.rows * p.group - t.row_first);
            const int last_node = (t.row_first + t.rows - 1) / p.group;
            t.upto = p.row_offsets ? t.g.s.len + last_node + 1 : t.g.s.len;
            t.tile1 = min(t.g.tile1, max((t.upto + AS_TN - 1) / AS_TN, t.g.tile0));
            t.n_tiles = t.tile1 - t.g.tile0;
            t.common = !p.row_offsets ? t.upto : kind == AT_CHAIN ? t.g.s.len + t.row_first / p.group + 1 : t.g.s.len;
            t.streams = t.rows > 128 ? 2 : 1;
            if (tid == 0) sh.odd = 0;
            __syncthreads();
            return true;
        }
    };
    auto end_unit = [&](const Unit &t) {
        done += t.n_tiles;
        if (t.n_tiles > 0) ++units;
        if (t.streams == 2) {
            done1 += t.n_tiles;
            if (t.n_tiles > 0) ++units1;
        }
    };

    if (warp < 8) {   // ---- a row per thread
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");   // (two groups of 216 and one of 72 are three of 168)
        const int stream = warp >> 2;
        const uint32_t s_at = tmem + ((uint32_t)((warp & 3) * 32) << 16) + stream * 256, o_at = s_at + 128;
        Unit t;
        while (next_unit(t)) {
            const AttnSegment &g = t.g;
            const int r = tid, u = t.row_first + r, node = u / p.group;
            const bool mine = r < t.rows;
            const size_t head = (size_t)(g.head * p.group + u % p.group);
            if (t.n_tiles > 0) {
                const __nv_bfloat16 *src = static_cast<const __nv_bfloat16 *>(p.q) + (mine ? (size_t)(g.s.row0 + node) * p.q_stride + head * D : 0);
#pragma unroll
                for (int c = 0; c < PIECES; ++c) cp_async_16(q_s + stream * TILE + as_at(r & 127, c), src + c * 8, mine);
                cp_async_wait_all();
                fence_proxy_async();
                mbar_arrive_warp(smem_u32(&sh.q_full), lane);
            }
            if (stream < t.streams) {
                const uint32_t seen_before = stream ? done1 : done;
                float m = -INFINITY, l = 0.f;   // m: of the raw scores, as the sums stand
                bool ok = true;
                for (int i = 0; i < t.n_tiles; ++i) {
                    const int tile = g.tile0 + i;
                    ok = wait(&sh.s_full[stream], (seen_before + i) & 1);
                    if (!ok) break;
                    tc_fence_after();
                    uint32_t x[128];
#pragma unroll
                    for (int c = 0; c < 4; ++c) GDN_TMEM_LD32(s_at + c * 32, (x + c * 32));
                    tmem_wait_ld();
                    bool hidden = (tile + 1) * AS_TN > t.common;   // from some row of this warp, some token
                    if (hidden) {
                        uint32_t see[4], all = ~0u;   // bit j: this row sees token tile * AS_TN + 32 c + j
#pragma unroll
                        for (int c = 0; c < 4; ++c) all &= see[c] = mine ? seen_word(p, kind, sh.anc, g.s, node, tile * AS_TN + c * 32) : ~0u;   // (no row: zeros, written nowhere)
                        hidden = __any_sync(0xffffffffu, all != ~0u);
                        if (hidden) {
#pragma unroll
                            for (int c = 0; c < 4; ++c)
#pragma unroll
                                for (int j = 0; j < 32; ++j)
                                    if (!(see[c] >> j & 1)) x[c * 32 + j] = 0xFF800000u;
                        }
                    }
                    float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int j = 0; j < 128; j += 8)
#pragma unroll
                        for (int k = 0; k < 4; ++k) t4[k] = max3_nan(t4[k], __uint_as_float(x[j + k]), __uint_as_float(x[j + 4 + k]));
                    const float top = max3_nan(max3_nan(t4[0], t4[1], t4[2]), t4[3], t4[3]);
                    // some score is +inf or no number, or all are -inf: the differences to the maximum may be no numbers, and stay that
                    const bool odd_scores = __any_sync(0xffffffffu, !(fabsf(top) < INFINITY));
                    const bool first = i == 0;
                    const bool raise = first || (top - m) * p.scale_log2 > AS_SLACK || (m == -INFINITY && top > -INFINITY);
                    float fade = 1.f;
                    if (raise) {
                        const float m_new = fmaxf(m, top);   // (of a number and none, the number)
                        fade = first || m == -INFINITY ? 0.f : power_of_two((m - m_new) * p.scale_log2);
                        m = m_new;
                        l *= fade;
                    }
                    if (!first && __any_sync(0xffffffffu, raise)) {
#pragma unroll 1
                        for (int c = 0; c < D / 16; ++c) {
                            uint32_t y[16];
                            GDN_TMEM_LD16(o_at + c * 16, y);
                            tmem_wait_ld();
#pragma unroll
                            for (int j = 0; j < 16; ++j) y[j] = __float_as_uint(__uint_as_float(y[j]) * fade);
                            GDN_TMEM_ST16(o_at + c * 16, y);
                        }
                    }
                    // (a hidden score of -inf gives 2^-inf = 0; scale > 0 keeps it -inf)
                    const float ref = m == -INFINITY ? 0.f : m * p.scale_log2;
                    const float2 scale2 = make_float2(p.scale_log2, p.scale_log2), ref2 = make_float2(-ref, -ref);
                    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t w[16];
                        auto weights = [&](auto by_products) {   // three of eight pairs go without the special function unit
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                float2 e = fma2(make_float2(__uint_as_float(x[c * 32 + 2 * j]), __uint_as_float(x[c * 32 + 2 * j + 1])), scale2, ref2);
                                if (decltype(by_products)::value && (j % 8 == 1 || j % 8 == 4 || j % 8 == 7)) e = power_of_two_by_products(e);
                                else e = make_float2(power_of_two(e.x), power_of_two(e.y));
                                sum[j & 1] = add2(sum[j & 1], e);
                                w[j] = pack_bf16(e.x, e.y);
                            }
                        };
                        if (hidden || odd_scores) weights(No{});
                        else weights(Yes{});
                        GDN_TMEM_ST16(s_at + c * 16, w);
                        if (c == 1 || c == 3) {   // half of the tile's weights: their part of the second product may begin
                            tmem_wait_st();
                            tc_fence_before();
                            mbar_arrive_warp(smem_u32(&sh.p_full[c >> 1][stream]), lane);
                        }
                    }
                    l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                }
                if (ok && t.n_tiles > 0) ok = wait(&sh.o_full[stream], (stream ? units1 : units) & 1);
                tc_fence_after();
                if (ok) {
                    const bool odd = sh.odd != 0;
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    __nv_bfloat16 *o = static_cast<__nv_bfloat16 *>(p.o) + ((size_t)(g.s.row0 + node) * p.h_q + head) * D;
                    const size_t part = (size_t)(g.slot < 0 ? 0 : g.slot) * AS_M;
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t x[32];
                        if (t.n_tiles > 0) {
                            GDN_TMEM_LD32(o_at + c * 32, x);
                            tmem_wait_ld();
                        } else {
#pragma unroll
                            for (int j = 0; j < 32; ++j) x[j] = 0;
                        }
                        if (odd && mine)
                            for (int j = t.common - g.s.len; j <= node; ++j) {
                                const int at_token = g.s.len + j;
                                if (at_token < g.tile0 * AS_TN || at_token >= t.tile1 * AS_TN || !attn_sees(p, kind, sh.anc, g.s.row0, node, j)) continue;
                                const long long at = attn_token_offset(p, g.b, at_token, t.upto);
                                if (at < 0) continue;
                                const __nv_bfloat16 *v = v_cache + at + g.head * p.head_stride + c * 32;
#pragma unroll
                                for (int e = 0; e < 32; ++e) {
                                    const float y = __bfloat162float(v[e]);
                                    if (!(fabsf(y) < INFINITY)) x[e] = __float_as_uint(__uint_as_float(x[e]) + y);
                                }
                            }
                        if (!mine) continue;
                        if (g.slot < 0) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                uint32_t w[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    w[k] = pack_bf16(__uint_as_float(x[8 * j + 2 * k]) * inv, __uint_as_float(x[8 * j + 2 * k + 1]) * inv);
                                *reinterpret_cast<uint4 *>(o + c * 32 + j * 8) = make_uint4(w[0], w[1], w[2], w[3]);
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j)   // [slot][D / 4][M][4]: a warp's rows lie side by side
                                *reinterpret_cast<uint4 *>(p.part_o + part * D + ((size_t)(c * 8 + j) * AS_M + r) * 4) =
                                    make_uint4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
                        }
                    }
                    if (mine && g.slot >= 0)
                        *reinterpret_cast<float2 *>(p.part_ml + (part + r) * 2) = make_float2(m == -INFINITY ? m : m * p.scale_log2, l);
                }
                tc_fence_before();
            }
            end_unit(t);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        Unit t;
        while (next_unit(t)) {
            const AttnSegment &g = t.g;
            // (by one warp) values of places that hold no token: zeros (their weights are 0, and 0 times what lies there may be no number);
            // of tokens that not every row sees: what is infinite or no number is taken out, and added at the end of the unit
            auto look_at_values = [&](int tile, uint32_t stage) {
                if ((tile + 1) * AS_TN <= t.common) return;
                for (int k = lane; k < AS_TN * PIECES; k += 32) {
                    const int row = k / PIECES, token = tile * AS_TN + row;
                    if (token < t.common) continue;
                    uint4 *at = reinterpret_cast<uint4 *>(data + (v_s - q_s) + stage * TILE + as_at(row, k % PIECES));
                    uint4 y = *at;
                    if (token >= t.upto) *at = make_uint4(0, 0, 0, 0);
                    else if (zero_odd(y)) {
                        *at = y;
                        sh.odd = 1;
                    }
                }
            };
            if (warp < 10) {   // ---- tiles, of keys or of values
                const bool keys = warp == 8;
                const uint32_t to = keys ? k_s : v_s, stages = keys ? K_STAGES : V_STAGES;
                unsigned long long *full = keys ? sh.k_full : sh.v_full, *empty = keys ? sh.k_empty : sh.v_empty;
                constexpr int ASKS = TMA ? 1 : 4;   // places that a lane looks up: of its box, or of four tokens
                const int box = TMA ? maps.box : 1;
                int page[ASKS];
                auto token_of = [&](int tile, int k) { return tile * AS_TN + (TMA ? lane * box : k * 32 + lane); };
                auto ask = [&](int tile) {
#pragma unroll
                    for (int k = 0; k < ASKS; ++k) {
                        const int token = token_of(tile, k);
                        page[k] = tile < t.tile1 && token < t.upto && (!TMA || lane * box < AS_TN)
                                      ? p.page_table[(size_t)g.b * p.max_pages + (p.page_shift >= 0 ? token >> p.page_shift : token / p.page_size)] : -1;
                    }
                };
                ask(g.tile0);
                for (int i = 0; i < t.n_tiles; ++i) {
                    const uint32_t n = done + i, stage = n % stages;
                    const int tile = g.tile0 + i;
                    bool good[ASKS];
                    int in_page[ASKS], at_page[ASKS];
#pragma unroll
                    for (int k = 0; k < ASKS; ++k) {
                        const int token = token_of(tile, k);
                        const bool wanted = token < t.upto && (!TMA || lane * box < AS_TN);
                        good[k] = wanted && page[k] >= 0 && page[k] < p.n_pages;
                        if (wanted && !good[k]) report_status(p.status_dev, GDN_ERR_PAGE);
                        at_page[k] = page[k];
                        in_page[k] = p.page_shift >= 0 ? token & (p.page_size - 1) : token % p.page_size;
                    }
                    ask(tile + 1);
                    if (n >= stages && !wait(&empty[stage], (n / stages - 1) & 1)) break;
                    if constexpr (TMA) {
                        const uint32_t bar = smem_u32(keys ? &sh.k_full[stage] : &sh.v_landed[stage]);
                        if (lane == 0) mbar_expect_tx(bar, TILE);
                        __syncwarp();
                        if (lane * box < AS_TN)   // (a page behind the last one reads as zeros)
#pragma unroll
                            for (int c = 0; c < D / 64; ++c)
                                tma_load_4d(to + stage * TILE + c * (AS_TN * 128) + lane * box * 128, keys ? &maps.k : &maps.v, c * 64, in_page[0], g.head,
                                            good[0] ? at_page[0] : p.n_pages, bar);
                    } else {
                        constexpr int ROWS = 32 / PIECES;   // rows that one access of the warp covers
                        const int col = lane % PIECES;
                        const __nv_bfloat16 *from_head = (keys ? k_cache : v_cache) + g.head * p.head_stride + col * 8;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const long long place = good[k] ? at_page[k] * p.page_stride + in_page[k] * p.token_stride : -1;
#pragma unroll 8
                            for (int h = 0; h < 32 / ROWS; ++h) {
                                const int in = h * ROWS + lane / PIECES;
                                const long long at = __shfl_sync(0xffffffffu, place, in);
                                cp_async_16(to + stage * TILE + as_at(k * 32 + in, col), from_head + (at < 0 ? 0 : at), at >= 0);
                            }
                        }
                        cp_async_wait_all();
                        __syncwarp();
                    }
                    if constexpr (!TMA) {
                        if (!keys) look_at_values(tile, stage);
                        fence_proxy_async();
                        mbar_arrive_warp(smem_u32(&full[stage]), lane);
                    }
                }
            } else if (TMA && warp == 11) {   // ---- values that have landed
                for (int i = 0; i < t.n_tiles; ++i) {
                    const uint32_t n = done + i, stage = n % V_STAGES;
                    if (!wait(&sh.v_landed[stage], (n / V_STAGES) & 1)) break;
                    look_at_values(g.tile0 + i, stage);
                    fence_proxy_async();
                    mbar_arrive_warp(smem_u32(&sh.v_full[stage]), lane);
                }
            } else if (warp == 10 && t.n_tiles > 0) {   // ---- products, by one thread: what it does between two of them the tensor cores may wait for
                if (elect_one()) {
                    constexpr uint32_t id_s = idesc_bf16(128, 128), id_o = idesc_bf16(128, D) | (1u << 16);
                    auto scores = [&](int s, uint32_t n) {
                        const uint64_t q_d = smem_desc_sw128(q_s + s * TILE), k_d = smem_desc_sw128(k_s + (n % K_STAGES) * TILE);
#pragma unroll
                        for (int k = 0; k < KS; ++k) {
                            const uint64_t on = ((k >> 2) * (AS_TN * 128) + (k & 3) * 32) >> 4;
                            umma_bf16(tmem + s * 256, q_d + on, k_d + on, id_s, k != 0);
                        }
                        umma_commit(smem_u32(&sh.s_full[s]));
                    };
                    bool ok = wait_alone(&sh.q_full, units & 1) && wait_alone(&sh.k_full[done % K_STAGES], (done / K_STAGES) & 1);
                    tc_fence_after();
                    if (ok) {
                        for (int s = 0; s < t.streams; ++s) scores(s, done);
                        umma_commit(smem_u32(&sh.k_empty[done % K_STAGES]));
                    }
                    for (int i = 0; i < t.n_tiles && ok; ++i) {
                        const uint32_t n = done + i, next = n + 1;
                        const uint32_t stage = n % V_STAGES;
                        const uint64_t v_d = desc_rows_along_k(v_s + stage * TILE);
                        const bool more = i + 1 < t.n_tiles;
                        ok = wait_alone(&sh.v_full[stage], (n / V_STAGES) & 1);
                        for (int s = 0; s < t.streams && ok; ++s) {
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                ok = ok && wait_alone(&sh.p_full[half][s], ((s ? done1 : done) + i) & 1);
                                if (!ok) break;
                                tc_fence_after();
#pragma unroll
                                for (int k = 0; k < AS_TN / 32; ++k) {
                                    const int at = half * (AS_TN / 32) + k;
                                    umma_bf16_ts_into(tmem + s * 256 + 128, tmem + s * 256 + at * 8, v_d + (at * 2048 >> 4), id_o, i > 0 || at > 0);
                                }
                            }
                            if (!ok) break;
                            if (!more) umma_commit(smem_u32(&sh.o_full[s]));
                            else {
                                if (s == 0) {
                                    ok = wait_alone(&sh.k_full[next % K_STAGES], (next / K_STAGES) & 1);
                                    tc_fence_after();
                                }
                                if (ok) scores(s, next);
                            }
                        }
                        if (ok) {
                            umma_commit(smem_u32(&sh.v_empty[stage]));
                            if (more) umma_commit(smem_u32(&sh.k_empty[next % K_STAGES]));
                        }
                    }
                }
                __syncwarp();
            }
            end_unit(t);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (*dead) {   // products and copies may still be on their way: a millisecond, far longer than what can be in their queues takes
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000) {}
        __syncthreads();
    }
    if (warp == 10) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

bool cache_map(CUtensorMap *tm, const void *cache, const AttnParams &p, int box)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)p.d, (cuuint64_t)p.page_size, (cuuint64_t)p.h_kv, (cuuint64_t)p.n_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)p.token_stride * 2, (cuuint64_t)p.head_stride * 2, (cuuint64_t)p.page_stride * 2};
    const cuuint32_t boxes[4] = {64, (cuuint32_t)box, 1, 1}, steps[4] = {1, 1, 1, 1};
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(cache), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

AttnTiling attn_sm100_tiling() { return {AS_M, AS_TN, 1, 4}; }

cudaError_t launch_attn_sm100(const AttnParams &p, int grid, cudaStream_t stream)
{
    static PerContext seen[4];
    using Kernel = void (*)(const AttnParams, const CacheMaps);
    static const Kernel kernels[4] = {attn_sm100_kernel<64, false>, attn_sm100_kernel<64, true>, attn_sm100_kernel<128, false>, attn_sm100_kernel<128, true>};
    CacheMaps maps{};
    // a box is the largest power of two of tokens that divides a page and a tile, so that none crosses a page's end; swizzled boxes begin
    // on 1024 bytes, so that one has eight rows or more; strides that a tensor map cannot have are the other kernel's
    maps.box = p.page_size & -p.page_size;
    if (maps.box > AS_TN) maps.box = AS_TN;
    const bool tma = maps.box >= 8 && cache_map(&maps.k, p.k_cache, p, maps.box) && cache_map(&maps.v, p.v_cache, p, maps.box);
    const int which = (p.d == 128 ? 2 : 0) + (tma ? 1 : 0);
    const size_t smem = p.d == 128 ? as_smem<128>() : as_smem<64>();
    int sms = 0;
    const cudaError_t e = device_sms(seen[which], reinterpret_cast<const void *>(kernels[which]), smem, &sms);
    if (e != cudaSuccess) return e;
    return launch_behind(kernels[which], dim3((unsigned)grid), AS_THREADS, smem, stream, p, maps);
}

}  // namespace gdn
