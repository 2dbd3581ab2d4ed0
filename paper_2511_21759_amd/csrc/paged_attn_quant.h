// Attention of new rows over pages of 8-bit codes (odb_paged_attention_quant): the kernels, for one kind of codes at a time.
//
// The work is laid out as for 16-bit pages (paged_attn.hip): a tile of query rows of one request and K/V head, S^T = K Q^T, then
// O^T = V^T P^T, with the keys split by the waves (few rows) or the rows (many).  What differs:
//
//   Codes become binary16 in registers, which holds every INT8 and E4M3 code, and go through binary16 MFMAs: one conversion of two
//         E4M3 codes, or a permutation of bytes and an addition of two halves for INT8 (1024 + code + 128 - 1152).
//   K:    score = (q . codes) * scale of the key: the scale multiplies a score, not the channels.
//   V:    O = sum of (p * scale of the key) codes: it multiplies a probability.  p * scale is rounded to binary16, so scales are
//         taken relative to a power of two beyond the largest that the row has seen (RowState), and O with them.
//   Sums of probabilities are those of p alone, rounded to binary16 like the operands.
#pragma once

#include "paged_attn_core.h"

namespace odb {

namespace {

template <int CODES> struct Code;
template <> struct Code<ODB_INT8> {
    static constexpr bool kOdd = false;                      // every code is a number
    static __device__ __forceinline__ uint2 halves(uint32_t w) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        const uint32_t u = w ^ 0x80808080u;
        const h2 off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
        uint2 r;
        r.x = __builtin_bit_cast(uint32_t, (h2)(__builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + off));
        r.y = __builtin_bit_cast(uint32_t, (h2)(__builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + off));
        return r;
    }
};
template <> struct Code<ODB_E4M3> {
    static constexpr bool kOdd = true;                       // 0x7f and 0xff are no numbers
    static __device__ __forceinline__ uint2 halves(uint32_t w) {
        return uint2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true))};
    }
};
template <int CODES>
__device__ __forceinline__ frag_t halves8(uint32_t a, uint32_t b) {
    const uint2 x = Code<CODES>::halves(a), y = Code<CODES>::halves(b);
    return frag_t{{x.x, x.y, y.x, y.y}};
}
// has one of 16 codes no value?
__device__ __forceinline__ int has_odd_code(const frag_t &v) {
    uint32_t odd = 0;
#pragma unroll
    for (int w = 0; w < 4; w++) odd |= ((v.w[w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    return odd != 0;
}

constexpr float kQuantBeyond = 1 << 27;          // scores times their scales are rounded before the reference is known: less room than kBeyond
__device__ __forceinline__ float checked_quant_sum(float at, float sum) { return fabsf(at) >= kQuantBeyond && at != kNone ? __builtin_bit_cast(float, -1) : sum; }

// Queries of a lane's row in operand order, binary16, and the factor of its scores.  bfloat16 has another range: the row is taken as
// multiples of 2^(e - 9), 2^e beyond its largest magnitude, which is 2^8 or more in them: its own eight bits are kept down to 2^-23 of 2^e, and
// below, half of binary16's smallest number, 2^-25, is within 2^-33 of the largest.
// PAIRS: the channels of two k-steps are those of 64 in the order in which a lane loads codes, sixteen at once.
template <int DH, bool PAIRS>
__device__ __forceinline__ void load_queries(const PagedAttn &a, const u16 *src, int g, frag_t (&q)[DH / 32], float &sc) {
#pragma unroll
    for (int k = 0; k < DH / 32; k++) q[k] = ld_frag(src + (PAIRS ? 64 * (k >> 1) + 16 * g + 8 * (k & 1) : 32 * k + 8 * g));
    sc = a.sc;
    if (a.pages.dtype != ODB_BF16) return;
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < DH / 32; k++)
#pragma unroll
        for (int w = 0; w < 4; w++) top = fmaxf(top, fmaxf(fabsf(bf2f((u16)q[k].w[w])), fabsf(bf2f((u16)(q[k].w[w] >> 16)))));
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const int e = __builtin_amdgcn_frexp_expf(fminf(fmaxf(top, 0x1p-100f), 0x1p126f));
#pragma unroll
    for (int k = 0; k < DH / 32; k++)
#pragma unroll
        for (int w = 0; w < 4; w++)
            q[k].w[w] = Num<_Float16>::pack(ldexpf(bf2f((u16)q[k].w[w]), 9 - e), ldexpf(bf2f((u16)(q[k].w[w] >> 16)), 9 - e));
    sc = fmaxf(ldexpf(sc, e - 9), 0x1p-126f);
}

__device__ __forceinline__ float most(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// What a row tile's rows carry through the keys, a row per lane and its four lanes the same: the reference of their probabilities (its limit in
// units of log2 here), and that of V's scales: a power of two, `unit`, that none of those a row has seen exceeds.  O is in multiples of it.
struct RowState { float at = kNone, limit = kNone, unit = 0.f, inverse = 1.f; };

// Scores z of keys that a row may not see are minus infinity.  What these are multiplied by, and V's scales, must not make more of them: where the
// lane's keys share a scale (EVEN) it is left out if the row sees none of them, else key by key.  A factor of nought becomes one beside it.
template <bool EVEN>
__device__ __forceinline__ void hide_scales(const f32x4 (&z)[2], float (&c)[2], f32x4 (&v)[2]) {
#pragma unroll
    for (int s = 0; s < 2; s++) {
        if (EVEN) {
            const bool any = !(fmaxf(fmaxf(z[s][0], z[s][1]), fmaxf(z[s][2], z[s][3])) == -INFINITY);
            c[s] = any ? __builtin_elementwise_maximum(c[s], 0x1p-126f) : 1.0f;
            v[s][0] = any ? v[s][0] : 0.f;
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++) v[s][e] = z[s][e] > -INFINITY ? v[s][e] : 0.f;
        }
    }
}

// Probabilities of 32 keys of a row tile from their scores z (keys that are not seen: -infinity): p as the operand that is summed, p times V's
// relative scales as that of the product.  c: what a score of the first and the second 16 keys is multiplied by; v: the keys' scales, of
// which with EVEN only the first of each 16 counts.  References are raised, and sums and O rescaled, as in probabilities().
template <int CT, bool EVEN>
__device__ __forceinline__ void quant_probabilities(const f32x4 (&z)[2], const float (&f2)[2], const f32x4 (&v)[2], RowState &st, f32x4 &lsum, f32x4 (&o)[CT],
                                                    frag_t &pf, frag_t &pv) {
    const float c0 = f2[0], c1 = f2[1];
    // (maxima that hand on a NaN, which the matrix cores' results need no instruction more for; a row with one is a NaN whatever its reference)
    float top = most(most(most(z[0][0], z[0][1]), most(z[0][2], z[0][3])) * c0, most(most(z[1][0], z[1][1]), most(z[1][2], z[1][3])) * c1);
    float top_v = most(v[0][0], v[1][0]);
    if (!EVEN)
#pragma unroll
        for (int e = 1; e < 4; e++) top_v = most(top_v, most(v[0][e], v[1][e]));
    if (__any((int)(top > st.limit) | (int)(top_v > st.unit))) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        top_v = fmaxf(top_v, __shfl_xor(top_v, 16));
        top_v = fmaxf(top_v, __shfl_xor(top_v, 32));
        // (only where the row's own scores ask for it: what other rows see does not move it)
        float up = top > st.limit ? fmaxf(st.at, top - kShift) : st.at, over = -INFINITY;
#pragma unroll
        for (int e = 0; e < 4; e++) over = fmaxf(over, fmaxf(__builtin_fmaf(z[0][e], c0, -up), __builtin_fmaf(z[1][e], c1, -up)));
        over = fmaxf(over, __shfl_xor(over, 16));
        over = fmaxf(over, __shfl_xor(over, 32));
        up += over > kRaise ? fabsf(up) * 0x1.8p-24f : 0.f;
        float f = __builtin_amdgcn_exp2f(st.at - up);
        lsum *= f;
        if (top_v > st.unit) {
            // (some room above: scales differ.  From 2^-124 to 2^127, so that the unit and its inverse are both numbers for subnormal scales too: an
            // inverse of infinity times the unit of nought that a row begins with would be no number)
            const int e = __builtin_amdgcn_frexp_expf(fminf(fmaxf(top_v, 0x1p-126f), 0x1p125f)) + 1;
            st.inverse = ldexpf(1.0f, -e);
            f *= st.unit * st.inverse;
            st.unit = ldexpf(1.0f, e);
        }
#pragma unroll
        for (int c = 0; c < CT; c++) o[c] *= f;
        st.at = up;
        st.limit = up + kRaise;
        st.limit -= up == kNone ? 0.f : fabsf(up) * 0x1p-22f;                  // (roundings of the limit and of the scores that are compared with it)
    }
    float p[2][4], w[2][4];
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            p[s][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[s][e], s ? c1 : c0, -st.at));
            w[s][e] = p[s][e] * (v[s][EVEN ? 0 : e] * st.inverse);
        }
    pf = frag_t{{Num<_Float16>::pack(p[0][0], p[0][1]), Num<_Float16>::pack(p[0][2], p[0][3]), Num<_Float16>::pack(p[1][0], p[1][1]), Num<_Float16>::pack(p[1][2], p[1][3])}};
    pv = frag_t{{Num<_Float16>::pack(w[0][0], w[0][1]), Num<_Float16>::pack(w[0][2], w[0][3]), Num<_Float16>::pack(w[1][0], w[1][1]), Num<_Float16>::pack(w[1][2], w[1][3])}};
}

__device__ __forceinline__ float ld_scalar_float(const float *p, long long i) {
    typedef const __attribute__((address_space(4))) float *ptr;
    return ((ptr)(uintptr_t)p)[i];
}

__device__ __forceinline__ void store_rounded8(const PagedAttn &a, int row, int head, int dim, int c, const float *x, float f) {
    uint4 v;
    if (a.pages.dtype == ODB_F16) {
        v.x = Num<_Float16>::pack(x[0] * f, x[1] * f); v.y = Num<_Float16>::pack(x[2] * f, x[3] * f);
        v.z = Num<_Float16>::pack(x[4] * f, x[5] * f); v.w = Num<_Float16>::pack(x[6] * f, x[7] * f);
    } else {
        v.x = Num<__bf16>::pack(x[0] * f, x[1] * f); v.y = Num<__bf16>::pack(x[2] * f, x[3] * f);
        v.z = Num<__bf16>::pack(x[4] * f, x[5] * f); v.w = Num<__bf16>::pack(x[6] * f, x[7] * f);
    }
    store_out8(a, row, head, dim, c, v);
}

// ---- few rows: the waves of a workgroup split the keys -----------------------------------------------------------------

// As paged_attn_kernel, with blocks of 32 keys.  V's codes lie in LDS as they come and are transposed as they are read (eight keys of a channel
// per lane).  EVEN: the 16 keys of a tile share their scales, which are then scalars of the wave; else every key has its own.
// Bound by HBM with single tokens (two of 1.9e5 positions, 799 MB, 125 us = 6.4 TB/s; 48 of 24 to 13524, 379 MB, 67 us = 5.7), by the latency of a
// block's loads where pairs are few: about 1.1 us a turn of a wave (one token of 800 / 2000 positions 12.5 / 21.8 us whole), 1.7 with 32 rows.
// Blocks of 64 keys, which have as many bytes on their way as 16-bit pages, need 194 registers and were slower nearly everywhere (48 tokens 84 / 86 us, but
// 32 of 1000 positions 19.3 / 15.9, 10 x 32 rows 52 / 35).
// COST: places in the list for a pair beside its blocks; they pass at twice the rate of 16-bit ones (48 tokens: 86 us with 6, 84 with 12, 86 with 20).
template <int DH>
struct QuantShape {
    static constexpr int SHIFT = 5, COST = 12;
};
constexpr int kLeastQuantPiece = 12;             // places

// Where the 16-byte piece c of a key lies in a wave's codes of V: the reads of 16 neighbouring lanes' keys fall on different banks.
template <int DH>
__device__ __forceinline__ constexpr int vq_piece(int key, int c) {
    constexpr int P = DH / 16;
    const int turn = DH == 64 ? ((key >> 2) & 1) | ((key >> 3) & 2) : DH == 128 ? ((key >> 1) & 3) | ((key >> 2) & 4) : (key & 7) | ((key >> 1) & 8);
    return key * P + (c ^ turn);
}

template <int CODES, int DH, int NT, bool EVEN>
__global__ __launch_bounds__(64 * NW, DH == 256 || NT == 4 ? 1 : 2) void quant_attn_kernel(PagedAttnQuant a) {
    typedef QuantShape<DH> Shape;
    constexpr int KB = 32, SHIFT = Shape::SHIFT, T = 2;          // keys and 16-key tiles of a block
    constexpr int CH = DH / 64, KS = DH / 32, CT = DH / 16;      // loads of a tile of K or V per lane, k-steps of S, channel tiles of O
    constexpr int KEYS = 1024 / DH;                              // keys per load of V
    constexpr int OSTRIDE = DH + 4, WAVE_LDS = 16 * OSTRIDE * 4;
    constexpr int TILE_ROWS = NT * 16;
    static_assert(KB * DH <= WAVE_LDS && KEYS * CH == 16, "V block");
    __shared__ __align__(16) unsigned char lds[NW * WAVE_LDS];
    __shared__ float2 stat[NW][TILE_ROWS];

    const int kv = a.pages.n_kv_heads, head = (int)(blockIdx.x % (unsigned)kv), x = (int)(blockIdx.x / (unsigned)kv);
    const bool split = a.split > 0;
    auto piece_of = [&](long long total) { return max((long long)kLeastQuantPiece, (total + a.split - 1) / max(a.split, 1)); };
    Place pl;
    if (!find_place<SHIFT, Shape::COST, true>(a, TILE_ROWS, split, [&](long long total) { return split ? piece_of(total) * x : (long long)x; }, pl)) return;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, li = lane & 15;
    const int G = a.group;
    const unsigned char *kp = (const unsigned char *)a.pages.k + (size_t)head * a.pages.head_stride, *vp = (const unsigned char *)a.pages.v + (size_t)head * a.pages.head_stride;
    const float *ksp = a.scales.k + (size_t)head * a.scales.head_stride, *vsp = a.scales.v + (size_t)head * a.scales.head_stride;
    const int page_mask = (1 << a.page_shift) - 1;
    const size_t pos_stride = a.pages.pos_stride, page_stride = a.pages.page_stride, scale_page = a.scales.page_stride;
    const int v_key = lane / (DH / 16), v_ch = lane % (DH / 16);
    const unsigned k_off = li * (unsigned)pos_stride + 16 * g, v_off = v_key * (unsigned)pos_stride + v_ch * 16;    // bytes
    unsigned char *mine = lds + wave * WAVE_LDS;
    const frag_t ones = {{Num<_Float16>::kOnes, Num<_Float16>::kOnes, Num<_Float16>::kOnes, Num<_Float16>::kOnes}};
    Request rq = pl.q;
    int request = pl.r, tiles = tiles_of(a, rq, TILE_ROWS), nb = split ? request_blocks<SHIFT>(a, rq) : 1;
    const int cost = split ? Shape::COST : 0;
    int tile = __builtin_amdgcn_readfirstlane((int)(pl.at / (nb + cost))), at = __builtin_amdgcn_readfirstlane((int)(pl.at - (long long)tile * (nb + cost)));
    const long long piece = piece_of(pl.total);
    long long left = split ? min(piece, pl.total - piece * x) : 1;
    if (!split) tile = tiles - 1 - tile;                          // the last rows of a causal request see the most: first

    for (;;) {
        const int end = split ? (int)min((long long)nb + cost, at + left) : 1;
        const int b_lo = max(0, at - cost), b_end = max(0, end - cost);
        if (b_end > b_lo) {
            const int n_rows = rq.m * G, rho0 = tile * TILE_ROWS;
            int ql = lane;
            asm volatile("" : "+v"(ql));
            int pmin, pmax;
            tile_span(rq, G, tile, TILE_ROWS, pmin, pmax);
            const Blocks bl = split ? blocks_of<SHIFT>(a, rq.len, rq.first, rq.first + rq.m - 1) : blocks_of<SHIFT>(a, rq.len, pmin, pmax);
            const int b_hi = split ? min(b_end, bl.count) : bl.count;
            const bool whole = b_lo == 0 && b_end == nb;

            frag_t q[NT][KS];
            float sc[NT];
            Sight sight[NT];                                          // of the lane's row of each tile
#pragma unroll
            for (int t = 0; t < NT; t++) {
                const int rho = min(rho0 + t * 16 + (ql & 15), n_rows - 1), i = rho / G, hq = head * G + (rho - i * G);
                sight[t] = sight_of(a, rq.len, rq.first + i);
                load_queries<DH, true>(a, (const u16 *)a.q + (size_t)(rq.row0 + i) * a.q_row + (size_t)hq * DH, ql >> 4, q[t], sc[t]);
            }

            f32x4 o[NT][CT], lsum[NT];
            RowState st[NT];
#pragma unroll
            for (int t = 0; t < NT; t++) {
                lsum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < CT; c++) o[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
            }

            // page of each 16-key tile of a block: -1 where no key of the tile is visible or the table names no page of the pool
            const int32_t *table = a.tables + (size_t)request * a.columns;
            auto page_of = [&](int key) -> int {
                const int id = key < rq.len ? ld_scalar(table, key >> a.page_shift) : -1;
                return id >= 0 && id < a.pages.n_pages ? id : -1;
            };
            frag_t kr[T][CH], vr[T][CH];
            f32x4 ks[T], vs[T];                                       // (EVEN: one number each, in all four)
            float nks[T], nvs[T];
            auto tile_base = [&](int page, int key) -> size_t { return (size_t)max(page, 0) * page_stride + (size_t)(key & page_mask) * pos_stride; };
            auto scale_base = [&](int page, int key) -> size_t { return (size_t)max(page, 0) * scale_page + (size_t)((key & page_mask) >> a.scales.group_shift); };
            auto load_k = [&](const size_t (&base)[T], unsigned off) {
#pragma unroll
                for (int t = 0; t < T; t++)
#pragma unroll
                    for (int c = 0; c < CH; c++) kr[t][c] = ld_at<NT == 1>((const u16 *)(kp + base[t] + 64 * c), off);
            };
            auto load_v = [&](const size_t (&base)[T], unsigned off) {
#pragma unroll
                for (int t = 0; t < T; t++)
#pragma unroll
                    for (int j = 0; j < CH; j++) vr[t][j] = ld_at<NT == 1>((const u16 *)(vp + base[t] + (size_t)(j * KEYS) * pos_stride), off);
            };
            // scales of the lane's keys, 4 g .. 4 g + 3 of each tile
            auto load_scales = [&](const float *p, const size_t (&base)[T], f32x4 (&s)[T], bool there) {
#pragma unroll
                for (int t = 0; t < T; t++) s[t] = __builtin_bit_cast(f32x4, ld_at<false>((const u16 *)(p + base[t]), there ? 16u * (unsigned)g : 0u));
            };

            int b = b_lo + wave;
            if (b < b_hi) {
                int key0 = block_key<SHIFT>(bl, b), pg[T], nkey = 0, npg[T];
                size_t base[T], sbase[T];
#pragma unroll
                for (int t = 0; t < T; t++) {
                    pg[t] = page_of(key0 + 16 * t);
                    npg[t] = -1;
                    base[t] = tile_base(pg[t], key0 + 16 * t);
                    sbase[t] = scale_base(pg[t], key0 + 16 * t);
                }
                load_k(base, k_off);
                if (!EVEN) load_scales(ksp, sbase, ks, true);
                __builtin_amdgcn_sched_barrier(0);                    // K first here too, or the loop's first wait would be for both
                load_v(base, v_off);
                if (!EVEN) load_scales(vsp, sbase, vs, true);
                if (EVEN)
#pragma unroll
                    for (int t = 0; t < T; t++) { nks[t] = ld_scalar_float(ksp, sbase[t]); nvs[t] = ld_scalar_float(vsp, sbase[t]); }
                if (b + NW < b_hi) {
                    nkey = block_key<SHIFT>(bl, b + NW);
#pragma unroll
                    for (int t = 0; t < T; t++) npg[t] = page_of(nkey + 16 * t);
                }
                for (; b < b_hi; b += NW) {
                    const bool more = b + NW < b_hi;
                    const unsigned k_next = more ? k_off : 0, v_next = more ? v_off : 0;
                    float cks[T], cvs[T];
                    bool plain = all_seen(a, rq.len, key0, KB, pmin, pmax);
#pragma unroll
                    for (int t = 0; t < T; t++) {
                        base[t] = tile_base(npg[t], nkey + 16 * t);
                        sbase[t] = scale_base(npg[t], nkey + 16 * t);
                        plain = plain && pg[t] >= 0;
                        if (EVEN) {
                            cks[t] = nks[t];
                            cvs[t] = nvs[t];
                            nks[t] = ld_scalar_float(ksp, sbase[t]);
                            nvs[t] = ld_scalar_float(vsp, sbase[t]);
                        }
                    }
                    // scores of all keys and row tiles first, which frees the registers of K for the next block
                    f32x4 z[NT][2];
#pragma unroll
                    for (int tile = 0; tile < T; tile++) {
                        frag_t kf[KS];
#pragma unroll
                        for (int c = 0; c < CH; c++) {
                            kf[2 * c] = halves8<CODES>(kr[tile][c].w[0], kr[tile][c].w[1]);
                            kf[2 * c + 1] = halves8<CODES>(kr[tile][c].w[2], kr[tile][c].w[3]);
                        }
#pragma unroll
                        for (int t = 0; t < NT; t++) {
                            f32x4 y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int k = 0; k < KS; k++) y = mfma16(kf[k], q[t][k], y);
                            if (!EVEN) y *= ks[tile];
                            z[t][tile] = y;
                        }
                    }
                    load_k(base, k_next);
                    if (!EVEN) load_scales(ksp, sbase, ks, more);
                    bool dirty = false;
                    if (Code<CODES>::kOdd && !plain) {
                        int odd = 0;
#pragma unroll
                        for (int t = 0; t < T; t++)
#pragma unroll
                            for (int j = 0; j < CH; j++) {
                                if (!((int)(key0 + 16 * t + j * KEYS + v_key < rq.len) & (int)(pg[t] >= 0))) vr[t][j] = frag_t{{0, 0, 0, 0}};
                                odd |= has_odd_code(vr[t][j]);
                            }
                        dirty = __any(odd);
                    }
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                    for (int t = 0; t < T; t++)
#pragma unroll
                        for (int j = 0; j < CH; j++) *reinterpret_cast<frag_t *>(mine + 16 * vq_piece<DH>(16 * t + j * KEYS + v_key, v_ch)) = vr[t][j];
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    load_v(base, v_next);
                    if (Code<CODES>::kOdd && __builtin_expect(dirty, 0)) {
                        // a code that is no number makes the rows that see it no numbers, and has a zero in its place for the others
                        int dl = lane;
                        asm volatile("" : "+v"(dl));
                        for (int key = 0; key < KB; key++) {
                            const int page = key & 16 ? pg[1] : pg[0];
#pragma unroll
                            for (int t = 0; t < NT; t++) {
                                const bool seen = sees(sight[t], key0 + key, page);
#pragma unroll
                                for (int c = 0; c < CT; c++)
#pragma unroll
                                    for (int d = 0; d < 4; d++) {
                                        const unsigned char w = mine[16 * vq_piece<DH>(key, c) + 4 * (dl >> 4) + d];
                                        if ((int)seen & (int)((w & 0x7f) == 0x7f)) o[t][c][d] = __builtin_nanf("");
                                    }
                            }
                        }
                        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                        for (int j = 0; j < KB * DH / 1024; j++) {
                            frag_t *at = reinterpret_cast<frag_t *>(mine + 16 * (dl + 64 * j)), v = *at;
#pragma unroll
                            for (int w = 0; w < 4; w++) {
                                const uint32_t odd = ((v.w[w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;      // the highest bit of such codes
                                v.w[w] &= ~((odd >> 7) * 0xffu);
                            }
                            *at = v;
                        }
                        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    }

                    f32x4 v[2];
#pragma unroll
                    for (int s = 0; s < 2; s++) v[s] = EVEN ? f32x4{cvs[s], 0.f, 0.f, 0.f} : vs[s];
                    auto v_codes = [&](int c) {
                        typedef int i32x2 __attribute__((ext_vector_type(2)));
                        typedef __attribute__((address_space(3))) i32x2 *lds_ptr;
                        const int r = li >> 1, key = (r & 3) + 4 * g + 4 * (r & 4);
                        const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_ptr)(mine + 16 * vq_piece<DH>(key, c) + 8 * (li & 1)));
                        return halves8<CODES>((uint32_t)w[0], (uint32_t)w[1]);
                    };
                    frag_t vt[NT > 1 ? CT : 1];                           // held for several row tiles
                    if (NT > 1)
#pragma unroll
                        for (int c = 0; c < CT; c++) vt[NT > 1 ? c : 0] = v_codes(c);
#pragma unroll
                    for (int t = 0; t < NT; t++) {
                        f32x4 (&zt)[2] = z[t];
                        frag_t pf, pv;
                        float c[2] = {EVEN ? sc[t] * cks[0] : sc[t], EVEN ? sc[t] * cks[1] : sc[t]};
                        f32x4 vt2[2] = {v[0], v[1]};
                        if (!plain) {
                            hide_unseen(zt, sight[t], key0, g, pg[0], pg[1]);
                            hide_scales<EVEN>(zt, c, vt2);
                        }
                        quant_probabilities<CT, EVEN>(zt, c, vt2, st[t], lsum[t], o[t], pf, pv);
                        lsum[t] = mfma16(ones, pf, lsum[t]);
#pragma unroll
                        for (int c = 0; c < CT; c++) o[t][c] = mfma16(NT > 1 ? vt[NT > 1 ? c : 0] : v_codes(c), pv, o[t][c]);
                    }
                    if (!EVEN) load_scales(vsp, sbase, vs, more);
                    key0 = nkey;
#pragma unroll
                    for (int t = 0; t < T; t++) pg[t] = npg[t];
                    if (b + 2 * NW < b_hi) {
                        nkey = block_key<SHIFT>(bl, b + 2 * NW);
#pragma unroll
                        for (int t = 0; t < T; t++) npg[t] = page_of(nkey + 16 * t);
                    }
                }
            }

            // ---- the waves' sums become one
            int tid = threadIdx.x;
            asm volatile("" : "+v"(tid));
            const int eg = (tid >> 4) & 3, el = tid & 15;
#pragma unroll
            for (int t = 0; t < NT; t++)
                if (eg == 0) stat[wave][t * 16 + el] = float2{st[t].at, lsum[t][0]};
            const long long place = (2ll * x + (b_lo == 0)) * kv + head;
            const int parts = whole ? 1 : (int)((piece * x + (min(piece, pl.total - piece * x) - left) - at + cost + nb - 1) / piece) - x + 1;
#pragma unroll
            for (int t = 0; t < NT; t++) {
                __syncthreads();
                {
                    float top = kNone;
#pragma unroll
                    for (int w = 0; w < NW; w++) top = fmaxf(top, stat[w][t * 16 + el].x);
                    const float f = __builtin_amdgcn_exp2f(st[t].at - top) * st[t].unit;
                    float *dst = reinterpret_cast<float *>(mine) + el * OSTRIDE + 4 * eg;
#pragma unroll
                    for (int c = 0; c < CT; c++) *reinterpret_cast<f32x4 *>(dst + c * 16) = o[t][c] * f;
                }
                __syncthreads();
                for (int e = tid; e < 2 * DH; e += 64 * NW) {
                    const int r = e / (DH / 8), c = (e % (DH / 8)) * 8, rho = rho0 + t * 16 + r;
                    if (rho >= n_rows) continue;
                    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, top = -INFINITY, l = 0.f;
#pragma unroll
                    for (int w = 0; w < NW; w++) top = fmaxf(top, stat[w][t * 16 + r].x);
#pragma unroll
                    for (int w = 0; w < NW; w++) {
                        const float2 s = stat[w][t * 16 + r];
                        l += s.y * __builtin_amdgcn_exp2f(s.x - top);
                        const float *src = reinterpret_cast<const float *>(lds + w * WAVE_LDS) + r * OSTRIDE + c;
                        const f32x4 u = *reinterpret_cast<const f32x4 *>(src), y = *reinterpret_cast<const f32x4 *>(src + 4);
#pragma unroll
                        for (int i = 0; i < 4; i++) { sum[i] += u[i]; sum[4 + i] += y[i]; }
                    }
                    l = checked_quant_sum(top, l);
                    const int i = rho / G, hq = head * G + (rho - i * G), row = rq.row0 + i;
                    if (!whole) {
                        float *dst = a.partial + ((size_t)place * TILE_ROWS + t * 16 + r) * DH + c;
                        *reinterpret_cast<f32x4 *>(dst) = f32x4{sum[0], sum[1], sum[2], sum[3]};
                        *reinterpret_cast<f32x4 *>(dst + 4) = f32x4{sum[4], sum[5], sum[6], sum[7]};
                        if (c == 0) {
                            a.ml[place * TILE_ROWS + t * 16 + r] = float2{top, l};
                            if (b_lo == 0) a.where[(size_t)row * a.heads + hq] = int2{x, parts * kRowsPlace + t * 16 + r};
                        }
                    } else {
                        // a row that sees nothing is zero
                        store_rounded8(a, row, hq, DH, c, sum, l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l);
                        if (split && c == 0) a.where[(size_t)row * a.heads + hq] = int2{x, 0};
                    }
                }
            }
            __syncthreads();
        }
        if (!split) return;
        left -= end - at;
        if (left <= 0) return;
        at = 0;
        if (++tile == tiles) {
            do {
                if (++request >= a.n) return;
                rq = request_of(a, request);
                tiles = tiles_of(a, rq, TILE_ROWS);
            } while (tiles == 0);
            tile = 0;
            nb = request_blocks<SHIFT>(a, rq);
        }
    }
}

// ---- many rows: the waves of a workgroup split the rows and share K and V in LDS ----------------------------------------

constexpr int kMostShares = 16;          // parts of a tile that is cut

// As paged_rows_kernel; codes become binary16 on their way to LDS, once for the four waves, and the keys' scales lie beside them.  A lane converts sixteen
// codes to two pieces beside each other and stores every second piece at once, which the swizzle is made for (PAIRS in k_piece and v_piece).
// Bound by vector and matrix instructions together: 74 of the one and 17 of the other for a row tile and 32 keys, 38 more than with 16-bit pages:
// 8 products and 4 conversions for p times V's scale, 8 conversions of codes, what the two references ask for.  Four requests of 4096 rows at 8192 positions, 32
// heads over 8 of 128: 2.63 ms with E4M3 codes and scales of 64 positions (836 TFLOP/s), 2.79 with INT8 codes and a scale a position (788), 16-bit pages 2.30.
template <int CODES, int DH, bool EVEN>
__global__ __launch_bounds__(256, 2) void quant_rows_kernel(PagedAttnQuant a) {
    typedef RowsShape<DH> Shape;
    constexpr int NT = Shape::NT, SK = Shape::SK, SHIFT = Shape::SHIFT, KS = DH / 32, CT = DH / 16;
    constexpr int WK = SK / 4, KEYS = 1024 / DH, LD = WK / KEYS;             // keys that a wave stages; per load; loads each of K and V
    constexpr int BUF = 2 * SK * DH * 2;                                    // bytes of a stage
    static_assert(LD >= 1 && LD * KEYS == WK, "stage");
    extern __shared__ __align__(1024) unsigned char stages[];
    __shared__ __align__(16) float scales[2][2][SK];                          // [buffer][K, V][key]
    __shared__ __align__(4) unsigned char flags[2][4];                        // of a wave's part of a stage: 1 odd values, 2 in no page

    const int kv = a.pages.n_kv_heads, head = (int)(blockIdx.x % (unsigned)kv), x = (int)(blockIdx.x / (unsigned)kv);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, li = lane & 15;
    const bool tail = a.slots > 0, split = a.split > 0 && !tail;
    const int cost = split ? kTileCost : 0;
    Request rq;
    int request, tiles, tile, at, left, piece = 1, total = 0;
    int share = 0, shares = 1, cut = 0;                                          // tail: this workgroup's part of a tile, of how many, its number among the cut ones
    if (split) {
        const int32_t *plan = reinterpret_cast<const int32_t *>(a.plan);
        request = ld_scalar(plan, 4 * x);
        if (request < 0) return;
        tile = ld_scalar(plan, 4 * x + 1);
        at = ld_scalar(plan, 4 * x + 2);
        piece = ld_scalar(plan, 4 * a.split);
        total = ld_scalar(plan, 4 * a.split + 1);
        left = min(piece, total - piece * x);
        rq = request_of(a, request);
        tiles = tiles_of(a, rq, Shape::TILE_ROWS);
    } else {
        Place pl;
        auto pick = [&](long long all) -> long long {
            if (!tail) return x;
            const int over = (int)(all % a.slots), full = (int)(all - over);
            if (x < full) return x;
            shares = over ? min(kMostShares, a.slots / over) : 1;
            cut = x - full;
            share = cut % shares;
            return cut < over * shares ? full + cut / shares : all;
        };
        if (!find_place<5, -1, true>(a, Shape::TILE_ROWS, tail, pick, pl)) return;
        request = pl.r;
        rq = pl.q;
        tiles = tiles_of(a, rq, Shape::TILE_ROWS);
        tile = tiles - 1 - __builtin_amdgcn_readfirstlane((int)pl.at);      // those that see the most first
        at = 0;
        left = 1;
    }
    const int G = a.group;
    const frag_t ones = {{Num<_Float16>::kOnes, Num<_Float16>::kOnes, Num<_Float16>::kOnes, Num<_Float16>::kOnes}};

    const unsigned char *kp = (const unsigned char *)a.pages.k + (size_t)head * a.pages.head_stride, *vp = (const unsigned char *)a.pages.v + (size_t)head * a.pages.head_stride;
    const float *ksp = a.scales.k + (size_t)head * a.scales.head_stride, *vsp = a.scales.v + (size_t)head * a.scales.head_stride;
    const int page_mask = (1 << a.page_shift) - 1;
    const size_t pos_stride = a.pages.pos_stride, page_stride = a.pages.page_stride;
    const int s_key = lane / (DH / 16), s_ch = lane % (DH / 16);
    const unsigned s_off = s_key * (unsigned)pos_stride + s_ch * 16, s_step = KEYS * (unsigned)pos_stride;      // bytes
    typedef __attribute__((address_space(3))) unsigned char *lds_bytes;
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_bytes)stages;
    auto lds_frag = [](unsigned at, int more) { return (frag_t *)((lds_bytes)(uintptr_t)at + more); };
    auto put = [](unsigned at, int more, const frag_t &f) {                     // (as one store of 16 bytes)
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        *(__attribute__((address_space(3))) u32x4 *)((lds_bytes)(uintptr_t)at + more) = __builtin_bit_cast(u32x4, f);
    };
    const unsigned k_put = lds0 + 16 * k_piece<DH, true>(WK * wave + s_key, 2 * s_ch), v_put = lds0 + SK * DH * 2 + 16 * v_piece<DH, true>(WK * wave + s_key, 2 * s_ch);
    const unsigned k_get = lds0 + 16 * k_piece<DH, true>(li, g), v_get = lds0 + SK * DH * 2 + v_lane<DH, true>(lane, 0);
    for (;;) {
        const int n_rows = rq.m * G, rho0 = (tile * 4 + wave) * 16 * NT;
        int pmin, pmax, wmin, wmax;                                             // positions of the tile's rows and of this wave's
        tile_span(rq, G, tile, Shape::TILE_ROWS, pmin, pmax);
        tile_span(rq, G, tile * 4 + wave, 16 * NT, wmin, wmax);
        const Blocks bl = blocks_of<SHIFT>(a, rq.len, pmin, pmax);
        const int nb = max(1, bl.count);
        if (tail) {
            shares = min(shares, max(1, nb / kLeastStages));
            if (share >= shares) return;
            at = (int)((long long)share * nb / shares);
        }
        const int end = split ? min(nb + cost, at + left) : tail ? (int)((long long)(share + 1) * nb / shares) : nb;
        const int b_lo = max(0, at - cost), b_hi = min(bl.count, end - cost);
        if (end - cost > b_lo) {
            const bool whole = b_lo == 0 && end - cost == nb;
            const bool idle = rho0 >= n_rows;                                       // (a wave without rows helps to load)
            const int32_t *table = a.tables + (size_t)request * a.columns;
            frag_t q[NT][KS];
            float sc[NT];
            Sight sight[NT];
#pragma unroll
            for (int t = 0; t < NT; t++) {
                const int rho = min(rho0 + t * 16 + li, n_rows - 1), i = rho / G, hq = head * G + (rho - i * G);
                sight[t] = sight_of(a, rq.len, rq.first + i);
                load_queries<DH, false>(a, (const u16 *)a.q + (size_t)(rq.row0 + i) * a.q_row + (size_t)hq * DH, g, q[t], sc[t]);
            }
            f32x4 o[NT][CT], lsum[NT];
            RowState st[NT];
#pragma unroll
            for (int t = 0; t < NT; t++) {
                lsum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < CT; c++) o[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            // Page and place in it of the keys that this wave stages, of 64 stages from `base` on, a stage per lane; page -1: in no page
            int places, inside;
            auto find_places = [&](int base) {
                const int b = base + lane, key = block_key<SHIFT>(bl, b) + WK * wave;
                int id = -1;
                if (b < b_hi && key < rq.len) id = table[key >> a.page_shift];
                places = id >= 0 && id < a.pages.n_pages ? id : -1;
                inside = key & page_mask;
                asm volatile("" : "+v"(places), "+v"(inside));                  // (the wait for the table is here, not in every stage)
            };
            frag_t kr[LD], vr[LD];
            float scale = 0.f;                                                  // of K for the first half of the lanes, of V for the others
            auto load = [&](int b) -> bool {
                const int i = (b - b_lo) & 63, page = __builtin_amdgcn_readlane(places, i), in = __builtin_amdgcn_readlane(inside, i);
                const size_t at = (size_t)max(page, 0) * page_stride + (page < 0 ? 0 : (size_t)in * pos_stride);
                const rsrc_t k_src = rsrc_of((const u16 *)(kp + at)), v_src = rsrc_of((const u16 *)(vp + at));
#pragma unroll
                for (int j = 0; j < LD; j++) kr[j] = ld_buffer(k_src, s_off, j * s_step);
#pragma unroll
                for (int j = 0; j < LD; j++) vr[j] = ld_buffer(v_src, s_off, j * s_step);
                if (lane < 2 * WK) {
                    const int key = (page < 0 ? 0 : in) + (lane & (WK - 1));
                    scale = (lane < WK ? ksp : vsp)[(size_t)max(page, 0) * a.scales.page_stride + (key >> a.scales.group_shift)];
                }
                return page >= 0;
            };
            auto store = [&](int buf, int key0, bool there, bool plain) {
                unsigned k_at = k_put + buf * BUF, v_at = v_put + buf * BUF;
                asm volatile("" : "+v"(k_at), "+v"(v_at));
                int odd = 0;
                const bool look = Code<CODES>::kOdd && (!plain || !there);
#pragma unroll
                for (int j = 0; j < LD; j++) {
                    if (look) {
                        if (!((int)(key0 + WK * wave + s_key + j * KEYS < rq.len) & (int)there)) vr[j] = frag_t{{0, 0, 0, 0}};
                        odd |= has_odd_code(vr[j]);
                    }
                    constexpr int P = KEYS * DH / 8;                            // (pieces of the keys of a load; sixteen codes become two pieces)
                    const int k_turn = 16 * (k_piece<DH, true>(j * KEYS, 0) - j * P), v_turn = 16 * (v_piece<DH, true>(j * KEYS, 0) - j * P);
                    put(k_at ^ k_turn, 16 * j * P, halves8<CODES>(kr[j].w[0], kr[j].w[1]));
                    put(k_at ^ (k_turn ^ 16), 16 * j * P, halves8<CODES>(kr[j].w[2], kr[j].w[3]));
                    put(v_at ^ v_turn, 16 * j * P, halves8<CODES>(vr[j].w[0], vr[j].w[1]));
                    put(v_at ^ (v_turn ^ 16), 16 * j * P, halves8<CODES>(vr[j].w[2], vr[j].w[3]));
                }
                if (lane < 2 * WK) {
                    const int key = WK * wave + (lane & (WK - 1));
                    scales[buf][lane >= WK][key] = scale;
                }
                odd = look && __any(odd);
                if (lane == 0) flags[buf][wave] = (unsigned char)(odd | (there ? 0 : 2));
            };
            const Sight tile_all = sight_of_all(a, rq.len, pmin, pmax), all = sight_of_all(a, rq.len, wmin, wmax);
            const Sight some = idle ? Sight{0, 0, 0} : sight_of_some(a, rq.len, wmin, wmax);

            if (b_hi > b_lo) {
                find_places(b_lo);
                int key0 = block_key<SHIFT>(bl, b_lo);
                bool there = load(b_lo), plain = all_of(tile_all, key0, SK);
                store(0, key0, there, plain);
                __syncthreads();
                for (int b = b_lo; b < b_hi; b++) {
                    const int buf = (b - b_lo) & 1, next = min(b + 1, b_hi - 1);      // (behind the last stage once more the same one)
                    if (next > b && ((next - b_lo) & 63) == 0) find_places(next);
                    there = load(next);
                    unsigned k_at = k_get + buf * BUF, v_at = v_get + buf * BUF;
                    asm volatile("" : "+v"(k_at), "+v"(v_at));
                    const uint32_t flag_word = *reinterpret_cast<const uint32_t *>(flags[buf]);
#pragma unroll
                    for (int h = 0; h < SK / 32; h++) {
                        const int key32 = key0 + 32 * h;
                        if (!any_of(some, key32, 32)) continue;
                        const unsigned char *block = stages + buf * BUF + SK * DH * 2 + 32 * h * DH * 2;
                        frag_t kf[2][KS];
#pragma unroll
                        for (int s = 0; s < 2; s++)
#pragma unroll
                            for (int k = 0; k < KS; k++) kf[s][k] = *lds_frag(k_at ^ (unsigned)(k << 6 ^ (DH > 64 ? pair_turn<DH>(0, 4 * k) << 4 : 0)), (32 * h + 16 * s) * DH * 2);
                        f32x4 ks[2], v[2];
#pragma unroll
                        for (int s = 0; s < 2; s++) {
                            const float *sk = &scales[buf][0][32 * h + 16 * s], *sv = &scales[buf][1][32 * h + 16 * s];
                            ks[s] = EVEN ? f32x4{sk[0], sk[0], sk[0], sk[0]} : *reinterpret_cast<const f32x4 *>(sk + 4 * g);
                            v[s] = EVEN ? f32x4{sv[0], sv[0], sv[0], sv[0]} : *reinterpret_cast<const f32x4 *>(sv + 4 * g);
                        }
                        f32x4 z[NT][2];
#pragma unroll
                        for (int t = 0; t < NT; t++)
#pragma unroll
                            for (int s = 0; s < 2; s++) {
                                z[t][s] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                                for (int k = 0; k < KS; k++) z[t][s] = mfma16(kf[s][k], q[t][k], z[t][s]);
                            }
                        frag_t vt[CT];
#pragma unroll
                        for (int c = 0; c < CT; c++) vt[c] = v_operand_at((const unsigned char *)lds_frag(v_at ^ (unsigned)(c << 5 ^ (DH > 64 ? pair_turn<DH>(0, 2 * c) << 4 : 0)), 32 * h * DH * 2), 16 * DH * 2);
                        const uint32_t fl = (uint32_t)__builtin_amdgcn_readfirstlane((int)flag_word);
                        const bool dirty = Code<CODES>::kOdd && (fl & 0x01010101u) != 0;
                        const int pg0 = -(int)(fl >> (8 * (2 * h * 16 / WK)) & 2), pg1 = -(int)(fl >> (8 * ((2 * h + 1) * 16 / WK)) & 2);
                        const bool masked = (pg0 | pg1) != 0 || !(plain || all_of(all, key32, 32));
                        if (__builtin_expect(dirty, 0))
#pragma unroll
                            for (int c = 0; c < CT; c++) clear_odd<_Float16>(vt[c]);
#pragma unroll
                        for (int t = 0; t < NT; t++) {
                            frag_t pf, pv;
                            if (!EVEN)
#pragma unroll
                                for (int s = 0; s < 2; s++) z[t][s] *= ks[s];
                            float c[2] = {EVEN ? sc[t] * ks[0][0] : sc[t], EVEN ? sc[t] * ks[1][0] : sc[t]};
                            f32x4 vt2[2] = {v[0], v[1]};
                            if (masked) {
                                hide_unseen(z[t], sight[t], key32, g, pg0, pg1);
                                hide_scales<EVEN>(z[t], c, vt2);
                            }
                            quant_probabilities<CT, EVEN>(z[t], c, vt2, st[t], lsum[t], o[t], pf, pv);
                            if (__builtin_expect(dirty, 0))
                                add_odd<_Float16, DH, true>(block, lane, pf, [&](int key) { return sees(sight[t], key32 + key, key & 16 ? pg1 : pg0); }, o[t]);
                            lsum[t] = mfma16(ones, pf, lsum[t]);
#pragma unroll
                            for (int c = 0; c < CT; c++) o[t][c] = mfma16(vt[c], pv, o[t][c]);
                        }
                    }
                    key0 = block_key<SHIFT>(bl, next);
                    plain = all_of(tile_all, key0, SK);
                    store(buf ^ 1, key0, there, plain);
                    __syncthreads();
                }
            }
            // ---- results, or sums for the joining kernel
            int tid = threadIdx.x;                                                  // (hidden, as above)
            asm volatile("" : "+v"(tid));
            const int part0 = tail ? cut : x, parts = whole ? 1 : tail ? shares : (piece * x + (min(piece, total - piece * x) - left) - at + cost + nb - 1) / piece - x + 1;
#pragma unroll
            for (int t = 0; t < NT; t++) {
                const int in_tile = wave * 16 * NT + t * 16 + (tid & 15), rho = tile * Shape::TILE_ROWS + in_tile, eg = (tid >> 4) & 3;
                if (rho >= n_rows) continue;
                const int i = rho / G, hq = head * G + (rho - i * G);
                const float l = checked_quant_sum(st[t].at, lsum[t][0]);
                if (!whole) {
                    const long long place = ((2ll * part0 + (b_lo == 0)) * kv + head) * Shape::TILE_ROWS + in_tile;
#pragma unroll
                    for (int c = 0; c < CT; c++) *reinterpret_cast<f32x4 *>(a.partial + place * DH + c * 16 + 4 * eg) = o[t][c] * st[t].unit;
                    if (eg == 0) {
                        a.ml[place] = float2{st[t].at, l};
                        if (b_lo == 0) a.where[(size_t)(rq.row0 + i) * a.heads + hq] = int2{part0, parts * kRowsPlace + in_tile};
                    }
                    continue;
                }
                const float f = (l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l) * st[t].unit;          // a row that sees nothing is zero
#pragma unroll
                for (int c = 0; c < CT; c++) {
                    const f32x4 y = o[t][c] * f;
                    const uint2 w = a.pages.dtype == ODB_F16 ? uint2{Num<_Float16>::pack(y[0], y[1]), Num<_Float16>::pack(y[2], y[3])}
                                                             : uint2{Num<__bf16>::pack(y[0], y[1]), Num<__bf16>::pack(y[2], y[3])};
                    store_out4(a, rq.row0 + i, hq, DH, c * 16 + 4 * eg, w);
                }
                if (a.split && eg == 0) a.where[(size_t)(rq.row0 + i) * a.heads + hq] = int2{part0, 0};
            }
        }
        if (!split) return;
        left -= end - at;
        if (left <= 0) return;
        at = 0;
        if (++tile == tiles) {
            do {
                if (++request >= a.n) return;
                rq = request_of(a, request);
                tiles = tiles_of(a, rq, Shape::TILE_ROWS);
            } while (tiles == 0);
            tile = 0;
        }
    }
}

template <int CODES, int DH, bool EVEN>
void launch_quant_dim(const PagedAttnQuant &a, int nt, hipStream_t s) {
    const dim3 grid((unsigned)(a.items * a.pages.n_kv_heads));
    if (nt == kManyRows) {
        constexpr int bytes = 2 * 2 * RowsShape<DH>::SK * DH * 2;
        allow_lds<quant_rows_kernel<CODES, DH, EVEN>>(bytes);
        if (a.split && !a.slots) launch_paged_plan(a, s);
        quant_rows_kernel<CODES, DH, EVEN><<<grid, 256, bytes, s>>>(a);
    } else if (nt == 1) {
        quant_attn_kernel<CODES, DH, 1, EVEN><<<grid, 256, 0, s>>>(a);
    } else if (nt == 2 || DH == 256) {
        quant_attn_kernel<CODES, DH, 2, EVEN><<<grid, 256, 0, s>>>(a);
    } else {
        if constexpr (DH != 256) quant_attn_kernel<CODES, DH, 4, EVEN><<<grid, 256, 0, s>>>(a);
    }
    if (a.split) launch_paged_join(a, s);
}

template <int CODES>
void launch_quant_codes(const PagedAttnQuant &a, int nt, hipStream_t s) {
    const bool even = a.scales.group_shift >= 4;
    switch (a.pages.head_dim) {
    case 64: return even ? launch_quant_dim<CODES, 64, true>(a, nt, s) : launch_quant_dim<CODES, 64, false>(a, nt, s);
    case 128: return even ? launch_quant_dim<CODES, 128, true>(a, nt, s) : launch_quant_dim<CODES, 128, false>(a, nt, s);
    default: return even ? launch_quant_dim<CODES, 256, true>(a, nt, s) : launch_quant_dim<CODES, 256, false>(a, nt, s);
    }
}

}  // namespace
}  // namespace odb
