// Paged K/V in 8 bits: rows stored as codes with scales (odb_qk_norm_rope_quant), and read back (odb_paged_read_quant).
#include "paged.h"
#include "paged_rope.h"

namespace odb {

namespace {

constexpr float kTiny = 0x1p-100f;             // a group whose values are all below has codes and scale zero
constexpr float kTinyScale = 0x1p-110f;        // no scale is smaller, but zero (2^-100 / 448); what is there below it counts as zero

// Four bytes of codes from numbers that are within the codes' range once clamped: to nearest, ties to even.
__device__ __forceinline__ uint32_t int8_codes(float a, float b, float c, float d) {
    // (1.5 * 2^23 added: the sum's last place is one, and its low byte the code)
    auto bits = [](float x) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(x, -127.f, 127.f) + 12582912.f); };
    const uint32_t ab = __builtin_amdgcn_perm(bits(b), bits(a), 0x0c0c0400u), cd = __builtin_amdgcn_perm(bits(d), bits(c), 0x04000c0cu);
    return ab | cd;
}
__device__ __forceinline__ uint32_t e4m3_codes(float a, float b, float c, float d) {
    auto in = [](float x) { return __builtin_amdgcn_fmed3f(x, -448.f, 448.f); };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(in(a), in(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(in(c), in(d), w, true);
}
__device__ __forceinline__ uint2 codes8(bool int8, const f32x8 &x) {
    return int8 ? uint2{int8_codes(x[0], x[1], x[2], x[3]), int8_codes(x[4], x[5], x[6], x[7])}
                : uint2{e4m3_codes(x[0], x[1], x[2], x[3]), e4m3_codes(x[4], x[5], x[6], x[7])};
}
// numbers of four codes
__device__ __forceinline__ f32x4 numbers4(bool int8, uint32_t w) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    f32x4 r;
    if (int8) {
#pragma unroll
        for (int i = 0; i < 4; i++) r[i] = (float)(int)(int8_t)(w >> (8 * i));
    } else {
        const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        r = f32x4{lo[0], lo[1], hi[0], hi[1]};
    }
    return r;
}

// x * times / over, rounded once after the product: over's reciprocal is rounded to nearest, and with it a quotient that is off by less than
// one place becomes the nearest one by its remainder (Markstein), so that values which lie between two codes are seen to.  An infinite x
// goes beyond the largest code.
struct Ratio { float times, over, per; };
__device__ __forceinline__ f32x8 divided(const f32x8 &x, const Ratio &r) {
    f32x8 y;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float t = x[i] * r.times, q = __builtin_amdgcn_fmed3f(t * r.per, -1024.f, 1024.f);
        y[i] = __builtin_fmaf(__builtin_fmaf(-q, r.over, t), r.per, q);
    }
    return y;
}

}  // namespace

// Spans of positions, aligned to their number, that a workgroup quantises at once: as many as its threads hold, or a group.
static int span_shift(int head_dim, int group_shift) {
    const int least = head_dim == 64 ? 6 : head_dim == 128 ? 5 : 4;
    return group_shift > least ? group_shift : least;
}
// Numbers of a request's spans: those of m rows fall into at most floor((m - 2) / span) + 2; request r's are numbered from floor(its first
// row / span) + 2 r on, which leaves room for them.
static long long quant_spans(int n, int rows, bool cu_rows, int rows_per_request, const QuantScales &s, int head_dim) {
    const int shift = span_shift(head_dim, s.group_shift), span = 1 << shift;
    return cu_rows ? (rows >> shift) + 2ll * n : (long long)n * ((rows_per_request + 2 * span - 2) >> shift);
}

static long long query_workgroups(int rows, int heads, int head_dim) {
    const int per_wave = 64 / (head_dim / 16);
    return ((long long)rows * ((heads + per_wave - 1) / per_wave) + 3) / 4;
}
long long quant_workgroups(int n, int rows, int heads, bool cu_rows, int rows_per_request, const odb_pages &p, const QuantScales &s) {
    return quant_spans(n, rows, cu_rows, rows_per_request, s, p.head_dim) * 2 * p.n_kv_heads + query_workgroups(rows, heads, p.head_dim);
}

// Two kinds of workgroups in one launch.  The last `span_groups` take a span of positions of one request, for one head, K or V:
// DH / 16 lanes a position with sixteen channels each, which stay in registers from the load to the codes; the largest magnitude of a group
// goes through lanes and LDS.  The others norm and turn queries, as qk_norm_rope_kernel does, a row and group of heads a wave.
// Bound by the memory: 11735 rows of four prompts, 48 heads of 128 in bfloat16, 267 MB, 62 us (4.3 TB/s; a copy 5.1; queries behind the spans 66, two rows of them a wave 72, stored
// past the caches 64).  Few rows are bound by loads that wait for each other - row offsets, lengths, page, scale: eleven tokens 4.7 us,
// 6 x 32 rows of 96 heads from 32 bits 7.0.
template <class TI, class TO, int DH, int PASSES>
__global__ __launch_bounds__(256) void qk_norm_rope_quant_kernel(QkNormRopeQuant a, unsigned span_groups) {
    constexpr int LANES = DH / 16, PER_WAVE = 64 / LANES, PER_PASS = 4 * PER_WAVE, SPAN = PER_PASS * PASSES;
    __shared__ float tops[4 * PASSES];
    __shared__ int states[4 * PASSES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane % LANES, slice = lane / LANES;
    const odb_pages &pg = a.pages;
    const int kv = pg.n_kv_heads;
    const HeadLane hl = a.interleaved ? head_lane<true>(l, a.rot) : head_lane<false>(l, a.rot);
    auto turn = [&](f32x8 &x, f32x8 &y, const float (&cs)[8], const float (&sn)[8]) {
        if (a.interleaved) turn_head<true>(x, y, cs, sn);
        else turn_head<false>(x, y, cs, sn);
    };
    const f32x8 zeros = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

    const unsigned query_groups = gridDim.x - span_groups;
    if (blockIdx.x < query_groups) {                            // queries
        const int waves_per_row = (a.heads + PER_WAVE - 1) / PER_WAVE;
        const unsigned w = blockIdx.x * 4u + wave;
        const int row = (int)(w / (unsigned)waves_per_row), head = (int)(w % (unsigned)waves_per_row) * PER_WAVE + slice;
        if (row >= a.rows || head >= a.heads) return;
        const int pos = a.positions[row];
        bool live = pos >= 0 && pos < a.n_pos;
        if (a.cu_rows) live = live && row >= a.cu_rows[0] && row < a.cu_rows[a.n];
        float cs[8], sn[8];
        if (hl.turns && live) load_angles(a.table + (size_t)pos * a.rot + l * 16, cs, sn);
        const TI *src = (const TI *)a.q + (size_t)row * a.q_row + (size_t)head * DH;
        f32x8 x = load8(src + hl.c0), y = load8(src + hl.c1);
        if (a.q_gain) norm_head<DH>(x, y, a.q_gain, a.eps, hl.c0, hl.c1);
        if (hl.turns) turn(x, y, cs, sn);
        if (!live) x = y = zeros;
        if (a.status) {                                         // (of the model's forward, whose type is binary16)
            int out = 0;
#pragma unroll
            for (int i = 0; i < 8; i += 4) out |= (int)out_of_f16(x[i], x[i + 1], x[i + 2], x[i + 3]) | (int)out_of_f16(y[i], y[i + 1], y[i + 2], y[i + 3]);
            if (out) {
                atomicOr(a.status, kStatusSaturated);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    x[i] = fminf(fmaxf(x[i], -65504.f), 65504.f);
                    y[i] = fminf(fmaxf(y[i], -65504.f), 65504.f);
                }
            }
        }
        TO *dst = (TO *)a.q_out + (size_t)row * a.q_out_row + (size_t)head * DH;
        store8(dst + hl.c0, x);
        store8(dst + hl.c1, y);
        return;
    }

    // ---- keys or values of a span: which
    const unsigned item = blockIdx.x - query_groups;
    const bool is_k = item & 1;
    const int head = (int)((item >> 1) % (unsigned)kv);
    int number = (int)((item >> 1) / (unsigned)kv), r = 0, lo, hi;
    constexpr int SHIFT = SPAN == 16 ? 4 : SPAN == 32 ? 5 : 6;
    static_assert(1 << SHIFT == SPAN, "span");
    if (a.cu_rows) {
        auto start = [&](int i, int row) { return 2 * i + (min(max(row, 0), a.rows) >> SHIFT); };
        for (int rest = a.n;;) {
            const int step = (rest + 63) >> 6, i = r + lane * step;
            const int c = __popcll(__ballot(i < r + rest && start(i, a.cu_rows[min(i, a.n - 1)]) <= number));
            if (c == 0) return;
            r += (c - 1) * step;
            if (step == 1) break;
            rest = min(step, rest - (c - 1) * step);
        }
        lo = min(max(a.cu_rows[r], 0), a.rows);
        hi = min(max(a.cu_rows[r + 1], 0), a.rows);
        number -= start(r, lo);
    } else {
        const int per = (a.rows_per_request + 2 * SPAN - 2) >> SHIFT;
        r = number / per;
        number -= r * per;
        if (r >= a.n) return;
        lo = r * a.rows_per_request;
        hi = lo + a.rows_per_request;
    }
    const int m = hi - lo, len = (int)min((long long)max(a.kv_len[r], 0), (long long)a.columns << a.page_shift);
    constexpr int kFar = 1 << 30;
    const int first = a.first ? min(max(a.first[r], -kFar), kFar) : len - m;
    const int span0 = ((first >> SHIFT) + number) << SHIFT;
    if (m <= 0 || span0 >= first + m || span0 >= len) return;

    // ---- the new values, turned
    const TI *base = (const TI *)(is_k ? a.k : a.v) + (size_t)head * DH;
    const long long row_stride = is_k ? a.k_row : a.v_row;
    const int c0 = is_k ? hl.c0 : l * 16, c1 = is_k ? hl.c1 : l * 16 + 8;
    const float limit = 3.402823466e38f;
    f32x8 x[PASSES], y[PASSES];
    int page[PASSES];
    bool fresh[PASSES], kept[PASSES];
    float top[PASSES];
#pragma unroll
    for (int j = 0; j < PASSES; j++) {
        const int p = span0 + j * PER_PASS + wave * PER_WAVE + slice, i = p - first;
        const bool mine = i >= 0 && i < m, inside = p >= 0 && p < len;
        int id = -1, pos = -1;
        if (inside) id = a.tables[(size_t)r * a.columns + (p >> a.page_shift)];
        if (mine) pos = a.positions[lo + i];
        x[j] = y[j] = zeros;
        if (mine) {
            const TI *src = base + (size_t)(lo + i) * row_stride;
            x[j] = load8(src + c0);
            y[j] = load8(src + c1);
        }
        const bool there = id >= 0 && id < pg.n_pages;
        page[j] = there ? id : -1;
        fresh[j] = there && mine && pos >= 0 && pos < a.n_pos;
        kept[j] = there && !fresh[j];
        if (is_k) {
            float cs[8], sn[8];
            if (hl.turns && fresh[j]) load_angles(a.table + (size_t)pos * a.rot + l * 16, cs, sn);
            if (a.k_gain) norm_head<DH>(x[j], y[j], a.k_gain, a.eps, c0, c1);
            if (hl.turns && fresh[j]) turn(x[j], y[j], cs, sn);
        }
        float t = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) t = __builtin_elementwise_maximum(t, __builtin_elementwise_maximum(fabsf(x[j][e]), fabsf(y[j][e])));
        if (fresh[j] && !(t <= limit)) {                          // rare: infinite, or no number
            if (a.odd) atomicOr(a.odd, a.odd_bit);
            t = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                x[j][e] = x[j][e] == x[j][e] ? x[j][e] : 0.f;
                y[j][e] = y[j][e] == y[j][e] ? y[j][e] : 0.f;
                t = fmaxf(t, fmaxf(fabsf(x[j][e]) <= limit ? fabsf(x[j][e]) : 0.f, fabsf(y[j][e]) <= limit ? fabsf(y[j][e]) : 0.f));
            }
        }
        top[j] = fresh[j] ? t : 0.f;
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) top[j] = fmaxf(top[j], __shfl_xor(top[j], o));
    }

    // ---- the groups' scales
    const bool alone = a.scales.group_shift == 0;               // a group per position
    bool any_kept[PASSES], any_fresh[PASSES];
    if (alone) {
#pragma unroll
        for (int j = 0; j < PASSES; j++) { any_fresh[j] = fresh[j]; any_kept[j] = false; }
    } else {
        // (a wave's positions of a pass are in one group: 16 at most)
#pragma unroll
        for (int j = 0; j < PASSES; j++) {
            float t = top[j];
#pragma unroll
            for (int o = LANES; o < 64; o <<= 1) t = fmaxf(t, __shfl_xor(t, o));
            const int flags = (__any(kept[j]) ? 1 : 0) | (__any(fresh[j]) ? 2 : 0);
            if (lane == 0) { tops[4 * j + wave] = t; states[4 * j + wave] = flags; }
        }
        __syncthreads();
        const int waves = max(1, (1 << a.scales.group_shift) / PER_WAVE);      // waves' passes of a group
#pragma unroll
        for (int j = 0; j < PASSES; j++) {
            const int w0 = (4 * j + wave) / waves * waves;
            float t = 0.f;
            int flags = 0;
            for (int w = w0; w < w0 + waves; w++) {
                t = fmaxf(t, tops[w]);
                flags |= states[w];
            }
            top[j] = t;
            any_kept[j] = flags & 1;
            any_fresh[j] = flags & 2;
        }
    }
    unsigned char *codes = (unsigned char *)(is_k ? pg.k : pg.v) + (size_t)head * pg.head_stride;
    float *scales = (is_k ? a.scales.k : a.scales.v) + (size_t)head * a.scales.head_stride;
    const bool int8 = a.scales.codes == ODB_INT8;
    // the scales that are there, all before any is written (a group's threads are several waves)
    float there[PASSES], old[PASSES];
    size_t scale_at[PASSES];
#pragma unroll
    for (int j = 0; j < PASSES; j++) {
        const int in = (span0 + j * PER_PASS + wave * PER_WAVE + slice) & ((1 << a.page_shift) - 1);
        scale_at[j] = (size_t)max(page[j], 0) * a.scales.page_stride + (in >> a.scales.group_shift);
        there[j] = page[j] >= 0 && any_kept[j] && any_fresh[j] ? scales[scale_at[j]] : 0.f;
        old[j] = there[j] >= kTinyScale && there[j] <= limit ? there[j] : 0.f;
    }
    if (!alone) __syncthreads();
#pragma unroll
    for (int j = 0; j < PASSES; j++) {
        if (page[j] < 0 || !any_fresh[j]) continue;
        const float most = int8 ? 127.f : 448.f, top_j = top[j] < kTiny ? 0.f : top[j], mine = top_j / most;
        const bool own = mine >= old[j];
        const float scale = own ? mine : old[j];
        // (M and a over 512: nothing leaves the range, and nothing is rounded by it)
        Ratio ratio{own ? most * 0x1p-9f : 1.f, own ? top_j * 0x1p-9f : old[j], 0.f};
        ratio.per = scale > 0.f ? 1.0f / ratio.over : 0.f;
        const int in = (span0 + j * PER_PASS + wave * PER_WAVE + slice) & ((1 << a.page_shift) - 1);
        unsigned char *dst = codes + (size_t)page[j] * pg.page_stride + (size_t)in * pg.pos_stride;
        if (fresh[j]) {
            const f32x8 u = scale > 0.f ? divided(x[j], ratio) : zeros, v = scale > 0.f ? divided(y[j], ratio) : zeros;
            *reinterpret_cast<uint2 *>(dst + c0) = codes8(int8, u);
            *reinterpret_cast<uint2 *>(dst + c1) = codes8(int8, v);
        } else if (mine > old[j]) {                               // what stays is rounded anew where the scale grows
            const float less = old[j] * ratio.times / ratio.over;
            uint4 w = *reinterpret_cast<const uint4 *>(dst + l * 16);
            auto again = [&](uint32_t z) {
                f32x4 u = numbers4(int8, z) * less;
#pragma unroll
                for (int e = 0; e < 4; e++) u[e] = u[e] == u[e] ? u[e] : 0.f;
                return int8 ? int8_codes(u[0], u[1], u[2], u[3]) : e4m3_codes(u[0], u[1], u[2], u[3]);
            };
            w = uint4{again(w.x), again(w.y), again(w.z), again(w.w)};
            *reinterpret_cast<uint4 *>(dst + l * 16) = w;
        }
        // (one position of a group writes it; there is one below its length in every group with a new row)
        const int p = span0 + j * PER_PASS + wave * PER_WAVE + slice, at = p & ((1 << a.scales.group_shift) - 1);
        if (l == 0 && (at == 0)) scales[scale_at[j]] = scale;
    }
}

template <class TI, class TO, int DH>
static void launch_quant_rows(const QkNormRopeQuant &a, int shift, hipStream_t s) {
    const unsigned spans = (unsigned)(quant_spans(a.n, a.rows, a.cu_rows, a.rows_per_request, a.scales, DH) * 2 * a.pages.n_kv_heads);
    const unsigned grid = spans + (unsigned)query_workgroups(a.rows, a.heads, DH);
    const int passes = (1 << shift) / (256 / (DH / 16));
    if (passes == 1) qk_norm_rope_quant_kernel<TI, TO, DH, 1><<<dim3(grid), 256, 0, s>>>(a, spans);
    if constexpr (DH > 64)
        if (passes == 2) qk_norm_rope_quant_kernel<TI, TO, DH, 2><<<dim3(grid), 256, 0, s>>>(a, spans);
    if constexpr (DH > 128)
        if (passes == 4) qk_norm_rope_quant_kernel<TI, TO, DH, 4><<<dim3(grid), 256, 0, s>>>(a, spans);
}

template <class TI, class TO>
static void launch_quant_types(const QkNormRopeQuant &a, hipStream_t s) {
    const int shift = span_shift(a.pages.head_dim, a.scales.group_shift);
    switch (a.pages.head_dim) {
    case 64: return launch_quant_rows<TI, TO, 64>(a, shift, s);
    case 128: return launch_quant_rows<TI, TO, 128>(a, shift, s);
    default: return launch_quant_rows<TI, TO, 256>(a, shift, s);
    }
}

void launch_qk_norm_rope_quant(const QkNormRopeQuant &a, hipStream_t s) {
    if (a.rows < 1) return;
    if (a.pages.dtype == ODB_F16) {
        if (a.in_dtype == ODB_F32) launch_quant_types<float, _Float16>(a, s);
        else launch_quant_types<_Float16, _Float16>(a, s);
    } else {
        if (a.in_dtype == ODB_F32) launch_quant_types<float, __bf16>(a, s);
        else launch_quant_types<__bf16, __bf16>(a, s);
    }
}

// ---- values read back ------------------------------------------------------------------------------------------------

// Sixteen bytes of values a lane, K and V of a row beside each other in the order of the lanes, of two rows whose loads are on their way
// together; stored past the caches.  Bound by the memory: 24001 positions of 8 heads of 128, 147 MB, 22.8 us (6.4 TB/s; with ordinary stores 34, one
// row 40), to 32 bits 39 (ordinary stores 65).  70 positions 2.6 us: a slot, then its codes.
constexpr int kReadRows = 2;
template <class TO>
__global__ __launch_bounds__(256) void paged_read_quant_kernel(PagedReadQuant a, unsigned per_row) {
    constexpr int CH = 16 / sizeof(TO), WORDS = CH / 4;
    typedef TO out_t __attribute__((ext_vector_type(CH)));
    typedef float f32_t __attribute__((ext_vector_type(CH)));
    const unsigned t = blockIdx.x * 256u + threadIdx.x, part = t / per_row, row0 = part * kReadRows;
    if (row0 >= (unsigned)a.rows) return;
    const odb_pages &pg = a.pages;
    const unsigned half = per_row >> 1, at = t - part * per_row, is_v = at >= half, e = (at - (is_v ? half : 0)) * CH, head = e / (unsigned)pg.head_dim, c = e % (unsigned)pg.head_dim;
    const unsigned char *codes = (const unsigned char *)(is_v ? pg.v : pg.k) + (size_t)head * pg.head_stride + c;
    const float *scales = (is_v ? a.scales.v : a.scales.k) + (size_t)head * a.scales.head_stride;
    uint32_t w[kReadRows][WORDS];
    float scale[kReadRows];
    bool there[kReadRows];
#pragma unroll
    for (int i = 0; i < kReadRows; i++) {
        const int slot = row0 + i < (unsigned)a.rows ? a.slots[row0 + i] : -1, page = slot >= 0 ? (int)((unsigned)slot / (unsigned)pg.page_size) : -1;
        there[i] = page >= 0 && page < pg.n_pages;
        const int in = there[i] ? slot - page * pg.page_size : 0;
        const size_t from = there[i] ? page : 0;
        const uint32_t *src = reinterpret_cast<const uint32_t *>(codes + from * pg.page_stride + (size_t)in * pg.pos_stride);
#pragma unroll
        for (int j = 0; j < WORDS; j++) w[i][j] = src[j];
        scale[i] = scales[from * a.scales.page_stride + (in >> a.scales.group_shift)];
    }
    const bool int8 = a.scales.codes == ODB_INT8;
    TO *out = (TO *)(is_v ? a.v : a.k) + e;
    const long long stride = is_v ? a.v_row : a.k_row;
#pragma unroll
    for (int i = 0; i < kReadRows; i++) {
        if (row0 + i >= (unsigned)a.rows) return;
        f32_t x;
#pragma unroll
        for (int j = 0; j < WORDS; j++) {
            const f32x4 u = numbers4(int8, w[i][j]) * scale[i];
#pragma unroll
            for (int k = 0; k < 4; k++) x[4 * j + k] = there[i] ? u[k] : 0.f;
        }
        out_t *dst = reinterpret_cast<out_t *>(out + (size_t)(row0 + i) * stride);
        __builtin_nontemporal_store(__builtin_convertvector(x, out_t), dst);
    }
}

void launch_paged_read_quant(const PagedReadQuant &a, hipStream_t s) {
    if (a.rows < 1) return;
    const unsigned per_row = 2u * a.pages.n_kv_heads * a.pages.head_dim / (a.out_dtype == ODB_F32 ? 4 : 8);
    const dim3 grid((unsigned)((((unsigned long long)a.rows + kReadRows - 1) / kReadRows * per_row + 255) / 256));
    if (a.out_dtype == ODB_F16) paged_read_quant_kernel<_Float16><<<grid, 256, 0, s>>>(a, per_row);
    else if (a.out_dtype == ODB_BF16) paged_read_quant_kernel<__bf16><<<grid, 256, 0, s>>>(a, per_row);
    else paged_read_quant_kernel<float><<<grid, 256, 0, s>>>(a, per_row);
}

}  // namespace odb
