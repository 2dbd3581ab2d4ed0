// Operators around a paged K/V cache: page tables and slot maps, the table of rotary angles, and the pass that norms and
// turns queries and keys and stores keys and values in their pages.  Attention over the pages is in paged_attn.hip.
#include "launch.h"
#include "paged.h"
#include "paged_rope.h"

namespace odb {

// ---- page tables ----------------------------------------------------------------------------------------------------

// Sums of these kernels saturate at 2^30 (more than any pool or row buffer has), so that lengths of any size cannot wrap them.
constexpr unsigned kSat = 1u << 30;
__device__ __forceinline__ unsigned sat_add(unsigned a, unsigned b) { return min(a + b, kSat); }

// index of the request whose part of the inclusive sums holds item i (sums[n - 1] > i)
__device__ __forceinline__ int owner(const unsigned *sums, int n, unsigned i) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] > i) hi = mid; else lo = mid + 1;
    }
    return lo;
}

// Pages that a request holds, needs, and whether its wanted length can be named by its table at all.
struct PageNeed { unsigned had, need; int held, wanted; bool fits; };
__device__ __forceinline__ PageNeed page_need(const PageTables &a, int held, int wanted) {
    PageNeed p;
    const int top = a.columns << a.page_shift, mask = (1 << a.page_shift) - 1;      // (at most 2^30)
    p.held = min(max(held, 0), top);
    p.wanted = wanted;
    p.fits = p.wanted >= 0 && p.wanted <= top;
    p.had = ((unsigned)p.held + mask) >> a.page_shift;
    p.need = p.fits ? ((unsigned)p.wanted + mask) >> a.page_shift : p.had;
    return p;
}

// One launch, no exchange between workgroups: each of them computes the three running sums over the requests (pages taken,
// pages given back, rows) for itself - a thread takes up to 16 neighbouring requests, then one scan over the threads - and keeps
// them in LDS with what else the items need; then it does its share of one kind of items: rows, pages given back, pages taken.  What one
// workgroup writes no other reads: entries behind a request's held pages are not looked up in the table but derived from the
// stack, and the stack's new top from the tables of those that gave back.  A second call with the same inputs therefore writes the
// same values again.  Bound by its chain of dependent reads: 24 requests 5.5 us, 700 with 2.2e5 rows 10.8 (1.9 MB, of which the memory
// takes 0.4); with all kinds of items done by every workgroup in turn 11.8, and with a read per request in the sums 12.8.
__global__ __launch_bounds__(256) void page_tables_kernel(PageTables a) {
    extern __shared__ unsigned lds[];
    __shared__ unsigned wave_sums[4][3], tops[4], misses[4];
    unsigned *taken = lds, *given = lds + a.n, *rows = lds + 2 * a.n, *had = lds + 3 * a.n, *need = lds + 4 * a.n;
    int *first = (int *)(lds + 5 * a.n), *length = (int *)(lds + 6 * a.n);
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int per = (a.n + 255) / 256, r0 = t * per, r1 = min(a.n, r0 + per);
    const unsigned n_free = (unsigned)min(max(*a.n_free, 0), a.n_pages);

    // the inputs first, neighbouring threads reading neighbouring requests: one latency for all of them
    int *in_held = (int *)had, *in_wanted = (int *)need, *in_count = (int *)rows;
#pragma unroll 4
    for (int r = t; r < a.n; r += 256) {
        const int h = a.held[r], w = a.wanted[r], c = a.count ? a.count[r] : 0, f = a.first ? a.first[r] : 0;
        in_held[r] = h;
        in_wanted[r] = w;
        in_count[r] = c;
        first[r] = f;
    }
    __syncthreads();
    unsigned sum[3] = {0, 0, 0};
    for (int r = r0; r < r1; r++) {
        const PageNeed p = page_need(a, in_held[r], in_wanted[r]);
        const int c = a.count ? in_count[r] : p.fits ? p.wanted - p.held : 0;
        taken[r] = sum[0] = sat_add(sum[0], p.need > p.had ? p.need - p.had : 0);
        given[r] = sum[1] = sat_add(sum[1], p.had > p.need ? p.had - p.need : 0);
        rows[r] = sum[2] = sat_add(sum[2], min((unsigned)max(c, 0), (unsigned)a.rows_cap));
        had[r] = p.had;
        need[r] = p.need;
        if (!a.first) first[r] = p.held;
        length[r] = p.fits ? p.wanted : ~p.held;                   // (a length that cannot be: the request is refused)
    }
    unsigned before[3], total[3] = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < 3; i++) {
        unsigned v = sum[i];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const unsigned up = __shfl_up(v, o);
            if (lane >= o) v = sat_add(v, up);
        }
        if (lane == 63) wave_sums[wave][i] = v;
        before[i] = __shfl_up(v, 1);
        if (lane == 0) before[i] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; i++)
        for (int w = 0; w < 4; w++) {
            if (w < wave) before[i] = sat_add(before[i], wave_sums[w][i]);
            total[i] = sat_add(total[i], wave_sums[w][i]);
        }
    const unsigned have = n_free + total[1], n_rows = min(total[2], (unsigned)a.rows_cap);
    unsigned refused = 0, most = 0;
    for (int r = r0; r < r1; r++) {
        taken[r] = sat_add(taken[r], before[0]);
        given[r] = sat_add(given[r], before[1]);
        rows[r] = sat_add(rows[r], before[2]);
        // pages of a request behind the first refused one are not granted either: the sums only rise
        const bool takes = need[r] > had[r], ok = length[r] >= 0 && (!takes || taken[r] <= have);
        const int held = length[r] < 0 ? ~length[r] : ok ? 0 : page_need(a, a.held[r], 0).held;
        length[r] = ok ? length[r] : held;
        refused += !ok;
        if (ok && takes) most = max(most, taken[r]);
        if (blockIdx.x == 0) {
            a.len[r] = length[r];
            a.cu_rows[r + 1] = (int)min(rows[r], (unsigned)a.rows_cap);
        }
    }
    __syncthreads();

    // The page that takes number i off the stack: those given back in this call lie on top.
    auto taken_page = [&](unsigned i) -> int {
        const unsigned at = have - 1 - i;
        if (at < n_free) return a.free_pages[at];
        const unsigned g = at - n_free;
        const int r = owner(given, a.n, g);
        return a.tables[(size_t)r * a.columns + need[r] + (g - (r ? given[r - 1] : 0))];
    };
    // rows: position and slot, four neighbouring ones per thread, which mostly share their request and often their page
    const int role = (int)blockIdx.x < a.row_groups ? 0 : (int)blockIdx.x < a.row_groups + a.page_groups ? 1 : 2;
    const unsigned step = (role ? a.page_groups : a.row_groups) * 256, item0 = (blockIdx.x - (role ? a.row_groups + (role - 1) * a.page_groups : 0)) * 256 + t;
    for (unsigned i0 = role == 0 ? item0 * 4 : n_rows; i0 < n_rows; i0 += step * 4) {
        int r = owner(rows, a.n, i0), page = -1;
        long long page_at = -1;                                    // r and page number that `page` was looked up for
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const unsigned i = i0 + k;
            if (i >= n_rows) break;
            while (rows[r] <= i) r++;
            const long long pos = (long long)first[r] + (i - (r ? rows[r - 1] : 0));
            int slot = -1;
            if (pos >= 0 && pos < length[r]) {
                const unsigned j = (unsigned)pos >> a.page_shift;
                const long long key = (long long)r << 32 | j;
                if (key != page_at) {
                    page = j < had[r] ? a.tables[(size_t)r * a.columns + j] : taken_page((r ? taken[r - 1] : 0) + (j - had[r]));
                    page_at = key;
                }
                if (page >= 0 && page < a.n_pages) slot = (page << a.page_shift) + ((int)pos & ((1 << a.page_shift) - 1));
            }
            a.slots[i] = slot;
            a.positions[i] = (int)min(pos, 0x7fffffffll);
        }
    }
    // pages given back go on the stack
    for (unsigned g = role == 1 ? item0 : total[1]; g < total[1]; g += step) {
        const int r = owner(given, a.n, g);
        if (n_free + g < (unsigned)a.n_pages) a.free_pages[n_free + g] = a.tables[(size_t)r * a.columns + need[r] + (g - (r ? given[r - 1] : 0))];
    }
    // pages taken go into the tables
    for (unsigned i = role == 2 ? item0 : total[0]; i < min(total[0], have); i += step) {
        const int r = owner(taken, a.n, i);
        if (taken[r] > have) break;
        a.tables[(size_t)r * a.columns + had[r] + (i - (r ? taken[r - 1] : 0))] = taken_page(i);
    }
    if (blockIdx.x) return;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        refused += __shfl_xor(refused, o);
        most = max(most, __shfl_xor(most, o));
    }
    if (lane == 0) { misses[wave] = refused; tops[wave] = most; }
    __syncthreads();
    if (t == 0) {
        most = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
        a.cu_rows[0] = 0;
        a.state[0] = (int)min(have - most, (unsigned)a.n_pages);
        a.state[1] = (int)most;
        a.state[2] = (int)total[1];
        a.state[3] = (int)(misses[0] + misses[1] + misses[2] + misses[3]);
    }
}

void launch_page_tables(PageTables a, hipStream_t s) {
    // four rows per thread up to two workgroups per CU (more would only repeat the sums), and one thread for every eight requests'
    // pages; the kinds of items are done beside each other, since each is a chain of dependent reads
    a.row_groups = a.rows_cap / 1024 + 1 < 512 ? a.rows_cap / 1024 + 1 : 512;
    a.page_groups = a.n / 32 + 1;
    if (a.n * 28 > 65536) allow_lds<page_tables_kernel>(kMaxRequests * 28);
    page_tables_kernel<<<dim3(a.row_groups + 2 * a.page_groups), 256, a.n * 28, s>>>(a);
}

// ---- rotary angles --------------------------------------------------------------------------------------------------

// cos and sin of 2 pi r for |r| <= 1/2 turn, by the quarter turn nearest to r and Taylor's series on the remaining eighth:
// |y| <= pi / 4, where the first terms left out, y^17 / 17! and y^16 / 16!, are below 1.1e-15: far below half a step of the
// float that is stored.
__device__ __forceinline__ void turn_sincos(double r, double &c, double &s) {
    const double q = rint(4.0 * r), y = 6.283185307179586476925 * (r - 0.25 * q), z = y * y;
    double ps = -7.647163731819816476e-13, pc = -1.147074559772972471e-11;     // -1/15!, -1/14!
    ps = fma(ps, z, 1.605904383682161460e-10); pc = fma(pc, z, 2.087675698786809898e-9);     // 1/13!, 1/12!
    ps = fma(ps, z, -2.505210838544171878e-8); pc = fma(pc, z, -2.755731922398589065e-7);    // -1/11!, -1/10!
    ps = fma(ps, z, 2.755731922398589065e-6); pc = fma(pc, z, 2.480158730158730159e-5);      // 1/9!, 1/8!
    ps = fma(ps, z, -1.984126984126984127e-4); pc = fma(pc, z, -1.388888888888888889e-3);    // -1/7!, -1/6!
    ps = fma(ps, z, 8.333333333333333333e-3); pc = fma(pc, z, 4.166666666666666667e-2);      // 1/5!, 1/4!
    ps = fma(ps, z, -1.666666666666666667e-1); pc = fma(pc, z, -0.5);
    const double sy = fma(ps * z, y, y), cy = fma(pc, z, 1.0);
    const int k = (int)q & 3;
    const double u = k & 1 ? sy : cy, w = k & 1 ? cy : sy;
    c = k == 1 || k == 2 ? -u : u;
    s = k >= 2 ? -w : w;
}

// The angle is counted in turns, p * (hi + lo), and its whole turns are dropped before anything is rounded to fewer bits, so a
// position of 2^22 has the same error as the first.  A thread computes one pair at every eighth position that way and turns on
// from there by the pair's own angle, seven times in 64 bits (an error of 7 * 2^-52 at most): 14 operations of 64 bits for an entry
// and not 36.  Pairs of a position lie beside each other: stores of 512 contiguous bytes per wave.  Bound by those: 131072 positions of
// 64 pairs, 67 MB, 12 us (5.3 TB/s; every entry by series 24 us).
constexpr int kAngleRun = 8;
__global__ __launch_bounds__(256) void rope_angles_kernel(RopeTable a) {
    const unsigned i = blockIdx.x * 256u + threadIdx.x, run = i / (unsigned)a.pairs, j = i - run * a.pairs;
    const int p0 = (int)run * kAngleRun;
    if (p0 >= a.n_pos) return;
    const double p = (double)p0, hi = a.hi[j], lo = a.lo[j], r = fma(p, hi, -rint(p * hi)) + p * lo, one = (hi - rint(hi)) + lo;
    double c, s, dc, ds;
    turn_sincos(r - rint(r), c, s);
    turn_sincos(one, dc, ds);
    c *= a.magnitude;
    s *= a.magnitude;
    float *out = a.table + 2 * ((size_t)p0 * a.pairs + j);
    const int n = min(kAngleRun, a.n_pos - p0);
    for (int k = 0; k < n; k++) {
        *reinterpret_cast<float2 *>(out + 2 * (size_t)k * a.pairs) = float2{(float)c, (float)s};
        const double u = fma(c, dc, -(s * ds)), w = fma(s, dc, c * ds);
        c = u;
        s = w;
    }
}

void launch_rope_angles(const RopeTable &a, hipStream_t s) {
    const long long total = ((long long)a.n_pos + kAngleRun - 1) / kAngleRun * a.pairs;          // at most 2^19 * 2^7
    rope_angles_kernel<<<dim3((unsigned)((total + 255) / 256)), 256, 0, s>>>(a);
}

// ---- norms and rotation of queries and keys, K/V to their pages ------------------------------------------------------

// A head is held by DH / 16 lanes with 16 channels each: in the half layout channel pair (j, j + rot / 2) sits in one lane as
// elements of its first and its second eight, in the interleaved layout (2j, 2j + 1) inside each eight.  Lanes behind the rotated
// part hold two neighbouring eights that pass through.  A wave does as many heads of one row as it has groups of lanes, and nothing
// else: with loops over more heads, which would load the row's angles once for all of them, the large call is slower.  Bound by the
// memory, every element read and written once: 16411 rows of 48 heads of 128 bfloat16, 408 MB, take 81 us (5.0 TB/s; a copy reaches
// 4.9), with two or three times as many heads per wave 84 to 89; loads past the caches take 100.  Few rows are bound by loads that wait
// for each other, position and slot, then angles, then the row (9 rows 3.8 us, 224 of 96 heads 5.6), though the row's address needs
// neither of the first.
template <class TI, class TO, int DH, bool INTER>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkNormRope a, int waves_per_row) {
    constexpr int LANES = DH / 16, HEADS = 64 / LANES;          // lanes per head, heads per wave
    const int lane = threadIdx.x & 63, l = lane % LANES, slice = lane / LANES;
    const unsigned w = blockIdx.x * 4u + (threadIdx.x >> 6);
    const int row = (int)(w / (unsigned)waves_per_row), part = (int)(w % (unsigned)waves_per_row);
    if (row >= a.rows) return;
    const odb_pages &pg = a.pages;
    const int pos = a.positions[row], slot = a.slots[row];
    // a padding row: queries become zero, nothing is stored
    const bool live = pos >= 0 && pos < a.n_pos && (!a.row_end || row < *a.row_end);
    const int page = slot >= 0 ? (int)((unsigned)slot / (unsigned)pg.page_size) : -1;
    const bool stored = live && page >= 0 && page < pg.n_pages;
    const size_t at = stored ? (size_t)page * pg.page_stride + (size_t)(slot - page * pg.page_size) * pg.pos_stride : 0;

    const HeadLane hl = head_lane<INTER>(l, a.rot);
    const int c0 = hl.c0, c1 = hl.c1;
    const bool turns = hl.turns;
    float cs[8], sn[8];
    if (turns && live) load_angles(a.table + (size_t)pos * a.rot + l * 16, cs, sn);
    const int kv = pg.n_kv_heads, total = a.heads + 2 * kv;
    const int h = part * HEADS + slice;
    if (h >= total) return;
    const bool is_q = h < a.heads, is_k = !is_q && h < a.heads + kv;
    const int head = is_q ? h : is_k ? h - a.heads : h - a.heads - kv;
    const TI *src = is_q ? (const TI *)a.q + (size_t)row * a.q_row : is_k ? (const TI *)a.k + (size_t)row * a.k_row
                                                                          : (const TI *)a.v + (size_t)row * a.v_row;
    src += (size_t)head * DH;
    f32x8 x = load8(src + c0), y = load8(src + c1);
    if (is_q || is_k) {
        const float *gain = is_q ? a.q_gain : a.k_gain;
        if (gain) norm_head<DH>(x, y, gain, a.eps, c0, c1);
        if (turns) turn_head<INTER>(x, y, cs, sn);
    }
    TO *dst;
    if (is_q) {
        dst = (TO *)a.q_out + (size_t)row * a.q_out_row + (size_t)head * DH;
        if (!live) x = y = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    } else {
        if (!stored) return;
        dst = (TO *)(is_k ? pg.k : pg.v) + at + (size_t)head * pg.head_stride;
    }
    if (a.status) {                                             // (of the model's forward, whose type is binary16)
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
    store8(dst + c0, x);
    store8(dst + c1, y);
}

template <class TI, class TO, int DH>
static void launch_rope_dim(const QkNormRope &a, hipStream_t s) {
    const int wpr = qk_waves_per_row(a.heads, a.pages);
    const unsigned grid = (unsigned)(((long long)a.rows * wpr + 3) / 4);
    if (a.interleaved) qk_norm_rope_kernel<TI, TO, DH, true><<<dim3(grid), 256, 0, s>>>(a, wpr);
    else qk_norm_rope_kernel<TI, TO, DH, false><<<dim3(grid), 256, 0, s>>>(a, wpr);
}

template <class TI, class TO>
static void launch_rope_types(const QkNormRope &a, hipStream_t s) {
    switch (a.pages.head_dim) {
    case 64: return launch_rope_dim<TI, TO, 64>(a, s);
    case 128: return launch_rope_dim<TI, TO, 128>(a, s);
    default: return launch_rope_dim<TI, TO, 256>(a, s);
    }
}

void launch_qk_norm_rope(const QkNormRope &a, hipStream_t s) {
    if (a.rows < 1) return;
    if (a.pages.dtype == ODB_F16) {
        if (a.in_dtype == ODB_F32) launch_rope_types<float, _Float16>(a, s);
        else launch_rope_types<_Float16, _Float16>(a, s);
    } else {
        if (a.in_dtype == ODB_F32) launch_rope_types<float, __bf16>(a, s);
        else launch_rope_types<__bf16, __bf16>(a, s);
    }
}

}  // namespace odb
