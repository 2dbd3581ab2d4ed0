// Operators around a paged K/V cache: page tables and slot maps, the table of rotary angles, and the pass that norms and
// turns queries and keys and stores keys and values in their pages.  Attention over the pages is in paged_attn.hip.
#include "paged.h"

namespace odb {

// ---- page tables ----------------------------------------------------------------------------------------------------

// Sums of these kernels saturate at 2^30 (more than any pool or row buffer has), so that lengths of any size cannot wrap them.
constexpr unsigned kSat = 1u << 30;
__device__ __forceinline__ unsigned sat_add(unsigned a, unsigned b) { return min(a + b, kSat); }

// Inclusive scan of one value per thread over the 256 threads of a workgroup, on top of `carry`; `carry` becomes the total.
__device__ __forceinline__ unsigned scan256(unsigned v, unsigned &carry, unsigned *wave_sums) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned up = __shfl_up(v, o);
        if (lane >= o) v = sat_add(v, up);
    }
    if (lane == 63) wave_sums[wave] = v;
    __syncthreads();
    unsigned before = carry;
    for (int w = 0; w < 4; w++) {
        if (w < wave) before = sat_add(before, wave_sums[w]);
        carry = sat_add(carry, wave_sums[w]);
    }
    __syncthreads();
    return sat_add(before, v);
}

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
__device__ __forceinline__ PageNeed page_need(const PageTables &a, int r) {
    PageNeed p;
    const long long most = (long long)a.columns << a.page_shift;
    const int top = (int)min(most, 0x7fffffffll), mask = (1 << a.page_shift) - 1;
    p.held = min(max(a.held[r], 0), top);
    p.wanted = a.wanted[r];
    p.fits = p.wanted >= 0 && p.wanted <= top;
    p.had = ((unsigned)p.held + mask) >> a.page_shift;
    p.need = p.fits ? ((unsigned)p.wanted + mask) >> a.page_shift : p.had;
    return p;
}

// One launch, no exchange between workgroups: each of them computes the three running sums over the requests (pages taken,
// pages given back, rows) for itself - at most 4096 requests, so at most 16 per thread - and then does its share of
// the items: rows, pages given back, pages taken.  What one workgroup writes no other reads: entries behind a request's held
// pages are not looked up in the table but derived from the stack, and the stack's new top from the tables of those that gave back.
// A second call with the same inputs therefore writes the same values again. 
__global__ __launch_bounds__(256) void page_tables_kernel(PageTables a) {
    extern __shared__ unsigned lds[];
    __shared__ unsigned wave_sums[4], granted_top[4];
    unsigned *taken = lds, *given = lds + a.n, *rows = lds + 2 * a.n;
    const int t = threadIdx.x;
    unsigned c_take = 0, c_give = 0, c_rows = 0;
    for (int r0 = 0; r0 < a.n; r0 += 256) {
        const int r = r0 + t;
        unsigned take = 0, give = 0, count = 0;
        if (r < a.n) {
            const PageNeed p = page_need(a, r);
            take = p.need > p.had ? p.need - p.had : 0;
            give = p.had > p.need ? p.had - p.need : 0;
            const int c = a.count ? a.count[r] : p.fits ? p.wanted - p.held : 0;
            count = min((unsigned)max(c, 0), (unsigned)a.rows_cap);
        }
        const unsigned st = scan256(take, c_take, wave_sums), sg = scan256(give, c_give, wave_sums), sr = scan256(count, c_rows, wave_sums);
        if (r < a.n) { taken[r] = st; given[r] = sg; rows[r] = sr; }
    }
    __syncthreads();
    const unsigned n_free = (unsigned)min(max(*a.n_free, 0), a.n_pages), have = n_free + c_give;
    const unsigned n_rows = min(c_rows, (unsigned)a.rows_cap);

    // The page that takes number i off the stack: those given back in this call lie on top.
    auto taken_page = [&](unsigned i) -> int {
        const unsigned at = have - 1 - i;
        if (at < n_free) return a.free_pages[at];
        const unsigned g = at - n_free;
        const int r = owner(given, a.n, g);
        const unsigned mine = g - (r ? given[r - 1] : 0);
        return a.tables[(size_t)r * a.columns + page_need(a, r).need + mine];
    };
    auto granted = [&](int r, const PageNeed &p) { return p.fits && (p.need <= p.had || taken[r] <= have); };

    // rows: position and slot
    const unsigned step = gridDim.x * 256, first = blockIdx.x * 256 + t;
    for (unsigned i = first; i < n_rows; i += step) {
        const int r = owner(rows, a.n, i);
        const PageNeed p = page_need(a, r);
        const bool ok = granted(r, p);
        const int len = ok ? p.wanted : p.held;
        const long long pos = (long long)(a.first ? a.first[r] : p.held) + (i - (r ? rows[r - 1] : 0));
        int slot = -1;
        if (pos >= 0 && pos < len) {
            const unsigned j = (unsigned)pos >> a.page_shift;
            const int page = j < p.had ? a.tables[(size_t)r * a.columns + j] : taken_page((r ? taken[r - 1] : 0) + (j - p.had));
            if (page >= 0 && page < a.n_pages) slot = (page << a.page_shift) + ((int)pos & ((1 << a.page_shift) - 1));
        }
        a.slots[i] = slot;
        a.positions[i] = (int)min(pos, 0x7fffffffll);
    }
    // pages given back go on the stack
    for (unsigned g = first; g < c_give; g += step) {
        const int r = owner(given, a.n, g);
        const unsigned mine = g - (r ? given[r - 1] : 0);
        if (n_free + g < (unsigned)a.n_pages) a.free_pages[n_free + g] = a.tables[(size_t)r * a.columns + page_need(a, r).need + mine];
    }
    // pages taken go into the tables (those of requests behind the first refused one are not granted: the sums only rise)
    for (unsigned i = first; i < min(c_take, have); i += step) {
        const int r = owner(taken, a.n, i);
        if (taken[r] > have) break;
        const unsigned mine = i - (r ? taken[r - 1] : 0);
        a.tables[(size_t)r * a.columns + page_need(a, r).had + mine] = taken_page(i);
    }
    if (blockIdx.x) return;
    unsigned refused = 0, most = 0;
    for (int r = t; r < a.n; r += 256) {
        const PageNeed p = page_need(a, r);
        const bool ok = granted(r, p);
        a.len[r] = ok ? p.wanted : p.held;
        a.cu_rows[r + 1] = (int)min(rows[r], (unsigned)a.rows_cap);
        if (!ok) refused++;
        else if (p.need > p.had) most = max(most, taken[r]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        refused += __shfl_xor(refused, o);
        most = max(most, __shfl_xor(most, o));
    }
    if ((t & 63) == 0) { wave_sums[t >> 6] = refused; granted_top[t >> 6] = most; }
    __syncthreads();
    if (t == 0) {
        refused = wave_sums[0] + wave_sums[1] + wave_sums[2] + wave_sums[3];
        most = max(max(granted_top[0], granted_top[1]), max(granted_top[2], granted_top[3]));
        a.cu_rows[0] = 0;
        a.state[0] = (int)min(have - most, (unsigned)a.n_pages);
        a.state[1] = (int)most;
        a.state[2] = (int)c_give;
        a.state[3] = (int)refused;
    }
}

void launch_page_tables(const PageTables &a, hipStream_t s) {
    // a workgroup per 256 rows up to two per CU; more would only repeat the sums
    const int wanted = a.rows_cap / 256 + 1;
    const int grid = wanted < 512 ? wanted : 512;
    page_tables_kernel<<<dim3(grid), 256, (size_t)a.n * 12, s>>>(a);
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
// position of 2^22 has the same error as the first.  One pair per thread, pairs of a position beside each other: stores of 512
// contiguous bytes per wave.
__global__ __launch_bounds__(256) void rope_angles_kernel(RopeTable a) {
    const unsigned i = blockIdx.x * 256u + threadIdx.x, pos = i / (unsigned)a.pairs, j = i - pos * a.pairs;
    if (pos >= (unsigned)a.n_pos) return;
    const double p = (double)pos, hi = a.hi[j], r = fma(p, hi, -rint(p * hi)) + p * a.lo[j];
    double c, s;
    turn_sincos(r - rint(r), c, s);
    *reinterpret_cast<float2 *>(a.table + 2 * (size_t)i) = float2{(float)(c * a.magnitude), (float)(s * a.magnitude)};
}

void launch_rope_angles(const RopeTable &a, hipStream_t s) {
    const long long total = (long long)a.n_pos * a.pairs;          // at most 2^22 * 2^7
    rope_angles_kernel<<<dim3((unsigned)((total + 255) / 256)), 256, 0, s>>>(a);
}

// ---- norms and rotation of queries and keys, K/V to their pages ------------------------------------------------------

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
template <class T> struct Vec;
template <> struct Vec<_Float16> { typedef f16x8 v8; };
template <> struct Vec<__bf16> { typedef bf16x8 v8; };
template <> struct Vec<float> { typedef f32x8 v8; };

template <class T>
__device__ __forceinline__ f32x8 load8(const T *p) {
    return __builtin_convertvector(*reinterpret_cast<const typename Vec<T>::v8 *>(p), f32x8);
}
// one rounding, to nearest even, of a value computed in 32 bits; beyond the type's range it becomes infinite
template <class T>
__device__ __forceinline__ void store8(T *p, f32x8 x) {
    *reinterpret_cast<typename Vec<T>::v8 *>(p) = __builtin_convertvector(x, typename Vec<T>::v8);
}

// A head is held by DH / 16 lanes with 16 channels each: in the half layout channel pair (j, j + rot / 2) sits in one lane as
// elements of its first and its second eight, in the interleaved layout (2j, 2j + 1) inside each eight.  Lanes behind the rotated
// part hold two neighbouring eights that pass through.  A wave does `per` groups of heads of one row, so the row's cosines and
// sines are loaded once into registers; its groups of lanes do different heads.  Bound by the memory: every element is read and written once.
template <class TI, class TO, int DH, bool INTER>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkNormRope a, int waves_per_row) {
    constexpr int LANES = DH / 16, HEADS = 64 / LANES;          // lanes per head, heads per wave
    const int lane = threadIdx.x & 63, l = lane % LANES, slice = lane / LANES;
    const unsigned w = blockIdx.x * 4u + (threadIdx.x >> 6);
    const int row = (int)(w / (unsigned)waves_per_row), part = (int)(w % (unsigned)waves_per_row);
    if (row >= a.rows) return;
    const odb_pages &pg = a.pages;
    const int pos = a.positions[row], slot = a.slots[row];
    const bool live = pos >= 0 && pos < a.n_pos;                // a padding row: queries become zero, nothing is stored
    const int page = slot >= 0 ? (int)((unsigned)slot / (unsigned)pg.page_size) : -1;
    const bool stored = live && page >= 0 && page < pg.n_pages;
    const size_t at = stored ? (size_t)page * pg.page_stride + (size_t)(slot - page * pg.page_size) * pg.pos_stride : 0;

    const int half = a.rot / 2, turning = a.rot / 16;           // lanes of a head that turn
    const bool turns = l < turning;
    int c0, c1;                                                 // first channels of the lane's two eights
    if (INTER) { c0 = l * 16; c1 = c0 + 8; }
    else if (turns) { c0 = l * 8; c1 = c0 + half; }
    else { c0 = a.rot + (l - turning) * 16; c1 = c0 + 8; }
    float cs[8], sn[8];
    if (turns && live) {
        const float *t = a.table + (size_t)pos * a.rot + l * 16;       // eight (cos, sin)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float4 x = *reinterpret_cast<const float4 *>(t + 4 * i);
            cs[2 * i] = x.x; sn[2 * i] = x.y; cs[2 * i + 1] = x.z; sn[2 * i + 1] = x.w;
        }
    }
    const int kv = pg.n_kv_heads, total = a.heads + 2 * kv;
    for (int h = part * HEADS + slice; h < total; h += waves_per_row * HEADS) {
        const bool is_q = h < a.heads, is_k = !is_q && h < a.heads + kv;
        const int head = is_q ? h : is_k ? h - a.heads : h - a.heads - kv;
        const TI *src = is_q ? (const TI *)a.q + (size_t)row * a.q_row : is_k ? (const TI *)a.k + (size_t)row * a.k_row
                                                                              : (const TI *)a.v + (size_t)row * a.v_row;
        src += (size_t)head * DH;
        f32x8 x = load8(src + c0), y = load8(src + c1);
        if (is_q || is_k) {
            const float *gain = is_q ? a.q_gain : a.k_gain;
            if (gain) {
                float ss = 0.f;
#pragma unroll
                for (int i = 0; i < 8; i++) ss += x[i] * x[i] + y[i] * y[i];
#pragma unroll
                for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
                const float r = 1.0f / sqrtf(ss / (float)DH + a.eps);
                const f32x8 g0 = load8(gain + c0), g1 = load8(gain + c1);
                x = x * r * g0;
                y = y * r * g1;
            }
            if (turns) {
                if (INTER) {
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const float u = x[2 * i], v = x[2 * i + 1], p = y[2 * i], q = y[2 * i + 1];
                        x[2 * i] = u * cs[i] - v * sn[i];
                        x[2 * i + 1] = v * cs[i] + u * sn[i];
                        y[2 * i] = p * cs[4 + i] - q * sn[4 + i];
                        y[2 * i + 1] = q * cs[4 + i] + p * sn[4 + i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const float u = x[i], v = y[i];
                        x[i] = u * cs[i] - v * sn[i];
                        y[i] = v * cs[i] + u * sn[i];
                    }
                }
            }
        }
        TO *dst;
        if (is_q) {
            dst = (TO *)a.q_out + (size_t)row * a.q_out_row + (size_t)head * DH;
            if (!live) x = y = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        } else {
            if (!stored) continue;
            dst = (TO *)(is_k ? pg.k : pg.v) + at + (size_t)head * pg.head_stride;
        }
        store8(dst + c0, x);
        store8(dst + c1, y);
    }
}

template <class TI, class TO, int DH>
static void launch_rope_dim(const QkNormRope &a, hipStream_t s) {
    // A wave that does all heads of its row loads the angles once; with few rows the heads are spread over more waves, up to
    // four per SIMD of the chip, which shortens the chain of loads that bounds a small call.
    const int per_wave = 64 / (DH / 16), total = a.heads + 2 * a.pages.n_kv_heads, most = (total + per_wave - 1) / per_wave;
    int wpr = 1;
    while (wpr < most && (long long)a.rows * wpr < 4096) wpr++;
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
