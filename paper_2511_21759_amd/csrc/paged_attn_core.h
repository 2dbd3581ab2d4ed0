// Device code that the kernels of attention over paged K/V share, whatever the pages hold: which keys a row sees, which work a workgroup
// has, and pieces of the loops.
#pragma once
#include "launch.h"
#include "paged.h"

namespace odb {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T> struct Num;
template <> struct Num<_Float16> {
    static constexpr uint32_t kOnes = 0x3c003c00u, kExp = 0x7c00u;
    static __device__ __forceinline__ f32x4 mfma(const frag_t &x, const frag_t &y, f32x4 c) { return mfma16(x, y, c); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2)); }
    static __device__ __forceinline__ float value(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (u16)b); }
};
template <> struct Num<__bf16> {
    static constexpr uint32_t kOnes = 0x3f803f80u, kExp = 0x7f80u;
    static __device__ __forceinline__ f32x4 mfma(const frag_t &x, const frag_t &y, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2)); }
    static __device__ __forceinline__ float value(uint32_t b) { return bf2f((u16)b); }
};

// Probabilities are exp2(score - reference) with the reference kShift below the maximum that it was taken from: the binary16
// form of a probability then keeps all its bits down to 2^-22 of the largest one.  The reference is raised when a score
// passes it by more than kRaise, so a probability is at most 2^kRaise, which binary16 holds.
// As long as a row has seen no key its reference is kNone, lower than any score: sums that are nought then stay so.
constexpr float kShift = 8.0f, kRaise = 15.0f, kNone = -3.402823466e38f;
struct Reference { float at = kNone, limit = kNone; };          // in units of log2; limit: the score beyond which it is raised

// A reference has 24 bits, so far from zero its own rounding moves the probabilities by a power of two: below kBeyond by up to 2^16 down and,
// where it would be more than 2^7 up, down instead, which keeps that of the largest score inside binary16 and not zero.  A row whose reference
// lies beyond gets no number for its sum (the one whose bits are all ones: others take a register).
constexpr float kBeyond = 1 << 29;
__device__ __forceinline__ float checked_sum(float at, float sum) { return fabsf(at) >= kBeyond && at != kNone ? __builtin_bit_cast(float, -1) : sum; }

// ---- which keys -------------------------------------------------------------------------------------------------------

constexpr int kFar = 1 << 30;                       // lengths, windows and positions are at most this
struct Request { int m, len, first, row0; };       // rows, visible positions, position of the first row, its index

// Lengths, tables and plans are read through the scalar cache where the index is the same for a whole wave: such a load does not
// queue behind the loads of K and V.  (No kernel writes what it reads so.)
typedef const __attribute__((address_space(4))) int32_t *scalar_ptr;
__device__ __forceinline__ int ld_scalar(const int32_t *p, int i) { return ((scalar_ptr)(uintptr_t)p)[i]; }

__device__ __forceinline__ Request request_of(const PagedAttn &a, int r) {
    Request q;
    int lo = r * a.rows_per_request, hi = lo + a.rows_per_request;
    if (a.cu_rows) { lo = ld_scalar(a.cu_rows, r); hi = ld_scalar(a.cu_rows, r + 1); }
    lo = min(max(lo, 0), a.rows);
    hi = min(max(hi, 0), a.rows);
    q.row0 = lo;
    q.m = max(hi - lo, 0);
    const long long most = (long long)a.columns << a.page_shift;
    q.len = (int)min((long long)max(ld_scalar(a.kv_len, r), 0), most);
    q.first = a.first ? min(max(ld_scalar(a.first, r), -kFar), kFar) : q.len - q.m;      // (differences of positions stay inside 32 bits)
    return q;
}

// The blocks of 2^SHIFT keys that rows at positions pmin .. pmax may see: `head` blocks from key 0 (the first positions that stay
// visible), then those from block `from` on; `count` in all.
struct Blocks { int head, from, count; };
template <int SHIFT = 5>
__device__ __forceinline__ Blocks blocks_of(const PagedAttn &a, int len, int pmin, int pmax) {
    int lo = 0, hi = len;
    if (a.causal) hi = min(hi, pmax + 1);
    if (a.window) {
        lo = max(0, pmin - a.window + 1);
        hi = min(hi, pmax > kFar - a.window ? kFar : pmax + a.window);
    }
    Blocks b;
    constexpr int M = (1 << SHIFT) - 1;
    int last = hi > lo ? (hi + M) >> SHIFT : 0;
    b.from = hi > lo ? lo >> SHIFT : 0;
    const int stay = min(a.window ? a.sinks : 0, a.causal ? min(len, pmax + 1) : len);
    b.head = stay > 0 ? (stay + M) >> SHIFT : 0;
    if (last > b.from) {
        last = max(last, b.head);                                // (positions that stay may reach beyond the window)
        b.head = min(b.head, b.from);
        b.count = b.head + last - b.from;
    } else {
        b.from = b.head;
        b.count = b.head;
    }
    return b;
}
template <int SHIFT = 5>
__device__ __forceinline__ int block_key(const Blocks &b, int i) { return (i < b.head ? i : b.from + i - b.head) << SHIFT; }

// positions of a tile's first and last row
__device__ __forceinline__ void tile_span(const Request &q, int group, int tile, int tile_rows, int &pmin, int &pmax) {
    pmin = q.first + tile * tile_rows / group;
    pmax = q.first + min(((tile + 1) * tile_rows - 1) / group, q.m - 1);
}

// ---- which work: every workgroup works it out for itself from the lengths ---------------------------------------------

constexpr int NW = 4;                    // waves of a workgroup
constexpr int kLookAtAll = 512;          // requests

struct Place { Request q; int r; long long at, total; };

__device__ __forceinline__ long long uniform(long long x) {
    return (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) |
                       (unsigned)__builtin_amdgcn_readfirstlane((int)x));
}

__device__ __forceinline__ int tiles_of(const PagedAttn &a, const Request &q, int tile_rows) {
    return (int)(((long long)q.m * a.group + tile_rows - 1) / tile_rows);
}
// blocks of keys that a request's rows see together (one where they see none, so that their zeros are written)
template <int SHIFT = 5>
__device__ __forceinline__ int request_blocks(const PagedAttn &a, const Request &q) {
    return max(1, blocks_of<SHIFT>(a, q.len, q.first, q.first + q.m - 1).count);
}
// A pair of request and row tile stands in the list with kPairCost places in front of those of its blocks: its queries, its first
// loads and its sums at the end take about as long as that many blocks (64 single tokens of 17 to 16384 positions: 97 us with 6,
// 98 with 8, 103 with 16, 107 without).
constexpr int kPairCost = 6;

// The requests' weights - row tiles, times blocks where keys are split - lie behind each other; finds the request that holds
// item pick(total) and the item's offset inside it.  False if there is none.  Up to 64 requests every wave does it alone.
// LONGEST: of up to 64 requests that are given out by whole tiles, those with the most positions lie first.
template <int SHIFT = 5, int COST = kPairCost, bool LONGEST = false, class Pick>
__device__ __forceinline__ bool find_place(const PagedAttn &a, int tile_rows, bool need_total, Pick pick, Place &p) {
    const int lane = threadIdx.x & 63;
    const bool by_blocks = a.split && COST >= 0;
    auto weigh = [&](const Request &q) -> long long {
        const int tiles = tiles_of(a, q, tile_rows);
        return by_blocks && tiles ? (long long)tiles * (request_blocks<SHIFT>(a, q) + COST) : tiles;
    };
    auto scan64 = [&](long long v) -> long long {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const long long up = __shfl_up(v, o);
            if (lane >= o) v += up;
        }
        return v;
    };
    if (a.n <= 64) {
        Request q{0, 0, 0, 0};
        if (lane < a.n) q = request_of(a, lane);
        long long v = weigh(q);
        int who = lane;
        if (LONGEST && !by_blocks && a.n > 1) {
            // a lane's place in the order, and back: which request is at a lane's place
            int before = 0;
            for (int j = 0; j < a.n; j++) {
                const int other = __builtin_amdgcn_readlane(q.len, j);
                before += (int)(other > q.len) | ((int)(other == q.len) & (int)(j < lane));
            }
            who = __builtin_amdgcn_ds_permute(4 * (lane < a.n ? before : lane), lane);
            v = __shfl((int)v, who);                                 // (tiles of one request: fewer than 2^30)
        }
        const long long end = scan64(v);
        p.total = uniform(__shfl(end, 63));
        const long long x = pick(p.total);
        const unsigned long long behind = __ballot(end > x);
        if (x >= p.total) return false;
        const int at = __builtin_amdgcn_readfirstlane(__ffsll(behind) - 1);
        p.at = x - uniform(__shfl(end - v, at));
        p.r = __builtin_amdgcn_readlane(who, at);
        p.q.m = __builtin_amdgcn_readlane(q.m, p.r);
        p.q.len = __builtin_amdgcn_readlane(q.len, p.r);
        p.q.first = __builtin_amdgcn_readlane(q.first, p.r);
        p.q.row0 = __builtin_amdgcn_readlane(q.row0, p.r);
        return true;
    }
    // Many requests, and no lengths to look at: request r's tiles are numbered from r + floor(its first row * group / tile_rows) on, which
    // leaves room for one that is not full in each, so the first rows alone, 64 requests at a time, tell whose tile it is.  Numbers that
    // no tile has lie between the others, every second one perhaps; workgroups take the numbers out of order, or those with nothing to
    // do fall on the same CUs.  Looking at all requests / this way: 4096 single tokens of 100 positions 956 / 504 us, 3000 x 3 rows of
    // 200 950 / 634, 1000 x 1 of 300 264 / 236, 300 x 4 of 900 201 / 208 (in order 301).
    if (!need_total && a.n > kLookAtAll) {
        int x = (int)pick(0), r = 0;
        if (!a.cu_rows) {
            const int per = (a.rows_per_request * a.group + tile_rows - 1) / tile_rows;
            r = x / per;
            x -= r * per;
            if (r >= a.n) return false;
        } else {
            x = (int)((long long)x * a.stride % a.items);
            auto start = [&](int i, int row) { return i + (int)((long long)min(max(row, 0), a.rows) * a.group / tile_rows); };
            for (int left = a.n;;) {
                const int step = (left + 63) >> 6, i = r + lane * step;
                const int c = __popcll(__ballot(i < r + left && start(i, a.cu_rows[min(i, a.n - 1)]) <= x));
                if (c == 0) return false;
                r += (c - 1) * step;
                if (step == 1) break;
                left = min(step, left - (c - 1) * step);
            }
            x -= start(r, ld_scalar(a.cu_rows, r));
        }
        p.r = r;
        p.at = x;
        p.q = request_of(a, r);
        return x >= 0 && x < tiles_of(a, p.q, tile_rows);
    }
    __shared__ long long sums[NW], found_at;
    __shared__ int found;
    const int t = threadIdx.x, wave = t >> 6;
    if (t == 0) found = -1;
    p.total = 0;
    if (need_total) {
        long long v = 0;
        for (int r = t; r < a.n; r += 64 * NW) v += weigh(request_of(a, r));
        v = scan64(v);
        if (lane == 63) sums[wave] = v;
        __syncthreads();
        v = 0;
        for (int w = 0; w < NW; w++) v += sums[w];
        p.total = uniform(v);
        __syncthreads();
        if (pick(p.total) >= p.total) return false;
    }
    const long long x = pick(p.total);
    long long carry = 0;
    for (int r0 = 0; r0 < a.n && carry <= x; r0 += 64 * NW) {
        const int r = r0 + t;
        const long long v = r < a.n ? weigh(request_of(a, r)) : 0, end0 = scan64(v);
        if (lane == 63) sums[wave] = end0;
        __syncthreads();
        long long end = carry + end0;
        for (int w = 0; w < NW; w++) {
            if (w < wave) end += sums[w];
            carry += sums[w];
        }
        if (x < end && x >= end - v) { found = r; found_at = x - (end - v); }
        __syncthreads();
    }
    p.r = __builtin_amdgcn_readfirstlane(found);
    if (p.r < 0) return false;
    p.at = uniform(found_at);
    p.q = request_of(a, p.r);
    return true;
}

__device__ __forceinline__ void store_out8(const PagedAttn &a, int row, int head, int dim, int c, const uint4 &v) {
    if (a.out_mt > 0) {
        const int kk = head * dim + c;
        u16 *p = (u16 *)a.out + ((size_t)(kk >> 5) * a.out_mt + (row >> 4)) * kTileElems + tile_elem(row & 15, kk & 31);
        *reinterpret_cast<uint4 *>(p) = v;
    } else {
        *reinterpret_cast<uint4 *>((u16 *)a.out + (size_t)row * a.out_row + (size_t)head * dim + c) = v;
    }
}

__device__ __forceinline__ void store_out4(const PagedAttn &a, int row, int head, int dim, int c, const uint2 &v) {
    if (a.out_mt > 0) {
        const int kk = head * dim + c;
        u16 *p = (u16 *)a.out + ((size_t)(kk >> 5) * a.out_mt + (row >> 4)) * kTileElems + tile_elem(row & 15, kk & 31);
        *reinterpret_cast<uint2 *>(p) = v;
    } else {
        *reinterpret_cast<uint2 *>((u16 *)a.out + (size_t)row * a.out_row + (size_t)head * dim + c) = v;
    }
}

// ---- pieces of the loops ----------------------------------------------------------------------------------------------

// Probabilities of 32 keys for NT row tiles from their scores z (keys that are not seen: -infinity), as the operand of the product
// with V; the reference is raised, and sums and O rescaled, where a score passes it by too much.  It is common to the four lanes of
// a row and only has to keep exp2 in range, so after the first blocks that is rare, and the common path has no exchange of lanes.
template <class T, int CT, int NT>
__device__ __forceinline__ void probabilities(f32x4 (*z)[2], float sc, Reference *ref, f32x4 *lsum, f32x4 (*o)[CT], frag_t *pf) {
    float top[NT];
    int over = 0;
#pragma unroll
    for (int t = 0; t < NT; t++) {
        top[t] = -INFINITY;
#pragma unroll
        for (int s = 0; s < 2; s++)
#pragma unroll
            for (int e = 0; e < 4; e++) top[t] = fmaxf(top[t], z[t][s][e]);
        over |= (int)(top[t] > ref[t].limit);
    }
    if (__any(over))                            // (one branch for all row tiles)
#pragma unroll
        for (int t = 0; t < NT; t++) {
            float m = fmaxf(top[t], __shfl_xor(top[t], 16));
            m = fmaxf(m, __shfl_xor(m, 32));
            float up = fmaxf(ref[t].at, m * sc - kShift);
            up += __builtin_fmaf(m, sc, -up) > kRaise ? fabsf(up) * 0x1.8p-24f : 0.f;      // (rounded down by more than 7: the next number)
            const float f = __builtin_amdgcn_exp2f(ref[t].at - up);
            lsum[t] *= f;
#pragma unroll
            for (int c = 0; c < CT; c++) o[t][c] *= f;
            ref[t].at = up;
            ref[t].limit = (up + kRaise) / sc;
            ref[t].limit -= fabsf(ref[t].limit) * 0x1p-22f;                               // (its own roundings)
        }
    // Probabilities are rounded to the type of V for the matrix cores; the sum that divides them at the end is that of the
    // rounded ones, so what equal rounding errors have in common drops out.
#pragma unroll
    for (int t = 0; t < NT; t++) {
        float p[2][4];
#pragma unroll
        for (int s = 0; s < 2; s++)
#pragma unroll
            for (int e = 0; e < 4; e++) p[s][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[t][s][e], sc, -ref[t].at));
        pf[t] = frag_t{{Num<T>::pack(p[0][0], p[0][1]), Num<T>::pack(p[0][2], p[0][3]), Num<T>::pack(p[1][0], p[1][1]), Num<T>::pack(p[1][2], p[1][3])}};
    }
}

// Values of V that are infinite or no number must not reach a row that does not see their key, not even times zero.  In blocks
// that not all rows see in full, keys that no row sees (whatever lies behind the last position, or in no page of the pool) become
// zero as they are loaded, and the others are looked at; where there are such values, they are added one by one to the rows that
// see them (add_odd) and the product has zeros in their place (clear_odd).
template <class T>
__device__ __forceinline__ int has_odd(const frag_t &v) {
    int odd = 0;
#pragma unroll
    for (int w = 0; w < 4; w++)
        odd |= (int)((v.w[w] & Num<T>::kExp) == Num<T>::kExp) | (int)(((v.w[w] >> 16) & Num<T>::kExp) == Num<T>::kExp);
    return odd;
}
template <class T>
__device__ __forceinline__ void clear_odd(frag_t &v) {
#pragma unroll
    for (int w = 0; w < 4; w++) {
        if ((v.w[w] & Num<T>::kExp) == Num<T>::kExp) v.w[w] &= 0xffff0000u;
        if (((v.w[w] >> 16) & Num<T>::kExp) == Num<T>::kExp) v.w[w] &= 0xffffu;
    }
}

// Where the 16-byte piece `c` of key row `key` lies in a block of V: pieces are exchanged inside 256 bytes so that the
// 8-byte reads of eight neighbouring keys, 32 bytes of each, fall on all 64 banks.
// PAIRS: written by lanes that hold two pieces beside each other each, every second piece at once: those of the upper half of 256 bytes, or of
// every second key of 128, are the other way round (eight lanes then write to all banks; a store of 1 KiB takes 13 clocks and not 16).
template <int DH>
__host__ __device__ constexpr int pair_turn(int key, int c) { return DH == 64 ? key & 1 : DH == 128 ? (c >> 3) & 1 : ((c >> 3) ^ (c >> 4)) & 1; }
template <int DH, bool PAIRS = false>
__host__ __device__ constexpr int v_piece(int key, int c) {
    return key * (DH / 8) + (c ^ (DH == 64 ? ((key >> 1) & 3) << 1 : (key & 7) << 1) ^ (PAIRS ? pair_turn<DH>(key, c) : 0));
}

template <class T, int DH, bool PAIRS = false, class See>
__device__ __forceinline__ void add_odd(const unsigned char *v_block, int lane, const frag_t &pf, See see, f32x4 (&o)[DH / 16]) {
    int dl = lane;                            // (hidden from the compiler, which else keeps this part's addresses in registers)
    asm volatile("" : "+v"(dl));
    for (int key = 0; key < 32; key++) {
        const int src = (dl & 15) + 16 * ((key >> 2) & 3);       // the lane that holds the row's probability of this key
        const uint32_t w0 = (uint32_t)__shfl((int)pf.w[0], src), w1 = (uint32_t)__shfl((int)pf.w[1], src);
        const uint32_t w2 = (uint32_t)__shfl((int)pf.w[2], src), w3 = (uint32_t)__shfl((int)pf.w[3], src);
        const uint32_t a0 = key & 16 ? w2 : w0, a1 = key & 16 ? w3 : w1, word = key & 2 ? a1 : a0;
        const float p = Num<T>::value(key & 1 ? word >> 16 : word & 0xffffu);
        const bool seen = see(key);
#pragma unroll
        for (int c = 0; c < DH / 16; c++)
#pragma unroll
            for (int d = 0; d < 4; d++) {
                const int ch = c * 16 + 4 * (dl >> 4) + d;
                const uint32_t v = *reinterpret_cast<const u16 *>(v_block + 16 * v_piece<DH, PAIRS>(key, ch >> 3) + 2 * (ch & 7));
                if ((int)seen & (int)((v & Num<T>::kExp) == Num<T>::kExp)) o[c][d] += p * Num<T>::value(v);
            }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// V^T of a 32-key block in operand order: a lane's channel is (lane & 15) of tile c, its keys 4 (lane >> 4) + 0..3 of each 16
__device__ __forceinline__ frag_t v_operand_at(const unsigned char *p0, int keys16) {
    typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
    const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p0));
    const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p0 + keys16)));
    return frag_t{{lo.x, lo.y, hi.x, hi.y}};
}
template <int DH, bool PAIRS = false>
__device__ __forceinline__ unsigned v_lane(int lane, int c) {             // bytes
    const int li = lane & 15, row = 4 * (lane >> 4) + (li >> 2), at = 2 * c + ((li >> 1) & 1);
    return 16 * v_piece<DH, PAIRS>(row, at) + 8 * (li & 1);
}
template <int DH>
__device__ __forceinline__ frag_t v_operand(const unsigned char *v_block, int lane, int c) {
    return v_operand_at(v_block + v_lane<DH>(lane, c), 16 * DH * 2);
}

// Load of 16 bytes at a scalar address plus a lane's offset.  STREAM: data that is read once, past the caches' replacement.
template <bool STREAM>
__device__ __forceinline__ frag_t ld_at(const u16 *uniform, unsigned lane_bytes) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    typedef const __attribute__((address_space(1))) char *global_bytes;
    typedef const __attribute__((address_space(1))) u32x4 *global_ptr;
    global_bytes base = (global_bytes)(uintptr_t)uniform;
    asm("" : "+s"(base));                                         // (keeps the sum of a scalar base and a 32-bit offset apart)
    const global_ptr p = (global_ptr)(base + lane_bytes);
    return __builtin_bit_cast(frag_t, STREAM ? __builtin_nontemporal_load(p) : *p);
}

// The same with the base in a buffer's description and one more scalar offset: no sums of addresses beside the load itself.  (The
// offsets of a lane and of the wave together are below 2^30, and the description has no other bound.)
typedef __amdgpu_buffer_rsrc_t rsrc_t;
__device__ __forceinline__ rsrc_t rsrc_of(const u16 *base) {
    return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, 0x7fffffff, 0x00027000);
}
__device__ __forceinline__ frag_t ld_buffer(rsrc_t r, unsigned lane_bytes, unsigned wave_bytes) {
    return __builtin_bit_cast(frag_t, __builtin_amdgcn_raw_buffer_load_b128(r, (int)lane_bytes, (int)wave_bytes, 0));
}

// the keys that a row at position p sees: lo .. hi - 1 and 0 .. stay - 1
struct Sight { int lo, hi, stay; };
__device__ __forceinline__ Sight sight_of(const PagedAttn &a, int len, int pos) {
    const int p = min(pos, kFar - 1), end = a.causal ? min(len, p + 1) : len;
    return Sight{a.window ? p - a.window + 1 : 0, a.window ? min(end, p + a.window) : end, a.window ? min(a.sinks, end) : 0};
}
// (no branches: bitwise operators)
__device__ __forceinline__ bool sees(const Sight &s, int key, int page) {
    return ((int)(page >= 0) & (((int)(key >= s.lo) & (int)(key < s.hi)) | (int)(key < s.stay))) != 0;
}
// scores of a 32-key block that a row does not see become -infinity
__device__ __forceinline__ void hide_unseen(f32x4 (&z)[2], const Sight &sight, int key0, int g, int page0, int page1) {
    int key = key0 + 4 * g;
    asm volatile("" : "+v"(key));             // (hidden from the compiler, which else computes the eight keys outside this rare part)
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
        for (int e = 0; e < 4; e++) z[s][e] = sees(sight, key + s * 16 + e, s ? page1 : page0) ? z[s][e] : -INFINITY;
}
// is every one of n keys from key0 on visible to every row at positions pmin .. pmax?
__device__ __forceinline__ bool all_seen(const PagedAttn &a, int len, int key0, int n, int pmin, int pmax) {
    const int last = key0 + n - 1;
    return last < len && (!a.causal || last <= pmin) && (!a.window || last < a.sinks || (key0 > pmax - a.window && last - pmin < a.window));
}

// Keys that some, or that all rows at positions pmin .. pmax see, as a Sight: is any, or every one, of n keys from key0 on among them?
__device__ __forceinline__ Sight sight_of_some(const PagedAttn &a, int len, int pmin, int pmax) {
    const Sight s = sight_of(a, len, pmin), e = sight_of(a, len, pmax);
    return Sight{s.lo, e.hi, e.stay};
}
__device__ __forceinline__ Sight sight_of_all(const PagedAttn &a, int len, int pmin, int pmax) {
    const Sight s = sight_of(a, len, pmin), e = sight_of(a, len, pmax);
    return Sight{e.lo, s.hi, s.stay};
}
__device__ __forceinline__ bool any_of(const Sight &s, int key0, int n) { return (key0 < s.hi && key0 + n > s.lo) || key0 < s.stay; }
__device__ __forceinline__ bool all_of(const Sight &s, int key0, int n) { return (key0 >= s.lo && key0 + n <= s.hi) || key0 + n <= s.stay; }

// ---- what the few- and many-row kernels have in common with the kernels that plan and join -------------------------------

constexpr int kRowsPlace = 256;          // `where` holds parts * kRowsPlace + row of the tile
constexpr int kTileCost = 3, kLeastStages = 4, kPlanTiles = 512;       // many rows: places of a tile beside its stages, stages of a piece at least

// Many rows: 16-row tiles of a wave, rows of a workgroup, keys of a stage
template <int DH>
struct RowsShape {
    static constexpr int NT = DH == 256 ? 1 : 2, TILE_ROWS = 64 * NT, SHIFT = DH == 256 ? 5 : 6, SK = 1 << SHIFT;
};
// Where piece c of a key of K lies: the 16 keys that one operand load reads fall on different banks.
template <int DH, bool PAIRS = false>
__host__ __device__ constexpr int k_piece(int key, int c) {
    return key * (DH / 8) + (c ^ (DH == 64 ? (key >> 1) & 7 : key & 15) ^ (PAIRS ? pair_turn<DH>(key, c) : 0));
}

}  // namespace
}  // namespace odb
