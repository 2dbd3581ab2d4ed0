// Attention of new rows over a paged K/V cache (odb_paged_attention).
//
// A workgroup takes a tile of R = 16 * NT query rows of one request and one K/V head - the rows of the request times the
// query heads that share the K/V head, row-major - and a part of the keys; its four waves take 32-key blocks in turn, each
// with its own running (reference, sum, O), and are merged through LDS in a fixed order.
//
//   S^T = K Q^T  (16 keys x 16 rows per MFMA): a lane holds scores of ONE row (lane & 15), keys 4 * (lane >> 4) + 0..3.
//   O^T = V^T P^T  over the 32 keys of a block: the probabilities are already where the second MFMA wants them if its key
//         order inside the block is the one that S^T left; V^T comes out of LDS through the transposing 64-bit read, which
//         hands a lane four consecutive keys of one channel from row-major [key][channel] storage.
//
// K goes from the pages straight to registers in operand order (16 bytes per lane, the 16 keys of a tile lie in one page);
// V goes through registers into a wave's own part of LDS, so waves never wait for each other inside the loop.  The loads of a
// block are issued while the block before it is worked on.
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
constexpr float kShift = 8.0f, kRaise = 15.0f;

// ---- which keys -------------------------------------------------------------------------------------------------------

constexpr int kFar = 1 << 30;                       // lengths, windows and positions are at most this
struct Request { int m, len, first, row0; };       // rows, visible positions, position of the first row, its index

__device__ __forceinline__ Request request_of(const PagedAttn &a, int r) {
    Request q;
    int lo = r, hi = r + 1;
    if (a.cu_rows) { lo = a.cu_rows[r]; hi = a.cu_rows[r + 1]; }
    lo = min(max(lo, 0), a.rows);
    hi = min(max(hi, 0), a.rows);
    q.row0 = lo;
    q.m = max(hi - lo, 0);
    const long long most = (long long)a.columns << a.page_shift;
    q.len = (int)min((long long)max(a.kv_len[r], 0), most);
    q.first = a.first ? min(max(a.first[r], -kFar), kFar) : q.len - q.m;      // (differences of positions stay inside 32 bits)
    return q;
}

// The 32-key blocks that rows at positions pmin .. pmax may see: `head` blocks from key 0 (the first positions that stay
// visible), then those from block `from` on; `count` in all.
struct Blocks { int head, from, count; };
__device__ __forceinline__ Blocks blocks_of(const PagedAttn &a, int len, int pmin, int pmax) {
    int lo = 0, hi = len;
    if (a.causal) hi = min(hi, pmax + 1);
    if (a.window) {
        lo = max(0, pmin - a.window + 1);
        hi = min(hi, pmax < 0 ? 0 : pmax > kFar - a.window ? kFar : pmax + a.window);
    }
    Blocks b;
    const int last = hi > lo ? (hi + 31) >> 5 : 0;
    b.from = hi > lo ? lo >> 5 : 0;
    const int stay = min(a.window ? a.sinks : 0, a.causal ? min(len, pmax + 1) : len);
    b.head = stay > 0 ? (stay + 31) >> 5 : 0;
    if (last > b.from) {
        b.head = min(b.head, b.from);
        b.count = b.head + last - b.from;
    } else {
        b.from = b.head;
        b.count = b.head;
    }
    return b;
}
__device__ __forceinline__ int block_key(const Blocks &b, int i) { return (i < b.head ? i : b.from + i - b.head) * 32; }

// positions of a tile's first and last row
__device__ __forceinline__ void tile_span(const Request &q, int group, int tile, int tile_rows, int &pmin, int &pmax) {
    pmin = q.first + tile * tile_rows / group;
    pmax = q.first + min(((tile + 1) * tile_rows - 1) / group, q.m - 1);
}

// ---- which work: every workgroup works it out for itself from the lengths ---------------------------------------------

__device__ __forceinline__ int scan256(int v, int &carry, int *wave_sums) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(v, o);
        if (lane >= o) v += up;
    }
    if (lane == 63) wave_sums[wave] = v;
    __syncthreads();
    int before = carry;
    for (int w = 0; w < 4; w++) {
        if (w < wave) before += wave_sums[w];
        carry += wave_sums[w];
    }
    __syncthreads();
    return before + v;
}

struct Item { int request, tile, part, parts, blocks_per_part; };

// Item number x of the list (request, row tile, part of the keys).  With a split, a part has as many blocks as bring about
// `split` parts in all, at least kLeastBlocks; without one every tile is one part.  Returns false behind the list's end.
constexpr int kLeastBlocks = 8;
__device__ __forceinline__ bool find_item(const PagedAttn &a, int x, int tile_rows, Item &it) {
    __shared__ int sums[4], found[4];
    const int t = threadIdx.x;
    int per = 1 << 30;
    int tiles0 = 0, count0 = 0;
    if (a.split > 0) {
        long long total = 0;
        for (int r = t; r < a.n; r += 256) {
            const Request q = request_of(a, r);
            const int tiles = (int)(((long long)q.m * a.group + tile_rows - 1) / tile_rows);
            const int count = tiles ? blocks_of(a, q.len, q.first, q.first + q.m - 1).count : 0;
            if (r == t) { tiles0 = tiles; count0 = count; }
            total += (long long)tiles * count;
        }
        __shared__ long long wide[4];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
        if ((t & 63) == 0) wide[t >> 6] = total;
        __syncthreads();
        total = wide[0] + wide[1] + wide[2] + wide[3];
        per = (int)max((long long)kLeastBlocks, (total + a.split - 1) / a.split);
    }
    if (t == 0) found[0] = -1;
    __syncthreads();
    int carry = 0;
    for (int r0 = 0; r0 < a.n; r0 += 256) {
        const int r = r0 + t;
        int tiles = 0, parts = 1;
        if (a.split > 0 && r0 == 0) {
            tiles = tiles0;
            parts = max(1, (count0 + per - 1) / per);
        } else if (r < a.n) {
            const Request q = request_of(a, r);
            tiles = (int)(((long long)q.m * a.group + tile_rows - 1) / tile_rows);
            if (a.split > 0 && tiles) parts = max(1, (blocks_of(a, q.len, q.first, q.first + q.m - 1).count + per - 1) / per);
        }
        const int mine = tiles * parts, end = scan256(mine, carry, sums);
        if (x < end && x >= end - mine) {
            found[0] = r;
            found[1] = parts;
            found[2] = x - (end - mine);
            found[3] = tiles;
        }
        if (carry > x) break;
    }
    __syncthreads();
    it.request = __builtin_amdgcn_readfirstlane(found[0]);
    if (it.request < 0) return false;
    it.parts = __builtin_amdgcn_readfirstlane(found[1]);
    const int at = __builtin_amdgcn_readfirstlane(found[2]);
    it.tile = at / it.parts;
    it.part = at - it.tile * it.parts;
    it.tile = __builtin_amdgcn_readfirstlane(found[3]) - 1 - it.tile;      // the last rows of a causal request see the most: first
    it.blocks_per_part = per;
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

// ---- the kernel -------------------------------------------------------------------------------------------------------

// Where the 16-byte piece `c` of key row `key` lies in a wave's V block: pieces are exchanged inside 256 bytes so that the
// 8-byte reads of eight neighbouring keys, 32 bytes of each, fall on all 64 banks.
template <int DH>
__device__ __forceinline__ int v_piece(int key, int c) {
    return key * (DH / 8) + (DH == 64 ? c ^ (((key >> 1) & 3) << 1) : c ^ ((key & 7) << 1));
}

template <class T, int DH, int NT>
__global__ __launch_bounds__(256, DH == 256 || NT == 4 ? 1 : 2) void paged_attn_kernel(PagedAttn a) {
    constexpr int KS = DH / 32, CT = DH / 16, VL = DH / 16;      // k-steps of S, channel tiles of O, V loads of a lane per block
    constexpr int KEYS = 1024 / DH * 8 / 16;                     // keys per V load of a wave: 64 lanes * 8 channels / DH
    constexpr int OSTRIDE = DH + 4, WAVE_LDS = 16 * OSTRIDE * 4; // a wave's 32 x DH block of V, later its 16 x DH tile of O in 32 bits
    static_assert(32 * DH * 2 <= WAVE_LDS && KEYS * VL == 32, "V block");
    __shared__ __align__(16) unsigned char lds[4 * WAVE_LDS];
    __shared__ float2 stat[4][NT * 16];

    const int kv = a.pages.n_kv_heads, head = (int)(blockIdx.x % (unsigned)kv);
    const int x = (int)(blockIdx.x / (unsigned)kv);
    Item it;
    if (!find_item(a, x, NT * 16, it)) return;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, li = lane & 15;
    const Request rq = request_of(a, it.request);
    const int G = a.group, tile_rows = NT * 16, n_rows = rq.m * G, rho0 = it.tile * tile_rows;
    int pmin, pmax;
    tile_span(rq, G, it.tile, tile_rows, pmin, pmax);
    const Blocks bl = it.parts > 1 ? blocks_of(a, rq.len, rq.first, rq.first + rq.m - 1) : blocks_of(a, rq.len, pmin, pmax);
    const int b_lo = it.parts > 1 ? it.part * it.blocks_per_part : 0;
    const int b_hi = it.parts > 1 ? min(bl.count, b_lo + it.blocks_per_part) : bl.count;

    // queries of the tile, in operand order; rows behind the last are zero
    frag_t q[NT][KS];
    int see_lo[NT], see_hi[NT], stay[NT];                         // the lane's row sees keys see_lo .. see_hi - 1 and 0 .. stay - 1
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const int rho = rho0 + t * 16 + li, i = rho / G, hq = head * G + (rho - i * G);
        const int p = min(rq.first + i, kFar - 1), end = a.causal ? min(rq.len, p + 1) : rq.len;
        see_lo[t] = a.window ? p - a.window + 1 : 0;
        see_hi[t] = a.window ? min(end, p + a.window) : end;
        stay[t] = a.window ? min(a.sinks, end) : 0;
        const u16 *src = (const u16 *)a.q + (size_t)(rq.row0 + min(i, rq.m - 1)) * a.q_row + (size_t)hq * DH + 8 * g;
#pragma unroll
        for (int k = 0; k < KS; k++) {
            q[t][k] = frag_t{{0, 0, 0, 0}};
            if (rho < n_rows) q[t][k] = ld_frag(src + 32 * k);
        }
    }

    f32x4 o[NT][CT], lsum[NT];
    float mref[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        mref[t] = -INFINITY;
        lsum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CT; c++) o[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const int32_t *table = a.tables + (size_t)it.request * a.columns;
    const u16 *kp = (const u16 *)a.pages.k + (size_t)head * a.pages.head_stride, *vp = (const u16 *)a.pages.v + (size_t)head * a.pages.head_stride;
    const int page_mask = (1 << a.page_shift) - 1;
    const size_t pos_stride = a.pages.pos_stride, page_stride = a.pages.page_stride;
    const int v_key = lane / (DH / 8), v_ch = lane % (DH / 8);
    const unsigned k_off = 2u * (li * (unsigned)pos_stride + 8 * g), v_off = 2u * (v_key * (unsigned)pos_stride + v_ch * 8);    // bytes
    auto ld = [](const u16 *uniform, unsigned lane_bytes) { return ld_frag((const u16 *)((const char *)uniform + lane_bytes)); };

    // page of each 16-key tile of a block: -1 where no key of the tile is visible or the table names no page of the pool
    auto page_of = [&](int key) -> int {
        const int id = key < rq.len ? __builtin_amdgcn_readfirstlane(table[key >> a.page_shift]) : -1;
        return id >= 0 && id < a.pages.n_pages ? id : -1;
    };
    frag_t kf[2][KS], vf[VL];
    auto tile_base = [&](int page, int key) -> size_t { return (size_t)max(page, 0) * page_stride + (size_t)(key & page_mask) * pos_stride; };
    auto load_k = [&](size_t base0, size_t base1) {
#pragma unroll
        for (int k = 0; k < KS; k++) kf[0][k] = ld(kp + base0 + 32 * k, k_off);
#pragma unroll
        for (int k = 0; k < KS; k++) kf[1][k] = ld(kp + base1 + 32 * k, k_off);
    };
    auto load_v = [&](size_t base0, size_t base1) {
#pragma unroll
        for (int j = 0; j < VL; j++) vf[j] = ld(vp + (j < VL / 2 ? base0 : base1) + (size_t)(j % (VL / 2) * KEYS) * pos_stride, v_off);
    };

    unsigned char *mine = lds + wave * WAVE_LDS;
    const frag_t ones = {{Num<T>::kOnes, Num<T>::kOnes, Num<T>::kOnes, Num<T>::kOnes}};

    int b = b_lo + wave;
    int key0 = 0, pg0 = -1, pg1 = -1, nkey = 0, npg0 = -1, npg1 = -1;
    size_t base0 = 0, base1 = 0;
    if (b < b_hi) {
        key0 = block_key(bl, b);
        pg0 = page_of(key0);
        pg1 = page_of(key0 + 16);
        base0 = tile_base(pg0, key0);
        base1 = tile_base(pg1, key0 + 16);
        load_k(base0, base1);
        load_v(base0, base1);
    }
    if (b + 4 < b_hi) {
        nkey = block_key(bl, b + 4);
        npg0 = page_of(nkey);
        npg1 = page_of(nkey + 16);
    }
    for (; b < b_hi; b += 4) {
        // scores, then the registers of K are free for the next block
        f32x4 st[NT][2];
#pragma unroll
        for (int t = 0; t < NT; t++)
#pragma unroll
            for (int s = 0; s < 2; s++) {
                st[t][s] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KS; k++) st[t][s] = Num<T>::mfma(kf[s][k], q[t][k], st[t][s]);
            }
        const bool more = b + 4 < b_hi;
        if (more) {
            base0 = tile_base(npg0, nkey);
            base1 = tile_base(npg1, nkey + 16);
            load_k(base0, base1);
        }
        // is every key of the block visible to every row of the tile?
        const bool plain = pg0 >= 0 && pg1 >= 0 && key0 + 31 < rq.len && (!a.causal || key0 + 31 <= pmin) &&
                           (!a.window || key0 + 31 < a.sinks || (key0 > pmax - a.window && key0 + 31 - pmin < a.window));
        bool dirty = false;
        if (!plain) {
            // a value that is no number must not reach a row that does not see its key, not even times zero
            int odd = 0;
#pragma unroll
            for (int j = 0; j < VL; j++)
#pragma unroll
                for (int w = 0; w < 4; w++)
                    odd |= (int)((vf[j].w[w] & Num<T>::kExp) == Num<T>::kExp) | (int)(((vf[j].w[w] >> 16) & Num<T>::kExp) == Num<T>::kExp);
            dirty = __any(odd);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int j = 0; j < VL; j++)
            *reinterpret_cast<frag_t *>(mine + 16 * v_piece<DH>((j < VL / 2 ? 0 : 16) + v_key + (j % (VL / 2)) * KEYS, v_ch)) = vf[j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (more) load_v(base0, base1);

        // probabilities
        // (no branches: bitwise operators)
        auto visible = [&](int t, int key, int page) -> bool {
            return ((int)(page >= 0) & (((int)(key >= see_lo[t]) & (int)(key < see_hi[t])) | (int)(key < stay[t]))) != 0;
        };
        frag_t pf[NT];
#pragma unroll
        for (int t = 0; t < NT; t++) {
            float top = -INFINITY;
            if (!plain) {
#pragma unroll
                for (int s = 0; s < 2; s++)
#pragma unroll
                    for (int e = 0; e < 4; e++) st[t][s][e] = visible(t, key0 + s * 16 + 4 * g + e, s ? pg1 : pg0) ? st[t][s][e] : -INFINITY;
            }
#pragma unroll
            for (int s = 0; s < 2; s++)
#pragma unroll
                for (int e = 0; e < 4; e++) top = fmaxf(top, st[t][s][e]);
            // The reference is common to the four lanes of a row and only has to keep exp2 in range: it is raised, with a
            // maximum across the lanes and a rescaling, when a score passes it by too much, which after the first blocks is rare.
            if (__any(top * a.sc > mref[t] + kRaise)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float up = fmaxf(mref[t], top * a.sc - kShift);
                const float f = __builtin_amdgcn_exp2f(mref[t] - (up == -INFINITY ? 0.f : up));
                lsum[t] *= f;
#pragma unroll
                for (int c = 0; c < CT; c++) o[t][c] *= f;
                mref[t] = up;
            }
            const float ref = mref[t] == -INFINITY ? 0.f : mref[t];
            float p[2][4];
#pragma unroll
            for (int s = 0; s < 2; s++)
#pragma unroll
                for (int e = 0; e < 4; e++) p[s][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[t][s][e], a.sc, -ref));
            // Probabilities are rounded to the type of V for the matrix cores; the sum that divides them at the end is that of the
            // rounded ones, so what equal rounding errors have in common drops out.
            pf[t].w[0] = Num<T>::pack(p[0][0], p[0][1]);
            pf[t].w[1] = Num<T>::pack(p[0][2], p[0][3]);
            pf[t].w[2] = Num<T>::pack(p[1][0], p[1][1]);
            pf[t].w[3] = Num<T>::pack(p[1][2], p[1][3]);
            lsum[t] = Num<T>::mfma(ones, pf[t], lsum[t]);
        }
        if (__builtin_expect(dirty, 0)) {
            // rare: values that are infinite or no number, in a block that not all rows see in full.  They are added one by one
            // to the rows that see them and left out of the product.
#pragma unroll
            for (int t = 0; t < NT; t++)
                for (int key = 0; key < 32; key++) {
                    const int src = li + 16 * ((key >> 2) & 3);       // the lane that holds the row's probability of this key
                    const uint32_t w0 = (uint32_t)__shfl((int)pf[t].w[0], src), w1 = (uint32_t)__shfl((int)pf[t].w[1], src);
                    const uint32_t w2 = (uint32_t)__shfl((int)pf[t].w[2], src), w3 = (uint32_t)__shfl((int)pf[t].w[3], src);
                    const uint32_t a0 = key & 16 ? w2 : w0, a1 = key & 16 ? w3 : w1, word = key & 2 ? a1 : a0;
                    const float p = Num<T>::value(key & 1 ? word >> 16 : word & 0xffffu);
                    const bool see = visible(t, key0 + key, key & 16 ? pg1 : pg0);
#pragma unroll
                    for (int c = 0; c < CT; c++)
#pragma unroll
                        for (int d = 0; d < 4; d++) {
                            const int ch = c * 16 + 4 * g + d;
                            const uint32_t v = *reinterpret_cast<const u16 *>(mine + 16 * v_piece<DH>(key, ch >> 3) + 2 * (ch & 7));
                            if ((int)see & (int)((v & Num<T>::kExp) == Num<T>::kExp)) o[t][c][d] += p * Num<T>::value(v);
                        }
                }
        }
        // values: a lane's channel is li of tile c, its keys 4 g .. 4 g + 3 of each 16
#pragma unroll
        for (int c = 0; c < CT; c++) {
            typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
            const int row = 4 * g + (li >> 2), piece = 2 * c + ((li >> 1) & 1);
            unsigned char *p0 = mine + 16 * v_piece<DH>(row, piece) + 8 * (li & 1), *p1 = mine + 16 * v_piece<DH>(16 + row, piece) + 8 * (li & 1);
            const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p0));
            const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p1));
            frag_t vt = {{lo.x, lo.y, hi.x, hi.y}};
            if (__builtin_expect(dirty, 0)) {
#pragma unroll
                for (int w = 0; w < 4; w++) {
                    if ((vt.w[w] & Num<T>::kExp) == Num<T>::kExp) vt.w[w] &= 0xffff0000u;
                    if (((vt.w[w] >> 16) & Num<T>::kExp) == Num<T>::kExp) vt.w[w] &= 0xffffu;
                }
            }
#pragma unroll
            for (int t = 0; t < NT; t++) o[t][c] = Num<T>::mfma(vt, pf[t], o[t][c]);
        }
        key0 = nkey; pg0 = npg0; pg1 = npg1;
        if (b + 8 < b_hi) {
            nkey = block_key(bl, b + 8);
            npg0 = page_of(nkey);
            npg1 = page_of(nkey + 16);
        }
    }

    // ---- the four waves' sums become one
#pragma unroll
    for (int t = 0; t < NT; t++)
        if (g == 0) stat[wave][t * 16 + li] = float2{mref[t], lsum[t][0]};
    const long long item = (long long)x * kv + head;
#pragma unroll
    for (int t = 0; t < NT; t++) {
        __syncthreads();
        {
            const float2 s0 = stat[0][t * 16 + li], s1 = stat[1][t * 16 + li], s2 = stat[2][t * 16 + li], s3 = stat[3][t * 16 + li];
            const float top = fmaxf(fmaxf(s0.x, s1.x), fmaxf(s2.x, s3.x));
            const float f = __builtin_amdgcn_exp2f(mref[t] - (top == -INFINITY ? 0.f : top));
            float *dst = reinterpret_cast<float *>(mine) + li * OSTRIDE + 4 * g;
#pragma unroll
            for (int c = 0; c < CT; c++) *reinterpret_cast<f32x4 *>(dst + c * 16) = o[t][c] * f;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 2 * DH; e += 256) {
            const int r = e / (DH / 8), c = (e % (DH / 8)) * 8, rho = rho0 + t * 16 + r;
            if (rho >= n_rows) continue;
            float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, top = -INFINITY, l = 0.f;
#pragma unroll
            for (int w = 0; w < 4; w++) top = fmaxf(top, stat[w][t * 16 + r].x);
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float2 s = stat[w][t * 16 + r];
                l += s.y * __builtin_amdgcn_exp2f(s.x - (top == -INFINITY ? 0.f : top));
                const float *src = reinterpret_cast<const float *>(lds + w * WAVE_LDS) + r * OSTRIDE + c;
                const f32x4 u = *reinterpret_cast<const f32x4 *>(src), v = *reinterpret_cast<const f32x4 *>(src + 4);
#pragma unroll
                for (int i = 0; i < 4; i++) { sum[i] += u[i]; sum[4 + i] += v[i]; }
            }
            const int i = rho / G, hq = head * G + (rho - i * G), row = rq.row0 + i;
            if (it.parts > 1) {
                float *dst = a.partial + ((size_t)item * tile_rows + t * 16 + r) * DH + c;
                *reinterpret_cast<f32x4 *>(dst) = f32x4{sum[0], sum[1], sum[2], sum[3]};
                *reinterpret_cast<f32x4 *>(dst + 4) = f32x4{sum[4], sum[5], sum[6], sum[7]};
                if (c == 0) {
                    a.ml[item * tile_rows + t * 16 + r] = float2{top, l};
                    if (it.part == 0) a.where[(size_t)row * a.heads + hq] = int2{x, it.parts};
                }
            } else {
                // a row that sees nothing is zero
                const float f = l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l;
                uint4 v;
                v.x = Num<T>::pack(sum[0] * f, sum[1] * f);
                v.y = Num<T>::pack(sum[2] * f, sum[3] * f);
                v.z = Num<T>::pack(sum[4] * f, sum[5] * f);
                v.w = Num<T>::pack(sum[6] * f, sum[7] * f);
                store_out8(a, row, hq, DH, c, v);
                if (a.split > 0 && c == 0) a.where[(size_t)row * a.heads + hq] = int2{x, 1};
            }
        }
    }
}

// Joins the parts of a row: four waves take them in turn, then wave sums are added in order.  One workgroup per (row, head).
template <class T, int DH>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttn a, int tile_rows) {
    __shared__ float sums[4][DH];
    __shared__ float tops[4], ls[4];
    const int row = (int)(blockIdx.x / (unsigned)a.heads), hq = (int)(blockIdx.x % (unsigned)a.heads);
    // rows that belong to no request are left alone
    if (a.cu_rows && (row < a.cu_rows[0] || row >= a.cu_rows[a.n])) return;
    const int2 w = a.where[(size_t)row * a.heads + hq];
    if (w.y <= 1 || w.x < 0 || (long long)w.x + w.y > a.items) return;
    const int kv = a.pages.n_kv_heads, head = hq / a.group;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int m0 = row;
    if (a.cu_rows) {
        int lo = 0, hi = a.n - 1;                       // the request: the last one that starts at or before the row
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.cu_rows[mid] <= row) lo = mid; else hi = mid - 1;
        }
        m0 = a.cu_rows[lo];
    }
    const int r = ((row - m0) * a.group + hq % a.group) % tile_rows;
    constexpr int V = DH / 64;                          // channels of a lane
    float acc[V], top = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < V; i++) acc[i] = 0.f;
#pragma unroll 4
    for (int p = wave; p < w.y; p += 4) {
        const size_t at = ((size_t)(w.x + p) * kv + head) * tile_rows + r;
        const float2 s = a.ml[at];
        const float *src = a.partial + at * DH + lane * V;
        float v[V];
#pragma unroll
        for (int i = 0; i < V; i++) v[i] = src[i];
        const float up = fmaxf(top, s.x), ref = up == -INFINITY ? 0.f : up;
        const float f = __builtin_amdgcn_exp2f(top - ref), h = __builtin_amdgcn_exp2f(s.x - ref);
        l = l * f + s.y * h;
#pragma unroll
        for (int i = 0; i < V; i++) acc[i] = acc[i] * f + v[i] * h;
        top = up;
    }
#pragma unroll
    for (int i = 0; i < V; i++) sums[wave][lane * V + i] = acc[i];
    if (lane == 0) { tops[wave] = top; ls[wave] = l; }
    __syncthreads();
    const int c = threadIdx.x * 8;
    if (c >= DH) return;
    float best = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    if (best == -INFINITY) best = 0.f;
    float total = 0.f, out[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const float f = __builtin_amdgcn_exp2f(tops[k] - best);
        total += ls[k] * f;
#pragma unroll
        for (int i = 0; i < 8; i++) out[i] += sums[k][c + i] * f;
    }
    const float f = total > 0.f ? 1.0f / total : total == 0.f ? 0.f : total;
    uint4 v;
    v.x = Num<T>::pack(out[0] * f, out[1] * f);
    v.y = Num<T>::pack(out[2] * f, out[3] * f);
    v.z = Num<T>::pack(out[4] * f, out[5] * f);
    v.w = Num<T>::pack(out[6] * f, out[7] * f);
    store_out8(a, row, hq, DH, c, v);
}

template <class T, int DH, int NT>
void launch_nt(const PagedAttn &a, hipStream_t s) {
    paged_attn_kernel<T, DH, NT><<<dim3((unsigned)(a.items * a.pages.n_kv_heads)), 256, 0, s>>>(a);
    if (a.split > 0) paged_join_kernel<T, DH><<<dim3((unsigned)a.rows * (unsigned)a.heads), 256, 0, s>>>(a, NT * 16);
}

template <class T, int DH>
void launch_dim(const PagedAttn &a, int nt, hipStream_t s) {
    if (nt == 1) return launch_nt<T, DH, 1>(a, s);
    if (nt == 2 || DH == 256) return launch_nt<T, DH, 2>(a, s);
    if constexpr (DH != 256) launch_nt<T, DH, 4>(a, s);
}

template <class T>
void launch_type(const PagedAttn &a, int nt, hipStream_t s) {
    switch (a.pages.head_dim) {
    case 64: return launch_dim<T, 64>(a, nt, s);
    case 128: return launch_dim<T, 128>(a, nt, s);
    default: return launch_dim<T, 256>(a, nt, s);
    }
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

int paged_attn_tiles(const odb_pages &p, int group, int max_rows) {
    const long long rows = (long long)max_rows * group;
    return rows <= 16 ? 1 : rows <= 32 || p.head_dim == 256 ? 2 : 4;
}

void paged_attn_split(const odb_pages &p, int n, int rows, int group, int nt, long long max_len, int *split, long long *items) {
    // Every request has at most one row tile that is not full.
    const long long tiles = (n < rows ? n : rows) + (long long)rows * group / (16 * nt);
    const long long blocks = (max_len + 31) / 32;
    const int aim = (2048 / nt + p.n_kv_heads - 1) / p.n_kv_heads;
    *split = tiles >= aim || blocks <= 2 * kLeastBlocks ? 0 : aim;
    *items = tiles + *split;
}

size_t paged_attn_workspace(const odb_pages &p, int rows, int heads, int nt, int split, long long items) {
    if (!split) return 0;
    const size_t tile_rows = (size_t)items * p.n_kv_heads * nt * 16;
    return up256(tile_rows * p.head_dim * 4) + up256(tile_rows * 8) + up256((size_t)rows * heads * 8);
}

void launch_paged_attention(PagedAttn a, int nt, void *workspace, hipStream_t s) {
    if (a.rows < 1) return;
    if (a.split > 0) {
        const size_t tile_rows = (size_t)a.items * a.pages.n_kv_heads * nt * 16;
        char *w = (char *)workspace;
        a.partial = (float *)w;
        a.ml = (float2 *)(w + up256(tile_rows * a.pages.head_dim * 4));
        a.where = (int2 *)((char *)a.ml + up256(tile_rows * 8));
    }
    if (a.pages.dtype == ODB_F16) launch_type<_Float16>(a, nt, s);
    else launch_type<__bf16>(a, nt, s);
}

}  // namespace odb
