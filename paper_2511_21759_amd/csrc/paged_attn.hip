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

// Lengths and tables are read through the scalar cache where the index is the same for a whole wave: such a load does not
// queue behind the loads of K and V.  (No kernel of this file writes them.)
typedef const __attribute__((address_space(4))) int32_t *scalar_ptr;
__device__ __forceinline__ int ld_scalar(const int32_t *p, int i) { return ((scalar_ptr)(uintptr_t)p)[i]; }

__device__ __forceinline__ Request request_of(const PagedAttn &a, int r) {
    Request q;
    int lo = r, hi = r + 1;
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

struct Place { Request q; int r; long long at, total; };

__device__ __forceinline__ long long uniform(long long x) {
    return (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) |
                       (unsigned)__builtin_amdgcn_readfirstlane((int)x));
}

__device__ __forceinline__ int tiles_of(const PagedAttn &a, const Request &q, int tile_rows) {
    return (int)(((long long)q.m * a.group + tile_rows - 1) / tile_rows);
}
// blocks of keys that a request's rows see together (one where they see none, so that their zeros are written)
__device__ __forceinline__ int request_blocks(const PagedAttn &a, const Request &q) {
    return max(1, blocks_of(a, q.len, q.first, q.first + q.m - 1).count);
}

// The requests' weights - row tiles, times blocks where keys are split - lie behind each other; finds the request that holds
// item pick(total) and the item's offset inside it.  False if there is none.  Up to 64 requests every wave does it alone.
template <class Pick>
__device__ __forceinline__ bool find_place(const PagedAttn &a, int tile_rows, bool need_total, Pick pick, Place &p) {
    const int lane = threadIdx.x & 63;
    auto weigh = [&](const Request &q) -> long long {
        const int tiles = tiles_of(a, q, tile_rows);
        return a.split && tiles ? (long long)tiles * request_blocks(a, q) : tiles;
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
        const long long v = weigh(q), end = scan64(v);
        p.total = uniform(__shfl(end, 63));
        const long long x = pick(p.total);
        const unsigned long long behind = __ballot(end > x);
        if (x >= p.total) return false;
        p.r = __builtin_amdgcn_readfirstlane(__ffsll(behind) - 1);
        p.at = x - uniform(__shfl(end - v, p.r));
        p.q.m = __builtin_amdgcn_readlane(q.m, p.r);
        p.q.len = __builtin_amdgcn_readlane(q.len, p.r);
        p.q.first = __builtin_amdgcn_readlane(q.first, p.r);
        p.q.row0 = __builtin_amdgcn_readlane(q.row0, p.r);
        return true;
    }
    __shared__ long long sums[4], found_at;
    __shared__ int found;
    const int t = threadIdx.x, wave = t >> 6;
    if (t == 0) found = -1;
    p.total = 0;
    if (need_total) {
        long long v = 0;
        for (int r = t; r < a.n; r += 256) v += weigh(request_of(a, r));
        v = scan64(v);
        if (lane == 63) sums[wave] = v;
        __syncthreads();
        p.total = uniform(sums[0] + sums[1] + sums[2] + sums[3]);
        __syncthreads();
        if (pick(p.total) >= p.total) return false;
    }
    const long long x = pick(p.total);
    long long carry = 0;
    for (int r0 = 0; r0 < a.n && carry <= x; r0 += 256) {
        const int r = r0 + t;
        const long long v = r < a.n ? weigh(request_of(a, r)) : 0, end0 = scan64(v);
        if (lane == 63) sums[wave] = end0;
        __syncthreads();
        long long end = carry + end0;
        for (int w = 0; w < 4; w++) {
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

// ---- the kernel -------------------------------------------------------------------------------------------------------

// Where the 16-byte piece `c` of key row `key` lies in a wave's V block: pieces are exchanged inside 256 bytes so that the
// 8-byte reads of eight neighbouring keys, 32 bytes of each, fall on all 64 banks.
template <int DH>
__device__ __forceinline__ int v_piece(int key, int c) {
    return key * (DH / 8) + (DH == 64 ? c ^ (((key >> 1) & 3) << 1) : c ^ ((key & 7) << 1));
}

// With keys split (a.split workgroups per K/V head), the blocks of all (request, row tile) pairs lie behind each other and every
// workgroup takes an equal piece of that list, wherever it starts and ends: all finish together, however ragged the lengths are.
// A pair that lies inside one piece is finished there; of the others each piece leaves its sums (reference, sum, O), which
// paged_join_kernel adds in order.  A piece has at most one pair that it does not start and one that it does not end, so two
// places per workgroup hold them: 2 w + 1 for a pair that starts in it, 2 w for one that started before.
constexpr int kLeastBlocks = 8;          // of a piece: two per wave; shorter ones cost more in sums than they save

template <class T, int DH, int NT>
__global__ __launch_bounds__(256, DH == 256 || NT == 4 ? 1 : 2) void paged_attn_kernel(PagedAttn a) {
    constexpr int KS = DH / 32, CT = DH / 16, VL = DH / 16;      // k-steps of S, channel tiles of O, V loads of a lane per block
    constexpr int KEYS = 1024 / DH * 8 / 16;                     // keys per V load of a wave: 64 lanes * 8 channels / DH
    constexpr int OSTRIDE = DH + 4, WAVE_LDS = 16 * OSTRIDE * 4; // a wave's 32 x DH block of V, later its 16 x DH tile of O in 32 bits
    constexpr int TILE_ROWS = NT * 16;
    static_assert(32 * DH * 2 <= WAVE_LDS && KEYS * VL == 32, "V block");
    __shared__ __align__(16) unsigned char lds[4 * WAVE_LDS];
    __shared__ float2 stat[4][TILE_ROWS];

    const int kv = a.pages.n_kv_heads, head = (int)(blockIdx.x % (unsigned)kv), x = (int)(blockIdx.x / (unsigned)kv);
    const bool split = a.split > 0;
    auto piece_of = [&](long long total) { return max((long long)kLeastBlocks, (total + a.split - 1) / max(a.split, 1)); };
    Place pl;
    if (!find_place(a, TILE_ROWS, split, [&](long long total) { return split ? piece_of(total) * x : (long long)x; }, pl)) return;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, li = lane & 15;
    const int G = a.group;
    const u16 *kp = (const u16 *)a.pages.k + (size_t)head * a.pages.head_stride, *vp = (const u16 *)a.pages.v + (size_t)head * a.pages.head_stride;
    const int page_mask = (1 << a.page_shift) - 1;
    const size_t pos_stride = a.pages.pos_stride, page_stride = a.pages.page_stride;
    const int v_key = lane / (DH / 8), v_ch = lane % (DH / 8);
    const unsigned k_off = 2u * (li * (unsigned)pos_stride + 8 * g), v_off = 2u * (v_key * (unsigned)pos_stride + v_ch * 8);    // bytes
    unsigned char *mine = lds + wave * WAVE_LDS;
    const frag_t ones = {{Num<T>::kOnes, Num<T>::kOnes, Num<T>::kOnes, Num<T>::kOnes}};
    // K/V of a request with one row tile are read once: past the caches' replacement
    auto ld = [](const u16 *uniform, unsigned lane_bytes) -> frag_t {
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        typedef const __attribute__((address_space(1))) char *global_bytes;
        typedef const __attribute__((address_space(1))) u32x4 *global_ptr;
        global_bytes base = (global_bytes)(uintptr_t)uniform;
        asm("" : "+s"(base));                                     // (keeps the sum of a scalar base and a 32-bit offset apart)
        const global_ptr p = (global_ptr)(base + lane_bytes);
        return __builtin_bit_cast(frag_t, NT == 1 ? __builtin_nontemporal_load(p) : *p);
    };

    Request rq = pl.q;
    int request = pl.r, tiles = tiles_of(a, rq, TILE_ROWS), nb = split ? request_blocks(a, rq) : 1;
    int tile = __builtin_amdgcn_readfirstlane((int)(pl.at / nb)), b_lo = __builtin_amdgcn_readfirstlane((int)(pl.at - (long long)tile * nb));
    // blocks of this piece that are left
    const long long piece = piece_of(pl.total);
    long long left = split ? min(piece, pl.total - piece * x) : 1;
    if (!split) tile = tiles - 1 - tile;                          // the last rows of a causal request see the most: first

    for (;;) {
        const int n_rows = rq.m * G, rho0 = tile * TILE_ROWS;
        int ql = lane;
        asm volatile("" : "+v"(ql));
        int pmin, pmax;
        tile_span(rq, G, tile, TILE_ROWS, pmin, pmax);
        const Blocks bl = split ? blocks_of(a, rq.len, rq.first, rq.first + rq.m - 1) : blocks_of(a, rq.len, pmin, pmax);
        const int b_end = split ? (int)min((long long)nb, b_lo + left) : 1;       // in units of the list
        const int b_hi = split ? min(b_end, bl.count) : bl.count;
        const bool whole = b_lo == 0 && b_end == nb;

        // queries of the tile, in operand order; rows behind the last repeat it and are not written
        frag_t q[NT][KS];
        int see_lo[NT], see_hi[NT], stay[NT];                     // the lane's row sees keys see_lo .. see_hi - 1 and 0 .. stay - 1
#pragma unroll
        for (int t = 0; t < NT; t++) {
            const int rho = min(rho0 + t * 16 + (ql & 15), n_rows - 1), i = rho / G, hq = head * G + (rho - i * G);
            const int p = min(rq.first + i, kFar - 1), end = a.causal ? min(rq.len, p + 1) : rq.len;
            see_lo[t] = a.window ? p - a.window + 1 : 0;
            see_hi[t] = a.window ? min(end, p + a.window) : end;
            stay[t] = a.window ? min(a.sinks, end) : 0;
            const u16 *src = (const u16 *)a.q + (size_t)(rq.row0 + i) * a.q_row + (size_t)hq * DH + 8 * (ql >> 4);
#pragma unroll
            for (int k = 0; k < KS; k++) q[t][k] = ld_frag(src + 32 * k);
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

        // page of each 16-key tile of a block: -1 where no key of the tile is visible or the table names no page of the pool
        const int32_t *table = a.tables + (size_t)request * a.columns;
        auto page_of = [&](int key) -> int {
            const int id = key < rq.len ? ld_scalar(table, key >> a.page_shift) : -1;
            return id >= 0 && id < a.pages.n_pages ? id : -1;
        };
        frag_t kf[2][KS], vf[VL];
        auto tile_base = [&](int page, int key) -> size_t { return (size_t)max(page, 0) * page_stride + (size_t)(key & page_mask) * pos_stride; };
        auto load_k = [&](size_t base0, size_t base1, unsigned off) {
#pragma unroll
            for (int k = 0; k < KS; k++) kf[0][k] = ld(kp + base0 + 32 * k, off);
#pragma unroll
            for (int k = 0; k < KS; k++) kf[1][k] = ld(kp + base1 + 32 * k, off);
        };
        auto load_v = [&](size_t base0, size_t base1, unsigned off) {
#pragma unroll
            for (int j = 0; j < VL; j++) vf[j] = ld(vp + (j < VL / 2 ? base0 : base1) + (size_t)(j % (VL / 2) * KEYS) * pos_stride, off);
        };

        int b = b_lo + wave;
        if (b < b_hi) {
            int key0 = block_key(bl, b), pg0 = page_of(key0), pg1 = page_of(key0 + 16), nkey = 0, npg0 = -1, npg1 = -1;
            size_t base0 = tile_base(pg0, key0), base1 = tile_base(pg1, key0 + 16);
            load_k(base0, base1, k_off);
            __builtin_amdgcn_sched_barrier(0);                    // K first here too, or the loop's first wait would be for both
            load_v(base0, base1, v_off);
#pragma unroll
            for (int t = 0; t < NT; t++)
#pragma unroll
                for (int k = 0; k < KS; k++) asm volatile("" ::"v"(q[t][k].w[0]));     // waits for the queries here, not in the loop
            if (b + 4 < b_hi) {
                nkey = block_key(bl, b + 4);
                npg0 = page_of(nkey);
                npg1 = page_of(nkey + 16);
            }
            for (; b < b_hi; b += 4) {
                // Behind the last block the loads are made all the same, of 16 bytes for all lanes: with no branch around them
                // the wait for K need not be one for V too.
                const bool more = b + 4 < b_hi;
                const unsigned k_next = more ? k_off : 0, v_next = more ? v_off : 0;
                base0 = tile_base(npg0, nkey);
                base1 = tile_base(npg1, nkey + 16);
                // is every key of the block visible to every row of the tile?
                const bool plain = pg0 >= 0 && pg1 >= 0 && key0 + 31 < rq.len && (!a.causal || key0 + 31 <= pmin) &&
                                   (!a.window || key0 + 31 < a.sinks || (key0 > pmax - a.window && key0 + 31 - pmin < a.window));
                // (no branches: bitwise operators)
                auto visible = [&](int t, int key, int page) -> bool {
                    return ((int)(page >= 0) & (((int)(key >= see_lo[t]) & (int)(key < see_hi[t])) | (int)(key < stay[t]))) != 0;
                };
                f32x4 st[2][2];                                       // scores of this row tile and the next
                auto scores = [&](int t) {
#pragma unroll
                    for (int s = 0; s < 2; s++) {
                        f32x4 z = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int k = 0; k < KS; k++) z = Num<T>::mfma(kf[s][k], q[t][k], z);
                        st[t & 1][s] = z;
                    }
                };
                scores(0);
                if (NT == 1) load_k(base0, base1, k_next);            // the registers of K are free for the next block
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
                    *reinterpret_cast<frag_t *>(mine + 16 * v_piece<DH>(v_key + j % (8 / KEYS) * KEYS, v_ch) + j / (8 / KEYS) * (8 * DH * 2)) = vf[j];
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                load_v(base0, base1, v_next);
                // V^T in operand order: a lane's channel is li of tile c, its keys 4 g .. 4 g + 3 of each 16
                auto v_tile = [&](int c) -> frag_t {
                    typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
                    const int row = 4 * g + (li >> 2), at = 2 * c + ((li >> 1) & 1);
                    unsigned char *p0 = mine + 16 * v_piece<DH>(row, at) + 8 * (li & 1), *p1 = p0 + 16 * DH * 2;
                    const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p0));
                    const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p1));
                    return frag_t{{lo.x, lo.y, hi.x, hi.y}};
                };
                auto clear_odd = [](frag_t &v) {
#pragma unroll
                    for (int w = 0; w < 4; w++) {
                        if ((v.w[w] & Num<T>::kExp) == Num<T>::kExp) v.w[w] &= 0xffff0000u;
                        if (((v.w[w] >> 16) & Num<T>::kExp) == Num<T>::kExp) v.w[w] &= 0xffffu;
                    }
                };
                frag_t vt[NT > 1 ? CT : 1];                           // held for several row tiles
                if (NT > 1) {
#pragma unroll
                    for (int c = 0; c < CT; c++) vt[c] = v_tile(c);
                    if (__builtin_expect(dirty, 0))
#pragma unroll
                        for (int c = 0; c < CT; c++) clear_odd(vt[c]);
                }

                // row tiles one after the other, the next one's scores under way in the matrix cores while this one's probabilities are made
#pragma unroll
                for (int t = 0; t < NT; t++) {
                    if (t + 1 < NT) scores(t + 1);
                    if (NT > 1 && t + 2 == NT) load_k(base0, base1, k_next);
                    f32x4 (&z)[2] = st[t & 1];
                    float top = -INFINITY;
                    if (!plain) {
#pragma unroll
                        for (int s = 0; s < 2; s++)
#pragma unroll
                            for (int e = 0; e < 4; e++) z[s][e] = visible(t, key0 + s * 16 + 4 * g + e, s ? pg1 : pg0) ? z[s][e] : -INFINITY;
                    }
#pragma unroll
                    for (int s = 0; s < 2; s++)
#pragma unroll
                        for (int e = 0; e < 4; e++) top = fmaxf(top, z[s][e]);
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
                        for (int e = 0; e < 4; e++) p[s][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[s][e], a.sc, -ref));
                    // Probabilities are rounded to the type of V for the matrix cores; the sum that divides them at the end is that of the
                    // rounded ones, so what equal rounding errors have in common drops out.
                    frag_t pf;
                    pf.w[0] = Num<T>::pack(p[0][0], p[0][1]);
                    pf.w[1] = Num<T>::pack(p[0][2], p[0][3]);
                    pf.w[2] = Num<T>::pack(p[1][0], p[1][1]);
                    pf.w[3] = Num<T>::pack(p[1][2], p[1][3]);
                    if (__builtin_expect(dirty, 0)) {
                        // rare: values that are infinite or no number, in a block that not all rows see in full.  They are added one by
                        // one to the rows that see them; the product has zeros in their place.
                        int dl = lane;                            // (hidden, as below)
                        asm volatile("" : "+v"(dl));
                        for (int key = 0; key < 32; key++) {
                            const int src = (dl & 15) + 16 * ((key >> 2) & 3);       // the lane that holds the row's probability of this key
                            const uint32_t w0 = (uint32_t)__shfl((int)pf.w[0], src), w1 = (uint32_t)__shfl((int)pf.w[1], src);
                            const uint32_t w2 = (uint32_t)__shfl((int)pf.w[2], src), w3 = (uint32_t)__shfl((int)pf.w[3], src);
                            const uint32_t a0 = key & 16 ? w2 : w0, a1 = key & 16 ? w3 : w1, word = key & 2 ? a1 : a0;
                            const float pk = Num<T>::value(key & 1 ? word >> 16 : word & 0xffffu);
                            const bool see = visible(t, key0 + key, key & 16 ? pg1 : pg0);
#pragma unroll
                            for (int c = 0; c < CT; c++)
#pragma unroll
                                for (int d = 0; d < 4; d++) {
                                    const int ch = c * 16 + 4 * (dl >> 4) + d;
                                    const uint32_t v = *reinterpret_cast<const u16 *>(mine + 16 * v_piece<DH>(key, ch >> 3) + 2 * (ch & 7));
                                    if ((int)see & (int)((v & Num<T>::kExp) == Num<T>::kExp)) o[t][c][d] += pk * Num<T>::value(v);
                                }
                        }
                        if (NT == 1) {
                            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                            for (int j = 0; j < VL; j++) {
                                frag_t *at = reinterpret_cast<frag_t *>(mine + 16 * (dl + 64 * j)), v = *at;
                                clear_odd(v);
                                *at = v;
                            }
                            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                        }
                    }
                    lsum[t] = Num<T>::mfma(ones, pf, lsum[t]);
#pragma unroll
                    for (int c = 0; c < CT; c++) o[t][c] = Num<T>::mfma(NT > 1 ? vt[c] : v_tile(c), pf, o[t][c]);
                }
                key0 = nkey; pg0 = npg0; pg1 = npg1;
                if (b + 8 < b_hi) {
                    nkey = block_key(bl, b + 8);
                    npg0 = page_of(nkey);
                    npg1 = page_of(nkey + 16);
            }
            }
        }

        // ---- the four waves' sums become one
        // (the thread's number is hidden from the compiler, which else keeps addresses of this part in registers through the loop)
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        const int eg = (tid >> 4) & 3, el = tid & 15;
#pragma unroll
        for (int t = 0; t < NT; t++)
            if (eg == 0) stat[wave][t * 16 + el] = float2{mref[t], lsum[t][0]};
        const long long place = (2ll * x + (b_lo == 0)) * kv + head;
        // parts of the pair: this piece, where it starts, to the one that holds its last block
        const int parts = whole ? 1 : (int)((piece * x + (min(piece, pl.total - piece * x) - left) - b_lo + nb - 1) / piece) - x + 1;
#pragma unroll
        for (int t = 0; t < NT; t++) {
            __syncthreads();
            {
                const float2 s0 = stat[0][t * 16 + el], s1 = stat[1][t * 16 + el], s2 = stat[2][t * 16 + el], s3 = stat[3][t * 16 + el];
                const float top = fmaxf(fmaxf(s0.x, s1.x), fmaxf(s2.x, s3.x));
                const float f = __builtin_amdgcn_exp2f(mref[t] - (top == -INFINITY ? 0.f : top));
                float *dst = reinterpret_cast<float *>(mine) + el * OSTRIDE + 4 * eg;
#pragma unroll
                for (int c = 0; c < CT; c++) *reinterpret_cast<f32x4 *>(dst + c * 16) = o[t][c] * f;
            }
            __syncthreads();
            for (int e = tid; e < 2 * DH; e += 256) {
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
                if (!whole) {
                    float *dst = a.partial + ((size_t)place * TILE_ROWS + t * 16 + r) * DH + c;
                    *reinterpret_cast<f32x4 *>(dst) = f32x4{sum[0], sum[1], sum[2], sum[3]};
                    *reinterpret_cast<f32x4 *>(dst + 4) = f32x4{sum[4], sum[5], sum[6], sum[7]};
                    if (c == 0) {
                        a.ml[place * TILE_ROWS + t * 16 + r] = float2{top, l};
                        if (b_lo == 0) a.where[(size_t)row * a.heads + hq] = int2{x, parts * 64 + t * 16 + r};
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
                    if (split && c == 0) a.where[(size_t)row * a.heads + hq] = int2{x, 0};
                }
            }
        }
        if (!split) return;
        left -= b_end - b_lo;
        if (left <= 0) return;
        b_lo = 0;
        if (++tile == tiles) {
            do {
                if (++request >= a.n) return;
                rq = request_of(a, request);
                tiles = tiles_of(a, rq, TILE_ROWS);
            } while (tiles == 0);
            tile = 0;
            nb = request_blocks(a, rq);
        }
        __syncthreads();
    }
}

// Adds the parts of a row in order.  WPR waves per (row, head) - one where there are many rows, which have few parts each, 16
// where there are few, which have many: the parts' references and sums first, a part per lane, then their O, a part per wave in turn.
template <class T, int DH, int WPR>
__global__ __launch_bounds__(WPR == 16 ? 1024 : 256) void paged_join_kernel(PagedAttn a) {
    constexpr int V = DH / 64, ROWS = WPR == 16 ? 1 : 4 / WPR;          // channels of a lane, rows of a workgroup
    __shared__ float sums[ROWS][WPR][DH];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = wave / WPR, w = wave % WPR;
    const long long unit = (long long)blockIdx.x * ROWS + sub;
    const int row = (int)(unit / a.heads), hq = (int)(unit % a.heads);
    // rows that belong to no request are left alone
    bool mine = row < a.rows && (!a.cu_rows || (row >= a.cu_rows[0] && row < a.cu_rows[a.n]));
    int2 at{0, 0};
    if (mine) at = a.where[(size_t)row * a.heads + hq];
    const int parts = at.y >> 6, r = at.y & 63, kv = a.pages.n_kv_heads, head = hq / a.group;
    mine = mine && parts > 1 && r < a.tile_rows && at.x >= 0 && (long long)at.x + parts <= a.split;
    auto place = [&](int p) { return ((size_t)(2ll * (at.x + p) + (p == 0)) * kv + head) * a.tile_rows + r; };
    float top = -INFINITY, total = 0.f, acc[V];
#pragma unroll
    for (int i = 0; i < V; i++) acc[i] = 0.f;
    if (mine) {
        for (int p = lane; p < parts; p += 64) top = fmaxf(top, a.ml[place(p)].x);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        if (top == -INFINITY) top = 0.f;
        for (int p = lane; p < parts; p += 64) {
            const float2 s = a.ml[place(p)];
            total += s.y * __builtin_amdgcn_exp2f(s.x - top);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
#pragma unroll 8
        for (int p = w; p < parts; p += WPR) {
            const size_t e = place(p);
            const float f = __builtin_amdgcn_exp2f(a.ml[e].x - top);
            const float *src = a.partial + e * DH + lane * V;
#pragma unroll
            for (int i = 0; i < V; i++) acc[i] += src[i] * f;
        }
    }
#pragma unroll
    for (int i = 0; i < V; i++) sums[sub][w][lane * V + i] = acc[i];
    __syncthreads();
    const int c = (w * 64 + lane) * 8;
    if (!mine || c >= DH) return;
    float out[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < WPR; k++)
#pragma unroll
        for (int i = 0; i < 8; i++) out[i] += sums[sub][k][c + i];
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
    if (!a.split) return;
    const long long units = (long long)a.rows * a.heads;
    if (units <= 512) paged_join_kernel<T, DH, 16><<<dim3((unsigned)units), 1024, 0, s>>>(a);
    else paged_join_kernel<T, DH, 1><<<dim3((unsigned)((units + 3) / 4)), 256, 0, s>>>(a);
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
    // One round of workgroups.  Two per CU hide each other's starts and ends where a tile is 16 rows (64 single tokens over 555 MB:
    // 107 us, with one 110, with four 107; two over 985 MB 156, 153, 158); with more rows every cut costs more sums (8 x 32 rows: one
    // 59 us, two 62, four 68).
    const int aim = (256 * (nt == 1 && p.head_dim != 256 ? 2 : 1) + p.n_kv_heads - 1) / p.n_kv_heads;
    // With four row tiles for every workgroup the lengths even out by themselves, and a tile then reads only the keys it sees.
    *split = tiles >= 4 * aim || blocks <= 2 * kLeastBlocks ? 0 : aim;
    *items = *split ? *split : tiles;
}

size_t paged_attn_workspace(const odb_pages &p, int rows, int heads, int nt, int split) {
    if (!split) return 0;
    const size_t tile_rows = 2 * (size_t)split * p.n_kv_heads * nt * 16;
    return up256(tile_rows * p.head_dim * 4) + up256(tile_rows * 8) + up256((size_t)rows * heads * 8);
}

void launch_paged_attention(PagedAttn a, int nt, void *workspace, hipStream_t s) {
    if (a.rows < 1) return;
    a.tile_rows = nt * 16;
    if (a.split > 0) {
        const size_t tile_rows = 2 * (size_t)a.split * a.pages.n_kv_heads * nt * 16;
        char *w = (char *)workspace;
        a.partial = (float *)w;
        a.ml = (float2 *)(w + up256(tile_rows * a.pages.head_dim * 4));
        a.where = (int2 *)((char *)a.ml + up256(tile_rows * 8));
    }
    if (a.pages.dtype == ODB_F16) launch_type<_Float16>(a, nt, s);
    else launch_type<__bf16>(a, nt, s);
}

}  // namespace odb
