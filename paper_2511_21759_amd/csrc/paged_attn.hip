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
// block are issued while the block before it is worked on.  That is the way for few rows (paged_attn_kernel); for tiles of many rows
// the waves split the rows and share K and V (paged_rows_kernel).  paged_attn_plan chooses.
#include "paged_attn_core.h"

namespace odb {

namespace {

// ---- few rows: the waves of a workgroup split the keys -----------------------------------------------------------------

// With keys split (a.split workgroups per K/V head), the blocks of all (request, row tile) pairs lie behind each other and every
// workgroup takes an equal piece of that list, wherever it starts and ends: all finish together, however ragged the lengths are.
// (A pair whose blocks all lie behind a piece's end is left to the next piece.)
// A pair that lies inside one piece is finished there; of the others each piece leaves its sums (reference, sum, O), which
// paged_join_kernel adds in order.  A piece has at most one pair that it does not start and one that it does not end, so two
// places per workgroup hold them: 2 w + 1 for a pair that starts in it, 2 w for one that started before.
// Bound by HBM with single tokens (two of 1e5 positions, 985 MB, 149 us = 6.6 TB/s; 64 of 17 to 16384, 555 MB, 91 us = 6.1), by the
// latency of its beginning and end where keys are few (333 positions 6.8 us).
// Places of a piece at least: 32 single tokens of 20 to 4000 positions, 28 heads over 4, take 18 us with 12, 19 with 16, 21 with 10.
constexpr int kLeastPiece = 12;

template <class T, int DH, int NT>
__global__ __launch_bounds__(64 * NW, DH == 256 || NT == 4 ? 1 : 2) void paged_attn_kernel(PagedAttn a) {
    constexpr int KS = DH / 32, CT = DH / 16, VL = DH / 16;      // k-steps of S, channel tiles of O, V loads of a lane per block
    constexpr int KEYS = 1024 / DH * 8 / 16;                     // keys per V load of a wave: 64 lanes * 8 channels / DH
    constexpr int OSTRIDE = DH + 4, WAVE_LDS = 16 * OSTRIDE * 4; // a wave's 32 x DH block of V, later its 16 x DH tile of O in 32 bits
    constexpr int TILE_ROWS = NT * 16;
    static_assert(32 * DH * 2 <= WAVE_LDS && KEYS * VL == 32, "V block");
    __shared__ __align__(16) unsigned char lds[NW * WAVE_LDS];
    __shared__ float2 stat[NW][TILE_ROWS];

    const int kv = a.pages.n_kv_heads, head = (int)(blockIdx.x % (unsigned)kv), x = (int)(blockIdx.x / (unsigned)kv);
    const bool split = a.split > 0;
    auto piece_of = [&](long long total) { return max((long long)kLeastPiece, (total + a.split - 1) / max(a.split, 1)); };
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
    Request rq = pl.q;
    int request = pl.r, tiles = tiles_of(a, rq, TILE_ROWS), nb = split ? request_blocks(a, rq) : 1;
    // place in the pair's part of the list where this piece starts
    const int cost = split ? kPairCost : 0;
    int tile = __builtin_amdgcn_readfirstlane((int)(pl.at / (nb + cost))), at = __builtin_amdgcn_readfirstlane((int)(pl.at - (long long)tile * (nb + cost)));
    // places of this piece that are left
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
            const Blocks bl = split ? blocks_of(a, rq.len, rq.first, rq.first + rq.m - 1) : blocks_of(a, rq.len, pmin, pmax);
            const int b_hi = split ? min(b_end, bl.count) : bl.count;
            const bool whole = b_lo == 0 && b_end == nb;

            // queries of the tile, in operand order; rows behind the last repeat it and are not written
            frag_t q[NT][KS];
            Sight sight[NT];                                          // of the lane's row of each tile
#pragma unroll
            for (int t = 0; t < NT; t++) {
                const int rho = min(rho0 + t * 16 + (ql & 15), n_rows - 1), i = rho / G, hq = head * G + (rho - i * G);
                sight[t] = sight_of(a, rq.len, rq.first + i);
                const u16 *src = (const u16 *)a.q + (size_t)(rq.row0 + i) * a.q_row + (size_t)hq * DH + 8 * (ql >> 4);
#pragma unroll
                for (int k = 0; k < KS; k++) q[t][k] = ld_frag(src + 32 * k);
            }

            f32x4 o[NT][CT], lsum[NT];
            Reference ref[NT];
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
            frag_t kf[2][KS], vf[VL];
            auto tile_base = [&](int page, int key) -> size_t { return (size_t)max(page, 0) * page_stride + (size_t)(key & page_mask) * pos_stride; };
            auto load_k = [&](size_t base0, size_t base1, unsigned off) {
#pragma unroll
                for (int k = 0; k < KS; k++) kf[0][k] = ld_at<NT == 1>(kp + base0 + 32 * k, off);     // (a request with one row tile reads its K/V once)
#pragma unroll
                for (int k = 0; k < KS; k++) kf[1][k] = ld_at<NT == 1>(kp + base1 + 32 * k, off);
            };
            auto load_v = [&](size_t base0, size_t base1, unsigned off) {
#pragma unroll
                for (int j = 0; j < VL; j++) vf[j] = ld_at<NT == 1>(vp + (j < VL / 2 ? base0 : base1) + (size_t)(j % (VL / 2) * KEYS) * pos_stride, off);
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
                if (b + NW < b_hi) {
                    nkey = block_key(bl, b + NW);
                    npg0 = page_of(nkey);
                    npg1 = page_of(nkey + 16);
                }
                for (; b < b_hi; b += NW) {
                    // Behind the last block the loads are made all the same, of 16 bytes for all lanes: with no branch around them
                    // the wait for K need not be one for V too.
                    const bool more = b + NW < b_hi;
                    const unsigned k_next = more ? k_off : 0, v_next = more ? v_off : 0;
                    base0 = tile_base(npg0, nkey);
                    base1 = tile_base(npg1, nkey + 16);
                    // is every key of the block visible to every row of the tile?
                    const bool plain = pg0 >= 0 && pg1 >= 0 && all_seen(a, rq.len, key0, 32, pmin, pmax);
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
                        int odd = 0;
#pragma unroll
                        for (int j = 0; j < VL; j++) {
                            const int key = key0 + (j < VL / 2 ? 0 : 16) + v_key + j % (VL / 2) * KEYS;
                            if (!((int)(key < rq.len) & (int)((j < VL / 2 ? pg0 : pg1) >= 0))) vf[j] = frag_t{{0, 0, 0, 0}};
                            odd |= has_odd<T>(vf[j]);
                        }
                        dirty = __any(odd);
                    }
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                    for (int j = 0; j < VL; j++)
                        *reinterpret_cast<frag_t *>(mine + 16 * v_piece<DH>(v_key + j % (8 / KEYS) * KEYS, v_ch) + j / (8 / KEYS) * (8 * DH * 2)) = vf[j];
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    load_v(base0, base1, v_next);
                    frag_t vt[NT > 1 ? CT : 1];                           // held for several row tiles
                    if (NT > 1) {
#pragma unroll
                        for (int c = 0; c < CT; c++) vt[c] = v_operand<DH>(mine, lane, c);
                        if (__builtin_expect(dirty, 0))
#pragma unroll
                            for (int c = 0; c < CT; c++) clear_odd<T>(vt[c]);
                    }

                    // row tiles one after the other, the next one's scores under way in the matrix cores while this one's probabilities are made
#pragma unroll
                    for (int t = 0; t < NT; t++) {
                        if (t + 1 < NT) scores(t + 1);
                        if (NT > 1 && t + 2 == NT) load_k(base0, base1, k_next);
                        f32x4 (&z)[2] = st[t & 1];
                        if (!plain) hide_unseen(z, sight[t], key0, g, pg0, pg1);
                        frag_t pf;
                        probabilities<T, CT, 1>(st + (t & 1), a.sc, ref + t, lsum + t, o + t, &pf);
                        if (__builtin_expect(dirty, 0)) {
                            add_odd<T, DH>(mine, lane, pf, [&](int key) { return sees(sight[t], key0 + key, key & 16 ? pg1 : pg0); }, o[t]);
                            if (NT == 1) {
                                int dl = lane;
                                asm volatile("" : "+v"(dl));
                                for (int j = 0; j < VL; j++) {
                                    frag_t *at = reinterpret_cast<frag_t *>(mine + 16 * (dl + 64 * j)), v = *at;
                                    clear_odd<T>(v);
                                    *at = v;
                                }
                                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                            }
                        }
                        lsum[t] = Num<T>::mfma(ones, pf, lsum[t]);
#pragma unroll
                        for (int c = 0; c < CT; c++) o[t][c] = Num<T>::mfma(NT > 1 ? vt[c] : v_operand<DH>(mine, lane, c), pf, o[t][c]);
                    }
                    key0 = nkey; pg0 = npg0; pg1 = npg1;
                    if (b + 2 * NW < b_hi) {
                        nkey = block_key(bl, b + 2 * NW);
                        npg0 = page_of(nkey);
                        npg1 = page_of(nkey + 16);
                    }
                }
            }

            // ---- the waves' sums become one
            // (the thread's number is hidden from the compiler, which else keeps addresses of this part in registers through the loop)
            int tid = threadIdx.x;
            asm volatile("" : "+v"(tid));
            const int eg = (tid >> 4) & 3, el = tid & 15;
#pragma unroll
            for (int t = 0; t < NT; t++)
                if (eg == 0) stat[wave][t * 16 + el] = float2{ref[t].at, lsum[t][0]};
            const long long place = (2ll * x + (b_lo == 0)) * kv + head;
            // parts of the pair: this piece, where it starts, to the one that holds its last block
            const int parts = whole ? 1 : (int)((piece * x + (min(piece, pl.total - piece * x) - left) - at + cost + nb - 1) / piece) - x + 1;
#pragma unroll
            for (int t = 0; t < NT; t++) {
                __syncthreads();
                {
                    float top = kNone;
#pragma unroll
                    for (int w = 0; w < NW; w++) top = fmaxf(top, stat[w][t * 16 + el].x);
                    const float f = __builtin_amdgcn_exp2f(ref[t].at - top);
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
                        const f32x4 u = *reinterpret_cast<const f32x4 *>(src), v = *reinterpret_cast<const f32x4 *>(src + 4);
#pragma unroll
                        for (int i = 0; i < 4; i++) { sum[i] += u[i]; sum[4 + i] += v[i]; }
                    }
                    l = checked_sum(top, l);
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
            nb = request_blocks(a, rq);
        }
    }
}

// ---- many rows: the waves of a workgroup split the rows and share K and V in LDS ----------------------------------------

// Stages of SK keys, K and V, are loaded through registers into one of two LDS buffers while the other is worked on, one barrier
// per stage; a wave holds NT row tiles for all keys, so nothing has to be merged at the end.  Bound by the matrix cores and the vector
// ALU together, which hardly overlap: 32 keys of a row tile are 17 MFMAs of 16 cycles, and 8 exponentials of 16 and about 20 other
// instructions of 4; scalar instructions count too (half as many of them, by looking 64 stages' pages up at once and comparing a
// stage with ranges that are worked out once, were worth 12 %).  Four requests of 4096 rows at 8192 positions, 32 query heads over 8 of
// 128, take 1.66 to 1.80 ms causal and 2.18 to 2.36 full, from card to card (1008 to 934 TFLOP/s; a library product reaches 1240).

// Where row tiles are too few to fill the chip, pieces of the list of their stages are given out as in paged_attn_kernel.  The stages
// that a tile sees differ from tile to tile, so a launch in front works out where each piece starts: a thread per tile.
template <int DH>
__global__ __launch_bounds__(kPlanTiles) void paged_plan_kernel(PagedAttn a) {
    typedef RowsShape<DH> Shape;
    __shared__ int request_end[kMaxRequests], tile_end[kPlanTiles], sums[kPlanTiles / 64];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    auto scan = [&](int v, int &carry) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(v, o);
            if (lane >= o) v += up;
        }
        if (lane == 63) sums[wave] = v;
        __syncthreads();
        v += carry;
        for (int w = 0; w < kPlanTiles / 64; w++) {
            if (w < wave) v += sums[w];
            carry += sums[w];
        }
        __syncthreads();
        return v;
    };
    auto first_behind = [](const int *ends, int n, int x) {            // first entry above x
        int lo = 0, hi = n - 1;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (ends[mid] > x) hi = mid; else lo = mid + 1;
        }
        return lo;
    };
    int n_tiles = 0;
    for (int r0 = 0; r0 < a.n; r0 += kPlanTiles) {
        const int r = r0 + t, tiles = r < a.n ? min(tiles_of(a, request_of(a, r), Shape::TILE_ROWS), kPlanTiles) : 0, end = scan(tiles, n_tiles);
        if (r < a.n) request_end[r] = end;
    }
    __syncthreads();
    n_tiles = min(n_tiles, kPlanTiles);                                     // (more only if cu_rows does not rise)
    int places = 0, total = 0;
    if (t < n_tiles) {
        const int r = first_behind(request_end, a.n, t);
        const Request q = request_of(a, r);
        int pmin, pmax;
        tile_span(q, a.group, t - (r ? request_end[r - 1] : 0), Shape::TILE_ROWS, pmin, pmax);
        places = max(1, blocks_of<Shape::SHIFT>(a, q.len, pmin, pmax).count) + kTileCost;
    }
    const int end = scan(places, total);
    tile_end[t] = end;
    __syncthreads();
    const int piece = max(kLeastStages + kTileCost, (total + a.split - 1) / a.split);
    for (int x = t; x < a.split; x += kPlanTiles) {
        const long long start = (long long)x * piece;
        int4 p{-1, 0, 0, 0};
        if (start < total) {
            const int y = first_behind(tile_end, n_tiles, (int)start), r = first_behind(request_end, a.n, y);
            p = int4{r, y - (r ? request_end[r - 1] : 0), (int)start - (y ? tile_end[y - 1] : 0), 0};
        }
        a.plan[x] = p;
    }
    if (t == 0) a.plan[a.split] = int4{piece, total, 0, 0};
}

template <class T, int DH>
__global__ __launch_bounds__(256, DH == 64 ? 3 : 2) void paged_rows_kernel(PagedAttn a) {
    typedef RowsShape<DH> Shape;
    constexpr int NT = Shape::NT, SK = Shape::SK, SHIFT = Shape::SHIFT, KS = DH / 32, CT = DH / 16;
    constexpr int WK = SK / 4, KEYS = 512 / DH, LD = WK / KEYS;              // keys that a wave stages; per load; loads each of K and V
    constexpr int BUF = 2 * SK * DH * 2;                                    // bytes of a stage
    extern __shared__ __align__(1024) unsigned char stages[];
    __shared__ __align__(4) unsigned char flags[2][4];                        // of a wave's part of a stage: 1 odd values, 2 in no page

    const int kv = a.pages.n_kv_heads, head = (int)(blockIdx.x % (unsigned)kv), x = (int)(blockIdx.x / (unsigned)kv);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, li = lane & 15;
    const bool split = a.split > 0;
    const int cost = split ? kTileCost : 0;
    // request and tile, the place in the tile's part of the list where this piece starts, and the places that are left
    Request rq;
    int request, tiles, tile, at, left, piece = 1, total = 0;
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
        if (!find_place(a, Shape::TILE_ROWS, false, [&](long long) { return (long long)x; }, pl)) return;
        request = pl.r;
        rq = pl.q;
        tiles = tiles_of(a, rq, Shape::TILE_ROWS);
        tile = tiles - 1 - __builtin_amdgcn_readfirstlane((int)pl.at);      // those that see the most first
        at = 0;
        left = 1;
    }
    const int G = a.group;
    const frag_t ones = {{Num<T>::kOnes, Num<T>::kOnes, Num<T>::kOnes, Num<T>::kOnes}};

    const u16 *kp = (const u16 *)a.pages.k + (size_t)head * a.pages.head_stride, *vp = (const u16 *)a.pages.v + (size_t)head * a.pages.head_stride;
    const int page_mask = (1 << a.page_shift) - 1;
    const size_t pos_stride = a.pages.pos_stride, page_stride = a.pages.page_stride;
    const int s_key = lane / (DH / 8), s_ch = lane % (DH / 8);
    const unsigned s_off = 2u * (s_key * (unsigned)pos_stride + s_ch * 8), s_step = 2u * KEYS * (unsigned)pos_stride;      // bytes
    // LDS addresses of the first stage where a lane writes and reads its pieces.  Those of other keys and channels differ from these by an
    // exclusive or, which takes no register of its own, and a constant.
    typedef __attribute__((address_space(3))) unsigned char *lds_bytes;
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_bytes)stages;               // (a multiple of the keys' size)
    auto lds_frag = [](unsigned at, int more) { return (frag_t *)((lds_bytes)(uintptr_t)at + more); };
    const unsigned k_put = lds0 + 16 * k_piece<DH>(WK * wave + s_key, s_ch), v_put = lds0 + SK * DH * 2 + 16 * v_piece<DH>(WK * wave + s_key, s_ch);
    const unsigned k_get = lds0 + 16 * k_piece<DH>(li, g), v_get = lds0 + SK * DH * 2 + v_lane<DH>(lane, 0);
    for (;;) {
        const int n_rows = rq.m * G, rho0 = (tile * 4 + wave) * 16 * NT;
        int pmin, pmax, wmin, wmax;                                             // positions of the tile's rows and of this wave's
        tile_span(rq, G, tile, Shape::TILE_ROWS, pmin, pmax);
        tile_span(rq, G, tile * 4 + wave, 16 * NT, wmin, wmax);
        const Blocks bl = blocks_of<SHIFT>(a, rq.len, pmin, pmax);
        const int nb = max(1, bl.count), end = split ? min(nb + cost, at + left) : nb;
        const int b_lo = max(0, at - cost), b_hi = min(bl.count, end - cost);
        if (end - cost > b_lo) {
            const bool whole = b_lo == 0 && end - cost == nb;
            const bool idle = rho0 >= n_rows;                                       // (a wave without rows helps to load)
            const int32_t *table = a.tables + (size_t)request * a.columns;
            frag_t q[NT][KS];
            Sight sight[NT];
#pragma unroll
            for (int t = 0; t < NT; t++) {
                const int rho = min(rho0 + t * 16 + li, n_rows - 1), i = rho / G, hq = head * G + (rho - i * G);
                sight[t] = sight_of(a, rq.len, rq.first + i);
                const u16 *src = (const u16 *)a.q + (size_t)(rq.row0 + i) * a.q_row + (size_t)hq * DH + 8 * g;
#pragma unroll
                for (int k = 0; k < KS; k++) q[t][k] = ld_frag(src + 32 * k);
            }
            f32x4 o[NT][CT], lsum[NT];
            Reference ref[NT];
#pragma unroll
            for (int t = 0; t < NT; t++) {
                lsum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < CT; c++) o[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            // Where the keys that this wave stages lie, of 64 stages from `base` on, a stage per lane: elements from the head's part of
            // the pool on, -1 for keys of no page.
            long long places;
            auto find_places = [&](int base) {
                const int b = base + lane, key = block_key<SHIFT>(bl, b) + WK * wave;
                int id = -1;
                if (b < b_hi && key < rq.len) id = table[key >> a.page_shift];
                places = id >= 0 && id < a.pages.n_pages ? id * (long long)page_stride + (key & page_mask) * (long long)pos_stride : -1;
                asm volatile("" : "+v"(places));                                // (the wait for the table is here, not in every stage)
            };
            frag_t kr[LD], vr[LD];
            auto load = [&](int b) -> bool {
                const int i = (b - b_lo) & 63, hi = __builtin_amdgcn_readlane((int)(places >> 32), i);
                const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)places, i);
                const size_t at = hi < 0 ? 0 : (size_t)hi << 32 | lo;
                const rsrc_t k_src = rsrc_of(kp + at), v_src = rsrc_of(vp + at);
#pragma unroll
                for (int j = 0; j < LD; j++) kr[j] = ld_buffer(k_src, s_off, j * s_step);
#pragma unroll
                for (int j = 0; j < LD; j++) vr[j] = ld_buffer(v_src, s_off, j * s_step);
                return hi >= 0;
            };
            // `plain`: every row of the tile sees every key of the stage, as far as there is a page
            auto store = [&](int buf, int key0, bool there, bool plain) {
                unsigned k_at = k_put + buf * BUF, v_at = v_put + buf * BUF;
                asm volatile("" : "+v"(k_at), "+v"(v_at));
                int odd = 0;
                const bool look = !plain || !there;
#pragma unroll
                for (int j = 0; j < LD; j++) {
                    if (look) {
                        if (!((int)(key0 + WK * wave + s_key + j * KEYS < rq.len) & (int)there)) vr[j] = frag_t{{0, 0, 0, 0}};
                        odd |= has_odd<T>(vr[j]);
                    }
                    constexpr int P = KEYS * DH / 8;                            // (pieces of the keys of a load)
                    const int k_turn = 16 * (k_piece<DH>(j * KEYS, 0) - j * P), v_turn = 16 * (v_piece<DH>(j * KEYS, 0) - j * P);
                    *lds_frag(k_at ^ k_turn, 16 * j * P) = kr[j];
                    *lds_frag(v_at ^ v_turn, 16 * j * P) = vr[j];
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
                        const unsigned char *block = stages + 32 * h * DH * 2;
                        frag_t kf[2][KS];
#pragma unroll
                        for (int s = 0; s < 2; s++)
#pragma unroll
                            for (int k = 0; k < KS; k++) kf[s][k] = *lds_frag(k_at ^ (unsigned)(k << 6), (32 * h + 16 * s) * DH * 2);
                        f32x4 z[NT][2];
#pragma unroll
                        for (int t = 0; t < NT; t++)
#pragma unroll
                            for (int s = 0; s < 2; s++) {
                                z[t][s] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                                for (int k = 0; k < KS; k++) z[t][s] = Num<T>::mfma(kf[s][k], q[t][k], z[t][s]);
                            }
                        frag_t vt[CT];
#pragma unroll
                        for (int c = 0; c < CT; c++) vt[c] = v_operand_at((const unsigned char *)lds_frag(v_at ^ (unsigned)(c << 5), 32 * h * DH * 2), 16 * DH * 2);
                        // (a 16-key tile lies in one page; its flags are those of the first wave that stages it)
                        const uint32_t fl = (uint32_t)__builtin_amdgcn_readfirstlane((int)flag_word);
                        const bool dirty = (fl & 0x01010101u) != 0;
                        const int pg0 = -(int)(fl >> (8 * (2 * h * 16 / WK)) & 2), pg1 = -(int)(fl >> (8 * ((2 * h + 1) * 16 / WK)) & 2);
                        const bool masked = (pg0 | pg1) != 0 || !(plain || all_of(all, key32, 32));
                        if (__builtin_expect(dirty, 0))
#pragma unroll
                            for (int c = 0; c < CT; c++) clear_odd<T>(vt[c]);
                        if (masked)
#pragma unroll
                            for (int t = 0; t < NT; t++) hide_unseen(z[t], sight[t], key32, g, pg0, pg1);
                        frag_t pf[NT];
                        probabilities<T, CT, NT>(z, a.sc, ref, lsum, o, pf);
                        if (__builtin_expect(dirty, 0))
#pragma unroll
                            for (int t = 0; t < NT; t++)
                                add_odd<T, DH>(block + buf * BUF + SK * DH * 2, lane, pf[t], [&](int key) { return sees(sight[t], key32 + key, key & 16 ? pg1 : pg0); }, o[t]);
#pragma unroll
                        for (int t = 0; t < NT; t++) {
                            lsum[t] = Num<T>::mfma(ones, pf[t], lsum[t]);
#pragma unroll
                            for (int c = 0; c < CT; c++) o[t][c] = Num<T>::mfma(vt[c], pf[t], o[t][c]);
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
            const int parts = whole ? 1 : (piece * x + (min(piece, total - piece * x) - left) - at + cost + nb - 1) / piece - x + 1;
#pragma unroll
            for (int t = 0; t < NT; t++) {
                const int in_tile = wave * 16 * NT + t * 16 + (tid & 15), rho = tile * Shape::TILE_ROWS + in_tile, eg = (tid >> 4) & 3;
                if (rho >= n_rows) continue;
                const int i = rho / G, hq = head * G + (rho - i * G);
                const float l = checked_sum(ref[t].at, lsum[t][0]);
                if (!whole) {
                    const long long place = ((2ll * x + (b_lo == 0)) * kv + head) * Shape::TILE_ROWS + in_tile;
#pragma unroll
                    for (int c = 0; c < CT; c++) *reinterpret_cast<f32x4 *>(a.partial + place * DH + c * 16 + 4 * eg) = o[t][c];
                    if (eg == 0) {
                        a.ml[place] = float2{ref[t].at, l};
                        if (b_lo == 0) a.where[(size_t)(rq.row0 + i) * a.heads + hq] = int2{x, parts * kRowsPlace + in_tile};
                    }
                    continue;
                }
                const float f = l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l;          // a row that sees nothing is zero
#pragma unroll
                for (int c = 0; c < CT; c++)
                    store_out4(a, rq.row0 + i, hq, DH, c * 16 + 4 * eg, uint2{Num<T>::pack(o[t][c][0] * f, o[t][c][1] * f), Num<T>::pack(o[t][c][2] * f, o[t][c][3] * f)});
                if (split && eg == 0) a.where[(size_t)(rq.row0 + i) * a.heads + hq] = int2{x, 0};
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

// Adds the parts of a row in order, WPR waves per (row, head) with a part each in turn.  Rows that belong to no request are left alone.
// Bound by its dependent reads: 2048 rows of mostly one part 4.6 us, 64 rows of 32 parts 4.9.
template <class T, int DH, int WPR>
__global__ __launch_bounds__(WPR == 16 ? 1024 : 256) void paged_join_kernel(PagedAttn a) {
    constexpr int V = DH / 64, ROWS = WPR == 16 ? 1 : 4 / WPR;          // channels of a lane, rows of a workgroup
    __shared__ float sums[ROWS][WPR][DH];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = wave / WPR, w = wave % WPR;
    const long long unit = (long long)blockIdx.x * ROWS + sub;
    const int row = (int)(unit / a.heads), hq = (int)(unit % a.heads);
    int2 at{0, 0};
    bool mine = row < a.rows;
    if (mine) {
        at = a.where[(size_t)row * a.heads + hq];
        mine = !a.cu_rows || (row >= a.cu_rows[0] && row < a.cu_rows[a.n]);
    }
    const int parts = at.y / kRowsPlace, r = at.y % kRowsPlace, kv = a.pages.n_kv_heads, head = hq / a.group;
    mine = mine && parts > 1 && r < a.tile_rows && at.x >= 0 && (long long)at.x + parts <= a.split;
    auto place = [&](int p) { return ((size_t)(2ll * (at.x + p) + (p == 0)) * kv + head) * a.tile_rows + r; };
    float top = -INFINITY, total = 0.f, acc[V];
#pragma unroll
    for (int i = 0; i < V; i++) acc[i] = 0.f;
    if (mine) {
        // the first parts' O are on their way while the references and sums are looked at, a part per lane
        constexpr int AHEAD = 4;
        float first[AHEAD][V];
#pragma unroll
        for (int j = 0; j < AHEAD; j++) {
            const float *src = a.partial + place(min(w + j * WPR, parts - 1)) * DH + lane * V;
#pragma unroll
            for (int i = 0; i < V; i++) first[j][i] = src[i];
        }
        const float2 s0 = a.ml[place(min(lane, parts - 1))];
        top = s0.x;
        for (int p = lane + 64; p < parts; p += 64) top = fmaxf(top, a.ml[place(p)].x);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        const float f0 = __builtin_amdgcn_exp2f(s0.x - top);
        if (lane < parts) total = s0.y * f0;
        for (int p = lane + 64; p < parts; p += 64) {
            const float2 s = a.ml[place(p)];
            total += s.y * __builtin_amdgcn_exp2f(s.x - top);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
#pragma unroll
        for (int j = 0; j < AHEAD; j++) {
            const int p = w + j * WPR;
            const float f = __shfl(f0, p);                             // (p < 64)
            if (p < parts)
#pragma unroll
                for (int i = 0; i < V; i++) acc[i] += first[j][i] * f;
        }
#pragma unroll 4
        for (int p = w + AHEAD * WPR; p < parts; p += WPR) {
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
#pragma unroll 4
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

template <class T, int DH>
void launch_join(const PagedAttn &a, hipStream_t s) {
    // parts of a row, where the lengths are equal
    const long long units = (long long)a.rows * a.heads, parts = a.split / a.tiles;
    if (parts > 16) paged_join_kernel<T, DH, 16><<<dim3((unsigned)units), 1024, 0, s>>>(a);
    else if (parts > 4) paged_join_kernel<T, DH, 4><<<dim3((unsigned)units), 256, 0, s>>>(a);
    else paged_join_kernel<T, DH, 1><<<dim3((unsigned)((units + 3) / 4)), 256, 0, s>>>(a);
}

template <class T, int DH, int NT>
void launch_nt(const PagedAttn &a, hipStream_t s) {
    paged_attn_kernel<T, DH, NT><<<dim3((unsigned)(a.items * a.pages.n_kv_heads)), 256, 0, s>>>(a);
    if (!a.split) return;
    launch_join<T, DH>(a, s);
}

template <class T, int DH>
void launch_rows(const PagedAttn &a, hipStream_t s) {
    constexpr int bytes = 2 * 2 * RowsShape<DH>::SK * DH * 2;
    allow_lds<paged_rows_kernel<T, DH>>(bytes);
    if (a.split) paged_plan_kernel<DH><<<dim3(1), kPlanTiles, 0, s>>>(a);
    paged_rows_kernel<T, DH><<<dim3((unsigned)(a.items * a.pages.n_kv_heads)), 256, bytes, s>>>(a);
    if (a.split) launch_join<T, DH>(a, s);
}

template <class T, int DH>
void launch_dim(const PagedAttn &a, int nt, hipStream_t s) {
    if (nt == kManyRows) return launch_rows<T, DH>(a, s);
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
inline int many_rows(const odb_pages &p) { return p.head_dim == 256 ? RowsShape<256>::TILE_ROWS : RowsShape<128>::TILE_ROWS; }

}  // namespace

void paged_attn_plan(const odb_pages &p, int n, int rows, int group, int max_rows, long long max_len, long long columns, int *nt, int *split,
                     long long *items) {
    const long long most = (long long)max_rows * group;
    // Every request has at most one row tile that is not full.
    auto tiles = [&](int tile_rows) { return (long long)(n < rows ? n : rows) + (long long)rows * group / tile_rows; };
    auto numbers = [&](int tile_rows) { return (n + (long long)rows * group / tile_rows) | 1; };      // (find_place; odd: no pattern survives)
    // Tiles of many rows, where more than half of one is full: whole if there is one for every CU, in pieces if fewer see long keys, or if
    // there may be requests whose lengths differ and leave CUs waiting for the longest.  Else the waves split the keys of smaller tiles,
    // which need cuts of their own if they are not far more than the CUs.  Whole / pieces / keys split by waves, us; full attention, 32
    // query heads over 8 of 128:
    //   rows of positions    512 of 512  21 / 35 / 19    600 of 600  25 / 42 / 39    704 of 2000  60 / 59 / 73    704 of 5000  130 / 95 / 127
    //                        256 of 2048 57 / 53 / 33    512 of 4096 107 / 68 / 63   512 of 8192  203 / 105 / 114  300 of 12000 295 / 113 / 117
    //   requests x rows      32 x 24 of 4000  114 / 126 / 135      64 x 24 of 300 to 5000  149 / 109 / 162      8 x 24 of 2000  58 / 38 / 39
    // 32 heads over 32: 8 x 80 of 700  28 / 44 / 43, 8 x 80 of 2000  63 / 76 / 81
    // Lengths themselves are not known here, so `ragged` is a guess: that requests of up to 64 stages are of like lengths, and longer ones
    // are not.  Whole / pieces where it is right and where it is not: 32 x 24 rows of 300 to 5000 115 / 64, of 8000 each 216 / 215, of 5000 each
    // 143 / 151, of 300 to 3600 93 / 56; 64 x 24 of 1000 to 8000 253 / 199, of 5000 each 241 / 249, of 300 to 3600 114 / 98.
    const int many = many_rows(p), keys = p.head_dim == 256 ? RowsShape<256>::SK : RowsShape<128>::SK;
    const long long likely = min(tiles(many), (long long)n * ((most + many - 1) / many));      // (max_rows may not hold)
    const long long groups = likely * p.n_kv_heads, stages = (max_len + keys - 1) / keys;
    if (2 * most > many) {
        // more of the smaller tiles than CUs
        const bool crowded = (long long)rows * group / (many / 2) * p.n_kv_heads > 256;
        // (the plan's sums are 32-bit, by the tables' columns: max_len may not hold)
        const bool fits = tiles(many) <= kPlanTiles && tiles(many) * (columns * p.page_size / keys + 8) < 1 << 30;
        const bool ragged = n > 1 && groups < 1024 && stages >= 64;
        const bool whole = groups >= 256 ? !(ragged && fits) : (crowded && stages <= 32) || (groups >= 128 && stages <= 12);
        const int pieces = (512 + p.n_kv_heads - 1) / p.n_kv_heads;
        if (whole || (fits && (groups >= 256 || likely * stages >= (crowded ? 12ll : 20ll) * pieces))) {
            *nt = kManyRows;
            *split = whole ? 0 : pieces;
            *items = whole ? numbers(many) : pieces;
            return;
        }
    }
    *nt = most <= 16 ? 1 : most <= 32 || p.head_dim == 256 ? 2 : 4;
    // One round of workgroups, two per CU where a tile is 16 rows (one / two / four: 64 single tokens over 555 MB 96 / 97 / 100 us, two over
    // 985 MB 152 / 154 / 157, 48 of 17 to 16384 positions over 32 heads 194 / 192 / 188); with more rows every cut costs more sums (8 x 32 rows
    // of 500 to 3000: 50 / 52 / 57).
    const int aim = (256 * (*nt == 1 && p.head_dim != 256 ? 2 : 1) + p.n_kv_heads - 1) / p.n_kv_heads;
    // Where the bound on the row tiles, which counts one more than the full ones for every request, is four of that round the keys stay
    // whole, and a tile reads only those that it sees.  Short keys are not worth the cuts and the join either.  Whole / pieces:
    //   equal lengths     64 single tokens of 2000, 32 heads over 32  333 / 326 us    16 x 32 rows of 1500  77 / 83    32 x 32 of 1500  147 / 158
    //   blocks, ragged    16 x 32 rows of 500 to 3000, 32 heads over 32  71 / 70       32 x 32  137 / 138
    //   tokens, ragged    64 of 17 to 16384, 32 heads over 32  457 / 284               256, 32 over 8  663 / 397
    // The last line is what this rule, which does not know the lengths, gives away: all workgroups of such a call run at once, and the longest
    // request sets its time.  Short keys, 32 heads over 8 of 128: 4 single tokens of 600 positions 14.2 / 15.8, 4 of 800 16.1 / 14.8, 16 of 800
    // 19.0 / 21.3, 32 of 1000 25.6 / 31.3, 65 of 1000 60 / 54; 4 x 32 rows of 1000, 32 heads over 32, 19.7 / 23.8.
    const int tile_rows = 16 * *nt;
    const long long pairs = min(tiles(tile_rows), (long long)n * ((most + tile_rows - 1) / tile_rows)) * p.n_kv_heads;
    const long long channels = (max_len + 31) / 32 * p.head_dim;
    const bool brief = channels <= 20 * 128 || (pairs >= 96 && pairs <= 512 && channels <= 32 * 128);
    *split = tiles(tile_rows) >= 4 * aim || brief ? 0 : aim;
    *items = *split ? *split : numbers(tile_rows);
}

// Half the bytes a key, and whole tiles of up to 64 requests are given out longest first.  nt, and many rows whole or in pieces, as above (whole longest first /
// pieces, us, 32 heads over 8 of 128 where nothing else is said: four pieces of prompts, 727 to 1449 rows of 2694 to 5995 positions, 304 / 321, in order of the
// requests 392; 32 x 24 rows of 300 to 5000 158 / 63, 100 x 24 212 / 157, 64 x 24 of 1000 to 8000 256 / 170, of 5000 each 219 / 229; 40 x 40 of 300 to 8000 250 /
// 131, 60 x 48 of 1000 to 6000 225 / 253; 2 x 1500 of 5000 to 9000 262 / 193, 3 x 900 338 / 351; 64 heads over 8 of 64, 32 x 12 of 300 to 5000 115 / 50; 16 over 2 of
// 256, 130 x 8 190 / 84).
// Where a last round of whole tiles' workgroups would hold a few only, these are cut, which costs a join and its workspace (three of 503 to 997 rows under a
// window of 900, 526 tiles and 512 workgroups at once: 83 / 107 us uncut; four pieces, two full rounds: 319 / 304).  Full rounds have nothing to cut (2048 rows of as
// many positions 79 us, 86 with the join; 4096 203, 218; 8192 688, 716).
// Few rows: cuts for two workgroups a CU with 32 rows too (8 x 32 rows of 500 to 3000, 32 heads over 32: 45 us, one 53); whole where the pairs are enough and
// the keys up to 1536, up to 768 with heads of 256 (whole / pieces, 32 heads over 32: 10 x 32 rows of 454 to 1364 24 / 31, of 900 to 1500 28 / 34, 14 x 32 of
// 1490 to 1500 41 / 53, 8 x 48 of 1400 to 1500 38 / 40; longer ones, 64 heads over 8 of 64, 20 x 4 rows of 300 to 3000 31 / 20, 40 x 4 of 1000 to 3000 34 / 32).
void paged_attn_quant_plan(const odb_pages &p, int n, int rows, int group, int max_rows, long long max_len, long long columns, int *nt, int *split,
                           long long *items, int *slots) {
    paged_attn_plan(p, n, rows, group, max_rows, max_len, columns, nt, split, items);
    *slots = 0;
    const int tile_rows = *nt == kManyRows ? many_rows(p) : 16 * *nt;
    const long long most = (long long)max_rows * group, full = (long long)rows * group / tile_rows, numbers = (n + full) | 1;
    const long long tiles = min((n < rows ? n : rows) + full, (long long)n * ((most + tile_rows - 1) / tile_rows)), pairs = tiles * p.n_kv_heads;
    if (*nt == kManyRows) {
        if (*split || pairs < 256) return;
        const int at_once = (512 + p.n_kv_heads - 1) / p.n_kv_heads;
        const long long over = tiles % at_once;
        if (n <= 64 && full >= at_once && full / at_once == tiles / at_once && over > 0 && 2 * over <= at_once && tiles <= 4ll * at_once) {
            *slots = *split = at_once;
            *items = (n < rows ? n : rows) + full + at_once;                   // (of all tiles that there can be: max_rows may not hold)
        }
        return;
    }
    if (!*split) return;
    if (*nt > 1 && n <= 64 && pairs >= 160 && pairs <= 512 && (max_len + 31) / 32 * max(p.head_dim, 128) <= 48 * 128) {
        *split = 0;
        *items = numbers;
    } else if (*nt == 2 && p.head_dim != 256) {
        *split = *items = (512 + p.n_kv_heads - 1) / p.n_kv_heads;
    }
}

size_t paged_attn_workspace(const odb_pages &p, int rows, int heads, int nt, int split) {
    if (!split) return 0;
    const size_t tile_rows = 2 * (size_t)split * p.n_kv_heads * (nt == kManyRows ? many_rows(p) : nt * 16);
    return up256(tile_rows * p.head_dim * 4) + up256(tile_rows * 8) + up256((size_t)rows * heads * 8) + up256(((size_t)split + 1) * 16);
}

void paged_attn_setup(PagedAttn &a, int nt, void *workspace) {
    a.tile_rows = nt == kManyRows ? many_rows(a.pages) : nt * 16;
    a.tiles = (int)max(1ll, (long long)min(a.n, a.rows) + (long long)a.rows * a.group / a.tile_rows);
    if (!a.split && a.cu_rows && a.n > kLookAtAll) {                       // far apart, and every item once: no common divisor
        auto common = [](long long x, long long y) { while (y) { const long long z = x % y; x = y; y = z; } return x; };
        for (a.stride = a.items * 0.618; a.stride > 1 && common(a.items, a.stride) > 1;) a.stride--;
    }
    if (a.split > 0) {
        const size_t tile_rows = 2 * (size_t)a.split * a.pages.n_kv_heads * a.tile_rows;
        char *w = (char *)workspace;
        auto take = [&](size_t bytes) { char *p = w; w += up256(bytes); return p; };
        a.partial = (float *)take(tile_rows * a.pages.head_dim * 4);
        a.ml = (float2 *)take(tile_rows * 8);
        a.where = (int2 *)take((size_t)a.rows * a.heads * 8);
        a.plan = (int4 *)take(((size_t)a.split + 1) * 16);
    }
}

void launch_paged_attention(PagedAttn a, int nt, void *workspace, hipStream_t s) {
    if (a.rows < 1) return;
    paged_attn_setup(a, nt, workspace);
    if (a.pages.dtype == ODB_F16) launch_type<_Float16>(a, nt, s);
    else launch_type<__bf16>(a, nt, s);
}

void launch_paged_attention_quant(PagedAttnQuant a, int nt, void *workspace, hipStream_t s) {
    if (a.rows < 1) return;
    paged_attn_setup(a, nt, workspace);
    if (a.scales.codes == ODB_INT8) launch_paged_attention_int8(a, nt, s);
    else launch_paged_attention_e4m3(a, nt, s);
}

void launch_paged_join(const PagedAttn &a, hipStream_t s) {
    const bool f16 = a.pages.dtype == ODB_F16;
    switch (a.pages.head_dim) {
    case 64: return f16 ? launch_join<_Float16, 64>(a, s) : launch_join<__bf16, 64>(a, s);
    case 128: return f16 ? launch_join<_Float16, 128>(a, s) : launch_join<__bf16, 128>(a, s);
    default: return f16 ? launch_join<_Float16, 256>(a, s) : launch_join<__bf16, 256>(a, s);
    }
}

void launch_paged_plan(const PagedAttn &a, hipStream_t s) {
    switch (a.pages.head_dim) {
    case 64: return paged_plan_kernel<64><<<dim3(1), kPlanTiles, 0, s>>>(a);
    case 128: return paged_plan_kernel<128><<<dim3(1), kPlanTiles, 0, s>>>(a);
    default: return paged_plan_kernel<256><<<dim3(1), kPlanTiles, 0, s>>>(a);
    }
}

}  // namespace odb
