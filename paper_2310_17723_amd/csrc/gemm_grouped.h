// What the kernels of products grouped by expert share: their arguments, and which rows of which expert a tile holds.
#pragma once
#include <math.h>
#include "gemm_common.h"

namespace hero_gemm {

constexpr int MAX_EXPERTS = 512;

// GemmArgs with g.M = R (rows of C); Bt, b_col_scale, bias and out_col_scale are expert 0's
struct GroupedArgs {
    GemmArgs g;
    const int32_t* offsets; const int32_t* row_index;
    int E, MA;                                  // experts, rows of A
    int64_t expert_stride;                      // bytes between the weights of two experts
    int epi, c_dt;                              // (for the kernel that asks at run time)
};

// what a kernel takes that has a grouped form
template <bool GROUPED> struct ArgsOf { using type = GemmArgs; };
template <> struct ArgsOf<true> { using type = GroupedArgs; };
__device__ __forceinline__ const GemmArgs& gemm_of(const GemmArgs& g) { return g; }
__device__ __forceinline__ const GemmArgs& gemm_of(const GroupedArgs& a) { return a.g; }
__device__ __forceinline__ bool source_is_gathered(const GemmArgs&) { return false; }
__device__ __forceinline__ bool source_is_gathered(const GroupedArgs& a) { return a.row_index != nullptr; }

// inclusive sum over the lanes of a wave
__device__ __forceinline__ int wave_scan_sum(int x) {
#define HERO_SHR(n) x += __builtin_amdgcn_update_dpp(0, x, 0x110 + n, 0xF, 0xF, true)
    HERO_SHR(1); HERO_SHR(2); HERO_SHR(4); HERO_SHR(8);         // row_shr within 16 lanes
#undef HERO_SHR
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);   // lane 15 of rows 0, 2 into rows 1, 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);   // lane 31 into rows 2, 3
    return x;
}
__device__ __forceinline__ int wave_scan_max(int x, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int y = __shfl_up(x, o); if (lane >= o) x = max(x, y); }
    return x;
}

// One piece of 64 experts, an expert to a lane: its rows [begin, end).  Offsets outside [0, R] and falling ones are taken as the largest
// up to them (`carry`: the end of the piece in front), so that whatever is handed over the rows lie within [0, R] and no row has two experts.
__device__ __forceinline__ void expert_rows(const GroupedArgs& a, int e0, int lane, int carry, int& begin, int& end) {
    const int e = e0 + lane, R = a.g.M;
    const int lo = a.offsets[min(e, a.E)], hi = a.offsets[min(e + 1, a.E)];
    begin = min(max(lo, 0), R);
    end = min(max(hi, 0), R);
    if (__ballot(end < begin || begin < carry)) {               // (rare)
        begin = wave_scan_max(max(begin, carry), lane);
        end = max(end, begin);
    }
}

// Rows of a tile: [row0, row0 + rows) of expert e; rows == 0: there is no such tile
struct GroupTile { int e, row0, rows, col_tile; };

// Tile `slot` of this XCD's share.  Tiles of BM rows; those of an expert lie together, and of them the row tiles of one column tile (they read the
// same weights).  Every XCD takes a contiguous range of the list.  Every lane of the wave calls it, and `slot` is uniform.
template <int BM>
__device__ __forceinline__ GroupTile group_tile(const GroupedArgs& a, int xcd, int slot, int ntn, int lane) {
    constexpr int PIECES = MAX_EXPERTS / 64;
    int begin[PIECES], end[PIECES], upto[PIECES], carry = 0, tiles = 0;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        begin[p] = end[p] = 0; upto[p] = 0;
        if (p * 64 < a.E) {
            expert_rows(a, p * 64, lane, carry, begin[p], end[p]);
            upto[p] = tiles + wave_scan_sum((end[p] - begin[p] + BM - 1) / BM);
            carry = __builtin_amdgcn_readlane(end[p], 63);
            tiles = __builtin_amdgcn_readlane(upto[p], 63);
        }
    }
    const int per = (int)(((int64_t)tiles * ntn + NUM_XCD - 1) / NUM_XCD);
    const int64_t seq = (int64_t)xcd * per + slot;
    GroupTile t{0, 0, 0, 0};
    if (slot >= per || seq >= (int64_t)tiles * ntn) return t;
    const int at = (int)(seq / ntn);                            // the expert is the first whose tiles reach beyond this row tile
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        if (p * 64 < a.E && t.rows == 0) {
            const unsigned long long beyond = __ballot(upto[p] > at);
            if (beyond) {
                const int l = __ffsll(beyond) - 1;
                const int b = __builtin_amdgcn_readlane(begin[p], l), n = __builtin_amdgcn_readlane(end[p], l) - b, mt = (n + BM - 1) / BM;
                const int first = __builtin_amdgcn_readlane(upto[p], l) - mt;
                const int64_t in = seq - (int64_t)first * ntn;
                const int m = (int)(in % mt);
                t.e = p * 64 + l; t.col_tile = (int)(in / mt);
                t.row0 = b + m * BM; t.rows = min(BM, n - m * BM);
            }
        }
    }
    return t;
}

// The tables of the tile kernels (in LDS, whole waves): row_begin [E + 1], tiles_upto [E] filled up to a multiple of 64 with the number of all
// row tiles, which is returned.  Tiles have `height` rows.
__device__ __forceinline__ int expert_tables(const GroupedArgs& a, int height, int* row_begin, int* tiles_upto, int lane) {
    int carry = 0, tiles = 0;
    for (int e0 = 0; e0 < a.E; e0 += 64) {
        int begin, end;
        expert_rows(a, e0, lane, carry, begin, end);
        const int upto = tiles + wave_scan_sum((end - begin + height - 1) / height);
        if (e0 + lane <= a.E) row_begin[e0 + lane] = begin;
        if (e0 + lane + 1 == a.E) row_begin[a.E] = end;
        tiles_upto[e0 + lane] = upto;
        carry = __builtin_amdgcn_readlane(end, 63);
        tiles = __builtin_amdgcn_readlane(upto, 63);
    }
    return tiles;
}

// What a tile of one to four quarters of the rows of 256 costs: its weights come in whole.  us, 1024 rows to each of eight experts x 4096 x 4096 in tiles of
// 64, 128, 192, 256 rows: INT8 250, 166, 135, 118, BF16 535, 305, 255, 219.  256 x 128 tiles go by the same figures: 8 experts of so many rows x 8192 x 4096, in % of the
// time with 256 rows, BF16 64, 77, 90, INT8 62, 77, 89 and E4M3 61, 74, 92, though that multiplies 128 rows at a time (the ones behind the last are that row again, which costs
// little power).  E4M3 256 x 128 held to heights of 128 and 256: over the 60 of the problems drawn where that changes the height 192 rows became 4.8 % slower, 64 as fast.
constexpr int GROUPED_COST[4] = {59, 76, 92, 100};
// The height at which the busiest workgroup has the least to do: the rows of the experts, which are known here only, make a number of tiles that the
// workgroups take in turn.  us, 256 rows always / this: INT8 3200 rows of 8 experts x 4096 x 4096 101 / 83, 6400 rows of 16 x 1024 x 4096 51 / 45.  (The last
// tiles of a workgroup cut into pieces instead, so that all of them end together: no gain, and 8192 rows of 8 experts x 4096 x 16384 517 -> 544: what idles
// at the end leaves the others its power.)
template <int BM>
__device__ __forceinline__ int best_height(const GroupedArgs& a, int workgroups, int lane) {
    int carry = 0, tiles[4] = {0, 0, 0, 0};
    for (int e0 = 0; e0 < a.E; e0 += 64) {
        int begin, end;
        expert_rows(a, e0, lane, carry, begin, end);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            constexpr int H = BM / 4;
            tiles[q] += __builtin_amdgcn_readlane(wave_scan_sum((end - begin + (q + 1) * H - 1) / ((q + 1) * H)), 63);
        }
        carry = __builtin_amdgcn_readlane(end, 63);
    }
    int best = 3;
    int64_t least = INT64_MAX;
#pragma unroll
    for (int q = 3; q >= 0; --q) {
        const int64_t cost = ((int64_t)tiles[q] * a.g.ntn + workgroups - 1) / workgroups * GROUPED_COST[q];
        if (cost < least) { least = cost; best = q; }
    }
    return (best + 1) * (BM / 4);
}

// Tile number s: rows [m0, end) of expert e.  Eight row tiles of an expert run through its columns together (tile_from_seq's order).
struct ExpertTile { int e, m0, end, col_tile; };
__device__ __forceinline__ ExpertTile expert_tile(const GroupedArgs& a, int height, const int* row_begin, const int* tiles_upto, int s, int lane) {
    const int ntn = a.g.ntn, at = s / ntn;
    int e0 = 0;
    unsigned long long beyond = __ballot(tiles_upto[lane] > at);
    while (!beyond) { e0 += 64; beyond = __ballot(tiles_upto[e0 + lane] > at); }       // (s is a tile: there is one)
    const int e = e0 + __ffsll(beyond) - 1;
    const int first = __builtin_amdgcn_readfirstlane(e ? tiles_upto[e - 1] : 0), mt = __builtin_amdgcn_readfirstlane(tiles_upto[e]) - first;
    const int begin = __builtin_amdgcn_readfirstlane(row_begin[e]), in = s - first * ntn;
    const int grp = in / (GROUP_M * ntn), rem = in - grp * (GROUP_M * ntn), rows = min(mt - grp * GROUP_M, GROUP_M);
    ExpertTile t;                               // (uniform, and said to be: the addresses of the direct loads are scalars)
    t.e = __builtin_amdgcn_readfirstlane(e);
    t.m0 = __builtin_amdgcn_readfirstlane(begin + (grp * GROUP_M + rem % rows) * height);
    t.end = __builtin_amdgcn_readfirstlane(min(row_begin[e + 1], t.m0 + height));
    t.col_tile = __builtin_amdgcn_readfirstlane(rem / rows);
    return t;
}

// The most tiles of BM rows that R rows of E experts can make
inline int64_t most_row_tiles(int64_t R, int64_t E, int BM) {
    return (R + (E < R ? E : R) * (BM - 1)) / BM;
}

// Which kernel: the numbers of include/hero_debug.h (hero_gemm_grouped_tile)
enum GroupedForm { GROUPED_ANY = 1, GROUPED_RING = 16 /* + RingForm */, GROUPED_128 = 128, GROUPED_256 = 256, GROUPED_256x128 = 384 };
// gemm_grouped_rows.hip: every size
hero_status launch_grouped_rows(const GroupedArgs& a, hero_dtype adt, hipStream_t st);
// gemm_ring.h: one tile per workgroup
template <int ADT, int EPI, int CDT> hero_status launch_grouped_ring(const GroupedArgs& a, RingForm f, hipStream_t st);
// gemm_persistent.h: tiles of 256 x 256, 256 x 128 or 128 x 128
template <int ADT, int EPI, int CDT> hero_status launch_grouped_tile(const GroupedArgs& a, int tile, hipStream_t st);
// The sizes that the ring kernel takes: whole slabs, and 32-bit offsets per lane (of a tile's rows, or of all rows that may be gathered)
inline bool grouped_ring_ok(const GroupedArgs& a) {
    return a.g.K % (2 * BK) == 0 && ring_ok(a.g.lda, a.g.ldb) && (!a.row_index || (int64_t)a.MA * a.g.lda <= (1LL << 32));
}
// .. and the persistent kernel, which looks ahead
inline bool grouped_tile_ok(const GroupedArgs& a) { return grouped_ring_ok(a) && a.g.K >= 8 * BK; }

// The choice goes by an estimate of each form's time (us) from what the host knows: a round of tiles takes start + slab times the 128-byte slabs of K, a first one
// that fills the slots to r only alone + (1 - alone) r of that, a last one between that and its share; the weights of the experts that can have a row come at 5.4 TB/s, and
// the lesser of the two times shows to 15 %.  Fitted, a form at a time, to 770 problems of 1 to 32768 rows, 2 to 256 experts, every type, drawn at random, weights from memory.  Over 180
// others the choice takes 1.014 times the best form's time (1.33 at most), over 270 of 40 to 700 rows an expert 1.031 (1.39); by the number of tiles to a CU alone 1.021 and 1.044.
struct FormTime { int form, bm, bn, slots; struct { float start, slab, alone; } few, many; };      // (few: up to 32 rows an expert)
constexpr FormTime FORM_TIMES[] = {
    {GROUPED_RING + RING_32x32_K4, 32, 32, 256, {3.94f, 0.098f, 0.78f}, {3.92f, 0.096f, 0.80f}},
    {GROUPED_RING + RING_32x64_K2, 32, 64, 256, {3.80f, 0.186f, 0.81f}, {3.60f, 0.182f, 0.85f}},
    {GROUPED_RING + RING_64x64_K2, 64, 64, 256, {4.05f, 0.219f, 0.76f}, {3.96f, 0.224f, 0.75f}},
    {GROUPED_RING + RING_64x64, 64, 64, 768, {4.89f, 0.458f, 0.49f}, {2.93f, 0.693f, 0.36f}},
    {GROUPED_RING + RING_128x64, 128, 64, 512, {4.93f, 0.492f, 0.58f}, {3.71f, 0.692f, 0.43f}},
    {GROUPED_128, 128, 128, 512, {3.67f, 1.054f, 0.48f}, {4.23f, 1.191f, 0.43f}},
    {GROUPED_256, 256, 256, 256, {}, {9.93f, 1.513f, 0.73f}},
    {GROUPED_256x128, 256, 128, 256, {}, {5.70f, 0.928f, 1.00f}}};
inline int grouped_form(const GroupedArgs& a) {
    if (!grouped_ring_ok(a)) return GROUPED_ANY;
    const bool tile_ok = grouped_tile_ok(a);
    const int R = a.g.M, N = a.g.N, active = a.E < R ? a.E : R;
    // experts are not equal: eight of them have 0.3, 0.5, .. 1.7 times the rows that each would have
    int of_eight[9] = {};                                           // their row tiles of 32, 64, 128, 192 and 256 rows, by 32 rows
    for (int i = 3; i <= 17; i += 2) {
        const int rows = (int)(((int64_t)R * i + 10 * active - 1) / (10 * active)), t64 = (rows + 63) >> 6;
        of_eight[1] += (rows + 31) >> 5;
        of_eight[2] += t64;
        of_eight[4] += (t64 + 1) >> 1;
        of_eight[6] += (t64 + 2) / 3;
        of_eight[8] += (t64 + 3) >> 2;
    }
    auto tiles = [&](int bm, int bn) {
        const float some = (float)of_eight[bm >> 5] * (float)active / 8, most = (float)((R + active * (bm - 1)) / bm), t = some < most ? some : most;
        return (t > 1 ? t : 1) * (float)((N + bn - 1) / bn);
    };
    const float slabs = (float)(a.g.K / (2 * BK)), stream = (float)active * (float)N * (float)a.g.K / 5.4e6f;
    int best = GROUPED_ANY;
    float least = INFINITY;
    const bool few = R / active <= 32;
    for (const FormTime& f : FORM_TIMES) {
        if ((f.form >= GROUPED_128 && !tile_ok) || (f.bm == 256 && few)) continue;
        const float start = few ? f.few.start : f.many.start, slab = few ? f.few.slab : f.many.slab, alone = few ? f.few.alone : f.many.alone;
        float time = INFINITY;
        for (int q = f.bm == 256 ? 0 : 3; q < 4; ++q) {             // (best_height())
            const float r = tiles(f.bm / 4 * (q + 1), f.bn) / (float)f.slots;
            if (f.form < GROUPED_RING + RING_64x64 && r > 1) continue;      // K groups: one round
            const float rounds = r <= 1 ? alone + (1 - alone) * r : r + 0.6f * alone * (ceilf(r) - r);
            const float t = rounds * (start + slab * slabs) * (f.bm == 256 ? GROUPED_COST[q] * 0.01f : 1.0f);
            time = t < time ? t : time;
        }
        time = time > stream ? time + 0.15f * stream : stream + 0.15f * time;
        if (time < least) { least = time; best = f.form; }
    }
    return best;
}

}  // namespace hero_gemm
