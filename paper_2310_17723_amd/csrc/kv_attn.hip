// 16-bit attention over the block-scaled 8-bit KV cache (hero_kv_attn): scores, softmax and products on the matrix cores in
// FP16 with fp32 sums, the cache's codes (exact in FP16) and scales taken apart in registers.
//
// The mathematics.  With K = ks c_k, V = vs c_v (scales of the key's block and head) and, base 2, a = scale log2(e) ks (q . c_k):
//   out = sum_k 2^a vs c_v / sum_k 2^a = sum_k 2^b c_v / sum_k 2^b / vs,     b = a + log2 vs
// so V's scale costs nothing per value: it is the addend of the fma that makes a score an exponent, and its reciprocal weighs a block's
// share of the denominator.  The running maximum m is that of b; P = 2^(b - m + 15) is what FP16 holds: at most 2^15 (many rows: 2^15.94), and a normal number
// down to 2^-29 of the row's largest (a long flat tail of small probabilities is not lost).  The denominator is summed before that rounding: a
// block whose V is small beside the others' has a small P and may still hold most of the weight.  q is made FP16 too: rows of BF16 are
// multiplied by a power of two that takes their largest value to [2^14, 2^15), which keeps every bit of values down to 2^-29 of it.
// Rows: the queries of all heads that share a head of the cache, row = token * group + head of the group.
#include "kv_cache.h"
#include <algorithm>

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

constexpr float LIFT = 15.0f;
constexpr int MOST_PIECES = 128;

struct AttnArgs {
    KvView c;
    const uint16_t* q; int64_t qs[3];                         // batch, token, head
    int B, Hq, Sq, group;
    float scale; int causal;
    const int32_t *kv_len, *new_len;
    uint16_t* out; int64_t ldo;
    int tiles, splits;                                        // tiles of rows; pieces of the keys
    FastDiv by_group, by_splits, by_tiles, by_heads, by_bh8;  // (bh8: eighths of the heads of all sequences, rounded up)
    float* part; float* part_ml;                              // [B][H][rows][splits][Dh], [..][2]: a piece's sum of P c_v; its m, its denominator
};

__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {       // v_cvt_pk_f16_f32 (round to nearest even)
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{lo, hi}), v2h));
}

// What the exponents of a row whose largest is `top` are taken against: LIFT less, or `top` itself where fp32 has no such number (from 2^24 on top - LIFT can lie 16
// below it, and P = 2^16 is none of FP16).  Sums are held against this number, so that a lift that changes is no factor lost.
__device__ __forceinline__ float against(float top) {
    const float below = top - LIFT;
    return top - below > LIFT ? top : below;
}

// ---- codes -> FP16 ----
// two codes of INT8 in the bytes that sel picks, as FP16: 0x64xx is 1024 + xx, xx = code + 128
__device__ __forceinline__ uint32_t i8x2_to_f16(uint32_t hi, uint32_t lo, uint32_t sel) {
    const uint32_t w = __builtin_amdgcn_perm(hi, lo, sel) ^ 0x64806480u;
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, w) + v2h{(_Float16)-1152.0f, (_Float16)-1152.0f});
}
template <bool HI> __device__ __forceinline__ uint32_t f8x2_to_f16(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, HI));
}
// eight neighbouring codes
template <int FMT> __device__ __forceinline__ v8h codes8(uint32_t w0, uint32_t w1) {
    v4i r;
    if constexpr (FMT == HERO_I8)
        r = v4i{(int)i8x2_to_f16(0, w0, 0x0c010c00u), (int)i8x2_to_f16(0, w0, 0x0c030c02u),
                (int)i8x2_to_f16(0, w1, 0x0c010c00u), (int)i8x2_to_f16(0, w1, 0x0c030c02u)};
    else r = v4i{(int)f8x2_to_f16<false>(w0), (int)f8x2_to_f16<true>(w0), (int)f8x2_to_f16<false>(w1), (int)f8x2_to_f16<true>(w1)};
    return __builtin_bit_cast(v8h, r);
}
// channels 2 p and 2 p + 1 (of the four in a dword) of two keys: the pair of keys per channel
template <int FMT, int P> __device__ __forceinline__ void pair_of_keys(uint32_t k0, uint32_t k1, uint32_t& c0, uint32_t& c1) {
    if constexpr (FMT == HERO_I8) {
        c0 = i8x2_to_f16(k1, k0, P ? 0x0c060c02u : 0x0c040c00u);
        c1 = i8x2_to_f16(k1, k0, P ? 0x0c070c03u : 0x0c050c01u);
    } else {
        const uint32_t w = __builtin_amdgcn_perm(k1, k0, P ? 0x07030602u : 0x05010400u);
        c0 = f8x2_to_f16<false>(w);
        c1 = f8x2_to_f16<true>(w);
    }
}

__device__ __forceinline__ float max_of_groups16(float x) {           // over the lanes l, l ^ 16, l ^ 32, l ^ 48
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_of_groups16(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// A row's queries as FP16 (lanes LANES apart hold its other channels), negated for a negative scale, and what a score is to be multiplied by (base 2).
template <int DT, int N, int LANES>
__device__ __forceinline__ float queries(const v4i (&raw)[N], float scale, v8h (&qf)[N]) {
    const float rc = fabsf(scale) * 1.44269504088896340736f;
    const uint32_t sign = scale < 0.0f ? 0x80008000u : 0;
    if constexpr (DT == HERO_F16) {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            v4i w = raw[t];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] ^= (int)sign;
            qf[t] = __builtin_bit_cast(v8h, w);
        }
        return rc;
    } else {
        uint32_t top = 0;
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t w = (uint32_t)raw[t][j] & 0x7fff7fffu;
                top = max(top, max(w & 0xffffu, w >> 16));
            }
#pragma unroll
        for (int o = LANES; o < 64; o *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        // the power of two that takes the largest value to [2^14, 2^15); 1 where it is no number; at most 2^100
        const int ex = (int)(top >> 7);                                   // biased exponent
        const int up = ex == 255 ? 0 : min(127 + 14 - ex, 100);
        const float by = __uint_as_float((uint32_t)(127 + up) << 23);
#pragma unroll
        for (int t = 0; t < N; ++t) {
            v4i w;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t x = (uint32_t)raw[t][j] ^ sign;
                w[j] = (int)f16x2(bf16_bits_to_f32(x & 0xffffu) * by, __uint_as_float(x & 0xffff0000u) * by);
            }
            qf[t] = __builtin_bit_cast(v8h, w);
        }
        return rc * __uint_as_float((uint32_t)(127 - up) << 23);
    }
}

// Vector loads from a wave-uniform address: offsets of 32 bits per lane and per wave beside a descriptor in scalar registers.  (Of a pointer
// plus an offset the compiler makes a 64-bit vector addition per load, and keeps the offsets in 64 bits.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t uniform_base(const void* p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, -1, 0x00020000);
}
__device__ __forceinline__ uint32_t load1(__amdgpu_buffer_rsrc_t base, uint32_t lane_offset, uint32_t wave_offset) {
    return __builtin_amdgcn_raw_buffer_load_b32(base, (int)lane_offset, (int)wave_offset, 0);
}
__device__ __forceinline__ v4i load4(__amdgpu_buffer_rsrc_t base, uint32_t lane_offset, uint32_t wave_offset) {
    return __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(base, (int)lane_offset, (int)wave_offset, 0));
}

// keys that row's query sees: [0, result).  (s + 1 <= n: no sum passes len)
__device__ __forceinline__ int keys_seen(const AttnArgs& a, int row, int len, int n) {
    const int s = a.by_group.div(row);
    if (row >= a.Sq * a.group || s >= n) return 0;
    return a.causal ? max(0, len + (s + 1 - n)) : len;
}

// ------------------------------------------------------------------------------------------
// Few rows: a wave owns 16 RT rows and 32 keys at a time, its K and V fragments straight from memory into registers (K: a lane's 16
// channels of its key; V: a lane's 8 (4) channels of 8 keys, paired up by byte permutes), and an online softmax of its own; the NW waves of
// a workgroup split the keys of its piece and meet in LDS.
// Bound by HBM: each code is read once for all rows that share its head (the matrix instructions work on 16 rows whether there are 1 or 16, 8 %
// of the time at that).  K's next codes are asked for behind the first product and V's behind the second, which leaves registers for four waves per SIMD with one
// row tile of heads of 128 (INT8 codes and FP16 rows: 132 registers, three), five with heads of 64; two row tiles of heads of 128 take 184-188, two waves.
// 4 x 8 heads x 4 rows over 131072 E4M3 keys: 1.03 GB in 174 us, 5.9 TB/s (a read-only stream 6.15); 64 x 32 heads x 1 row
// over 1100 .. 2048 INT8 keys, 0.82 GB: 152 us, 5.4 TB/s; 16 x 8 heads x 20 rows (two tiles) over 3000 .. 4096: 26-27 us, 4.4 TB/s.
// ------------------------------------------------------------------------------------------
template <int DH, int FMT, int DT, int RT, int NW>
__global__ __launch_bounds__(64 * NW) void kv_attn_rows_kernel(AttnArgs a) {
    constexpr int KS = DH / 32;                // matrix steps over the head's width
    constexpr int CT = DH / 16;                // tiles of 16 output channels; tile i: channels CT c + i
    constexpr int VW = DH / 64;                // dwords of V per lane and key
    constexpr int ROWS = 16 * RT, OLD = DH + 4;
    __shared__ __attribute__((aligned(16))) float so[NW][16][OLD];
    __shared__ float sm[NW][ROWS], sl[NW][ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
    int split = blockIdx.x, tile = a.by_splits.divmod(split), h = a.by_tiles.divmod(tile);
    const int b = a.by_heads.divmod(h);
    const int block = 1 << a.c.log2_block;
    const int len = min(max(a.kv_len[b], 0), a.c.max_blocks << a.c.log2_block);
    const int n = a.new_len ? min(max(a.new_len[b], 0), a.Sq) : a.Sq;
    const int row0 = tile * ROWS, nrows = a.Sq * a.group;

    // what the rows see: all of them the keys before `all`, none those from `last` on (a later token sees more, until n)
    int seen[RT], all, last;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) seen[rt] = keys_seen(a, row0 + rt * 16 + c, len, n);
    {
        const int hi_row = min(row0 + ROWS, nrows) - 1;
        last = max(keys_seen(a, row0, len, n), keys_seen(a, min(hi_row, n * a.group - 1), len, n));
        if (row0 >= n * a.group) last = 0;
        all = min(keys_seen(a, row0, len, n), keys_seen(a, hi_row, len, n));
    }
    last = __builtin_amdgcn_readfirstlane(last);
    all = __builtin_amdgcn_readfirstlane(all);

    // queries
    v8h qf[RT][KS];
    float rc[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = min(row0 + rt * 16 + c, nrows - 1), s = a.by_group.div(row);
        const uint16_t* const qp = a.q + (int64_t)b * a.qs[0] + (int64_t)s * a.qs[1] + (int64_t)(h * a.group + row - s * a.group) * a.qs[2] + g * 16;
        v4i raw[KS];
#pragma unroll
        for (int t = 0; t < KS; ++t) raw[t] = *reinterpret_cast<const v4i*>(qp + (t >> 1) * 64 + (t & 1) * 8);
        rc[rt] = queries<DT, KS, 16>(raw, a.scale, qf[rt]);
    }

    v4f o[RT][CT];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -INFINITY; l[rt] = 0.0f;
#pragma unroll
        for (int i = 0; i < CT; ++i) o[rt][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // this piece's keys, in steps of 32.  A step's codes are asked for as soon as the registers of the last one's are free; its blocks a step before.
    const int steps = (last + 31) / 32, per = (steps + a.splits - 1) / a.splits;
    const int s_end = min((split + 1) * per, steps);
    v4i kr[2][VW];                               // [half][64 channels]
    uint32_t vr[8][VW];
    float ks[2], vs[2];
    int blk[2], nblk[2];
    const uint32_t koff = (uint32_t)(c * (int)a.c.k.s_row + g * 16), voff = (uint32_t)(g * 4 * (int)a.c.v.s_row + c * (DH / 16));
    auto find = [&](int step, int (&to)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int key = step * 32 + hf * 16;
            to[hf] = key < last ? a.c.block_of(b, key >> a.c.log2_block) : -1;
        }
    };
    auto from = [&](const KvSide& sd, int step, int hf) __attribute__((always_inline)) -> const uint8_t* {   // (a half without a block reads block 0, hidden below)
        return sd.codes + (int64_t)max(blk[hf], 0) * sd.s_block + (int64_t)((step * 32 + hf * 16) & (block - 1)) * sd.s_row + (int64_t)h * sd.s_head;
    };
    auto load_k = [&](int step) __attribute__((always_inline)) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const uint8_t* const kp = from(a.c.k, step, hf);
            const int64_t at = (int64_t)max(blk[hf], 0) * a.c.H + h;
            ks[hf] = a.c.k.scale[at];
            vs[hf] = a.c.v.scale[at];
#pragma unroll
            for (int t = 0; t < VW; ++t) kr[hf][t] = *reinterpret_cast<const v4i*>(kp + koff + t * 64);
        }
    };
    auto load_v = [&](int step) __attribute__((always_inline)) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const uint8_t* const vp = from(a.c.v, step, hf);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (VW == 2) {
                    const v2i w = *reinterpret_cast<const v2i*>(vp + voff + (uint32_t)j * (uint32_t)a.c.v.s_row);
                    vr[hf * 4 + j][0] = (uint32_t)w[0]; vr[hf * 4 + j][1] = (uint32_t)w[1];
                } else vr[hf * 4 + j][0] = *reinterpret_cast<const uint32_t*>(vp + voff + (uint32_t)j * (uint32_t)a.c.v.s_row);
            }
        }
    };
    int step = split * per + wave;
    if (step < s_end) {
        find(step, blk);
        load_k(step);
        load_v(step);
        find(step + NW, nblk);
    }
    for (; step < s_end; step += NW) {
        const int key0 = step * 32;
        const bool edge = key0 + 32 > all || blk[0] < 0 || blk[1] < 0;
        float kc[2], lv[2], iv[2];
        int lim[2];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            kc[hf] = ks[hf]; lv[hf] = __builtin_amdgcn_logf(vs[hf]); iv[hf] = __builtin_amdgcn_rcpf(vs[hf]);
            lim[hf] = blk[hf] < 0 ? 0 : 0x7fffffff;
        }
        if (edge)                                                         // what lies behind the last key is no code
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool there = key0 + (j >> 2) * 16 + g * 4 + (j & 3) < len && blk[j >> 2] >= 0;
#pragma unroll
                for (int t = 0; t < VW; ++t) vr[j][t] = there ? vr[j][t] : 0u;
            }
        const bool more = step + NW < s_end;
        v4f acc[RT][2];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            v8h kf[KS];
#pragma unroll
            for (int t = 0; t < VW; ++t) {
                kf[2 * t] = codes8<FMT>((uint32_t)kr[hf][t][0], (uint32_t)kr[hf][t][1]);
                kf[2 * t + 1] = codes8<FMT>((uint32_t)kr[hf][t][2], (uint32_t)kr[hf][t][3]);
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                acc[rt][hf] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int t = 0; t < KS; ++t) acc[rt][hf] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[t], qf[rt][t], acc[rt][hf], 0, 0, 0);
            }
        }
        if (more) {
            blk[0] = nblk[0]; blk[1] = nblk[1];
            load_k(step + NW);
        }
        uint32_t p[RT][4];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float x[8], top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = fmaf(acc[rt][j >> 2][j & 3], rc[rt] * kc[j >> 2], lv[j >> 2]);
            if (edge) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int key = key0 + (j >> 2) * 16 + g * 4 + (j & 3);
                    x[j] = key < min(seen[rt], lim[j >> 2]) ? x[j] : -INFINITY;
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, x[j]);
            top = max_of_groups16(top);
            const float mn = fmaxf(m[rt], against(top)), ms = mn > -INFINITY ? mn : 0.0f;
            const float resc = __builtin_amdgcn_exp2f(m[rt] - ms);
            float sum[2] = {0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float e0 = __builtin_amdgcn_exp2f(x[j] - ms), e1 = __builtin_amdgcn_exp2f(x[j + 1] - ms);
                p[rt][j >> 1] = f16x2(e0, e1);
                sum[j >> 2] += e0 + e1;
            }
            // (a block that a row does not see may have a scale that is NaN)
            l[rt] = fmaf(l[rt], resc, (sum[0] == 0.0f ? 0.0f : sum[0] * iv[0]) + (sum[1] == 0.0f ? 0.0f : sum[1] * iv[1]));
            if (__builtin_amdgcn_ballot_w64(mn != m[rt]) != 0) {
#pragma unroll
                for (int i = 0; i < CT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[rt][i][r] *= resc;
            }
            m[rt] = mn;
        }
#pragma unroll
        for (int t = 0; t < VW; ++t) {
            uint32_t w[4][4];                    // [channel][pair of keys]
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                pair_of_keys<FMT, 0>(vr[2 * j][t], vr[2 * j + 1][t], w[0][j], w[1][j]);
                pair_of_keys<FMT, 1>(vr[2 * j][t], vr[2 * j + 1][t], w[2][j], w[3][j]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const v8h vf = __builtin_bit_cast(v8h, v4i{(int)w[i][0], (int)w[i][1], (int)w[i][2], (int)w[i][3]});
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const v8h pf = __builtin_bit_cast(v8h, v4i{(int)p[rt][0], (int)p[rt][1], (int)p[rt][2], (int)p[rt][3]});
                    o[rt][t * 4 + i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf, o[rt][t * 4 + i], 0, 0, 0);
                }
            }
        }
        if (more) {
            load_v(step + NW);
            find(step + 2 * NW, nblk);
        }
    }

    // the waves meet: each one's sums at the common maximum, added in the order of the waves
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] = sum_of_groups16(l[rt]);
        if (g == 0) { sm[wave][rt * 16 + c] = m[rt]; sl[wave][rt * 16 + c] = l[rt]; }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        __syncthreads();
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, sm[w][rt * 16 + c]);
        const float f = M > -INFINITY ? __builtin_amdgcn_exp2f(m[rt] - M) : 0.0f;
#pragma unroll
        for (int i = 0; i < CT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) so[wave][c][(g * 4 + r) * CT + i] = o[rt][i][r] * f;
        __syncthreads();
        for (int at = tid; at < 16 * (DH / 4); at += 64 * NW) {
            const int rr = at / (DH / 4), e = (at % (DH / 4)) * 4, row = row0 + rt * 16 + rr;
            if (row >= nrows) continue;
            float top = -INFINITY, L = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w) top = fmaxf(top, sm[w][rt * 16 + rr]);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float lw = sl[w][rt * 16 + rr];
                if (!(lw == 0.0f)) L = fmaf(lw, __builtin_amdgcn_exp2f(sm[w][rt * 16 + rr] - top), L);
            }
            v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const v4f p = *reinterpret_cast<const v4f*>(&so[w][rr][e]);
#pragma unroll
                for (int t = 0; t < 4; ++t) sum[t] += p[t];
            }
            if (a.splits > 1) {
                const int64_t pr = (((int64_t)b * a.c.H + h) * nrows + row) * a.splits + split;
                *reinterpret_cast<v4f*>(a.part + pr * DH + e) = sum;
                if (e == 0) { a.part_ml[pr * 2] = top; a.part_ml[pr * 2 + 1] = L; }
            } else {
                // (a score beyond fp32 has no exponent: NaN; no key: 0)
                const float inv = top == INFINITY ? __builtin_nanf("") : (L == 0.0f ? 0.0f : 1.0f / L);
                const int s = a.by_group.div(row);
                uint16_t* const op = a.out + ((int64_t)b * a.Sq + s) * a.ldo + (int64_t)(h * a.group + row - s * a.group) * DH + e;
                *reinterpret_cast<v2i*>(op) = v2i{(int)pack2_hp<DT>(sum[0] * inv, sum[1] * inv), (int)pack2_hp<DT>(sum[2] * inv, sum[3] * inv)};
            }
        }
    }
}

// ------------------------------------------------------------------------------------------
// Many rows: a workgroup of eight waves owns 256 rows (heads of 64: of four, 128), a wave 32 of them; K and V of 64 keys at a time are made FP16 once, on their way
// into LDS (K by rows, V by channels), three tiles deep, so that one barrier per tile is enough: a tile is written while the one before it is
// worked on.  Scores are computed transposed (S^T = K Q^T): a lane owns query lane % 32, and the exponentials are the second product's operand
// as they stand.  A step makes the scores of 32 keys, takes the exponentials of the 32 before them and multiplies V by those of the 32 before
// those, in one block of instructions.
// The maximum is taken of every step's exponents before P is made of them, and the sums so far are rescaled only where a row's has risen by more than SLACK: the
// largest P of a row lies in [2^15, 2^15.94], its normal numbers reach down to 2^-29 of it as in the kernel of few rows.  (Exponentials against the last maximum, raised
// behind a step whose P came near FP16's end, need 7 bits of room there: P was normal down to 2^-22 of the largest only, and a flat tail at 2^-28.5 behind a key with V = 0
// off by 3 %.  us for the two cases below, so / as it is, with queries of a quarter, the listed and 2.5 times the size: 82 / 96, 88 / 96, 98 / 96 and 170 / 192,
// 182 / 198, 207 / 199.)
// K's rows are 16 bytes longer than they need to be, V's 16-byte pieces XOR-swizzled by their row: fragment reads (turns of lanes 0-3, 12-15,
// 20-27 and so on) meet no bank conflict.
// 8 x 32 heads x 256 rows behind 2304 E4M3 keys 95-97 us (755 TFLOP/s; a library product of 8192^3 runs at 1270), 4 x 32 x 2048 causal INT8 197 us
// (697), 4 x 32 heads of 64 x 2048 causal INT8 113.  In clocks per tile and CU of the first: 4600 at 2.14 GHz, 2048 of them matrix instructions, 310 rescaled sums (in two
// steps of five; 120 with queries of a quarter of the size, 440 with 2.5 times).  Against a late maximum it was 3793 at 1.94 GHz, of which without fragment
// reads 2783, without staging and loads 2877, without exponentials 3528, without any of them 2335; the clock that the power limit allows fell with what was left (1.73 GHz),
// so that orders of instructions, priorities and loads that nothing waits for changed a launch by 2 % or not at all.  64 rows to a wave halve the
// reads, but leave one wave per SIMD and too few registers: half as long again.  Beside the loop a workgroup takes 7 us (arguments, lengths, first tile, result); two
// row tiles to a workgroup cost the loop more (8 %) than they saved.
// ------------------------------------------------------------------------------------------
constexpr float SLACK = 0.9375f;                            // P stays below 2^15.95, FP16's end is 65504

// The order of a step's instructions: an exponential and an LDS read behind each matrix instruction.
template <int COUNT>
__device__ __forceinline__ void step_order() {
    constexpr int LDS_READ = 0x100, MATRIX = 0x008, EXP = 0x400;
    __builtin_amdgcn_sched_group_barrier(LDS_READ, 4, 0);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        __builtin_amdgcn_sched_group_barrier(MATRIX, 1, 0);
        __builtin_amdgcn_sched_group_barrier(LDS_READ, 1, 0);
        __builtin_amdgcn_sched_group_barrier(EXP, 16 / COUNT, 0);
    }
}

// A thread stages one unit of K and one of V per tile of 64 keys, which for heads of 64 gives work to 256 threads; three such workgroups fit a CU.  us against eight
// waves whose halves stage the same (both against a late maximum): 4 x 32 heads of 64 x 2048 rows causal INT8 136 -> 105, 8 x 12 x 512 causal 20.1 -> 16.9, 16 x 12 x 128 over 1024 34.0 -> 26.9.
constexpr int tile_waves(int Dh) { return Dh == 64 ? 4 : 8; }

template <int DH, int FMT, int DT, int NI>                   // NI: blocks that a tile's 64 keys lie in
__global__ __launch_bounds__(64 * tile_waves(DH), DH == 64 ? 3 : 2) void kv_attn_tile_kernel(AttnArgs a) {
    constexpr int NW = tile_waves(DH), ROWS = 32 * NW;
    constexpr int DS = DH / 16, CT = DH / 32, KROW = DH * 2 + 16, NB = 3;
    constexpr int GH = NI == 4 ? 2 : 1, GE = 16 / GH;        // groups of keys with scales of their own in 32 keys
    constexpr int OROW = DH * 2 + 16;                        // a row of the result on its way out
    __shared__ __attribute__((aligned(1024))) uint8_t pool[NB * (64 * KROW + DH * 128)];
    static_assert(NW * 32 * OROW <= sizeof(pool), "every wave's rows of the result fit");
    uint8_t (* const sK)[64 * KROW] = reinterpret_cast<uint8_t (*)[64 * KROW]>(pool);
    uint8_t (* const sV)[DH * 128] = reinterpret_cast<uint8_t (*)[DH * 128]>(pool + NB * 64 * KROW);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hh = lane >> 5, ql = lane & 31;
    const int nrows = a.Sq * a.group;
    // workgroups go round-robin to the XCDs: a head's row tiles to one of them; the last rows (which see the most keys) first
    int split = (int)(blockIdx.x >> 3), bh8 = a.by_splits.divmod(split);
    const int tile = a.tiles - 1 - a.by_bh8.divmod(bh8), bh = bh8 * 8 + (int)(blockIdx.x & 7);
    if (bh >= a.B * a.c.H) return;
    int h = bh;
    const int b = a.by_heads.divmod(h);
    const int len = min(max(a.kv_len[b], 0), a.c.max_blocks << a.c.log2_block);
    const int n = a.new_len ? min(max(a.new_len[b], 0), a.Sq) : a.Sq;
    const int row0 = tile * ROWS, wrow = row0 + wave * 32, row = wrow + ql;
    auto range = [&](int r0, int count, int& all, int& last) {           // of rows [r0, r0 + count): keys that all / any of them see
        const int r1 = min(r0 + count, nrows) - 1;
        last = r0 >= n * a.group ? 0 : max(keys_seen(a, r0, len, n), keys_seen(a, min(r1, n * a.group - 1), len, n));
        all = min(keys_seen(a, r0, len, n), keys_seen(a, r1, len, n));
        last = __builtin_amdgcn_readfirstlane(last);
        all = __builtin_amdgcn_readfirstlane(all);
    };
    int all, last, wall, wlast;
    range(row0, ROWS, all, last);
    range(wrow, 32, wall, wlast);
    const int seen = keys_seen(a, row, len, n);
    const int total = (last + 63) / 64, per = (total + a.splits - 1) / a.splits;
    const int t0 = min(split * per, total), t1 = min(t0 + per, total), wt = min(t1, (wlast + 63) / 64), te = t1 - 1;

    // ---- staging.  K: a thread's unit is 16 codes of a key; V: 4 channels of 4 keys.
    v4i kr;
    uint32_t vr[4];
    int vend;                                                            // how many keys there are from V's unit's first on
    const int kch = tid % (DH / 16), krow = tid / (DH / 16);
    const int vch = tid % (DH / 4), vq = tid / (DH / 4);
    // A wave's units all lie in one group of 16 keys; a tile's keys in NI blocks (the same one, of 64 tokens or more).  The table is read three
    // tiles ahead, the codes two, the scales one; as vector loads, since a scalar load's wait would be one for all LDS reads too.
    const int group16 = wave * 4 / NW;
    const int kstride = (int)a.c.k.s_row, vstride = (int)a.c.v.s_row;    // (a block's rows span less than 2^31 elements)
    const uint32_t koff = (uint32_t)((krow & 15) * kstride + kch * 16);
    const uint32_t voff = (uint32_t)((vq & 3) * 4 * vstride + vch * 4);
    typedef int Ids[NI];
    const int32_t* const table = a.c.table + (int64_t)b * a.c.max_blocks;
    auto place = [&](int t, int i) __attribute__((always_inline)) { return min((t * 64 + i * (64 / NI)) >> a.c.log2_block, a.c.max_blocks - 1); };
    auto look = [&](int t, Ids& raw) __attribute__((always_inline)) {    // (without a table nothing, not even a register, is touched: it could be waited for)
        if (a.c.table)
#pragma unroll
            for (int i = 0; i < NI; ++i) raw[i] = (int)load1(uniform_base(table + place(t, i)), 0, 0);
    };
    auto settle = [&](int t, const Ids& raw, Ids& id) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NI; ++i) id[i] = (int)((uint32_t)b * (uint32_t)a.c.max_blocks + (uint32_t)place(t, i));
        if (a.c.table)
#pragma unroll
            for (int i = 0; i < NI; ++i) id[i] = __builtin_amdgcn_readfirstlane(raw[i]);
#pragma unroll
        for (int i = 0; i < NI; ++i) id[i] = (unsigned)id[i] < (unsigned)a.c.n_blocks ? id[i] : -1;
    };
    const uint8_t* const khead = a.c.k.codes + (int64_t)h * a.c.k.s_head;
    const uint8_t* const vhead = a.c.v.codes + (int64_t)h * a.c.v.s_head;
    auto fetch = [&](int t, const Ids& id) __attribute__((always_inline)) {
        int blk = 0;                             // id[group16 NI / 4], by masks: an index that is not known would put the array into memory
#pragma unroll
        for (int i = 0; i < NI; ++i) blk |= id[i] & -(int)(group16 * NI / 4 == i);
        const int first = t * 64 + group16 * 16, at = first & ((1 << a.c.log2_block) - 1);
        const uint8_t* const kp = khead + (int64_t)max(blk, 0) * a.c.k.s_block + (uint32_t)(at * kstride);
        const uint8_t* const vp = vhead + (int64_t)max(blk, 0) * a.c.v.s_block + (uint32_t)(at * vstride);
        kr = load4(uniform_base(kp), koff, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) vr[j] = load1(uniform_base(vp), voff, (uint32_t)(j * vstride));
        vend = blk < 0 ? 0 : len - first - (vq & 3) * 4;
    };
    float sk[NI], sv[NI];
    const float* const kscale = a.c.k.scale + h;
    const float* const vscale = a.c.v.scale + h;
    auto scales = [&](const Ids& id) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int64_t at = (int64_t)max(id[i], 0) * a.c.H;
            sk[i] = __uint_as_float(load1(uniform_base(kscale + at), 0, 0));
            sv[i] = __uint_as_float(load1(uniform_base(vscale + at), 0, 0));
        }
    };
    // what lies behind the last key, or where no block is, is no code
    auto blank = [&]() __attribute__((always_inline)) {
        if (__builtin_amdgcn_ballot_w64(vend < 4) != 0)
#pragma unroll
            for (int j = 0; j < 4; ++j) vr[j] = j < vend ? vr[j] : 0u;
    };
    // a half of 16 keys: its lanes hold keys 0-3, 8-11 / 4-7, 12-15 of them
    const uint32_t kput = krow * KROW + kch * 32;
    const uint32_t vput = vch * 512 + ((vq >> 2) * 2 + (vq & 1)) * 16 + ((vq >> 1) & 1) * 8;
    auto stage = [&](int buf) __attribute__((always_inline)) {
        const v8h x0 = codes8<FMT>((uint32_t)kr[0], (uint32_t)kr[1]), x1 = codes8<FMT>((uint32_t)kr[2], (uint32_t)kr[3]);
        *reinterpret_cast<v8h*>(&sK[buf][kput]) = x0;
        *reinterpret_cast<v8h*>(&sK[buf][kput + 16]) = x1;
        uint32_t w[4][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            pair_of_keys<FMT, 0>(vr[2 * j], vr[2 * j + 1], w[0][j], w[1][j]);
            pair_of_keys<FMT, 1>(vr[2 * j], vr[2 * j + 1], w[2][j], w[3][j]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int rr = (vch * 4 + i) >> 1;
            *reinterpret_cast<v2i*>(&sV[buf][(vput ^ (((rr & 7) ^ ((rr >> 3) & 1)) * 16)) + i * 128]) = v2i{(int)w[i][0], (int)w[i][1]};
        }
    };
    // what was written to LDS is there for the other waves, and global loads stay in flight
    auto meet = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    };

    // ---- the arithmetic
    v8h qf[DS];
    v16f o[CT];
    float rc, m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[c][r] = 0.0f;
    // scores of 32 keys (s of the tile in buf)
    const uint32_t kget = ql * KROW + hh * 16;
    const uint32_t vget = ql * 128 + (hh ^ ((ql >> 1) & 7) ^ (ql >> 4)) * 16;
    auto scores = [&](int buf, int s) __attribute__((always_inline)) -> v16f {
        v16f acc = {};
        const uint8_t* const from = &sK[buf][s * 32 * KROW];
#pragma unroll
        for (int d = 0; d < DS; ++d) acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const v8h*>(from + kget + d * 32), qf[d], acc, 0, 0, 0);
        return acc;
    };
    // of the scales that have come: what the exponents are made of (score * ck + lv); a group without a block has no keys
    struct Group { float ks, lv, iv; int lim; };
    auto groups = [&](const Ids& id, Group (&gr)[2][GH]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const Group x = {sk[i], __builtin_amdgcn_logf(sv[i]), __builtin_amdgcn_rcpf(sv[i]), id[i] < 0 ? 0 : 0x7fffffff};
            if constexpr (NI == 1) gr[0][0] = gr[1][0] = x;
            else gr[i / GH][i % GH] = x;
        }
    };
    float sum[GH], resc;
    uint32_t p[8] = {0, 0, 0, 0, 0, 0, 0, 0}, q[8];                      // of the step before (nothing yet), of this one
    // scores -> exponents, and what the largest makes of the row's maximum.  (A row by its own scores alone: its result does not depend on the others of its wave.)
    auto exponents = [&](int t, int s, v16f& acc, const Group (&gr)[GH], bool edge) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < GH; ++g) {
            const float ck = rc * gr[g].ks;
#pragma unroll
            for (int r = g * GE; r < (g + 1) * GE; ++r) acc[r] = fmaf(acc[r], ck, gr[g].lv);
        }
        if (edge) {                              // hidden keys (of scales that may be NaN)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int key = t * 64 + s * 32 + (r >> 2) * 8 + hh * 4 + (r & 3);
                acc[r] = key < min(seen, gr[r / GE].lim) ? acc[r] : -INFINITY;
            }
        }
        float top = acc[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, acc[r]);
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
        const float mn = top - m > LIFT + SLACK ? against(top) : m;      // (m is -inf before the first key)
        resc = mn > m ? __builtin_amdgcn_exp2f(m - mn) : 1.0f;
        m = mn;
    };
    auto weigh = [&](const v16f& acc) __attribute__((always_inline)) {
        const float sub = m > -INFINITY ? m : 0.0f;
#pragma unroll
        for (int g = 0; g < GH; ++g) {
            sum[g] = 0.0f;
#pragma unroll
            for (int r = g * GE; r < (g + 1) * GE; r += 2) {
                const float e0 = __builtin_amdgcn_exp2f(acc[r] - sub), e1 = __builtin_amdgcn_exp2f(acc[r + 1] - sub);
                sum[g] += e0 + e1;
                q[r >> 1] = f16x2(e0, e1);
            }
        }
    };
    // behind the products, which were of the P before: all sums at the maximum of this step
    auto settled = [&](const Group (&gr)[GH]) __attribute__((always_inline)) {
        if (__builtin_amdgcn_ballot_w64(resc != 1.0f) != 0) {
            l *= resc;
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[c][r] *= resc;
        }
#pragma unroll
        for (int g = 0; g < GH; ++g) l += sum[g] == 0.0f ? 0.0f : sum[g] * gr[g].iv;
#pragma unroll
        for (int r = 0; r < 8; ++r) p[r] = q[r];
    };
    auto product = [&](int buf, int s, int i) __attribute__((always_inline)) {      // the i-th of its 2 CT matrix instructions
        const int st = i / CT, c = i % CT;
        const v8h pf = __builtin_bit_cast(v8h, v4i{(int)p[4 * st], (int)p[4 * st + 1], (int)p[4 * st + 2], (int)p[4 * st + 3]});
        o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const v8h*>(&sV[buf][(vget ^ ((s * 2 + st) * 32)) + c * 4096]), pf, o[c], 0, 0, 0);
    };
    // the two products of a step, one matrix instruction of each after the other: the first's eight are a chain
    static_assert(DS == 2 * CT, "as many of the one as of the other");
    auto products = [&](int kbuf, int ks, int vbuf, int vs) __attribute__((always_inline)) -> v16f {
        v16f acc = {};
        const uint8_t* const from = &sK[kbuf][ks * 32 * KROW];
#pragma unroll
        for (int d = 0; d < DS; ++d) {
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const v8h*>(from + kget + d * 32), qf[d], acc, 0, 0, 0);
            product(vbuf, vs, d);
        }
        return acc;
    };

    // ---- the first tile.  (The blocks are looked up and the scales asked for in front of the codes here as in the loop: what waits for them there
    // is not to wait for codes.)
    Ids raw = {}, id, id1, id2;                                               // blocks of tile t + 3 as they come, of t, t + 1, t + 2
    v4i qraw[DS];
    if (t0 < t1) {
        Ids raw1 = {}, raw2 = {};
        look(t0, raw1);
        look(min(t0 + 1, te), raw2);
        look(min(t0 + 2, te), raw);
        settle(t0, raw1, id1);
        settle(min(t0 + 1, te), raw2, id2);
        scales(id1);
        fetch(t0, id1);
    }
    {
        const int rr = min(row, nrows - 1), s = a.by_group.div(rr);
        const uint16_t* const qp = a.q + (int64_t)b * a.qs[0] + (int64_t)s * a.qs[1] + (int64_t)(h * a.group + rr - s * a.group) * a.qs[2] + hh * 8;
#pragma unroll
        for (int t = 0; t < DS; ++t) qraw[t] = *reinterpret_cast<const v4i*>(qp + t * 16);
    }
    if (t0 < t1) {
        blank();
        stage(t0 % NB);
        fetch(min(t0 + 1, te), id2);
    }
    rc = queries<DT, DS, 32>(qraw, a.scale, qf);
    __syncthreads();
    v16f acc = {}, next;
    if (t0 < wt) acc = scores(t0 % NB, 0);
    auto next_ids = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NI; ++i) { id[i] = id1[i]; id1[i] = id2[i]; }
        settle(min(t + 2, te), raw, id2);
        look(min(t + 3, te), raw);
    };
    // (behind the last tile the last one is fetched and staged again, and scores are made that nobody takes: no branch in the middle)
    int t = t0, before = t0 % NB;                                        // (a first product of nothing by a tile that is there)
    for (; t < wt; ++t) {
        const int buf = t % NB, after = (t + 1) % NB;
        Group gr[2][GH];
        next_ids(t);
        groups(id, gr);
        scales(id1);                             // (in front of the codes of this iteration, whose arrival the next one's start does not wait for)
        bool edge = t * 64 + 64 > wall;
#pragma unroll
        for (int i = 0; i < NI; ++i) edge |= id[i] < 0;
        blank();
        exponents(t, 0, acc, gr[0], edge);
        next = products(buf, 1, before, 1);
        weigh(acc);
        stage(after);
        fetch(min(t + 2, te), id2);
        step_order<DS + 2 * CT>();
        settled(gr[0]);
        meet();
        exponents(t, 1, next, gr[1], edge);
        acc = products(after, 0, buf, 0);
        weigh(next);
        step_order<DS + 2 * CT>();
        settled(gr[1]);
        before = buf;
    }
    if (t0 < wt)
#pragma unroll
        for (int i = 0; i < DS; ++i) product(before, 1, i);
    for (; t < t1; ++t) {                                                // tiles that other waves' rows see
        next_ids(t);
        blank();
        stage((t + 1) % NB);
        fetch(min(t + 2, te), id2);
        meet();
    }

    l += __shfl_xor(l, 32);
    if (a.splits > 1) {
        if (row >= nrows) return;
        const int64_t pr = ((int64_t)bh * nrows + row) * a.splits + split;
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<v4f*>(a.part + pr * DH + c * 32 + g * 8 + hh * 4) = v4f{o[c][4 * g], o[c][4 * g + 1], o[c][4 * g + 2], o[c][4 * g + 3]};
        if (hh == 0) { a.part_ml[pr * 2] = m; a.part_ml[pr * 2 + 1] = l; }
        return;
    }
    // by way of LDS (each wave its own part, once all have read their last tile), so that a store covers whole rows
    __syncthreads();
    uint8_t* const mine = pool + wave * (32 * OROW);
    const float inv = m == INFINITY ? __builtin_nanf("") : (l == 0.0f ? 0.0f : 1.0f / l);
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<v2i*>(mine + ql * OROW + (c * 32 + g * 8 + hh * 4) * 2) =
                v2i{(int)pack2_hp<DT>(o[c][4 * g] * inv, o[c][4 * g + 1] * inv), (int)pack2_hp<DT>(o[c][4 * g + 2] * inv, o[c][4 * g + 3] * inv)};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    constexpr int LPR = DH / 4, RPS = 64 / LPR;              // lanes to a row, rows to a store
#pragma unroll
    for (int i = 0; i < 32 / RPS; ++i) {
        const int rr = i * RPS + lane / LPR, r = wrow + rr, e = lane % LPR * 4;
        const v2i w = *reinterpret_cast<const v2i*>(mine + rr * OROW + e * 2);
        if (r >= nrows) continue;
        const int s = a.by_group.div(r);
        *reinterpret_cast<v2i*>(a.out + ((int64_t)b * a.Sq + s) * a.ldo + (int64_t)(h * a.group + r - s * a.group) * DH + e) = w;
    }
}

// ------------------------------------------------------------------------------------------
// The pieces of the keys joined: a row is the business of GPR groups of DH / 4 threads, each of which takes every GPR-th piece, four at a time
// in flight; the groups meet in LDS.  All in a fixed order.  (One group whose loads waited for each other: 31 us for 32 pieces of 128 rows, eight
// groups 4; eight groups for the 4 pieces of 2560 rows 4.8, one 3.)
// ------------------------------------------------------------------------------------------
template <int DH, int DT, int GPR>
__global__ __launch_bounds__(256) void kv_attn_join_kernel(AttnArgs a) {
    constexpr int TPR = DH / 4, RPB = 256 / TPR / GPR;
    __shared__ __attribute__((aligned(16))) float so[GPR > 1 ? GPR : 1][DH];
    __shared__ float sm[GPR], sl[GPR];
    static_assert(GPR == 1 || RPB == 1, "one row where groups meet");
    const int nrows = a.Sq * a.group, tid = threadIdx.x, grp = GPR > 1 ? tid / TPR : 0, e = (tid % TPR) * 4;
    const int64_t r = (int64_t)blockIdx.x * RPB + (GPR > 1 ? 0 : tid / TPR);
    if (r >= (int64_t)a.B * a.c.H * nrows) return;
    const float* const ml = a.part_ml + r * a.splits * 2;
    const float* const p = a.part + r * a.splits * DH + e;
    v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
    float M = -INFINITY, L = 0.0f;
    for (int s0 = grp; s0 < a.splits; s0 += 4 * GPR) {
        v4f x[4];
        float m[4], l[4], top = M;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = min(s0 + i * GPR, a.splits - 1);
            x[i] = *reinterpret_cast<const v4f*>(p + (int64_t)s * DH);
            m[i] = ml[2 * s];
            l[i] = s0 + i * GPR < a.splits ? ml[2 * s + 1] : 0.0f;        // (0: no key in it; its maximum is -inf)
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, m[i]);
        const float base = top > -INFINITY ? top : 0.0f, f0 = __builtin_amdgcn_exp2f(M - base);
        L *= f0;
#pragma unroll
        for (int t = 0; t < 4; ++t) sum[t] *= f0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (l[i] == 0.0f) continue;
            const float f = __builtin_amdgcn_exp2f(m[i] - base);
            L = fmaf(l[i], f, L);
#pragma unroll
            for (int t = 0; t < 4; ++t) sum[t] = fmaf(x[i][t], f, sum[t]);
        }
        M = top;
    }
    if constexpr (GPR > 1) {
        *reinterpret_cast<v4f*>(&so[grp][e]) = sum;
        if (e == 0) { sm[grp] = M; sl[grp] = L; }
        __syncthreads();
        if (grp) return;
#pragma unroll
        for (int i = 1; i < GPR; ++i) M = fmaxf(M, sm[i]);
        sum = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        L = 0.0f;
#pragma unroll
        for (int i = 0; i < GPR; ++i) {
            const v4f x = *reinterpret_cast<const v4f*>(&so[i][e]);
            const float l = sl[i];
            if (l == 0.0f) continue;
            const float f = __builtin_amdgcn_exp2f(sm[i] - (M > -INFINITY ? M : 0.0f));
            L = fmaf(l, f, L);
#pragma unroll
            for (int t = 0; t < 4; ++t) sum[t] = fmaf(x[t], f, sum[t]);
        }
    }
    const float inv = M == INFINITY ? __builtin_nanf("") : (L == 0.0f ? 0.0f : 1.0f / L);
    const int bh = (int)(r / nrows), row = (int)(r - (int64_t)bh * nrows), s = a.by_group.div(row);
    int h = bh;
    const int b = a.by_heads.divmod(h);
    uint16_t* const op = a.out + ((int64_t)b * a.Sq + s) * a.ldo + (int64_t)(h * a.group + row - s * a.group) * DH + e;
    *reinterpret_cast<v2i*>(op) = v2i{(int)pack2_hp<DT>(sum[0] * inv, sum[1] * inv), (int)pack2_hp<DT>(sum[2] * inv, sum[3] * inv)};
}

__global__ void kv_attn_zero_kernel(uint16_t* out, int64_t rows, int64_t cols, int64_t ld) {
    const int64_t step = (int64_t)gridDim.x * 1024;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < rows * cols; i += step)
        *reinterpret_cast<v2i*>(out + (i / cols) * ld + i % cols) = v2i{0, 0};
}

// How a call is cut: 16 rt rows to a tile of the kernel of few rows, or 256 (heads of 64: 128) to one of that of many (rt = 0); the keys into pieces.
// The kernel of many rows reads K and V once per such tile, and takes longer to begin and end.  us, few / many, by the multiply-adds of rows x keys (in G; neither the
// mask nor the sequences' lengths are known here: the table's width stands for the keys):
//   0.3: 128 rows of 8 heads over 2048 keys 16 / 24      0.5: 256 of 8 over 2048 18 / 32              0.7: 160 of 8 over 4000 24 / 32
//   1.0: 200 of 128 heads of 64 over 600 21 / 19         1.0: 128 of 128 heads of 64 over 1000 20 / 24   1.3: 100 of 48 heads of 64 over 4096 33 / 28
//   1.6: 512 of 96 heads of 64 over 512 25 / 21          1.9: 300 of 24 heads of 64 over 4096 33 / 36    2.1: 128 of 32 over 4096 30 / 29
//   4.3: 1024 of 32 over 1024 causal 46 / 40             4.3: 512 of 8 over 8192 47 / 42              5.2: 80 of 512 over 1000 72 / 67
//   10: 160 of 128 over 4000 126 / 83                    17: 2048 of 32 over 2048 causal 130 / 78     69: 4096 of 32 over 4096 causal 372 / 174
// and up to 64 rows, which the kernel of few rows reads once too: 36 rows of 512 heads over 2048 keys 91 / 115, 64 of 8 over 65536 49 / 61.
struct Plan { int rt, tiles, splits; };

// forced: 0, or the rows of a tile (16, 32, 256 for the kernel of many rows)
Plan plan(const hero_kv_cache* c, int64_t Hq, int64_t Sq, int forced) {
    Plan p;
    const int64_t rows = Sq * (Hq / c->H), bh = c->B * c->H, keys = c->max_blocks * c->block, steps = (keys + 31) / 32;
    p.rt = rows <= 16 ? 1 : rows > 64 && (double)rows * bh * keys * c->Dh >= 1.5e9 ? 0 : 2;
    if (forced) p.rt = forced == 256 ? 0 : forced / 16;
    const int64_t tile = p.rt ? 16 * p.rt : 32 * tile_waves(c->Dh);
    p.tiles = (int)((rows + tile - 1) / tile);
    const int64_t units = bh * p.tiles;
    // Pieces of 16 steps or more while there are fewer than two workgroups per CU (one, of many rows of heads of 128).  us, towards 256 / 512 / 1024 workgroups:
    // 4 x 8 heads x 4 rows over 131072 keys 192 / 179 / 184, 16 x 8 heads x 20 rows over 4096 keys (its write with it) 49 / 41 / 46.  Many rows, towards
    // 256 / 512 / 768: 4 x 8 heads of 64 x 512 rows over 8192 keys 89 / 69 / 69, heads of 128 94 / 108 / 124.
    // Pieces of 8 / 16 / 24 steps or more: 12 heads of 64 x 1 row over 512 keys 12.2 / 10.0 / 9.8, 4 x 8 x 4 rows over 2048 12.3 / 12.0 / 15.3, 3 x 2 x 539 over 1111 14.2 / 14.5 / 15.9.
    int64_t s = ((p.rt == 0 && c->Dh == 128 ? 256 : 512) + units - 1) / units;
    s = s < steps / 16 ? s : steps / 16;
    p.splits = (int)(s < 1 ? 1 : s > MOST_PIECES ? MOST_PIECES : s);
    return p;
}

hero_status check_sizes(const hero_kv_cache* c, int64_t Hq, int64_t Sq) {
    if (Hq < 0 || Sq < 0 || Hq > 65535 || Sq > (1LL << 30)) return HERO_ERR_SHAPE;
    if (c->H == 0 ? Hq != 0 : Hq % c->H != 0) return HERO_ERR_SHAPE;
    if (c->H && Sq * (Hq / c->H) > (1LL << 30)) return HERO_ERR_SHAPE;
    return HERO_OK;
}

size_t part_bytes(const hero_kv_cache* c, int64_t Hq, int64_t Sq, int splits) {
    return splits > 1 ? (size_t)(c->B * Sq * Hq) * splits * (c->Dh + 2) * 4 : 0;
}

template <int DH, int FMT, int DT>
hero_status launch(const AttnArgs& a, const Plan& p, hipStream_t st) {
    const dim3 block(256);
    if (p.rt == 0) {
        const dim3 grid((unsigned)(((int64_t)a.B * a.c.H + 7) / 8 * 8 * a.tiles * a.splits));
        if (a.c.log2_block == 4) hipLaunchKernelGGL((kv_attn_tile_kernel<DH, FMT, DT, 4>), grid, dim3(64 * tile_waves(DH)), 0, st, a);
        else if (a.c.log2_block == 5) hipLaunchKernelGGL((kv_attn_tile_kernel<DH, FMT, DT, 2>), grid, dim3(64 * tile_waves(DH)), 0, st, a);
        else hipLaunchKernelGGL((kv_attn_tile_kernel<DH, FMT, DT, 1>), grid, dim3(64 * tile_waves(DH)), 0, st, a);
    } else {
        const dim3 grid((unsigned)((int64_t)a.B * a.c.H * a.tiles * a.splits));
        if (p.rt == 1) hipLaunchKernelGGL((kv_attn_rows_kernel<DH, FMT, DT, 1, 4>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((kv_attn_rows_kernel<DH, FMT, DT, 2, 4>), grid, block, 0, st, a);
    }
    hero_status r = hero_launch_status();
    if (r != HERO_OK || a.splits == 1) return r;
    const int64_t rows = (int64_t)a.B * a.c.H * a.Sq * a.group;
    constexpr int NG = 256 / (DH / 4);
    if (a.splits <= 8) hipLaunchKernelGGL((kv_attn_join_kernel<DH, DT, 1>), dim3((unsigned)((rows + NG - 1) / NG)), block, 0, st, a);
    else hipLaunchKernelGGL((kv_attn_join_kernel<DH, DT, NG>), dim3((unsigned)rows), block, 0, st, a);
    return hero_launch_status();
}

}  // namespace

extern "C" size_t hero_kv_attn_workspace_bytes(const hero_kv_cache* cache, int64_t Hq, int64_t Sq) {
    if (kv_check(cache) != HERO_OK || check_sizes(cache, Hq, Sq) != HERO_OK || cache->B == 0 || Hq == 0 || Sq == 0) return 0;
    return part_bytes(cache, Hq, Sq, plan(cache, Hq, Sq, 0).splits);
}

extern "C" hero_status hero_kv_attn(const hero_kv_cache* cache, const void* q, const int64_t q_strides[4], hero_dtype dt,
                                    int64_t Hq, int64_t Sq, float scale, hero_mask mask, const int32_t* kv_len, const int32_t* new_len,
                                    void* out, int64_t ldo, void* workspace, size_t workspace_bytes, void* stream) {
    return hero_kv_attn_tile(cache, q, q_strides, dt, Hq, Sq, scale, mask, kv_len, new_len, out, ldo, workspace, workspace_bytes, stream, 0);
}

extern "C" hero_status hero_kv_attn_tile(const hero_kv_cache* cache, const void* q, const int64_t q_strides[4], hero_dtype dt,
                                         int64_t Hq, int64_t Sq, float scale, hero_mask mask, const int32_t* kv_len, const int32_t* new_len,
                                         void* out, int64_t ldo, void* workspace, size_t workspace_bytes, void* stream, int forced) {
    hero_status r = kv_check(cache);
    if (r != HERO_OK) return r;
    if (forced != 0 && forced != 16 && forced != 32 && forced != 256) return HERO_ERR_UNSUPPORTED;
    if (dt != HERO_BF16 && dt != HERO_F16) return HERO_ERR_UNSUPPORTED;
    if (mask != HERO_MASK_NONE && mask != HERO_MASK_CAUSAL) return HERO_ERR_UNSUPPORTED;
    if ((r = check_sizes(cache, Hq, Sq)) != HERO_OK) return r;
    if (cache->B == 0 || Hq == 0 || Sq == 0) return HERO_OK;
    if (!out || !kv_len) return HERO_ERR_NULL;
    if ((r = kv_check_rows(q, q_strides)) != HERO_OK) return r;
    const int Dh = cache->Dh;
    if (ldo < Hq * Dh) return HERO_ERR_SHAPE;
    if (ldo % 4 || !hero_aligned16(out) || ((uintptr_t)kv_len & 3) || ((uintptr_t)new_len & 3)) return HERO_ERR_ALIGN;
    if (workspace && ((uintptr_t)workspace & 255)) return HERO_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    if (cache->n_blocks == 0 || cache->max_blocks == 0) {                // no key anywhere
        if (cache->B * Sq * Hq > 0x7fffffffLL) return HERO_ERR_SHAPE;
        const int64_t groups = (cache->B * Sq * Hq * Dh + 1023) / 1024;
        hipLaunchKernelGGL(kv_attn_zero_kernel, dim3((unsigned)std::min<int64_t>(groups, 8192)), dim3(256), 0, st, (uint16_t*)out, cache->B * Sq, Hq * Dh, ldo);
        return hero_launch_status();
    }
    Plan p = plan(cache, Hq, Sq, forced);
    if (!workspace || workspace_bytes < part_bytes(cache, Hq, Sq, p.splits)) p.splits = 1;
    const int64_t nb = (cache->B * cache->H + 7) / 8 * 8 * p.tiles * p.splits;
    if (!kv_launchable(nb, p.rt ? 256 : 64 * tile_waves(Dh)) || cache->B * Sq * Hq > 0x7fffffffLL) return HERO_ERR_SHAPE;
    AttnArgs a;
    a.c = kv_view(cache);
    a.q = (const uint16_t*)q;
    for (int t = 0; t < 3; ++t) a.qs[t] = q_strides[t];
    a.B = (int)cache->B; a.Hq = (int)Hq; a.Sq = (int)Sq; a.group = (int)(Hq / cache->H);
    a.scale = scale; a.causal = mask == HERO_MASK_CAUSAL; a.kv_len = kv_len; a.new_len = new_len;
    a.out = (uint16_t*)out; a.ldo = ldo; a.tiles = p.tiles; a.splits = p.splits;
    a.by_group = fast_div(a.group); a.by_splits = fast_div(p.splits); a.by_tiles = fast_div(p.tiles);
    a.by_heads = fast_div(a.c.H); a.by_bh8 = fast_div((cache->B * cache->H + 7) / 8);
    a.part = (float*)workspace; a.part_ml = a.part + (p.splits > 1 ? cache->B * Sq * Hq * p.splits * Dh : 0);
#define HERO_KVA(DH, FMT) (dt == HERO_BF16 ? launch<DH, FMT, HERO_BF16>(a, p, st) : launch<DH, FMT, HERO_F16>(a, p, st))
    if (cache->dt == HERO_I8) return Dh == 64 ? HERO_KVA(64, HERO_I8) : HERO_KVA(128, HERO_I8);
    return Dh == 64 ? HERO_KVA(64, HERO_F8E4M3) : HERO_KVA(128, HERO_F8E4M3);
#undef HERO_KVA
}
