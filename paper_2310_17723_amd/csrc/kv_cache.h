// The block-scaled 8-bit KV cache as its kernels see it (kv_cache.hip: written and read back; kv_attn.hip: attended over).
#pragma once
#include "hero_common.h"

// n / d for 0 <= n < 2^31 without a division: (floor(m n / 2^32) + n) >> s with 2^s >= d, m = floor(2^32 (2^s - d) / d) + 1 (Granlund and
// Montgomery's division by an invariant integer)
struct FastDiv {
    uint32_t m, s, d;
    __device__ __forceinline__ int div(int n) const { return (int)((__umulhi((uint32_t)n, m) + (uint32_t)n) >> s); }
    __device__ __forceinline__ int divmod(int& n) const {                  // the remainder stays in n
        const int q = div(n);
        n -= q * (int)d;
        return q;
    }
};
static inline FastDiv fast_div(int64_t d) {
    FastDiv f{0, 0, (uint32_t)d};
    while ((1ULL << f.s) < (uint64_t)d) ++f.s;
    f.m = (uint32_t)((((1ULL << f.s) - (uint64_t)d) << 32) / (uint64_t)d) + 1;
    return f;
}

struct KvSide { uint8_t* codes; float* scale; int64_t s_block, s_row, s_head; };       // element strides

struct KvView {
    KvSide k, v;
    const int32_t* table;                  // [B][max_blocks], or NULL: block b max_blocks + j
    int n_blocks, max_blocks, H, log2_block;
    // the block that holds positions [j block, (j + 1) block) of sequence b, or -1 (a table's index outside the pool)
    __device__ __forceinline__ int block_of(int b, int j) const {
        const int64_t at = (int64_t)b * max_blocks + j;
        const int blk = table ? table[at] : (int)at;
        return (unsigned)blk < (unsigned)n_blocks ? blk : -1;
    }
};

// Everything about a cache that the host can check; HERO_OK with B, H, max_blocks or n_blocks 0 too.
static inline hero_status kv_check(const hero_kv_cache* c) {
    if (!c) return HERO_ERR_NULL;
    if (c->B < 0 || c->max_blocks < 0 || c->n_blocks < 0 || c->H < 0) return HERO_ERR_SHAPE;
    if (c->Dh != 64 && c->Dh != 128) return HERO_ERR_UNSUPPORTED;
    if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != 128) return HERO_ERR_UNSUPPORTED;
    if (c->dt != HERO_I8 && c->dt != HERO_F8E4M3) return HERO_ERR_UNSUPPORTED;
    if (c->B > 65535 || c->H > 65535 || c->n_blocks > 0x7fffffffLL || c->max_blocks > (1LL << 30) / c->block) return HERO_ERR_SHAPE;
    if (c->B == 0 || c->H == 0) return HERO_OK;
    if (!c->block_table && c->n_blocks < c->B * c->max_blocks) return HERO_ERR_SHAPE;
    if (c->n_blocks > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale)) return HERO_ERR_NULL;
    for (const int64_t* s : {c->k_strides, c->v_strides}) {
        if (s[3] != 1) return HERO_ERR_UNSUPPORTED;
        if (s[0] % 16 || s[1] % 16 || s[2] % 16) return HERO_ERR_ALIGN;
        if (s[0] < 0 || s[1] < 0 || s[2] < 0 || s[1] > 0x7fffffffLL / c->block) return HERO_ERR_SHAPE;
    }
    if (!hero_aligned16(c->k) || !hero_aligned16(c->v) || ((uintptr_t)c->k_scale & 3) || ((uintptr_t)c->v_scale & 3) ||
        ((uintptr_t)c->block_table & 3)) return HERO_ERR_ALIGN;
    return HERO_OK;
}

static inline KvView kv_view(const hero_kv_cache* c) {
    KvView v;
    v.k = {(uint8_t*)c->k, c->k_scale, c->k_strides[0], c->k_strides[1], c->k_strides[2]};
    v.v = {(uint8_t*)c->v, c->v_scale, c->v_strides[0], c->v_strides[1], c->v_strides[2]};
    v.table = c->block_table;
    v.n_blocks = (int)c->n_blocks; v.max_blocks = (int)c->max_blocks; v.H = c->H;
    v.log2_block = c->block == 16 ? 4 : c->block == 32 ? 5 : c->block == 64 ? 6 : 7;
    return v;
}

// whether `groups` workgroups can be launched: HIP counts a dimension's threads in 32 bits
static inline bool kv_launchable(int64_t groups, int threads) { return groups <= 0xffffffffLL / threads; }

// strides of [B, S, heads, Dh] rows: unit channels, the others multiples of 8 elements
static inline hero_status kv_check_rows(const void* p, const int64_t* s) {
    if (!p || !s) return HERO_ERR_NULL;
    if (s[3] != 1) return HERO_ERR_UNSUPPORTED;
    if (s[0] % 8 || s[1] % 8 || s[2] % 8 || !hero_aligned16(p)) return HERO_ERR_ALIGN;
    return HERO_OK;
}
