// The block-scaled 8-bit KV cache written and read back: hero_kv_write, hero_kv_read.
#include "kv_cache.h"

namespace {

constexpr float SMALLEST = 0x1p-64f;       // no scale is smaller: the logarithm and the reciprocal that the attention takes of one stay in range

struct WriteArgs {
    KvView c;
    FastDiv by_heads;
    const uint16_t* x[2];                  // K, V
    int64_t xs[2][3];                      // batch, token, head
    int B, S, touched;
    const int32_t *kv_len, *new_len;
};

template <int FMT> struct Fmt;
template <> struct Fmt<HERO_I8> { static constexpr float most = 127.0f; };
template <> struct Fmt<HERO_F8E4M3> { static constexpr float most = 448.0f; };

// The definition's IEEE quotient x / s without a division: of r = 1 / s, rounded to nearest, x r is two units off at most, one correction with the
// exact remainder makes it one of the quotient's neighbours and the next the quotient rounded to nearest (Markstein's theorem; for every 11-bit
// mantissa of x and every mantissa of s it is, by trial).  The
// remainder is exact where a code can depend on it: |x / s| >= 2^-10 with s >= 2^-64 leaves it above 2^-100.  At a scale that is not finite: 0 for
// every finite x.
struct Divisor {
    float s, r;
    __device__ __forceinline__ explicit Divisor(float scale) {
        const bool ok = scale == scale && scale < INFINITY;
        s = ok ? scale : 1.0f;
        r = ok ? __fdiv_rn(1.0f, s) : 0.0f;
    }
    __device__ __forceinline__ float quotient(float x) const {
        float q = x * r;
        q = fmaf(fmaf(-q, s, x), r, q);
        return fmaf(fmaf(-q, s, x), r, q);
    }
};

// four codes of finite values in fp32 at a scale
template <int FMT>
__device__ __forceinline__ uint32_t codes4(const float* x, const Divisor& by) {
    float y[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) y[t] = by.quotient(x[t]);
    if constexpr (FMT == HERO_I8) return quant4_sat(y[0], y[1], y[2], y[3]);
    else return fp8x4_sat(y[0], y[1], y[2], y[3]);
}

template <int FMT>
__device__ __forceinline__ void values4(uint32_t w, float (&x)[4]) {
    if constexpr (FMT == HERO_I8) {
#pragma unroll
        for (int t = 0; t < 4; ++t) x[t] = (float)(int8_t)(w >> (8 * t));
    } else {
        const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
    }
}

// ------------------------------------------------------------------------------------------
// One unit = the new tokens of one block of one head, K or V: TPU threads hold them in registers (CH pieces of 8 values
// each), so that they are read once for the maximum and the codes.  The maximum is one of bit patterns: NaN > infinity > numbers.
// A unit whose block holds older tokens and whose maximum grows codes those anew from the cache.
// Up to 2048 values (a few tokens, or pages of 16) a unit is one wave's, else a workgroup's.  Bound by HBM and, in small calls, by the chain of length, block,
// scale and rows: 8 x 2048 tokens of 32 heads of 128 in 87 us, 4.6 TB/s (and read back 158, a large copy's rate; with IEEE
// divisions 176); 64 x 1 token 5 us, 16 x 301 in pages of 16 9 us (12.5 with the divisions, the look-up in front of the rows and 64-bit index arithmetic).
// ------------------------------------------------------------------------------------------
template <int FMT, int DT, int DH, int TPU, int CH>
__global__ __launch_bounds__(256) void kv_write_kernel(WriteArgs a) {
    constexpr int UPB = 256 / TPU;
    __shared__ uint32_t part[4];
    constexpr int cpr = DH / 8;
    const int tid = threadIdx.x % TPU;
    int h = (int)blockIdx.x * UPB + __builtin_amdgcn_readfirstlane((int)(threadIdx.x / TPU));
    const int t = a.by_heads.divmod(h), b = blockIdx.y, side = blockIdx.z;
    const int block = 1 << a.c.log2_block, cap = a.c.max_blocks << a.c.log2_block;
    const int len = a.kv_len[b], n = a.new_len ? min(max(a.new_len[b], 0), a.S) : a.S;
    const int64_t origin = (int64_t)len - n;                             // the position of row 0
    if (origin >= cap) return;
    const int begin = (int)max(origin, (int64_t)0), end = min(len, cap);
    const int64_t first = ((int64_t)(begin >> a.c.log2_block) + t) << a.c.log2_block;
    const int lo = (int)max((int64_t)begin, first), hi = (int)min((int64_t)end, first + block);
    if (lo >= hi) return;
    const uint16_t* const x = a.x[side] + (int64_t)b * a.xs[side][0] + (lo - origin) * a.xs[side][1] + (int64_t)h * a.xs[side][2];
    const int chunks = (hi - lo) * cpr;
    v4i raw[CH];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int at = tid + i * TPU;
        raw[i] = v4i{0, 0, 0, 0};
        if (at < chunks) raw[i] = *reinterpret_cast<const v4i*>(x + (int64_t)(at / cpr) * a.xs[side][1] + (at % cpr) * 8);
    }
    // (the rows are on their way while the block is looked up)
    const int blk = a.c.block_of(b, (int)(first >> a.c.log2_block));
    if (blk < 0) return;
    const KvSide sd = side ? a.c.v : a.c.k;
    float* const scale = sd.scale + (int64_t)blk * a.c.H + h;
    const bool older = lo > first;
    const float s_old = older ? *scale : 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t w = (uint32_t)raw[i][j] & 0x7fff7fffu;
            top = max(top, max(w & 0xffffu, w >> 16));
        }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if constexpr (TPU > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
        __syncthreads();                                                 // (every thread has read the scale, too)
        top = max(max(part[0], part[1]), max(part[2], part[3]));
    }
    const bool finite = top < (DT == HERO_BF16 ? 0x7f80u : 0x7c00u);
    const float wanted = fmaxf(__fdiv_rn(hp_to_f32<DT>(top), Fmt<FMT>::most), SMALLEST);
    const float s = !finite || s_old != s_old ? __builtin_nanf("") : fmaxf(fabsf(s_old), wanted);      // (a scale from elsewhere may be negative: coded anew then)
    if (tid == 0) *scale = s;
    const Divisor by(s);                                                 // (codes at a scale that is NaN: 0, whatever the values)
    uint8_t* const out = sd.codes + (int64_t)blk * sd.s_block + (int64_t)h * sd.s_head;
    const int r0 = (int)(lo - first);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int at = tid + i * TPU;
        if (at >= chunks) break;
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float y = hp_to_f32<DT>(((uint32_t)raw[i][j >> 1] >> (16 * (j & 1))) & 0xffffu);
            f[j] = finite ? y : 0.0f;
        }
        *reinterpret_cast<v2i*>(out + (int64_t)(r0 + at / cpr) * sd.s_row + (at % cpr) * 8) =
            v2i{(int)codes4<FMT>(f, by), (int)codes4<FMT>(f + 4, by)};
    }
    if (older && !(s == s_old)) {
        for (int at = tid; at < r0 * cpr; at += TPU) {
            v2i* const p = reinterpret_cast<v2i*>(out + (int64_t)(at / cpr) * sd.s_row + (at % cpr) * 8);
            v2i w = *p;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float f[4];
                values4<FMT>((uint32_t)w[j], f);
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = s == s ? f[e] * s_old : 0.0f;   // (of a scale that was NaN, too)
                w[j] = (int)codes4<FMT>(f, by);
            }
            *p = w;
        }
    }
}

struct ReadArgs {
    KvView c;
    void* out[2];
    int64_t os[2][3];
    int S, sides;                          // sides: 0 K, 1 V, 2 both
    const int32_t *start, *kv_len;
};

// A thread reads 16 codes of a row, a row being a head of a position, heads fastest (the order of the output).  Bound by HBM: 4 x 32768 positions of
// 8 heads of 128 in 139-140 us, 5.7 TB/s, above a large copy's rate (an earlier form in 159: with the index taken apart by 64-bit divisions 207; with two, four, eight rows to a
// thread 156, 172, 184; with streaming stores 219 and more).
template <int FMT, int DT, int DH>
__global__ __launch_bounds__(256) void kv_read_kernel(ReadArgs a) {
    constexpr int CPR = DH / 16, RPB = 256 / CPR;
    const int side = a.sides == 2 ? (int)blockIdx.z : a.sides, b = blockIdx.y;
    const uint32_t row0 = blockIdx.x * RPB, i0 = row0 / (uint32_t)a.c.H, h0 = row0 - i0 * (uint32_t)a.c.H;
    const uint32_t at = h0 + threadIdx.x / CPR, di = at / (uint32_t)a.c.H;
    const int h = (int)(at - di * (uint32_t)a.c.H), ch = threadIdx.x % CPR;
    const int64_t i = (int64_t)i0 + di, pos = (a.start ? (int64_t)a.start[b] : 0) + i;
    if (i >= a.S || pos < 0 || pos >= min(a.kv_len[b], a.c.max_blocks << a.c.log2_block)) return;
    const int blk = a.c.block_of(b, (int)(pos >> a.c.log2_block));
    const KvSide sd = side ? a.c.v : a.c.k;
    v4i w = {0, 0, 0, 0};
    float s = 0.0f;
    if (blk >= 0) {
        w = *reinterpret_cast<const v4i*>(sd.codes + (int64_t)blk * sd.s_block + (pos & ((1 << a.c.log2_block) - 1)) * sd.s_row +
                                          (int64_t)h * sd.s_head + ch * 16);
        s = sd.scale[(int64_t)blk * a.c.H + h];
    }
    const int64_t to = (int64_t)b * a.os[side][0] + i * a.os[side][1] + (int64_t)h * a.os[side][2] + ch * 16;
    float f[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        values4<FMT>((uint32_t)w[j], f[j]);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[j][e] *= s;
    }
    if constexpr (DT == HERO_F32) {
        float* const o = (float*)a.out[side] + to;
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<v4f*>(o + 4 * j) = v4f{f[j][0], f[j][1], f[j][2], f[j][3]};
    } else {
        uint16_t* const o = (uint16_t*)a.out[side] + to;
#pragma unroll
        for (int j = 0; j < 4; j += 2)
            *reinterpret_cast<v4i*>(o + 4 * j) = v4i{(int)pack2_hp<DT>(f[j][0], f[j][1]), (int)pack2_hp<DT>(f[j][2], f[j][3]),
                                                     (int)pack2_hp<DT>(f[j + 1][0], f[j + 1][1]), (int)pack2_hp<DT>(f[j + 1][2], f[j + 1][3])};
    }
}

template <int FMT, int DT, int DH>
hero_status launch_write(const WriteArgs& a, int rows, hipStream_t st) {
    const int64_t units = (int64_t)a.touched * a.c.H;                    // of a sequence's K (or V)
    const int chunks = rows * (DH / 8);                                  // of the fullest unit
    const int upb = chunks <= 256 ? 4 : 1;
    const int64_t nb = (units + upb - 1) / upb;
    if (!kv_launchable(nb, 256) || units > 0x7ffffff0LL) return HERO_ERR_SHAPE;
    const dim3 grid((unsigned)nb, (unsigned)a.B, 2), block(256);
#define HERO_KVW(TPU, CH) hipLaunchKernelGGL((kv_write_kernel<FMT, DT, DH, TPU, CH>), grid, block, 0, st, a)
    if (chunks <= 64) HERO_KVW(64, 1);
    else if (chunks <= 256) HERO_KVW(64, 4);
    else if (chunks <= 1024) HERO_KVW(256, 4);
    else HERO_KVW(256, 8);
#undef HERO_KVW
    return hero_launch_status();
}

}  // namespace

extern "C" hero_status hero_kv_write(const hero_kv_cache* cache, const void* k, const int64_t k_strides[4],
                                     const void* v, const int64_t v_strides[4], hero_dtype dt, int64_t S,
                                     const int32_t* kv_len, const int32_t* new_len, void* stream) {
    const hero_status ok = kv_check(cache);
    if (ok != HERO_OK) return ok;
    if (dt != HERO_BF16 && dt != HERO_F16) return HERO_ERR_UNSUPPORTED;
    if (S < 0 || S > (1LL << 30)) return HERO_ERR_SHAPE;
    if (cache->B == 0 || cache->H == 0 || S == 0) return HERO_OK;
    for (int side = 0; side < 2; ++side) {
        const hero_status r = kv_check_rows(side ? v : k, side ? v_strides : k_strides);
        if (r != HERO_OK) return r;
    }
    if (!kv_len) return HERO_ERR_NULL;
    if (((uintptr_t)kv_len & 3) || ((uintptr_t)new_len & 3)) return HERO_ERR_ALIGN;
    if (cache->n_blocks == 0 || cache->max_blocks == 0) return HERO_OK;  // nowhere to write to
    WriteArgs a;
    a.c = kv_view(cache);
    a.x[0] = (const uint16_t*)k; a.x[1] = (const uint16_t*)v;
    for (int t = 0; t < 3; ++t) { a.xs[0][t] = k_strides[t]; a.xs[1][t] = v_strides[t]; }
    a.B = (int)cache->B; a.S = (int)S; a.kv_len = kv_len; a.new_len = new_len;
    a.touched = (int)((S + cache->block - 2) / cache->block + 1);        // S tokens lie in at most so many blocks
    if (a.touched > a.c.max_blocks) a.touched = a.c.max_blocks;
    const int rows = S < cache->block ? (int)S : cache->block;
    a.by_heads = fast_div(a.c.H);
    hipStream_t st = (hipStream_t)stream;
#define HERO_KVW(FMT, DT) (cache->Dh == 64 ? launch_write<FMT, DT, 64>(a, rows, st) : launch_write<FMT, DT, 128>(a, rows, st))
    if (cache->dt == HERO_I8) return dt == HERO_BF16 ? HERO_KVW(HERO_I8, HERO_BF16) : HERO_KVW(HERO_I8, HERO_F16);
    return dt == HERO_BF16 ? HERO_KVW(HERO_F8E4M3, HERO_BF16) : HERO_KVW(HERO_F8E4M3, HERO_F16);
#undef HERO_KVW
}

extern "C" hero_status hero_kv_read(const hero_kv_cache* cache, void* k_out, const int64_t k_strides[4],
                                    void* v_out, const int64_t v_strides[4], hero_dtype out_dt, int64_t S,
                                    const int32_t* start, const int32_t* kv_len, void* stream) {
    const hero_status ok = kv_check(cache);
    if (ok != HERO_OK) return ok;
    if (out_dt != HERO_BF16 && out_dt != HERO_F16 && out_dt != HERO_F32) return HERO_ERR_UNSUPPORTED;
    if (S < 0 || S > (1LL << 30)) return HERO_ERR_SHAPE;
    if (cache->B == 0 || cache->H == 0 || S == 0) return HERO_OK;
    if (!k_out && !v_out) return HERO_ERR_NULL;
    for (int side = 0; side < 2; ++side) {
        if (!(side ? v_out : k_out)) continue;
        const hero_status r = kv_check_rows(side ? v_out : k_out, side ? v_strides : k_strides);
        if (r != HERO_OK) return r;
    }
    if (!kv_len) return HERO_ERR_NULL;
    if (((uintptr_t)kv_len & 3) || ((uintptr_t)start & 3)) return HERO_ERR_ALIGN;
    ReadArgs a;
    a.c = kv_view(cache);
    a.out[0] = k_out; a.out[1] = v_out;
    for (int t = 0; t < 3; ++t) { a.os[0][t] = k_out ? k_strides[t] : 0; a.os[1][t] = v_out ? v_strides[t] : 0; }
    a.S = (int)S; a.start = start; a.kv_len = kv_len;
    a.sides = k_out && v_out ? 2 : (v_out ? 1 : 0);
    const int64_t per = 256 / (cache->Dh / 16), nb = (S * cache->H + per - 1) / per;
    if (!kv_launchable(nb, 256) || S * cache->H > 0x7fffff00LL) return HERO_ERR_SHAPE;
    hipStream_t st = (hipStream_t)stream;
    const dim3 block(256), grid((unsigned)nb, (unsigned)cache->B, a.sides == 2 ? 2 : 1);
#define HERO_KVR(FMT, DT) do { if (cache->Dh == 64) hipLaunchKernelGGL((kv_read_kernel<FMT, DT, 64>), grid, block, 0, st, a); \
                               else hipLaunchKernelGGL((kv_read_kernel<FMT, DT, 128>), grid, block, 0, st, a); } while (0)
    if (cache->dt == HERO_I8) {
        if (out_dt == HERO_BF16) HERO_KVR(HERO_I8, HERO_BF16);
        else if (out_dt == HERO_F16) HERO_KVR(HERO_I8, HERO_F16);
        else HERO_KVR(HERO_I8, HERO_F32);
    } else {
        if (out_dt == HERO_BF16) HERO_KVR(HERO_F8E4M3, HERO_BF16);
        else if (out_dt == HERO_F16) HERO_KVR(HERO_F8E4M3, HERO_F16);
        else HERO_KVR(HERO_F8E4M3, HERO_F32);
    }
#undef HERO_KVR
    return hero_launch_status();
}
