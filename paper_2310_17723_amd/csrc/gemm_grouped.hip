// The entry points of the products grouped by expert: hero_int8_gemm_grouped, hero_fp8_gemm_grouped, hero_hp_gemm_grouped.
#include "gemm_grouped.h"

using namespace hero_gemm;

namespace {

struct Request {
    const void* A; int64_t lda, MA; const float* a_row_scale; const int32_t* row_index;
    const void* Bt; int64_t ldb, expert_stride; const float* b_col_scale; const float* bias;
    hero_epilogue epi; const float* out_col_scale; void* C; hero_dtype c_dt; int64_t ldc;
    const int32_t* offsets; int64_t E, R, N, K;
};

bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

// Everything that can be checked, before anything is launched.  *noop: nothing to do.
hero_status check(const Request& q, hero_dtype dt, bool* noop) {
    *noop = false;
    const bool hp = dt == HERO_BF16 || dt == HERO_F16;
    const int es = hp ? 2 : 1;
    if (q.E < 0 || q.R < 0 || q.N < 0 || q.K <= 0 || q.MA < 0) return HERO_ERR_SHAPE;
    if (q.R >= (1LL << 23) || q.N > 0x7fffff00LL || q.K > 0x7fffffffLL / es || q.MA > 0x7fffffffLL) return HERO_ERR_SHAPE;
    if (q.E > MAX_EXPERTS || q.K * es % KMULT != 0) return HERO_ERR_UNSUPPORTED;
    if (q.lda < q.K || q.ldb < q.K || q.ldc < q.N || q.expert_stride < 0) return HERO_ERR_SHAPE;
    const bool c16 = q.c_dt == HERO_F16 || q.c_dt == HERO_BF16;
    switch (q.epi) {
    case HERO_EPI_DEQUANT: case HERO_EPI_DEQUANT_GELU:
        if (!c16 || (hp && q.c_dt != dt)) return HERO_ERR_UNSUPPORTED;
        break;
    case HERO_EPI_REQUANT: case HERO_EPI_GELU_REQUANT:
        if (hp || q.c_dt != dt) return HERO_ERR_UNSUPPORTED;
        break;
    default: return HERO_ERR_UNSUPPORTED;
    }
    if (q.E == 0 || q.R == 0 || q.N == 0) { *noop = true; return HERO_OK; }
    if (q.row_index ? q.MA == 0 : q.MA != q.R) return HERO_ERR_SHAPE;
    if (!q.A || !q.Bt || !q.C || !q.offsets) return HERO_ERR_NULL;
    if (!hp && !q.b_col_scale) return HERO_ERR_NULL;
    if (q.epi == HERO_EPI_GELU_REQUANT && !q.out_col_scale) return HERO_ERR_NULL;
    const int64_t unit = 16 / es;
    if (q.lda % unit != 0 || q.ldb % unit != 0 || q.expert_stride % unit != 0 || q.ldc % 4 != 0) return HERO_ERR_ALIGN;
    if (!hero_aligned16(q.A) || !hero_aligned16(q.Bt) || !hero_aligned16(q.C)) return HERO_ERR_ALIGN;
    if (!aligned4(q.offsets) || !aligned4(q.row_index) || !aligned4(q.a_row_scale) || !aligned4(q.b_col_scale) || !aligned4(q.bias) ||
        !aligned4(q.out_col_scale)) return HERO_ERR_ALIGN;
    return HERO_OK;
}

template <int ADT, int EPI, int CDT>
hero_status launch_tile(const GroupedArgs& a, int tile, hipStream_t st) {
    return tile < GROUPED_128 ? launch_grouped_ring<ADT, EPI, CDT>(a, (RingForm)(tile - GROUPED_RING), st) : launch_grouped_tile<ADT, EPI, CDT>(a, tile, st);
}
template <int ADT, int CDT8>
hero_status launch_tile8(const GroupedArgs& a, int tile, hipStream_t st) {
    const bool bf = a.c_dt == HERO_BF16;
    switch (a.epi) {
    case HERO_EPI_REQUANT: return launch_tile<ADT, HERO_EPI_REQUANT, CDT8>(a, tile, st);
    case HERO_EPI_GELU_REQUANT: return launch_tile<ADT, HERO_EPI_GELU_REQUANT, CDT8>(a, tile, st);
    case HERO_EPI_DEQUANT: return bf ? launch_tile<ADT, HERO_EPI_DEQUANT, HERO_BF16>(a, tile, st) : launch_tile<ADT, HERO_EPI_DEQUANT, HERO_F16>(a, tile, st);
    default: return bf ? launch_tile<ADT, HERO_EPI_DEQUANT_GELU, HERO_BF16>(a, tile, st) : launch_tile<ADT, HERO_EPI_DEQUANT_GELU, HERO_F16>(a, tile, st);
    }
}
template <int DT>
hero_status launch_tile16(const GroupedArgs& a, int tile, hipStream_t st) {
    return a.epi == HERO_EPI_DEQUANT_GELU ? launch_tile<DT, HERO_EPI_DEQUANT_GELU, DT>(a, tile, st) : launch_tile<DT, HERO_EPI_DEQUANT, DT>(a, tile, st);
}

hero_status run(const Request& q, hero_dtype dt, int tile, void* stream) {
    bool noop = false;
    const hero_status cs = check(q, dt, &noop);
    if (cs != HERO_OK || noop) return cs;
    const int es = dt == HERO_BF16 || dt == HERO_F16 ? 2 : 1;
    GroupedArgs a;
    GemmArgs& g = a.g;
    g.A = (const int8_t*)q.A; g.lda = q.lda * es; g.a_row_scale = es == 1 ? q.a_row_scale : nullptr;
    g.Bt = (const int8_t*)q.Bt; g.ldb = q.ldb * es; g.b_col_scale = q.b_col_scale; g.bias = q.bias;
    g.residual = nullptr; g.ldr = 0; g.out_col_scale = q.out_col_scale;
    g.C = q.C; g.ldc = q.ldc; g.M = (int)q.R; g.N = (int)q.N; g.K = (int)(q.K * es);
    g.ntm = g.ntn = g.per_xcd = 0; g.ksplit = 1; g.kslabs = 0;
    a.offsets = q.offsets; a.row_index = q.row_index; a.E = (int)q.E; a.MA = (int)q.MA;
    a.expert_stride = q.expert_stride * es; a.epi = q.epi; a.c_dt = q.c_dt;
    hipStream_t st = (hipStream_t)stream;
    if (tile == 0) tile = grouped_form(a);
    if (tile == GROUPED_ANY) return launch_grouped_rows(a, dt, st);
    if (!(tile < GROUPED_128 ? grouped_ring_ok(a) : grouped_tile_ok(a))) return HERO_ERR_UNSUPPORTED;
    switch (dt) {
    case HERO_I8: return launch_tile8<HERO_I8, HERO_I8>(a, tile, st);
    case HERO_F8E4M3: return launch_tile8<HERO_F8E4M3, HERO_F8E4M3>(a, tile, st);
    case HERO_BF16: return launch_tile16<HERO_BF16>(a, tile, st);
    default: return launch_tile16<HERO_F16>(a, tile, st);
    }
}

}  // namespace

extern "C" hero_status hero_int8_gemm_grouped(const int8_t* A, int64_t lda, int64_t MA, const float* a_row_scale, const int32_t* row_index,
                                              const int8_t* Bt, int64_t ldb, int64_t expert_stride, const float* b_col_scale, const float* bias,
                                              hero_epilogue epi, const float* out_col_scale, void* C, hero_dtype c_dt, int64_t ldc,
                                              const int32_t* offsets, int64_t E, int64_t R, int64_t N, int64_t K, void* stream) {
    const Request q{A, lda, MA, a_row_scale, row_index, Bt, ldb, expert_stride, b_col_scale, bias, epi, out_col_scale, C, c_dt, ldc, offsets, E, R, N, K};
    return run(q, HERO_I8, 0, stream);
}

extern "C" hero_status hero_fp8_gemm_grouped(const void* A, int64_t lda, int64_t MA, const float* a_row_scale, const int32_t* row_index,
                                             const void* Bt, int64_t ldb, int64_t expert_stride, const float* b_col_scale, const float* bias,
                                             hero_epilogue epi, const float* out_col_scale, void* C, hero_dtype c_dt, int64_t ldc,
                                             const int32_t* offsets, int64_t E, int64_t R, int64_t N, int64_t K, void* stream) {
    const Request q{A, lda, MA, a_row_scale, row_index, Bt, ldb, expert_stride, b_col_scale, bias, epi, out_col_scale, C, c_dt, ldc, offsets, E, R, N, K};
    return run(q, HERO_F8E4M3, 0, stream);
}

extern "C" hero_status hero_hp_gemm_grouped(const void* A, int64_t lda, int64_t MA, const int32_t* row_index,
                                            const void* Bt, int64_t ldb, int64_t expert_stride, const float* bias, int gelu,
                                            void* C, int64_t ldc, const int32_t* offsets, int64_t E, int64_t R, int64_t N, int64_t K,
                                            hero_dtype dt, void* stream) {
    if (dt != HERO_BF16 && dt != HERO_F16) return HERO_ERR_UNSUPPORTED;
    const Request q{A, lda, MA, nullptr, row_index, Bt, ldb, expert_stride, nullptr, bias, gelu ? HERO_EPI_DEQUANT_GELU : HERO_EPI_DEQUANT, nullptr,
                    C, dt, ldc, offsets, E, R, N, K};
    return run(q, dt, 0, stream);
}

extern "C" hero_status hero_gemm_grouped_tile(hero_dtype dt, const void* A, int64_t lda, int64_t MA, const float* a_row_scale, const int32_t* row_index,
                                              const void* Bt, int64_t ldb, int64_t expert_stride, const float* b_col_scale, const float* bias,
                                              hero_epilogue epi, const float* out_col_scale, void* C, hero_dtype c_dt, int64_t ldc,
                                              const int32_t* offsets, int64_t E, int64_t R, int64_t N, int64_t K, void* stream, int tile) {
    if (dt != HERO_I8 && dt != HERO_F8E4M3 && dt != HERO_BF16 && dt != HERO_F16) return HERO_ERR_UNSUPPORTED;
    if (tile < 0 || (tile > GROUPED_ANY && tile < GROUPED_RING) || (tile > GROUPED_RING + RING_128x64 && tile != GROUPED_128 && tile != GROUPED_256 && tile != GROUPED_256x128)) return HERO_ERR_UNSUPPORTED;

    const Request q{A, lda, MA, a_row_scale, row_index, Bt, ldb, expert_stride, b_col_scale, bias, epi, out_col_scale, C, c_dt, ldc, offsets, E, R, N, K};
    return run(q, dt, tile, stream);
}
