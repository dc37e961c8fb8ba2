// Products grouped by expert, of every size: what the faster kernels do not take (a K that ends in half a slab, rows that lie 16 MB or more apart, rows
// gathered from more than 4 GB).  Both operands come straight from memory into the operands of the matrix instructions, by 64-bit addresses.
#include "gemm_grouped.h"

using namespace hero_gemm;

namespace {

constexpr int ROW_WAVES = 8;

template <int ADT, typename ACC>
__device__ __forceinline__ ACC mfma_step128(const v4i (&w)[2], const v4i (&a)[2], ACC c) {
    if constexpr (ADT == HERO_F8E4M3) {
        const v8i w8 = {w[0][0], w[0][1], w[0][2], w[0][3], w[1][0], w[1][1], w[1][2], w[1][3]};
        const v8i a8 = {a[0][0], a[0][1], a[0][2], a[0][3], a[1][0], a[1][1], a[1][2], a[1][3]};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w8, a8, c, 0, 0, 0, 0, 0, 0);
    } else {
#pragma unroll
        for (int s = 0; s < 2; ++s) c = mfma16_step<ADT>(w[s], a[s], c);
        return c;
    }
}

// A workgroup owns 16 TM rows of one expert and 16 CT columns; its eight waves share K, taking steps of 128 bytes in turn, DEPTH of
// which a wave has under way.  Lane l holds 16 bytes of row l % 16 of each operand, piece l / 16 of the step's lower 64 bytes and of its upper
// ones; the result of lane l are the columns 4 (l / 16) .. + 3 of row l % 16.  The eight partial sums meet in LDS, in the order of the waves.
template <int ADT, int TM, int CT, int DEPTH>
__global__ __launch_bounds__(ROW_WAVES * 64, 4) void grouped_rows_kernel(GroupedArgs a) {
    using ACC = typename Acc4Of<ADT>::type;
    constexpr bool HP = ADT == HERO_BF16 || ADT == HERO_F16;
    constexpr int SLOTS = TM * CT * 64;
    static_assert(SLOTS <= ROW_WAVES * 64, "a thread for every four results");
    __shared__ ACC part[ROW_WAVES * SLOTS];
    const GemmArgs& g = a.g;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const GroupTile t = group_tile<16 * TM>(a, blockIdx.x % NUM_XCD, blockIdx.x / NUM_XCD, g.ntn, lane);
    if (t.rows == 0) return;
    const int n0 = t.col_tile * (16 * CT);
    auto source = [&](int row) { return a.row_index ? min(max(a.row_index[row], 0), a.MA - 1) : row; };

    const int r16 = lane & 15, piece = (lane >> 4) * 16;
    const int8_t* pa[TM]; const int8_t* pw[CT];
#pragma unroll
    for (int i = 0; i < TM; ++i) pa[i] = g.A + (int64_t)source(t.row0 + min(i * 16 + r16, t.rows - 1)) * g.lda + piece;
#pragma unroll
    for (int c = 0; c < CT; ++c) pw[c] = g.Bt + (int64_t)t.e * a.expert_stride + (int64_t)min(n0 + c * 16 + r16, g.N - 1) * g.ldb + piece;

    const int steps = (g.K >> 7) + ((g.K >> 6) & 1), half = (g.K & 64) ? steps - 1 : -1;      // (the last step may be half a one; K goes up to 2^31 - 64)
    v4i fa[DEPTH][TM][2], fw[DEPTH][CT][2];
    auto load = [&](int s, v4i (&xa)[TM][2], v4i (&xw)[CT][2]) {
        if (s >= steps) return;                                     // (uniform)
        const int64_t k = (int64_t)s * 128;
#pragma unroll
        for (int c = 0; c < CT; ++c) xw[c][0] = *reinterpret_cast<const v4i*>(pw[c] + k);
#pragma unroll
        for (int i = 0; i < TM; ++i) xa[i][0] = *reinterpret_cast<const v4i*>(pa[i] + k);
        if (s != half) {
#pragma unroll
            for (int c = 0; c < CT; ++c) xw[c][1] = *reinterpret_cast<const v4i*>(pw[c] + k + 64);
#pragma unroll
            for (int i = 0; i < TM; ++i) xa[i][1] = *reinterpret_cast<const v4i*>(pa[i] + k + 64);
        } else {
#pragma unroll
            for (int c = 0; c < CT; ++c) xw[c][1] = v4i{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < TM; ++i) xa[i][1] = v4i{0, 0, 0, 0};
        }
    };
    ACC acc[CT][TM];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[c][i] = ACC{0, 0, 0, 0};
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load(wave + d * ROW_WAVES, fa[d], fw[d]);
    for (int s0 = wave; s0 < steps; s0 += DEPTH * ROW_WAVES) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int s = s0 + d * ROW_WAVES;
            if (s < steps) {
#pragma unroll
                for (int c = 0; c < CT; ++c)
#pragma unroll
                    for (int i = 0; i < TM; ++i) acc[c][i] = mfma_step128<ADT>(fw[d][c], fa[d][i], acc[c][i]);
                load(s + DEPTH * ROW_WAVES, fa[d], fw[d]);
            }
        }
    }
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < TM; ++i) part[wave * SLOTS + (c * TM + i) * 64 + lane] = acc[c][i];
    __syncthreads();
    if (tid >= SLOTS) return;
    const int c = (tid >> 6) / TM, m = ((tid >> 6) % TM) * 16 + r16, n = n0 + c * 16 + (lane >> 4) * 4;
    if (m >= t.rows || n >= g.N) return;
    const int row = t.row0 + m;
    ACC sum = part[tid];
#pragma unroll
    for (int w = 1; w < ROW_WAVES; ++w) {
        const ACC p = part[w * SLOTS + tid];
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] += p[k];
    }
    const bool gelu = a.epi == HERO_EPI_DEQUANT_GELU || a.epi == HERO_EPI_GELU_REQUANT;
    const float rs = !HP && g.a_row_scale ? g.a_row_scale[source(row)] : 1.0f;
    const int64_t v0 = (int64_t)t.e * g.N;
    float y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t at = v0 + min(n + k, g.N - 1);
        const float b = g.bias ? g.bias[at] : 0.0f;
        float v = (float)sum[k];
        v = HP ? v + b : fmaf(v * rs, g.b_col_scale[at], b);        // (no row scale: 1)
        if (gelu) v = gelu_erf(v);
        if (a.epi == HERO_EPI_GELU_REQUANT) v = v * __fdiv_rn(1.0f, g.out_col_scale[at]);
        y[k] = v;
    }
    const int64_t o = (int64_t)row * g.ldc + n;
    const int left = g.N - n;
    if (a.c_dt == HERO_I8 || a.c_dt == HERO_F8E4M3) {
        const uint32_t w = a.c_dt == HERO_I8 ? quant4_sat(y[0], y[1], y[2], y[3]) : fp8x4_sat(y[0], y[1], y[2], y[3]);
        if (left >= 4) *reinterpret_cast<uint32_t*>((int8_t*)g.C + o) = w;
        else for (int k = 0; k < left; ++k) ((int8_t*)g.C)[o + k] = (int8_t)(w >> (8 * k));
    } else {
        const bool bf = a.c_dt == HERO_BF16;
        const uint32_t lo = bf ? pack2_hp<HERO_BF16>(y[0], y[1]) : pack2_hp<HERO_F16>(y[0], y[1]);
        const uint32_t hi = bf ? pack2_hp<HERO_BF16>(y[2], y[3]) : pack2_hp<HERO_F16>(y[2], y[3]);
        if (left >= 4) *reinterpret_cast<v2i*>((uint16_t*)g.C + o) = v2i{(int)lo, (int)hi};
        else for (int k = 0; k < left; ++k) ((uint16_t*)g.C)[o + k] = (uint16_t)((k < 2 ? lo : hi) >> (16 * (k & 1)));
    }
}

template <int ADT, int TM, int CT, int DEPTH>
hero_status launch(const GroupedArgs& ga, hipStream_t st) {
    GroupedArgs a = ga;
    a.g.ntn = (a.g.N + 16 * CT - 1) / (16 * CT);
    const int64_t tiles = most_row_tiles(a.g.M, a.E, 16 * TM) * a.g.ntn, per = (tiles + NUM_XCD - 1) / NUM_XCD;
    if (per * NUM_XCD * ROW_WAVES * 64 > 0xffffffffLL) return HERO_ERR_SHAPE;
    hipLaunchKernelGGL((grouped_rows_kernel<ADT, TM, CT, DEPTH>), dim3((unsigned)(per * NUM_XCD)), dim3(ROW_WAVES * 64), 0, st, a);
    return hero_launch_status();
}

}  // namespace

namespace hero_gemm {
hero_status launch_grouped_rows(const GroupedArgs& a, hero_dtype adt, hipStream_t st) {
    switch (adt) {
    case HERO_I8: return launch<HERO_I8, 2, 2, 2>(a, st);
    case HERO_F8E4M3: return launch<HERO_F8E4M3, 2, 2, 2>(a, st);
    case HERO_BF16: return launch<HERO_BF16, 2, 2, 2>(a, st);
    case HERO_F16: return launch<HERO_F16, 2, 2, 2>(a, st);
    default: return HERO_ERR_UNSUPPORTED;
    }
}
}  // namespace hero_gemm
