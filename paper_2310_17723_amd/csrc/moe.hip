// The router of a mixture-of-experts MLP (choice of experts, order of their rows) and the weighted sum behind the experts:
// hero_moe_route, hero_moe_combine.
#include "hero_common.h"
#include <float.h>

namespace {

constexpr int MAX_E = 512, MAX_K = 16;
constexpr int TOKENS = 64;                  // of a workgroup: at most 1024 choices, one for each of its threads
constexpr int THREADS = 1024, WAVES = THREADS / 64;

struct RouteArgs {
    const void* logits; int64_t ldl;
    int T, E, k, renorm, nb;                // nb workgroups of TOKENS tokens
    int32_t* expert; float* weight; int32_t* slot; int32_t* row_token; int32_t* offsets;
    int32_t* counts;                        // [E][nb]: choices of each workgroup; behind the scan those of the workgroups before it
    int32_t* totals;                        // [E]
};

template <int DT>
__device__ __forceinline__ float logit_at(const void* p, int64_t i) {
    if constexpr (DT == HERO_F32) return ((const float*)p)[i];
    else return hp_to_f32<DT>(((const uint16_t*)p)[i]);
}

// A wave chooses the experts of one token: lane l holds the logits of experts l V .. l V + V - 1, so that the first lane (and of its
// experts the first) of those that hold the maximum is the lowest index.  k rounds of a maximum over the wave and a ballot.
template <int DT, int V>
__device__ __forceinline__ void choose(const RouteArgs& a, int t, int lane, int32_t* chosen) {
    float l[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = lane * V + v;
        const float x = logit_at<DT>(a.logits, (int64_t)t * a.ldl + min(e, a.E - 1));
        l[v] = e < a.E && x == x ? fminf(x, FLT_MAX) : -INFINITY;
    }
    float top = 0.0f, mine = -INFINITY, all = 0.0f;               // lane j keeps the logit of choice j
    int who = -1;
    for (int j = 0; j < a.k; ++j) {
        float best = l[0];
#pragma unroll
        for (int v = 1; v < V; ++v) best = fmaxf(best, l[v]);
        const float m = wave_reduce<true>(best);
        if (j == 0) {
            top = m > -INFINITY ? m : 0.0f;
            if (!a.renorm) {
#pragma unroll
                for (int v = 0; v < V; ++v) all += expf(l[v] - top);
            }
        }
        if (!(m > -INFINITY)) break;                              // (uniform)
        const int first = __ffsll((unsigned long long)__ballot(best == m)) - 1;
        int at = V - 1;
#pragma unroll
        for (int v = V - 2; v >= 0; --v) if (l[v] == m) at = v;
        at = __builtin_amdgcn_readlane(at, first);
        if (lane == j) { mine = m; who = first * V + at; }
#pragma unroll
        for (int v = 0; v < V; ++v) if (lane == first && v == at) l[v] = -INFINITY;
    }
    const float p = who >= 0 ? expf(mine - top) : 0.0f;
    const float total = wave_reduce<false>(a.renorm ? p : all);
    if (lane < a.k) {
        a.expert[(int64_t)t * a.k + lane] = who;
        a.weight[(int64_t)t * a.k + lane] = who >= 0 ? __fdiv_rn(p, total) : 0.0f;
        if (chosen) chosen[lane] = who;
    }
}

// Choice c of this workgroup, one to a thread: how many choices of the same expert come before it in its wave, and in the workgroup's
// earlier waves (`before` [WAVES][E]).  Equal experts of a wave are found bit by bit of their number.
__device__ __forceinline__ int rank_in_group(int e, int E, int* before, int* group_total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < WAVES * E; i += THREADS) before[i] = 0;
    __syncthreads();
    unsigned long long same = __ballot(e >= 0);
#pragma unroll
    for (int b = 0; b < 9; ++b) {
        const unsigned long long set = __ballot((e >> b) & 1);
        same &= (e >> b) & 1 ? set : ~set;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    if (e >= 0 && rank == 0) before[wave * E + e] = __popcll(same);
    __syncthreads();
    for (int i = threadIdx.x; i < E; i += THREADS) {
        int sum = 0;
        for (int w = 0; w < WAVES; ++w) { const int n = before[w * E + i]; before[w * E + i] = sum; sum += n; }
        if (group_total) group_total[i] = sum;
    }
    __syncthreads();
    return rank + (e >= 0 ? before[wave * E + e] : 0);
}

// start[e] = sum of total[0 .. e - 1] for e <= E, by the first wave (eight experts to a lane)
__device__ __forceinline__ void starts(const int* total, int E, int* start) {
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        int n[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) { n[i] = lane * 8 + i < E ? total[lane * 8 + i] : 0; sum += n[i]; }
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const int x = __shfl_up(upto, o); if (lane >= o) upto += x; }
        int at = upto - sum;
#pragma unroll
        for (int i = 0; i < 8; ++i) { if (lane * 8 + i <= E) start[lane * 8 + i] = at; at += n[i]; }
        if (lane == 63 && E == 512) start[512] = at;
    }
    __syncthreads();
}

// Choices of TOKENS tokens, a wave for each in turn.  ONE: the only workgroup of the call, which orders the rows as well; else it leaves
// behind how many of its choices fall to each expert.
template <int DT, int V, bool ONE>
__global__ __launch_bounds__(THREADS) void route_choose_kernel(RouteArgs a) {
    __shared__ int32_t chosen[TOKENS * MAX_K];
    __shared__ int before[ONE ? WAVES * MAX_E : MAX_E], total[ONE ? MAX_E : 1], start[ONE ? MAX_E + 1 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int t0 = blockIdx.x * TOKENS, nt = min(TOKENS, a.T - t0);
    if (!ONE) {
        for (int i = threadIdx.x; i < a.E; i += THREADS) before[i] = 0;
        __syncthreads();
    }
    for (int t = wave; t < nt; t += WAVES) choose<DT, V>(a, t0 + t, lane, chosen + t * a.k);
    __syncthreads();
    const int c = threadIdx.x, e = c < nt * a.k ? chosen[c] : -1;
    if constexpr (ONE) {
        const int r = rank_in_group(e, a.E, before, total);
        starts(total, a.E, start);
        if (c < nt * a.k) a.slot[c] = e >= 0 ? start[e] + r : -1;
        if (e >= 0) a.row_token[start[e] + r] = c / a.k;
        if (c < nt * a.k && c >= start[a.E]) a.row_token[c] = -1;
        for (int i = threadIdx.x; i <= a.E; i += THREADS) a.offsets[i] = start[i];
    } else {
        if (e >= 0) atomicAdd(&before[e], 1);                       // (counts: their order does not show)
        __syncthreads();
        for (int i = threadIdx.x; i < a.E; i += THREADS) a.counts[(int64_t)i * a.nb + blockIdx.x] = before[i];
    }
}

// counts[e][b] -> choices of e in the workgroups before b; totals[e].  A workgroup per expert.
__global__ __launch_bounds__(256) void route_scan_kernel(RouteArgs a) {
    __shared__ int part[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t* const row = a.counts + (int64_t)blockIdx.x * a.nb;
    int carry = 0;
    for (int b0 = 0; b0 < a.nb; b0 += 256) {
        const int b = b0 + threadIdx.x, n = b < a.nb ? row[b] : 0;
        int upto = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const int x = __shfl_up(upto, o); if (lane >= o) upto += x; }
        __syncthreads();
        if (lane == 63) part[wave] = upto;
        __syncthreads();
        int base = carry;
        for (int w = 0; w < wave; ++w) base += part[w];
        if (b < a.nb) row[b] = base + upto - n;
        carry += part[0] + part[1] + part[2] + part[3];
    }
    if (threadIdx.x == 0) a.totals[blockIdx.x] = carry;
}

__global__ __launch_bounds__(THREADS) void route_place_kernel(RouteArgs a) {
    __shared__ int before[WAVES * MAX_E], start[MAX_E + 1];
    const int t0 = blockIdx.x * TOKENS, n = min(TOKENS, a.T - t0) * a.k, c = threadIdx.x;
    const int64_t i = (int64_t)t0 * a.k + c;
    const int e = c < n ? a.expert[i] : -1;
    const int r = rank_in_group(e, a.E, before, nullptr);
    starts(a.totals, a.E, start);
    if (c < n) {
        const int s = e >= 0 ? start[e] + a.counts[(int64_t)e * a.nb + blockIdx.x] + r : -1;
        a.slot[i] = s;
        if (e >= 0) a.row_token[s] = t0 + c / a.k;
        if (i >= start[a.E]) a.row_token[i] = -1;
    }
    if (blockIdx.x == 0)
        for (int j = threadIdx.x; j <= a.E; j += THREADS) a.offsets[j] = start[j];
}

template <int DT, int V>
hero_status launch_route(const RouteArgs& a, hipStream_t st) {
    if (a.nb <= 1) {
        hipLaunchKernelGGL((route_choose_kernel<DT, V, true>), dim3(1), dim3(THREADS), 0, st, a);
        return hero_launch_status();
    }
    hipLaunchKernelGGL((route_choose_kernel<DT, V, false>), dim3((unsigned)a.nb), dim3(THREADS), 0, st, a);
    hipLaunchKernelGGL(route_scan_kernel, dim3((unsigned)a.E), dim3(256), 0, st, a);
    hipLaunchKernelGGL(route_place_kernel, dim3((unsigned)a.nb), dim3(THREADS), 0, st, a);
    return hero_launch_status();
}
template <int DT>
hero_status launch_route(const RouteArgs& a, hipStream_t st) {
    return a.E <= 64 ? launch_route<DT, 1>(a, st) : a.E <= 128 ? launch_route<DT, 2>(a, st) : a.E <= 256 ? launch_route<DT, 4>(a, st) : launch_route<DT, 8>(a, st);
}

struct CombineArgs {
    const uint16_t* y; int64_t ldy;
    const int32_t* slot; const float* weight;
    const uint16_t* residual; int64_t ldr;
    uint16_t* out; int64_t ldo;
    int T, k, R, chunks;                    // chunks of 8 values to a row
};

// A thread adds 8 values of one token.  Bound by HBM: the rows, the residual and the result once.
template <int DT, int K>
__global__ __launch_bounds__(256) void combine_kernel(CombineArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t t = i / a.chunks;
    if (t >= a.T) return;
    const int c = (int)(i - t * a.chunks) * 8, k = K ? K : a.k;
    const int32_t* const slot = a.slot + t * k;
    const float* const weight = a.weight + t * k;
    float sum[8];
#pragma unroll
    for (int v = 0; v < 8; ++v) sum[v] = 0.0f;
    auto add = [&](int s, float w) {
        if (s < 0 || s >= a.R) return;
        const v4i x = *reinterpret_cast<const v4i*>(a.y + (int64_t)s * a.ldy + c);
#pragma unroll
        for (int v = 0; v < 8; ++v) sum[v] = fmaf(w, hp_to_f32<DT>(((uint32_t)x[v >> 1] >> (16 * (v & 1))) & 0xffffu), sum[v]);
    };
    for (int j = 0; j < k; ++j) add(slot[j], weight[j]);
    if (a.residual) {
        const v4i x = *reinterpret_cast<const v4i*>(a.residual + t * a.ldr + c);
#pragma unroll
        for (int v = 0; v < 8; ++v) sum[v] += hp_to_f32<DT>(((uint32_t)x[v >> 1] >> (16 * (v & 1))) & 0xffffu);
    }
    v4i o;
#pragma unroll
    for (int v = 0; v < 4; ++v) o[v] = (int)pack2_hp<DT>(sum[2 * v], sum[2 * v + 1]);
    *reinterpret_cast<v4i*>(a.out + t * a.ldo + c) = o;
}

inline bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

}  // namespace

extern "C" size_t hero_moe_route_workspace_bytes(int64_t T, int64_t E, int64_t top_k) {
    if (T <= TOKENS || E < 1 || E > MAX_E || top_k < 1 || top_k > MAX_K || T > 0x7fffffffLL / top_k) return 0;
    const size_t nb = (size_t)((T + TOKENS - 1) / TOKENS);
    return ((nb + 1) * (size_t)E * 4 + 255) / 256 * 256;
}

extern "C" hero_status hero_moe_route(const void* logits, hero_dtype dt, int64_t ldl, int64_t T, int64_t E, int64_t top_k, int renorm,
                                      int32_t* expert, float* weight, int32_t* slot, int32_t* row_token, int32_t* offsets,
                                      void* workspace, size_t workspace_bytes, void* stream) {
    if (dt != HERO_F32 && dt != HERO_BF16 && dt != HERO_F16) return HERO_ERR_UNSUPPORTED;
    if (T < 0 || E < 1 || top_k < 1 || top_k > E || ldl < E) return HERO_ERR_SHAPE;
    if (E > MAX_E || top_k > MAX_K) return HERO_ERR_UNSUPPORTED;
    if (T > 0x7fffffffLL / top_k) return HERO_ERR_SHAPE;
    if (!offsets || (T > 0 && (!logits || !expert || !weight || !slot || !row_token))) return HERO_ERR_NULL;
    if (!aligned4(offsets) || !aligned4(expert) || !aligned4(weight) || !aligned4(slot) || !aligned4(row_token)) return HERO_ERR_ALIGN;
    if ((uintptr_t)logits & (dt == HERO_F32 ? 3 : 1)) return HERO_ERR_ALIGN;
    if (workspace && ((uintptr_t)workspace & 255)) return HERO_ERR_WORKSPACE;
    const size_t need = hero_moe_route_workspace_bytes(T, E, top_k);
    if (need && (!workspace || workspace_bytes < need)) return HERO_ERR_WORKSPACE;
    RouteArgs a;
    a.logits = logits; a.ldl = ldl; a.T = (int)T; a.E = (int)E; a.k = (int)top_k; a.renorm = renorm != 0;
    a.nb = (int)((T + TOKENS - 1) / TOKENS);
    a.expert = expert; a.weight = weight; a.slot = slot; a.row_token = row_token; a.offsets = offsets;
    a.counts = (int32_t*)workspace; a.totals = a.counts ? a.counts + (int64_t)a.nb * E : nullptr;
    if ((int64_t)a.nb * THREADS > 0xffffffffLL) return HERO_ERR_SHAPE;
    hipStream_t st = (hipStream_t)stream;
    return dt == HERO_F32 ? launch_route<HERO_F32>(a, st) : dt == HERO_BF16 ? launch_route<HERO_BF16>(a, st) : launch_route<HERO_F16>(a, st);
}

extern "C" hero_status hero_moe_combine(const void* y, int64_t ldy, int64_t R, const int32_t* slot, const float* weight,
                                        const void* residual, int64_t ldr, void* out, int64_t ldo,
                                        int64_t T, int64_t top_k, int64_t D, hero_dtype dt, void* stream) {
    if (dt != HERO_BF16 && dt != HERO_F16) return HERO_ERR_UNSUPPORTED;
    if (T < 0 || D < 0 || R < 0 || R > 0x7fffffffLL || T > 0x7fffffffLL || D > 0x7fffffffLL || top_k < 1) return HERO_ERR_SHAPE;
    if (top_k > MAX_K || D % 8 != 0) return HERO_ERR_UNSUPPORTED;
    if (ldy < D || ldo < D || (residual && ldr < D)) return HERO_ERR_SHAPE;
    if (T == 0 || D == 0) return HERO_OK;
    if (!slot || !weight || !out || (R > 0 && !y)) return HERO_ERR_NULL;
    if (ldy % 8 != 0 || ldo % 8 != 0 || (residual && ldr % 8 != 0)) return HERO_ERR_ALIGN;
    if (!hero_aligned16(y) || !hero_aligned16(out) || !hero_aligned16(residual) || !aligned4(slot) || !aligned4(weight)) return HERO_ERR_ALIGN;
    if (residual == out && ldr != ldo) return HERO_ERR_SHAPE;
    CombineArgs a;
    a.y = (const uint16_t*)y; a.ldy = ldy; a.slot = slot; a.weight = weight; a.residual = (const uint16_t*)residual; a.ldr = ldr;
    a.out = (uint16_t*)out; a.ldo = ldo; a.T = (int)T; a.k = (int)top_k; a.R = (int)R; a.chunks = (int)(D / 8);
    if (T > 0xffffff00LL / a.chunks) return HERO_ERR_SHAPE;
    const dim3 grid((unsigned)((T * a.chunks + 255) / 256)), block(256);
    hipStream_t st = (hipStream_t)stream;
    if (dt == HERO_BF16) hipLaunchKernelGGL((combine_kernel<HERO_BF16, 0>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((combine_kernel<HERO_F16, 0>), grid, block, 0, st, a);
    return hero_launch_status();
}
