// The router of a mixture-of-experts MLP (choice of experts, order of their rows) and the weighted sum behind the experts:
// hero_moe_route, hero_moe_combine.
#include "hero_common.h"
#include <float.h>
#include <type_traits>

namespace {

constexpr int MAX_E = 512, MAX_K = 16;
// Tokens of a workgroup, sixteen threads to each: for few tokens one workgroup of up to 64 of them, for many workgroups of 16
constexpr int ONE_TOKENS = 64, TOKENS = 16, MAX_WAVES = ONE_TOKENS / 4;
// Counts of 16 tokens fit a byte each.  While they are few, the workgroups that place the rows (64 tokens each) add up all of them themselves, each a stretch
// of every expert's; else a scan of 32-bit ones runs between.  (Sums of two experts share a word: less than 65536 tokens.)  us, with the scan / added:
// 256 tokens x 16 experts 9.9 / 8.2, 2048 x 256 12.0 / 10.4, 8192 x 64 11.4 / 9.6, 5001 x 160 (fp32) 12.4 / 11.6, 8192 x 128 12.2 / 11.3;  behind the limit 16384 x 128
// 14.9 / 14.7, 16384 x 256 18.0 / 20.3.
constexpr int64_t BYTES_TO_ADD = 1 << 16;
inline bool adds_itself(int64_t T, int64_t E) { return T <= 32768 && (T + TOKENS - 1) / TOKENS * ((E + 3) / 4 * 4) <= BYTES_TO_ADD; }

struct RouteArgs {
    const void* logits; int64_t ldl;
    int T, E, k, renorm, nb;                // nb workgroups
    int32_t* expert; float* weight; int32_t* slot; int32_t* row_token; int32_t* offsets;
    int32_t* counts;                        // [nb][E]: choices of each workgroup; behind the scan those of the workgroups before it.  Without: bytes [nb][E up to 4]
    int32_t* totals;                        // [E]
};

// reductions over rows of 16 lanes; every lane of a row gets the result
template <int CTRL> __device__ __forceinline__ int row_swap(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, true); }
template <typename T, typename F>
__device__ __forceinline__ T row_reduce(T x, F f) {
    auto step = [&](auto C) { x = f(x, __builtin_bit_cast(T, row_swap<decltype(C)::value>(__builtin_bit_cast(int, x)))); };
    step(std::integral_constant<int, 0xB1>{});                    // quad_perm [1,0,3,2]
    step(std::integral_constant<int, 0x4E>{});                    // quad_perm [2,3,0,1]
    step(std::integral_constant<int, 0x141>{});                   // row_half_mirror
    step(std::integral_constant<int, 0x140>{});                   // row_mirror
    return x;
}

// Sixteen lanes choose the experts of one token, a wave those of four: lane l holds the logits of experts 16 v + l.  top_k rounds of a maximum; ties
// go to the lowest index.  Bound by the instructions of the rounds: a logit of 16 bits shares a word with its index, so that the maximum is
// one of words, all different, 3 V instructions a round for V logits to a lane; 32 bits take 5 V (value, then index).  us, a wave to a token ->
// this: 16384 tokens x 256 bf16, 8 chosen 17.8 -> 8.2, 5001 x 160 f32, 6 chosen 15.0 -> 5.5.
template <int DT, int V>
__device__ __forceinline__ void choose(const RouteArgs& a, int t, int t_end, int lane, int32_t* chosen) {
    const int l16 = lane & 15;
    const bool real = t < t_end;
    const int64_t row = (int64_t)min(t, t_end - 1) * a.ldl + l16;
    auto max_of = [](auto x, auto y) { return x > y ? x : y; };
    auto sum_of = [](float x, float y) { return x + y; };
    float top = -INFINITY, all = 0.0f, mine = -INFINITY;          // lane j of the row keeps choice j
    int who = -1;
    if constexpr (DT != HERO_F32) {
        // w: the type's bits, turned so that they order as unsigned numbers (-0 as +0), above the index from above; 0: no expert (-infinity, NaN)
        constexpr uint32_t INF = DT == HERO_BF16 ? 0x7f80u : 0x7c00u;
        auto value = [](uint32_t b) { return fminf(hp_to_f32<DT>(b), FLT_MAX); };
        auto bits = [](uint32_t w) { const uint32_t b = w >> 16; return b & 0x8000u ? b & 0x7fffu : 0xffffu ^ b; };
        uint32_t w[V];
#pragma unroll
        for (int v = 0; v < V; ++v) w[v] = v * 16 + l16 < a.E ? ((const uint16_t*)a.logits)[row + v * 16] : INF | 0x8000u;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            uint32_t b = w[v] == 0x8000u ? 0u : w[v];
            const bool none = (b & 0x7fffu) > INF || b == (INF | 0x8000u);
            b = b & 0x8000u ? 0xffffu ^ b : b | 0x8000u;
            w[v] = none ? 0u : (b << 16) | (0xffffu - (uint32_t)(v * 16 + l16));
        }
        uint32_t m = 0;
        for (int j = 0; j < a.k; ++j) {
            uint32_t next = w[0];
#pragma unroll
            for (int v = 1; v < V; ++v) next = max(next, w[v]);
            m = row_reduce(next, max_of);
            if (j == 0) {
                top = m ? value(bits(m)) : 0.0f;
                if (!a.renorm) {
#pragma unroll
                    for (int v = 0; v < V; ++v) all += w[v] ? expf(value(bits(w[v])) - top) : 0.0f;
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) w[v] = w[v] == m ? 0u : w[v];
            if (l16 == j && m) { who = 0xffff - (int)(m & 0xffffu); mine = value(bits(m)); }
        }
    } else {
        float l[V];
#pragma unroll
        for (int v = 0; v < V; ++v) l[v] = v * 16 + l16 < a.E ? ((const float*)a.logits)[row + v * 16] : -INFINITY;
#pragma unroll
        for (int v = 0; v < V; ++v) l[v] = l[v] == l[v] ? fminf(l[v], FLT_MAX) : -INFINITY;
        for (int j = 0; j < a.k; ++j) {
            float m = l[0];
#pragma unroll
            for (int v = 1; v < V; ++v) m = fmaxf(m, l[v]);
            m = row_reduce(m, [](float x, float y) { return fmaxf(x, y); });
            if (j == 0) {
                top = m > -INFINITY ? m : 0.0f;
                if (!a.renorm) {
#pragma unroll
                    for (int v = 0; v < V; ++v) all += expf(l[v] - top);
                }
            }
            int at = V;
#pragma unroll
            for (int v = V - 1; v >= 0; --v) at = l[v] == m ? v : at;
            const int index = at * 16 + l16, first = row_reduce(index, [](int x, int y) { return min(x, y); });
            at = index == first ? at : V;
#pragma unroll
            for (int v = 0; v < V; ++v) l[v] = v == at ? -INFINITY : l[v];
            if (l16 == j && m > -INFINITY) { who = first; mine = m; }
        }
    }
    const float p = who >= 0 ? expf(mine - top) : 0.0f;
    const float total = row_reduce(a.renorm ? p : all, sum_of);
    if (real && l16 < a.k) {
        a.expert[(int64_t)t * a.k + l16] = who;
        a.weight[(int64_t)t * a.k + l16] = who >= 0 ? __fdiv_rn(p, total) : 0.0f;
        chosen[l16] = who;
    }
}

// Choice c of this workgroup, one to a thread: how many choices of the same expert come before it in its wave, and in the workgroup's
// earlier waves (`before` [waves][E]).  Equal experts of a wave are found bit by bit of their number.
__device__ __forceinline__ int rank_in_group(int e, int E, int* before, int* group_total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, threads = blockDim.x, waves = threads >> 6;
    for (int i = threadIdx.x; i < waves * E; i += threads) before[i] = 0;
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
    for (int i = threadIdx.x; i < E; i += threads) {
        int sum = 0;
        for (int w = 0; w < waves; ++w) { const int n = before[w * E + i]; before[w * E + i] = sum; sum += n; }
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

// ONE: the only workgroup of the call (of as many waves as it needs), which orders the rows as well; else a workgroup leaves behind how many of its
// choices fall to each expert (BYTES: in bytes).
template <int DT, int V, bool ONE, bool BYTES>
__global__ __launch_bounds__(ONE ? ONE_TOKENS * 16 : TOKENS * 16) void route_choose_kernel(RouteArgs a) {
    constexpr int NTOK = ONE ? ONE_TOKENS : TOKENS;
    __shared__ int32_t chosen[NTOK * MAX_K];
    __shared__ int before[ONE ? MAX_WAVES * MAX_E : MAX_E], total[ONE ? MAX_E : 1], start[ONE ? MAX_E + 1 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int t0 = blockIdx.x * NTOK, nt = min(NTOK, a.T - t0), t = wave * 4 + (lane >> 4);
    if (!ONE)
        for (int i = threadIdx.x; i < a.E; i += TOKENS * 16) before[i] = 0;
    if (wave * 4 < nt) choose<DT, V>(a, t0 + t, t0 + nt, lane, chosen + t * a.k);
    __syncthreads();
    const int c = threadIdx.x, e = c < nt * a.k ? chosen[c] : -1;
    if constexpr (ONE) {
        const int r = rank_in_group(e, a.E, before, total);
        starts(total, a.E, start);
        if (c < nt * a.k) a.slot[c] = e >= 0 ? start[e] + r : -1;
        if (e >= 0) a.row_token[start[e] + r] = c / a.k;
        if (c < nt * a.k && c >= start[a.E]) a.row_token[c] = -1;
        for (int i = threadIdx.x; i <= a.E; i += blockDim.x) a.offsets[i] = start[i];
    } else {
        if (e >= 0) atomicAdd(&before[e], 1);                       // (counts: their order does not show)
        __syncthreads();
        if constexpr (BYTES) {
            const int words = (a.E + 3) >> 2;
            for (int i = threadIdx.x; i < words; i += TOKENS * 16) {
                int x = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) x |= i * 4 + j < a.E ? before[i * 4 + j] << (8 * j) : 0;
                a.counts[blockIdx.x * words + i] = x;
            }
        } else
            for (int i = threadIdx.x; i < a.E; i += TOKENS * 16) a.counts[(int64_t)blockIdx.x * a.E + i] = before[i];
    }
}

// counts[b][e] -> choices of e in the workgroups before b; totals[e].  A workgroup for 16 experts: 64 threads to each, a stretch of the workgroups to
// every one of them.
__global__ __launch_bounds__(1024) void route_scan_kernel(RouteArgs a) {
    constexpr int ROWS = 16;                                            // of a stretch
    __shared__ int part[64][17], whole[16];
    const int col = threadIdx.x & 15, seg = threadIdx.x >> 4, e = blockIdx.x * 16 + col;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int carry = 0;                                                      // (of this thread's expert)
    for (int b0 = seg * ROWS; b0 - seg * ROWS < a.nb; b0 += 64 * ROWS) {
        int x[ROWS], sum = 0;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) x[i] = e < a.E && b0 + i < a.nb ? a.counts[(int64_t)(b0 + i) * a.E + e] : 0;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) { const int n = x[i]; x[i] = sum; sum += n; }
        part[seg][col] = sum;
        __syncthreads();
        const int n = part[lane][wave];                                 // wave w scans the 64 stretches of expert w
        int upto = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const int y = __shfl_up(upto, o); if (lane >= o) upto += y; }
        part[lane][wave] = upto - n;
        if (lane == 63) whole[wave] = upto;
        __syncthreads();
        const int at = carry + part[seg][col];
        carry += whole[col];
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
            if (e < a.E && b0 + i < a.nb) a.counts[(int64_t)(b0 + i) * a.E + e] = at + x[i];
        __syncthreads();
    }
    if (seg == 0 && e < a.E) a.totals[e] = carry;
}

// Rows of `NTOK` tokens.  BYTES: the counts of all workgroups are added here, a word of four experts and a stretch of the workgroups to a thread.
template <int NTOK, bool BYTES>
__global__ __launch_bounds__(NTOK * 16) void route_place_kernel(RouteArgs a) {
    __shared__ int before[NTOK / 4 * MAX_E], start[MAX_E + 1], total[BYTES ? MAX_E : 1], front[BYTES ? MAX_E : 1];
    const int t0 = blockIdx.x * NTOK, n = min(NTOK, a.T - t0) * a.k, c = threadIdx.x;
    const int64_t i = (int64_t)t0 * a.k + c;
    const int e = c < n ? a.expert[i] : -1;
    int earlier = 0;
    if constexpr (BYTES) {
        // (few words: a power of two of threads, so that those of the same word lie as far apart in every wave, which adds them up first)
        const int words = (a.E + 3) >> 2, across = words > 16 ? words : words <= 1 ? 1 : 1 << (32 - __clz(words - 1)), stretches = (NTOK * 16) / across;
        const int w = c % across, first = c / across, mine = blockIdx.x * (NTOK / TOKENS);
        for (int x = c; x < a.E; x += NTOK * 16) total[x] = front[x] = 0;
        __syncthreads();
        uint32_t sum[4] = {0, 0, 0, 0};                                 // experts 4 w, 4 w + 2 of all workgroups;  4 w + 1, 4 w + 3;  likewise of those in front
        constexpr int AT_ONCE = 8;
        for (int b0 = first < stretches ? first : a.nb; b0 < a.nb; b0 += AT_ONCE * stretches) {
            uint32_t x[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) x[i] = (uint32_t)a.counts[min(b0 + i * stretches, a.nb - 1) * words + min(w, words - 1)];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int b = b0 + i * stretches;
                const uint32_t y = b < a.nb ? x[i] : 0u, y0 = y & 0x00ff00ffu, y1 = (y >> 8) & 0x00ff00ffu;
                sum[0] += y0; sum[1] += y1;
                sum[2] += b < mine ? y0 : 0u; sum[3] += b < mine ? y1 : 0u;
            }
        }
        if (across <= 16)
            for (int o = across; o < 64; o <<= 1)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] += __shfl_xor(sum[j], o);
        if (across > 16 ? first < stretches : (c & 63) < across && w < words) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (w * 4 + j < a.E) {
                    atomicAdd(&total[w * 4 + j], (int)((sum[j & 1] >> (j & 2) * 8) & 0xffffu));
                    atomicAdd(&front[w * 4 + j], (int)((sum[2 + (j & 1)] >> (j & 2) * 8) & 0xffffu));
                }
        }
        __syncthreads();
        earlier = e >= 0 ? front[e] : 0;
    } else earlier = e >= 0 ? a.counts[(int64_t)blockIdx.x * a.E + e] : 0;
    const int r = rank_in_group(e, a.E, before, nullptr);
    starts(BYTES ? total : a.totals, a.E, start);
    if (c < n) {
        const int s = e >= 0 ? start[e] + earlier + r : -1;
        a.slot[i] = s;
        if (e >= 0) a.row_token[s] = t0 + c / a.k;
        if (i >= start[a.E]) a.row_token[i] = -1;
    }
    if (blockIdx.x == 0)
        for (int j = threadIdx.x; j <= a.E; j += NTOK * 16) a.offsets[j] = start[j];
}

template <int DT, int V>
hero_status launch_route(const RouteArgs& a, hipStream_t st) {
    if (a.T <= ONE_TOKENS) {
        const int waves = (a.T + 3) / 4;
        hipLaunchKernelGGL((route_choose_kernel<DT, V, true, false>), dim3(1), dim3(64 * (waves < 1 ? 1 : waves)), 0, st, a);
        return hero_launch_status();
    }
    if (adds_itself(a.T, a.E)) {
        hipLaunchKernelGGL((route_choose_kernel<DT, V, false, true>), dim3((unsigned)a.nb), dim3(TOKENS * 16), 0, st, a);
        hipLaunchKernelGGL((route_place_kernel<ONE_TOKENS, true>), dim3((unsigned)(a.T + ONE_TOKENS - 1) / ONE_TOKENS), dim3(ONE_TOKENS * 16), 0, st, a);
        return hero_launch_status();
    }
    hipLaunchKernelGGL((route_choose_kernel<DT, V, false, false>), dim3((unsigned)a.nb), dim3(TOKENS * 16), 0, st, a);
    hipLaunchKernelGGL(route_scan_kernel, dim3((unsigned)(a.E + 15) / 16), dim3(1024), 0, st, a);
    hipLaunchKernelGGL((route_place_kernel<TOKENS, false>), dim3((unsigned)a.nb), dim3(TOKENS * 16), 0, st, a);
    return hero_launch_status();
}
template <int DT>
hero_status launch_route(const RouteArgs& a, hipStream_t st) {
    const int v = (a.E + 15) / 16;
#define HERO_ROUTE(V) if (v <= V) return launch_route<DT, V>(a, st)
    HERO_ROUTE(1); HERO_ROUTE(2); HERO_ROUTE(4); HERO_ROUTE(8); HERO_ROUTE(12); HERO_ROUTE(16); HERO_ROUTE(24);
#undef HERO_ROUTE
    return launch_route<DT, 32>(a, st);
}

struct CombineArgs {
    const uint16_t* y; int64_t ldy;
    const int32_t* slot; const float* weight;
    const uint16_t* residual; int64_t ldr;
    uint16_t* out; int64_t ldo;
    int T, k, R, chunks;                    // chunks of 8 values to a row
};

// A thread adds 8 values of one token: the slots and weights of up to four choices, then their rows, then the sums, so that one wait covers the
// loads of each kind (a choice after the other: 32 tokens x 4 x 1024 4.7 us, 1 x 2 x 768 2.2).  Bound by HBM: the rows, the residual and the result
// once, 16384 tokens x 2 x 4096 in 99 us, 5.4 TB/s, a large copy's rate.
// y is in 16 bits, half the bytes of fp32 on both sides of this kernel, which is nothing but bytes: every row is rounded before the weighted sum and the sum
// after.  Root mean square error of a whole MLP (BF16) relative to its result, rows in fp32 / this: 32 tokens x 4 of 16 experts x 1024 x 4096 1.66e-3 / 1.84e-3,
// 4096 x 2 of 8 x 4096 x 16384 1.66e-3 / 1.95e-3 (1.66e-3 is the rounding of the result alone).
template <int DT, int K>
__global__ __launch_bounds__(256) void combine_kernel(CombineArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t t = i / a.chunks;
    if (t >= a.T) return;
    const int c = (int)(i - t * a.chunks) * 8;
    const int32_t* const slot = a.slot + t * a.k;
    const float* const weight = a.weight + t * a.k;
    auto value = [](const v4i& x, int v) { return hp_to_f32<DT>(((uint32_t)x[v >> 1] >> (16 * (v & 1))) & 0xffffu); };
    float sum[8];
#pragma unroll
    for (int v = 0; v < 8; ++v) sum[v] = 0.0f;
    v4i res = {0, 0, 0, 0};
    if (a.residual) res = *reinterpret_cast<const v4i*>(a.residual + t * a.ldr + c);
    for (int j0 = 0; j0 < a.k; j0 += K) {
        int s[K];
        float w[K];
        v4i x[K];
#pragma unroll
        for (int j = 0; j < K; ++j) {
            s[j] = j0 + j < a.k ? slot[j0 + j] : -1;
            w[j] = j0 + j < a.k ? weight[j0 + j] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < K; ++j)
            if ((uint32_t)s[j] < (uint32_t)a.R) x[j] = *reinterpret_cast<const v4i*>(a.y + (int64_t)s[j] * a.ldy + c);
#pragma unroll
        for (int j = 0; j < K; ++j)
            if ((uint32_t)s[j] < (uint32_t)a.R) {
#pragma unroll
                for (int v = 0; v < 8; ++v) sum[v] = fmaf(w[j], value(x[j], v), sum[v]);
            }
    }
    if (a.residual) {
#pragma unroll
        for (int v = 0; v < 8; ++v) sum[v] += value(res, v);
    }
    v4i o;
#pragma unroll
    for (int v = 0; v < 4; ++v) o[v] = (int)pack2_hp<DT>(sum[2 * v], sum[2 * v + 1]);
    *reinterpret_cast<v4i*>(a.out + t * a.ldo + c) = o;
}
template <int DT>
void launch_combine(const CombineArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)(((int64_t)a.T * a.chunks + 255) / 256)), block(256);
    if (a.k <= 1) hipLaunchKernelGGL((combine_kernel<DT, 1>), grid, block, 0, st, a);
    else if (a.k <= 2) hipLaunchKernelGGL((combine_kernel<DT, 2>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((combine_kernel<DT, 4>), grid, block, 0, st, a);
}

inline bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

}  // namespace

extern "C" size_t hero_moe_route_workspace_bytes(int64_t T, int64_t E, int64_t top_k) {
    if (T <= ONE_TOKENS || E < 1 || E > MAX_E || top_k < 1 || top_k > MAX_K || T > 0x7fffffffLL / top_k) return 0;
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
    if ((int64_t)a.nb * TOKENS * 16 > 0xffffffffLL) return HERO_ERR_SHAPE;
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
    hipStream_t st = (hipStream_t)stream;
    if (dt == HERO_BF16) launch_combine<HERO_BF16>(a, st);
    else launch_combine<HERO_F16>(a, st);
    return hero_launch_status();
}
