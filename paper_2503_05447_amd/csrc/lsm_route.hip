// Routing of tokens to experts and the plan that sorts (token, expert) pairs by expert (include/lsm_train.h).
//   k_route       G lanes a token, eight of its logits in each: top_k rounds of the largest key, then the weights
//   k_route_bwd   the same lanes: softmax, the chosen experts' gradients, a row of d_logits
//   k_plan_count  pairs of each expert in each block's share
//   k_plan_place  every block adds up the shares before its own and places its pairs; a block that has all pairs counts them itself
// Bound: the large cases by latency, each kernel being a chain of a few loads, reductions over lanes and stores (32768 tokens, 64 bf16
// logits, 8 a token: 7.6 us for the routing, 2.9 and 8.6 for the plan, 10.2 for the gradient, where the bytes are 1 to 2 us each); a
// few tokens by the launches (four tokens: 3.8 and 2.8 us).  A token's logits stay in registers: eight in each of 8, 16 or 32 lanes, so
// that a round of the selection is seven comparisons and three to five exchanges between lanes.  The plan is a counting sort: each
// wave places 64 pairs at a time, their ranks among equal ones from ballots, so that the order needs no second pass.
#include "lsm_train_dev.h"

namespace lsm {
namespace {

constexpr float kLargest = 3.402823466e38f;

template <typename TIO> __device__ __forceinline__ float load1(const TIO* p);
template <> __device__ __forceinline__ float load1<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float load1<uint16_t>(const uint16_t* p) { return __uint_as_float(uint32_t(*p) << 16); }
template <typename TIO> __device__ __forceinline__ void store1(TIO* p, float x);
template <> __device__ __forceinline__ void store1<float>(float* p, float x) { *p = x; }
template <> __device__ __forceinline__ void store1<uint16_t>(uint16_t* p, float x) { *p = uint16_t(pack2(x, 0.f)); }

// The largest (smallest) over aligned groups of G lanes, in every lane.
template <int CTRL> __device__ __forceinline__ uint32_t dpp_u(uint32_t x) {
    return uint32_t(__builtin_amdgcn_mov_dpp(int(x), CTRL, 0xf, 0xf, true));
}
template <int G> __device__ __forceinline__ uint32_t group_max(uint32_t x) {
    x = max(x, dpp_u<0xB1>(x));
    x = max(x, dpp_u<0x4E>(x));
    x = max(x, dpp_u<0x141>(x));
    if (G >= 16) x = max(x, dpp_u<0x140>(x));
    if (G >= 32) x = max(x, uint32_t(__shfl_xor(int(x), 16, 64)));
    return x;
}

// Keys in the order of the numbers: 0 for what is never chosen (-inf, NaN), +inf as the largest finite number, -0 as 0.
__device__ __forceinline__ float as_logit(float x, float largest) {
    if (x != x) return -__builtin_inff();
    return fminf(x, largest) + 0.f;
}
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x);
    return x == -__builtin_inff() ? 0u : u >> 31 ? ~u : u | 0x80000000u;
}
template <typename TIO> constexpr float kMost = kLargest;
template <> constexpr float kMost<uint16_t> = 3.38953139e38f;  // bf16

constexpr int kHeld = 8;  // logits a lane

// Experts of a token: e = G r + lane, so that neighbouring lanes read neighbouring logits.
template <typename TIO, int G>
__global__ __launch_bounds__(256) void k_route(const TIO* logits, float* weights, int* chosen, int n, int E, int top_k, int renormalise) {
    const int g = threadIdx.x % G, t = (blockIdx.x * 256 + threadIdx.x) / G;
    if (t >= n) return;  // whole groups
    uint32_t key[kHeld];
    float x[kHeld];
    _Pragma("unroll") for (int r = 0; r < kHeld; ++r) {
        const int e = G * r + g;
        x[r] = e < E ? as_logit(load1(logits + size_t(t) * E + e), kMost<TIO>) : -__builtin_inff();
        key[r] = key_of(x[r]);
    }
    constexpr int SLOTS = kMostTop / G > 1 ? kMostTop / G : 1;
    int mine[SLOTS];
    float value[SLOTS], first = 0.f;
    _Pragma("unroll") for (int s = 0; s < SLOTS; ++s) { mine[s] = -1; value[s] = -__builtin_inff(); }
    for (int j = 0; j < top_k; ++j) {
        uint32_t most = key[0];
        _Pragma("unroll") for (int r = 1; r < kHeld; ++r) most = max(most, key[r]);
        most = group_max<G>(most);
        if (most == 0) break;  // the same in all lanes of the group
        uint32_t e = 0;  // of the equal ones that of the lowest index, as the largest of ~e
        _Pragma("unroll") for (int r = kHeld - 1; r >= 0; --r)
            if (key[r] == most) e = ~uint32_t(G * r + g);
        e = ~group_max<G>(e);
        _Pragma("unroll") for (int r = 0; r < kHeld; ++r)
            if (e == uint32_t(G * r + g)) key[r] = 0;
        const float v = __uint_as_float(most >> 31 ? most & 0x7fffffffu : ~most);
        if (j == 0) first = v;
        _Pragma("unroll") for (int s = 0; s < SLOTS; ++s)
            if (j == s * G + g) { mine[s] = int(e); value[s] = v; }
    }
    float sum = 0.f;
    if (renormalise) {
        _Pragma("unroll") for (int s = 0; s < SLOTS; ++s) sum += expf(value[s] - first);
    } else {
        _Pragma("unroll") for (int r = 0; r < kHeld; ++r) sum += expf(x[r] - first);
    }
    sum = group_sum<G>(sum);
    _Pragma("unroll") for (int s = 0; s < SLOTS; ++s) {
        const int j = s * G + g;
        if (j >= top_k) break;
        weights[size_t(t) * top_k + j] = mine[s] < 0 ? 0.f : expf(value[s] - first) / sum;
        chosen[size_t(t) * top_k + j] = mine[s];
    }
}

template <typename TIO, int G>
__global__ __launch_bounds__(256) void k_route_bwd(const TIO* logits, const int* chosen, const float* d_weights, TIO* d_logits, int n, int E,
                                                   int top_k, int renormalise) {
    const int g = threadIdx.x % G, t = (blockIdx.x * 256 + threadIdx.x) / G;
    if (t >= n) return;
    float x[kHeld], d[kHeld];
    bool in[kHeld];
    _Pragma("unroll") for (int r = 0; r < kHeld; ++r) {
        const int e = G * r + g;
        x[r] = e < E ? as_logit(load1(logits + size_t(t) * E + e), kMost<TIO>) : -__builtin_inff();
        d[r] = 0.f;
        in[r] = false;
    }
    for (int j = 0; j < top_k; ++j) {
        const int e = chosen[size_t(t) * top_k + j];
        const float dw = d_weights[size_t(t) * top_k + j];
        _Pragma("unroll") for (int r = 0; r < kHeld; ++r)
            if (e == G * r + g && e < E) { d[r] += dw; in[r] = true; }
    }
    uint32_t most = 0;
    _Pragma("unroll") for (int r = 0; r < kHeld; ++r)
        if (in[r] || !renormalise) most = max(most, key_of(x[r]));
    most = group_max<G>(most);
    const float top = most == 0 ? 0.f : __uint_as_float(most >> 31 ? most & 0x7fffffffu : ~most);
    float p[kHeld], sum = 0.f, along = 0.f;
    _Pragma("unroll") for (int r = 0; r < kHeld; ++r) {
        p[r] = in[r] || !renormalise ? expf(x[r] - top) : 0.f;
        sum += p[r];
    }
    sum = group_sum<G>(sum);
    const float scale = most == 0 ? 0.f : 1.f / sum;
    _Pragma("unroll") for (int r = 0; r < kHeld; ++r) {
        p[r] *= scale;
        if (!(p[r] > 0.f)) d[r] = 0.f;  // nothing through an expert of -inf
        along += p[r] * d[r];
    }
    along = group_sum<G>(along);
    _Pragma("unroll") for (int r = 0; r < kHeld; ++r) {
        const int e = G * r + g;
        if (e < E) store1(d_logits + size_t(t) * E + e, p[r] > 0.f ? p[r] * (d[r] - along) : 0.f);
    }
}

// ---- the plan ------------------------------------------------------------------------------------------------------
constexpr int kPlanThreads = 512, kPlanWaves = kPlanThreads / 64, kPlanAlone = 8192, kPlanBlocks = 256;

struct PlanArgs {
    const int32_t* id;
    int32_t *offsets, *order, *place, *hist;  // hist: [blocks][groups + 1], the last for what is left out
    int count, groups, limit, share;          // share: items of a block, a multiple of 64 kPlanWaves
};
// The groups of items i, i + step and so on below `end` (-1: no item), requested together (3000 pairs in one block: 18 -> 9 us, with the waves'
// shares even; 16 at a time: as fast, but three tokens 1.5 us slower for the longer code).
constexpr int kRead = 4;
__device__ __forceinline__ void groups_of(const PlanArgs& a, int i, int step, int end, int (&g)[kRead]) {
    _Pragma("unroll") for (int u = 0; u < kRead; ++u) g[u] = i + u * step < end ? a.id[i + u * step] : 0;
    _Pragma("unroll") for (int u = 0; u < kRead; ++u) {
        const int id = g[u];
        g[u] = i + u * step >= end ? -1 : id >= 0 && id < a.limit ? (a.groups == 1 ? 0 : id) : a.groups;
    }
}
// Counts groups g in n[], lane 0 among the lanes that are there.  With one group each wave adds its lanes up first: 64 additions to one address
// wait for one another (8191 tokens: 14.4 -> 12.3 us).
__device__ __forceinline__ void count_groups(int* n, const int (&g)[kRead], int groups) {
    _Pragma("unroll") for (int u = 0; u < kRead; ++u) {
        if (groups > 1) {
            if (g[u] >= 0) atomicAdd(&n[g[u]], 1);
            continue;
        }
        const int in = lanes(__ballot(g[u] == 0)), out = lanes(__ballot(g[u] == 1));
        if ((threadIdx.x & 63) == 0) {
            atomicAdd(&n[0], in);
            atomicAdd(&n[1], out);
        }
    }
}

__global__ __launch_bounds__(kPlanThreads) void k_plan_count(PlanArgs a) {
    __shared__ int n[kMostExperts + 1];
    for (int g = threadIdx.x; g <= a.groups; g += kPlanThreads) n[g] = 0;
    __syncthreads();
    const int i0 = int(blockIdx.x) * a.share, i1 = min(a.count, i0 + a.share);
    for (int i = i0 + int(threadIdx.x); i < i1; i += kRead * kPlanThreads) {
        int g[kRead];
        groups_of(a, i, kPlanThreads, i1, g);
        count_groups(n, g, a.groups);
    }
    __syncthreads();
    for (int g = threadIdx.x; g <= a.groups; g += kPlanThreads) a.hist[size_t(blockIdx.x) * (a.groups + 1) + g] = n[g];
}

// Items of one group keep their order: a wave's items are neighbours, its places follow those of the waves before it.
__global__ __launch_bounds__(kPlanThreads) void k_plan_place(PlanArgs a) {
    __shared__ int mine[kPlanWaves][kMostExperts + 1];  // items of each wave, then where they begin
    __shared__ int before[kMostExperts + 1], all[kMostExperts + 1], part[kPlanWaves];
    const int G = a.groups + 1, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int g = threadIdx.x; g < G; g += kPlanThreads) {
        before[g] = all[g] = 0;
        _Pragma("unroll") for (int w = 0; w < kPlanWaves; ++w) mine[w][g] = 0;
    }
    __syncthreads();
    const int i0 = int(blockIdx.x) * a.share, each = a.share / kPlanWaves, w0 = i0 + wave * each, w1 = min(a.count, w0 + each);
    for (int i = w0 + lane; i < w1; i += kRead * 64) {
        int g[kRead];
        groups_of(a, i, 64, w1, g);
        count_groups(mine[wave], g, a.groups);
    }
    if (gridDim.x > 1) {
        const int rows = kPlanThreads / G > 0 ? kPlanThreads / G : 1, g = int(threadIdx.x) % G, r0 = int(threadIdx.x) / G;
        int b = 0, s = 0;
        if (r0 < rows)
            for (int r = r0; r < int(gridDim.x); r += 8 * rows) {  // eight of them requested at a time
                int c[8];
                _Pragma("unroll") for (int u = 0; u < 8; ++u) c[u] = r + u * rows < int(gridDim.x) ? a.hist[size_t(r + u * rows) * G + g] : 0;
                _Pragma("unroll") for (int u = 0; u < 8; ++u) {
                    s += c[u];
                    if (r + u * rows < int(blockIdx.x)) b += c[u];
                }
            }
        if (r0 < rows) {
            atomicAdd(&before[g], b);
            atomicAdd(&all[g], s);
        }
        __syncthreads();
    } else {
        __syncthreads();
        for (int g = threadIdx.x; g < G; g += kPlanThreads) {
            int s = 0;
            _Pragma("unroll") for (int w = 0; w < kPlanWaves; ++w) s += mine[w][g];
            all[g] = s;
        }
        __syncthreads();
    }
    // where each group begins: a running sum over the groups, at most one a thread (257 groups at most)
    const int own = int(threadIdx.x) < G ? all[threadIdx.x] : 0;
    int upto = own;
    for (int off = 1; off < 64; off <<= 1) {
        const int t = __shfl_up(upto, off, 64);
        if (lane >= off) upto += t;
    }
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += part[w];
    if (int(threadIdx.x) < G) {
        const int g = threadIdx.x;
        int at = upto - own;
        if (blockIdx.x == 0) a.offsets[g] = at;
        at += before[g];
        _Pragma("unroll") for (int w = 0; w < kPlanWaves; ++w) {
            const int c = mine[w][g];
            mine[w][g] = at;
            at += c;
        }
    }
    __syncthreads();
    volatile int* next = mine[wave];
    for (int first = w0; first < w1; first += kRead * 64) {
        int groups[kRead];
        groups_of(a, first + lane, 64, w1, groups);
        _Pragma("unroll") for (int u = 0; u < kRead; ++u) {
            if (first + u * 64 >= w1) break;
            const int i = first + u * 64 + lane, g = groups[u];
            const bool there = g >= 0;
            unsigned long long same = __ballot(there);
            for (int b = 0; (a.groups >> b) != 0; ++b) {
                const unsigned long long set = __ballot((g >> b) & 1);
                same &= (g >> b) & 1 ? set : ~set;
            }
            if (there) {
                const int rank = lanes(same & ((1ull << lane) - 1)), at = next[g] + rank;
                const bool in = g < a.groups;
                a.order[at] = in ? i : -1;
                a.place[i] = in ? at : -1;
            }
            __builtin_amdgcn_wave_barrier();
            if (there && (same >> lane) == 1ull) next[g] = next[g] + lanes(same);  // the last of the equal ones
            __builtin_amdgcn_wave_barrier();
        }
    }
}

int check(const lsm_route_params* p, bool logits) {
    if (!p) return LSM_ERR_NULL;
    if (p->struct_size != sizeof(lsm_route_params)) return LSM_ERR_SHAPE;
    if (p->n < 1 || p->E < 1 || p->top_k < 1 || p->top_k > p->E) return LSM_ERR_SHAPE;
    if (p->E > kMostExperts || p->top_k > kMostTop) return LSM_ERR_UNSUPPORTED;
    if (int64_t(p->n) * p->top_k > kMostPairs) return LSM_ERR_SHAPE;
    if (!logits) return LSM_OK;
    if (p->dtype != LSM_DTYPE_F32 && p->dtype != LSM_DTYPE_BF16) return LSM_ERR_UNSUPPORTED;
    if (p->renormalise != 0 && p->renormalise != 1) return LSM_ERR_UNSUPPORTED;
    return LSM_OK;
}

int plan_share(int64_t count) {  // items of a block
    const int64_t each = count <= kPlanAlone ? count : (count + kPlanBlocks - 1) / kPlanBlocks, unit = 64 * kPlanWaves;
    return int((each + unit - 1) / unit * unit);
}

template <typename TIO, int G>
void launch_route(const lsm_route_params& p, const void* logits, float* weights, int32_t* chosen, hipStream_t st) {
    hipLaunchKernelGGL((k_route<TIO, G>), dim3(unsigned((int64_t(p.n) * G + 255) / 256)), dim3(256), 0, st, static_cast<const TIO*>(logits),
                       weights, chosen, p.n, p.E, p.top_k, p.renormalise);
}
template <typename TIO, int G>
void launch_route_bwd(const lsm_route_params& p, const void* logits, const int32_t* chosen, const float* dw, void* dl, hipStream_t st) {
    hipLaunchKernelGGL((k_route_bwd<TIO, G>), dim3(unsigned((int64_t(p.n) * G + 255) / 256)), dim3(256), 0, st,
                       static_cast<const TIO*>(logits), chosen, dw, static_cast<TIO*>(dl), p.n, p.E, p.top_k, p.renormalise);
}

}  // namespace

size_t plan_space(int64_t count, int groups) {
    if (count <= kPlanAlone) return 0;
    const int64_t share = plan_share(count), blocks = (count + share - 1) / share;
    return align256(size_t(blocks) * (groups + 1) * 4);
}
bool enqueue_plan(const int32_t* id, int64_t count, int groups, int limit, int32_t* offsets, int32_t* order, int32_t* place,
                  int32_t* hist, hipStream_t st) {
    const int share = plan_share(count), blocks = int((count + share - 1) / share);
    const PlanArgs a{id, offsets, order, place, hist, int(count), groups, limit, share};
    if (blocks > 1) {
        ProfScope ps(KID_PLAN, st);
        hipLaunchKernelGGL(k_plan_count, dim3(blocks), dim3(kPlanThreads), 0, st, a);
        if (!launched()) return false;
    }
    ProfScope ps(KID_PLAN, st);
    hipLaunchKernelGGL(k_plan_place, dim3(blocks), dim3(kPlanThreads), 0, st, a);
    return launched();
}

}  // namespace lsm

extern "C" {

int lsm_moe_route(const lsm_route_params* p, const void* logits, float* weights, int32_t* chosen, void* stream) {
    using namespace lsm;
    const int rc = check(p, true);
    if (rc != LSM_OK) return rc;
    if (!logits || !weights || !chosen) return LSM_ERR_NULL;
    if (misaligned(logits) || misaligned(weights) || misaligned(chosen)) return LSM_ERR_ALIGN;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    ProfScope ps(KID_ROUTE, st);
    if (p->dtype == LSM_DTYPE_BF16) {
        if (p->E <= 64) launch_route<uint16_t, 8>(*p, logits, weights, chosen, st);
        else if (p->E <= 128) launch_route<uint16_t, 16>(*p, logits, weights, chosen, st);
        else launch_route<uint16_t, 32>(*p, logits, weights, chosen, st);
    } else {
        if (p->E <= 64) launch_route<float, 8>(*p, logits, weights, chosen, st);
        else if (p->E <= 128) launch_route<float, 16>(*p, logits, weights, chosen, st);
        else launch_route<float, 32>(*p, logits, weights, chosen, st);
    }
    return launched() ? LSM_OK : LSM_ERR_LAUNCH;
}

int lsm_moe_route_bwd(const lsm_route_params* p, const void* logits, const int32_t* chosen, const float* d_weights,
                      void* d_logits, void* stream) {
    using namespace lsm;
    const int rc = check(p, true);
    if (rc != LSM_OK) return rc;
    if (!logits || !chosen || !d_weights || !d_logits) return LSM_ERR_NULL;
    if (misaligned(logits) || misaligned(chosen) || misaligned(d_weights) || misaligned(d_logits)) return LSM_ERR_ALIGN;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    ProfScope ps(KID_ROUTE, st);
    if (p->dtype == LSM_DTYPE_BF16) {
        if (p->E <= 64) launch_route_bwd<uint16_t, 8>(*p, logits, chosen, d_weights, d_logits, st);
        else if (p->E <= 128) launch_route_bwd<uint16_t, 16>(*p, logits, chosen, d_weights, d_logits, st);
        else launch_route_bwd<uint16_t, 32>(*p, logits, chosen, d_weights, d_logits, st);
    } else {
        if (p->E <= 64) launch_route_bwd<float, 8>(*p, logits, chosen, d_weights, d_logits, st);
        else if (p->E <= 128) launch_route_bwd<float, 16>(*p, logits, chosen, d_weights, d_logits, st);
        else launch_route_bwd<float, 32>(*p, logits, chosen, d_weights, d_logits, st);
    }
    return launched() ? LSM_OK : LSM_ERR_LAUNCH;
}

size_t lsm_moe_plan_workspace_bytes(const lsm_route_params* p) {
    using namespace lsm;
    return check(p, false) == LSM_OK ? plan_space(int64_t(p->n) * p->top_k, p->E) : 0;
}
int lsm_moe_plan(const lsm_route_params* p, const int32_t* chosen, int32_t* offsets, int32_t* order, int32_t* place,
                 void* workspace, size_t workspace_bytes, void* stream) {
    using namespace lsm;
    const int rc = check(p, false);
    if (rc != LSM_OK) return rc;
    if (!chosen || !offsets || !order || !place) return LSM_ERR_NULL;
    if (misaligned(chosen) || misaligned(offsets) || misaligned(order) || misaligned(place) || misaligned(workspace)) return LSM_ERR_ALIGN;
    const size_t need = lsm_moe_plan_workspace_bytes(p);
    if (need > 0 && (!workspace || workspace_bytes < need)) return LSM_ERR_WORKSPACE;
    return enqueue_plan(chosen, int64_t(p->n) * p->top_k, p->E, p->E, offsets, order, place, static_cast<int32_t*>(workspace),
                        static_cast<hipStream_t>(stream)) ? LSM_OK : LSM_ERR_LAUNCH;
}

}  // extern "C"
