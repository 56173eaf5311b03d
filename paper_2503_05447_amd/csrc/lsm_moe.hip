// A mixture-of-experts layer for a few tokens (include/lsm_block.h), in four launches:
//   k_moe_router   a workgroup per 16 tokens: router outputs, softmax, the top_k experts of each token
//   k_moe_gate_up  a workgroup per active expert and 16 hidden features: h = w silu(Wg x) * (Wu x) for the expert's tokens
//   k_moe_down     a workgroup per active expert and 16 output features: Wd h, one row for each (token, expert) pair
//   k_moe_sum      y = residual + the sum of a token's rows, in the order of the experts
//
// Bound: the active experts' weights, read once from HBM: with a token or two an expert there are a few operations to a byte.
// A weight matrix is the first operand of 16 x 16 matrix products (its rows are the product's rows; a lane loads 16 bytes of
// a row straight into the operand's registers, no staging), the expert's tokens are the columns: up to 16 tokens cost what one
// does.  Four waves share the tile's rows by splitting the contraction and are summed through LDS in a fixed order.
#include "lsm_block_dev.h"

namespace lsm {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kMaxTokens = 128, kMaxExperts = 256, kMaxTop = 16;

// One step of a 16 x 16 product: both operands hold, in lane l, 16 bytes of row (column) l % 16 from element kPiece (l / 16) on.
__device__ __forceinline__ f32x4 product(const u32x4& a, const u32x4& b, f32x4 c, uint16_t) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 product(const u32x4& a, const u32x4& b, f32x4 c, float) {
    _Pragma("unroll") for (int i = 0; i < 4; ++i)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
    return c;
}
// The result's lane l holds column l % 16, rows 4 (l / 16) .. + 3.

struct MoeArgs {
    const void *x, *router, *w_gate_up, *w_down, *residual;
    void* y;
    int* chosen;      // [n][top_k] experts, rising
    float* weight;    // [n][top_k]
    void *h, *h_rem;  // [n top_k][F] hidden activations times the expert's weight (bf16: head and remainder)
    float* part;      // [n top_k][D]
    int n, D, F, E, top_k, renormalise;
    bool by_pair;     // fewer (token, expert) pairs than experts: the grid counts pairs
};

// 16 bytes of row `row` from element k on; 0 beyond the row's K elements
template <typename TIO>
__device__ __forceinline__ u32x4 operand(const TIO* m, size_t row, int K, int k) {
    if (k >= K) return u32x4{0, 0, 0, 0};
    return *reinterpret_cast<const u32x4*>(m + row * size_t(K) + k);
}

// Router of 16 tokens: 16 waves take the tiles of 16 experts, several waves a tile splitting the contraction where there are
// fewer tiles than waves.  Then a wave per token: softmax over the experts, four to a lane, and the top_k by the bits of the
// top_k-th largest output, found one by one by counting.  Experts of equal output go by index.
template <typename TIO>
__global__ __launch_bounds__(1024) void k_moe_router(MoeArgs a) {
    constexpr int E = kPiece<TIO>, STEP = 4 * E;
    __shared__ f32x4 part[16][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, t0 = int(blockIdx.x) * 16;
    const int tiles = (a.E + 15) / 16, split = 16 / tiles;
    {
        const int tile = wave / split, piece = wave % split;
        f32x4 c = {0.f, 0.f, 0.f, 0.f};
        if (tile < tiles) {
            const int steps = (a.D + STEP - 1) / STEP, per = (steps + split - 1) / split;
            const size_t er = min(tile * 16 + (lane & 15), a.E - 1), tr = min(t0 + (lane & 15), a.n - 1);
            const int k0 = E * (lane >> 4);
            constexpr int U = 4;
            for (int s = piece * per; s < min(steps, (piece + 1) * per); s += U) {
                u32x4 wr[U], xr[U];
                const int last = min(steps, (piece + 1) * per);
                _Pragma("unroll") for (int u = 0; u < U; ++u) {
                    const int k = s + u < last ? (s + u) * STEP + k0 : a.D;
                    wr[u] = operand(static_cast<const TIO*>(a.router), er, a.D, k);
                    xr[u] = operand(static_cast<const TIO*>(a.x), tr, a.D, k);
                }
                _Pragma("unroll") for (int u = 0; u < U; ++u) c = product(wr[u], xr[u], c, TIO());
            }
        }
        part[wave][lane] = c;
    }
    __syncthreads();
    const int t = t0 + wave;
    if (t >= a.n) return;
    constexpr int R = kMaxExperts / 64;
    float out[R], p[R];
    uint32_t key[R];
    float m = -__builtin_inff();
    _Pragma("unroll") for (int r = 0; r < R; ++r) {
        const int e = 64 * r + lane;
        out[r] = -__builtin_inff();
        key[r] = 0;
        if (e < a.E) {
            float s = 0.f;
            for (int i = 0; i < split; ++i) s += part[(e / 16) * split + i][16 * ((e % 16) / 4) + wave][e % 4];
            out[r] = s;
            const uint32_t u = __float_as_uint(s + 0.f);
            key[r] = s == s ? u ^ (uint32_t(int(u) >> 31) | 0x80000000u) : 1u;  // not a number: after all numbers
            m = fmaxf(m, s);
        }
    }
    _Pragma("unroll") for (int off = 1; off < 64; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    float all = 0.f;
    _Pragma("unroll") for (int r = 0; r < R; ++r) {
        p[r] = 64 * r + lane < a.E ? expf(out[r] - m) : 0.f;
        all += p[r];
    }
    all = group_sum<64>(all);
    uint32_t bound = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t trial = bound | (1u << bit);
        int c = 0;
        _Pragma("unroll") for (int r = 0; r < R; ++r) c += lanes(__ballot(key[r] >= trial));
        if (c >= a.top_k) bound = trial;
    }
    int left = a.top_k;  // places for experts at the bound
    _Pragma("unroll") for (int r = 0; r < R; ++r) left -= lanes(__ballot(key[r] > bound));
    const unsigned long long below = (1ull << lane) - 1;
    bool in[R];
    float sum = 0.f;
    _Pragma("unroll") for (int r = 0; r < R; ++r) {
        const unsigned long long at = __ballot(key[r] == bound);
        in[r] = key[r] > bound || (key[r] == bound && lanes(at & below) < left);
        left = max(0, left - lanes(at));
        sum += in[r] ? p[r] : 0.f;
    }
    sum = group_sum<64>(sum);
    const float over = all == all ? (a.renormalise ? sum : all) : all;
    int place = t * a.top_k;
    _Pragma("unroll") for (int r = 0; r < R; ++r) {
        const unsigned long long who = __ballot(in[r]);
        if (in[r]) {
            const int i = place + lanes(who & below);
            a.chosen[i] = 64 * r + lane;
            a.weight[i] = p[r] / over;
        }
        place += lanes(who);
    }
}

// The pairs (token * top_k + place) of this workgroup's expert in the order of the tokens; -1: nothing to do for it.
__device__ __forceinline__ int expert_pairs(const MoeArgs& a, int y, int* pairs, int* counts, int* expert) {
    constexpr int M = kMaxTokens * kMaxTop / 256;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, total = a.n * a.top_k;
    const int e = a.by_pair ? a.chosen[y] : y;
    unsigned long long who[M];
    _Pragma("unroll") for (int i = 0; i < M; ++i) {
        const int at = i * 256 + tid;
        who[i] = __ballot(i * 256 < total && at < total && a.chosen[at < total ? at : 0] == e);
        if (lane == 0) counts[i * 4 + wave] = lanes(who[i]);
    }
    __syncthreads();
    int n = 0;
    _Pragma("unroll") for (int i = 0; i < M; ++i)
        _Pragma("unroll") for (int w = 0; w < 4; ++w) {
            if (w == wave && (who[i] >> lane & 1)) pairs[n + lanes(who[i] & ((1ull << lane) - 1))] = i * 256 + tid;
            n += counts[i * 4 + w];
        }
    __syncthreads();
    *expert = e;
    if (n == 0 || (a.by_pair && pairs[0] != y)) return -1;
    return n;
}

constexpr int kSteps = 4;  // steps of the contraction requested at a time

// NG: groups of 16 tokens that an expert may have
template <typename TIO, int NG>
__global__ __launch_bounds__(256) void k_moe_gate_up(MoeArgs a) {
    constexpr int E = kPiece<TIO>, STEP = 4 * E;
    __shared__ int pairs[kMaxTokens], counts[kMaxTokens * kMaxTop / 64];
    __shared__ f32x4 part[4][2 * NG][64];
    int e;
    const int m = expert_pairs(a, blockIdx.y, pairs, counts, &e);
    if (m < 0) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, groups = (m + 15) / 16;
    const int f0 = int(blockIdx.x) * 16;
    const size_t row = size_t(e) * 2 * a.F + min(f0 + (lane & 15), a.F - 1);
    const TIO* w = static_cast<const TIO*>(a.w_gate_up);
    const TIO* x = static_cast<const TIO*>(a.x);
    size_t token[NG];
    _Pragma("unroll") for (int g = 0; g < NG; ++g) token[g] = pairs[min(g * 16 + (lane & 15), m - 1)] / a.top_k;
    f32x4 c[2][NG];
    _Pragma("unroll") for (int g = 0; g < NG; ++g) c[0][g] = c[1][g] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int steps = (a.D + STEP - 1) / STEP, per = (steps + 3) / 4, last = min(steps, (wave + 1) * per);
    for (int s = wave * per; s < last; s += kSteps) {
        u32x4 wr[2][kSteps];
        int k[kSteps];
        _Pragma("unroll") for (int u = 0; u < kSteps; ++u) {
            k[u] = s + u < last ? (s + u) * STEP + E * (lane >> 4) : a.D;
            wr[0][u] = operand(w, row, a.D, k[u]);
            wr[1][u] = operand(w, row + a.F, a.D, k[u]);
        }
        _Pragma("unroll") for (int g = 0; g < NG; ++g) {
            if (g >= groups) break;
            u32x4 xr[kSteps];
            _Pragma("unroll") for (int u = 0; u < kSteps; ++u) xr[u] = operand(x, token[g], a.D, k[u]);
            _Pragma("unroll") for (int u = 0; u < kSteps; ++u) {
                c[0][g] = product(wr[0][u], xr[u], c[0][g], TIO());
                c[1][g] = product(wr[1][u], xr[u], c[1][g], TIO());
            }
        }
    }
    _Pragma("unroll") for (int g = 0; g < NG; ++g) {
        part[wave][2 * g][lane] = c[0][g];
        part[wave][2 * g + 1][lane] = c[1][g];
    }
    __syncthreads();
    const int f = f0 + 4 * (lane >> 4);  // F is a multiple of 8: the four features of a lane are all there or none
    for (int g = wave; g < groups; g += 4) {
        const int i = g * 16 + (lane & 15);
        if (i >= m || f >= a.F) continue;
        f32x4 s[2];
        _Pragma("unroll") for (int n = 0; n < 2; ++n)
            s[n] = (part[0][2 * g + n][lane] + part[1][2 * g + n][lane]) + (part[2][2 * g + n][lane] + part[3][2 * g + n][lane]);
        const int pair = pairs[i];
        const float p = a.weight[pair];
        float h[4];
        _Pragma("unroll") for (int j = 0; j < 4; ++j) h[j] = p * (s[0][j] / (1.f + expf(-s[0][j])) * s[1][j]);
        const size_t at = size_t(pair) * a.F + f;
        if (sizeof(TIO) == 4) {
            *reinterpret_cast<f32x4*>(static_cast<float*>(a.h) + at) = f32x4{h[0], h[1], h[2], h[3]};
        } else {
            const u32x2 hi = {pack2(h[0], h[1]), pack2(h[2], h[3])};
            *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.h) + at) = hi;
            *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.h_rem) + at) =
                u32x2{pack2(h[0] - bf16_lo(hi.x), h[1] - bf16_hi(hi.x)), pack2(h[2] - bf16_lo(hi.y), h[3] - bf16_hi(hi.y))};
        }
    }
}

template <typename TIO, int NG>
__global__ __launch_bounds__(256) void k_moe_down(MoeArgs a) {
    constexpr int E = kPiece<TIO>, STEP = 4 * E;
    constexpr bool REM = sizeof(TIO) == 2;
    __shared__ int pairs[kMaxTokens], counts[kMaxTokens * kMaxTop / 64];
    __shared__ f32x4 part[4][NG][64];
    int e;
    const int m = expert_pairs(a, blockIdx.y, pairs, counts, &e);
    if (m < 0) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, groups = (m + 15) / 16;
    const int d0 = int(blockIdx.x) * 16;
    const size_t row = size_t(e) * a.D + min(d0 + (lane & 15), a.D - 1);
    const TIO* w = static_cast<const TIO*>(a.w_down);
    size_t pair[NG];
    _Pragma("unroll") for (int g = 0; g < NG; ++g) pair[g] = pairs[min(g * 16 + (lane & 15), m - 1)];
    f32x4 c[NG];
    _Pragma("unroll") for (int g = 0; g < NG; ++g) c[g] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int steps = (a.F + STEP - 1) / STEP, per = (steps + 3) / 4, last = min(steps, (wave + 1) * per);
    for (int s = wave * per; s < last; s += kSteps) {
        u32x4 wr[kSteps];
        int k[kSteps];
        _Pragma("unroll") for (int u = 0; u < kSteps; ++u) {
            k[u] = s + u < last ? (s + u) * STEP + E * (lane >> 4) : a.F;
            wr[u] = operand(w, row, a.F, k[u]);
        }
        _Pragma("unroll") for (int g = 0; g < NG; ++g) {
            if (g >= groups) break;
            u32x4 hr[kSteps], rr[kSteps];
            _Pragma("unroll") for (int u = 0; u < kSteps; ++u) {
                hr[u] = operand(static_cast<const TIO*>(a.h), pair[g], a.F, k[u]);
                if (REM) rr[u] = operand(static_cast<const TIO*>(a.h_rem), pair[g], a.F, k[u]);
            }
            _Pragma("unroll") for (int u = 0; u < kSteps; ++u) {
                c[g] = product(wr[u], hr[u], c[g], TIO());
                if (REM) c[g] = product(wr[u], rr[u], c[g], TIO());
            }
        }
    }
    _Pragma("unroll") for (int g = 0; g < NG; ++g) part[wave][g][lane] = c[g];
    __syncthreads();
    const int d = d0 + 4 * (lane >> 4);
    for (int g = wave; g < groups; g += 4) {
        const int i = g * 16 + (lane & 15);
        if (i >= m || d >= a.D) continue;
        *reinterpret_cast<f32x4*>(a.part + size_t(pairs[i]) * a.D + d) =
            (part[0][g][lane] + part[1][g][lane]) + (part[2][g][lane] + part[3][g][lane]);
    }
}

template <typename TIO>
__device__ __forceinline__ f32x4 load4(const TIO* p) {
    if (sizeof(TIO) == 4) return *reinterpret_cast<const f32x4*>(p);
    const u32x2 v = *reinterpret_cast<const u32x2*>(p);
    return f32x4{bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)};
}
template <typename TIO>
__global__ __launch_bounds__(256) void k_moe_sum(MoeArgs a) {
    const size_t i = (size_t(blockIdx.x) * 256 + threadIdx.x) * 4;
    if (i >= size_t(a.n) * a.D) return;
    const int t = int(i / a.D), d = int(i - size_t(t) * a.D);
    f32x4 s = a.residual ? load4(static_cast<const TIO*>(a.residual) + i) : f32x4{0.f, 0.f, 0.f, 0.f};
    const float* p = a.part + size_t(t) * a.top_k * a.D + d;
    for (int j = 0; j < a.top_k; ++j) s += *reinterpret_cast<const f32x4*>(p + size_t(j) * a.D);
    if (sizeof(TIO) == 4) *reinterpret_cast<f32x4*>(static_cast<float*>(a.y) + i) = s;
    else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.y) + i) = u32x2{pack2(s[0], s[1]), pack2(s[2], s[3])};
}

// ---- host ------------------------------------------------------------------------------------------------------------
int check(const lsm_moe_params* p) {
    if (!p) return LSM_ERR_NULL;
    if (p->struct_size != sizeof(lsm_moe_params)) return LSM_ERR_SHAPE;
    if (p->n < 1 || p->D < 1 || p->F < 1 || p->E < 1 || p->top_k < 1 || p->top_k > p->E) return LSM_ERR_SHAPE;
    if (p->dtype != LSM_DTYPE_F32 && p->dtype != LSM_DTYPE_BF16) return LSM_ERR_UNSUPPORTED;
    if (p->n > kMaxTokens || p->E > kMaxExperts || p->top_k > kMaxTop || p->D % 8 || p->F % 8 || p->D > 65536 || p->F > 65536)
        return LSM_ERR_UNSUPPORTED;
    if (p->renormalise != 0 && p->renormalise != 1) return LSM_ERR_UNSUPPORTED;
    return LSM_OK;
}
struct MoeSpace { size_t chosen, weight, h, h_rem, part, bytes; };
MoeSpace space(const lsm_moe_params& p) {
    const size_t pairs = size_t(p.n) * p.top_k, el = p.dtype == LSM_DTYPE_BF16 ? 2 : 4;
    MoeSpace s{};
    s.chosen = 0;
    s.weight = align256(pairs * 4);
    s.h = s.weight + align256(pairs * 4);
    s.h_rem = s.h + align256(pairs * p.F * el);
    s.part = s.h_rem + (el == 2 ? align256(pairs * p.F * el) : 0);
    s.bytes = s.part + align256(pairs * p.D * 4);
    return s;
}
template <typename TIO, int NG>
void launch_experts(const MoeArgs& a, hipStream_t st) {
    const int y = a.by_pair ? a.n * a.top_k : a.E;
    {
        ProfScope ps(KID_MOE_GATE_UP, st);
        hipLaunchKernelGGL((k_moe_gate_up<TIO, NG>), dim3((a.F + 15) / 16, y), dim3(256), 0, st, a);
    }
    ProfScope ps(KID_MOE_DOWN, st);
    hipLaunchKernelGGL((k_moe_down<TIO, NG>), dim3((a.D + 15) / 16, y), dim3(256), 0, st, a);
}
template <typename TIO>
void launch(const MoeArgs& a, hipStream_t st) {
    {
        ProfScope ps(KID_MOE_ROUTER, st);
        hipLaunchKernelGGL((k_moe_router<TIO>), dim3((a.n + 15) / 16), dim3(1024), 0, st, a);
    }
    if (a.n <= 16) launch_experts<TIO, 1>(a, st);
    else if (a.n <= 32) launch_experts<TIO, 2>(a, st);
    else if (a.n <= 64) launch_experts<TIO, 4>(a, st);
    else launch_experts<TIO, 8>(a, st);
    ProfScope ps(KID_MOE_SUM, st);
    hipLaunchKernelGGL((k_moe_sum<TIO>), dim3(unsigned((size_t(a.n) * a.D / 4 + 255) / 256)), dim3(256), 0, st, a);
}

}  // namespace
}  // namespace lsm

extern "C" {

size_t lsm_moe_step_workspace_bytes(const lsm_moe_params* p) {
    using namespace lsm;
    return check(p) == LSM_OK ? space(*p).bytes : 0;
}

int lsm_moe_step(const lsm_moe_params* p, const void* x, const void* router, const void* w_gate_up, const void* w_down,
                 const void* residual, void* y, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace lsm;
    const int rc = check(p);
    if (rc != LSM_OK) return rc;
    if (!x || !router || !w_gate_up || !w_down || !y) return LSM_ERR_NULL;
    if (misaligned(x) || misaligned(router) || misaligned(w_gate_up) || misaligned(w_down) || misaligned(residual) || misaligned(y) ||
        misaligned(workspace))
        return LSM_ERR_ALIGN;
    const MoeSpace s = space(*p);
    if (!workspace || workspace_bytes < s.bytes) return LSM_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    const MoeArgs a{x, router, w_gate_up, w_down, residual, y, reinterpret_cast<int*>(ws + s.chosen),
                    reinterpret_cast<float*>(ws + s.weight), ws + s.h, ws + s.h_rem, reinterpret_cast<float*>(ws + s.part),
                    p->n, p->D, p->F, p->E, p->top_k, p->renormalise, p->n * p->top_k < p->E};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (p->dtype == LSM_DTYPE_BF16) launch<uint16_t>(a, st);
    else launch<float>(a, st);
    return hipGetLastError() == hipSuccess ? LSM_OK : LSM_ERR_LAUNCH;
}

}  // extern "C"
