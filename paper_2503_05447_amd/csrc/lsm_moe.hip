// A mixture-of-experts layer for a few tokens (include/lsm_block.h), in five launches:
//   k_moe_router   a workgroup per expert and 16 tokens: router outputs
//   k_moe_route    a wave per token: softmax, the top_k experts, their weights; a bit per token in each expert's mask (for up to
//                  four tokens the next kernel's workgroups do this themselves)
//   k_moe_gate_up  a workgroup per active expert and tile of hidden features: h = w silu(Wg x) * (Wu x) for the expert's tokens
//   k_moe_down     a workgroup per active expert and tile of output features: Wd h, one row for each (token, expert) pair
//   k_moe_sum      y = residual + the sum of a token's rows, in the order of the experts
//
// Bound: the active experts' weights, read once from HBM: with a token or two an expert there are a few operations to a byte.
// A weight matrix is the first operand of 16 x 16 matrix products (its rows are the product's rows; a lane loads 16 bytes of
// a row straight into the operand's registers, no staging), the expert's tokens are the columns: up to 16 tokens cost what one
// does.  What is requested for a step is used a step later, so that a wave always has a request under way.
//
// Measured, bf16: 128 tokens, 64 experts of 1536 x 2048, 6 a token: k_moe_gate_up 148 us (5.4 TB/s), k_moe_down 91 (4.4: it reads
// its columns, head and remainder, beside the weights), the other three 17; 16 tokens, 64 of 1032 x 2048, 8 a token: 86 and 54; one
// token, 64 of 1024 x 1024: 10.4 and 6.2, 3.6 and 3.8 for the other two.  A read-only stream reaches 6.1 TB/s here.
//
// Not kept: the sum by the last workgroup of a tile (the fences across the dies cost more than they save: 128 tokens 250 -> 650 us);
// all experts' rows of 16 outputs by one workgroup (one token: 64 workgroups, 5 us more than both kernels); an expert's tiles on
// one die (16 tokens 4 % slower, 128 tokens the same); weights loaded past the caches (8 % slower); eight waves a workgroup.
#include "lsm_block_dev.h"

namespace lsm {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

typedef unsigned long long u64;

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
    float* logits;    // [n][E]
    int* chosen;      // [n][top_k] experts, rising
    f32x2* place;     // [n][E], where chosen: the weight, and (as an int) the place in `chosen`
    u64* mask;        // [E][2] the tokens of each expert
    void *h, *h_rem;  // [n top_k][F] hidden activations times the expert's weight (bf16: head and remainder)
    float* part;      // [n top_k][D]
    int n, D, F, E, top_k, renormalise;
    bool by_pair;     // fewer (token, expert) pairs than experts: the grid counts pairs
};

// Router outputs of 16 tokens for one expert, four tokens a wave: lanes along the row, 16 bytes each, four pieces of the expert's row
// and of every token's requested at a time.  (As 16 x 16 products by one workgroup for all experts: 22 us at a hidden size of
// 2048, where the rows are 4 KiB apart and meet in one channel.)
template <typename TIO>
__global__ __launch_bounds__(256) void k_moe_router(MoeArgs a) {
    constexpr int E = kPiece<TIO>, U = 4;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, e = blockIdx.x, t0 = int(blockIdx.y) * 16 + wave;
    if (blockIdx.y == 0 && threadIdx.x < 2) a.mask[2 * e + threadIdx.x] = 0;  // filled by the next kernel
    if (t0 >= a.n) return;
    const TIO* w = static_cast<const TIO*>(a.router) + size_t(e) * a.D;
    const TIO* x[4];
    float sum[4];
    _Pragma("unroll") for (int i = 0; i < 4; ++i) {
        x[i] = static_cast<const TIO*>(a.x) + size_t(min(t0 + 4 * i, a.n - 1)) * a.D;
        sum[i] = 0.f;
    }
    for (int k0 = lane * E; k0 < a.D; k0 += U * 64 * E) {
        u32x4 wr[U], xr[4][U];
        _Pragma("unroll") for (int u = 0; u < U; ++u) {
            const int k = min(k0 + u * 64 * E, a.D - E);
            wr[u] = *reinterpret_cast<const u32x4*>(w + k);
            _Pragma("unroll") for (int i = 0; i < 4; ++i) xr[i][u] = *reinterpret_cast<const u32x4*>(x[i] + k);
        }
        _Pragma("unroll") for (int u = 0; u < U; ++u) {
            if (k0 + u * 64 * E >= a.D) break;
            float wf[E];
            unpack(wr[u], wf);
            _Pragma("unroll") for (int i = 0; i < 4; ++i) {
                float xf[E];
                unpack(xr[i][u], xf);
                _Pragma("unroll") for (int c = 0; c < E; ++c) sum[i] += wf[c] * xf[c];
            }
        }
    }
    _Pragma("unroll") for (int i = 0; i < 4; ++i) {
        sum[i] = group_sum<64>(sum[i]);
        if (lane == 0 && t0 + 4 * i < a.n) a.logits[size_t(t0 + 4 * i) * a.E + e] = sum[i];
    }
}

// The experts of token t, by a wave: softmax over the experts, R to a lane, and the top_k by the bits of the top_k-th largest
// output, found one by one by counting.  Experts of equal output go by index.  emit(place, expert, weight), places rising with
// the experts.
template <int R, typename Emit>
__device__ __forceinline__ void route(const MoeArgs& a, int t, int lane, Emit emit) {
    float out[R], p[R];
    uint32_t key[R];
    float m = -__builtin_inff();
    _Pragma("unroll") for (int r = 0; r < R; ++r) {
        const int e = 64 * r + lane;
        out[r] = -__builtin_inff();
        key[r] = 0;
        if (e < a.E) {
            const float s = a.logits[size_t(t) * a.E + e];
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
    int place = 0;
    _Pragma("unroll") for (int r = 0; r < R; ++r) {
        const unsigned long long who = __ballot(in[r]);
        if (in[r]) emit(place + lanes(who & below), 64 * r + lane, p[r] / over);
        place += lanes(who);
    }
}
constexpr int kWide = kMaxExperts / 64;

template <int R>
__global__ __launch_bounds__(256) void k_moe_route(MoeArgs a) {
    const int lane = threadIdx.x & 63, t = int(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (t >= a.n) return;
    route<R>(a, t, lane, [&](int i, int e, float w) {
        a.chosen[t * a.top_k + i] = e;
        a.place[size_t(t) * a.E + e] = f32x2{w, __int_as_float(t * a.top_k + i)};
        atomicOr(a.mask + 2 * e + (t >> 6), u64(1) << (t & 63));  // bits: the order of the tokens does not matter
    });
}

// The tokens of this workgroup's expert.
struct Tokens {
    u64 low, high;
    int e, m;  // expert and how many; 0: nothing to do here
    // For up to four tokens, which every workgroup of the first product routes for itself (a wave per token; a launch less): low is
    // the set of the expert's pairs.  The first workgroup leaves what the next kernel needs.
    __device__ __forceinline__ Tokens(const MoeArgs& a, int* chosen, float* weight) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, pairs = a.n * a.top_k;
        auto emit = [&](int i, int e_, float w) {
            chosen[wave * a.top_k + i] = e_;
            weight[wave * a.top_k + i] = w;
        };
        if (wave < a.n) a.E <= 64 ? route<1>(a, wave, lane, emit) : route<kWide>(a, wave, lane, emit);
        __syncthreads();
        const int mine = lane < pairs ? chosen[lane] : -1;
        if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < pairs) {
            u64 mask = 0;
            for (int i = 0; i < pairs; ++i) mask |= u64(chosen[i] == mine ? 1 : 0) << (i / a.top_k);
            a.chosen[lane] = mine;
            a.place[size_t(lane / a.top_k) * a.E + mine] = f32x2{weight[lane], __int_as_float(lane)};
            a.mask[2 * mine] = mask;
            a.mask[2 * mine + 1] = 0;
        }
        const int y = blockIdx.y;
        e = __builtin_amdgcn_readfirstlane(chosen[a.by_pair ? y : 0]);
        if (!a.by_pair) e = y;
        low = __ballot(mine == e);
        high = 0;
        m = lanes(low);
        if (a.by_pair && __builtin_ctzll(low) != y) m = 0;  // an earlier pair has the expert
    }
    __device__ __forceinline__ explicit Tokens(const MoeArgs& a) {
        const int y = blockIdx.y;
        e = a.by_pair ? a.chosen[y] : y;
        low = a.mask[2 * e];
        high = a.mask[2 * e + 1];
        m = lanes(low) + lanes(high);
        if (a.by_pair && m > 0 && (low ? __builtin_ctzll(low) : 64 + __builtin_ctzll(high)) != y / a.top_k) m = 0;  // an earlier pair has it
    }
    // the i-th of them, i < m: the position of a bit by halves
    __device__ __forceinline__ int at(int i) const {
        int n = lanes(low), t = 0;
        u64 w = low;
        if (i >= n) { i -= n; w = high; t = 64; }
        n = lanes(w & 0xffffffffu);
        uint32_t v = uint32_t(w);
        if (i >= n) { i -= n; v = uint32_t(w >> 32); t += 32; }
        _Pragma("unroll") for (int half = 16; half > 0; half /= 2) {
            n = __builtin_popcount(v & ((1u << half) - 1));
            if (i >= n) { i -= n; v >>= half; t += half; }
        }
        return t;
    }
};


// A workgroup of either product takes NT tiles of 16 rows (of the gate and of the factor half each, or all of the down matrix), so
// that a request of the columns serves them all; its four waves split the contraction and are summed through LDS.
// NG: groups of 16 columns at a time; an expert with more tokens takes another pass.  PLANES: of the columns (head, remainder).
template <typename TIO, int NT, int NG, int PLANES>
struct Product {
    static constexpr int E = kPiece<TIO>, STEP = 4 * E;
    static constexpr int kSteps = NT == 1 ? 4 : 2;  // steps of the contraction in a request
    f32x4 c[NT][NG];
    const TIO *w[NT], *col[PLANES][NG];  // this lane's row of each tile and its columns, from the first element that it loads
    int K, first, last, groups;

    struct Request { u32x4 w[NT][kSteps], x[PLANES][NG][kSteps]; };

    __device__ __forceinline__ void range(int contraction, int wave) {
        K = contraction;
        const int steps = (K + STEP - 1) / STEP, per = (steps + 3) / 4;
        first = wave * per;
        last = min(steps, first + per);
    }
    __device__ __forceinline__ void request(Request& r, int s) const {
        const int k = s * STEP;
        if (s + kSteps <= last && k + kSteps * STEP <= K) {
            _Pragma("unroll") for (int u = 0; u < kSteps; ++u)
                _Pragma("unroll") for (int n = 0; n < NT; ++n) r.w[n][u] = *reinterpret_cast<const u32x4*>(w[n] + k + u * STEP);
            _Pragma("unroll") for (int g = 0; g < NG; ++g) {
                if (g >= groups) break;
                _Pragma("unroll") for (int u = 0; u < kSteps; ++u)
                    _Pragma("unroll") for (int n = 0; n < PLANES; ++n)
                        r.x[n][g][u] = *reinterpret_cast<const u32x4*>(col[n][g] + k + u * STEP);
            }
            return;
        }
        const int mine = E * int((threadIdx.x & 63) >> 4);  // beyond the end of the contraction: zeros
        _Pragma("unroll") for (int u = 0; u < kSteps; ++u) {
            const bool in = s + u < last && k + u * STEP + mine < K;
            const u32x4 zero = {0, 0, 0, 0};
            _Pragma("unroll") for (int n = 0; n < NT; ++n) r.w[n][u] = in ? *reinterpret_cast<const u32x4*>(w[n] + k + u * STEP) : zero;
            _Pragma("unroll") for (int g = 0; g < NG; ++g) {
                if (g >= groups) break;
                _Pragma("unroll") for (int n = 0; n < PLANES; ++n)
                    r.x[n][g][u] = in ? *reinterpret_cast<const u32x4*>(col[n][g] + k + u * STEP) : zero;
            }
        }
    }
    __device__ __forceinline__ void take(const Request& r) {
        _Pragma("unroll") for (int g = 0; g < NG; ++g) {
            if (g >= groups) break;
            _Pragma("unroll") for (int u = 0; u < kSteps; ++u)
                _Pragma("unroll") for (int n = 0; n < PLANES; ++n)
                    _Pragma("unroll") for (int i = 0; i < NT; ++i) c[i][g] = product(r.w[i][u], r.x[n][g][u], c[i][g], TIO());
        }
    }
    __device__ __forceinline__ void walk() {
        _Pragma("unroll") for (int g = 0; g < NG; ++g)
            _Pragma("unroll") for (int i = 0; i < NT; ++i) c[i][g] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (first >= last) return;
        Request a, b;
        request(a, first);
        for (int s = first;;) {
            s += kSteps;
            if (s < last) request(b, s);
            take(a);
            if (s >= last) break;
            s += kSteps;
            if (s < last) request(a, s);
            take(b);
            if (s >= last) break;
        }
    }
    __device__ __forceinline__ void join(f32x4 (*part)[NT * NG][64], int wave, int lane, bool again) {
        if (again) __syncthreads();
        _Pragma("unroll") for (int g = 0; g < NG; ++g)
            _Pragma("unroll") for (int i = 0; i < NT; ++i) part[wave][NT * g + i][lane] = c[i][g];
        __syncthreads();
    }
    __device__ __forceinline__ static f32x4 sum(const f32x4 (*part)[NT * NG][64], int i, int g, int lane) {
        const int at = NT * g + i;
        return (part[0][at][lane] + part[1][at][lane]) + (part[2][at][lane] + part[3][at][lane]);
    }
};

// ROUTE: at most four tokens, see Tokens
template <typename TIO, int NT, int NG, bool ROUTE>
__global__ __launch_bounds__(256) void k_moe_gate_up(MoeArgs a) {
    // Tiles of the gate, and of the factor; NT = 1: one tile of eight rows of either.
    constexpr bool SHARED = NT == 1;
    constexpr int HT = SHARED ? 1 : NT / 2, ROWS = SHARED ? 8 : 16;
    __shared__ f32x4 part[4][NT * NG][64];
    __shared__ int chosen[ROUTE ? 4 * kMaxTop : 1];
    __shared__ float weight[ROUTE ? 4 * kMaxTop : 1];
    Tokens tok = ROUTE ? Tokens(a, chosen, weight) : Tokens(a);
    if (tok.m == 0) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    typedef Product<TIO, NT, NG, 1> P;
    P p;
    p.range(a.D, wave);
    const int row0 = int(blockIdx.x) * ROWS * HT, mine = P::E * (lane >> 4);
    const TIO* w = static_cast<const TIO*>(a.w_gate_up) + size_t(tok.e) * 2 * a.F * a.D + mine;
    if (SHARED) {
        p.w[0] = w + size_t((lane & 8 ? a.F : 0) + row0 + (lane & 7)) * a.D;  // F is a multiple of 8
    } else {
        _Pragma("unroll") for (int i = 0; i < HT; ++i) {
            p.w[i] = w + size_t(min(row0 + 16 * i + (lane & 15), a.F - 1)) * a.D;
            p.w[(HT + i) % NT] = p.w[i] + size_t(a.F) * a.D;
        }
    }
    for (int i0 = 0; i0 < tok.m; i0 += 16 * NG) {
        p.groups = min(NG, (tok.m - i0 + 15) / 16);
        int token[NG];
        _Pragma("unroll") for (int g = 0; g < NG; ++g) {
            token[g] = tok.at(min(i0 + g * 16 + (lane & 15), tok.m - 1));  // with ROUTE the pair
            p.col[0][g] = static_cast<const TIO*>(a.x) + size_t(ROUTE ? token[g] / a.top_k : token[g]) * a.D + mine;
        }
        p.walk();
        p.join(part, wave, lane, i0 > 0);
        _Pragma("unroll") for (int u = 0; u < NG * HT; ++u) {
            const int g = u / HT, i = u % HT, f = row0 + 16 * i + 4 * (lane >> 4);  // F is a multiple of 8: a lane's four are all there or none
            if (g >= p.groups || u % 4 != wave || i0 + g * 16 + (lane & 15) >= tok.m || f >= a.F || (SHARED && lane >= 32)) continue;
            const f32x4 gate = P::sum(part, i, g, lane), up = SHARED ? P::sum(part, 0, g, lane + 32) : P::sum(part, HT + i, g, lane);
            const f32x2 to = ROUTE ? f32x2{weight[token[g]], __int_as_float(token[g])} : a.place[size_t(token[g]) * a.E + tok.e];
            float h[4];
            _Pragma("unroll") for (int j = 0; j < 4; ++j) h[j] = to.x * (gate[j] / (1.f + expf(-gate[j])) * up[j]);
            const size_t at = size_t(__float_as_int(to.y)) * a.F + f;
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
}

template <typename TIO, int NT, int NG>
__global__ __launch_bounds__(256) void k_moe_down(MoeArgs a) {
    __shared__ f32x4 part[4][NT * NG][64];
    const Tokens tok(a);
    if (tok.m == 0) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    constexpr int PLANES = sizeof(TIO) == 2 ? 2 : 1;
    typedef Product<TIO, NT, NG, PLANES> P;
    P p;
    p.range(a.F, wave);
    const int row0 = int(blockIdx.x) * 16 * NT, mine = P::E * (lane >> 4);
    _Pragma("unroll") for (int i = 0; i < NT; ++i)
        p.w[i] = static_cast<const TIO*>(a.w_down) + (size_t(tok.e) * a.D + min(row0 + 16 * i + (lane & 15), a.D - 1)) * a.F + mine;
    for (int i0 = 0; i0 < tok.m; i0 += 16 * NG) {
        p.groups = min(NG, (tok.m - i0 + 15) / 16);
        int pair[NG];
        _Pragma("unroll") for (int g = 0; g < NG; ++g) {
            const int token = tok.at(min(i0 + g * 16 + (lane & 15), tok.m - 1));
            pair[g] = __float_as_int(a.place[size_t(token) * a.E + tok.e].y);
            p.col[0][g] = static_cast<const TIO*>(a.h) + size_t(pair[g]) * a.F + mine;
            if (PLANES == 2) p.col[PLANES - 1][g] = static_cast<const TIO*>(a.h_rem) + size_t(pair[g]) * a.F + mine;
        }
        p.walk();
        p.join(part, wave, lane, i0 > 0);
        _Pragma("unroll") for (int u = 0; u < NG * NT; ++u) {
            const int g = u / NT, i = u % NT, d = row0 + 16 * i + 4 * (lane >> 4);
            if (g >= p.groups || u % 4 != wave || i0 + g * 16 + (lane & 15) >= tok.m || d >= a.D) continue;
            *reinterpret_cast<f32x4*>(a.part + size_t(pair[g]) * a.D + d) = P::sum(part, i, g, lane);
        }
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
struct MoeSpace { size_t logits, chosen, place, mask, h, h_rem, part, bytes; };
MoeSpace space(const lsm_moe_params& p) {
    const size_t pairs = size_t(p.n) * p.top_k, el = p.dtype == LSM_DTYPE_BF16 ? 2 : 4;
    MoeSpace s{};
    s.logits = 0;
    s.chosen = s.logits + align256(size_t(p.n) * p.E * 4);
    s.place = s.chosen + align256(pairs * 4);
    s.mask = s.place + align256(size_t(p.n) * p.E * sizeof(f32x2));
    s.h = s.mask + align256(size_t(p.E) * 2 * sizeof(u64));
    s.h_rem = s.h + align256(pairs * p.F * el);
    s.part = s.h_rem + (el == 2 ? align256(pairs * p.F * el) : 0);
    s.bytes = s.part + align256(pairs * p.D * 4);
    return s;
}
constexpr int kRouteAlong = 4;  // tokens that the first product's workgroups route themselves

// The launches: whether each could be enqueued, and nothing after one that could not.
template <typename TIO, int NT, int NG>
bool launch_gate_up(const MoeArgs& a, int y, hipStream_t st) {
    ProfScope ps(KID_MOE_GATE_UP, st);
    const dim3 grid((a.F + 8 * NT - 1) / (8 * NT), y);
    constexpr bool ALONG = NG == 1 && NT < 4;
    if (ALONG && a.n <= kRouteAlong) hipLaunchKernelGGL((k_moe_gate_up<TIO, NT, NG, ALONG>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_moe_gate_up<TIO, NT, NG, false>), grid, dim3(256), 0, st, a);
    return launched();
}
template <typename TIO, int NT, int NG>
bool launch_down(const MoeArgs& a, int y, hipStream_t st) {
    ProfScope ps(KID_MOE_DOWN, st);
    hipLaunchKernelGGL((k_moe_down<TIO, NT, NG>), dim3((a.D + 16 * NT - 1) / (16 * NT), y), dim3(256), 0, st, a);
    return launched();
}
// Tiles: four where columns are half full, so that they are requested half as often (128 tokens, 12 an expert: 277 -> 259 us), else
// two (16 tokens 167 -> 162 us, one token 28 -> 25).  Half as many where the workgroups are too few for the chip, or few and long, so
// that a compute unit with one more than another has much more to do (110 tokens, 8 experts of 168 x 376, all active: 33.5 -> 29.6 us;
// 64 tokens, 8 experts of 1024 x 1024 in fp32: 59 -> 49; 4 tokens, 8 of 2000 x 3000 in fp32: 117 -> 102).  Not where they are few
// but short: the columns would be requested more often (90 tokens, 8 of 648 x 472, first product 11.1 -> 13.5 us).
int tiles(int rows, int experts, bool half_full, int64_t row_bytes) {
    int nt = half_full ? 4 : 2;
    for (; nt > 1; nt /= 2) {
        const int64_t groups = int64_t(experts) * ((rows + 16 * nt - 1) / (16 * nt)), bytes = 16 * nt * row_bytes;
        if (groups >= 128 && (groups >= 512 || bytes <= (96 << 10)) && (groups >= 2048 || bytes <= (256 << 10))) break;
    }
    return nt;
}
template <typename TIO, int NG>
bool launch_experts(const MoeArgs& a, bool half_full, hipStream_t st) {
    const int pairs = a.n * a.top_k, y = a.by_pair ? pairs : a.E;
    const int up = tiles(2 * a.F, y, half_full, int64_t(a.D) * int(sizeof(TIO))),
              down = tiles(a.D, y, half_full, int64_t(a.F) * int(sizeof(TIO)));
    if (!(up == 4 ? launch_gate_up<TIO, 4, NG>(a, y, st) : up == 2 ? launch_gate_up<TIO, 2, NG>(a, y, st)
                                                                   : launch_gate_up<TIO, 1, NG>(a, y, st)))
        return false;
    if (!(down == 4 ? launch_down<TIO, 4, NG>(a, y, st) : down == 2 ? launch_down<TIO, 2, NG>(a, y, st)
                                                                    : launch_down<TIO, 1, NG>(a, y, st)))
        return false;
    ProfScope ps(KID_MOE_SUM, st);
    hipLaunchKernelGGL((k_moe_sum<TIO>), dim3(unsigned((size_t(a.n) * a.D / 4 + 255) / 256)), dim3(256), 0, st, a);
    return launched();
}
template <typename TIO>
bool launch(const MoeArgs& a, hipStream_t st) {
    {
        ProfScope ps(KID_MOE_ROUTER, st);
        hipLaunchKernelGGL((k_moe_router<TIO>), dim3(a.E, (a.n + 15) / 16), dim3(256), 0, st, a);
    }
    if (!launched()) return false;
    if (a.n > kRouteAlong) {
        ProfScope ps(KID_MOE_ROUTER, st);
        if (a.E <= 64) hipLaunchKernelGGL((k_moe_route<1>), dim3((a.n + 3) / 4), dim3(256), 0, st, a);
        else hipLaunchKernelGGL((k_moe_route<kWide>), dim3((a.n + 3) / 4), dim3(256), 0, st, a);
        if (!launched()) return false;
    }
    // Columns: as many groups of 16 as an expert has tokens, give or take the spread of chance (more take another pass; with
    // groups that are rarely used the registers would be missing: 128 tokens, 12 an expert: 4 groups 296 us, 2 groups 259).
    const float mean = float(a.n) * a.top_k / a.E, most = mean + 2.f * sqrtf(mean);
    const bool half_full = mean >= 8.f;
    if (a.n <= 16) return launch_experts<TIO, 1>(a, half_full, st);
    if (a.n <= 32 || most <= 32.f) return launch_experts<TIO, 2>(a, half_full, st);
    return launch_experts<TIO, 4>(a, half_full, st);
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
    const MoeArgs a{x, router, w_gate_up, w_down, residual, y, reinterpret_cast<float*>(ws + s.logits),
                    reinterpret_cast<int*>(ws + s.chosen), reinterpret_cast<f32x2*>(ws + s.place), reinterpret_cast<u64*>(ws + s.mask),
                    ws + s.h, ws + s.h_rem, reinterpret_cast<float*>(ws + s.part), p->n, p->D, p->F, p->E, p->top_k, p->renormalise,
                    p->n * p->top_k < p->E};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return (p->dtype == LSM_DTYPE_BF16 ? launch<uint16_t>(a, st) : launch<float>(a, st)) ? LSM_OK : LSM_ERR_LAUNCH;
}

}  // extern "C"
