// The experts' products for many tokens, forward and backward (include/lsm_train.h), over pairs sorted by expert (lsm_route.hip):
//   k_up           h = silu(Wg x) * (Wu x) of every pair, x taken through the plan's order
//   k_down         Wd h, fp32, a row a pair
//   k_sum          the weighted sum of a token's pairs and the residual; backward the sum of dx and of the weights' gradients
//   k_hidden_grad  both products of the hidden layer again and t = Wd^T dy; from them the gradients of gate and factor, the
//                  activations times their weight, and the part of <t, h> that belongs to the tile
//   k_dx           the gradients of gate and factor times Wg, Wu, fp32, a row a pair
//   k_dw           both weights' gradients, an expert's pairs being the long axis
// An expert's rows are whole tiles but the last; a workgroup finds its expert and tile from the offsets, which stay on the device.
//
// Bound: the matrix products for many tokens, the weights' bytes for few.  16384 tokens of 1024, 64 experts of 1024, 8 a token, bf16: up
// 511 us (1.08 PFLOP/s; matrix cores busy 0.59 of the clocks), down 327 (0.84, 0.45), sum 131 (4.6 TB/s), hidden_grad 1053 (0.78, 0.41: one tile's
// products and the other's follow each other, with a fresh start each), dx 545 (1.01, 0.55), dw 830 to 915 for both (0.90 to 0.99, 0.56: a mean of 2048
// pairs is 64 steps a tile), against 1.17 to 1.42 of large library products.  Five tokens: 26, 17 and 4 us for 168 and 84 MB of weights.  fp32, 1500
// tokens of 512, 8 experts of 776, 2 a token: 55, 38, 5, 86, 69, 7 and 121 us, 50 to 82 TFLOP/s (busy 0.61 to 0.72).
// Nothing is saved by the forward call: gate and factor formed again cost 500 us there, kept they would be 0.5 GB a layer.  A pair's result is a
// row of its own, added up by k_sum in a fixed order: adding to the token's row at once would need atomics, whose order is not fixed.
// These rows are parts of a token's sum and stay in fp32: as fp16 with a power of two for each stretch of a row they would take half the bytes
// (16384 tokens forward and backward 3520 -> 3365 us, five tokens 44.4 -> 46.1), and change five tokens' results by 5e-4 of their size.
#include "lsm_product_dev.h"

namespace lsm {
namespace {

struct ExpertArgs {
    const void *x, *w_gate_up, *w_down, *residual, *d_y;
    const float* weights;
    const int32_t *offsets, *order, *place;
    void *y, *d_w_gate_up, *d_w_down;
    float* d_weights;
    void *h, *da;         // [pairs][F]: activations (backward: times their weight); [pairs][2 F]; rows from line to line
    float *part, *weight_part;  // [pairs][D]; [tiles of F][pairs]
    int n, D, F, E, top_k, parts;
    int halves;             // rows of a pair in h (forward) or da (backward): 2 where a remainder follows what was rounded
    uint32_t x_bytes, dy_bytes, h_bytes, da_bytes;  // between rows
};

// What the plan says, kept inside the buffers whatever stands there.
__device__ __forceinline__ int offset_of(const ExpertArgs& a, int e) { return min(max(a.offsets[e], 0), a.n * a.top_k); }
__device__ __forceinline__ uint32_t pair_of(const ExpertArgs& a, int at) { return min(uint32_t(a.order[at]), uint32_t(a.n * a.top_k - 1)); }
__device__ __forceinline__ uint32_t token_of(const ExpertArgs& a, int at) { return pair_of(a, at) / uint32_t(a.top_k); }

template <typename TIO> __device__ __forceinline__ TIO* row_of(void* rows, int at, uint32_t bytes) {
    return reinterpret_cast<TIO*>(static_cast<char*>(rows) + size_t(at) * bytes);
}

__device__ __forceinline__ f32x4 remainders(const f32x4& x) {
    return f32x4{remainder_of(x[0]), remainder_of(x[1]), remainder_of(x[2]), remainder_of(x[3])};
}
struct Where { int e, first, count, r, c; };  // expert, its first place and its pairs, the tile's number along rows and columns

// The tiles of a workgroup, of all experts' tiles of BR rows x `cols` columns in the order expert, column, row.  Workgroups are dealt out
// to the eight dies in turn; a die gets neighbouring tiles, which share operands in its L2.
template <int BR>
struct Finder {
    int o[5], tiles[4], upto, own;  // of four experts a lane: where they begin, their row tiles; row tiles up to and of this lane
    __device__ __forceinline__ Finder(const ExpertArgs& a, int halves = 1) {
        const int lane = threadIdx.x & 63;
        own = 0;
        _Pragma("unroll") for (int i = 0; i < 5; ++i) o[i] = offset_of(a, min(4 * lane + i, a.E)) * halves;
        _Pragma("unroll") for (int i = 0; i < 4; ++i) {
            tiles[i] = max(o[i + 1] - o[i] + BR - 1, 0) / BR;
            own += tiles[i];
        }
        upto = own;
        for (int off = 1; off < 64; off <<= 1) {
            const int t = __shfl_up(upto, off, 64);
            if (lane >= off) upto += t;
        }
    }
    // The n-th tile of this workgroup; false: there is none.
    __device__ __forceinline__ bool find(int n, int cols, Where& w) const {
        const int all = min(__builtin_amdgcn_readlane(upto, 63), int(kMostTiles) / cols) * cols, die = (all + 7) / 8;
        const int at = int(blockIdx.x) / 8 + n * (int(gridDim.x) / 8), id = (int(blockIdx.x) % 8) * die + at;
        if (at >= die || id >= all) return false;
        const int l = lanes(__ballot(upto <= id / cols));
        int rest = id - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(own, l)) * cols;
        _Pragma("unroll") for (int i = 0; i < 4; ++i) {
            const int t = __builtin_amdgcn_readlane(tiles[i], l);
            if (rest < t * cols) {
                w.e = 4 * l + i;
                w.first = __builtin_amdgcn_readlane(o[i], l);
                w.count = __builtin_amdgcn_readlane(o[i + 1], l) - w.first;
                w.c = rest / t;
                w.r = rest - w.c * t;
                return true;
            }
            rest -= t * cols;
        }
        return false;
    }
};

// The rows of gate and factor for the same features are blocks i and i + TC / 2 of one wave.
template <typename T>
__device__ __forceinline__ uint32_t gate_up_row(const ExpertArgs& a, int c, int q) {
    constexpr int HALF = T::TC / 2;
    const int wave = q / (T::TC * 16), i = q / 16 % T::TC, f = c * (T::BC / 2) + (wave * HALF + i % HALF) * 16 + q % 16;
    return f < a.F ? uint32_t((i >= HALF ? a.F : 0) + f) * uint32_t(a.D) * uint32_t(sizeof(typename T::TIO)) : kBeyond;
}
// pair_at(i): the pair of row i of the tile
template <typename T, typename PairAt>
__device__ __forceinline__ void start_gate_up(const T& t, typename T::C& c, typename T::R& r, const ExpertArgs& a, const Where& w, PairAt pair_at) {
    typedef typename T::TIO TIO;
    r.start_rows(a.x, t.wave, t.lane, [&](int i) { return w.r * T::BR + i < w.count ? pair_at(i) / uint32_t(a.top_k) * a.x_bytes : kBeyond; });
    c.start_rows(static_cast<const TIO*>(a.w_gate_up) + size_t(w.e) * 2 * a.F * a.D, t.wave, t.lane,
                 [&](int q) { return gate_up_row<T>(a, w.c, q); });
}
template <typename T>
__device__ __forceinline__ void start_gate_up(T& t, const ExpertArgs& a, const Where& w) {
    start_gate_up(t, t.c, t.r, a, w, [&](int i) { return pair_of(a, w.first + w.r * T::BR + i); });
}

template <typename T>
__global__ __launch_bounds__(T::THREADS) void k_up(ExpertArgs a) {
    typedef typename T::TIO TIO;
    __shared__ __attribute__((aligned(1024))) char shared[T::LDS];
    const int cols = (a.F + T::BC / 2 - 1) / (T::BC / 2);
    const Finder<T::BR> finder(a);
    Where w;
    if (!finder.find(0, cols, w)) return;
    T t(shared);
    start_gate_up(t, a, w);
    for (int n = 1;; ++n) {
        Where next{};
        const bool more = T::FOLLOWED && finder.find(n, cols, next);
        if (more) t.bring(a.order + next.first + next.r * T::BR, next.count - next.r * T::BR);
        else next.count = 0;
        f32x4 acc[T::TC][T::TR];
        clear<T>(acc);
        t.walk(acc, a.D, typename T::Nothing(), [&]() {
            start_gate_up(t, t.c2, t.r2, a, next, [&](int i) { return min(uint32_t(t.brought(i)), uint32_t(a.n * a.top_k - 1)); });
        });
        constexpr int HALF = T::TC / 2;
        const int f0 = w.c * (T::BC / 2) + t.wc * HALF * 16;
        const int halves = kMayHalve<T> ? a.halves : 1;
        _Pragma("unroll") for (int j = 0; j < T::TR; ++j) {
            _Pragma("unroll") for (int i = 0; i < HALF; ++i)
                _Pragma("unroll") for (int e = 0; e < 4; ++e) {
                    const float gate = acc[i][j][e];
                    acc[i][j][e] = gate * sigmoid(gate, TIO()) * acc[i + HALF][j][e];
                }
            const auto line = [&](int half) {
                return [=, &w](int r) {
                    const int at = w.r * T::BR + r;
                    return at < w.count ? row_of<TIO>(a.h, (w.first + at) * halves + half, a.h_bytes) + f0 : nullptr;
                };
            };
            t.template store<HALF, TIO>(j, a.F - f0, [&](int i) { return acc[i][j]; }, line(0));
            if constexpr (kMayHalve<T>)
                if (halves == 2) t.template store<HALF, TIO>(j, a.F - f0, [&](int i) { return remainders(acc[i][j]); }, line(1));
        }
        if (!more) return;
        t.go_on();
        w = next;
    }
}

// rows of `part` = the tile's
template <typename T>
__device__ __forceinline__ void finish_part(const T& t, const ExpertArgs& a, const Where& w, f32x4 (&acc)[T::TC][T::TR]) {
    const int d0 = (w.c * T::WC + t.wc) * T::TC * 16, halves = kMayHalve<T> ? a.halves : 1;
    if constexpr (kMayHalve<T>)
        if (halves == 2)  // both rows of a pair, in neighbouring lanes
            _Pragma("unroll") for (int i = 0; i < T::TC; ++i)
                _Pragma("unroll") for (int j = 0; j < T::TR; ++j)
                    _Pragma("unroll") for (int e = 0; e < 4; ++e) acc[i][j][e] += dpp<0xB1>(acc[i][j][e]);
    _Pragma("unroll") for (int j = 0; j < T::TR; ++j)
        t.template store<T::TC, float>(j, a.D - d0, [&](int i) { return acc[i][j]; }, [&](int r) {
            const int row = w.r * T::BR + r;
            return row < w.count && (row & (halves - 1)) == 0 ? a.part + size_t((w.first + row) >> (halves - 1)) * a.D + d0 : nullptr;
        });
}
// rows of the pairs of this tile, `bytes` each, one after the other
template <typename T>
__device__ __forceinline__ void start_pairs(const T& t, typename T::R& r, const void* rows, const Where& w, uint32_t bytes) {
    r.start_rows(static_cast<const char*>(rows) + size_t(w.first + w.r * T::BR) * bytes, t.wave, t.lane,
                 [&](int i) { return w.r * T::BR + i < w.count ? uint32_t(i) * bytes : kBeyond; });
}

// `part` of all tiles of [pairs][D]: start(t, c, r, w) sets a tile's operands, K long
template <typename T, typename Start>
__device__ __forceinline__ void part_tiles(char* shared, const ExpertArgs& a, int K, Start start) {
    const int cols = (a.D + T::BC - 1) / T::BC;
    const Finder<T::BR> finder(a, kMayHalve<T> ? a.halves : 1);
    Where w;
    if (!finder.find(0, cols, w)) return;
    T t(shared);
    start(t, t.c, t.r, w);
    for (int n = 1;; ++n) {
        Where next{};
        const bool more = T::FOLLOWED && finder.find(n, cols, next);
        if (!more) next.count = 0;
        f32x4 acc[T::TC][T::TR];
        clear<T>(acc);
        t.walk(acc, K, typename T::Nothing(), [&]() { start(t, t.c2, t.r2, next); });
        finish_part(t, a, w, acc);
        if (!more) return;
        t.go_on();
        w = next;
    }
}

template <typename T>
__global__ __launch_bounds__(T::THREADS) void k_down(ExpertArgs a) {
    typedef typename T::TIO TIO;
    __shared__ __attribute__((aligned(1024))) char shared[T::LDS];
    const uint32_t bytes = uint32_t(a.F) * uint32_t(sizeof(TIO));
    part_tiles<T>(shared, a, a.F, [&](const T& t, typename T::C& c, typename T::R& r, const Where& w) {
        start_pairs(t, r, a.h, w, a.h_bytes);
        c.start_rows(static_cast<const TIO*>(a.w_down) + size_t(w.e) * a.D * a.F, t.wave, t.lane, [&](int q) {
            const int d = w.c * T::BC + q;
            return d < a.D ? uint32_t(d) * bytes : kBeyond;
        });
    });
}

template <typename T>
__global__ __launch_bounds__(T::THREADS) void k_dx(ExpertArgs a) {
    typedef typename T::TIO TIO;
    __shared__ __attribute__((aligned(1024))) char shared[T::LDS];
    part_tiles<T>(shared, a, 2 * a.F, [&](const T& t, typename T::C& c, typename T::R& r, const Where& w) {
        start_pairs(t, r, a.da, w, a.da_bytes);
        c.start_cols(static_cast<const TIO*>(a.w_gate_up) + size_t(w.e) * 2 * a.F * a.D, a.D * int(sizeof(TIO)), w.c * T::BC, a.D, t.wave, t.lane, 0);
    });
}

// H: the products of gate and factor; T: that of dy with the columns of Wd for the same features.
template <typename H, typename T>
__global__ __launch_bounds__(T::THREADS) void k_hidden_grad(ExpertArgs a) {
    typedef typename T::TIO TIO;
    static_assert(H::TC == 2 * T::TC && H::TR == T::TR && H::WC == T::WC && H::WR == T::WR, "the same features in the same lanes");
    __shared__ __attribute__((aligned(1024))) char shared[H::LDS > T::LDS ? H::LDS : T::LDS];
    Where w;
    if (!Finder<T::BR>(a).find(0, (a.F + T::BC - 1) / T::BC, w)) return;
    f32x4 gu[H::TC][H::TR], tt[T::TC][T::TR];
    float weight[T::TR];
    {
        H t(shared);
        start_gate_up(t, a, w);
        clear<H>(gu);
        t.walk(gu, a.D);
    }
    T t(shared);
    t.r.start_rows(a.d_y, t.wave, t.lane, [&](int i) {
        const int at = w.r * T::BR + i;
        return at < w.count ? token_of(a, w.first + at) * a.dy_bytes : kBeyond;
    });
    t.c.start_cols(static_cast<const TIO*>(a.w_down) + size_t(w.e) * a.D * a.F, a.F * int(sizeof(TIO)), w.c * T::BC, a.F, t.wave, t.lane, 0);
    clear<T>(tt);
    t.walk(tt, a.D);
    _Pragma("unroll") for (int j = 0; j < T::TR; ++j)
        weight[j] = w.r * T::BR + t.row(j) < w.count ? a.weights[pair_of(a, w.first + w.r * T::BR + t.row(j))] : 0.f;
    const int f0 = w.c * T::BC + t.wc * T::TC * 16;
    _Pragma("unroll") for (int j = 0; j < T::TR; ++j) {
        const int at = w.r * T::BR + t.row(j);
        const float p = weight[j];
        float along = 0.f;
        _Pragma("unroll") for (int i = 0; i < T::TC; ++i)
            _Pragma("unroll") for (int r = 0; r < 4; ++r) {
                const float gate = gu[i][j][r], up = gu[i + T::TC][j][r], d = tt[i][j][r];
                const float sig = sigmoid(gate, TIO()), s = gate * sig, h = s * up, dh = p * d;
                along += d * h;
                gu[i][j][r] = dh * up * (sig + s * (1.f - sig));
                gu[i + T::TC][j][r] = dh * s;
                tt[i][j][r] = p * h;
            }
        along = T::row_sum(along);
        if (t.lane < 16 && at < w.count) a.weight_part[size_t(w.c * T::WC + t.wc) * (size_t(a.n) * a.top_k) + w.first + at] = along;
        const int halves = kMayHalve<T> ? a.halves : 1;
        const auto line = [&](void* base, uint32_t bytes, int shift, int by, int which) {
            return [=, &w](int r) {
                const int q = w.r * T::BR + r;
                return q < w.count ? row_of<TIO>(base, (w.first + q) * by + which, bytes) + shift + f0 : nullptr;
            };
        };
        _Pragma("unroll") for (int half = 0; half < 2; ++half)
            t.template store<T::TC, TIO>(j, a.F - f0, [&](int i) { return gu[half * T::TC + i][j]; }, line(a.da, a.da_bytes, half * a.F, halves, 0));
        if constexpr (kMayHalve<T>)
            if (halves == 2)
                _Pragma("unroll") for (int half = 0; half < 2; ++half)
                    t.template store<T::TC, TIO>(j, a.F - f0, [&](int i) { return remainders(gu[half * T::TC + i][j]); },
                                                 line(a.da, a.da_bytes, half * a.F, halves, 1));
        t.template store<T::TC, TIO>(j, a.F - f0, [&](int i) { return tt[i][j]; }, line(a.h, a.h_bytes, 0, 1, 0));
    }
}

// DOWN: d_w_down [D][F] = sum over the expert's pairs of dy (rows) and weighted activations (columns); else d_w_gate_up [2 F][D] of the
// gradients of gate and factor (rows) and x (columns).
template <typename T, bool DOWN>
__global__ __launch_bounds__(T::THREADS) void k_dw(ExpertArgs a, int row_tiles, int col_tiles) {
    typedef typename T::TIO TIO;
    constexpr int EL = int(sizeof(TIO));
    __shared__ __attribute__((aligned(1024))) char shared[T::LDS];
    const int all = a.E * row_tiles * col_tiles, die = (all + 7) / 8, slot = int(blockIdx.x) / 8, id = (int(blockIdx.x) % 8) * die + slot;
    if (slot >= die || id >= all) return;
    const int e = id / (row_tiles * col_tiles), rest = id - e * row_tiles * col_tiles, c = rest / row_tiles, r0 = rest - c * row_tiles;
    const int first = uniform(offset_of(a, e)), count = max(uniform(offset_of(a, e + 1)) - first, 0);
    const int rows = DOWN ? a.D : 2 * a.F, cols = DOWN ? a.F : a.D;
    T t(shared);
    if (DOWN) {
        t.r.start_cols(a.d_y, int(a.dy_bytes), r0 * T::BR, rows, t.wave, t.lane, t.list_at());
        t.c.start_cols(row_of<TIO>(a.h, first, a.h_bytes), int(a.h_bytes), c * T::BC, cols, t.wave, t.lane, 0);
    } else {
        t.r.start_cols(row_of<TIO>(a.da, first * a.halves, a.da_bytes), int(a.da_bytes) * a.halves, r0 * T::BR, rows, t.wave, t.lane, 0);
        t.c.start_cols(a.x, int(a.x_bytes), c * T::BC, cols, t.wave, t.lane, t.list_at());
    }
    f32x4 acc[T::TC][T::TR];
    clear<T>(acc);
    t.walk(acc, count, [&](int k) { return token_of(a, first + k); });
    TIO* out = static_cast<TIO*>(DOWN ? a.d_w_down : a.d_w_gate_up) + size_t(e) * rows * cols;
    const int c0 = c * T::BC + t.wc * T::TC * 16;
    _Pragma("unroll") for (int j = 0; j < T::TR; ++j) {
        t.template store<T::TC, TIO>(j, cols - c0, [&](int i) { return acc[i][j]; }, [&](int r) {
            const int row = r0 * T::BR + r;
            return row < rows ? out + size_t(row) * cols + c0 : nullptr;
        });
    }
}

// Four (fp32) or eight (bf16) neighbouring elements of a token; WEIGHTED: forward.
template <typename TIO, bool WEIGHTED>
__global__ __launch_bounds__(256) void k_sum(ExpertArgs a) {
    constexpr int E = kPiece<TIO>;
    const int pieces = a.D / E;
    const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (!WEIGHTED && id < int64_t(a.n) * a.top_k) {
        const int at = a.place[id];
        float s = 0.f;
        if (uint32_t(at) < uint32_t(a.n * a.top_k))
            for (int b = 0; b < a.parts; b += 16) {  // requested together
                float x[16];
                _Pragma("unroll") for (int u = 0; u < 16; ++u)
                    x[u] = b + u < a.parts ? a.weight_part[size_t(b + u) * (size_t(a.n) * a.top_k) + at] : 0.f;
                _Pragma("unroll") for (int u = 0; u < 16; ++u) s += x[u];
            }
        a.d_weights[id] = s;
    }
    if (id >= int64_t(a.n) * pieces) return;
    const int t = int(id / pieces), d = int(id - int64_t(t) * pieces) * E;
    float s[E];
    if (WEIGHTED && a.residual) unpack(*reinterpret_cast<const u32x4*>(static_cast<const TIO*>(a.residual) + size_t(t) * a.D + d), s);
    else _Pragma("unroll") for (int e = 0; e < E; ++e) s[e] = 0.f;
    constexpr int U = 4;  // pairs requested at a time
    for (int j0 = 0; j0 < a.top_k; j0 += U) {
        int at[U];
        float p[U];
        f32x4 z[U][E / 4];
        _Pragma("unroll") for (int u = 0; u < U; ++u) {
            at[u] = j0 + u < a.top_k ? a.place[size_t(t) * a.top_k + j0 + u] : -1;
            if (uint32_t(at[u]) >= uint32_t(a.n * a.top_k)) at[u] = -1;
            p[u] = !WEIGHTED ? 1.f : at[u] < 0 ? 0.f : a.weights[size_t(t) * a.top_k + j0 + u];
        }
        _Pragma("unroll") for (int u = 0; u < U; ++u) {
            if (at[u] < 0) continue;
            _Pragma("unroll") for (int i = 0; i < E / 4; ++i)
                z[u][i] = *reinterpret_cast<const f32x4*>(a.part + size_t(at[u]) * a.D + d + 4 * i);
        }
        _Pragma("unroll") for (int u = 0; u < U; ++u) {
            if (at[u] < 0) continue;
            _Pragma("unroll") for (int i = 0; i < E / 4; ++i)
                _Pragma("unroll") for (int e = 0; e < 4; ++e) s[4 * i + e] += p[u] * z[u][i][e];
        }
    }
    *reinterpret_cast<u32x4*>(static_cast<TIO*>(a.y) + size_t(t) * a.D + d) = pack(s);
}

// ---- host ------------------------------------------------------------------------------------------------------------
bool fits(const lsm_experts_params& p, bool backward);
int check(const lsm_experts_params* p, bool backward) {
    if (!p) return LSM_ERR_NULL;
    if (p->struct_size != sizeof(lsm_experts_params)) return LSM_ERR_SHAPE;
    if (p->n < 1 || p->D < 1 || p->F < 1 || p->E < 1 || p->top_k < 1 || p->top_k > p->E) return LSM_ERR_SHAPE;
    if (p->dtype != LSM_DTYPE_F32 && p->dtype != LSM_DTYPE_BF16) return LSM_ERR_UNSUPPORTED;
    if (p->E > kMostExperts || p->top_k > kMostTop || p->D % 8 || p->F % 8 || p->D > 65536 || p->F > 65536 || p->reserved != 0)
        return LSM_ERR_UNSUPPORTED;
    const int64_t el = p->dtype == LSM_DTYPE_BF16 ? 2 : 4;
    if (int64_t(p->n) * p->top_k > kMostPairs || 2 * int64_t(p->F) * p->D * el >= int64_t(kBeyond)) return LSM_ERR_SHAPE;
    for (const int64_t s : {p->x_stride, backward ? p->dy_stride : int64_t(p->x_stride)}) {
        if (s < p->D || s > (int64_t(1) << 31) || p->n * s * el >= int64_t(kBeyond)) return LSM_ERR_SHAPE;
        if (s % 8) return LSM_ERR_ALIGN;
    }
    return fits(*p, backward) ? LSM_OK : LSM_ERR_SHAPE;
}

// In calls of up to 16 tokens the rounding of what goes from one product into the next is kept as a row of its own behind it: an expert's rows
// are still one tile, the weights are read once, and with bf16 elements the result's rounding is the only one that counts (without: errors
// of 1.41 times it; 64 experts of 1024 x 1024, 8 a token, forward: five tokens 38.0 -> 38.8 us, 16 tokens 74 -> 76).  With more tokens the
// products that take the second rows would be twice as long.
int halves_of(const lsm_experts_params& p) { return p.dtype == LSM_DTYPE_BF16 && p.n <= 16 ? 2 : 1; }

// Tiles of the products over pairs, whose rows are ragged, and of the weights' gradients.
struct Plan { int up, down, hidden, dx, dw1, dw2; };
int64_t tiles_of_rows(const lsm_experts_params& p, int rows) {  // about: every expert's last tile is half empty
    const int64_t pairs = int64_t(p.n) * p.top_k, active = pairs < p.E ? pairs : p.E, full = pairs / rows + active / 2;
    return full > active ? full : active;
}
Plan plan_of(const lsm_experts_params& p) {
    const bool f32 = p.dtype == LSM_DTYPE_F32;
    const auto rows = [&](int cols, int K, int parts) {
        return pick_tile(f32, K, [&](const TileSize& t) { return tiles_of_rows(p, t.rows) * up(cols, t.cols / parts); },
                         halves_of(p) == 2 ? 0x78 : f32 ? 0x7e : 0x7f);
    };
    const int64_t mean = (int64_t(p.n) * p.top_k + p.E - 1) / p.E;
    const auto square = [&](int r, int c) {
        return pick_tile(f32, mean, [&](const TileSize& t) { return int64_t(p.E) * up(r, t.rows) * up(c, t.cols); }, (f32 ? 0 : 1 << 0) | 1 << 2 | 1 << 5);
    };
    return Plan{rows(p.F, p.D, 2), rows(p.D, p.F, 1), rows(p.F, p.D + p.D / 2, 2), rows(p.D, 2 * p.F, 1), square(2 * p.F, p.D), square(p.D, p.F)};
}
int weight_parts(const lsm_experts_params& p, int kind) { return up(p.F, kTiles[kind].cols / 2) * kTiles[kind].waves; }
// The most tiles there can be: every expert's last one may be almost empty.
int64_t most_tiles(int64_t pairs, int E, int rows, int cols, int halves) {
    return (pairs * halves / rows + (pairs < E ? pairs : int64_t(E))) * cols;
}
bool fits(const lsm_experts_params& p, bool backward) {
    const Plan q = plan_of(p);
    const auto rows = [&](int kind, int cols, int parts) {
        return most_tiles(int64_t(p.n) * p.top_k, p.E, kTiles[kind].rows, up(cols, kTiles[kind].cols / parts), halves_of(p)) < kMostTiles;
    };
    const auto square = [&](int kind, int r, int c) { return int64_t(p.E) * up(r, kTiles[kind].rows) * up(c, kTiles[kind].cols) < kMostTiles; };
    if (!backward) return rows(q.up, p.F, 2) && rows(q.down, p.D, 1);
    return rows(q.hidden, p.F, 2) && rows(q.dx, p.D, 1) && square(q.dw1, 2 * p.F, p.D) && square(q.dw2, p.D, p.F);
}
template <typename T>
unsigned grid_of(const ExpertArgs& a, int cols, int halves = 1) {
    const unsigned all = unsigned((most_tiles(int64_t(a.n) * a.top_k, a.E, T::BR, cols, halves) + 7) / 8 * 8);
    return T::FOLLOWED && all > 256 ? 256 : all;  // one for each compute unit
}

// Rows of own buffers begin with a line of the caches: a step's 64 bytes of a row are in one line, where else they lie across two if the
// width is not whole lines (2047 tokens, 64 experts of 1032: Wd h 173 -> 163 us).
size_t line_bytes(size_t bytes) { return (bytes + 127) / 128 * 128; }

struct Space { size_t h, da, part, weight_part, bytes; };
Space space(const lsm_experts_params& p, bool backward) {
    const size_t pairs = size_t(p.n) * p.top_k, el = p.dtype == LSM_DTYPE_BF16 ? 2 : 4;
    const Plan q = plan_of(p);
    Space s{};
    s.h = 0;
    s.part = align256(pairs * (backward ? 1 : halves_of(p)) * line_bytes(p.F * el));
    s.da = s.part + align256(pairs * p.D * 4);
    s.weight_part = s.da + (backward ? align256(pairs * halves_of(p) * line_bytes(2 * p.F * el)) : 0);
    s.bytes = s.weight_part + (backward ? align256(pairs * weight_parts(p, q.hidden) * 4) : 0);
    return s;
}

template <typename TIO, bool WEIGHTED>
bool launch_sum(const ExpertArgs& a, hipStream_t st) {
    int64_t items = int64_t(a.n) * (a.D / kPiece<TIO>);
    if (!WEIGHTED && items < int64_t(a.n) * a.top_k) items = int64_t(a.n) * a.top_k;
    ProfScope ps(KID_EXPERTS_SUM, st);
    hipLaunchKernelGGL((k_sum<TIO, WEIGHTED>), dim3(unsigned((items + 255) / 256)), dim3(256), 0, st, a);
    return launched();
}

template <typename TIO, int KIND>
bool launch_up(const ExpertArgs& a, hipStream_t st) {
    typedef typename TileOf<TIO, BY_ROWS, BY_ROWS, KIND, false, false, false, true>::type T;
    ProfScope ps(KID_EXPERTS_UP, st);
    hipLaunchKernelGGL((k_up<T>), dim3(grid_of<T>(a, up(a.F, T::BC / 2))), dim3(T::THREADS), 0, st, a);
    return launched();
}
template <typename TIO, int KIND>
bool launch_down(const ExpertArgs& a, hipStream_t st) {
    typedef typename TileOf<TIO, BY_ROWS, BY_ROWS, KIND, false, false, false, true>::type T;
    ProfScope ps(KID_EXPERTS_DOWN, st);
    hipLaunchKernelGGL((k_down<T>), dim3(grid_of<T>(a, up(a.D, T::BC), a.halves)), dim3(T::THREADS), 0, st, a);
    return launched();
}
template <typename TIO, int KIND>
bool launch_hidden(const ExpertArgs& a, hipStream_t st) {
    typedef typename TileOf<TIO, BY_ROWS, BY_ROWS, KIND>::type H;
    typedef typename TileOf<TIO, BY_COLS, BY_ROWS, KIND, true>::type T;
    ProfScope ps(KID_EXPERTS_HIDDEN_GRAD, st);
    hipLaunchKernelGGL((k_hidden_grad<H, T>), dim3(grid_of<T>(a, up(a.F, T::BC))), dim3(T::THREADS), 0, st, a);
    return launched();
}
template <typename TIO, int KIND>
bool launch_dx(const ExpertArgs& a, hipStream_t st) {
    typedef typename TileOf<TIO, BY_COLS, BY_ROWS, KIND, false, false, false, true>::type T;
    ProfScope ps(KID_EXPERTS_DX, st);
    hipLaunchKernelGGL((k_dx<T>), dim3(grid_of<T>(a, up(a.D, T::BC), a.halves)), dim3(T::THREADS), 0, st, a);
    return launched();
}
template <typename TIO, int KIND, bool DOWN>
bool launch_dw(const ExpertArgs& a, hipStream_t st) {
    typedef typename TileOf<TIO, BY_COLS, BY_COLS, KIND, false, !DOWN, DOWN>::type T;
    const int rt = up(DOWN ? a.D : 2 * a.F, T::BR), ct = up(DOWN ? a.F : a.D, T::BC);
    ProfScope ps(KID_EXPERTS_DW, st);
    hipLaunchKernelGGL((k_dw<T, DOWN>), dim3(unsigned((int64_t(a.E) * rt * ct + 7) / 8 * 8)), dim3(T::THREADS), 0, st, a, rt, ct);
    return launched();
}

template <typename TIO>
bool launch(const lsm_experts_params& p, ExpertArgs a, bool backward, hipStream_t st) {
    const Plan q = plan_of(p);
    a.parts = weight_parts(p, q.hidden);
#define LSM_UP(K) launch_up<TIO, K>(a, st)
#define LSM_DOWN(K) launch_down<TIO, K>(a, st)
#define LSM_HIDDEN(K) launch_hidden<TIO, K>(a, st)
#define LSM_DX(K) launch_dx<TIO, K>(a, st)
    if (!backward) return LSM_KIND(LSM_UP, q.up) && LSM_KIND(LSM_DOWN, q.down) && launch_sum<TIO, true>(a, st);
    if (!(LSM_KIND(LSM_HIDDEN, q.hidden) && LSM_KIND(LSM_DX, q.dx) && launch_sum<TIO, false>(a, st))) return false;
    if (!a.d_w_down) return true;
    return (q.dw1 == 0 ? launch_dw<TIO, 0, false>(a, st) : q.dw1 == 2 ? launch_dw<TIO, 2, false>(a, st) : launch_dw<TIO, 5, false>(a, st)) &&
           (q.dw2 == 0 ? launch_dw<TIO, 0, true>(a, st) : q.dw2 == 2 ? launch_dw<TIO, 2, true>(a, st) : launch_dw<TIO, 5, true>(a, st));
#undef LSM_UP
#undef LSM_DOWN
#undef LSM_HIDDEN
#undef LSM_DX
}

}  // namespace
}  // namespace lsm

extern "C" {

size_t lsm_moe_experts_workspace_bytes(const lsm_experts_params* p) {
    using namespace lsm;
    return check(p, false) == LSM_OK ? space(*p, false).bytes : 0;
}
size_t lsm_moe_experts_bwd_workspace_bytes(const lsm_experts_params* p) {
    using namespace lsm;
    return check(p, true) == LSM_OK ? space(*p, true).bytes : 0;
}

int lsm_moe_experts(const lsm_experts_params* p, const void* x, const float* weights, const int32_t* offsets, const int32_t* order,
                    const int32_t* place, const void* w_gate_up, const void* w_down, const void* residual, void* y,
                    void* workspace, size_t workspace_bytes, void* stream) {
    using namespace lsm;
    const int rc = check(p, false);
    if (rc != LSM_OK) return rc;
    if (!x || !weights || !offsets || !order || !place || !w_gate_up || !w_down || !y) return LSM_ERR_NULL;
    for (const void* q : {x, static_cast<const void*>(weights), static_cast<const void*>(offsets), static_cast<const void*>(order),
                          static_cast<const void*>(place), w_gate_up, w_down, residual, static_cast<const void*>(y), static_cast<const void*>(workspace)})
        if (misaligned(q)) return LSM_ERR_ALIGN;
    const Space s = space(*p, false);
    if (!workspace || workspace_bytes < s.bytes) return LSM_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    const uint32_t el = p->dtype == LSM_DTYPE_BF16 ? 2 : 4;
    ExpertArgs a{};
    a.x = x; a.w_gate_up = w_gate_up; a.w_down = w_down; a.residual = residual; a.weights = weights;
    a.offsets = offsets; a.order = order; a.place = place; a.y = y;
    a.h = ws + s.h; a.part = reinterpret_cast<float*>(ws + s.part);
    a.n = p->n; a.D = p->D; a.F = p->F; a.E = p->E; a.top_k = p->top_k; a.halves = halves_of(*p);
    a.x_bytes = uint32_t(p->x_stride) * el;
    a.h_bytes = uint32_t(line_bytes(p->F * el));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return (el == 2 ? launch<uint16_t>(*p, a, false, st) : launch<float>(*p, a, false, st)) ? LSM_OK : LSM_ERR_LAUNCH;
}

int lsm_moe_experts_bwd(const lsm_experts_params* p, const void* x, const float* weights, const int32_t* offsets,
                        const int32_t* order, const int32_t* place, const void* w_gate_up, const void* w_down, const void* d_y,
                        void* dx, float* d_weights, void* d_w_gate_up, void* d_w_down,
                        void* workspace, size_t workspace_bytes, void* stream) {
    using namespace lsm;
    const int rc = check(p, true);
    if (rc != LSM_OK) return rc;
    if (!x || !weights || !offsets || !order || !place || !w_gate_up || !w_down || !d_y || !dx || !d_weights || !d_w_gate_up != !d_w_down)
        return LSM_ERR_NULL;
    for (const void* q : {x, static_cast<const void*>(weights), static_cast<const void*>(offsets), static_cast<const void*>(order),
                          static_cast<const void*>(place), w_gate_up, w_down, d_y, static_cast<const void*>(dx), static_cast<const void*>(d_weights),
                          static_cast<const void*>(d_w_gate_up), static_cast<const void*>(d_w_down), static_cast<const void*>(workspace)})
        if (misaligned(q)) return LSM_ERR_ALIGN;
    const Space s = space(*p, true);
    if (!workspace || workspace_bytes < s.bytes) return LSM_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    const uint32_t el = p->dtype == LSM_DTYPE_BF16 ? 2 : 4;
    ExpertArgs a{};
    a.x = x; a.w_gate_up = w_gate_up; a.w_down = w_down; a.d_y = d_y; a.weights = weights;
    a.offsets = offsets; a.order = order; a.place = place; a.y = dx; a.d_weights = d_weights;
    a.d_w_gate_up = d_w_gate_up; a.d_w_down = d_w_down;
    a.h = ws + s.h; a.part = reinterpret_cast<float*>(ws + s.part);
    a.da = ws + s.da; a.weight_part = reinterpret_cast<float*>(ws + s.weight_part);
    a.n = p->n; a.D = p->D; a.F = p->F; a.E = p->E; a.top_k = p->top_k; a.halves = halves_of(*p);
    a.x_bytes = uint32_t(p->x_stride) * el;
    a.h_bytes = uint32_t(line_bytes(p->F * el));
    a.dy_bytes = uint32_t(p->dy_stride) * el;
    a.da_bytes = uint32_t(line_bytes(2 * p->F * el));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return (el == 2 ? launch<uint16_t>(*p, a, true, st) : launch<float>(*p, a, true, st)) ? LSM_OK : LSM_ERR_LAUNCH;
}

}  // extern "C"
