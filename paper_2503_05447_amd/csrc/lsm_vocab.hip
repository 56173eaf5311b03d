// Losses over a large vocabulary without its logits (include/lsm_train.h).
//   k_teacher   a wave per token: the teacher's probabilities and their entropy, entry by entry; whether the token counts
//   (plan)      the tokens that count, in their order (lsm_route.hip, one group): everything below works on these alone
//   k_logits    a tile of x w^T: of each row the maximum, the sum of exponentials and the logits at its entries
//   k_join      a token's loss from its tiles' maxima and sums
//   k_grad      a tile of x w^T again: the logits' gradient, for a piece of the vocabulary
//   k_dw        gradient^T x for the piece, all tokens being the long axis
//   k_dx        gradient w, the piece's vocabulary being the long axis, in several shares of it, added to the pieces before
//   k_dx_join   the shares' sum
// Bound: the matrix products, three forward and backward and a fourth for the logits formed again; for few tokens the weights, read once.
// 8191 tokens of 2048 of which 5734 count, 50257 columns, bf16: logits 946 us (1.25 PFLOP/s, a plain library product of that size is
// 1.24; matrix cores busy 0.67 of the clocks), grad 1112 (1.06, 0.60: 576 MB leave through LDS), dw 994 (1.19, 0.64), dx 1174 (1.00, 0.65: 184 tiles of
// 256 x 256 for 256 compute units); join 10, dx's sum 15, the plan 13 a call.  700 tokens of 512, 32003 columns, fp32: 218, 224, 202 and 215 us,
// 103 to 113 TFLOP/s (busy 0.77 to 0.79).  Three tokens of 1024, 50257 columns: 22 us, 4.7 TB/s; backward 22, 33 and 20 us.  4096 tokens of 1024
// with a teacher's 64 entries, 32000 columns: 260, 271, 206 and 206 us.
// The logits' gradient is formed a piece of the vocabulary at a time, so that workspaces do not grow with it; that pieces of 256 MB fit the
// memory-side cache makes no difference (512 MB and 1 GB: within 1 %).
#include "lsm_product_dev.h"

namespace lsm {
namespace {

constexpr int kMostEntries = 256, kGroup = 512;

// dx of a piece: rows of a tile, in how many shares its columns are taken with all tokens, the most it is worth taking them in
struct Shares { int rows, least, most; };
constexpr int kPieceKinds = 2;  // whole pieces, what is left

struct VocabArgs {
    const void *x, *w;
    const int32_t *index, *offsets, *order, *place;
    const float *teacher, *lse_in, *d_loss;
    int32_t *count, *entry;   // [n] 0: counts, -1: not; [K][n] tokens
    float *share, *entropy;   // [K][n] probabilities; [n]
    uint16_t* begin;          // [groups + 1][n] how many of a token's entries are below kGroup g
    f32x2* stats;             // [parts][n] maximum, sum
    float* at_entry;          // [max(K, 1)][n] logits
    float *loss, *lse;
    void *grad, *dx, *dw;     // gradient [n][piece]
    float* part;              // [shares][tokens that count][D]
    int n, D, V, K, parts, groups;  // groups: of kGroup columns
    int v0, width, piece;     // the piece: its first column, how many, and how many the gradient's rows hold (a multiple of 256)
    Shares here, before[kPieceKinds];  // of this piece, of the kinds of pieces that were before
    int kinds;                // of them
    int halves;               // rows of a token in grad: 2 where a remainder follows what was rounded
    uint32_t x_bytes;
    float scale;              // 1 / temperature
};

__device__ __forceinline__ int rows_of(const VocabArgs& a) { return uniform(min(max(a.offsets[1], 0), a.n)); }
__device__ __forceinline__ uint32_t token_of(const VocabArgs& a, int at) { return min(uint32_t(a.order[at]), uint32_t(a.n - 1)); }

template <int R>  // entries a lane
__global__ __launch_bounds__(1024) void k_teacher(VocabArgs a) {
    __shared__ int entry[64 * R][17];
    __shared__ float share[64 * R][17];
    const int t0 = int(blockIdx.x) * 16, slot = threadIdx.x >> 6, t = min(t0 + slot, a.n - 1), lane = threadIdx.x & 63;
    float z[R], m = -__builtin_inff();
    int v[R];
    _Pragma("unroll") for (int i = 0; i < R; ++i) {
        const int j = 64 * i + lane;
        v[i] = -1;
        z[i] = -__builtin_inff();
        if (j < a.K) {
            v[i] = a.index[size_t(t) * a.K + j];
            z[i] = a.teacher[size_t(t) * a.K + j];
            if (z[i] != z[i] || v[i] < 0 || v[i] >= a.V) z[i] = -__builtin_inff();
            z[i] = fminf(z[i], 3.402823466e38f);
            if (z[i] == -__builtin_inff()) v[i] = -1;
        }
        m = fmaxf(m, z[i]);
    }
    for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    const bool counts = m > -__builtin_inff();
    float sum = 0.f, d[R];
    _Pragma("unroll") for (int i = 0; i < R; ++i) {
        d[i] = v[i] >= 0 ? (z[i] - m) * a.scale : -__builtin_inff();
        sum += v[i] >= 0 ? expf(d[i]) : 0.f;
    }
    sum = group_sum<64>(sum);
    const float log_sum = logf(sum);
    float entropy = 0.f, p[R];
    _Pragma("unroll") for (int i = 0; i < R; ++i) {
        p[i] = v[i] >= 0 ? expf(d[i]) / sum : 0.f;
        if (p[i] > 0.f) entropy += p[i] * (d[i] - log_sum);
        else v[i] = -1;
    }
    // Entries of the same token become one, the first of them, and the entries of a row are sorted by their token: those of a tile's columns
    // then follow one another, and where they begin is written down for every kGroup columns.  (4096 tokens, 64 entries, 32000 columns: logits 287 -> 256 us, their gradient
    // 303 -> 269, against a look through all entries in every tile; every 64 columns instead: 12 us more here.)
    int rank[R], there = 0;
    _Pragma("unroll") for (int i = 0; i < R; ++i) rank[i] = 0;
    for (int e = 0; e < a.K; ++e) {
        int w = v[0];
        _Pragma("unroll") for (int i = 1; i < R; ++i)
            if (e >= 64 * i) w = v[i];
        w = __builtin_amdgcn_readlane(w, e & 63);
        if (w < 0) continue;
        ++there;
        float more = 0.f;
        bool again = false;
        _Pragma("unroll") for (int i = 0; i < R; ++i) {
            rank[i] += w < v[i] ? 1 : 0;
            if (v[i] == w && 64 * i + lane > e) { more += p[i]; v[i] = -1; p[i] = 0.f; again = true; }
        }
        if (__ballot(again) == 0) continue;
        more = group_sum<64>(more);
        _Pragma("unroll") for (int i = 0; i < R; ++i)
            if (64 * i + lane == e) p[i] += more;
    }
    _Pragma("unroll") for (int i = 0; i < R; ++i) {
        if (64 * i + lane >= there && 64 * i + lane < a.K) {
            entry[64 * i + lane][slot] = -1;
            share[64 * i + lane][slot] = 0.f;
        }
    }
    _Pragma("unroll") for (int i = 0; i < R; ++i) {
        if (v[i] < 0) continue;
        entry[rank[i]][slot] = v[i];
        share[rank[i]][slot] = p[i];
    }
    entropy = group_sum<64>(entropy);
    if (lane == 0) {
        a.count[t] = counts ? 0 : -1;
        a.entropy[t] = entropy;
    }
    __syncthreads();
    for (int g = lane; g <= a.groups; g += 64) {
        int below = 0, above = there;  // the answer is one of below .. above
        while (below < above) {
            const int mid = (below + above) / 2;
            if (entry[mid][slot] < kGroup * g) below = mid + 1;
            else above = mid;
        }
        a.begin[size_t(g) * a.n + t] = uint16_t(below);
    }
    for (int q = threadIdx.x; q < a.K * 16; q += 1024) {  // entry by entry, the tokens of one next to each other
        const int j = q >> 4, token = t0 + (q & 15);
        if (token >= a.n) continue;
        a.entry[size_t(j) * a.n + token] = entry[j][q & 15];
        a.share[size_t(j) * a.n + token] = share[j][q & 15];
    }
}

// The entries of a wave's rows, row(j) a lane, among its `width` columns from `first` on: the four lanes of a row take every fourth; the first
// ones, and with SHARE their probabilities, are requested for all rows together.
template <int ROWS, bool SHARE>
struct Entries {
    int e[ROWS], end[ROWS], v[ROWS];
    float share[ROWS];
    __device__ __forceinline__ static size_t cell(const VocabArgs& a, int e, int token) {
        return uint32_t(e) * uint32_t(a.n) + uint32_t(token);  // (n K is at most 2^28)
    }
    __device__ __forceinline__ void load(const VocabArgs& a, const int (&tokens)[ROWS], int first, int width, int lane) {
        const size_t g0 = size_t(min(first / kGroup, a.groups)) * a.n, g1 = size_t(min((first + width + kGroup - 1) / kGroup, a.groups)) * a.n;
        _Pragma("unroll") for (int j = 0; j < ROWS; ++j) {
            e[j] = tokens[j] < 0 ? 0 : int(a.begin[g0 + tokens[j]]);
            end[j] = tokens[j] < 0 ? 0 : int(a.begin[g1 + tokens[j]]);
        }
        _Pragma("unroll") for (int j = 0; j < ROWS; ++j) {
            e[j] += lane >> 4;
            v[j] = e[j] < end[j] ? a.entry[cell(a, e[j], tokens[j])] : -1;
            share[j] = SHARE && e[j] < end[j] ? a.share[cell(a, e[j], tokens[j])] : 0.f;
        }
    }
    // found(e, column - first, probability) for those of columns first .. first + width
    template <typename Found>
    __device__ __forceinline__ void find(const VocabArgs& a, int j, int token, int first, int width, Found found) const {
        int at = e[j], column = v[j];
        float p = share[j];
        while (__ballot(at < end[j])) {
            if (at >= end[j]) continue;
            if (uint32_t(column - first) < uint32_t(width)) found(at, column - first, p);
            at += 4;
            if (at >= end[j]) continue;
            column = a.entry[cell(a, at, token)];
            if (SHARE) p = a.share[cell(a, at, token)];
        }
    }
};

// Tile number id of rt x ct: eight rows of tiles at a time, the column changing more slowly than the row among them, so that the workgroups of
// a die, whose numbers are neighbours, hold a block of about eight by four tiles.
__device__ __forceinline__ void tile_at(int id, int rt, int ct, int& r, int& c) {
    const int band = id / (8 * ct), rest = id - band * 8 * ct, rows = min(8, rt - 8 * band);
    c = rest / rows;
    r = 8 * band + rest - c * rows;
}
__device__ __forceinline__ int number_of_tile(int all, int n = 0) {  // the n-th of this workgroup; -1: none left.  A die's numbers are neighbours
    const int die = (all + 7) / 8, at = int(blockIdx.x) / 8 + n * (int(gridDim.x) / 8), id = (int(blockIdx.x) % 8) * die + at;
    return at < die && id < all ? id : -1;
}

// The logits of all tiles of the tokens that count and the vocabulary from v0 to end, one after the other: finish(t, rows, r0, c, acc) with
// the tile's first row, its number along the columns and its logits, still without their scale.
template <typename T, typename Finish>
__device__ __forceinline__ void logit_tiles(char* shared, const VocabArgs& a, int v0, int end, Finish finish) {
    typedef typename T::TIO TIO;
    const int rows = rows_of(a), rt = (rows + T::BR - 1) / T::BR, ct = (end - v0 + T::BC - 1) / T::BC;
    int id = number_of_tile(rt * ct), r, c;
    if (id < 0) return;
    tile_at(id, rt, ct, r, c);
    T t(shared);
    const auto start = [&](typename T::C& to_c, typename T::R& to_r, bool there, int r0, int c0, auto token_at) {
        const uint32_t bytes = uint32_t(a.D) * uint32_t(sizeof(TIO));
        to_r.start_rows(a.x, t.wave, t.lane, [&](int i) { return there && r0 + i < rows ? token_at(i) * a.x_bytes : kBeyond; });
        to_c.start_rows(static_cast<const TIO*>(a.w) + size_t(v0 + c0) * a.D, t.wave, t.lane,
                        [&](int q) { return there && v0 + c0 + q < end ? uint32_t(q) * bytes : kBeyond; });
    };
    start(t.c, t.r, true, r * T::BR, c * T::BC, [&](int i) { return token_of(a, r * T::BR + i); });
    for (int n = 1;; ++n) {
        int next = -1, r2 = 0, c2 = 0;
        if (T::FOLLOWED) next = number_of_tile(rt * ct, n);
        if (next >= 0) {
            tile_at(next, rt, ct, r2, c2);
            t.bring(a.order + r2 * T::BR, rows - r2 * T::BR);
        }
        f32x4 acc[T::TC][T::TR];
        clear<T>(acc);
        t.walk(acc, a.D, typename T::Nothing(), [&]() {
            start(t.c2, t.r2, next >= 0, r2 * T::BR, c2 * T::BC, [&](int i) { return min(uint32_t(t.brought(i)), uint32_t(a.n - 1)); });
        });
        finish(t, rows, r * T::BR, c, acc);
        if (next < 0) return;
        t.go_on();
        r = r2;
        c = c2;
    }
}

template <typename T, bool TEACHER>
__global__ __launch_bounds__(T::THREADS) void k_logits(VocabArgs a) {
    typedef typename T::TIO TIO;
    __shared__ __attribute__((aligned(1024))) char shared[T::LDS];
    logit_tiles<T>(shared, a, 0, a.V, [&](const T& t, int rows, int r0, int c, f32x4 (&acc)[T::TC][T::TR]) {
        const int first = c * T::BC + t.wc * T::TC * 16, mine = first + 4 * (t.lane >> 4);  // of the wave, of the lane
        const float log2_scale = a.scale * kLog2e;
        const bool edge = first + T::TC * 16 > a.V;
        int tokens[T::TR], wants[T::TR];
        _Pragma("unroll") for (int j = 0; j < T::TR; ++j) tokens[j] = r0 + t.row(j) < rows ? int(token_of(a, r0 + t.row(j))) : -1;
        _Pragma("unroll") for (int j = 0; j < T::TR; ++j) wants[j] = TEACHER || tokens[j] < 0 ? -1 : a.index[tokens[j]];
        Entries<T::TR, false> entries;
        if (TEACHER) entries.load(a, tokens, first, T::TC * 16, t.lane);
        t.settle();
        _Pragma("unroll") for (int j = 0; j < T::TR; ++j) {
            const int at = r0 + t.row(j);
            float m = -__builtin_inff(), sum = 0.f;
            _Pragma("unroll") for (int i = 0; i < T::TC; ++i)
                _Pragma("unroll") for (int q = 0; q < 4; ++q) {
                    if (edge && mine + i * 16 + q >= a.V) acc[i][j][q] = -__builtin_inff();
                    m = fmaxf(m, acc[i][j][q]);
                }
            m = T::row_max(m);  // of the logits without their scale, which is positive
            const float top = m == -__builtin_inff() ? 0.f : m * log2_scale;
            _Pragma("unroll") for (int i = 0; i < T::TC; ++i)
                _Pragma("unroll") for (int q = 0; q < 4; ++q) sum += power(__builtin_fmaf(acc[i][j][q], log2_scale, -top), TIO());
            sum = T::row_sum(sum);
            if (t.lane < 16 && at < rows) a.stats[size_t(c * T::WC + t.wc) * a.n + at] = f32x2{m * a.scale, sum};
            if (!TEACHER) {
                const int want = wants[j];
                if (__ballot(uint32_t(want - first) < uint32_t(T::TC * 16)) == 0) continue;
                _Pragma("unroll") for (int i = 0; i < T::TC; ++i)
                    _Pragma("unroll") for (int q = 0; q < 4; ++q)
                        if (want == mine + i * 16 + q) a.at_entry[at] = acc[i][j][q] * a.scale;
            } else {
                constexpr int N = T::CHUNK;
                _Pragma("unroll") for (int i0 = 0; i0 < T::TC; i0 += N) {
                    t.template put<N>([&](int i) { return acc[i0 + i][j]; });
                    entries.find(a, j, tokens[j], first + i0 * 16, N * 16, [&](int e, int d, float) {
                        a.at_entry[size_t(e) * a.n + at] =
                            a.scale * *reinterpret_cast<__attribute__((address_space(3))) const float*>(uintptr_t(t.template cell<N>(t.lane & 15, d)));
                    });
                }
            }
        }
    });
}

// TOKENS tokens by a workgroup, every SLICES-th part (and entry) by a thread: 64 of them where tokens are many, four where a token's parts
// are what there is to do (three tokens, 788 parts: 24 us by 64, 7 by four).
template <int TOKENS, typename Join>
__device__ __forceinline__ float join(float (&all)[1024], float x, Join with) {
    constexpr int SLICES = 1024 / TOKENS;
    __syncthreads();
    all[threadIdx.x] = x;
    _Pragma("unroll") for (int half = SLICES / 2; half > 0; half /= 2) {
        __syncthreads();
        if (int(threadIdx.x) < half * TOKENS) all[threadIdx.x] = with(all[threadIdx.x], all[threadIdx.x + half * TOKENS]);
    }
    __syncthreads();
    return all[threadIdx.x % TOKENS];
}
template <int TOKENS>
__global__ __launch_bounds__(1024) void k_join(VocabArgs a) {
    __shared__ float all[1024];
    constexpr int SLICES = 1024 / TOKENS, U = 4;
    const auto larger = [](float x, float y) { return fmaxf(x, y); };
    const auto add = [](float x, float y) { return x + y; };
    const int slice = threadIdx.x / TOKENS, token = int(blockIdx.x) * TOKENS + int(threadIdx.x) % TOKENS;
    const int at = token < a.n ? a.place[token] : -1;
    float m = -__builtin_inff(), s = 0.f;
    if (at >= 0 && at < a.n)
        for (int p0 = slice; p0 < a.parts; p0 += U * SLICES) {  // a running maximum and sum, U parts at a time
            f32x2 v[U];
            float top = m;
            _Pragma("unroll") for (int u = 0; u < U; ++u) {
                v[u] = p0 + u * SLICES < a.parts ? a.stats[size_t(p0 + u * SLICES) * a.n + at] : f32x2{-__builtin_inff(), 0.f};
                top = fmaxf(top, v[u].x);
            }
            const float base = top == -__builtin_inff() ? 0.f : top;
            s *= expf(m - base);
            _Pragma("unroll") for (int u = 0; u < U; ++u) s += v[u].y * expf(v[u].x - base);
            m = top;
        }
    const float top = join<TOKENS>(all, m, larger), base = top == -__builtin_inff() ? 0.f : top;
    const float lse = base + logf(join<TOKENS>(all, m == -__builtin_inff() ? s : s * expf(m - base), add));
    float part = 0.f;
    if (a.K > 0 && at >= 0)
        for (int e = slice; e < a.K; e += SLICES) {
            const float p = a.share[size_t(e) * a.n + token];
            if (p > 0.f) part += p * (lse - a.at_entry[size_t(e) * a.n + at]);
        }
    if (a.K > 0) part = join<TOKENS>(all, part, add);
    if (slice != 0 || token >= a.n) return;
    a.loss[token] = at < 0 ? 0.f : a.K > 0 ? a.entropy[token] + part : lse - a.at_entry[at];
    a.lse[token] = at < 0 ? 0.f : lse;
}

template <typename T, bool TEACHER>
__global__ __launch_bounds__(T::THREADS) void k_grad(VocabArgs a) {
    typedef typename T::TIO TIO;
    __shared__ __attribute__((aligned(1024))) char shared[T::LDS];
    const int end = a.v0 + a.width;
    logit_tiles<T>(shared, a, a.v0, end, [&](const T& t, int rows, int r0, int c, f32x4 (&acc)[T::TC][T::TR]) {
        const int column = c * T::BC + t.wc * T::TC * 16, first = a.v0 + column, mine = first + 4 * (t.lane >> 4);
        const float log2_scale = a.scale * kLog2e;
        const bool edge = first + T::TC * 16 > end;
        int tokens[T::TR], wants[T::TR];
        float tops[T::TR], weights[T::TR];
        _Pragma("unroll") for (int j = 0; j < T::TR; ++j) tokens[j] = r0 + t.row(j) < rows ? int(token_of(a, r0 + t.row(j))) : -1;
        _Pragma("unroll") for (int j = 0; j < T::TR; ++j) {
            wants[j] = TEACHER || tokens[j] < 0 ? -1 : a.index[tokens[j]];
            tops[j] = tokens[j] < 0 ? 0.f : a.lse_in[tokens[j]] * kLog2e;
            weights[j] = tokens[j] < 0 ? 0.f : a.d_loss[tokens[j]] * a.scale;
        }
        Entries<T::TR, true> entries;
        if (TEACHER) entries.load(a, tokens, first, T::TC * 16, t.lane);
        t.settle();
        _Pragma("unroll") for (int j = 0; j < T::TR; ++j) {
            const int want = wants[j];
            const float top = tops[j], weight = weights[j];
            const bool here = !TEACHER && __ballot(uint32_t(want - first) < uint32_t(T::TC * 16)) != 0;
            constexpr int N = T::CHUNK;
            _Pragma("unroll") for (int i0 = 0; i0 < T::TC; i0 += N) {
                t.template put<N>([&](int i) {
                    f32x4 v;
                    _Pragma("unroll") for (int e = 0; e < 4; ++e) {
                        const int col = mine + (i0 + i) * 16 + e;
                        float p = power(__builtin_fmaf(acc[i0 + i][j][e], log2_scale, -top), TIO());
                        if (here && col == want) p -= 1.f;
                        v[e] = edge && col >= end ? 0.f : weight * p;
                    }
                    return v;
                });
                if (TEACHER) {
                    entries.find(a, j, tokens[j], first + i0 * 16, N * 16, [&](int, int d, float p) {  // no two entries of a row are the same
                        auto* at = reinterpret_cast<__attribute__((address_space(3))) float*>(uintptr_t(t.template cell<N>(t.lane & 15, d)));
                        *at = *at - weight * p;
                    });
                }
                // the columns behind the vocabulary's end are zeros that the next products read
                const int halves = kMayHalve<T> ? a.halves : 1;
                const auto line = [&](int half) {
                    return [=](int q) {
                        return r0 + q < rows ? static_cast<TIO*>(a.grad) + size_t((r0 + q) * halves + half) * a.piece + column + i0 * 16 : nullptr;
                    };
                };
                t.template take<N, TIO>(j, a.piece - column - i0 * 16, line(0));
                if constexpr (kMayHalve<T>)
                    if (halves == 2) t.template take<N, TIO, false, true>(j, a.piece - column - i0 * 16, line(1));
            }
        }
    });
}

template <typename T>
__global__ __launch_bounds__(T::THREADS) void k_dw(VocabArgs a) {
    typedef typename T::TIO TIO;
    constexpr int EL = int(sizeof(TIO));
    __shared__ __attribute__((aligned(1024))) char shared[T::LDS];
    const int width = a.width, rows = rows_of(a);
    const int rt = (width + T::BR - 1) / T::BR, ct = (a.D + T::BC - 1) / T::BC, id = number_of_tile(rt * ct);
    if (id < 0) return;
    int r, c;
    tile_at(id, rt, ct, r, c);
    T t(shared);
    t.r.start_cols(a.grad, a.piece * EL, r * T::BR, a.piece, t.wave, t.lane, 0);
    t.c.start_cols(a.x, int(a.x_bytes), c * T::BC, a.D, t.wave, t.lane, t.list_at());
    f32x4 acc[T::TC][T::TR];
    clear<T>(acc);
    t.walk(acc, rows * a.halves, [&](int k) { return token_of(a, k >> (a.halves - 1)); });
    const int c0 = c * T::BC + t.wc * T::TC * 16;
    _Pragma("unroll") for (int j = 0; j < T::TR; ++j) {
        t.template store<T::TC, TIO>(j, a.D - c0, [&](int i) { return acc[i][j]; }, [&](int q) {
            const int v = r * T::BR + q;
            return v < width ? static_cast<TIO*>(a.dw) + size_t(a.v0 + v) * a.D + c0 : nullptr;
        });
    }
}

// In how many shares a piece's columns are taken: where few of the tokens count, as many times more as workgroups would have nothing to do
// (8191 tokens, 50257 x 2048, 60 % of them left out: dx 1118 -> 705 us).
__device__ __forceinline__ int shares_of(const Shares& s, int n, int rows) {
    const int all = (n + s.rows - 1) / s.rows, there = max((rows + s.rows - 1) / s.rows, 1);
    return max(s.least, min(s.most, int(int64_t(s.least) * all / there)));
}
__device__ __forceinline__ int shares_before(const VocabArgs& a, int rows) {  // so many have a sum
    int most = 0;
    _Pragma("unroll") for (int i = 0; i < kPieceKinds; ++i)
        if (i < a.kinds) most = max(most, shares_of(a.before[i], a.n, rows));
    return most;
}

template <typename T>
__global__ __launch_bounds__(T::THREADS) void k_dx(VocabArgs a) {
    typedef typename T::TIO TIO;
    constexpr int EL = int(sizeof(TIO)), STEP = kStepBytes / EL;
    __shared__ __attribute__((aligned(1024))) char shared[T::LDS];
    const int width = a.width, tokens = rows_of(a), halves = kMayHalve<T> ? a.halves : 1, rows = tokens * halves;
    const int rt = (rows + T::BR - 1) / T::BR, ct = (a.D + T::BC - 1) / T::BC, shares = shares_of(a.here, a.n, tokens), id = number_of_tile(rt * ct * shares);
    if (id < 0) return;
    const int share = id / (rt * ct);
    int r, c;
    tile_at(id - share * rt * ct, rt, ct, r, c);
    const int steps = (width + STEP - 1) / STEP, k0 = steps * share / shares * STEP, k1 = min(width, steps * (share + 1) / shares * STEP);
    const int r0 = r * T::BR, begun = shares_before(a, tokens);
    const uint32_t bytes = uint32_t(a.piece) * EL;
    T t(shared);
    t.r.start_rows(static_cast<const TIO*>(a.grad) + size_t(r0) * a.piece + k0, t.wave, t.lane,
                   [&](int i) { return r0 + i < rows ? uint32_t(i) * bytes : kBeyond; });
    t.c.start_cols(static_cast<const TIO*>(a.w) + size_t(a.v0 + k0) * a.D, a.D * EL, c * T::BC, a.D, t.wave, t.lane, 0);
    f32x4 acc[T::TC][T::TR];
    clear<T>(acc);
    t.walk(acc, k1 - k0);
    const int c0 = c * T::BC + t.wc * T::TC * 16;
    if constexpr (kMayHalve<T>)
        if (halves == 2)  // both rows of a token, in neighbouring lanes
            _Pragma("unroll") for (int i = 0; i < T::TC; ++i)
                _Pragma("unroll") for (int j = 0; j < T::TR; ++j)
                    _Pragma("unroll") for (int e = 0; e < 4; ++e) acc[i][j][e] += dpp<0xB1>(acc[i][j][e]);
    const auto line = [&](int q) {
        const int at = r0 + q;
        return at < rows && (at & (halves - 1)) == 0 ? a.part + (size_t(share) * tokens + (at >> (halves - 1))) * a.D + c0 : nullptr;
    };
    _Pragma("unroll") for (int j = 0; j < T::TR; ++j) {
        if (share >= begun) t.template store<T::TC, float>(j, a.D - c0, [&](int i) { return acc[i][j]; }, line);
        else t.template store<T::TC, float, true>(j, a.D - c0, [&](int i) { return acc[i][j]; }, line);
    }
}

template <typename TIO>
__global__ __launch_bounds__(256) void k_dx_join(VocabArgs a) {
    constexpr int E = kPiece<TIO>;
    const int pieces = a.D / E;
    const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (id >= int64_t(a.n) * pieces) return;
    const int token = int(id / pieces), d = int(id - int64_t(token) * pieces) * E, at = a.place[token];
    float s[E];
    _Pragma("unroll") for (int e = 0; e < E; ++e) s[e] = 0.f;
    const int rows = rows_of(a), begun = shares_before(a, rows);
    if (at >= 0 && at < rows)
        for (int q = 0; q < begun; ++q) {
            const f32x4* z = reinterpret_cast<const f32x4*>(a.part + (size_t(q) * rows + at) * a.D + d);
            _Pragma("unroll") for (int i = 0; i < E / 4; ++i)
                _Pragma("unroll") for (int e = 0; e < 4; ++e) s[4 * i + e] += z[i][e];
        }
    *reinterpret_cast<u32x4*>(static_cast<TIO*>(a.dx) + size_t(token) * a.D + d) = pack(s);
}

// ---- host ------------------------------------------------------------------------------------------------------------
constexpr int64_t kPieceBytes = int64_t(256) << 20;  // of the logits' gradient at a time: what the memory-side cache holds

struct Pieces;
bool fits(const lsm_vocab_params& p, Pieces* backward);
int check(const lsm_vocab_params* p, Pieces* backward) {  // backward: where its pieces go, null for the forward call
    if (!p) return LSM_ERR_NULL;
    if (p->struct_size != sizeof(lsm_vocab_params)) return LSM_ERR_SHAPE;
    if (p->n < 1 || p->D < 1 || p->V < 1 || p->K < 0 || p->n > kMostPairs || p->V > (1 << 24)) return LSM_ERR_SHAPE;
    if (int64_t(p->n) * p->K > (1 << 28)) return LSM_ERR_SHAPE;
    if (!(p->temperature > 0.f) || !(1.f / p->temperature * kLog2e < 3.4e38f) || !(1.f / p->temperature > 0.f)) return LSM_ERR_SHAPE;  // (the kernels' own scale)
    if (p->dtype != LSM_DTYPE_F32 && p->dtype != LSM_DTYPE_BF16) return LSM_ERR_UNSUPPORTED;
    if (p->K > kMostEntries || p->D % 8 || p->D > 65536 || p->reserved != 0) return LSM_ERR_UNSUPPORTED;
    const int64_t el = p->dtype == LSM_DTYPE_BF16 ? 2 : 4;
    if (p->x_stride < p->D || p->x_stride > (int64_t(1) << 31) || p->n * p->x_stride * el >= int64_t(kBeyond)) return LSM_ERR_SHAPE;
    if (p->x_stride % 8) return LSM_ERR_ALIGN;
    return fits(*p, backward) ? LSM_OK : LSM_ERR_SHAPE;
}
int logits_tile(const lsm_vocab_params& p) {
    const bool f32 = p.dtype == LSM_DTYPE_F32;
    return pick_tile(f32, p.D, [&](const TileSize& t) { return int64_t(up(p.n, t.rows)) * up(p.V, t.cols); }, f32 ? 0x7e : 0x7f);
}
// In calls of up to 16 tokens the rounding of the logits' gradient is kept as a row of its own behind it: the rows are still one tile, the
// products take no longer (three tokens, 50257 x 1024, backward: 91 -> 92 us), and with bf16 elements the results' rounding is the only one that counts
// (without: errors of 1.41 times it, and up to twice where a result hangs on one number, as those of a single token or a target that no other token
// has).  With more tokens the products that take the second rows would be twice as long; how many of the tokens count is not known here.
int halves_of(const lsm_vocab_params& p) { return p.dtype == LSM_DTYPE_BF16 && p.n <= 16 ? 2 : 1; }

// A piece of the vocabulary backward: how many columns, the tiles of the logits' gradient, of dw and dx, into how many shares dx takes the piece.
struct Piece { int width, grad, dw, dx, shares; int64_t tiles, rows; };  // tiles: the most of its launches; rows: of sums for dx
Piece piece_of(const lsm_vocab_params& p, int width) {
    const bool f32 = p.dtype == LSM_DTYPE_F32;
    const unsigned kinds = halves_of(p) == 2 ? 0x78 : f32 ? 0x7e : 0x7f;
    Piece q{};
    q.width = width;
    q.grad = pick_tile(f32, p.D, [&](const TileSize& t) { return int64_t(up(p.n, t.rows)) * up(q.width, t.cols); }, kinds);
    q.dw = pick_tile(f32, p.n, [&](const TileSize& t) { return int64_t(up(q.width, t.rows)) * up(p.D, t.cols); },
                     (f32 ? 0 : 1 << 0) | 1 << 2 | 1 << 5);
    // the fewest shares with which the last round of workgroups is nine tenths full, or the best of some
    const auto shares = [&](const TileSize& t) {
        const int64_t n = int64_t(up(p.n, t.rows)) * up(p.D, t.cols), room = 256 * t.at_once;
        double best = 0;
        int least = 1;
        for (int k = 1; k <= 64 && k * 512 <= q.width + 511; ++k) {
            const double full = double(n * k) / (double(up(n * k, room)) * room);
            if (full > best + 0.02) { best = full; least = k; }
            if (best >= 0.9 || (k >= 8 && n * k >= room)) break;
        }
        return least;
    };
    q.dx = pick_tile_of(f32, [&](const TileSize& t) { return int64_t(up(p.n, t.rows)) * up(p.D, t.cols) * shares(t); },
                        [&](const TileSize& t) { return up(q.width, shares(t)); }, kinds);
    q.shares = shares(kTiles[q.dx]);
    const auto tiles_of = [](int rows, int cols, int kind) { return int64_t(up(rows, kTiles[kind].rows)) * up(cols, kTiles[kind].cols); };
    q.rows = int64_t(q.shares) * up(p.n, kTiles[q.dx].rows) * kTiles[q.dx].rows;
    for (const int64_t n : {tiles_of(p.n, q.width, q.grad), tiles_of(q.width, p.D, q.dw), tiles_of(p.n, p.D, q.dx) * q.shares})
        if (n > q.tiles) q.tiles = n;
    return q;
}
// The pieces of a call: `count` whole ones and what is left of the vocabulary, one column at least.
// dw's products are as long as there are tokens, so that a last round of a few tiles takes as long as a full one: a whole piece ends with a
// full round where less than half of the next one would be left (8191 tokens, 50257 x 1032, 64 columns of tiles at a time against 51: 3640 -> 3080 us
// backward; 12000 tokens, 50257 x 2048, 43 against 32: 7580 -> 6970).  What fits into one piece stays one: another piece costs three launches and another
// pass over dx's sums (3 tokens, 50257 x 1024, 192 and 5 columns of tiles against 197: 109 -> 92 us; 2048 tokens, 50257 x 2048: 1205 -> 1135; 6000
// tokens, 33000 x 2048, 87, 32 and 10 against 87 and 42: 2365 -> 2300).
struct Pieces { Piece whole, last; int count; };
Pieces pieces_of(const lsm_vocab_params& p) {
    const bool f32 = p.dtype == LSM_DTYPE_F32;
    int64_t most = kPieceBytes / (int64_t(p.n) * (f32 ? 4 : 2)) / 256;  // in tiles of 256 columns
    if (most < 1) most = 1;
    const int64_t tiles = up(p.V, 256), round = 256 / up(p.D, 256), over = most % (round ? round : 1);
    const int64_t whole = !f32 && round > 1 && most > round && 2 * over < round ? most - over : most;
    Pieces q{};
    q.count = tiles > most ? up(tiles - most, whole) : 0;
    if (q.count) q.whole = piece_of(p, int(whole * 256));
    q.last = piece_of(p, int(p.V - q.count * whole * 256));
    return q;
}
// The most of any piece: columns (whole tiles), tiles, rows of sums.
Piece largest_of(const Pieces& all) {
    Piece most{};
    for (const Piece& q : {all.whole, all.last}) {
        if (up(q.width, 256) * 256 > most.width) most.width = up(q.width, 256) * 256;
        if (q.rows > most.rows) most.rows = q.rows;
        if (q.tiles > most.tiles) most.tiles = q.tiles;
    }
    return most;
}
bool fits(const lsm_vocab_params& p, Pieces* backward) {
    if (backward) return largest_of(*backward = pieces_of(p)).tiles < kMostTiles;
    const TileSize& t = kTiles[logits_tile(p)];
    return int64_t(up(p.n, t.rows)) * up(p.V, t.cols) < kMostTiles;
}
int parts_of(const lsm_vocab_params& p, int kind) { return up(p.V, kTiles[kind].cols) * kTiles[kind].waves; }

int groups_of(const lsm_vocab_params& p) { return up(p.V, kGroup); }

struct Space { size_t offsets, order, place, hist, count, entry, share, begin, entropy, stats, at_entry, grad, part, bytes; };
Space space(const lsm_vocab_params& p, const Pieces* backward) {
    const size_t n = p.n, el = p.dtype == LSM_DTYPE_BF16 ? 2 : 4, K = p.K;
    Space s{};
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t here = at; at += align256(bytes); return here; };
    s.offsets = take(8);
    s.order = take(n * 4);
    s.place = take(n * 4);
    s.hist = take(plan_space(p.n, 1));
    s.count = take(K ? n * 4 : 0);
    s.entry = take(K * n * 4);
    s.share = take(K * n * 4);
    s.begin = take(K ? (size_t(groups_of(p)) + 1) * n * 2 : 0);
    s.entropy = take(K ? n * 4 : 0);
    if (!backward) {
        s.stats = take(size_t(parts_of(p, logits_tile(p))) * n * sizeof(f32x2));
        s.at_entry = take((K ? K : 1) * n * 4);
    } else {
        const Piece q = largest_of(*backward);
        s.grad = take(n * halves_of(p) * q.width * el);
        s.part = take(size_t(q.rows) * p.D * 4);
    }
    s.bytes = at;
    return s;
}

VocabArgs arguments(const lsm_vocab_params& p, const Space& s, char* ws, const void* x, const void* w, const int32_t* index, const float* teacher) {
    VocabArgs a{};
    a.x = x; a.w = w; a.index = index; a.teacher = teacher;
    a.offsets = reinterpret_cast<int32_t*>(ws + s.offsets);
    a.order = reinterpret_cast<int32_t*>(ws + s.order);
    a.place = reinterpret_cast<int32_t*>(ws + s.place);
    a.count = reinterpret_cast<int32_t*>(ws + s.count);
    a.entry = reinterpret_cast<int32_t*>(ws + s.entry);
    a.share = reinterpret_cast<float*>(ws + s.share);
    a.begin = reinterpret_cast<uint16_t*>(ws + s.begin);
    a.entropy = reinterpret_cast<float*>(ws + s.entropy);
    a.stats = reinterpret_cast<f32x2*>(ws + s.stats);
    a.at_entry = reinterpret_cast<float*>(ws + s.at_entry);
    a.grad = ws + s.grad;
    a.part = reinterpret_cast<float*>(ws + s.part);
    a.n = p.n; a.D = p.D; a.V = p.V; a.K = p.K; a.groups = groups_of(p);
    a.halves = halves_of(p);
    a.x_bytes = uint32_t(p.x_stride) * (p.dtype == LSM_DTYPE_BF16 ? 2 : 4);
    a.scale = 1.f / p.temperature;
    return a;
}
// The tokens that count.
bool enqueue_rows(const VocabArgs& a, const Space& s, char* ws, hipStream_t st) {
    if (a.K > 0) {
        ProfScope ps(KID_VOCAB_ROWS, st);
        if (a.K <= 64) hipLaunchKernelGGL(k_teacher<1>, dim3(up(a.n, 16)), dim3(1024), 0, st, a);
        else hipLaunchKernelGGL(k_teacher<4>, dim3(up(a.n, 16)), dim3(1024), 0, st, a);
        if (!launched()) return false;
    }
    return enqueue_plan(a.K ? a.count : a.index, a.n, 1, a.K ? 1 : a.V, reinterpret_cast<int32_t*>(ws + s.offsets),
                        reinterpret_cast<int32_t*>(ws + s.order), reinterpret_cast<int32_t*>(ws + s.place),
                        reinterpret_cast<int32_t*>(ws + s.hist), st);
}
template <typename T>
unsigned grid_of(int64_t tiles) {
    const unsigned all = unsigned((tiles + 7) / 8 * 8);
    return T::FOLLOWED && all > 256 ? 256 : all;  // one for each compute unit
}

template <typename TIO, int KIND>
bool launch_logits(const VocabArgs& a, hipStream_t st) {
    typedef typename TileOf<TIO, BY_ROWS, BY_ROWS, KIND, false, false, false, true>::type T;
    typedef typename TileOf<TIO, BY_ROWS, BY_ROWS, KIND>::type TT;  // with a teacher: followed, its tiles take as long
    ProfScope ps(KID_VOCAB_LOGITS, st);
    const int64_t tiles = int64_t(up(a.n, T::BR)) * up(a.V, T::BC);
    if (a.K) hipLaunchKernelGGL((k_logits<TT, true>), dim3(grid_of<TT>(tiles)), dim3(T::THREADS), 0, st, a);
    else hipLaunchKernelGGL((k_logits<T, false>), dim3(grid_of<T>(tiles)), dim3(T::THREADS), 0, st, a);
    return launched();
}
template <typename TIO, int KIND>
bool launch_grad(const VocabArgs& a, int width, hipStream_t st) {
    typedef typename TileOf<TIO, BY_ROWS, BY_ROWS, KIND, false, false, false, true>::type T;
    typedef typename TileOf<TIO, BY_ROWS, BY_ROWS, KIND>::type TT;  // followed: as long, and k_dw and k_dx behind it 202 -> 209 us each
    ProfScope ps(KID_VOCAB_GRAD, st);
    const int64_t tiles = int64_t(up(a.n, T::BR)) * up(width, T::BC);
    if (a.K) hipLaunchKernelGGL((k_grad<TT, true>), dim3(grid_of<TT>(tiles)), dim3(T::THREADS), 0, st, a);
    else hipLaunchKernelGGL((k_grad<T, false>), dim3(grid_of<T>(tiles)), dim3(T::THREADS), 0, st, a);
    return launched();
}
template <typename TIO, int KIND>
bool launch_dw(const VocabArgs& a, int width, hipStream_t st) {
    typedef typename TileOf<TIO, BY_COLS, BY_COLS, KIND, false, true>::type T;
    ProfScope ps(KID_VOCAB_DW, st);
    hipLaunchKernelGGL((k_dw<T>), dim3(grid_of<T>(int64_t(up(width, T::BR)) * up(a.D, T::BC))), dim3(T::THREADS), 0, st, a);
    return launched();
}
template <typename TIO, int KIND>
bool launch_dx(const VocabArgs& a, hipStream_t st) {
    typedef typename TileOf<TIO, BY_COLS, BY_ROWS, KIND>::type T;
    ProfScope ps(KID_VOCAB_DX, st);
    hipLaunchKernelGGL((k_dx<T>), dim3(grid_of<T>(int64_t(up(a.n, T::BR)) * up(a.D, T::BC) * a.here.least)), dim3(T::THREADS), 0, st, a);
    return launched();
}

template <typename TIO>
bool launch(VocabArgs a, const lsm_vocab_params& p, const Pieces* backward, hipStream_t st) {
#define LSM_LOGITS(K) launch_logits<TIO, K>(a, st)
#define LSM_GRAD(K) launch_grad<TIO, K>(a, q.width, st)
#define LSM_DX(K) launch_dx<TIO, K>(a, st)
    if (!backward) {
        const int kind = logits_tile(p);
        a.parts = parts_of(p, kind);
        if (!LSM_KIND(LSM_LOGITS, kind)) return false;
        ProfScope ps(KID_VOCAB_JOIN, st);
        if (a.n > 1024) hipLaunchKernelGGL(k_join<64>, dim3(up(a.n, 64)), dim3(1024), 0, st, a);
        else hipLaunchKernelGGL(k_join<4>, dim3(up(a.n, 4)), dim3(1024), 0, st, a);
        return launched();
    }
    for (int i = 0; i <= backward->count; ++i) {
        const Piece& q = i < backward->count ? backward->whole : backward->last;
        a.width = q.width;
        a.piece = up(q.width, 256) * 256;
        a.here = Shares{kTiles[q.dx].rows, q.shares, q.width / 512};
        if (!LSM_KIND(LSM_GRAD, q.grad)) return false;
        if (a.dw && !(q.dw == 0 ? launch_dw<TIO, 0>(a, q.width, st) : q.dw == 2 ? launch_dw<TIO, 2>(a, q.width, st) : launch_dw<TIO, 5>(a, q.width, st)))
            return false;
        if (!LSM_KIND(LSM_DX, q.dx)) return false;
        if (i == 0 || i == backward->count) a.before[a.kinds++] = a.here;
        a.v0 += q.width;
    }
    ProfScope ps(KID_VOCAB_JOIN, st);
    hipLaunchKernelGGL((k_dx_join<TIO>), dim3(up(int64_t(a.n) * (a.D / kPiece<TIO>), 256)), dim3(256), 0, st, a);
    return launched();
#undef LSM_LOGITS
#undef LSM_GRAD
#undef LSM_DX
}

}  // namespace
}  // namespace lsm

extern "C" {

size_t lsm_vocab_loss_workspace_bytes(const lsm_vocab_params* p) {
    using namespace lsm;
    return check(p, nullptr) == LSM_OK ? space(*p, nullptr).bytes : 0;
}
size_t lsm_vocab_loss_bwd_workspace_bytes(const lsm_vocab_params* p) {
    using namespace lsm;
    Pieces pieces;
    return check(p, &pieces) == LSM_OK ? space(*p, &pieces).bytes : 0;
}

int lsm_vocab_loss(const lsm_vocab_params* p, const void* x, const void* w, const int32_t* index, const float* teacher,
                   float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace lsm;
    const int rc = check(p, nullptr);
    if (rc != LSM_OK) return rc;
    if (!x || !w || !index || !teacher != !p->K || !loss || !lse) return LSM_ERR_NULL;
    if (misaligned(x) || misaligned(w) || misaligned(index) || misaligned(teacher) || misaligned(loss) || misaligned(lse) || misaligned(workspace))
        return LSM_ERR_ALIGN;
    const Space s = space(*p, nullptr);
    if (!workspace || workspace_bytes < s.bytes) return LSM_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    VocabArgs a = arguments(*p, s, ws, x, w, index, teacher);
    a.loss = loss;
    a.lse = lse;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (!enqueue_rows(a, s, ws, st)) return LSM_ERR_LAUNCH;
    return (p->dtype == LSM_DTYPE_BF16 ? launch<uint16_t>(a, *p, nullptr, st) : launch<float>(a, *p, nullptr, st)) ? LSM_OK : LSM_ERR_LAUNCH;
}

int lsm_vocab_loss_bwd(const lsm_vocab_params* p, const void* x, const void* w, const int32_t* index, const float* teacher,
                       const float* lse, const float* d_loss, void* dx, void* dw, void* workspace, size_t workspace_bytes,
                       void* stream) {
    using namespace lsm;
    Pieces pieces;
    const int rc = check(p, &pieces);
    if (rc != LSM_OK) return rc;
    if (!x || !w || !index || !teacher != !p->K || !lse || !d_loss || !dx) return LSM_ERR_NULL;
    if (misaligned(x) || misaligned(w) || misaligned(index) || misaligned(teacher) || misaligned(lse) || misaligned(d_loss) || misaligned(dx) ||
        misaligned(dw) || misaligned(workspace))
        return LSM_ERR_ALIGN;
    const Space s = space(*p, &pieces);
    if (!workspace || workspace_bytes < s.bytes) return LSM_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    VocabArgs a = arguments(*p, s, ws, x, w, index, teacher);
    a.lse_in = lse;
    a.d_loss = d_loss;
    a.dx = dx;
    a.dw = dw;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (!enqueue_rows(a, s, ws, st)) return LSM_ERR_LAUNCH;
    return (p->dtype == LSM_DTYPE_BF16 ? launch<uint16_t>(a, *p, &pieces, st) : launch<float>(a, *p, &pieces, st)) ? LSM_OK : LSM_ERR_LAUNCH;
}

}  // extern "C"
