// One step of a beam search: the best candidates of beams x vocabulary, and the beams' states rearranged (include/lsm_block.h).
//
// Selection is two kernels.  k_beam_slices: a workgroup reads a slice of one beam's logits once and leaves the slice's maximum, its
// sum of exponentials and its n_out + 1 best logits (value descending, token ascending).  k_beam_merge: a workgroup per sequence
// joins the slices' sums to each beam's log-normaliser, turns the kept logits into scores and takes the n_out best.  Scores fall
// with the logits of a beam, but not strictly (rounding makes equal scores of close logits), and equal scores go by token: where a
// slice's last kept score reaches the n_out-th best, dropped ones might be due, and the merge takes the candidates at exactly
// that score from the logits themselves, in order.
//
// To find the best n of what a workgroup holds without sorting it: the n-th largest of its lanes' maxima bounds the n-th best from
// below; its bits come one by one from counting the maxima above a trial value (a comparison and a population count each).  Few
// elements reach the bound; they are collected in LDS and ranked by counting.  The merge does the same with the slices' lists: the
// n-th largest of their first entries, say, is a bound.
//
// Bound, large batches: vector instructions and waiting, each in part.  Counted for 16 x 16 beams of 131071 bf16 logits, 32
// candidates: 16.6 vector instructions a logit (8 of them the exponential, the sum and the maximum) fill about two thirds of the
// kernel's cycles; a wave waits in 55 % of its own, since nothing is requested while a tile is worked on.  k_beam_slices 24.6 us
// (2.7 TB/s; the bytes alone would take 13), k_beam_merge 7.8, a workgroup a sequence: its chain of loads and barriers.  Small
// ones: the latency of two launches (one sequence of 4 beams: 6.0 and 4.6 us, the host needs 15).
// k_state_reorder: 391 us for 32 x 8 beams with 1 GiB of states, of which 1.25 GB have to move (about 220 rows of 256 change, 76 are
// some other beam's parent): 3.2 TB/s.  Not HBM: for K <= 8 a thread's loads, each under its own condition, are compiled to one
// after the other.
#include "lsm_block_dev.h"

#include <algorithm>

namespace lsm {
namespace {

typedef unsigned long long u64;

constexpr float kInf = __builtin_inff(), kLog2E = 1.44269504f;
constexpr float kLargest = 3.402823466e38f;
template <typename TIO> constexpr float kLargestOf = sizeof(TIO) == 4 ? kLargest : 3.389531390e38f;  // finite, of the logits' type
constexpr int kMaxOut = 32;      // n_out and K
constexpr int kWaveList = 512;   // a wave's candidates
constexpr int kPieces = 4;       // 16-byte pieces that a lane holds: tiles of 8192 logits, in fp32 4096

// unsigned numbers in the order of the floats (no NaN); -0 counts as 0
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ (uint32_t(int(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t o) {
    return __uint_as_float(o ^ ((o & 0x80000000u) ? 0x80000000u : 0xffffffffu));
}
constexpr uint32_t kOrderedNegInf = 0x007fffffu;
// value (or score) descending, index ascending = key descending; 0 is below every key
__device__ __forceinline__ u64 make_key(float x, uint32_t index) { return (u64(ordered(x)) << 32) | (0xffffffffu - index); }
__device__ __forceinline__ uint32_t key_index(u64 k) { return 0xffffffffu - uint32_t(k); }

__device__ __forceinline__ float sane(float x, float largest) { return x != x ? -kInf : fminf(x, largest); }
// Maximum that passes over quiet NaNs, without the compiler's canonicalisation of operands that it cannot tell from
// signalling ones (with one of those among them the result is of no use, and neither is the sum that is checked after it).
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float group_max(float x, int width) {  // of 16, 32 or 64 lanes
    x = fmaxf(x, dpp<0xB1>(x));
    x = fmaxf(x, dpp<0x4E>(x));
    x = fmaxf(x, dpp<0x141>(x));
    x = fmaxf(x, dpp<0x140>(x));
    if (width >= 32) x = fmaxf(x, __shfl_xor(x, 16, 64));
    if (width >= 64) x = fmaxf(x, __shfl_xor(x, 32, 64));
    return x;
}

// how many of a list's n keys are above x; eight are on their way at a time
__device__ __forceinline__ int rank_in(const u64* list, int n, u64 x) {
    int rank = 0, k = 0;
    for (; k + 8 <= n; k += 8) {
        u64 y[8];
        _Pragma("unroll") for (int i = 0; i < 8; ++i) y[i] = list[k + i];
        _Pragma("unroll") for (int i = 0; i < 8; ++i) rank += y[i] > x ? 1 : 0;
    }
    for (; k < n; ++k) rank += list[k] > x ? 1 : 0;
    return rank;
}

struct BeamArgs {
    const char* logits;
    const float* scores;
    const uint8_t* finished;
    float* out_scores;
    int32_t *parent, *token;
    uint8_t* out_finished;
    f32x2* sums;      // [B K][slices] maximum and sum of exponentials
    u64* kept;        // [B K][slices][n_out + 1] keys of logits, descending; 0 = none
    int64_t row_bytes;
    int rows, K, V, n_out, eos, bf16, slices, tiles, row_tiles;  // tiles of a slice and of a row
};

// The pieces of 16 bytes that a beam's logits lie in, counted from the one with its first logit; `lead` elements of that one
// come before it.  Elements that are not the beam's read as -inf, which is never kept and adds nothing to a sum.
template <typename TIO>
struct Row {
    static constexpr int E = kPiece<TIO>;
    const char* p;
    int lead, end;
    bool tail;  // so near the end of all logits that nothing may be read behind this row's last one
    __device__ __forceinline__ Row(const BeamArgs& a, int row) {
        const char* x = a.logits + row * a.row_bytes;
        lead = int(reinterpret_cast<uintptr_t>(x) & 15u) / int(sizeof(TIO));
        p = x - lead * int(sizeof(TIO));
        end = lead + a.V;
        tail = (a.rows - 1 - row) * a.row_bytes < 16;
    }
    // `at`: a piece's first element, a multiple of E
    __device__ __forceinline__ u32x4 whole(int at) const { return *reinterpret_cast<const u32x4*>(p + size_t(at) * sizeof(TIO)); }
    __device__ __forceinline__ u32x4 part(int at) const {
        constexpr uint32_t none = sizeof(TIO) == 4 ? 0xff800000u : 0xff80ff80u;
        u32x4 v = {none, none, none, none};
        if (at >= end) return v;
        if (at + E <= end || !tail) {
            v = whole(at);
        } else {
            TIO e[E];
            _Pragma("unroll") for (int i = 0; i < E; ++i) e[i] = reinterpret_cast<const TIO*>(p)[min(at + i, end - 1)];
            __builtin_memcpy(&v, e, 16);
        }
        _Pragma("unroll") for (int i = 0; i < 4; ++i) {
            if (sizeof(TIO) == 4) {
                if (at + i < lead || at + i >= end) v[i] = none;
            } else {
                const int e = at + 2 * i;
                if (e < lead || e >= end) v[i] = (v[i] & 0xffff0000u) | 0xff80u;
                if (e + 1 < lead || e + 1 >= end) v[i] = (v[i] & 0xffffu) | 0xff800000u;
            }
        }
        return v;
    }
};

// The k-th largest of the values that a wave's lanes hold, W each, or something a little below it: of fp32 the upper 16 bits do,
// unless many lanes share them (bf16 has no others).
template <typename TIO, int W>
__device__ __forceinline__ uint32_t kth_largest(const uint32_t (&v)[W], int k) {
    auto above = [&](uint32_t x) {
        int c = 0;
        _Pragma("unroll") for (int i = 0; i < W; ++i) c += lanes(__ballot(v[i] >= x));
        return c;
    };
    uint32_t bound = 0;
    _Pragma("unroll") for (int bit = 31; bit >= 16; --bit)
        if (above(bound | (1u << bit)) >= k) bound |= 1u << bit;
    if (sizeof(TIO) == 2) return bound | (bound & 0x80000000u ? 0u : 0xffffu);
    if (above(bound) > 2 * k)
        for (int bit = 15; bit >= 0; --bit)
            if (above(bound | (1u << bit)) >= k) bound |= 1u << bit;
    return bound;
}

template <typename TIO>
__global__ __launch_bounds__(256) void k_beam_slices(BeamArgs a) {
    constexpr int E = kPiece<TIO>, NP = kPieces, TILE = 256 * E * NP;
    __shared__ u64 list[4][kWaveList];
    __shared__ uint32_t lane_top[256], wave_bound[4];
    __shared__ f32x2 wave_sum[4];
    __shared__ int wave_count[4];
    __shared__ u64 wave_best[4];
    const int row = int(blockIdx.x) / a.slices, slice = int(blockIdx.x) - row * a.slices;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, keep = a.n_out + 1, quarter = (keep + 3) / 4;
    const u64 below = (u64(1) << lane) - 1;
    if (a.finished && a.finished[row]) return;
    const Row<TIO> r(a, row);
    const int tile0 = slice * a.tiles, tiles = min(a.tiles, a.row_tiles - tile0);
    auto first_of = [&](int tile, int j) { return tile * TILE + (j * 256 + tid) * E; };  // element of a lane's piece j
    auto fetch = [&](u32x4 (&raw)[NP], int tile) {
        if (tile * TILE >= r.lead && (tile + 1) * TILE <= r.end) {
            _Pragma("unroll") for (int j = 0; j < NP; ++j) raw[j] = r.whole(first_of(tile, j));
        } else {
            _Pragma("unroll") for (int j = 0; j < NP; ++j) raw[j] = r.part(first_of(tile, j));
        }
    };
    auto make_sane = [&](u32x4 (&raw)[NP]) {
        _Pragma("unroll") for (int j = 0; j < NP; ++j) {
            float x[E];
            unpack(raw[j], x);
            _Pragma("unroll") for (int i = 0; i < E; ++i) x[i] = sane(x[i], kLargestOf<TIO>);
            raw[j] = pack(x);
        }
    };
    int count = 0;       // candidates of this wave; beyond the list's end they are only counted
    bool fits = true;
    f32x2 sums[4];
    bool not_numbers = false;  // a NaN or +inf among the slice's logits: seen by the sum, and then all of it once more with those replaced
    for (;;) {
        float m = -kInf, from = -kLargest, s = 0.f, least = 0.f;
        float best = -kInf;  // this lane's largest so far
        int equal = 0;       // elements met at the bound
        bool in_order = true;
        for (int t = 0; t < tiles; ++t) {
            u32x4 raw[NP];
            fetch(raw, tile0 + t);
            if (not_numbers) make_sane(raw);
            float top = -kInf, piece_top[NP];
            _Pragma("unroll") for (int j = 0; j < NP; ++j) {
                float x[E];
                unpack(raw[j], x);
                piece_top[j] = max3(x[0], x[1], x[2]);
                _Pragma("unroll") for (int i = 3; i < E; i += 2) piece_top[j] = max3(piece_top[j], x[i], x[i + 1 < E ? i + 1 : i]);
                top = fmaxf(top, piece_top[j]);
            }
            if (__ballot(top > m)) {
                m = fmaxf(m, group_max(top, 64));
                const float to = fmaxf(m, -kLargest);
                s *= __builtin_amdgcn_exp2f((from - to) * kLog2E);
                from = to;
            }
            _Pragma("unroll") for (int j = 0; j < NP; ++j) {
                float x[E];
                unpack(raw[j], x);
                _Pragma("unroll") for (int i = 0; i < E; ++i) s += __builtin_amdgcn_exp2f((x[i] - from) * kLog2E);
            }
            // Bound: of the first tile the keep-th largest of the workgroup's 256 lane maxima.  Later also a value that quarter =
            // ceil(keep / 4) lanes of each wave have reached so far; the waves' own only rise, so an old one of another wave will do.
            best = fmaxf(best, top);
            if (t == 0) {
                lane_top[tid] = ordered(top);
                if (lane == 0) wave_bound[wave] = 0;
                __syncthreads();
                uint32_t tops[4];
                _Pragma("unroll") for (int i = 0; i < 4; ++i) tops[i] = lane_top[64 * i + lane];
                least = from_ordered(max(kth_largest<TIO>(tops, keep), kOrderedNegInf));
            } else if (__ballot(top > least)) {
                const uint32_t bests[1] = {ordered(best)};
                uint32_t all = kth_largest<TIO>(bests, quarter);
                if (lane == 0) __atomic_store_n(&wave_bound[wave], all, __ATOMIC_RELAXED);
                _Pragma("unroll") for (int w = 0; w < 4; ++w)
                    if (w != wave) all = min(all, __atomic_load_n(&wave_bound[w], __ATOMIC_RELAXED));
                if (all > ordered(least)) {
                    least = from_ordered(all);
                    equal = 0;
                    in_order = false;
                }
            }
            // Elements above the bound, and of those at it the wave's first `keep` (a mask's value may stand in every place).  At the first
            // tile's bound `keep` have come before those of later tiles; another wave may have met a later bound further on.
            const bool at_bound = (t == 0 || !in_order) && least > -kInf;
            const float bar = at_bound ? least : from_ordered(ordered(least) + 1);
            _Pragma("unroll") for (int j = 0; j < NP; ++j) {
                const int hit = lanes(__ballot(piece_top[j] >= bar));
                if (hit == 0) continue;
                float x[E];
                unpack(raw[j], x);
                const uint32_t token0 = uint32_t(first_of(tile0 + t, j) - r.lead);
                const bool few = !at_bound || hit <= 8;  // all of those at the bound will do
                const float from_here = few ? bar : from_ordered(ordered(least) + 1);
                int same = 0;
                _Pragma("unroll") for (int i = 0; i < E; ++i) {
                    const u64 who = __ballot(x[i] >= from_here);
                    if (who) {
                        const int at = count + lanes(who & below);
                        if (x[i] >= from_here && at < kWaveList) list[wave][at] = make_key(x[i], token0 + i);
                        count += lanes(who);
                    }
                }
                if (few || equal >= keep) continue;
                _Pragma("unroll") for (int i = 0; i < E; ++i) same += x[i] == least ? 1 : 0;
                if (__ballot(same > 0) == 0) continue;
                int upto = same;
                _Pragma("unroll") for (int off = 1; off < 64; off <<= 1) {
                    const int before = __shfl_up(upto, off, 64);
                    if (lane >= off) upto += before;
                }
                int place = equal + upto - same;
                const int all = __builtin_amdgcn_readlane(upto, 63);
                _Pragma("unroll") for (int i = 0; i < E; ++i)
                    if (x[i] == least) {
                        const int at = count + place - equal;
                        if (place < keep && at < kWaveList) list[wave][at] = make_key(x[i], token0 + i);
                        ++place;
                    }
                count += min(all, keep - equal);
                equal += all;
            }
            fits = fits && count <= kWaveList;
            if (fits && count > kWaveList / 2) {  // only the wave's own best go on
                constexpr int M = kWaveList / 64;
                u64 key[M];
                int rank[M];
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                _Pragma("unroll") for (int i = 0; i < M; ++i) {
                    key[i] = 64 * i + lane < count ? list[wave][64 * i + lane] : 0;
                    rank[i] = 0;
                }
                for (int k = 0; k < count; ++k) {
                    const u64 other = list[wave][k];
                    _Pragma("unroll") for (int i = 0; i < M; ++i) rank[i] += other > key[i] ? 1 : 0;
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                _Pragma("unroll") for (int i = 0; i < M; ++i)
                    if (key[i] != 0 && rank[i] < keep) list[wave][rank[i]] = key[i];
                count = keep;
            }
        }
        s = group_sum<64>(s);
        if (lane == 0) {
            wave_sum[wave] = f32x2{m, s};
            wave_count[wave] = fits ? count : kWaveList + 1;
        }
        __syncthreads();
        _Pragma("unroll") for (int w = 0; w < 4; ++w) sums[w] = wave_sum[w];
        const float any = sums[0].y + sums[1].y + sums[2].y + sums[3].y;
        if (any == any || not_numbers) break;
        not_numbers = true;
        count = 0;
        fits = true;
        __syncthreads();
    }
    if (tid == 0) {
        float all = -kInf, sum = 0.f;
        _Pragma("unroll") for (int w = 0; w < 4; ++w) all = fmaxf(all, sums[w].x);
        if (all > -kInf)
            _Pragma("unroll") for (int w = 0; w < 4; ++w) sum += sums[w].y * expf(sums[w].x - all);
        a.sums[blockIdx.x] = f32x2{all, sum};
    }
    u64* out = a.kept + size_t(blockIdx.x) * keep;
    int n = 0;
    fits = true;
    _Pragma("unroll") for (int w = 0; w < 4; ++w) {
        n += wave_count[w];
        fits = fits && wave_count[w] <= kWaveList;
    }
    if (fits) {
        for (int i = lane; i < count; i += 64) {
            const u64 key = list[wave][i];
            int rank = 0;
            _Pragma("unroll") for (int w = 0; w < 4; ++w) rank += rank_in(list[w], wave_count[w], key);
            if (rank < keep) out[rank] = key;
        }
        for (int i = n + tid; i < keep; i += 256) out[i] = 0;
        return;
    }
    // More than a list holds above one bound (whole lanes of the largest): the best one by one, from the logits.
    u64 last = ~u64(0);
    for (int k = 0; k < keep; ++k) {
        u64 best = 0;
        for (int t = 0; t < tiles; ++t) {
            u32x4 raw[NP];
            fetch(raw, tile0 + t);
            if (not_numbers) make_sane(raw);
            _Pragma("unroll") for (int j = 0; j < NP; ++j) {
                float x[E];
                unpack(raw[j], x);
                _Pragma("unroll") for (int i = 0; i < E; ++i) {
                    const u64 key = make_key(x[i], uint32_t(first_of(tile0 + t, j) - r.lead + i));
                    if (x[i] > -kInf && key < last && key > best) best = key;
                }
            }
        }
        _Pragma("unroll") for (int off = 1; off < 64; off <<= 1) {
            const u64 o = __shfl_xor(best, off, 64);
            best = o > best ? o : best;
        }
        __syncthreads();
        if (lane == 0) wave_best[wave] = best;
        __syncthreads();
        _Pragma("unroll") for (int w = 0; w < 4; ++w) best = wave_best[w] > best ? wave_best[w] : best;
        if (tid == 0) out[k] = best;
        last = best;  // 0 from here on once there is none left
    }
}

constexpr int kMergeThreads = 512, kMergeWaves = kMergeThreads / 64;
constexpr int kMergeAhead = 8;    // entries of the lists requested at once by a lane
constexpr int kMaxLists = 4160;   // K * slices, see check()
constexpr int kFewLists = 256;    // with so many, bounds from up to six depths of the lists
constexpr int kMergeList = kMaxOut * (kMaxOut + 2);  // candidates that can reach the bound, see there

__global__ __launch_bounds__(kMergeThreads) void k_beam_merge(BeamArgs a) {
    __shared__ u64 nth_of[kMaxLists], list[kMergeList], best[kMaxOut], the_bound;
    __shared__ float row_max[kMaxOut], row_log[kMaxOut], row_score[kMaxOut];
    __shared__ int row_done[kMaxOut], counts[kMergeWaves], count, hazard;
    const int b = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, K = a.K, n = a.n_out, keep = n + 1;
    const int lists = K * a.slices;
    if (tid == 0) { count = 0; hazard = 0; the_bound = 0; }
    // What comes from memory is requested first: entries of the lists (see the bound below), and the lists from their beginning.  Those
    // of a finished beam's lists are not written and not used.
    const int r0 = min(n, (n + lists - 1) / lists);
    int levels = 1;
    while (lists <= kFewLists && (r0 << (levels - 1)) < n) ++levels;
    const u64* kept = a.kept + size_t(b) * lists * keep;
    auto nth_entry = [&](int i) { return kept[size_t(i % lists) * keep + min(n, r0 << (i / lists)) - 1]; };
    u64 ahead[kMergeAhead];
    const u64 my_nth = tid < levels * lists ? nth_entry(tid) : 0;
    auto request = [&](int i0) {
        _Pragma("unroll") for (int j = 0; j < kMergeAhead; ++j) {
            const int i = i0 + j * kMergeThreads + tid;
            ahead[j] = i < lists * keep ? kept[i] : 0;
        }
    };
    request(0);
    const int width = K > 16 ? 16 : K > 8 ? 32 : 64, k = tid / width;  // lanes to a beam: all beams at once
    if (k < K) {
        const int row = b * K + k;
        const bool done = a.finished && a.finished[row];
        const float so_far = a.scores[row];
        float m = -kInf, s = 0.f;
        if (!done) {
            const f32x2* p = a.sums + size_t(row) * a.slices;
            for (int i = tid % width; i < a.slices; i += width) {  // joined as they come
                const f32x2 x = p[i];
                const float to = fmaxf(m, x.x);
                if (to > -kInf) s = s * expf(m - to) + x.y * expf(x.x - to);
                m = to;
            }
            const float mine = m;
            m = group_max(m, width);
            s = group_sum<16>(mine > -kInf ? s * expf(mine - m) : 0.f);
            if (width >= 32) s += __shfl_xor(s, 16, 64);
            if (width >= 64) s += __shfl_xor(s, 32, 64);
        }
        if (tid % width == 0) {
            row_max[k] = m;
            row_log[k] = logf(s);
            row_score[k] = so_far;
            row_done[k] = done;
        }
    }
    __syncthreads();
    auto score = [&](int k, float x) {  // x: sane
        const float y = row_score[k] + ((x - row_max[k]) - row_log[k]);
        return y == y ? y : -kInf;
    };
    const float per_list = 1.f / float(a.slices), per_entry = 1.f / float(keep);
    auto quotient = [](int x, int by, float inverse) {  // below 2^24: the product is at most one off
        int q = int(float(x) * inverse);
        if (q * by > x) --q;
        if ((q + 1) * by <= x) ++q;
        return q;
    };
    // a kept logit of list l as a key of scores; 0: none
    auto scored = [&](int l, u64 kept) {
        const int k = quotient(l, a.slices, per_list);
        if (kept == 0 || row_done[k]) return u64(0);
        return make_key(score(k, from_ordered(uint32_t(kept >> 32))), uint32_t(k) * uint32_t(a.V) + key_index(kept));
    };
    // Bound: ceil(n / r) lists have their first r entries at or above the ceil(n / r)-th largest of the lists' r-th entries, so this
    // bounds the n-th best from below; the largest of these over some r does.  (r = 1 alone leaves 800 candidates where the best
    // beams' lists hold most of them.)  At most n (n + 1) candidates reach it: r = 1: n lists reach it with an entry or more.
    // r0 > 1: there are fewer than n lists.  (Nothing bounds from below where too few lists have r entries: then there are no more
    // candidates than that either.)
    for (int i = tid; i < levels * lists; i += kMergeThreads) nth_of[i] = scored(i % lists, i == tid ? my_nth : nth_entry(i));
    if (tid < K && row_done[tid]) {  // a finished beam's one candidate
        const float y = row_score[tid];
        list[atomicAdd(&count, 1)] = make_key(y == y ? y : -kInf, uint32_t(tid) * uint32_t(a.V) + uint32_t(a.eos));
    }
    __syncthreads();
    for (int i = tid; i < levels * lists; i += kMergeThreads) {
        const int level = i / lists, r = min(n, r0 << level);
        const u64 x = nth_of[i];
        // (a list is in the order of its logits: its first r entries reach the r-th one's score, not its key)
        if (x != 0 && rank_in(nth_of + level * lists, lists, x) == (n + r - 1) / r - 1)
            atomicMax(&the_bound, r == 1 ? x : x & ~u64(0xffffffffu));
    }
    __syncthreads();
    const u64 bound = the_bound;
    uint32_t last_kept = 0;  // largest score at which a list of this lane's stopped keeping
    for (int i0 = 0; i0 < lists * keep; i0 += kMergeAhead * kMergeThreads) {
        if (i0 > 0) request(i0);
        _Pragma("unroll") for (int j = 0; j < kMergeAhead; ++j) {
            if (ahead[j] == 0) continue;
            const int i = i0 + j * kMergeThreads + tid, l = quotient(i, keep, per_entry);
            const u64 key = scored(l, ahead[j]);
            if (key != 0 && i - l * keep == n) last_kept = max(last_kept, uint32_t(key >> 32));
            if (key != 0 && key >= bound) list[atomicAdd(&count, 1)] = key;
        }
    }
    __syncthreads();
    const int c = count, have = min(c, n);
    for (int i = tid; i < c; i += kMergeThreads) {
        const u64 x = list[i];
        const int rank = rank_in(list, c, x);
        if (rank < n) best[rank] = x;
    }
    __syncthreads();
    const uint32_t bar = have == n ? uint32_t(best[n - 1] >> 32) : kOrderedNegInf;
    if (last_kept >= bar || bar <= kOrderedNegInf) hazard = 1;
    __syncthreads();
    auto put = [&](int place, uint32_t o, uint32_t index) {
        const int k = int(index / uint32_t(a.V)), t = int(index - uint32_t(k) * uint32_t(a.V));
        const size_t i = size_t(b) * n + place;
        a.out_scores[i] = from_ordered(o);
        a.parent[i] = k;
        a.token[i] = t;
        if (a.out_finished) a.out_finished[i] = row_done[k] || t == a.eos;
    };
    if (!hazard) {
        if (tid < n) put(tid, uint32_t(best[tid] >> 32), key_index(best[tid]));
        return;
    }
    // Those above the n-th best score are known; those at it come by index, from the logits of the slices that have any.
    int above = 0;
    for (int i = 0; i < have; ++i) above += uint32_t(best[i] >> 32) > bar ? 1 : 0;
    if (tid < above) put(tid, uint32_t(best[tid] >> 32), key_index(best[tid]));
    int found = above;
    for (int k = 0; k < K && found < n; ++k) {
        const char* x = a.logits + (b * K + k) * a.row_bytes;
        for (int s = 0; s < a.slices && found < n; ++s) {
            const size_t slot = size_t(b * K + k) * a.slices + s;
            // a slice of the first kernel starts at a whole piece of 16 bytes
            const int lead = int(reinterpret_cast<uintptr_t>(x) & 15u) / (a.bf16 ? 2 : 4);
            const int per_slice = a.tiles * 256 * kPieces * (a.bf16 ? 8 : 4);
            const int t0 = max(s * per_slice - lead, 0), t1 = min((s + 1) * per_slice - lead, a.V);
            if (bar > kOrderedNegInf && row_done[k]) {
                if (a.eos < t0 || a.eos >= t1) continue;
            } else if (bar > kOrderedNegInf) {
                const u64 first = a.kept[slot * keep];
                if (first == 0 || ordered(score(k, from_ordered(uint32_t(first >> 32)))) < bar) continue;
            }
            for (int at = t0; at < t1 && found < n; at += kMergeThreads) {
                const int t = at + tid;
                bool hit = false;
                if (t < t1) {
                    float y;
                    if (row_done[k]) {
                        y = t == a.eos && row_score[k] == row_score[k] ? row_score[k] : -kInf;
                    } else {
                        const float v = a.bf16 ? bf16_lo(reinterpret_cast<const uint16_t*>(x)[t]) : reinterpret_cast<const float*>(x)[t];
                        y = score(k, sane(v, a.bf16 ? kLargestOf<uint16_t> : kLargest));
                    }
                    hit = ordered(y) == bar;
                }
                const u64 hits = __ballot(hit);
                if (lane == 0) counts[wave] = lanes(hits);
                __syncthreads();
                int before = 0, all = 0;
                _Pragma("unroll") for (int w = 0; w < kMergeWaves; ++w) {
                    before += w < wave ? counts[w] : 0;
                    all += counts[w];
                }
                const int place = found + before + lanes(hits & ((u64(1) << lane) - 1));
                if (hit && place < n) put(place, bar, uint32_t(k) * uint32_t(a.V) + uint32_t(t));
                found += all;
                __syncthreads();
            }
        }
    }
}

// ---- the states follow their beams ---------------------------------------------------------------------------------
// A thread owns the same 16 bytes (or 4) of the K rows of a sequence: it has read what each row is to become, from the rows of the
// parents, before it stores the first one, so that the rows can change in place.  Nothing is moved for a beam that stays.
constexpr int kMaxStates = 64;
struct ReorderArgs {
    char* state[kMaxStates];
    size_t row_bytes[kMaxStates];
    const int32_t* parent;
    int K;
};

template <typename V, int KM>
__device__ __forceinline__ void reorder_column(char* rows, size_t row_bytes, size_t at, const int* from, int K) {
    V v[KM];
    _Pragma("unroll") for (int i = 0; i < KM; ++i)
        if (i < K && from[i] != i) v[i] = *reinterpret_cast<const V*>(rows + (from[i] < 0 ? 0 : from[i]) * row_bytes + at);
    _Pragma("unroll") for (int i = 0; i < KM; ++i)
        if (i < K && from[i] != i) {
            if (from[i] < 0) v[i] = V(0xffffffffu);
            *reinterpret_cast<V*>(rows + i * row_bytes + at) = v[i];
        }
}

template <int KM>
__global__ __launch_bounds__(256) void k_state_reorder(ReorderArgs a) {
    const size_t bytes = a.row_bytes[blockIdx.z];
    const bool wide = bytes % 16 == 0;
    const size_t at = (size_t(blockIdx.x) * 256 + threadIdx.x) * (wide ? 16 : 4);
    int from[KM];
    _Pragma("unroll") for (int i = 0; i < KM; ++i) {
        const int p = i < a.K ? a.parent[size_t(blockIdx.y) * a.K + i] : i;
        from[i] = p < 0 || p >= a.K ? (i < a.K ? -1 : i) : p;
    }
    char* rows = a.state[blockIdx.z] + size_t(blockIdx.y) * a.K * bytes;
    if (at >= bytes) return;
    if (wide) reorder_column<u32x4, KM>(rows, bytes, at, from, a.K);
    else reorder_column<uint32_t, KM>(rows, bytes, at, from, a.K);
}

// ---- host ------------------------------------------------------------------------------------------------------------
constexpr int kSlices = 1024, kMaxTiles = 8;
// Slices of so many tiles that there are a few workgroups for each compute unit, or of one.
struct BeamPlan { int row_tiles, tiles, slices; };
BeamPlan plan(const lsm_beam_params& p) {
    const int piece = p.dtype == LSM_DTYPE_BF16 ? 8 : 4, tile = 256 * piece * kPieces;
    BeamPlan pl{};
    pl.row_tiles = int((int64_t(p.V) + piece - 1 + tile - 1) / tile);  // a row may start inside a piece
    const int64_t all = int64_t(p.B) * p.K * pl.row_tiles;
    pl.tiles = int(all < 2 * kSlices ? 1 : all / kSlices < kMaxTiles ? all / kSlices : kMaxTiles);
    if (pl.tiles > pl.row_tiles) pl.tiles = pl.row_tiles;
    pl.slices = (pl.row_tiles + pl.tiles - 1) / pl.tiles;
    return pl;
}
int check(const lsm_beam_params* p) {
    if (!p) return LSM_ERR_NULL;
    if (p->struct_size != sizeof(lsm_beam_params)) return LSM_ERR_SHAPE;
    if (p->B < 1 || p->K < 1 || p->V < 1 || p->n_out < 1 || p->row_stride < p->V) return LSM_ERR_SHAPE;
    if (p->dtype != LSM_DTYPE_F32 && p->dtype != LSM_DTYPE_BF16) return LSM_ERR_UNSUPPORTED;
    if (p->K > kMaxOut || p->n_out > kMaxOut || p->reserved != 0) return LSM_ERR_UNSUPPORTED;
    const int64_t all = int64_t(p->K) * p->V;
    if (all > (int64_t(1) << 25) || p->n_out > all || p->eos < -1 || p->eos >= p->V) return LSM_ERR_SHAPE;
    // a sequence's lists: one a tile where there are fewer than 2 kSlices tiles, else a fraction of at most 2^25 / 4096 + K tiles
    static_assert(2 * kSlices <= kMaxLists && ((1 << 25) / 4096 + kMaxOut) / 2 + kMaxOut <= kMaxLists, "lists of a sequence");
    if (p->row_stride > (int64_t(1) << 40)) return LSM_ERR_SHAPE;
    if (int64_t(p->B) * p->K * plan(*p).slices * 256 > kAxisThreads || int64_t(p->B) * kMergeThreads > kAxisThreads) return LSM_ERR_SHAPE;
    return LSM_OK;
}
size_t sums_bytes(const lsm_beam_params& p, const BeamPlan& pl) { return align256(size_t(p.B) * p.K * pl.slices * sizeof(f32x2)); }

}  // namespace
}  // namespace lsm

extern "C" {

size_t lsm_beam_select_workspace_bytes(const lsm_beam_params* p) {
    using namespace lsm;
    if (check(p) != LSM_OK) return 0;
    const BeamPlan pl = plan(*p);
    return sums_bytes(*p, pl) + align256(size_t(p->B) * p->K * pl.slices * (p->n_out + 1) * sizeof(u64));
}

int lsm_beam_select(const lsm_beam_params* p, const void* logits, const float* scores, const uint8_t* finished,
                    float* out_scores, int32_t* parent, int32_t* token, uint8_t* out_finished, void* workspace,
                    size_t workspace_bytes, void* stream) {
    using namespace lsm;
    const int rc = check(p);
    if (rc != LSM_OK) return rc;
    if (!logits || !scores || !out_scores || !parent || !token) return LSM_ERR_NULL;
    if (p->eos < 0 && (finished || out_finished)) return LSM_ERR_NULL;
    if (misaligned(logits) || misaligned(scores) || misaligned(finished) || misaligned(out_scores) || misaligned(parent) ||
        misaligned(token) || misaligned(out_finished) || misaligned(workspace))
        return LSM_ERR_ALIGN;
    if (!workspace || workspace_bytes < lsm_beam_select_workspace_bytes(p)) return LSM_ERR_WORKSPACE;
    const BeamPlan pl = plan(*p);
    const bool bf16 = p->dtype == LSM_DTYPE_BF16;
    const BeamArgs a{static_cast<const char*>(logits), scores, finished, out_scores, parent, token, out_finished,
                     static_cast<f32x2*>(workspace), reinterpret_cast<u64*>(static_cast<char*>(workspace) + sums_bytes(*p, pl)),
                     p->row_stride * (bf16 ? 2 : 4), p->B * p->K, p->K, p->V, p->n_out, p->eos, bf16, pl.slices, pl.tiles, pl.row_tiles};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const unsigned blocks = unsigned(p->B) * p->K * pl.slices;
    {
        ProfScope ps(KID_BEAM_SLICES, st);
        if (bf16) hipLaunchKernelGGL((k_beam_slices<uint16_t>), dim3(blocks), dim3(256), 0, st, a);
        else hipLaunchKernelGGL((k_beam_slices<float>), dim3(blocks), dim3(256), 0, st, a);
    }
    if (!launched()) return LSM_ERR_LAUNCH;
    {
        ProfScope ps(KID_BEAM_MERGE, st);
        hipLaunchKernelGGL(k_beam_merge, dim3(p->B), dim3(kMergeThreads), 0, st, a);
    }
    return launched() ? LSM_OK : LSM_ERR_LAUNCH;
}

int lsm_state_reorder(void* const* states, const size_t* row_bytes, int n_states, const int32_t* parent, int B, int K,
                      void* stream) {
    using namespace lsm;
    if (!states || !row_bytes || !parent) return LSM_ERR_NULL;
    if (n_states < 1 || n_states > kMaxStates || B < 1 || B > 65535 || K < 1) return LSM_ERR_SHAPE;
    if (K > kMaxOut) return LSM_ERR_UNSUPPORTED;
    ReorderArgs a{};
    size_t columns = 0;
    for (int i = 0; i < n_states; ++i) {
        if (!states[i]) return LSM_ERR_NULL;
        if (row_bytes[i] == 0 || row_bytes[i] % 4 != 0) return LSM_ERR_SHAPE;
        a.state[i] = static_cast<char*>(states[i]);
        a.row_bytes[i] = row_bytes[i];
        const size_t c = row_bytes[i] / (row_bytes[i] % 16 == 0 ? 16 : 4);
        columns = c > columns ? c : columns;
    }
    if (columns > (size_t(1) << 31)) return LSM_ERR_SHAPE;
    // Tensors that share memory, with each other or with the parents, would be read while others' workgroups change them.
    struct Range { uintptr_t from, to; } range[kMaxStates + 1];
    const auto place = [](const void* p, size_t bytes) { return Range{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes}; };
    for (int i = 0; i < n_states; ++i) range[i] = place(states[i], row_bytes[i] * size_t(B) * K);
    range[n_states] = place(parent, size_t(B) * K * sizeof(int32_t));
    std::sort(range, range + n_states + 1, [](const Range& x, const Range& y) { return x.from < y.from; });
    for (int i = 0; i < n_states; ++i)
        if (range[i].to > range[i + 1].from) return LSM_ERR_SHAPE;
    for (int i = 0; i < n_states; ++i)
        if (misaligned(states[i])) return LSM_ERR_ALIGN;
    if (misaligned(parent)) return LSM_ERR_ALIGN;
    a.parent = parent;
    a.K = K;
    const dim3 grid(unsigned((columns + 255) / 256), B, n_states), block(256);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    ProfScope ps(KID_REORDER, st);
    if (K <= 4) hipLaunchKernelGGL((k_state_reorder<4>), grid, block, 0, st, a);
    else if (K <= 8) hipLaunchKernelGGL((k_state_reorder<8>), grid, block, 0, st, a);
    else if (K <= 16) hipLaunchKernelGGL((k_state_reorder<16>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_state_reorder<32>), grid, block, 0, st, a);
    return launched() ? LSM_OK : LSM_ERR_LAUNCH;
}

}  // extern "C"
