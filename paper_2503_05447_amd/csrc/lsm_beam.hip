// One step of a beam search: the best candidates of beams x vocabulary, and the beams' states rearranged (include/lsm_block.h).
//
// Selection is two kernels.  k_beam_slices: a workgroup reads a slice of one beam's logits once, into registers, and leaves the
// slice's maximum, its sum of exponentials and its n_out + 1 best logits (value descending, token ascending).  k_beam_merge: a
// workgroup per sequence joins the slices' sums to each beam's log-normaliser, turns the kept logits into scores and takes the
// n_out best.  Scores fall with the logits of a beam, but not strictly (rounding makes equal scores of close logits), and equal
// scores go by token: where a slice's last kept score reaches the n_out-th best, dropped ones might be due, and the merge takes
// the candidates at exactly that score from the logits themselves, in order.
//
// To find the best n of what a wave holds without sorting it: the n-th largest of its 64 lanes' maxima bounds the n-th best from
// below; its upper bits come from counting lanes above a trial value, bit by bit (a comparison and a population count
// each).  Few elements reach the bound; they are collected in LDS and ranked by counting.
//
// Bound: HBM (the logits once) for large batches; a latency of two launches for small ones.
#include "lsm_block_dev.h"

namespace lsm {
namespace {

typedef unsigned long long u64;

constexpr float kInf = __builtin_inff();
constexpr float kLargest = 3.402823466e38f;
template <typename TIO> constexpr float kLargestOf = sizeof(TIO) == 4 ? kLargest : 3.389531390e38f;  // finite, of the logits' type
constexpr int kMaxOut = 32;      // n_out and K
constexpr int kSliceList = 1024; // candidates of a slice that are ranked at once

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
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, dpp<0xB1>(x));
    x = fmaxf(x, dpp<0x4E>(x));
    x = fmaxf(x, dpp<0x141>(x));
    x = fmaxf(x, dpp<0x140>(x));
    x = fmaxf(x, __shfl_xor(x, 16, 64));
    return fmaxf(x, __shfl_xor(x, 32, 64));
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
    int K, V, n_out, eos, slices, bf16, per_slice;
};

// The pieces of 16 bytes that a beam's logits lie in, counted from the one with its first logit; `lead` elements of that one
// come before it.  Elements that are not the beam's read as -inf, which is never kept and adds nothing to a sum.
template <typename TIO>
struct Row {
    const char* p;
    int lead, end;
    __device__ __forceinline__ Row(const BeamArgs& a, int row) {
        const char* x = a.logits + row * a.row_bytes;
        lead = int(reinterpret_cast<uintptr_t>(x) & 15u) / int(sizeof(TIO));
        p = x - lead * int(sizeof(TIO));
        end = lead + a.V;
    }
    __device__ __forceinline__ u32x4 piece(int at) const {  // at: its first element, a multiple of kPiece<TIO>
        constexpr int E = kPiece<TIO>;
        if (at >= lead && at + E <= end) return *reinterpret_cast<const u32x4*>(p + size_t(at) * sizeof(TIO));
        u32x4 v;
        _Pragma("unroll") for (int i = 0; i < 4; ++i) {
            if (sizeof(TIO) == 4) {
                v[i] = at + i >= lead && at + i < end ? reinterpret_cast<const uint32_t*>(p)[at + i] : 0xff800000u;
            } else {
                uint32_t w = 0;
                _Pragma("unroll") for (int j = 0; j < 2; ++j) {
                    const int e = at + 2 * i + j;
                    w |= (e >= lead && e < end ? uint32_t(reinterpret_cast<const uint16_t*>(p)[e]) : 0xff80u) << (16 * j);
                }
                v[i] = w;
            }
        }
        return v;
    }
};

// A workgroup's list of candidates; `count` goes on beyond its end.
template <int CAP>
__device__ __forceinline__ void append(u64* list, int* count, u64 key) {
    const int at = atomicAdd(count, 1);
    if (at < CAP) list[at] = key;
}

template <typename TIO, int NP>
__global__ __launch_bounds__(256) void k_beam_slices(BeamArgs a) {
    constexpr int E = kPiece<TIO>;
    __shared__ u64 list[kSliceList];
    __shared__ f32x2 wave_sum[4];
    __shared__ uint32_t wave_bound[4];
    __shared__ u64 wave_best[4];
    __shared__ int count;
    const int row = int(blockIdx.x) / a.slices, slice = int(blockIdx.x) - row * a.slices;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, keep = a.n_out + 1;
    if (a.finished && a.finished[row]) return;
    if (tid == 0) count = 0;
    const Row<TIO> r(a, row);
    const int at0 = (slice * NP * 256 + tid) * E;  // this lane's pieces are 256 pieces apart
    u32x4 raw[NP];
    _Pragma("unroll") for (int j = 0; j < NP; ++j) raw[j] = r.piece(at0 + j * 256 * E);

    float top = -kInf, m = 0.f, s = 0.f;
    auto normaliser = [&]() {
        top = -kInf;
        _Pragma("unroll") for (int j = 0; j < NP; ++j) {
            float x[E];
            unpack(raw[j], x);
            _Pragma("unroll") for (int i = 0; i < E; i += 2) top = max3(top, x[i], x[i + 1]);
        }
        m = wave_max(top);
        const float from = fmaxf(m, -kLargest);
        s = 0.f;
        _Pragma("unroll") for (int j = 0; j < NP; ++j) {
            float x[E];
            unpack(raw[j], x);
            _Pragma("unroll") for (int i = 0; i < E; ++i) s += __builtin_amdgcn_exp2f((x[i] - from) * 1.44269504f);
        }
        s = group_sum<64>(s);
    };
    normaliser();
    if (s != s) {  // a NaN or +inf among the wave's logits (the sum is the same in all lanes)
        _Pragma("unroll") for (int j = 0; j < NP; ++j) {
            float x[E];
            unpack(raw[j], x);
            _Pragma("unroll") for (int i = 0; i < E; ++i) x[i] = sane(x[i], kLargestOf<TIO>);
            raw[j] = pack(x);
        }
        normaliser();
    }
    // bound: the keep-th largest lane maximum; in fp32 its upper 16 bits do, unless many lanes share them
    uint32_t bound = 0;
    const uint32_t mine = ordered(top);
    _Pragma("unroll") for (int bit = 31; bit >= 16; --bit) {
        const uint32_t trial = bound | (1u << bit);
        if (lanes(__ballot(mine >= trial)) >= keep) bound = trial;
    }
    if (sizeof(TIO) == 2) {
        bound |= bound & 0x80000000u ? 0u : 0xffffu;
    } else if (lanes(__ballot(mine >= bound)) > 2 * keep) {
        for (int bit = 15; bit >= 0; --bit) {
            const uint32_t trial = bound | (1u << bit);
            if (lanes(__ballot(mine >= trial)) >= keep) bound = trial;
        }
    }
    if (lane == 0) {
        wave_sum[wave] = f32x2{m, s};
        wave_bound[wave] = bound;
    }
    __syncthreads();
    bound = max(max(wave_bound[0], wave_bound[1]), max(wave_bound[2], wave_bound[3]));
    if (tid == 0) {
        float all = -kInf, sum = 0.f;
        _Pragma("unroll") for (int w = 0; w < 4; ++w) all = fmaxf(all, wave_sum[w].x);
        if (all > -kInf)
            _Pragma("unroll") for (int w = 0; w < 4; ++w) sum += wave_sum[w].y * expf(wave_sum[w].x - all);
        a.sums[blockIdx.x] = f32x2{all, sum};
    }
    // Elements above the bound, and of those at it the wave's first `keep` (a mask's value may stand in every place).
    const float least = from_ordered(max(bound, kOrderedNegInf + 1));
    int equal = 0;
    _Pragma("unroll") for (int j = 0; j < NP; ++j) {
        float x[E], best = -kInf;
        unpack(raw[j], x);
        _Pragma("unroll") for (int i = 0; i < E; i += 2) best = max3(best, x[i], x[i + 1]);
        if (__ballot(best >= least) == 0) continue;
        const uint32_t token0 = uint32_t(at0 + j * 256 * E - r.lead);
        int same = 0;
        _Pragma("unroll") for (int i = 0; i < E; ++i) {
            if (x[i] > least) append<kSliceList>(list, &count, make_key(x[i], token0 + i));
            same += x[i] == least ? 1 : 0;
        }
        if (equal >= keep || __ballot(same > 0) == 0) continue;
        int upto = same;
        _Pragma("unroll") for (int off = 1; off < 64; off <<= 1) {
            const int t = __shfl_up(upto, off, 64);
            if (lane >= off) upto += t;
        }
        int place = equal + upto - same;
        _Pragma("unroll") for (int i = 0; i < E; ++i)
            if (x[i] == least) {
                if (place < keep) append<kSliceList>(list, &count, make_key(x[i], token0 + i));
                ++place;
            }
        equal += __builtin_amdgcn_readlane(upto, 63);
    }
    __syncthreads();
    u64* out = a.kept + size_t(blockIdx.x) * keep;
    const int n = count;
    if (n <= kSliceList) {
        for (int i = tid; i < n; i += 256) {
            const u64 key = list[i];
            int rank = 0;
            for (int k = 0; k < n; ++k) rank += list[k] > key ? 1 : 0;
            if (rank < keep) out[rank] = key;
        }
        for (int i = n + tid; i < keep; i += 256) out[i] = 0;
        return;
    }
    // More than the list holds above one bound (long runs of neighbours among the largest): the best one by one.
    u64 last = ~u64(0);
    for (int k = 0; k < keep; ++k) {
        u64 best = 0;
        _Pragma("unroll") for (int j = 0; j < NP; ++j) {
            float x[E];
            unpack(raw[j], x);
            _Pragma("unroll") for (int i = 0; i < E; ++i) {
                const u64 key = make_key(x[i], uint32_t(at0 + j * 256 * E - r.lead + i));
                if (x[i] > -kInf && key < last && key > best) best = key;
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

constexpr int kMergeThreads = 1024, kMergePer = 8, kMergeWaves = kMergeThreads / 64;

__global__ __launch_bounds__(kMergeThreads) void k_beam_merge(BeamArgs a) {
    __shared__ u64 list[kMaxOut + kMergeThreads * kMergePer];
    __shared__ u64 best[kMaxOut];
    __shared__ u64 wave_bound[kMergeWaves];
    __shared__ float row_max[kMaxOut], row_log[kMaxOut], row_score[kMaxOut];
    __shared__ int row_done[kMaxOut], counts[kMergeWaves], count, hazard;
    const int b = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, K = a.K, n = a.n_out, keep = n + 1;
    if (tid == 0) { count = 0; hazard = 0; }
    for (int k = wave; k < K; k += kMergeWaves) {
        const int row = b * K + k;
        const bool done = a.finished && a.finished[row];
        float m = -kInf, s = 0.f;
        if (!done) {
            const f32x2* p = a.sums + size_t(row) * a.slices;
            for (int i = lane; i < a.slices; i += 64) m = fmaxf(m, p[i].x);
            m = wave_max(m);
            if (m > -kInf)
                for (int i = lane; i < a.slices; i += 64) s += p[i].y * expf(p[i].x - m);
            s = group_sum<64>(s);
        }
        if (lane == 0) {
            row_max[k] = m;
            row_log[k] = logf(s);
            row_score[k] = a.scores[row];
            row_done[k] = done;
        }
    }
    __syncthreads();
    auto score = [&](int k, float x) {  // x: sane
        const float y = row_score[k] + ((x - row_max[k]) - row_log[k]);
        return y == y ? y : -kInf;
    };
    int have = 0;  // best[0 .. have): the best so far, descending
    if (tid < K && row_done[tid]) {
        const float y = row_score[tid];
        append<kMaxOut>(list, &count, make_key(y == y ? y : -kInf, uint32_t(tid) * uint32_t(a.V) + uint32_t(a.eos)));
    }
    __syncthreads();
    const int per_row = a.slices * keep, total = K * per_row;
    uint32_t last_kept = 0;  // largest score at which a slice of this thread's stopped keeping
    for (int base = 0; base == 0 || base < total; base += kMergeThreads * kMergePer) {
        u64 key[kMergePer], top = 0;
        _Pragma("unroll") for (int j = 0; j < kMergePer; ++j) {
            const int i = base + tid + j * kMergeThreads, k = i / per_row;
            key[j] = 0;
            if (i >= total || row_done[k]) continue;
            const u64 kept = a.kept[size_t(b) * total + i];
            if (kept == 0) continue;
            key[j] = make_key(score(k, from_ordered(uint32_t(kept >> 32))), uint32_t(k) * uint32_t(a.V) + key_index(kept));
            top = key[j] > top ? key[j] : top;
            if (i % keep == n) last_kept = max(last_kept, uint32_t(key[j] >> 32));
        }
        // bound: the n-th largest of the lanes' best, down to the last bit only where many lanes share its score
        u64 bound = 0;
        for (int bit = 63; bit >= 0; --bit) {
            const u64 trial = bound | (u64(1) << bit);
            if (lanes(__ballot(top >= trial)) >= n) bound = trial;
            if (bit == 32 && lanes(__ballot(top >= bound)) <= 2 * n) break;
        }
        if (lane == 0) wave_bound[wave] = bound;
        __syncthreads();
        _Pragma("unroll") for (int w = 0; w < kMergeWaves; ++w) bound = wave_bound[w] > bound ? wave_bound[w] : bound;
        if (bound == 0) bound = 1;
        _Pragma("unroll") for (int j = 0; j < kMergePer; ++j)
            if (key[j] >= bound) append<kMaxOut + kMergeThreads * kMergePer>(list, &count, key[j]);
        __syncthreads();
        const int c = count;
        for (int i = tid; i < c; i += kMergeThreads) {
            const u64 x = list[i];
            int rank = 0;
            for (int k = 0; k < c; ++k) rank += list[k] > x ? 1 : 0;
            if (rank < n) best[rank] = x;
        }
        __syncthreads();
        have = min(c, n);
        if (tid < have) list[tid] = best[tid];
        if (tid == 0) count = have;
        __syncthreads();
    }
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
            const int t0 = max(s * a.per_slice - lead, 0), t1 = min((s + 1) * a.per_slice - lead, a.V);
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
// A thread owns the same 16 bytes (or 4) of the K rows of a sequence: it requests what each row is to become, from the rows of the
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
constexpr int kFewPieces = 2, kManyPieces = 8;  // 16-byte pieces a lane (in fp32 twice as many): slices of 4096 or 16384 logits

struct BeamPlan { int per_slice, slices; bool many; };
BeamPlan plan(const lsm_beam_params& p) {
    const int piece = p.dtype == LSM_DTYPE_BF16 ? 8 : 4;
    auto slices = [&](int64_t n) { return int64_t(p.V + piece - 1 + n - 1) / n; };  // a row may start inside a piece
    const int few = 256 * 8 * kFewPieces, large = 256 * 8 * kManyPieces;
    const bool many = int64_t(p.B) * p.K * slices(large) >= 512;
    const int n = many ? large : few;
    return BeamPlan{n, int(slices(n)), many};
}
int check(const lsm_beam_params* p) {
    if (!p) return LSM_ERR_NULL;
    if (p->struct_size != sizeof(lsm_beam_params)) return LSM_ERR_SHAPE;
    if (p->B < 1 || p->K < 1 || p->V < 1 || p->n_out < 1 || p->row_stride < p->V) return LSM_ERR_SHAPE;
    if (p->dtype != LSM_DTYPE_F32 && p->dtype != LSM_DTYPE_BF16) return LSM_ERR_UNSUPPORTED;
    if (p->K > kMaxOut || p->n_out > kMaxOut || p->reserved != 0) return LSM_ERR_UNSUPPORTED;
    const int64_t all = int64_t(p->K) * p->V;
    if (all > (int64_t(1) << 30) || p->n_out > all || p->eos < -1 || p->eos >= p->V) return LSM_ERR_SHAPE;
    if (p->row_stride > (int64_t(1) << 40) || int64_t(p->B) * p->K * plan(*p).slices > 0x7fffffff) return LSM_ERR_SHAPE;
    return LSM_OK;
}
size_t sums_bytes(const lsm_beam_params& p, const BeamPlan& pl) { return align256(size_t(p.B) * p.K * pl.slices * sizeof(f32x2)); }

template <typename TIO, int F>
void launch_slices(const BeamArgs& a, bool many, unsigned blocks, hipStream_t st) {
    ProfScope ps(KID_BEAM_SLICES, st);
    if (many) hipLaunchKernelGGL((k_beam_slices<TIO, F * kManyPieces>), dim3(blocks), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_beam_slices<TIO, F * kFewPieces>), dim3(blocks), dim3(256), 0, st, a);
}

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
                     p->row_stride * (bf16 ? 2 : 4), p->K, p->V, p->n_out, p->eos, pl.slices, bf16, pl.per_slice};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const unsigned blocks = unsigned(p->B) * p->K * pl.slices;
    if (bf16) launch_slices<uint16_t, 1>(a, pl.many, blocks, st);
    else launch_slices<float, 2>(a, pl.many, blocks, st);
    {
        ProfScope ps(KID_BEAM_MERGE, st);
        hipLaunchKernelGGL(k_beam_merge, dim3(p->B), dim3(kMergeThreads), 0, st, a);
    }
    return hipGetLastError() == hipSuccess ? LSM_OK : LSM_ERR_LAUNCH;
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
        if (misaligned(states[i])) return LSM_ERR_ALIGN;
        if (row_bytes[i] == 0 || row_bytes[i] % 4 != 0) return LSM_ERR_SHAPE;
        a.state[i] = static_cast<char*>(states[i]);
        a.row_bytes[i] = row_bytes[i];
        const size_t c = row_bytes[i] / (row_bytes[i] % 16 == 0 ? 16 : 4);
        columns = c > columns ? c : columns;
    }
    if (misaligned(parent)) return LSM_ERR_ALIGN;
    if (columns > (size_t(1) << 31)) return LSM_ERR_SHAPE;
    a.parent = parent;
    a.K = K;
    const dim3 grid(unsigned((columns + 255) / 256), B, n_states), block(256);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    ProfScope ps(KID_REORDER, st);
    if (K <= 4) hipLaunchKernelGGL((k_state_reorder<4>), grid, block, 0, st, a);
    else if (K <= 8) hipLaunchKernelGGL((k_state_reorder<8>), grid, block, 0, st, a);
    else if (K <= 16) hipLaunchKernelGGL((k_state_reorder<16>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_state_reorder<32>), grid, block, 0, st, a);
    return hipGetLastError() == hipSuccess ? LSM_OK : LSM_ERR_LAUNCH;
}

}  // extern "C"
