// Norm of every head of q and k with the rotation by position, one pass forward and one backward (include/lsm_block.h).
//
// A row x (one head of one token, d elements) becomes y = scale R_p (w * (r x)).  With the partner x' of each rotated
// element this is y_i = r (x_i c_i + x'_i s_i), c_i = scale w_i cos, s_i = -/+ scale w'_i sin: two coefficients per feature
// that depend on the token but not on the head.  A row is held by d / 8 lanes (bf16; d / 4 in fp32), 16 bytes a lane, so a
// wave takes the rows of a few tokens for one head at a time, keeps its tokens' coefficients in registers and walks over the
// heads, four rows requested at a time.  The partner of the halves' form lies in another lane of the row: it comes by a
// lane permutation of the packed elements.
//
// Bound: HBM.  Forward reads and writes each element once, backward reads x and dy and writes dx.  B=4, T=8192, 16 + 16 heads of 128,
// bf16: forward 110 us (4.9 TB/s), backward 165 (4.9 TB/s) and 5 for the weights' sums, 272 one after another: the rate of a large
// copy.  One token of 4 sequences: 5.9 us, the latency of the launch and of position, table, weights and rows, one after the other.
#include "lsm_block_dev.h"

#include <algorithm>

namespace lsm {
namespace {

struct QkSide {  // q or k
    const void* x;
    const void* g;  // gradient of the output (backward)
    void* y;        // output, or the gradient of the input (backward)
    const float* w;
    float scale;
    int H;
    lsm_strides xs, gs, ys;
};
struct QkArgs {
    QkSide side[2];
    int T, tokens;  // tokens per sequence, B * T
    int rot, n_pos, norm;
    float eps;
    const float* cos_sin;
    const int* positions;
    int groups, splits, per;  // work items: groups of a wave's tokens x ranges of `per` heads (q's, then k's)
    float* part;              // backward: [2][gridDim.x][D] sums of a workgroup's rows for the weights' gradients
};

// A wave's tokens and the part of a row that a lane holds.
template <typename TIO, int D>
struct QkLane {
    static constexpr int E = kPiece<TIO>, L = D / E, R = 64 / L;  // elements a lane, lanes a row, rows a wave
    int f0;          // first feature
    bool live;
    int b, t, partner;
    float cs[E], sn[E];  // cosine, and the sine with the sign that it has for this side of the pair
    uint32_t turned;     // all bits where this lane's features are rotated: what they are not turned with counts as 0, an infinity too

    __device__ __forceinline__ QkLane(const QkArgs& a, int group, bool pairs) {
        const int lane = threadIdx.x & 63;
        f0 = (lane % L) * E;
        const int at = group * R + lane / L;
        live = at < a.tokens;
        const int token = min(at, a.tokens - 1);
        b = token / a.T;
        t = token - b * a.T;
        partner = lane;
        turned = 0;
        _Pragma("unroll") for (int i = 0; i < E; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
        if (a.rot == 0) return;
        const int pos = a.positions ? a.positions[token] : t;
        if (pos < 0 || pos >= a.n_pos) {
            _Pragma("unroll") for (int i = 0; i < E; ++i) cs[i] = __uint_as_float(0x7fc00000u);
            return;
        }
        if (f0 >= a.rot) return;
        turned = 0xffffffffu;
        const int half = a.rot / 2;
        const float* row = a.cos_sin + size_t(pos) * a.rot;
        if (pairs) {
            _Pragma("unroll") for (int i = 0; i < E / 2; ++i) {
                cs[2 * i] = cs[2 * i + 1] = row[f0 / 2 + i];
                sn[2 * i + 1] = row[half + f0 / 2 + i];
                sn[2 * i] = -sn[2 * i + 1];
            }
        } else {
            const bool second = f0 >= half;
            const int c0 = second ? f0 - half : f0;
            partner = second ? lane - half / E : lane + half / E;
            _Pragma("unroll") for (int i = 0; i < E; i += 4) {
                const f32x4 c = *reinterpret_cast<const f32x4*>(row + c0 + i), s = *reinterpret_cast<const f32x4*>(row + half + c0 + i);
                _Pragma("unroll") for (int j = 0; j < 4; ++j) { cs[i + j] = c[j]; sn[i + j] = second ? s[j] : -s[j]; }
            }
        }
    }
    __device__ __forceinline__ size_t at(const lsm_strides& s) const { return size_t(b * s.batch + t * s.token) + f0; }
    __device__ __forceinline__ int partner_feature(int i, bool pairs) const {
        return pairs ? f0 + (i ^ 1) : f0 + (partner - int(threadIdx.x & 63)) * E + i;
    }
};
template <typename TIO>
__device__ __forceinline__ u32x4 row_load(const TIO* p) { return *reinterpret_cast<const u32x4*>(p); }
// results do not stay in a cache that is full of what is still to be read (fp32 step of 2047 tokens 66 -> 62 us, bf16 of 8192 284 -> 279)
template <typename TIO>
__device__ __forceinline__ void row_store(TIO* p, const u32x4& v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p)); }

// the elements that a lane's elements are turned with, 0 where they are not
template <bool PAIRS, int E>
__device__ __forceinline__ void partners(const u32x4& raw, int partner, uint32_t turned, float (&xp)[E]) {
    u32x4 o;
    _Pragma("unroll") for (int i = 0; i < 4; ++i)
        o[i] = (PAIRS ? raw[i] : uint32_t(__builtin_amdgcn_ds_bpermute(4 * partner, int(raw[i])))) & turned;
    if (PAIRS) {
        float x[E];
        unpack(o, x);
        _Pragma("unroll") for (int i = 0; i < E; ++i) xp[i] = x[i ^ 1];
    } else {
        unpack(o, xp);
    }
}

constexpr int kAhead = 4;  // rows requested at a time

template <typename TIO, int D, bool PAIRS>
__global__ __launch_bounds__(256) void k_qk(QkArgs a) {
    typedef QkLane<TIO, D> Lane;
    constexpr int E = Lane::E;
    const int item = int(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (item >= a.groups * a.splits) return;
    const Lane ln(a, item / a.splits, PAIRS);
    const int lo = (item % a.splits) * a.per, hi = lo + a.per;
    int first = 0;
    _Pragma("unroll") for (int n = 0; n < 2; ++n) {
        const QkSide& s = a.side[n];
        const int h0 = max(lo - first, 0), h1 = min(hi - first, s.H);
        first += s.H;
        if (h0 >= h1) continue;
        float c[E], sp[E];
        _Pragma("unroll") for (int i = 0; i < E; ++i) {
            c[i] = s.scale * ln.cs[i] * (s.w ? s.w[ln.f0 + i] : 1.f);
            sp[i] = s.scale * ln.sn[i] * (s.w ? s.w[ln.partner_feature(i, PAIRS)] : 1.f);
        }
        const TIO* x = static_cast<const TIO*>(s.x) + ln.at(s.xs);
        TIO* y = static_cast<TIO*>(s.y) + ln.at(s.ys);
        for (int h = h0; h < h1; h += kAhead) {
            u32x4 raw[kAhead];
            _Pragma("unroll") for (int u = 0; u < kAhead; ++u)
                if (h + u < h1) raw[u] = row_load(x + (h + u) * s.xs.head);
            _Pragma("unroll") for (int u = 0; u < kAhead; ++u) {
                if (h + u >= h1) break;
                float v[E], vp[E];
                unpack(raw[u], v);
                partners<PAIRS>(raw[u], ln.partner, ln.turned, vp);
                float r = 1.f;
                if (a.norm != LSM_NORM_NONE) {
                    float ss = 0.f;
                    _Pragma("unroll") for (int i = 0; i < E; ++i) ss += v[i] * v[i];
                    ss = group_sum<Lane::L>(ss);
                    r = rsqrtf((a.norm == LSM_NORM_RMS ? ss * (1.f / D) : ss) + a.eps);
                }
                _Pragma("unroll") for (int i = 0; i < E; ++i) v[i] = r * (v[i] * c[i] + vp[i] * sp[i]);
                if (ln.live) row_store(y + (h + u) * s.ys.head, pack(v));
            }
        }
    }
}

// Backward: u = scale R_p^T dy, z = w * u, dx = r (z - r x (r x . z) / d) (L2: without the 1 / d; no norm: z), dw = sum over rows of u * r x.
// The rows of x and dy are read once; a lane adds up its features' part of dw over all its rows, the workgroup's lanes are
// joined at its end and k_qk_weights sums the workgroups in a fixed order.
template <typename TIO, int D, bool PAIRS>
__global__ __launch_bounds__(256) void k_qk_bwd(QkArgs a) {
    typedef QkLane<TIO, D> Lane;
    constexpr int E = Lane::E;
    __shared__ float joined[2][4][D];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    float dw[2][E];
    _Pragma("unroll") for (int i = 0; i < E; ++i) dw[0][i] = dw[1][i] = 0.f;
    for (int item = int(blockIdx.x) * 4 + wave; item < a.groups * a.splits; item += int(gridDim.x) * 4) {
        const Lane ln(a, item / a.splits, PAIRS);
        const int lo = (item % a.splits) * a.per, hi = lo + a.per;
        int first = 0;
        _Pragma("unroll") for (int n = 0; n < 2; ++n) {
            const QkSide& s = a.side[n];
            const int h0 = max(lo - first, 0), h1 = min(hi - first, s.H);
            first += s.H;
            if (h0 >= h1) continue;
            float w[E], ct[E], st[E];
            _Pragma("unroll") for (int i = 0; i < E; ++i) {
                w[i] = s.w ? s.w[ln.f0 + i] : 1.f;
                ct[i] = s.scale * ln.cs[i];
                st[i] = -s.scale * ln.sn[i];
            }
            const TIO* x = static_cast<const TIO*>(s.x) + ln.at(s.xs);
            const TIO* g = static_cast<const TIO*>(s.g) + ln.at(s.gs);
            TIO* dx = static_cast<TIO*>(s.y) + ln.at(s.ys);
            for (int h = h0; h < h1; h += kAhead) {
                u32x4 rx[kAhead], rg[kAhead];
                _Pragma("unroll") for (int u = 0; u < kAhead; ++u) {
                    rx[u] = rg[u] = u32x4{0, 0, 0, 0};  // a row past the last token adds nothing to dw
                    if (h + u < h1 && ln.live) {
                        rx[u] = row_load(x + (h + u) * s.xs.head);
                        rg[u] = row_load(g + (h + u) * s.gs.head);
                    }
                }
                _Pragma("unroll") for (int u = 0; u < kAhead; ++u) {
                    if (h + u >= h1) break;
                    float v[E], z[E], zp[E];
                    unpack(rx[u], v);
                    unpack(rg[u], z);
                    partners<PAIRS>(rg[u], ln.partner, ln.turned, zp);
                    float ss = 0.f, along = 0.f, r = 1.f;
                    _Pragma("unroll") for (int i = 0; i < E; ++i) {
                        z[i] = z[i] * ct[i] + zp[i] * st[i];
                        ss += v[i] * v[i];
                        along += v[i] * (z[i] * w[i]);
                    }
                    if (a.norm != LSM_NORM_NONE) {
                        ss = group_sum<Lane::L>(ss);
                        along = group_sum<Lane::L>(along);
                        r = rsqrtf((a.norm == LSM_NORM_RMS ? ss * (1.f / D) : ss) + a.eps);
                        along *= a.norm == LSM_NORM_RMS ? r * r * (1.f / D) : r * r;
                    }
                    _Pragma("unroll") for (int i = 0; i < E; ++i) {
                        dw[n][i] += z[i] * (r * v[i]);
                        // without a norm x does not enter, whatever it is
                        z[i] = a.norm != LSM_NORM_NONE ? r * (z[i] * w[i] - v[i] * along) : z[i] * w[i];
                    }
                    if (ln.live) row_store(dx + (h + u) * s.ys.head, pack(z));
                }
            }
        }
    }
    if (!a.part) return;
    _Pragma("unroll") for (int n = 0; n < 2; ++n)
        _Pragma("unroll") for (int i = 0; i < E; ++i) {
            _Pragma("unroll") for (int m = Lane::L; m < 64; m *= 2) dw[n][i] += __shfl_xor(dw[n][i], m, 64);
            if (lane < Lane::L) joined[n][wave][lane * E + i] = dw[n][i];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += 256) {
        const int n = i / D, f = i % D;
        a.part[(size_t(n) * gridDim.x + blockIdx.x) * D + f] =
            (joined[n][0][f] + joined[n][1][f]) + (joined[n][2][f] + joined[n][3][f]);
    }
}

// dw of 16 features of q (blockIdx.y = 0) or k: 64 rows of threads over the workgroups' sums, then a tree.
__global__ __launch_bounds__(1024) void k_qk_weights(const float* part, int n, int D, float* dq_w, float* dk_w) {
    __shared__ float s[64][17];
    float* out = blockIdx.y ? dk_w : dq_w;
    if (!out) return;
    const int c = threadIdx.x & 15, r = threadIdx.x >> 4, f = int(blockIdx.x) * 16 + c;
    const float* p = part + size_t(blockIdx.y) * n * D + f;
    float x = 0.f;
    for (int i = r; i < n; i += 64) x += p[size_t(i) * D];
    s[r][c] = x;
    _Pragma("unroll") for (int m = 32; m > 0; m /= 2) {
        __syncthreads();
        if (r < m) s[r][c] += s[r + m][c];
    }
    if (r == 0) out[f] = s[0][c];
}

constexpr int kWaves = 4096;        // waves wanted: heads of a token are split over several where tokens are few
// Most workgroups of the backward kernel, each of which leaves 2 d sums: two a compute unit, eight rows of x and dy on their way in
// each of eight waves (B=4, T=8192, 16 + 16 heads of 128: 256: 196 us, 512: 174, 1024: 206, 2048: 187 and 7 more for the sums).
constexpr int kBwdGroups = 512;

int rows_per_wave(const lsm_qk_params& p) { return 64 / (p.d / (p.dtype == LSM_DTYPE_BF16 ? 8 : 4)); }

void plan(const lsm_qk_params& p, QkArgs& a) {
    const int heads = p.H_q + p.H_k, rows = rows_per_wave(p);
    a.groups = int((int64_t(p.B) * p.T + rows - 1) / rows);
    const int splits = a.groups >= kWaves ? 1 : (kWaves + a.groups - 1) / a.groups;
    a.per = splits >= heads ? 1 : (heads + splits - 1) / splits;
    a.splits = (heads + a.per - 1) / a.per;
}
int bwd_groups(const QkArgs& a) {
    const int64_t blocks = (int64_t(a.groups) * a.splits + 3) / 4;
    return int(blocks < kBwdGroups ? blocks : kBwdGroups);
}

bool stride_ok(const lsm_qk_params& p, const lsm_strides& s, int H) {
    const int64_t piece = p.dtype == LSM_DTYPE_BF16 ? 8 : 4;
    return (p.B == 1 || s.batch % piece == 0) && (H == 1 || s.head % piece == 0) && (p.T == 1 || s.token % piece == 0);
}

// Whether no two of a result's rows share an element (those of inputs may: an expanded gradient has strides of 0).
bool writable(const lsm_qk_params& p, const lsm_strides& s, int H) {
    struct Axis { int64_t n; __int128 step; };
    Axis axis[3] = {{p.B, s.batch}, {H, s.head}, {p.T, s.token}};
    for (Axis& a : axis) a.step = a.n == 1 ? 0 : a.step < 0 ? -a.step : a.step;
    // Axes in which each holds all of what the smaller ones reach: any order of a dense tensor, and slices of it.
    std::sort(axis, axis + 3, [](const Axis& x, const Axis& y) { return x.step < y.step; });
    __int128 reach = p.d;
    bool nested = true;
    for (const Axis& a : axis) {
        nested = nested && (a.n == 1 || a.step >= reach);
        reach += a.step * (a.n - 1);
    }
    if (nested) return true;
    if (__int128(p.B) * H * p.T * p.d > reach) return false;
    // Two rows are apart by (x, y, z) steps of the axes: for every x, y of the two shorter axes the z that brings them nearest.
    std::sort(axis, axis + 3, [](const Axis& x, const Axis& y) { return x.n < y.n; });
    const Axis& last = axis[2];
    if (last.step < p.d) return false;
    for (int64_t x = 0; x < axis[0].n; ++x)
        for (int64_t y = 1 - axis[1].n; y < axis[1].n; ++y) {
            if (x == 0 && y == 0) continue;
            const __int128 at = axis[0].step * x + axis[1].step * y, size = at < 0 ? -at : at;
            __int128 z = size / last.step;
            if (z > last.n - 1) z = last.n - 1;
            if (size - z * last.step < p.d || (z + 1 < last.n && (z + 1) * last.step - size < p.d)) return false;
        }
    return true;
}

// Results at their input's own address: the same rows in the same places, or some wave's results meet rows that another has yet to read.
bool in_place_ok(const lsm_qk_params& p, const void* x, const lsm_strides& xs, const void* y, const lsm_strides& ys, int H) {
    return x != y || ((p.B == 1 || xs.batch == ys.batch) && (H == 1 || xs.head == ys.head) && (p.T == 1 || xs.token == ys.token));
}

int check(const lsm_qk_params* p, bool backward) {
    if (!p) return LSM_ERR_NULL;
    if (p->struct_size != sizeof(lsm_qk_params)) return LSM_ERR_SHAPE;
    if (p->B < 1 || p->T < 1 || p->H_q < 1 || p->H_k < 0 || p->rot_dim < 0 || p->n_pos < 0) return LSM_ERR_SHAPE;
    if (p->dtype != LSM_DTYPE_F32 && p->dtype != LSM_DTYPE_BF16) return LSM_ERR_UNSUPPORTED;
    if (p->d != 64 && p->d != 128 && p->d != 256) return LSM_ERR_UNSUPPORTED;
    if (p->norm < LSM_NORM_NONE || p->norm > LSM_NORM_L2) return LSM_ERR_UNSUPPORTED;
    if (p->rotation != LSM_ROT_HALVES && p->rotation != LSM_ROT_PAIRS) return LSM_ERR_UNSUPPORTED;
    if (p->rot_dim % 16 != 0 || p->rot_dim > p->d || p->reserved != 0) return LSM_ERR_UNSUPPORTED;
    if (p->norm != LSM_NORM_NONE && !(p->eps > 0.f && p->eps < 3e38f)) return LSM_ERR_SHAPE;
    // the work items (token groups x head ranges) are counted in 32 bits
    if (int64_t(p->B) * p->T > (1 << 30) || int64_t(p->H_q) + p->H_k > (1 << 20)) return LSM_ERR_SHAPE;
    if (p->rot_dim && p->n_pos < 1) return LSM_ERR_SHAPE;
    if (!stride_ok(*p, p->q, p->H_q) || !stride_ok(*p, p->q_out, p->H_q) || (backward && !stride_ok(*p, p->dq, p->H_q)))
        return LSM_ERR_ALIGN;
    if (p->H_k && (!stride_ok(*p, p->k, p->H_k) || !stride_ok(*p, p->k_out, p->H_k) || (backward && !stride_ok(*p, p->dk, p->H_k))))
        return LSM_ERR_ALIGN;
    return LSM_OK;
}

int check_pointers(const lsm_qk_params& p, const void* q, const void* k, const float* qw, const float* kw, const float* cos_sin,
                   const int32_t* positions) {
    if (!q || (p.H_k > 0) != (k != nullptr) || (!k && kw)) return LSM_ERR_NULL;
    if ((p.rot_dim > 0) != (cos_sin != nullptr)) return LSM_ERR_NULL;
    if (p.rot_dim && !positions && p.T > p.n_pos) return LSM_ERR_SHAPE;
    if (misaligned(q) || misaligned(k) || misaligned(qw) || misaligned(kw) || misaligned(cos_sin) || misaligned(positions))
        return LSM_ERR_ALIGN;
    return LSM_OK;
}

QkArgs arguments(const lsm_qk_params& p, const void* q, const void* k, const float* qw, const float* kw, const float* cos_sin,
                 const int32_t* positions) {
    QkArgs a{};
    a.side[0] = QkSide{q, nullptr, nullptr, qw, p.q_scale, p.H_q, p.q, p.q_out, p.q_out};
    a.side[1] = QkSide{k, nullptr, nullptr, kw, p.k_scale, p.H_k, p.k, p.k_out, p.k_out};
    a.T = p.T;
    a.tokens = p.B * p.T;
    a.rot = p.rot_dim; a.n_pos = p.n_pos; a.norm = p.norm; a.eps = p.eps;
    a.cos_sin = cos_sin; a.positions = positions;
    plan(p, a);
    return a;
}

template <typename TIO, int D>
void launch(const QkArgs& a, bool pairs, bool backward, int blocks, hipStream_t st) {
    ProfScope ps(backward ? KID_QK_BWD : KID_QK, st);
    if (!backward && pairs) hipLaunchKernelGGL((k_qk<TIO, D, true>), dim3(blocks), dim3(256), 0, st, a);
    else if (!backward) hipLaunchKernelGGL((k_qk<TIO, D, false>), dim3(blocks), dim3(256), 0, st, a);
    else if (pairs) hipLaunchKernelGGL((k_qk_bwd<TIO, D, true>), dim3(blocks), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_qk_bwd<TIO, D, false>), dim3(blocks), dim3(256), 0, st, a);
}
template <typename TIO>
void launch(const lsm_qk_params& p, const QkArgs& a, bool backward, int blocks, hipStream_t st) {
    const bool pairs = p.rotation == LSM_ROT_PAIRS;
    if (p.d == 64) launch<TIO, 64>(a, pairs, backward, blocks, st);
    else if (p.d == 128) launch<TIO, 128>(a, pairs, backward, blocks, st);
    else launch<TIO, 256>(a, pairs, backward, blocks, st);
}

}  // namespace
}  // namespace lsm

extern "C" {

int lsm_qk_norm_rope(const lsm_qk_params* p, const void* q, const void* k, const float* q_weight, const float* k_weight,
                     const float* cos_sin, const int32_t* positions, void* q_out, void* k_out, void* stream) {
    using namespace lsm;
    int rc = check(p, false);
    if (rc == LSM_OK) rc = check_pointers(*p, q, k, q_weight, k_weight, cos_sin, positions);
    if (rc != LSM_OK) return rc;
    if (!q_out || (p->H_k > 0) != (k_out != nullptr)) return LSM_ERR_NULL;
    QkArgs a = arguments(*p, q, k, q_weight, k_weight, cos_sin, positions);
    const int64_t blocks = (int64_t(a.groups) * a.splits + 3) / 4;
    if (blocks * 256 > kAxisThreads) return LSM_ERR_SHAPE;
    if (!writable(*p, p->q_out, p->H_q) || (p->H_k && !writable(*p, p->k_out, p->H_k))) return LSM_ERR_SHAPE;
    if (!in_place_ok(*p, q, p->q, q_out, p->q_out, p->H_q) || (p->H_k && !in_place_ok(*p, k, p->k, k_out, p->k_out, p->H_k)))
        return LSM_ERR_SHAPE;
    if (misaligned(q_out) || misaligned(k_out)) return LSM_ERR_ALIGN;
    a.side[0].y = q_out;
    a.side[1].y = k_out;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (p->dtype == LSM_DTYPE_BF16) launch<uint16_t>(*p, a, false, int(blocks), st);
    else launch<float>(*p, a, false, int(blocks), st);
    return launched() ? LSM_OK : LSM_ERR_LAUNCH;
}

size_t lsm_qk_norm_rope_bwd_workspace_bytes(const lsm_qk_params* p) {
    using namespace lsm;
    if (check(p, true) != LSM_OK) return 0;
    QkArgs a{};
    plan(*p, a);
    return align256(size_t(2) * bwd_groups(a) * p->d * sizeof(float));
}

int lsm_qk_norm_rope_bwd(const lsm_qk_params* p, const void* q, const void* k, const float* q_weight, const float* k_weight,
                         const float* cos_sin, const int32_t* positions, const void* d_q_out, const void* d_k_out, void* dq,
                         void* dk, float* d_q_weight, float* d_k_weight, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace lsm;
    int rc = check(p, true);
    if (rc == LSM_OK) rc = check_pointers(*p, q, k, q_weight, k_weight, cos_sin, positions);
    if (rc != LSM_OK) return rc;
    const bool has_k = p->H_k > 0;
    if (!d_q_out || !dq || has_k != (d_k_out != nullptr) || has_k != (dk != nullptr)) return LSM_ERR_NULL;
    if ((d_q_weight && !q_weight) || (d_k_weight && !k_weight)) return LSM_ERR_NULL;
    if (misaligned(d_q_out) || misaligned(d_k_out) || misaligned(dq) || misaligned(dk) || misaligned(d_q_weight) ||
        misaligned(d_k_weight) || misaligned(workspace))
        return LSM_ERR_ALIGN;
    if (!writable(*p, p->dq, p->H_q) || (has_k && !writable(*p, p->dk, p->H_k))) return LSM_ERR_SHAPE;
    if (!workspace || workspace_bytes < lsm_qk_norm_rope_bwd_workspace_bytes(p)) return LSM_ERR_WORKSPACE;
    QkArgs a = arguments(*p, q, k, q_weight, k_weight, cos_sin, positions);
    a.side[0].g = d_q_out; a.side[0].y = dq; a.side[0].ys = p->dq;
    a.side[1].g = d_k_out; a.side[1].y = dk; a.side[1].ys = p->dk;
    const bool weights = d_q_weight || d_k_weight;
    a.part = weights ? static_cast<float*>(workspace) : nullptr;
    const int blocks = bwd_groups(a);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (p->dtype == LSM_DTYPE_BF16) launch<uint16_t>(*p, a, true, blocks, st);
    else launch<float>(*p, a, true, blocks, st);
    if (!launched()) return LSM_ERR_LAUNCH;
    if (weights) {
        ProfScope ps(KID_QK_WEIGHTS, st);
        hipLaunchKernelGGL(k_qk_weights, dim3(p->d / 16, 2), dim3(1024), 0, st, a.part, blocks, p->d, d_q_weight, d_k_weight);
        if (!launched()) return LSM_ERR_LAUNCH;
    }
    return LSM_OK;
}

}  // extern "C"
