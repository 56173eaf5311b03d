// Matrix products of the training operators (lsm_train.h): one workgroup forms a tile out[r][c] = sum_k R[r][k] C[c][k], the c
// of which lie next to each other in memory, with either operand by rows ([i][k], k contiguous) or by columns ([k][i], i
// contiguous), rows taken through a list where one is given.
//
// The product is formed as C R^T: c is the first operand of the 16 x 16 matrix instructions, so that a lane holds one row r and four
// neighbouring c's in four registers, and what is done along a row (maximum, sum, gate with factor) stays in a few lanes.  (With all
// matrix cores busy the clock is bound by power: from registers alone 16 x 16 x 32 reaches 1.9 PFLOP/s here, 32 x 32 x 16 1.7.)
//
// Pieces of 64 bytes of k a row (32 of bf16, 16 of fp32) go straight from memory into LDS, NBUF of them in a ring, 16 bytes a lane;
// a lane that has nothing to load (behind the last row, behind the last k) asks beyond the buffer's bound and gets zeros.
// Where a lane's 16 bytes land is fixed by the hardware (one after the other), so rows are spread over the banks by which
// 16 bytes of the row a lane asks for: slot s of row i holds piece s ^ f(i).  (By the counters no clock of LDS goes to bank conflicts in 256 x 256 tiles that follow one
// another, up to 0.055 of its clocks in others, whose results pass through rows 16 bytes further apart than they are long; with conflicts in the
// steps the clocks of LDS double.)
//
// Bound by the matrix cores: from registers alone the instruction reaches 1.9 PFLOP/s here, the steps of a 256 x 256 tile 1.4, a whole product
// 0.84 to 1.25 with its start, its results and a last round of tiles that is not full (a large library product 1.17 to 1.42).  fp32
// products are bound by the instruction's 154 TFLOP/s, of which long ones reach 117.
// Where tiles follow one another in a workgroup there are as many workgroups as there is room for.
//
// While the matrix instructions of step t run, the operands of step t + 1 are read, each into the registers whose last use has just
// been: piece t + 1 is complete before step t begins, piece t + NBUF - 1 is requested in it, and nothing is read from piece t.
#pragma once
#include "lsm_train_dev.h"

namespace lsm {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kBeyond = 0xfffff000u;  // offset and size of a buffer: at or behind it nothing is read and zeros come
constexpr int kStepBytes = kTileStepBytes;

enum Layout { BY_ROWS, BY_COLS };

template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }
__device__ __forceinline__ void fence_schedule() { __builtin_amdgcn_sched_barrier(0); }

__device__ __forceinline__ uint64_t uniform(uint64_t x) {
    return uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(x))))) |
           uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(x >> 32))))) << 32;
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// 16 bytes a lane from base + offset to LDS address `to` + 16 lane.  `base` and `to` are the same in all lanes.  (In assembly, so that the
// waits are those written below and not one for every read of LDS.  m0 is set and used here; nothing else in these kernels
// holds a value in it: no register is indexed by a variable.)
__device__ __forceinline__ void load_to_lds(uint64_t base, uint32_t offset, uint32_t to) {
    const uint64_t from = uniform(base);
    const u32x4 buffer = {uint32_t(from), uint32_t(from >> 32) & 0xffffu, kBeyond, 0x00020000u};
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(buffer)
                 : "memory");
}
// The same with 4 bytes a lane, to `to` + 4 lane.
__device__ __forceinline__ void load4_to_lds(uint64_t base, uint32_t offset, uint32_t to) {
    const uint64_t from = uniform(base);
    const u32x4 buffer = {uint32_t(from), uint32_t(from >> 32) & 0xffffu, kBeyond, 0x00020000u};
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(buffer) : "memory");
}
// One step of a 16 x 16 product: both operands hold, in lane l, 16 bytes of row l % 16 from byte 16 (l / 16) of the step on.
__device__ __forceinline__ f32x4 product(const u32x4& a, const u32x4& b, f32x4 c, uint16_t) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 product(const u32x4& a, const u32x4& b, f32x4 c, float) {
    _Pragma("unroll") for (int i = 0; i < 4; ++i)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
    return c;
}

// N rows of an operand and a step's k of each, as a workgroup of WAVES waves brings them to LDS and reads them.
template <typename TIO, Layout L, int N, int WAVES, bool LISTED>
struct Operand {
    static constexpr int EL = int(sizeof(TIO)), KSTEP = kStepBytes / EL, BYTES = N * kStepBytes;
    static constexpr int PIECES = N / 16, LOADS = PIECES >= WAVES ? PIECES / WAVES : 1;  // 1 KiB a load; of a wave
    static_assert(N % 32 == 0 && (PIECES % WAVES == 0 || WAVES % PIECES == 0), "even shares");
    static constexpr int kList = 2048;  // rows of a list that are in LDS at a time
    static constexpr int LINE = L == BY_ROWS ? kStepBytes : N * EL;   // bytes of a line in LDS
    static constexpr int LANES = LINE / 16, LINES = 64 / LANES;       // lanes of a line, lines of a load
    // By columns slot s of line k holds piece s ^ turn(k): the lines k .. k + 3 and k + 8 .. k + 11 that half a wave reads at a time, 32
    // bytes of each, lie in different banks; of fp32 the lines k, k + 4, k + 8 and k + 12, 64 bytes of each.
    static __device__ __forceinline__ int turn(int k) {
        const int low = LINE >= 256 ? k & 3 : LINE == 128 ? (k >> 1) & 1 : 0, bits = LINE >= 256 ? 2 : LINE == 128 ? 1 : 0;
        if (EL == 4) return 4 * ((k >> 2) & (LINE >= 256 ? 3 : LINE == 128 ? 1 : 0));
        return 2 * (low | ((k >> 3) & 1) << bits);
    }

    uint64_t base;
    uint32_t off[LOADS];
    int row_bytes;
    int list;             // LDS address of the list of rows (LISTED, by columns)
    uint32_t row[LOADS];  // LISTED: the rows of the next request

    __device__ __forceinline__ static int piece(int wave, int j) { return (wave * LOADS + j) % PIECES; }
    // the row (by rows) or the first of eight (four) neighbouring ones (by columns) that load j of this lane brings
    __device__ __forceinline__ static int mine(int wave, int lane, int j) {
        if (L == BY_ROWS) return piece(wave, j) * LINES + lane / LANES;
        return ((lane % LANES) ^ turn(line(wave, lane, j))) * (16 / EL);
    }
    __device__ __forceinline__ static int line(int wave, int lane, int j) { return piece(wave, j) * LINES + lane / LANES; }
    // By rows slot s of row i holds piece s ^ 2 (i / 8 % 2): a wave reads 16 lanes at a time, of which those of rows 0..3 and 12..15 and those
    // of rows 4..11 go together, the latter one piece further on.
    __device__ __forceinline__ static int k_piece(int lane) { return (lane & 3) ^ (2 * (lane >> 5)); }

    // By rows: row_at(i) is the row's offset in bytes from `from` (kBeyond: none) for i of the tile.
    template <typename RowAt>
    __device__ __forceinline__ void start_rows(const void* from, int wave, int lane, RowAt row_at) {
        base = uniform(reinterpret_cast<uint64_t>(from));
        _Pragma("unroll") for (int j = 0; j < LOADS; ++j) {
            const uint32_t at = row_at(mine(wave, lane, j));
            off[j] = at == kBeyond ? kBeyond : at + 16 * k_piece(lane);
        }
    }
    // By columns: columns first .. first + N of [k][..] rows of `stride` bytes, `width` columns in all.
    __device__ __forceinline__ void start_cols(const void* from, int stride, int first, int width, int wave, int lane, int rows_at) {
        base = uniform(reinterpret_cast<uint64_t>(from)) + uint64_t(first) * EL;
        row_bytes = stride;
        list = rows_at;
        _Pragma("unroll") for (int j = 0; j < LOADS; ++j) {
            const int c = mine(wave, lane, j);
            off[j] = first + c < width ? uint32_t(c * EL) + (LISTED ? 0u : uint32_t(line(wave, lane, j)) * uint32_t(stride)) : kBeyond;
        }
    }
    __device__ __forceinline__ uint32_t listed(int k) const {
        return *reinterpret_cast<__attribute__((address_space(3))) const uint32_t*>(uintptr_t(list + 4 * (k % kList)));
    }
    __device__ __forceinline__ void first_rows(int wave, int lane) {
        _Pragma("unroll") for (int j = 0; j < LOADS; ++j) row[j] = LISTED ? listed(line(wave, lane, j)) : 0;
    }
    // Request load j of the pieces from k0 on, of K k's; nothing behind the last.
    __device__ __forceinline__ void request(uint32_t to, int k0, int K, int wave, int lane, int j) {
        uint32_t o = off[j];
        uint64_t from = base;
        if (L == BY_ROWS) {
            if (k0 + k_piece(lane) * (16 / EL) >= K) o = kBeyond;
            from += uint64_t(k0) * EL;
        } else {
            const int k = k0 + line(wave, lane, j);
            if (LISTED) {
                const uint32_t at = o + row[j] * uint32_t(row_bytes);
                o = o == kBeyond ? kBeyond : at;
                row[j] = listed(k + KSTEP);
            } else {
                from += uint64_t(k0) * uint64_t(uint32_t(row_bytes));
            }
            if (k >= K) o = kBeyond;
        }
        load_to_lds(from, o, uniform(int(to + piece(wave, j) * 1024)));
    }

    // Rows first .. first + 15 as an operand.
    __device__ __forceinline__ static u32x4 read(uint32_t at, int first, int lane) {
        const int r = lane & 15, q = lane >> 4;
        if (L == BY_ROWS)
            return *reinterpret_cast<__attribute__((address_space(3))) const u32x4*>(
                uintptr_t(at + first * kStepBytes + r * kStepBytes + ((q ^ (2 * (r >> 3))) * 16)));
        if (EL == 4) {
            u32x4 v;
            const uint32_t p = at + 4 * q * LINE + (((first + r) >> 2) ^ turn(4 * q)) * 16 + (r & 3) * 4;
            _Pragma("unroll") for (int i = 0; i < 4; ++i)
                v[i] = *reinterpret_cast<__attribute__((address_space(3))) const uint32_t*>(uintptr_t(p + i * LINE));
            return v;
        }
        // 16 lanes read four lines' 16 columns and get a column of four lines each
        const int k = 8 * q + (r >> 2), slot = ((first >> 3) + ((r >> 1) & 1)) ^ turn(k);
        const uint32_t p = at + k * LINE + slot * 16 + 8 * (r & 1);
        typedef s16x4 __attribute__((address_space(3))) * tr_t;
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)(uintptr_t(p))));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)(uintptr_t(p + 4 * LINE))));
        return u32x4{lo.x, lo.y, hi.x, hi.y};
    }
};

// What rounding x to bf16 leaves; nothing where it is not finite.
__device__ __forceinline__ float remainder_of(float x) {
    const float r = x - bf16_lo(pack2(x, 0.f));
    return fabsf(r) < __builtin_inff() ? r : 0.f;
}

// A tile: WC x WR waves of TC x TR blocks of 16 x 16.  FOLLOWED: the workgroup goes on to another tile with the same kinds of operands and
// the same K; the first pieces of that one are requested in the last steps of this one, and come while its results are written.
template <typename TIO_, Layout LC, Layout LR, int WC_, int WR_, int TC_, int TR_, int NBUF_, bool LIST_C = false, bool LIST_R = false,
          bool FOLLOWED_ = false>
struct Tile {
    typedef TIO_ TIO;
    static constexpr bool FOLLOWED = FOLLOWED_;
    static constexpr int WC = WC_, WR = WR_, TC = TC_, TR = TR_, NBUF = NBUF_, WAVES = WC * WR, THREADS = 64 * WAVES;
    static constexpr int BC = WC * TC * 16, BR = WR * TR * 16;
    typedef Operand<TIO, LC, BC, WAVES, LIST_C> C;
    typedef Operand<TIO, LR, BR, WAVES, LIST_R> R;
    static constexpr int STAGE = C::BYTES + R::BYTES, LOADS = C::LOADS + R::LOADS, AHEAD = NBUF - 1, RING = NBUF * STAGE;
    static constexpr int LIST = LIST_C || LIST_R ? 4 * C::kList : 0, ROWS = FOLLOWED ? 4 * BR : 0;  // the following tile's rows
    static constexpr int LDS = RING + LIST + ROWS;
    static_assert(LDS <= 160 * 1024 && NBUF >= 3 && !(FOLLOWED && LIST), "LDS");
    // Results on their way out: 16 rows of CHUNK of a wave's blocks at a time, in fp32; each wave has its own place in the ring, where
    // another tile follows in the one piece of it that nothing is on its way to.
    static constexpr int CHUNK = FOLLOWED && TC > 4 ? 4 : TC, PAD = FOLLOWED ? 0 : 16;
    static_assert(WAVES * 16 * (64 * CHUNK + PAD) <= (FOLLOWED ? STAGE : RING), "LDS");

    C c, c2;
    R r, r2;
    int wave, lane, wc, wr, slot = 0;  // slot: of step 0 in the ring
    bool ahead = false;                // the first pieces are there
    uint32_t lds;

    __device__ __forceinline__ Tile(const char* shared) {
        wave = uniform(int(threadIdx.x >> 6));
        lane = threadIdx.x & 63;
        wc = wave % WC;
        wr = wave / WC;
        lds = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)shared));
    }
    __device__ __forceinline__ uint32_t list_at() const { return lds + RING; }
    __device__ __forceinline__ uint32_t at(int step) const { return lds + uint32_t((slot + step) % NBUF) * STAGE; }

    // The numbers list[i] for rows i < n of the following tile, to LDS, and one of them.
    __device__ __forceinline__ void bring(const int32_t* list, int n) const {
        if (wave < (BR + 63) / 64)
            load4_to_lds(reinterpret_cast<uint64_t>(list), 64 * wave + lane < n ? uint32_t(4 * (64 * wave + lane)) : kBeyond,
                         uniform(int(lds + RING + LIST + 256 * wave)));
    }
    __device__ __forceinline__ int brought(int i) const {
        return *reinterpret_cast<__attribute__((address_space(3))) const int*>(uintptr_t(lds + RING + LIST + 4 * i));
    }

    // Load n of step t of `steps`; behind them of the following tile's.
    __device__ __forceinline__ void request(int t, int steps, int K, int n) {
        const bool own = !FOLLOWED || t < steps;
        const int k0 = (own ? t : t - steps) * C::KSTEP;
        if (n < C::LOADS) {
            if constexpr (FOLLOWED) {
                C x = c;
                x.base = own ? c.base : c2.base;
                x.off[n] = own ? c.off[n] : c2.off[n];
                x.request(at(t), k0, K, wave, lane, n);
            } else {
                c.request(at(t), k0, K, wave, lane, n);
            }
        } else {
            const int m = n - C::LOADS;
            if constexpr (FOLLOWED) {
                R x = r;
                x.base = own ? r.base : r2.base;
                x.off[m] = own ? r.off[m] : r2.off[m];
                x.request(at(t) + C::BYTES, k0, K, wave, lane, m);
            } else {
                r.request(at(t) + C::BYTES, k0, K, wave, lane, m);
            }
        }
    }
    __device__ __forceinline__ u32x4 read_c(int step, int i) const { return C::read(at(step), (wc * TC + i) * 16, lane); }
    __device__ __forceinline__ u32x4 read_r(int step, int j) const { return R::read(at(step) + C::BYTES, (wr * TR + j) * 16, lane); }
    // The rows of k0 .. k0 + n - 1 for an operand that is taken through a list.
    template <typename RowOf>
    __device__ __forceinline__ void fill(RowOf row_of, int k0, int n, int K) const {
        for (int k = k0 + int(threadIdx.x); k < min(k0 + n, K); k += THREADS)
            *reinterpret_cast<__attribute__((address_space(3))) uint32_t*>(uintptr_t(list_at() + 4 * (k % C::kList))) = row_of(k);
        wait_lds();
    }
    struct Nothing {
        __device__ __forceinline__ uint32_t operator()(int) const { return 0; }
        __device__ __forceinline__ void operator()() const {}
    };
    __device__ __forceinline__ void walk(f32x4 (&acc)[TC][TR], int K) { walk(acc, K, Nothing(), Nothing()); }
    template <typename RowOf>
    __device__ __forceinline__ void walk(f32x4 (&acc)[TC][TR], int K, RowOf row_of) { walk(acc, K, row_of, Nothing()); }

    // acc += the product over k = 0 .. K - 1; row_of(k): the row of k in a list; follow(): sets c2 and r2, called when what was brought
    // is there.  Begins with LDS free, but for what is ahead, and ends so.
    template <typename RowOf, typename Follow>
    __device__ __forceinline__ void walk(f32x4 (&acc)[TC][TR], int K, RowOf row_of, Follow follow) {
        int steps = (K + C::KSTEP - 1) / C::KSTEP;
        if (FOLLOWED) steps = max(steps, AHEAD + 2);  // so that two ends of steps are between bring() and follow()
        if (steps == 0) return;
        if (LIST) {
            fill(row_of, 0, C::kList, K);
            barrier();
            c.first_rows(wave, lane);
            r.first_rows(wave, lane);
        }
        if (!FOLLOWED || !ahead) {
            _Pragma("unroll") for (int s = 0; s < AHEAD; ++s)
                _Pragma("unroll") for (int n = 0; n < LOADS; ++n) request(s, steps, K, n);
            wait_loads<(AHEAD - 2) * LOADS>();
            barrier();
        }
        u32x4 a[TC], b[TR], next[TR];
        _Pragma("unroll") for (int j = 0; j < TR; ++j) b[j] = read_r(0, j);
        _Pragma("unroll") for (int i = 0; i < TC; ++i) a[i] = read_c(0, i);
        if constexpr (FOLD > 0) {
            f32x4 part[TC][TR];
            for (int t0 = 0; t0 < steps; t0 += FOLD) {
                _Pragma("unroll") for (int i = 0; i < TC; ++i)
                    _Pragma("unroll") for (int j = 0; j < TR; ++j) part[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
                walk_steps(part, a, b, next, t0, min(t0 + FOLD, steps), steps, K, row_of);
                _Pragma("unroll") for (int i = 0; i < TC; ++i)
                    _Pragma("unroll") for (int j = 0; j < TR; ++j) acc[i][j] += part[i][j];
            }
        } else if constexpr (FOLLOWED) {
            walk_steps(acc, a, b, next, 0, steps - AHEAD, steps, K, row_of);
            follow();
            walk_steps(acc, a, b, next, steps - AHEAD, steps, steps, K, row_of);
        } else {
            walk_steps(acc, a, b, next, 0, steps, steps, K, row_of);
        }
        slot = (slot + steps) % NBUF;
        if (!FOLLOWED) {
            wait_lds();
            wait_loads<0>();
            barrier();
        }
    }
    // fp32 elements: sums of 128 k's are added up apart, so that a sum over some thousand is as exact as one over a few hundred.
    static constexpr int FOLD = sizeof(TIO) == 4 ? 8 : 0;

    template <typename RowOf>
    __device__ __forceinline__ void walk_steps(f32x4 (&acc)[TC][TR], u32x4 (&a)[TC], u32x4 (&b)[TR], u32x4 (&next)[TR], int t0, int t1, int steps,
                                               int K, RowOf row_of) {
        int t = t0;
        if constexpr (TC == TR || FOLLOWED || LIST > 0) {
            for (; t < t1; ++t) lean_step(acc, a, b, t, steps, K, row_of);
        } else {
            for (; t + 1 < t1; t += 2) {
                step(acc, a, b, next, t, steps, K, row_of);
                step(acc, a, next, b, t + 1, steps, K, row_of);
            }
            if (t >= t1) return;
            step(acc, a, b, next, t, steps, K, row_of);
            _Pragma("unroll") for (int j = 0; j < TR; ++j) b[j] = next[j];
        }
    }
    template <typename RowOf>
    __device__ __forceinline__ void refill(RowOf row_of, int t, int K) const {
        if (!LIST) return;  // the next half of the list, a step before its first row is read; the half that it replaces is used up
        const int k = (t + AHEAD + 2) * C::KSTEP;
        if (k >= C::kList && k % (C::kList / 2) == 0) fill(row_of, k, C::kList / 2, K);
    }
    __device__ __forceinline__ void end_step(int t) const {
        if (!FOLLOWED || !ahead || t > 0) wait_loads<(AHEAD - 2) * LOADS>();  // piece t + 2 is there
        barrier();
    }
    // Reads and requests are spread among the matrix instructions: behind one another they keep the wave from its next product until the
    // last of them is accepted.
    template <typename RowOf>
    __device__ __forceinline__ void step(f32x4 (&acc)[TC][TR], u32x4 (&a)[TC], const u32x4 (&b)[TR], u32x4 (&next)[TR], int t, int steps, int K,
                                         RowOf row_of) {
        constexpr int ALL = TC * TR;
        refill(row_of, t, K);
        fence_schedule();
        _Pragma("unroll") for (int i = 0; i < TC; ++i)
            _Pragma("unroll") for (int j = 0; j < TR; ++j) {
                acc[i][j] = product(a[i], b[j], acc[i][j], TIO());
                fence_schedule();
                const int m = i * TR + j;
                _Pragma("unroll") for (int n = m * TR / ALL; n < (m + 1) * TR / ALL; ++n) next[n] = read_r(t + 1, n);
                _Pragma("unroll") for (int n = m * LOADS / ALL; n < (m + 1) * LOADS / ALL; ++n) request(t + AHEAD, steps, K, n);
                if (j == TR - 1) a[i] = read_c(t + 1, i);
                fence_schedule();
            }
        end_step(t);
    }
    // The same without a second set of registers for r: first all products with the first operand of the shorter side (and as many of the
    // longer one as belong to it), then those with the second and so on, so that operands are free, and read anew, long before all
    // products are formed.  (8 x 4 blocks alone, with registers to spare: 4 % slower, but through a list 2 % faster; followed, the second set costs 29 to 59
    // registers in scratch and 15 to 20 %.)
    template <typename RowOf>
    __device__ __forceinline__ void lean_step(f32x4 (&acc)[TC][TR], u32x4 (&a)[TC], u32x4 (&b)[TR], int t, int steps, int K, RowOf row_of) {
        constexpr int GROUPS = TC < TR ? TC : TR, A = TC / GROUPS, B = TR / GROUPS, ALL = TC * TR;
        refill(row_of, t, K);
        fence_schedule();
        int m = 0;
        const auto multiply = [&](int i, int j) {
            acc[i][j] = product(a[i], b[j], acc[i][j], TIO());
            fence_schedule();
            _Pragma("unroll") for (int n = m * LOADS / ALL; n < (m + 1) * LOADS / ALL; ++n) request(t + AHEAD, steps, K, n);
            fence_schedule();
            ++m;
        };
        _Pragma("unroll") for (int d = 0; d < GROUPS; ++d) {
            _Pragma("unroll") for (int j = d * B; j < (d + 1) * B; ++j)
                _Pragma("unroll") for (int i = d * A; i < TC; ++i) multiply(i, j);
            _Pragma("unroll") for (int j = d * B; j < (d + 1) * B; ++j) b[j] = read_r(t + 1, j);
            _Pragma("unroll") for (int j = (d + 1) * B; j < TR; ++j)
                _Pragma("unroll") for (int i = d * A; i < (d + 1) * A; ++i) multiply(i, j);
            _Pragma("unroll") for (int i = d * A; i < (d + 1) * A; ++i) a[i] = read_c(t + 1, i);
            fence_schedule();
        }
        end_step(t);
    }
    // On to the following tile, when all that this wave had to write is on its way.  Pieces are requested into its place of the ring next, so
    // what it wrote there is waited for: a wave that stores nothing (rows behind the last, columns behind the width) has read none of it back.
    __device__ __forceinline__ void go_on() {
        c = c2;
        r = r2;
        ahead = true;
        wait_lds();
        barrier();
    }

    // Values of block (i, j): element e of a lane is row(j), column 16 (wc TC + i) + 4 (lane / 16) + e of the tile.
    __device__ __forceinline__ int row(int j) const { return (wr * TR + j) * 16 + (lane & 15); }
    // Sum and maximum over the lanes of a row.
    static __device__ __forceinline__ float row_sum(float x) {
        x += __shfl_xor(x, 16, 64);
        return x + __shfl_xor(x, 32, 64);
    }
    static __device__ __forceinline__ float row_max(float x) {
        x = fmaxf(x, __shfl_xor(x, 16, 64));
        return fmaxf(x, __shfl_xor(x, 32, 64));
    }

    // Results to memory, whole lines at a time: row block j of N neighbouring blocks goes through the wave's own place in LDS and leaves
    // in 16-byte pieces.  Rows are 16 bytes further apart than they are long or, where there is no room for that, piece p of row r is at
    // p ^ r: neither the lanes of a column nor those of a row meet in a bank.
    template <int N> __device__ __forceinline__ uint32_t cell(int row16, int column) const {
        static_assert(N <= CHUNK, "the wave's own place");
        const uint32_t own = (FOLLOWED ? at(AHEAD) : lds) + uint32_t(wave) * (16 * (64 * CHUNK + PAD)) + uint32_t(row16) * (N * 64 + PAD);
        return own + uint32_t(FOLLOWED ? ((column >> 2) ^ (row16 % (4 * N))) * 16 + (column & 3) * 4 : column * 4);
    }
    // Between what lanes of a wave write there and what others read: no lane's part may be moved across, nor taken apart from the others' as
    // where branches follow one another on the same condition.
    static __device__ __forceinline__ void wave_meets() {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    // value(i): four results of block i of the N.
    template <int N, typename Value>
    __device__ __forceinline__ void put(Value value) const {
        wave_meets();
        _Pragma("unroll") for (int i = 0; i < N; ++i)
            *reinterpret_cast<__attribute__((address_space(3))) f32x4*>(uintptr_t(cell<N>(lane & 15, i * 16 + 4 * (lane >> 4)))) = value(i);
        wave_meets();
    }
    // line(r): where row r of the tile goes, from the first of the N blocks' columns on, or null; width: columns that there are from there on.
    // ADD: to what is there already (TOUT's own sum); REST: what rounding to bf16 leaves of the results.
    template <int N, typename TOUT, bool ADD = false, bool REST = false, typename Line>
    __device__ __forceinline__ void take(int j, int width, Line line) const {
        constexpr int E = 16 / int(sizeof(TOUT)), LANES = N * 16 / E, ROWS_ = 64 / LANES;
        wave_meets();
        _Pragma("unroll") for (int it = 0; it < (16 + ROWS_ - 1) / ROWS_; ++it) {
            const int row = it * ROWS_ + lane / LANES, c = (lane % LANES) * E;
            if (ROWS_ > 16 && row >= 16) continue;
            float v[E];
            _Pragma("unroll") for (int q = 0; q < E / 4; ++q) {
                const f32x4 x = *reinterpret_cast<__attribute__((address_space(3))) const f32x4*>(uintptr_t(cell<N>(row, c + 4 * q)));
                _Pragma("unroll") for (int e = 0; e < 4; ++e) v[4 * q + e] = REST ? remainder_of(x[e]) : x[e];
            }
            TOUT* to = line((wr * TR + j) * 16 + row);
            if (!to || c >= width) continue;
            if (ADD) {
                float old[E];
                unpack(*reinterpret_cast<const u32x4*>(to + c), old);
                _Pragma("unroll") for (int e = 0; e < E; ++e) v[e] += old[e];
            }
            *reinterpret_cast<u32x4*>(to + c) = pack(v);
        }
    }
    // What was requested ahead is there before the first result is written: a wait for it later would be one for the results too.
    __device__ __forceinline__ void settle() const {
        if (FOLLOWED) wait_loads<0>();
    }
    // B blocks, CHUNK at a time; width, line from the first of them on.
    template <int B, typename TOUT, bool ADD = false, typename Value, typename Line>
    __device__ __forceinline__ void store(int j, int width, Value value, Line line) const {
        constexpr int N = CHUNK < B ? CHUNK : B;
        _Pragma("unroll") for (int i0 = 0; i0 < B; i0 += N) {
            put<N>([&](int i) { return value(i0 + i); });
            if (j == 0 && i0 == 0) settle();
            take<N, TOUT, ADD>(j, width - i0 * 16, [&](int r) {
                TOUT* p = line(r);
                return p ? p + i0 * 16 : nullptr;
            });
        }
    }
};

// Tiles that are taken for few rows: they can hold two rows of a result, with what its rounding leaves.
template <typename T> constexpr bool kMayHalve = sizeof(typename T::TIO) == 2 && T::BR <= 64;

// 2^x and 1 / (1 + 2^-x) of x = log2(e) y.  For bf16 elements the hardware's power and reciprocal, each within 2^-23: what they give is
// rounded to bf16 or summed over many; for fp32 elements the library's functions.
constexpr float kLog2e = 1.442695041f;
__device__ __forceinline__ float power(float x, float) { return exp2f(x); }
__device__ __forceinline__ float power(float x, uint16_t) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float sigmoid(float y, float) { return 1.f / (1.f + expf(-y)); }
__device__ __forceinline__ float sigmoid(float y, uint16_t) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * y)); }

template <typename T>
__device__ __forceinline__ void clear(f32x4 (&acc)[T::TC][T::TR]) {
    _Pragma("unroll") for (int i = 0; i < T::TC; ++i)
        _Pragma("unroll") for (int j = 0; j < T::TR; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// The tiles there are, by number (kTiles in lsm_train_dev.h has their sizes).  HALF: half the columns, for columns that go with pairs of them.
template <typename TIO, Layout LC, Layout LR, int KIND, bool HALF = false, bool LIST_C = false, bool LIST_R = false, bool FOLLOWED = false> struct TileOf;
// (fp32 has no tile of 256 x 256: its sums are kept in two sets of registers.)
#define LSM_TILE(KIND, WC, WR, TC, TR)                                                                                      \
    template <typename TIO, Layout LC, Layout LR, bool HALF, bool LIST_C, bool LIST_R, bool FOLLOWED>                         \
    struct TileOf<TIO, LC, LR, KIND, HALF, LIST_C, LIST_R, FOLLOWED> {                                                                  \
        typedef Tile<TIO, LC, LR, WC, WR, HALF ? (TC) / 2 : (TC), TR, 4, LIST_C, LIST_R, FOLLOWED && (KIND) == 0> type;       \
        static_assert(kTiles[KIND].rows == (WR) * (TR) * 16 && kTiles[KIND].cols == (WC) * (TC) * 16 && kTiles[KIND].waves == (WC), ""); \
    }
LSM_TILE(0, 2, 4, 8, 4);
LSM_TILE(1, 4, 2, 4, 4);
LSM_TILE(2, 2, 2, 4, 4);
LSM_TILE(3, 4, 1, 4, 4);
LSM_TILE(4, 4, 1, 4, 2);
LSM_TILE(5, 2, 2, 2, 2);
LSM_TILE(6, 4, 1, 2, 2);
#undef LSM_TILE
template <Layout LC, Layout LR, bool HALF, bool LIST_C, bool LIST_R, bool FOLLOWED>
struct TileOf<float, LC, LR, 0, HALF, LIST_C, LIST_R, FOLLOWED> : TileOf<float, LC, LR, 2, HALF, LIST_C, LIST_R> {};
// FOLLOWED: the largest tiles, one workgroup a compute unit, on and on; the others' workgroups are each other's company.

}  // namespace
}  // namespace lsm
