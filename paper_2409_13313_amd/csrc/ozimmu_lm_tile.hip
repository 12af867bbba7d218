// Products of 16-bit matrices on the matrix cores in tiles of 256 x 256, and what the loss makes of their sums (ozimmu_lm.h, Kind).
#include "ozimmu_lm.h"
#include <type_traits>

namespace {

using namespace mxk;
using lmk::BAD_TARGET;
using lmk::Tile;

constexpr int64_t COMPUTE_UNITS = 256;
constexpr int NXCD = 8, TILE = 256, STAGE_K = 64;
constexpr int OPERAND_BYTES = TILE * STAGE_K * 2, PLACE_BYTES = 2 * OPERAND_BYTES, COPIES = 8;  // 32 KiB, 64 KiB; copies a wave and operand
constexpr float LOG2E = 1.44269504088896341f;

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) const v4i* lds_v4i;

template <int TYPE> __device__ inline v4f mfma(v4i b, v4i a, v4f c)
{
    if constexpr (TYPE == BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, b), __builtin_bit_cast(v8bf, a), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, b), __builtin_bit_cast(v8h, a), c, 0, 0, 0);
}

template <int I, int N, class F> __device__ __attribute__((always_inline)) inline void static_for(F&& f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<I + 1, N>(f);
    }
}

__device__ inline void wait_lds()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0), by the builtin: the compiler then knows
    asm volatile("" ::: "memory");
}
template <int N> __device__ inline void wait_vmcnt() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// M0: where in LDS the next copy goes.  (At least one instruction has to stand between this and the copy.)
template <int PART> __device__ inline void copy_to(uint32_t place) { asm volatile("s_add_u32 m0, %0, %1" ::"s"(place), "n"(PART) : "memory", "scc"); }
__device__ inline void copy(uint32_t voff, v4i source, uint32_t soff)
{
    asm volatile("buffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(voff), "s"(source), "s"(soff) : "memory");
}

// Rows (or columns) of a tile by fragment (0 .. 15) and place (0 .. 15): a lane's four sums of a product are four places in a row, so that with
// those of the next fragment it holds 8 neighbouring columns.
__host__ __device__ constexpr int row_of(int fragment, int place) { return fragment / 2 * 32 + place / 4 * 8 + fragment % 2 * 4 + place % 4; }

// What a kernel is given: sizes in tiles and stages, operands in bytes
struct Args {
    int64_t m, n, p, b_rows;
    uint64_t A, B;
    uint32_t lda, ldb;
    int TM, TP, KT, splits;
    void* D;
    int64_t ldd;
    int dtype;
    float alpha, beta;
    const float* alpha_at;
    int64_t split_stride;
    const int* targets;
    int column0;
    const float* lse2;
    float* at_target;
    float2* parts;
    int64_t parts_ld;
};

// Workgroup b runs on XCD b % 8.  The items (output tiles, for each split of the inner dimension) are cut into eight contiguous ranges, one an
// XCD, in bands of eight tile rows walked column by column: the 32 tiles that an XCD works on at a time share 8 panels of A and 4 of B in its L2.
struct Order {
    static constexpr int BAND = 8;
    int TM, TP, KT, splits, next, last, step;
    __device__ inline explicit Order(const Args& g) : TM(g.TM), TP(g.TP), KT(g.KT), splits(g.splits)
    {
        const int T = TM * TP * splits, xcd = blockIdx.x % NXCD, begin = xcd * (T / NXCD) + (xcd < T % NXCD ? xcd : T % NXCD);
        next = begin + blockIdx.x / NXCD;
        last = begin + T / NXCD + (xcd < T % NXCD ? 1 : 0);
        step = gridDim.x / NXCD + (xcd < (int)(gridDim.x % NXCD) ? 1 : 0);
    }
    // the next item of this workgroup: tile, split, and its stages k0 .. k1 - 1; false behind the last
    __device__ inline bool take(int& tm, int& tp, int& split, int& k0, int& k1)
    {
        if (next >= last) return false;
        const int s = next / (TM * TP), in_split = next % (TM * TP);
        const int band = in_split / (BAND * TP), in_band = in_split % (BAND * TP);
        const int height = TM - band * BAND < BAND ? TM - band * BAND : BAND;
        split = __builtin_amdgcn_readfirstlane(s);
        tm = __builtin_amdgcn_readfirstlane(band * BAND + in_band % height);
        tp = __builtin_amdgcn_readfirstlane(in_band / height);
        k0 = __builtin_amdgcn_readfirstlane((int)((int64_t)KT * s / splits));
        k1 = __builtin_amdgcn_readfirstlane((int)((int64_t)KT * (s + 1) / splits));
        next += step;
        return true;
    }
};

// An operand on its way: a stage (64 inner elements of a tile's 256 rows) is 32 copies of 1 KiB, eight a wave.
//
// ACROSS false: rows lie along the inner dimension.  A copy takes 128 bytes of eight rows, a row by eight neighbouring lanes.  In LDS a fragment (16
// rows) is 2 KiB, its rows one behind the other, the eight 16-byte pieces of a row exchanged by the row's last three bits: the 16 lanes that
// read one piece of each row fall on different banks.
// ACROSS true: the inner dimension lies across the rows.  A copy takes 512 bytes of two inner positions.  In LDS they lie one behind the other, the
// eight pieces of 64 bytes (two fragments) of a position exchanged by bits 0, 1 and 3 of its number; the transposing read gives a lane
// four inner positions of its column, 16 lanes of it read four positions on different banks.
template <bool ACROSS> struct Operand {
    v4i now;          // the buffer: this tile's panel
    uint32_t off;     // of the stage that is copied next
    uint32_t stride;  // between stages
    uint32_t part[COPIES];
    uint32_t voff[ACROSS ? 4 : 1], tail;
    bool tail_lane;
    uint32_t at[ACROSS ? 4 : 2];

    __device__ inline void set(uint32_t ld, uint32_t lds, int wave, int half, int lane, int64_t n)
    {
        if constexpr (ACROSS) {
            stride = STAGE_K * ld;
#pragma unroll
            for (int i = 0; i < COPIES; ++i) part[i] = (uint32_t)(16 * wave + 2 * i) * ld;
#pragma unroll
            for (int v = 0; v < 4; ++v)  // copy i: v = i % 2 + 2 (i / 4)
                voff[v] = (uint32_t)(lane >> 5) * ld + (uint32_t)(((lane & 31) >> 2) ^ (2 * (v & 1) + (lane >> 5) + 4 * (v >> 1))) * 64u + (lane & 3) * 16u;
            const int i = lane & 15, q = lane >> 4;
#pragma unroll
            for (int f = 0; f < 4; ++f)
                at[f] = lds + (8 * q + (i >> 2)) * 512 + ((half ^ (q & 1)) * 4 + (f ^ (i >> 2))) * 64 + (i & 3) * 16;
        } else {
            stride = STAGE_K * 2;
#pragma unroll
            for (int i = 0; i < COPIES; ++i) part[i] = (uint32_t)((2 * wave + i / 4) * 32 + (i / 2 % 2) * 4 + (i % 2) * 16) * ld;
            const int r = lane >> 3, piece = (lane & 7) ^ r;
            voff[0] = (uint32_t)row_of(0, r) * ld + (uint32_t)piece * 16u;
            // pieces behind the end of a row, in the last stage: out of the buffer, which gives zeros
            tail_lane = (n - 1) / STAGE_K * STAGE_K + piece * 8 >= n;
            const int place = lane & 15, q = lane >> 4;
            at[0] = lds + half * (OPERAND_BYTES / 2) + (place >> 3) * 1024 + (place & 7) * 128 + ((q ^ (place & 7)) << 4);
            at[1] = at[0] ^ 64u;
        }
    }
    // the panel of a tile, from stage k0 on; `rows`: of the operand (along the tile), `n`: inner
    __device__ inline void point(uint64_t base, uint32_t ld, int tile, int k0, int64_t rows, int64_t n)
    {
        uint64_t from;
        int64_t bytes;
        if constexpr (ACROSS) {
            from = base + (uint64_t)tile * (TILE * 2);
            // (rows to whole eights: what stands in memory there is read as whole dwords, or not at all)
            bytes = (n - 1) * ld + ((rows + 7) / 8 * 8 - (int64_t)tile * TILE) * 2;
        } else {
            const int64_t left = rows - (int64_t)tile * TILE;
            from = base + (uint64_t)tile * TILE * ld;
            bytes = ((left < TILE ? left : TILE) - 1) * ld + n * 2;
        }
        now = v4i{(int)(uint32_t)from, (int)(uint32_t)(from >> 32), (int)(uint32_t)bytes, 0x00020000};
        off = (uint32_t)k0 * stride;
    }
    __device__ inline void nothing()
    {
        now = v4i{0, 0, 0, 0x00020000};
        off = 0;
        stride = 0;
    }
    __device__ inline void last_stage(bool is) { if constexpr (!ACROSS) tail = is && tail_lane ? 0x70000000u : voff[0]; }
    template <int I> __device__ inline void issue() const
    {
        if constexpr (ACROSS)
            copy(voff[I % 2 + 2 * (I / 4)], now, off + part[I]);
        else
            copy(tail, now, off + part[I]);
    }
    __device__ inline void turn() { for (auto& a : at) a ^= PLACE_BYTES; }
    // fragment F (0 .. 7 of the wave's half) of the stage's inner elements 32 KS .. + 31
    template <int F, int KS> __device__ inline v4i fetch() const
    {
        if constexpr (ACROSS) {
            typedef __attribute__((address_space(3))) v4s* lds_v4s;
            constexpr int D = F % 2 * 8 + KS * 32 * 512;
            const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(uintptr_t)(at[F / 2] + D));
            const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(uintptr_t)(at[F / 2] + D + 4 * 512));
            return __builtin_bit_cast(v4i, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return *(lds_v4i)(uintptr_t)(at[KS] + F * 2048);
        }
    }
};

__device__ inline float over_quarters_max(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ inline float over_quarters_sum(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

template <int TYPE, int DTYPE> __device__ inline void put(const Args& g, float alpha, int64_t row, int64_t col, const float* v)
{
    typedef typename Elem<DTYPE>::Bits Bits;
    if (row >= g.m || col >= g.p) return;
    Bits* const out = (Bits*)g.D + row * g.ldd + col;
    const int64_t left = g.p - col;
    Bits x[8];
    if (g.beta != 0.0f) {
        load_row<DTYPE, 8>(out, left, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = from_float<DTYPE>(alpha * v[e] + g.beta * to_float<DTYPE>(x[e]));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = from_float<DTYPE>(alpha * v[e]);
    }
    store_row<DTYPE, 8>(out, left, x);
}

// A workgroup of four waves, 128 x 128 sums each in 256 registers a lane, one wave a SIMD, takes one item after the other.  A stage is 64
// inner elements of A and B, 64 KiB, and LDS holds two: while one is multiplied the other arrives, and the stages of all items are one
// stream, so that the first of an item arrive while the sums of the one before are written out.  A stage is two steps of 64 matrix instructions a
// wave, each run as four quarters of 4 x 4 fragments on four sets of four: (A lo, B lo), (A lo, B hi), (A hi, B lo), (A hi, B hi), each fetching
// the set that the quarter after the next needs.  One barrier a stage, before the last two quarters: behind it the stage's place takes the
// copies of the stage after the next.
template <int TYPE, int KIND> __global__ __launch_bounds__(256) void k_lm_tile(Args g)
{
    constexpr bool A_ACROSS = KIND == lmk::WEIGHTS, B_ACROSS = KIND == lmk::WEIGHTS || KIND == lmk::STATES;
    __shared__ __align__(16) uint8_t ring[2 * PLACE_BYTES];
    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)ring;

    Operand<A_ACROSS> a;
    Operand<B_ACROSS> b;
    a.set(g.lda, lds, wave, wm, lane, g.n);
    b.set(g.ldb, lds + OPERAND_BYTES, wave, wn, lane, g.n);
    Order copy_order(g);
    int stages_left = 0, stage_now = 0;
    auto look_up = [&]() {
        int tm, tp, split, k0, k1;
        if (copy_order.take(tm, tp, split, k0, k1)) {
            a.point(g.A, g.lda, tm, k0, g.m, g.n);
            b.point(g.B, g.ldb, tp, k0, g.p, B_ACROSS ? g.b_rows : g.n);
            stages_left = k1 - k0;
            stage_now = k0;
        } else {
            a.nothing();
            b.nothing();
            stages_left = 1 << 30;
            stage_now = -(1 << 30);
        }
    };
    auto begin_copies = [&]() {
        const bool last = stage_now == g.KT - 1;
        a.last_stage(last);
        b.last_stage(last);
    };
    auto end_copies = [&]() {
        a.off += a.stride;
        b.off += b.stride;
        ++stage_now;
        if (--stages_left == 0) look_up();
    };
    uint32_t to = lds + wave * (COPIES * 1024);  // the place that is copied to, this wave's part
    look_up();
    static_for<0, 2>([&](auto) {
        begin_copies();
        static_for<0, COPIES>([&](auto I) {
            constexpr int i = decltype(I)::value;
            copy_to<i * 1024>(to);
            asm volatile("s_nop 4");
            a.template issue<i>();
            copy_to<OPERAND_BYTES + i * 1024>(to);
            asm volatile("s_nop 4");
            b.template issue<i>();
        });
        end_copies();
        to = to + PLACE_BYTES < lds + 2 * PLACE_BYTES ? to + PLACE_BYTES : to - PLACE_BYTES;
    });

    v4f acc[8][8];
    v4i faL[4], faH[4], fbL[4], fbH[4];
    // matrix instruction X of a quarter, there and back over the fragments of A
    auto math = [&](const v4i* fa, const v4i* fb, auto I0, auto J0, auto X) __attribute__((always_inline)) {
        constexpr int j = decltype(X)::value / 4, x = decltype(X)::value % 4, i = (j & 1) ? 3 - x : x;
        v4f& c = acc[decltype(I0)::value + i][decltype(J0)::value + j];
        c = mfma<TYPE>(fb[j], fa[i], c);
    };
    typedef std::integral_constant<int, 0> N0;
    typedef std::integral_constant<int, 4> N4;

    wait_vmcnt<2 * COPIES>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    static_for<0, 4>([&](auto Q) {
        constexpr int q = decltype(Q)::value;
        faL[q] = a.template fetch<q, 0>();
        fbL[q] = b.template fetch<q, 0>();
    });

    auto stage = [&]() __attribute__((always_inline)) {
        static_for<0, 2>([&](auto KS) __attribute__((always_inline)) {
            constexpr int ks = decltype(KS)::value;
            static_for<0, 16>([&](auto X) __attribute__((always_inline)) {
                constexpr int x = decltype(X)::value;
                if constexpr (x % 2 == 0 && x < 8) fbH[x / 2] = b.template fetch<4 + x / 2, ks>();
                math(faL, fbL, N0{}, N0{}, X);
                __builtin_amdgcn_sched_barrier(0);
            });
            static_for<0, 16>([&](auto X) __attribute__((always_inline)) {
                constexpr int x = decltype(X)::value;
                if constexpr (x % 2 == 0 && x < 8) faH[x / 2] = a.template fetch<4 + x / 2, ks>();
                math(faL, fbH, N0{}, N4{}, X);
                __builtin_amdgcn_sched_barrier(0);
            });
            if constexpr (ks == 1) {
                wait_vmcnt<0>();
                wait_lds();
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                a.turn();
                b.turn();
                begin_copies();
            }
            static_for<0, 16>([&](auto X) __attribute__((always_inline)) {
                constexpr int x = decltype(X)::value;
                if constexpr (ks == 1) {
                    // copies: B's eight here, A's in the next quarter
                    if constexpr (x % 2 == 0) copy_to<OPERAND_BYTES + x / 2 * 1024>(to);
                    if constexpr (x % 2 == 1) b.template issue<x / 2>();
                }
                if constexpr (x % 2 == 0 && x < 8) faL[x / 2] = a.template fetch<x / 2, 1 - ks>();
                math(faH, fbL, N4{}, N0{}, X);
                __builtin_amdgcn_sched_barrier(0);
            });
            static_for<0, 16>([&](auto X) __attribute__((always_inline)) {
                constexpr int x = decltype(X)::value;
                if constexpr (ks == 1) {
                    if constexpr (x % 2 == 0) copy_to<x / 2 * 1024>(to);
                    if constexpr (x % 2 == 1) a.template issue<x / 2>();
                }
                if constexpr (x % 2 == 0 && x < 8) fbL[x / 2] = b.template fetch<x / 2, 1 - ks>();
                math(faH, fbH, N4{}, N4{}, X);
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        end_copies();
        to = to < lds + PLACE_BYTES ? to + PLACE_BYTES : to - PLACE_BYTES;
    };

    Order order(g);
    int tm, tp, split, k0, k1;
    while (order.take(tm, tp, split, k0, k1)) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                acc[i][j] = v4f{0, 0, 0, 0};
                asm volatile("" : "+a"(acc[i][j]));  // (in its accumulation registers from here on)
            }
#pragma clang loop unroll(disable)
        for (int k = k0; k < k1; ++k) stage();

        // (read by asm statements, or the register allocator parks sums in scratch memory; the wait states behind the last matrix instruction are
        // written out)
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) asm volatile("" : "+a"(acc[i][j]));
        asm volatile("s_nop 15\n\ts_nop 15");
        int lr = lane & 15, lc = lane >> 4;
        asm volatile("" : "+v"(lr), "+v"(lc));
        const int64_t row0 = (int64_t)tm * TILE + wm * 128 + row_of(0, lr), col0 = (int64_t)tp * TILE + wn * 128;
        const int row_lane = wm * 128 + row_of(0, lr);
        // this lane's 32 sums of a row, eight neighbouring columns at a time: v[8 J + e] is column 32 J + 8 lc + e
        auto rows = [&](auto&& f) __attribute__((always_inline)) {
            static_for<0, 8>([&](auto I) __attribute__((always_inline)) {
                constexpr int i = decltype(I)::value;
                float v[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v[e]) : "a"(acc[i][e / 8 * 2 + e / 4 % 2][e % 4]));
                f(I, std::integral_constant<int, row_of(i, 0)>{}, v);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        if constexpr (KIND == lmk::LOSS || KIND == lmk::SLOPE) {
            // the targets of the lane's rows, as columns of this wave's 128
            int target[8];
            bool any = false;
            static_for<0, 8>([&](auto I) {
                constexpr int i = decltype(I)::value;
                target[i] = g.targets[(int64_t)tm * TILE + row_lane + row_of(i, 0)];
                const int c = target[i] - g.column0 - (int)col0;
                target[i] = target[i] < 0 ? target[i] : (c >= 0 && c < 128 ? c : 128);
                any |= target[i] >= 0 && target[i] < 128;
            });
            const bool found = __any(any), edge = col0 + 128 > g.p;
            const int cols = (int)(g.p - col0 < 128 ? g.p - col0 : 128);
            if constexpr (KIND == lmk::LOSS) {
                if (col0 < g.p)
                    rows([&](auto I, auto RI, float* v) __attribute__((always_inline)) {
                        constexpr int i = decltype(I)::value, ri = decltype(RI)::value;
                        const float none = -__builtin_inff();
                        if (edge)
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e] = e / 8 * 32 + lc * 8 + e % 8 < cols ? v[e] : none;
                        if (found) {
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (target[i] == e / 8 * 32 + lc * 8 + e % 8) {
                                    g.at_target[row0 + ri] = v[e];
                                    v[e] = none;
                                }
                        }
                        float m = none;
#pragma unroll
                        for (int e = 0; e < 32; ++e) m = fmaxf(m, v[e]);
                        m = over_quarters_max(m) * LOG2E;
                        const float m2 = m == none ? 0.0f : m;
                        float s = 0.0f;
#pragma unroll
                        for (int e = 0; e < 32; ++e) s += __builtin_amdgcn_exp2f(__builtin_fmaf(v[e], LOG2E, -m2));
                        s = over_quarters_sum(s);
                        if (lc == 0) g.parts[(col0 >> 7) * g.parts_ld + row0 + ri] = make_float2(m, s);
                    });
            } else {
                float lse2[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) lse2[i] = g.lse2[(int64_t)tm * TILE + row_lane + row_of(i, 0)];
                typedef typename Elem<TYPE>::Bits Bits;
                rows([&](auto I, auto RI, float* v) __attribute__((always_inline)) {
                    constexpr int i = decltype(I)::value, ri = decltype(RI)::value;
                    constexpr float SCALE = TYPE == F16 ? lmk::SLOPE_SCALE_F16 : 1.0f;
                    float target_slope = 0.0f;
                    if (found) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (target[i] == e / 8 * 32 + lc * 8 + e % 8) target_slope = expm1f((v[e] * LOG2E - lse2[i]) * 0.693147180559945309f);
                    }
                    const uint32_t keep = target[i] == lmk::NO_TARGET ? 0u : 0xffffffffu;
                    Bits* const out = (Bits*)g.D + (row0 + ri) * g.ldd + col0 + lc * 8;
#pragma unroll
                    for (int jj = 0; jj < 4; ++jj) {
                        Bits x[8];
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            float d = __builtin_amdgcn_exp2f(__builtin_fmaf(v[8 * jj + e], LOG2E, -lse2[i]));
                            if (edge) d = jj * 32 + lc * 8 + e < cols ? d : 0.0f;
                            if (found) d = target[i] == jj * 32 + lc * 8 + e ? target_slope : d;
                            x[e] = from_float<TYPE>(SCALE * d);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = ((uint32_t)x[2 * e] | (uint32_t)x[2 * e + 1] << 16) & keep;
                        __builtin_memcpy(out + jj * 32, w, 16);
                    }
                });
            }
        } else if constexpr (KIND == lmk::STATES) {
            rows([&](auto, auto RI, float* v) __attribute__((always_inline)) {
                constexpr int ri = decltype(RI)::value;
                float* const out = (float*)g.D + split * g.split_stride + (row0 + ri) * g.ldd + col0 + lc * 8;
                if (g.beta != 0.0f) {
                    v4f old[8];
#pragma unroll
                    for (int jj = 0; jj < 8; ++jj) old[jj] = *(const v4f*)(out + jj / 2 * 32 + jj % 2 * 4);
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] += old[e / 4][e % 4];
                }
#pragma unroll
                for (int jj = 0; jj < 8; ++jj) *(v4f*)(out + jj / 2 * 32 + jj % 2 * 4) = v4f{v[4 * jj], v[4 * jj + 1], v[4 * jj + 2], v[4 * jj + 3]};
            });
        } else {
            float alpha = g.alpha;
            if constexpr (KIND == lmk::WEIGHTS) alpha *= *g.alpha_at;
            rows([&](auto, auto RI, float* v) __attribute__((always_inline)) {
                constexpr int ri = decltype(RI)::value;
#pragma unroll
                for (int jj = 0; jj < 4; ++jj) {
                    if (g.dtype == F32) put<TYPE, F32>(g, alpha, row0 + ri, col0 + jj * 32 + lc * 8, v + 8 * jj);
                    if (g.dtype == BF16) put<TYPE, BF16>(g, alpha, row0 + ri, col0 + jj * 32 + lc * 8, v + 8 * jj);
                    if (g.dtype == F16) put<TYPE, F16>(g, alpha, row0 + ri, col0 + jj * 32 + lc * 8, v + 8 * jj);
                }
            });
        }
    }
    wait_vmcnt<0>();  // no copy may still be writing LDS when the workgroup retires
}

template <int TYPE, int KIND> void run(const Args& g, hipStream_t st)
{
    const int64_t items = (int64_t)g.TM * g.TP * g.splits;
    k_lm_tile<TYPE, KIND><<<dim3((unsigned)(items < COMPUTE_UNITS ? items : COMPUTE_UNITS)), dim3(256), 0, st>>>(g);
}
template <int TYPE> void run(int kind, const Args& g, hipStream_t st)
{
    if (kind == lmk::LINEAR) run<TYPE, lmk::LINEAR>(g, st);
    if (kind == lmk::LOSS) run<TYPE, lmk::LOSS>(g, st);
    if (kind == lmk::SLOPE) run<TYPE, lmk::SLOPE>(g, st);
    if (kind == lmk::STATES) run<TYPE, lmk::STATES>(g, st);
    if (kind == lmk::WEIGHTS) run<TYPE, lmk::WEIGHTS>(g, st);
}

}  // namespace

namespace lmk {

// (32-bit offsets inside a panel, 30 bits where rows lie along the inner dimension: pieces behind a row's end are sent behind those)
bool tile_fits(const Tile& t)
{
    auto along = [](int64_t ld) { return ld * 2 < (1 << 22); };
    auto across = [&](int64_t ld) { return t.n * ld * 2 < ((int64_t)1 << 32) - (1 << 20); };
    const bool a = t.kind == WEIGHTS ? across(t.lda) : along(t.lda);
    const bool b = t.kind == WEIGHTS || t.kind == STATES ? across(t.ldb) : along(t.ldb);
    return a && b && t.n > 0 && (t.m + TILE - 1) / TILE * ((t.p + TILE - 1) / TILE) * t.splits < ((int64_t)1 << 28);
}

hipError_t launch_tile(const Tile& t, hipStream_t st)
{
    const Args g = {t.m, t.n, t.p, t.b_rows, (uint64_t)(uintptr_t)t.A, (uint64_t)(uintptr_t)t.B, (uint32_t)(t.lda * 2), (uint32_t)(t.ldb * 2),
                    (int)((t.m + TILE - 1) / TILE), (int)((t.p + TILE - 1) / TILE), (int)((t.n + STAGE_K - 1) / STAGE_K), t.splits, t.D, t.ldd, t.dtype,
                    t.alpha, t.beta, t.alpha_at, t.split_stride, t.targets, t.column0, t.lse2, t.at_target, t.parts, t.parts_ld};
    if (t.type == BF16) run<BF16>(t.kind, g, st);
    if (t.type == F16) run<F16>(t.kind, g, st);
    return hipGetLastError();
}

}  // namespace lmk
