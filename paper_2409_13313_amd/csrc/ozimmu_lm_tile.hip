// Products of 16-bit matrices on the matrix cores in tiles of up to 256 x 256, and what the loss makes of their sums (ozimmu_lm.h, Kind).
#include "ozimmu_lm.h"
#include <type_traits>

namespace {

using namespace mxk;
using lmk::Tile;

constexpr int64_t COMPUTE_UNITS = 256;
constexpr int NXCD = 8, STAGE_K = 64;
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
    lmk::Targets targets;
    const int* known;
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

// An operand on its way: a stage (64 inner elements of a tile's 32 F rows) is 4 F copies of 1 KiB, F a wave, into one of PLACES places.
//
// ACROSS false: rows lie along the inner dimension.  A copy takes 128 bytes, a whole line, of eight rows, a row by eight neighbouring lanes.  In
// LDS a fragment (16 rows) is 2 KiB, its rows one behind the other, the eight 16-byte pieces of a row exchanged by the last three bits of its
// place: the lanes that read one piece of eight rows fall on different banks.
// ACROSS true: the inner dimension lies across the rows.  A copy takes 1 KiB of two (F = 4: four) inner positions.  In LDS they lie one behind the other, the
// pieces of 32 bytes (a fragment) of a position exchanged by bits 0, 1 and 3 of its number: the transposing read, which gives a lane four inner
// positions of its column, has 32 lanes read eight positions, which then fall on different banks.
template <bool ACROSS, int F, int PLACES> struct Operand {
    static constexpr int TILE = 32 * F, COPIES = F, BYTES = TILE * STAGE_K * 2, ROW = 2 * TILE;  // of a stage in LDS; of an inner position there
    static constexpr int POSITIONS = 1024 / ROW, LANES = 64 / POSITIONS;  // ACROSS: of a copy; lanes for each
    static constexpr int VOFFS = F == 8 ? 4 : 2;
    v4i now;          // the buffer: this tile's panel
    uint32_t off;     // of this wave's part of the stage that is copied next
    uint32_t stride;  // between stages
    uint32_t step[2]; // between its copies (from an even one, from an odd one)
    uint32_t at_copy; // offset of the next copy
    uint32_t wave_part;
    uint32_t voff[ACROSS ? VOFFS : 1], tail;
    bool tail_lane;
    uint32_t base[ACROSS ? F : 2], at[ACROSS ? F : 2];
    uint32_t to;      // where this wave's copies go next
    uint32_t first;   // .. in the first place
    uint32_t from;    // offset of the place that is read

    __device__ inline void set(uint32_t ld, uint32_t lds, int wave, int half, int lane, int64_t n)
    {
        stride = ACROSS ? STAGE_K * ld : STAGE_K * 2;
        first = to = lds + wave * (COPIES * 1024);
        if constexpr (ACROSS) {
            wave_part = (uint32_t)(16 * wave) * ld;
            step[0] = step[1] = POSITIONS * ld;
            const int position = lane / LANES, slot = lane % LANES;
#pragma unroll
            for (int v = 0; v < VOFFS; ++v) {  // of copy i: F = 8: v = i % 2 + 2 (i / 4), F = 4: v = i / 2
                const int swap = F == 8 ? 2 * (v & 1) + position + 4 * (v >> 1) : position + 4 * v;
                voff[v] = (uint32_t)position * ld + (uint32_t)((slot >> 1) ^ swap) * 32u + (slot & 1) * 16u;
            }
            const int i = lane & 15, q = lane >> 4;
#pragma unroll
            for (int f = 0; f < F; ++f) base[f] = lds + (8 * q + (i >> 2)) * ROW + ((half * F + f) ^ ((i >> 2) + 4 * (q & 1))) * 32 + (i & 3) * 8;
        } else {
            // (the halves of two fragments in turn, the first ones first: rows 0, 4, 16, 20 and so on)
            wave_part = (uint32_t)row_of(wave * (F / 2), 0) * ld;
            step[0] = 4 * ld;
            step[1] = 12 * ld;
            const int r = lane >> 3, piece = (lane & 7) ^ r;
            voff[0] = (uint32_t)row_of(0, r) * ld + (uint32_t)piece * 16u;
            // pieces behind the end of a row, in the last stage: out of the buffer, which gives zeros
            tail_lane = (n - 1) / STAGE_K * STAGE_K + piece * 8 >= n;
            const int place = lane & 15, q = lane >> 4;
            base[0] = lds + half * (BYTES / 2) + (place >> 3) * 1024 + (place & 7) * 128 + ((q ^ (place & 7)) << 4);
            base[1] = base[0] ^ 64u;
        }
        from = 0;
        read_from();
    }
    __device__ inline void read_from()
    {
#pragma unroll
        for (int f = 0; f < (ACROSS ? F : 2); ++f) at[f] = base[f] + from;
    }
    __device__ inline void read_next()
    {
        from = from == (PLACES - 1) * BYTES ? 0 : from + BYTES;
        read_from();
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
        off = (uint32_t)k0 * stride + wave_part;
    }
    __device__ inline void nothing()
    {
        now = v4i{0, 0, 0, 0x00020000};
        off = 0;
        stride = 0;
    }
    __device__ inline void begin_stage(bool last)
    {
        at_copy = off;
        if constexpr (!ACROSS) tail = last && tail_lane ? 0x70000000u : voff[0];
    }
    template <int I> __device__ inline void set_m0() const { copy_to<(ACROSS ? I : I / 4 * 4 + I % 2 * 2 + I / 2 % 2) * 1024>(to); }
    template <int I> __device__ inline void issue()
    {
        if constexpr (ACROSS)
            copy(voff[F == 8 ? I % 2 + 2 * (I / 4) : I / 2], now, at_copy);
        else
            copy(tail, now, at_copy);
        at_copy += step[I % 2];
    }
    __device__ inline void issued()
    {
        off += stride;
        to = to == first + (PLACES - 1) * BYTES ? first : to + BYTES;
    }
    // fragment I (0 .. F - 1 of the wave's half) of the stage's inner elements 32 KS .. + 31
    template <int I, int KS> __device__ inline v4i fetch() const
    {
        if constexpr (ACROSS) {
            typedef __attribute__((address_space(3))) v4s* lds_v4s;
            const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(uintptr_t)(at[I] + KS * 32 * ROW));
            const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(uintptr_t)(at[I] + KS * 32 * ROW + 4 * ROW));
            return __builtin_bit_cast(v4i, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return *(lds_v4i)(uintptr_t)(at[KS] + I * 2048);
        }
    }
    // row (column) of fragment f's place in the tile's half
    static __host__ __device__ constexpr int row(int fragment, int place) { return ACROSS ? 16 * fragment + place : row_of(fragment, place); }
};

// One operand's way through the items of a workgroup, some stages ahead of the products
template <bool ACROSS, int F, int PLACES, bool IS_A> struct Stream : Operand<ACROSS, F, PLACES> {
    Order order;
    int left = 0, stage = 0;
    __device__ inline explicit Stream(const Args& g) : order(g) {}
    __device__ inline void look_up(const Args& g)
    {
        int tm, tp, split, k0, k1;
        if (order.take(tm, tp, split, k0, k1)) {
            if constexpr (IS_A)
                this->point(g.A, g.lda, tm, k0, g.m, g.n);
            else
                this->point(g.B, g.ldb, tp, k0, g.p, ACROSS ? g.b_rows : g.n);
            left = k1 - k0;
            stage = k0;
        } else {
            this->nothing();
            left = 1 << 30;
            stage = -(1 << 30);
        }
    }
    __device__ inline void begin(const Args& g) { this->begin_stage(stage == g.KT - 1); }
    __device__ inline void end(const Args& g)
    {
        this->issued();
        ++stage;
        if (--left == 0) look_up(g);
    }
};

// over the four lanes l, l ^ 16, l ^ 32, l ^ 48
template <class F> __device__ inline float over_quarters(float v, F&& f)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// vmcnt(N), by the builtin: the compiler then knows what loads of its own are there
template <int N> __device__ inline void wait_vmcnt_known()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0xf70);
    asm volatile("" ::: "memory");
}

// Eight neighbouring sums into D.  EDGE: of which not all need lie in D.
template <int DTYPE, bool BETA, bool EDGE>
__device__ inline void put(const Args& g, float alpha, int64_t row, int64_t col, const float* v)
{
    typedef typename Elem<DTYPE>::Bits Bits;
    Bits* const out = (Bits*)g.D + row * g.ldd + col;
    Bits x[8];
    if constexpr (EDGE) {
        if (row >= g.m) return;
        const int left = (int)(g.p - col);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) out[e] = from_float<DTYPE>(BETA ? alpha * v[e] + g.beta * to_float<DTYPE>(out[e]) : alpha * v[e]);
    } else {
        if constexpr (BETA) __builtin_memcpy(x, out, sizeof(x));
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = from_float<DTYPE>(BETA ? alpha * v[e] + g.beta * to_float<DTYPE>(x[e]) : alpha * v[e]);
        __builtin_memcpy(out, x, sizeof(x));
    }
}

// A workgroup of four waves, 128 x 128 sums each in 256 registers a lane, one wave a SIMD, takes one item after the other.  A stage is 64
// inner elements of A and B.  The stages of all items are one stream, so that the first of an item arrive while the sums of the one before are
// written out.  A stage is two halves of 64 matrix instructions a wave; during each the 16 fragments of the next half come from LDS into a second
// set of registers.  So both places of a stage are free at the end of its first half, where the one barrier of a stage is; behind it they take
// the copies of A two stages and of B three stages on.
//
// A wave has FA fragments of A and FB of B, a workgroup 32 FA x 32 FB sums: 256 x 256, one workgroup a compute unit; 128 x 256 and 128 x 128 (two
// workgroups a compute unit, the one at work while the other begins or ends) for outputs of too few tiles.
//
// Bound by the matrix cores at the clock that power leaves them: 4096 x 4096 x 131072 in BF16 2.9 to 3.2 ms with the loss in its epilogue, 1.38 to 1.5 PFLOP/s
// (a library's product of that size, which stores it, 1.46).  On the way there, in ms: two places of 64 and no second set of registers 3.42; five places of 32
// 3.51, with a second set 3.32; whole lines in two and three places of 64 3.22; epilogues without waits for copies 3.14.  Of pieces of 16384 words (us; in
// brackets without epilogue): slopes 383 to 404 (363), states 372 to 400 (383), weights 372 to 412 (356).
template <int TYPE, int KIND, int FA, int FB> __global__ __launch_bounds__(256, FB == 4 ? 2 : 1) void k_lm_tile(Args g)
{
    constexpr bool A_ACROSS = KIND == lmk::WEIGHTS, B_ACROSS = KIND == lmk::WEIGHTS || KIND == lmk::STATES;
    constexpr int A_PLACES = FA == 8 || FB == 4 ? 2 : 3, B_PLACES = 3, M = FA * FB, TILE_A = 32 * FA, TILE_B = 32 * FB, N = 4 * FB;
    typedef Stream<A_ACROSS, FA, A_PLACES, true> StreamA;
    typedef Stream<B_ACROSS, FB, B_PLACES, false> StreamB;
    __shared__ __align__(16) uint8_t places[A_PLACES * StreamA::BYTES + B_PLACES * StreamB::BYTES];  // 160, 144, 80 KiB
    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)places;

    StreamA a(g);
    StreamB b(g);
    a.set(g.lda, lds, wave, wm, lane, g.n);
    b.set(g.ldb, lds + A_PLACES * StreamA::BYTES, wave, wn, lane, g.n);
    // Of the rows that a lane has of an item: targets as columns of the wave's (none of them: TILE_B; SLOPE: also NO_TARGET, BAD_TARGET), and
    // log2(e) lse.  They come an item ahead, so that no wait for them is one for the copies.
    struct Rows {
        int target[FA];
        float lse2[FA];
    };
    constexpr bool BY_ROW = KIND == lmk::LOSS || KIND == lmk::SLOPE;
    auto look_at = [&](int tm, int tp, Rows& o) __attribute__((always_inline)) {
        const int first = tm * TILE_A + wm * (TILE_A / 2) + row_of(0, lane & 15), col0 = tp * TILE_B + wn * (TILE_B / 2) + g.column0;
        static_for<0, FA>([&](auto I) __attribute__((always_inline)) {
            constexpr int i = decltype(I)::value;
            const int row = first + row_of(i, 0);
            if constexpr (KIND == lmk::LOSS) {
                // (rows behind the last one: its target, for nothing)
                const int64_t y = g.targets.y[min(row, (int)g.m - 1) * g.targets.stride], c = y - col0;
                o.target[i] = y != g.targets.ignore && (uint64_t)c < TILE_B / 2 ? (int)c : TILE_B;
            } else {
                const int target = g.known[row], c = target - col0;
                o.target[i] = target < 0 ? target : ((uint32_t)c < TILE_B / 2 ? c : TILE_B);
                o.lse2[i] = g.lse2[row];
            }
        });
    };
    Order order(g);
    int tm = 0, tp = 0, split = 0, k0 = 0, k1 = 0;
    bool any = order.take(tm, tp, split, k0, k1);
    Rows coming;
    if constexpr (BY_ROW) {
        look_at(tm, tp, coming);
        wait_vmcnt_known<0>();
    }
    a.look_up(g);
    b.look_up(g);
    auto whole_stage = [&](auto& o) __attribute__((always_inline)) {
        o.begin(g);
        static_for<0, std::remove_reference_t<decltype(o)>::COPIES>([&](auto I) __attribute__((always_inline)) {
            o.template set_m0<decltype(I)::value>();
            asm volatile("s_nop 4");
            o.template issue<decltype(I)::value>();
        });
        o.end(g);
    };
#pragma clang loop unroll(disable)
    for (int place = 0; place < B_PLACES; ++place) {
        whole_stage(b);
        if (place < A_PLACES) whole_stage(a);
    }
    constexpr int ON_THE_WAY = (A_PLACES - 2) * FA + FB;  // copies of a wave that need not be there yet when the next stage is looked at

    v4f acc[FA][FB];
    v4i fa[2][FA], fb[2][FB];   // the fragments of this half and of the next
    wait_vmcnt<FA + FB + ON_THE_WAY>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    static_for<0, FA>([&](auto F) __attribute__((always_inline)) { fa[0][decltype(F)::value] = a.template fetch<decltype(F)::value, 0>(); });
    static_for<0, FB>([&](auto F) __attribute__((always_inline)) { fb[0][decltype(F)::value] = b.template fetch<decltype(F)::value, 0>(); });

    // FIRST: of an item, whose sums begin here
    auto half = [&](auto H, auto FIRST, auto&& wait) __attribute__((always_inline)) {
        constexpr int h = decltype(H)::value, READS = FA + FB, EVERY = M / READS;
        if constexpr (h == 1) {
            a.begin(g);
            b.begin(g);
        }
        static_for<0, M>([&](auto X) __attribute__((always_inline)) {
            constexpr int x = decltype(X)::value, j = x / FA, i = j & 1 ? FA - 1 - x % FA : x % FA;
            // (early, so that the last of them is there at the end: three steps of four)
            constexpr int f = x * READS / (M * 3 / 4);
            if constexpr (f < READS && f * (M * 3 / 4) / READS + ((f * (M * 3 / 4)) % READS != 0) == x) {
                if constexpr (f < FA)
                    fa[1 - h][f % FA] = a.template fetch<f % FA, 1 - h>();
                else
                    fb[1 - h][f % READS - FA] = b.template fetch<(f - FA) & (FB - 1), 1 - h>();
            }
            if constexpr (h == 1) {
                constexpr int c = x / EVERY;
                if constexpr (x % EVERY == 0 && c < FA) a.template set_m0<c>();
                if constexpr (x % EVERY == 1 && c < FA) a.template issue<c>();
                if constexpr (x % EVERY == 0 && c >= FA && c < READS) b.template set_m0<c - FA>();
                if constexpr (x % EVERY == 1 && c >= FA && c < READS) b.template issue<c - FA>();
            }
            if constexpr (decltype(FIRST)::value) {
                acc[i][j] = mfma<TYPE>(fb[h][j], fa[h][i], v4f{0, 0, 0, 0});
                asm volatile("" : "+a"(acc[i][j]));  // (in its accumulation registers from here on)
            } else {
                acc[i][j] = mfma<TYPE>(fb[h][j], fa[h][i], acc[i][j]);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (h == 0) {
            // all of this stage is read, and the next one is there
            wait();
            wait_lds();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            a.read_next();
            b.read_next();
        } else {
            a.end(g);
            b.end(g);
        }
    };

    const float alpha = KIND == lmk::WEIGHTS || (KIND == lmk::LINEAR && TYPE == F16 && g.alpha_at) ? g.alpha * *g.alpha_at : g.alpha;
    typedef std::integral_constant<int, 0> N0;
    typedef std::integral_constant<int, 1> N1;
    const auto usual = [] { wait_vmcnt<ON_THE_WAY>(); };
    // The stores of an item stand behind the copies that its successor's first stage waits for, and need not be over then.  SLOPE: nor before them
    // the loads of `coming`.
    constexpr int STORES = KIND == lmk::STATES ? FA * FB : FA * FB / 2, LATER = ON_THE_WAY + STORES < 63 ? ON_THE_WAY + STORES : 63;
    bool stored = false;  // that many of them, by the last item
    while (any) {
        if constexpr (KIND == lmk::SLOPE)
            half(N0{}, std::true_type{}, [&]() __attribute__((always_inline)) {
                if (stored)
                    wait_vmcnt_known<STORES>();
                else
                    wait_vmcnt_known<0>();
            });
        else if constexpr (KIND == lmk::LOSS)
            half(N0{}, std::true_type{}, [] { wait_vmcnt_known<0>(); });
        else
            half(N0{}, std::true_type{}, [&]() __attribute__((always_inline)) {
                if (stored)
                    wait_vmcnt<LATER>();
                else
                    wait_vmcnt<ON_THE_WAY>();
            });
        half(N1{}, std::false_type{}, usual);
#pragma clang loop unroll(disable)
        for (int k = k0 + 1; k < k1; ++k) {
            half(N0{}, std::false_type{}, usual);
            half(N1{}, std::false_type{}, usual);
        }

        // (read by asm statements, or the register allocator parks sums in scratch memory; the wait states behind the last matrix instruction are
        // written out)
#pragma unroll
        for (int i = 0; i < FA; ++i)
#pragma unroll
            for (int j = 0; j < FB; ++j) asm volatile("" : "+a"(acc[i][j]));
        asm volatile("s_nop 15\n\ts_nop 15");
        int lr = lane & 15, lc = lane >> 4;
        asm volatile("" : "+v"(lr), "+v"(lc));
        const int64_t row0 = (int64_t)tm * TILE_A + wm * (TILE_A / 2) + a.row(0, lr), col0 = (int64_t)tp * TILE_B + wn * (TILE_B / 2);
        // this lane's N sums of a row: v[4 j + r] is of place 4 lc + r of B's fragment j (B along: v[8 J + e] is column 32 J + 8 lc + e)
        auto rows = [&](auto&& f) __attribute__((always_inline)) {
            static_for<0, FA>([&](auto I) __attribute__((always_inline)) {
                constexpr int i = decltype(I)::value;
                float v[N];
#pragma unroll
                for (int e = 0; e < N; ++e) asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v[e]) : "a"(acc[i][e / 8 * 2 + e / 4 % 2][e % 4]));
                f(I, std::integral_constant<int, a.row(i, 0)>{}, v);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        // the item at hand, and the next one
        const int this_split = split;
        const bool inside = (int64_t)(tm + 1) * TILE_A <= g.m && (int64_t)(tp + 1) * TILE_B <= g.p, whole = inside && g.beta == 0.0f;
        const Rows mine = coming;
        any = order.take(tm, tp, split, k0, k1);
        if constexpr (BY_ROW) {
            look_at(tm, tp, coming);
            uint32_t least = TILE_B;
#pragma unroll
            for (int i = 0; i < FA; ++i) least = min(least, (uint32_t)mine.target[i]);
            const bool found = __any(least < TILE_B / 2), edge = col0 + TILE_B / 2 > g.p;
            const int cols = (int)(g.p - col0 < TILE_B / 2 ? g.p - col0 : TILE_B / 2);
            // f(e, column - this lane's column e), one after the other.  (The column is made opaque each time, and nothing moves between them: their
            // comparisons, kept for all rows or made side by side, would take all scalar registers.)
            auto compared = [&](int column, auto&& f) __attribute__((always_inline)) {
                column -= lc * 8;
                asm volatile("" : "+v"(column));
                static_for<0, N>([&](auto E) __attribute__((always_inline)) {
                    constexpr int e = decltype(E)::value;
                    f(e, column - (e / 8 * 32 + e % 8));
                    if constexpr (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                });
            };
            if constexpr (KIND == lmk::LOSS) {
                if (col0 < g.p)
                    rows([&](auto I, auto RI, float* v) __attribute__((always_inline)) {
                        constexpr int i = decltype(I)::value, ri = decltype(RI)::value;
                        const int target = mine.target[i];
                        const float none = -__builtin_inff();
                        if (edge) compared(cols, [&](int e, int c) { v[e] = c > 0 ? v[e] : none; });
                        if (found) {
                            float z = 0.0f;
                            compared(target, [&](int e, int c) {
                                z = c == 0 ? v[e] : z;
                                v[e] = c == 0 ? none : v[e];
                            });
                            if ((uint32_t)target < TILE_B / 2 && (target >> 3 & 3) == lc) g.at_target[row0 + ri] = z;
                        }
                        float m = none;
#pragma unroll
                        for (int e = 0; e < N; ++e) m = fmaxf(m, v[e]);
                        m = over_quarters(m, [](float p, float q) { return fmaxf(p, q); }) * LOG2E;
                        const float m2 = m == none ? 0.0f : m;
                        float s[4] = {0, 0, 0, 0};
#pragma unroll
                        for (int e = 0; e < N; ++e) s[e % 4] += __builtin_amdgcn_exp2f(__builtin_fmaf(v[e], LOG2E, -m2));
                        const float sum = over_quarters((s[0] + s[1]) + (s[2] + s[3]), [](float p, float q) { return p + q; });
                        if (lc == 0) g.parts[col0 / (TILE_B / 2) * g.parts_ld + row0 + ri] = make_float2(m, sum);
                    });
            } else {
                typedef typename Elem<TYPE>::Bits Bits;
                rows([&](auto I, auto RI, float* v) __attribute__((always_inline)) {
                    constexpr int i = decltype(I)::value, ri = decltype(RI)::value;
                    constexpr float SCALE = TYPE == F16 ? lmk::SLOPE_SCALE_F16 : 1.0f;
                    const int target = mine.target[i];
                    const float lse2 = mine.lse2[i];
                    float own = 0.0f;
                    if (found) {
                        float z = 0.0f;
                        compared(target, [&](int e, int c) { z = c == 0 ? v[e] : z; });
                        own = expm1f((z * LOG2E - lse2) * 0.693147180559945309f);
                    }
                    const uint32_t keep = target == lmk::NO_TARGET ? 0u : 0xffffffffu;
                    Bits* const out = (Bits*)g.D + (row0 + ri) * g.ldd + col0 + lc * 8;
#pragma unroll
                    for (int e = 0; e < N; ++e) v[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(v[e], LOG2E, -lse2));
                    if (edge) compared(cols, [&](int e, int c) { v[e] = c > 0 ? v[e] : 0.0f; });
                    if (found) compared(target, [&](int e, int c) { v[e] = c == 0 ? own : v[e]; });
#pragma unroll
                    for (int jj = 0; jj < FB / 2; ++jj) {
                        v4i w;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            w[e] = (int)(((uint32_t)from_float<TYPE>(SCALE * v[8 * jj + 2 * e]) | (uint32_t)from_float<TYPE>(SCALE * v[8 * jj + 2 * e + 1]) << 16) & keep);
                        *(v4i*)(out + jj * 32) = w;
                    }
                });
            }
        } else if constexpr (KIND == lmk::STATES) {
            rows([&](auto, auto RI, float* v) __attribute__((always_inline)) {
                constexpr int ri = decltype(RI)::value;
                float* const out = (float*)g.D + this_split * g.split_stride + (row0 + ri) * g.ldd + col0 + lc * 4;
                if (g.beta != 0.0f) {
                    v4f old[FB];
#pragma unroll
                    for (int j = 0; j < FB; ++j) old[j] = *(const v4f*)(out + 16 * j);
#pragma unroll
                    for (int e = 0; e < N; ++e) v[e] += old[e / 4][e % 4];
                }
#pragma unroll
                for (int j = 0; j < FB; ++j) *(v4f*)(out + 16 * j) = v4f{v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
            });
        } else {
            // (each type and case a piece of code of its own, taken as a whole: woven into each other they do not fit the instruction cache, and a
            // gradient of weights of 256 x 256 sums took 25 us to write, so 14)
            auto write = [&](auto DTYPE, auto BETA, auto EDGE) __attribute__((always_inline)) {
                rows([&](auto, auto RI, float* v) __attribute__((always_inline)) {
                    constexpr int ri = decltype(RI)::value;
                    if constexpr (B_ACROSS) {
                        // two fragments' fours into eights: the odd sixteens of lanes give theirs of the first for the even ones' of the second
#pragma unroll
                        for (int e = 0; e < N; ++e)
                            if (e / 4 % 2 == 0) {
                                const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[e]), __float_as_uint(v[e + 4]), false, false);
                                v[e] = __uint_as_float(x[0]);
                                v[e + 4] = __uint_as_float(x[1]);
                            }
                    }
                    const int eight = B_ACROSS ? (lc & 1) * 16 + (lc >> 1) * 8 : lc * 8;  // of 32 columns
#pragma unroll
                    for (int jj = 0; jj < FB / 2; ++jj)
                        put<decltype(DTYPE)::value, decltype(BETA)::value, decltype(EDGE)::value>(g, alpha, row0 + ri, col0 + jj * 32 + eight, v + 8 * jj);
                });
            };
            auto write_as = [&](auto DTYPE) __attribute__((always_inline)) {
                if (whole)
                    write(DTYPE, std::false_type{}, std::false_type{});
                else if (inside)
                    write(DTYPE, std::true_type{}, std::false_type{});
                else if (g.beta == 0.0f)
                    write(DTYPE, std::false_type{}, std::true_type{});
                else
                    write(DTYPE, std::true_type{}, std::true_type{});
            };
            if (g.dtype == F32) write_as(std::integral_constant<int, F32>{});
            if (g.dtype == BF16) write_as(std::integral_constant<int, BF16>{});
            if (g.dtype == F16) write_as(std::integral_constant<int, F16>{});
        }
        stored = KIND == lmk::STATES || KIND == lmk::SLOPE || whole;
    }
    wait_vmcnt<0>();  // no copy may still be writing LDS when the workgroup retires
}

template <int TYPE, int KIND, int FA, int FB> void run(Args g, hipStream_t st)
{
    g.TM = (int)((g.m + 32 * FA - 1) / (32 * FA));
    g.TP = (int)((g.p + 32 * FB - 1) / (32 * FB));
    const int64_t items = (int64_t)g.TM * g.TP * g.splits, most = FB == 4 ? 2 * COMPUTE_UNITS : COMPUTE_UNITS;
    k_lm_tile<TYPE, KIND, FA, FB><<<dim3((unsigned)(items < most ? items : most)), dim3(256), 0, st>>>(g);
}
template <int TYPE, int KIND> void run(const Args& g, int shape, hipStream_t st)
{
    if (shape == lmk::TILE_256) run<TYPE, KIND, 8, 8>(g, st);
    if (shape == lmk::TILE_128_256) run<TYPE, KIND, 4, 8>(g, st);
    if (shape == lmk::TILE_128) run<TYPE, KIND, 4, 4>(g, st);
}

}  // namespace

namespace lmk {

// LM_TYPE: the element type that this compilation is of (the instances of both take long)
#define NAME2(type) launch_tile_##type
#define NAME(type) NAME2(type)
hipError_t NAME(LM_TYPE)(const Tile& t, hipStream_t st)
{
    const Args g = {t.m, t.n, t.p, t.b_rows, (uint64_t)(uintptr_t)t.A, (uint64_t)(uintptr_t)t.B, (uint32_t)(t.lda * 2), (uint32_t)(t.ldb * 2),
                    0, 0, (int)((t.n + STAGE_K - 1) / STAGE_K), t.splits, t.D, t.ldd, t.dtype,
                    t.alpha, t.beta, t.alpha_at, t.split_stride, t.targets, t.known, t.column0, t.lse2, t.at_target, t.parts, t.parts_ld};
    if (t.kind == LINEAR) run<LM_TYPE, LINEAR>(g, t.shape, st);
    if (t.kind == LOSS) run<LM_TYPE, LOSS>(g, t.shape, st);
    if (t.kind == SLOPE) run<LM_TYPE, SLOPE>(g, t.shape, st);
    if (t.kind == STATES) run<LM_TYPE, STATES>(g, t.shape, st);
    if (t.kind == WEIGHTS) run<LM_TYPE, WEIGHTS>(g, t.shape, st);
    return hipGetLastError();
}

}  // namespace lmk
