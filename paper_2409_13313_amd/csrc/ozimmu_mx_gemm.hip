// Product of microscaled 4-bit matrices on the matrix cores: D <- alpha A B^T + beta D (include/ozimmu_mx.h).
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 elements of 4 bits, every block of 32 with its scale, and adds
// to 16 x 16 FP32 sums: 16 cycles of a SIMD, 4096 operations a cycle.  The fragments of B are its first operand, so that a lane's four
// sums are four neighbouring columns of one row of D.
#include "ozimmu_mx_convert.h"
#include <type_traits>

namespace {

using namespace mxk;
using namespace mxl;

__device__ inline v8i operand(v4i x) { return __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1); }

template <int SEL_B, int SEL_A> __device__ inline v4f mfma(v4i b, int sb, v4i a, int sa, v4f acc)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(b), operand(a), acc, 4, 4, SEL_B, sb, SEL_A, sa);
}

constexpr int64_t COMPUTE_UNITS = 256;

// v: N sums of one row, from column col on, into D
template <int TYPE, int N> __device__ inline void finish(const Gemm& g, int64_t row, int64_t col, const float* v)
{
    typedef typename Elem<TYPE>::Bits Bits;
    if (row >= g.m || col >= g.p) return;
    Bits* const out = (Bits*)g.D + row * g.ldd + col;
    const int64_t left = g.p - col;
    Bits x[N];
    if (g.beta != 0.0f) {
        load_row<TYPE, N>(out, left, x);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = from_float<TYPE>(g.alpha * v[e] + g.beta * to_float<TYPE>(x[e]));
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = from_float<TYPE>(g.alpha * v[e]);
    }
    store_row<TYPE, N>(out, left, x);
}

template <int I, int N, class F> __device__ inline void static_for(F&& f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<I + 1, N>(f);
    }
}

// v: N sums of one row in FP32, into D of whatever type
template <int N> __device__ inline void finish_any(const Gemm& g, int64_t row, int64_t col, const float* v)
{
    if (g.dtype == F32) finish<F32, N>(g, row, col, v);
    if (g.dtype == BF16) finish<BF16, N>(g, row, col, v);
    if (g.dtype == F16) finish<F16, N>(g, row, col, v);
}

// ---- 64 rows x FB fragments of B (16 columns each) by a workgroup, operands straight from memory into registers ----
//
// For outputs too small for the tiles below, where the time is that of a launch, of the way of the operands and of one wave's share of the inner
// dimension: the waves share the inner tiles, each has one on its way at a time, and their sums meet in LDS, in a fixed order.  256 x 4096 x
// 4096 6.8 us (10 MB, 1.3 PF; a launch alone is 2.5), 512 x 4096 x 4096 9.5; beyond that operands read again by every workgroup bound it.
constexpr int DIRECT_SLOTS = 4;
template <int FB> constexpr int direct_pitch() { return 16 * FB + 4; }  // floats between the rows of a wave's sums: rows fall on different banks

template <int FB, int WAVES> __device__ inline void direct_block(const Gemm& g, int64_t block_row, int64_t block_col, float* sums)
{
    constexpr int PITCH = direct_pitch<FB>(), SLOTS = DIRECT_SLOTS;
    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t KT = inner_tiles(g.n), row0 = block_row * 64, col0 = block_col / (4 / FB) * QUARTER_R;
    const int f0 = (int)(block_col % (4 / FB)) * FB;  // first of the workgroup's fragments of the quarter
    const uint8_t* const A = g.A + row0 / TILE_R * KT * TILE_BYTES + row0 % TILE_R / QUARTER_R * QUARTER_BYTES;
    const uint8_t* const B = g.B + col0 / TILE_R * KT * TILE_BYTES + col0 % TILE_R / QUARTER_R * QUARTER_BYTES;
    v4f acc[4][FB];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < FB; ++j) acc[i][j] = v4f{0, 0, 0, 0};
    for (int64_t kt = wave; kt < KT; kt += WAVES) {
        v4i fa[4], fb[FB];
        const uint8_t* const ta = A + kt * TILE_BYTES;
        const uint8_t* const tb = B + kt * TILE_BYTES;
#pragma unroll
        for (int j = 0; j < FB; ++j) fb[j] = *(const v4i*)(tb + SCALE_BYTES + (f0 + j) * FRAGMENT_BYTES + lane * 16);
        const int sb = *(const int*)(tb + lane * 4) >> (8 * f0);
#pragma unroll
        for (int i = 0; i < 4; ++i) fa[i] = *(const v4i*)(ta + SCALE_BYTES + i * FRAGMENT_BYTES + lane * 16);
        const int sa = *(const int*)(ta + lane * 4);
        static_for<0, 4>([&](auto I) {
            static_for<0, FB>([&](auto J) {
                constexpr int i = decltype(I)::value, j = decltype(J)::value;
                acc[i][j] = mfma<j, i>(fb[j], sb, fa[i], sa, acc[i][j]);
            });
        });
    }
    // of the row at place l % 16 of fragment i, lane l holds the columns at places 4 (l / 16) .. + 3 of fragment j
    auto slot = [&](int w, int i, int j) { return (v4f*)(sums + (w * 64 + row_of(i, lane & 15)) * PITCH + j * 16 + (lane >> 4 << 2)); };
    if constexpr (WAVES > SLOTS) {
        // (as many waves again: theirs are added first)
        static_assert(WAVES == 2 * SLOTS, "two waves to a slot");
        if (wave >= SLOTS)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < FB; ++j) *slot(wave - SLOTS, i, j) = acc[i][j];
        __syncthreads();
        if (wave < SLOTS)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < FB; ++j) *slot(wave, i, j) += acc[i][j];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < FB; ++j) *slot(wave, i, j) = acc[i][j];
    }
    __syncthreads();
    constexpr int GROUPS = 64 * 4 * FB;  // of four columns
#pragma unroll
    for (int u = 0; u < (GROUPS + 64 * WAVES - 1) / (64 * WAVES); ++u) {
        const int at = u * 64 * WAVES + t;
        if (GROUPS % (64 * WAVES) != 0 && at >= GROUPS) break;
        // neighbouring threads, neighbouring columns: place 4 a + .. of fragment j is column 8 a + 4 j + .. (of 32)
        const int r = at / (4 * FB), q = at % (4 * FB), j = FB == 1 ? 0 : (q & 1) + q / 8 * 2, a = FB == 1 ? q : q / 2 % 4;
        v4f s = *(const v4f*)(sums + r * PITCH + j * 16 + 4 * a);
#pragma unroll
        for (int w = 1; w < SLOTS; ++w) s += *(const v4f*)(sums + (w * 64 + r) * PITCH + j * 16 + 4 * a);
        const float v[4] = {s[0], s[1], s[2], s[3]};
        finish_any<4>(g, row0 + r, col0 + row_of(f0 + j, 4 * a), v);
    }
}

template <int FB, int WAVES> __global__ __launch_bounds__(64 * WAVES) void k_mx_direct(Gemm g)
{
    __shared__ __align__(16) float sums[DIRECT_SLOTS * 64 * direct_pitch<FB>()];
    direct_block<FB, WAVES>(g, blockIdx.y, blockIdx.x, sums);
}

// Two products in one launch (the gradients of a small layer)
template <int FB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_mx_direct2(Gemm a, Gemm b, uint32_t cols_a, uint32_t cols_b, uint32_t blocks_a)
{
    __shared__ __align__(16) float sums[DIRECT_SLOTS * 64 * direct_pitch<FB>()];
    const bool first = blockIdx.x < blocks_a;
    const uint32_t at = first ? blockIdx.x : blockIdx.x - blocks_a, cols = first ? cols_a : cols_b;
    const Gemm g = first ? a : b;
    direct_block<FB, WAVES>(g, at / cols, at % cols, sums);
}

inline int64_t direct_units(const Gemm& g) { return (g.p + QUARTER_R - 1) / QUARTER_R * ((g.m + 63) / 64); }

template <int FB, int WAVES> void direct(const Gemm& g, const Gemm* also, hipStream_t st)
{
    const unsigned cols = (unsigned)((g.p + QUARTER_R - 1) / QUARTER_R * (4 / FB)), rows = (unsigned)((g.m + 63) / 64);
    if (!also) {
        k_mx_direct<FB, WAVES><<<dim3(cols, rows), dim3(64 * WAVES), 0, st>>>(g);
    } else {
        const unsigned cols_b = (unsigned)((also->p + QUARTER_R - 1) / QUARTER_R * (4 / FB)), rows_b = (unsigned)((also->m + 63) / 64);
        k_mx_direct2<FB, WAVES><<<dim3(cols * rows + cols_b * rows_b), dim3(64 * WAVES), 0, st>>>(g, *also, cols, cols_b, cols * rows);
    }
}

// Fewer fragments of B a workgroup where there are few workgroups (64 x 4096 x 4096, 1, 2, 4 fragments: 5.5, 5.9, 7.4 us; 256 rows: 8.0,
// 7.2, 7.7; 1024 rows: 24, 18.9, 16.7); eight waves where they all run at once and have four tiles each (64 x 8192 x 1024, 8 and 4 waves: 7.5 and
// 8.2 us; 64 x 2048 x 2048: 3.7 and 3.6).
void direct(const Gemm& g, const Gemm* also, hipStream_t st)
{
    const int64_t units = direct_units(g) + (also ? direct_units(*also) : 0);
    const bool deep = inner_tiles(g.n) >= 32 || (also && inner_tiles(also->n) >= 32);
    if (units * 4 <= COMPUTE_UNITS)
        deep ? direct<1, 8>(g, also, st) : direct<1, 4>(g, also, st);
    else if (units <= COMPUTE_UNITS * 5 / 4)
        deep && units * 2 <= COMPUTE_UNITS ? direct<2, 8>(g, also, st) : direct<2, 4>(g, also, st);
    else
        direct<4, 4>(g, also, st);
}

// ---- 256 x 256 outputs by a workgroup of four waves, 128 x 128 each: 256 FP32 sums a lane, one wave a SIMD ----
//
// A workgroup per compute unit takes one tile of the output after the other.  A stage is one tile of A and one of B (128 inner
// elements, 34 KiB).  The stages of all its output tiles are one stream from memory straight into a ring of four in LDS, four stages ahead
// of the products: while a tile's sums are written out, the first stages of the next one arrive.  A stage is one step of 64
// matrix instructions a wave, run as four quarters of 4 x 4 fragments on four sets of four fragments (16 bytes a lane each) and one
// register of scales: (A lo, B lo), (A lo, B hi), (A hi, B lo), (A hi, B hi).  Quarter 0 fetches B hi, quarter 1 A hi, quarters 2 and 3
// A lo and B lo of the next stage, so that a fragment is on its way 8 to 16 matrix instructions ahead of its first use.
// A scaled matrix instruction takes three of its four issue slots itself (a second instruction beside it costs 4 cycles, a branch 40 and more),
// so a stage has 52 other instructions for its 64, one behind a product at a time, and no branch but the one at its end.
// One barrier a stage, in its middle, where every wave has fetched all of the stage and its own copies of the next one have landed: behind
// it the stage's place in the ring takes the copies of the fourth stage from here.  Ten copies a wave and stage; those behind the last
// stage are out of the buffer's range: they read nothing, but count, so that every stage waits alike.
// Bound by power where the product is large: 8192 x 8192 x 16384 440 to 546 us (5.0 to 4.0 PF) on random operands, by what ran before (416 the
// least seen), 325 to 420 on zeros, which are the same instructions.  A register-only loop of the instruction gives 7.6 PF (with 32 x 32 x 64 6.7).  8192 x 4096 x 8192 112 us.
constexpr int RING = 4, STAGE_BYTES = 2 * TILE_BYTES, COPIES = 10;
constexpr int NXCD = 8;
constexpr int64_t MEMORY_SIDE_CACHE = (int64_t)256 << 20;

// (by the builtin: the compiler then knows, and waits for none of them again)
template <int N> __device__ inline void wait_lds()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f | N << 8);  // lgkmcnt(N)
    asm volatile("" ::: "memory");
}
template <int N> __device__ inline void wait_vmcnt() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// Workgroup b runs on XCD b % 8.  The tiles are cut into eight contiguous ranges, one an XCD, in bands of BAND tile rows walked column by
// column: the 32 tiles that an XCD works on at a time share BAND panels of A and 32 / BAND of B in its L2.  8 for tiles of 256 x 256, 4 for
// those of 256 x 128, where 8 would take a quarter more of A and B together (a linear layer of 2048 x 4096 x 4096, its quantisation included,
// 27.3 and 27.8 us).
template <int BAND> struct Order {
    int TM, TP, next, last, step;
    __device__ inline Order(int TM_, int TP_) : TM(TM_), TP(TP_)
    {
        const int T = TM * TP, xcd = blockIdx.x % NXCD, begin = xcd * (T / NXCD) + (xcd < T % NXCD ? xcd : T % NXCD);
        next = begin + blockIdx.x / NXCD;
        last = begin + T / NXCD + (xcd < T % NXCD ? 1 : 0);
        step = gridDim.x / NXCD + (xcd < (int)(gridDim.x % NXCD) ? 1 : 0);
    }
    // the next tile of this workgroup; false behind its last one
    __device__ inline bool take(int& tm, int& tp)
    {
        if (next >= last) return false;
        const int band = next / (BAND * TP), in_band = next % (BAND * TP);
        const int height = TM - band * BAND < BAND ? TM - band * BAND : BAND;
        tm = __builtin_amdgcn_readfirstlane(band * BAND + in_band % height);
        tp = __builtin_amdgcn_readfirstlane(in_band / height);
        next += step;
        return true;
    }
};

// Where the copies of an operand come from, as buffers: of the output tile at hand, and of the next one (no bytes: behind the last; nothing is
// read).  The copy of a stage is at the start of the buffer + the stage's offset, which runs from 0 to `stages` tiles in every output tile and
// is the same for A and B; the copies are AHEAD stages ahead, so the buffer of this output tile starts that much later, and that of the next
// one, which takes over within the loop, that much before its tiles.  The bytes are all that any offset reaches.  (All of it stays in scalar
// registers that scalar instructions write: the copies below are asm statements, and the compiler would not put the wait states between a
// vector instruction that writes their operands and them.)
struct Source {
    v4i now;
    uint64_t after;
    int bytes_after;
    __device__ inline void point(uint64_t at, int bytes) { now = v4i{(int)(uint32_t)at, (int)(uint32_t)(at >> 32), bytes, 0x00020000}; }
    __device__ inline uint64_t at() const { return (uint64_t)(uint32_t)now[1] << 32 | (uint32_t)now[0]; }
    __device__ inline void move(int64_t by) { point(at() + by, now[2]); }
    // the next output tile from here on: copies of its stage 0 at offset `stage` x TILE_BYTES
    __device__ inline void switch_over(int stage) { point(after - (uint64_t)stage * TILE_BYTES, bytes_after); }
};

// M0: the place in LDS that the next copies go to.  (At least one instruction has to stand between this and the first of them.)
__device__ inline void copy_to(uint32_t place, uint32_t wave_part) { asm volatile("s_add_u32 m0, %0, %1" ::"s"(place), "s"(wave_part) : "memory", "scc"); }

// Copy Q of a quarter of a tile: 256 bytes of scales (Q = 0) or a fragment.  Lane i writes LDS bytes [M0 + the instruction's offset + its 4 or
// 16 bytes); that offset moves both addresses alike, `off` only the one in memory.
template <int Q> __device__ inline void copy_quarter(uint32_t voff4, uint32_t voff16, v4i source, uint32_t off)
{
    if constexpr (Q == 0)
        asm volatile("buffer_load_dword %0, %1, %2 offen lds" ::"v"(voff4), "s"(source), "s"(off) : "memory");
    else
        asm volatile("buffer_load_dwordx4 %0, %1, %2 offen offset:%3 lds" ::"v"(voff16), "s"(source), "s"(off), "n"(SCALE_BYTES + (Q - 1) * FRAGMENT_BYTES)
                     : "memory");
}

// Eight neighbouring sums of a row into D; `left`: columns of D from the first of them on.
template <int TYPE, bool BETA>
__device__ inline void put8(__attribute__((address_space(1))) typename Elem<TYPE>::Bits* out, int left, float alpha, float beta, const float* v)
{
    typename Elem<TYPE>::Bits x[8];
    if (left >= 8) {
        if constexpr (BETA) __builtin_memcpy(x, out, sizeof(x));
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = from_float<TYPE>(BETA ? alpha * v[e] + beta * to_float<TYPE>(x[e]) : alpha * v[e]);
        __builtin_memcpy(out, x, sizeof(x));
    } else if (left > 0) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < left) out[e] = from_float<TYPE>(BETA ? alpha * v[e] + beta * to_float<TYPE>(out[e]) : alpha * v[e]);
    }
}

// The same where all eight lie inside D and its old values do not matter: written through the L2, so that the kernel's end has nothing
// left to write back (4096 x 2048 x 4096: 21.1 us, 22.5 with plain stores; 8192 x 2048 x 8192: 70 and 73.5).  STREAM: past the caches, for
// outputs that with the operands exceed the memory-side cache (8192 x 8192 x 16384, 268 MB of D: 434 us, written through 471, plain 477;
// 134 MB of D, inner dimension 4096: 128, 119, 117).  Two wait states keep what follows off the registers of a 16-byte store.
// EDGE: by the lanes alone of which NEED columns or more are left.
enum Stores { THROUGH, STREAM, EDGE };
template <int HOW, int OFFSET, int NEED> __device__ inline void store16(uint64_t base, uint32_t off, v4i y, int left)
{
    if constexpr (HOW == EDGE) {
        uint64_t all;
        asm volatile("v_cmp_le_i32 vcc, %5, %4\n\ts_and_saveexec_b64 %0, vcc\n\tglobal_store_dwordx4 %1, %2, %3 offset:%6 sc0 sc1\n\ts_nop 1\n\ts_mov_b64 exec, %0"
                     : "=&s"(all)
                     : "v"(off), "v"(y), "s"(base), "v"(left), "n"(NEED), "n"(OFFSET)
                     : "memory", "vcc", "scc");
    } else if constexpr (HOW == STREAM)
        asm volatile("global_store_dwordx4 %0, %1, %2 offset:%3 sc1 nt\n\ts_nop 1" ::"v"(off), "v"(y), "s"(base), "n"(OFFSET) : "memory");
    else
        asm volatile("global_store_dwordx4 %0, %1, %2 offset:%3 sc0 sc1\n\ts_nop 1" ::"v"(off), "v"(y), "s"(base), "n"(OFFSET) : "memory");
}
// 16-bit types: a lane stores its eight, and the four lanes of a row 64 bytes.  FP32: the lanes of a row first exchange theirs, so that
// each of two stores covers 64 bytes of a row there too (16 bytes of every 32 at a time, written through: 210 us for 8192 x 8192 x 4096).
template <int TYPE, int HOW, int COLUMN>
__device__ inline void put8_whole(uint64_t base, uint32_t off, float alpha, const float* v, int left)
{
    if constexpr (TYPE == F32) {
        v4i lo, hi;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            // quarters of the wave, first four columns p, other four q: (p0 p1 p2 p3, q0 q1 q2 q3) -> (p0 q0 p2 q2, p1 q1 p3 q3) -> (p0 q0 p1 q1, p2 q2 p3 q3)
            const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(alpha * v[e]), __float_as_uint(alpha * v[4 + e]), false, false);
            const auto y = __builtin_amdgcn_permlane32_swap(x[0], x[1], false, false);
            lo[e] = (int)y[0];
            hi[e] = (int)y[1];
        }
        store16<HOW, COLUMN * 4, 4>(base, off, lo, left);
        store16<HOW, COLUMN * 4 + 64, 20>(base, off, hi, left);
    } else {
        typename Elem<TYPE>::Bits x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = from_float<TYPE>(alpha * v[e]);
        v4i y;
        __builtin_memcpy(&y, x, 16);
        store16<HOW, COLUMN * 2, 8>(base, off, y, left);
    }
}

// A wave's sums into D: 8 x NJ fragments from row row0, column col0 on.  Fragment (i, j), register r: row at place l % 16 of fragment i % 4 of
// A's quarter i / 4, column at place 4 (l / 16) + r of fragment j % 4 of B's quarter j / 4; fragments j and j + 1 (j even) are 8 neighbouring
// columns.  whole: all of the workgroup's tile lies inside D; true is returned where that many stores were made, one for every two fragments (in
// FP32: each).
template <int TYPE, int NJ>
__device__ __attribute__((always_inline)) inline bool put_tile(const Gemm& g, v4f (&acc)[8][NJ], int64_t row0, int64_t col0, bool whole_tile, bool stream, int lane)
{
    typedef typename Elem<TYPE>::Bits Bits;
    typedef __attribute__((address_space(1))) Bits Global;
    // (left alone, the register allocator parks accumulators in scratch memory and copies all of them at once; so they are read by asm
    // statements below, and the wait states behind the last matrix instruction are written out)
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) asm volatile("" : "+a"(acc[i][j]));
    asm volatile("s_nop 15\n\ts_nop 15");
    // (lane parts made opaque here, or they are formed at kernel entry and live through everything; addresses are a uniform base and a
    // 32-bit lane offset)
    int lr = lane & 15, lc = lane >> 4;
    asm volatile("" : "+v"(lr), "+v"(lc));
    const int row_lane = row_of(0, lr), col_lane = row_of(0, lc << 2);
    const uint32_t off = ((uint32_t)row_lane * (uint32_t)g.ldd + (uint32_t)col_lane) * (uint32_t)sizeof(Bits);
    // eight sums at a time: v, the row (but for the lane's part) and the column
    auto each = [&](auto&& f) {
        static_for<0, 8>([&](auto I) {
            constexpr int i = decltype(I)::value, ri = i / 4 * 64 + row_of(i % 4, 0);
            uint64_t base = (uint64_t)(uintptr_t)((Bits*)g.D + (row0 + ri) * g.ldd + col0);
            asm volatile("" : "+s"(base));
            static_for<0, NJ / 2>([&](auto J) {
                constexpr int j = 2 * decltype(J)::value, cj = j / 4 * 64 + row_of(j % 4, 0);
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v[e]) : "a"(acc[i][j + e / 4][e % 4]));
                f(base, std::integral_constant<int, ri>{}, std::integral_constant<int, cj>{}, v);
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    };
    // rows and columns of D from this lane's first ones on (FP32: it stores columns 4 lc .. 4 lc + 3 and the 16th behind them)
    const int rows_left = (int)(g.m - row0 < 128 ? g.m - row0 : 128) - row_lane, cols = (int)(g.p - col0 < 128 ? g.p - col0 : 128);
    // (none in rows behind the last one; by a minimum: conditions kept in scalar registers spilled others)
    auto left = [&](int ri, int columns) { return min(columns, (rows_left - ri) * 256); };
    auto eights = [&](auto HOW) {
        const uint32_t off16 = TYPE == F32 ? ((uint32_t)row_lane * (uint32_t)g.ldd + (uint32_t)lc * 4u) * 4u : off;
        const int cols_left = cols - (TYPE == F32 ? lc * 4 : col_lane);
        each([&](uint64_t base, auto RI, auto CJ, const float* v) {
            constexpr int ri = decltype(RI)::value, cj = decltype(CJ)::value;
            put8_whole<TYPE, decltype(HOW)::value, cj>(base, off16, g.alpha, v, left(ri, cols_left - cj));
        });
    };
    auto ones = [&](auto BETA) {
        each([&](uint64_t base, auto RI, auto CJ, const float* v) {
            constexpr int ri = decltype(RI)::value, cj = decltype(CJ)::value;
            const int here = left(ri, cols - col_lane - cj);
            put8<TYPE, decltype(BETA)::value>((Global*)(base + off) + cj, decltype(BETA)::value || here < 8 ? here : 0, g.alpha, g.beta, v);
        });
    };
    if (g.beta != 0.0f) {
        ones(std::true_type{});
    } else if (!whole_tile) {
        eights(std::integral_constant<int, EDGE>{});
        if (cols > 0 && cols & 7) ones(std::false_type{});  // (the columns behind the last whole eight of a row)
    } else {
        if (stream)
            eights(std::integral_constant<int, STREAM>{});
        else
            eights(std::integral_constant<int, THROUGH>{});
        return true;
    }
    return false;
}

template <int TYPE> __global__ __launch_bounds__(256) void k_mx_tile(Gemm g, int KT, int TM, int TP, int stream)
{
    __shared__ __align__(16) uint8_t ring[RING * STAGE_BYTES];
    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)ring;
    const uint32_t voff4 = wave * QUARTER_BYTES + lane * 4, voff16 = wave * QUARTER_BYTES + lane * 16;
    const uint32_t m0_a = lds + wave * QUARTER_BYTES, m0_b = m0_a + TILE_BYTES;
    typedef __attribute__((address_space(3))) const v4i* lds_v4i;
    typedef __attribute__((address_space(3))) const int* lds_int;
    // this lane's bytes of fragment 0 and of the scales in the wave's first quarter of A and of B, in ring place 0
    const uint32_t fragA = lds + 2 * wm * QUARTER_BYTES + SCALE_BYTES + lane * 16;
    const uint32_t fragB = lds + TILE_BYTES + 2 * wn * QUARTER_BYTES + SCALE_BYTES + lane * 16;
    const uint32_t scaleA = lds + 2 * wm * QUARTER_BYTES + lane * 4;
    const uint32_t scaleB = lds + TILE_BYTES + 2 * wn * QUARTER_BYTES + lane * 4;

    Source a, b;
    Order<8> copy_order(TM, TP);
    const int operand_bytes = KT * TILE_BYTES;
    auto look_up = [&]() {
        int tm, tp;
        const bool any = copy_order.take(tm, tp);
        a.bytes_after = b.bytes_after = any ? operand_bytes : 0;
        if (any) {
            a.after = (uint64_t)(uintptr_t)g.A + (uint64_t)tm * operand_bytes;
            b.after = (uint64_t)(uintptr_t)g.B + (uint64_t)tp * operand_bytes;
        }
    };
    a.after = b.after = 0;
    look_up();
    a.switch_over(0);
    b.switch_over(0);
    uint32_t here = 0, to = 0;  // ring offsets: the current stage, the stage that is copied
    auto advance = [](uint32_t& place) { place = place == (RING - 1) * STAGE_BYTES ? 0 : place + STAGE_BYTES; };
    uint32_t off = 0;  // of the stage, in the operands' buffers
    auto copy_a = [&](auto Q) { copy_quarter<decltype(Q)::value>(voff4, voff16, a.now, off); };
    auto copy_b = [&](auto Q) { copy_quarter<decltype(Q)::value>(voff4, voff16, b.now, off); };
    static_for<0, RING>([&](auto S) {
        copy_to(to, m0_a);
        asm volatile("s_nop 0");
        static_for<0, COPIES / 2>(copy_a);
        if constexpr (decltype(S)::value < RING - 1) {  // (the main loop begins with the last one's B)
            copy_to(to, m0_b);
            asm volatile("s_nop 0");
            static_for<0, COPIES / 2>(copy_b);
            advance(to);
            off += TILE_BYTES;
        }
    });
    a.move(RING * TILE_BYTES);
    b.move((RING - 1) * TILE_BYTES);

    v4f acc[8][8];
    v4i faL[4], faH[4], fbL[4], fbH[4];
    int saL, saH, sbL, sbH;
    // matrix instruction X of a quarter: four on each fragment of the set that was fetched last (B's with BY_B), there and back over the other
    auto math = [&](const v4i* fa, int sa, const v4i* fb, int sb, auto I0, auto J0, auto X, auto BY_B) {
        constexpr int s = decltype(X)::value / 4, x = decltype(X)::value % 4, y = (s & 1) ? 3 - x : x;
        constexpr int i = decltype(BY_B)::value ? y : s, j = decltype(BY_B)::value ? s : y;
        v4f& c = acc[decltype(I0)::value + i][decltype(J0)::value + j];
        c = mfma<j, i>(fb[j], sb, fa[i], sa, c);
    };
    typedef std::integral_constant<int, 0> N0;
    typedef std::integral_constant<int, 4> N4;
    typedef std::true_type ByB;
    typedef std::false_type ByA;

    wait_vmcnt<(RING - 1) * COPIES - COPIES / 2>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    // addresses of the current stage and, from the middle of a stage on, of the next one
    uint32_t fa_at = fragA, fb_at = fragB, sa_at = scaleA, sb_at = scaleB;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        faL[q] = *(lds_v4i)(uintptr_t)(fa_at + q * FRAGMENT_BYTES);
        fbL[q] = *(lds_v4i)(uintptr_t)(fb_at + q * FRAGMENT_BYTES);
    }
    saL = *(lds_int)(uintptr_t)sa_at;
    sbL = *(lds_int)(uintptr_t)sb_at;

    // Stores count as copies do.  In the two stages behind the end of a tile, all of whose STORES stores were made, they are newer than
    // the copies that are waited for and need not be over; those stages have a loop of their own (with the choice between two waits in one
    // loop: a stage of k_mx_half 772 cycles, without 726).
    constexpr int STORES = TYPE == F32 ? 64 : 32, NEWER = (RING - 2) * COPIES;
    constexpr int NEWER_STORES = NEWER + STORES < 63 ? NEWER + STORES : 63;
    uint32_t fresh = 0;  // the offset of the first stage of the others
    // (forced inline: the state that it captures has to stay in registers)
    auto stage = [&](auto FRESH) __attribute__((always_inline)) {
        wait_lds<0>();
        // quarter 0: the upper half of B comes in, the first copies of B go out
        static_for<0, 16>([&](auto X) {
            constexpr int x = decltype(X)::value;
            if constexpr (x % 3 == 0 && x < 12) fbH[x / 3] = *(lds_v4i)(uintptr_t)(fb_at + QUARTER_BYTES + x / 3 * FRAGMENT_BYTES);
            if constexpr (x == 1) copy_to(to, m0_b);
            if constexpr (x == 2) copy_b(std::integral_constant<int, 0>{});
            if constexpr (x == 4) sbH = *(lds_int)(uintptr_t)(sb_at + QUARTER_BYTES);
            if constexpr (x == 5) saH = *(lds_int)(uintptr_t)(sa_at + QUARTER_BYTES);
            if constexpr (x == 8) copy_b(std::integral_constant<int, 1>{});
            if constexpr (x == 14) copy_b(std::integral_constant<int, 2>{});
            math(faL, saL, fbL, sbL, N0{}, N0{}, X, ByB{});
            __builtin_amdgcn_sched_barrier(0);
        });
        wait_lds<0>();
        // quarter 1: the upper half of A, early, so that it is there at the barrier
        static_for<0, 16>([&](auto X) {
            constexpr int x = decltype(X)::value;
            if constexpr (x % 2 == 0 && x < 8) faH[x / 2] = *(lds_v4i)(uintptr_t)(fa_at + QUARTER_BYTES + x / 2 * FRAGMENT_BYTES);
            if constexpr (x == 3) copy_b(std::integral_constant<int, 3>{});
            if constexpr (x == 9) copy_b(std::integral_constant<int, 4>{});
            if constexpr (x == 10) {
                to = here;
                advance(here);
            }
            if constexpr (x == 12) fa_at = fragA + here;
            if constexpr (x == 13) fb_at = fragB + here;
            if constexpr (x == 14) sa_at = scaleA + here;
            if constexpr (x == 15) sb_at = scaleB + here;
            math(faL, saL, fbH, sbH, N0{}, N4{}, X, ByB{});
            __builtin_amdgcn_sched_barrier(0);
        });
        wait_vmcnt<decltype(FRESH)::value ? NEWER_STORES : NEWER>();
        wait_lds<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // quarter 2: the lower half of A of the next stage (behind the last one: what the ring holds, unused); copies of A
        static_for<0, 16>([&](auto X) {
            constexpr int x = decltype(X)::value;
            if constexpr (x % 3 == 0 && x < 12) faL[x / 3] = *(lds_v4i)(uintptr_t)(fa_at + x / 3 * FRAGMENT_BYTES);
            if constexpr (x == 1) copy_to(to, m0_a);
            if constexpr (x == 2) copy_a(std::integral_constant<int, 0>{});
            if constexpr (x == 4) saL = *(lds_int)(uintptr_t)sa_at;
            if constexpr (x == 8) copy_a(std::integral_constant<int, 1>{});
            if constexpr (x == 14) copy_a(std::integral_constant<int, 2>{});
            math(faH, saH, fbL, sbL, N4{}, N0{}, X, ByA{});
            __builtin_amdgcn_sched_barrier(0);
        });
        // quarter 3: its lower half of B
        static_for<0, 16>([&](auto X) {
            constexpr int x = decltype(X)::value;
            if constexpr (x % 2 == 0 && x < 8) fbL[x / 2] = *(lds_v4i)(uintptr_t)(fb_at + x / 2 * FRAGMENT_BYTES);
            if constexpr (x == 1) sbL = *(lds_int)(uintptr_t)sb_at;
            if constexpr (x == 4) copy_a(std::integral_constant<int, 3>{});
            if constexpr (x == 10) copy_a(std::integral_constant<int, 4>{});
            math(faH, saH, fbH, sbH, N4{}, N4{}, X, ByA{});
            __builtin_amdgcn_sched_barrier(0);
        });
        off += TILE_BYTES;
    };
    Order<8> order(TM, TP);
    int tm, tp;
    while (order.take(tm, tp)) {
        look_up();
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                acc[i][j] = v4f{0, 0, 0, 0};
                asm volatile("" : "+a"(acc[i][j]));  // (in its accumulation registers from here on)
            }
        off = 0;
        while (off != fresh) stage(std::true_type{});
        // until the copies of A are the next output tile's, until those of B are, to the end (fresh stages end before)
        uint32_t until = (uint32_t)(KT - RING) * TILE_BYTES;
#pragma clang loop unroll(disable)
        for (int part = 0; part < 3; ++part) {
#pragma clang loop unroll(disable)
            while (off != until) stage(std::false_type{});
            if (part == 0) a.switch_over(KT - RING);
            if (part == 1) b.switch_over(KT - RING + 1);
            until = part == 0 ? (uint32_t)(KT - RING + 1) * TILE_BYTES : (uint32_t)operand_bytes;
        }
        a.move(operand_bytes);
        b.move(operand_bytes);
        fresh = put_tile<TYPE, 8>(g, acc, (int64_t)tm * TILE_R + wm * 128, (int64_t)tp * TILE_R + wn * 128,
                                  (int64_t)(tm + 1) * TILE_R <= g.m && (int64_t)(tp + 1) * TILE_R <= g.p, stream, lane)
                    ? (uint32_t)(KT - RING < RING - 2 ? KT - RING : RING - 2) * TILE_BYTES
                    : 0;
    }
    wait_vmcnt<0>();  // no copy may still be writing LDS when the workgroup retires
}

// Whether D goes past the caches.  What the next work reads is kept where it fits (8192 x 4096 x 8192, a layer and the quantisation of its
// output: 182 us kept, 198 past; the layer alone 168 and 162).  A gradient of weights is read when the other layers are done: past the
// caches from 16 MB on, so that the operands and the gradient handed on stay in them (backward and the quantisation of dX, dW of 34 MB:
// 70.5 kept, 68.0 past; 67 MB: 191.8 and 190.2; 134 MB: 330 and 323; dW scaled at once, kept ahead: 16 MB the same, 67 MB 191 and 201).
template <int TYPE> int streams(const Gemm& g)
{
    const int64_t bytes = g.m * g.p * (int64_t)sizeof(typename Elem<TYPE>::Bits);
    if (g.read_later) return bytes > MEMORY_SIDE_CACHE / 16;
    return packed_bytes(g.m, g.n) + packed_bytes(g.p, g.n) + bytes > MEMORY_SIDE_CACHE;
}
inline unsigned one_each(int64_t tiles) { return (unsigned)(tiles < COMPUTE_UNITS ? tiles : COMPUTE_UNITS); }

template <int TYPE> void tile(const Gemm& g, hipStream_t st)
{
    const int TM = (int)row_tiles(g.m), TP = (int)row_tiles(g.p);
    k_mx_tile<TYPE><<<dim3(one_each((int64_t)TM * TP)), dim3(256), 0, st>>>(g, (int)inner_tiles(g.n), TM, TP, streams<TYPE>(g));
}

// ---- few rows of X, quantised on the way: 16 rows and FB fragments of W's (16 columns each) by a workgroup ----
//
// The time of such a call is that of reading W once and of its launches, so this is one launch: the waves share the inner tiles, each
// takes its fragments of W straight from memory into registers, TILES of its tiles at a time, and quantises the blocks of X that meet them - a lane
// holds a block as the matrix instruction wants it, so that its scale takes no exchange between lanes.  The waves' sums meet in LDS.
// Every workgroup quantises all of X: FB is as large as leaves a workgroup for every compute unit.
// 16 rows through 16384 x 8192: 13.8 us, 72 MB at 5.2 TB/s, a large copy's rate; one row through 4096 x 4096: 4.9 us on the GPU.
constexpr int FEW_ROWS = 16;

template <int XTYPE, int FB, int WAVES, int TILES>
__global__ __launch_bounds__(64 * WAVES) void k_mx_few(Gemm g, const typename Elem<XTYPE>::Bits* X, int64_t ldx, int64_t KT)
{
    typedef typename Elem<XTYPE>::Bits Bits;
    __shared__ __align__(16) v4f sums[WAVES][FB][64];
    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t row0 = (int64_t)blockIdx.y * FEW_ROWS, col0 = (int64_t)blockIdx.x / (4 / FB) * QUARTER_R;
    const int f0 = (int)(blockIdx.x % (4 / FB)) * FB;  // first of the workgroup's fragments of the quarter
    const uint8_t* const W = g.B + col0 / TILE_R * KT * TILE_BYTES + col0 % TILE_R / QUARTER_R * QUARTER_BYTES;
    const int64_t row = row0 + (lane & 15);
    const Bits* const x_lane = X + row * ldx + (lane >> 4) * BLOCK;
    // elements of the row from the lane's block of tile 0 on
    const int64_t here = row < g.m ? g.n - (lane >> 4) * BLOCK : 0;

    v4f acc[FB];
#pragma unroll
    for (int f = 0; f < FB; ++f) acc[f] = v4f{0, 0, 0, 0};
    auto block = [&](const Bits* x, v4i& codes) -> int {
        const uint32_t b = scale_byte(f32_bits<XTYPE>(max_magnitude<XTYPE, BLOCK>(x)));
        const float s = scale_value(b);
#pragma unroll
        for (int q = 0; q < 4; ++q) codes[q] = (int)codes8<XTYPE>(x + 8 * q, s);
        return (int)b;
    };
    auto multiply = [&](const v4i* w, int sw, v4i x, int sx) {
        sw >>= 8 * f0;
        static_for<0, FB>([&](auto F) { acc[decltype(F)::value] = mfma<decltype(F)::value, 0>(w[decltype(F)::value], sw, x, sx, acc[decltype(F)::value]); });
    };
    for (int64_t kt0 = wave; kt0 < KT; kt0 += WAVES * TILES) {
        v4i w[TILES][FB];
        int sw[TILES];
        Bits x[TILES][BLOCK];
#pragma unroll
        for (int u = 0; u < TILES; ++u) {
            // (a tile behind the last one: the last one again, with zeros for X)
            const int64_t kt = kt0 + u * WAVES, at = kt < KT ? kt : KT - 1;
            const uint8_t* const tile = W + at * TILE_BYTES;
#pragma unroll
            for (int f = 0; f < FB; ++f) w[u][f] = *(const v4i*)(tile + SCALE_BYTES + (f0 + f) * FRAGMENT_BYTES + lane * 16);
            sw[u] = *(const int*)(tile + lane * 4);
            if (kt < KT && here - kt * TILE_K >= BLOCK) {
                __builtin_memcpy(x[u], x_lane + kt * TILE_K, sizeof(x[u]));
            } else {
#pragma unroll
                for (int e = 0; e < BLOCK; ++e) x[u][e] = 0;
            }
        }
#pragma unroll
        for (int u = 0; u < TILES; ++u) {
            v4i codes;
            const int sx = block(x[u], codes);
            multiply(w[u], sw[u], codes, sx);
        }
    }
    // the block that a row ends in, where it is not a whole one: zeros for the others
    if (g.n % BLOCK != 0 && wave == (int)((KT - 1) % WAVES)) {
        const uint8_t* const tile = W + (KT - 1) * TILE_BYTES;
        const int64_t left = here - (KT - 1) * TILE_K;
        v4i w[FB], codes;
        Bits x[BLOCK];
#pragma unroll
        for (int f = 0; f < FB; ++f) w[f] = *(const v4i*)(tile + SCALE_BYTES + (f0 + f) * FRAGMENT_BYTES + lane * 16);
        const int sw = *(const int*)(tile + lane * 4);
#pragma unroll
        for (int e = 0; e < BLOCK; ++e) x[e] = left < BLOCK && e < left ? x_lane[(KT - 1) * TILE_K + e] : 0;
        const int sx = block(x, codes);
        multiply(w, sw, codes, sx);
    }
#pragma unroll
    for (int f = 0; f < FB; ++f) sums[wave][f][lane] = acc[f];
    __syncthreads();
    // lane l of fragment f: columns at places 4 (l / 16) .. + 3 for row l % 16
    if (t < FB * 64) {
        const int f = t >> 6;
        v4f s = sums[0][f][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) s += sums[w][f][lane];
        const float v[4] = {s[0], s[1], s[2], s[3]};
        finish_any<4>(g, row, col0 + row_of(f0 + f, lane >> 4 << 2), v);
    }
}

template <int XTYPE, int FB, int WAVES, int TILES> void few(const Gemm& g, const void* X, int64_t ldx, hipStream_t st)
{
    const dim3 grid((unsigned)((g.p + QUARTER_R - 1) / QUARTER_R * (4 / FB)), (unsigned)((g.m + FEW_ROWS - 1) / FEW_ROWS));
    k_mx_few<XTYPE, FB, WAVES, TILES><<<grid, dim3(64 * WAVES), 0, st>>>(g, (const typename Elem<XTYPE>::Bits*)X, ldx, inner_tiles(g.n));
}

// One round of workgroups on the 256 compute units (beyond that two launches are faster: 48 rows through 8192 x 8192 19.3 us in two, 22.1 in
// one; 32 rows 18.8 and 13.6), up to 64 rows (64 rows through 4096 x 4096 7.8 us, in two 8.7; 96 rows 12.1 and 9.2), of as few fragments each as that allows: the more workgroups, the more of W on its way at a time (16 rows
// through 4096 x 4096: 1, 2, 4 fragments 6.9, 7.0, 7.5 us; 4096 x 14336: 18.4, 11.4, 8.8).  Up to 16 rows any number of rounds.
inline int64_t few_units(int64_t m, int64_t p) { return (p + QUARTER_R - 1) / QUARTER_R * ((m + FEW_ROWS - 1) / FEW_ROWS); }

// Four rows and fewer: little of the time goes into X, and sixteen waves with one tile each bring W in sooner than eight with two (one row
// through 16384 x 4096: 11.4 and 15.3 us; twelve rows: 20.2 and 17.2).
template <int XTYPE> void few(const Gemm& g, const void* X, int64_t ldx, hipStream_t st)
{
    const int64_t units = few_units(g.m, g.p);
    if (units * 4 <= COMPUTE_UNITS)
        g.m <= 4 ? few<XTYPE, 1, 16, 1>(g, X, ldx, st) : few<XTYPE, 1, 8, 2>(g, X, ldx, st);
    else if (units * 2 <= COMPUTE_UNITS)
        g.m <= 4 ? few<XTYPE, 2, 16, 1>(g, X, ldx, st) : few<XTYPE, 2, 8, 2>(g, X, ldx, st);
    else
        // (one tile each: also where there are no more, 12 rows through 1024 x 65536 9.2 and 11.2 us)
        g.m <= 8 || inner_tiles(g.n) <= 8 ? few<XTYPE, 4, 8, 1>(g, X, ldx, st) : few<XTYPE, 4, 8, 2>(g, X, ldx, st);
}

// ---- 256 x 128 outputs by a workgroup: the same with half a tile of B, for outputs of too few tiles ----
//
// A wave has 128 x 64 outputs; a stage (26 KiB) is 32 matrix instructions of it, (A lo, B) and (A hi, B), and the ring has six places.  A fragment
// of B gives way to the next stage's as soon as its last four products are done.  In LDS B is four pieces of two fragments, each behind the
// scales of its quarter, one from each wave.
// 2048 x 4096 x 4096, one tile for each compute unit: 20.3 us (3.4 PF), of 37000 cycles 23000 the stages (726 each; 512 were the matrix
// instructions alone, 70 the loop, 55 the barrier, 45 the copies, 30 LDS), 5000 the ring's first filling, 5000 the stores, 2000 their end.  A ring of four: within 2 %.
constexpr int HALF_RING = 6, PIECE_BYTES = SCALE_BYTES + 2 * FRAGMENT_BYTES, HALF_STAGE_BYTES = TILE_BYTES + 4 * PIECE_BYTES, HALF_COPIES = 8;

template <int TYPE> __global__ __launch_bounds__(256) void k_mx_half(Gemm g, int KT, int TM, int TP, int stream)
{
    __shared__ __align__(16) uint8_t ring[HALF_RING * HALF_STAGE_BYTES];
    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)ring;
    const uint32_t voffA4 = wave * QUARTER_BYTES + lane * 4, voffA16 = wave * QUARTER_BYTES + lane * 16;
    const uint32_t voffB4 = (wave >> 1) * QUARTER_BYTES + lane * 4, voffB16 = (wave >> 1) * QUARTER_BYTES + (wave & 1) * 2 * FRAGMENT_BYTES + lane * 16;
    const uint32_t m0_a = lds + wave * QUARTER_BYTES, m0_b = lds + TILE_BYTES + wave * PIECE_BYTES;
    typedef __attribute__((address_space(3))) const v4i* lds_v4i;
    typedef __attribute__((address_space(3))) const int* lds_int;
    const uint32_t fragA = lds + 2 * wm * QUARTER_BYTES + SCALE_BYTES + lane * 16, scaleA = lds + 2 * wm * QUARTER_BYTES + lane * 4;
    const uint32_t fragB = lds + TILE_BYTES + 2 * wn * PIECE_BYTES + SCALE_BYTES + lane * 16, scaleB = lds + TILE_BYTES + 2 * wn * PIECE_BYTES + lane * 4;

    Source a, b;
    Order<4> copy_order(TM, TP);
    const int operand_bytes = KT * TILE_BYTES;
    auto look_up = [&]() {
        int tm, tp;
        const bool any = copy_order.take(tm, tp);
        a.bytes_after = b.bytes_after = any ? operand_bytes : 0;
        if (any) {
            a.after = (uint64_t)(uintptr_t)g.A + (uint64_t)tm * operand_bytes;
            b.after = (uint64_t)(uintptr_t)g.B + (uint64_t)(tp >> 1) * operand_bytes + (uint64_t)(tp & 1) * 2 * QUARTER_BYTES;
        }
    };
    a.after = b.after = 0;
    look_up();
    a.switch_over(0);
    b.switch_over(0);
    uint32_t here = 0, to = 0;  // ring offsets: the current stage, the stage that is copied
    auto advance = [](uint32_t& place) { place = place == (HALF_RING - 1) * HALF_STAGE_BYTES ? 0 : place + HALF_STAGE_BYTES; };
    uint32_t off = 0;
    auto copy_a = [&](auto Q) { copy_quarter<decltype(Q)::value>(voffA4, voffA16, a.now, off); };
    auto copy_b = [&](auto Q) { copy_quarter<decltype(Q)::value>(voffB4, voffB16, b.now, off); };
    static_for<0, HALF_RING>([&](auto S) {
        copy_to(to, m0_a);
        asm volatile("s_nop 0");
        static_for<0, 5>(copy_a);
        if constexpr (decltype(S)::value < HALF_RING - 1) {  // (the main loop begins with the last one's B)
            copy_to(to, m0_b);
            asm volatile("s_nop 0");
            static_for<0, 3>(copy_b);
            advance(to);
            off += TILE_BYTES;
        }
    });
    a.move(HALF_RING * TILE_BYTES);
    b.move((HALF_RING - 1) * TILE_BYTES);

    v4f acc[8][4];
    v4i faL[4], faH[4], fb[4];
    int saL, saH, sb;
    // matrix instruction X of a half of A: four on each fragment of B, there and back over those of A
    auto math = [&](const v4i* fa, int sa, auto I0, auto X) {
        constexpr int j = decltype(X)::value / 4, x = decltype(X)::value % 4, i = (j & 1) ? 3 - x : x;
        v4f& c = acc[decltype(I0)::value + i][j];
        c = mfma<j, i>(fb[j], sb, fa[i], sa, c);
    };
    typedef std::integral_constant<int, 0> N0;
    typedef std::integral_constant<int, 4> N4;

    wait_vmcnt<(HALF_RING - 1) * HALF_COPIES - 3>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    uint32_t fa_at = fragA, fb_at = fragB, sa_at = scaleA, sb_at = scaleB;
    auto piece = [](int f) { return f / 2 * PIECE_BYTES + f % 2 * FRAGMENT_BYTES; };
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        faL[q] = *(lds_v4i)(uintptr_t)(fa_at + q * FRAGMENT_BYTES);
        fb[q] = *(lds_v4i)(uintptr_t)(fb_at + piece(q));
    }
    saL = *(lds_int)(uintptr_t)sa_at;
    sb = *(lds_int)(uintptr_t)sb_at;

    // (as above: stores newer than the copies that are waited for need not be over; here in the four stages behind a tile)
    constexpr int STORES = TYPE == F32 ? 32 : 16, NEWER = (HALF_RING - 2) * HALF_COPIES;
    constexpr int NEWER_STORES = NEWER + STORES < 63 ? NEWER + STORES : 63;
    uint32_t fresh = 0;
    // (forced inline: the state that it captures has to stay in registers)
    auto stage = [&](auto FRESH) __attribute__((always_inline)) {
        // (A lo, B): the upper half of A comes in, early, so that it is there at the barrier; copies of B
        static_for<0, 16>([&](auto X) {
            constexpr int x = decltype(X)::value;
            if constexpr (x % 2 == 0 && x < 8) faH[x / 2] = *(lds_v4i)(uintptr_t)(fa_at + QUARTER_BYTES + x / 2 * FRAGMENT_BYTES);
            if constexpr (x == 1) copy_to(to, m0_b);
            if constexpr (x == 3) copy_b(std::integral_constant<int, 0>{});
            if constexpr (x == 5) saH = *(lds_int)(uintptr_t)(sa_at + QUARTER_BYTES);
            if constexpr (x == 7) copy_b(std::integral_constant<int, 1>{});
            if constexpr (x == 9) copy_b(std::integral_constant<int, 2>{});
            if constexpr (x == 10) {
                to = here;
                advance(here);
            }
            if constexpr (x == 12) fa_at = fragA + here;
            if constexpr (x == 13) fb_at = fragB + here;
            if constexpr (x == 14) sa_at = scaleA + here;
            if constexpr (x == 15) sb_at = scaleB + here;
            math(faL, saL, N0{}, X);
            __builtin_amdgcn_sched_barrier(0);
        });
        wait_vmcnt<decltype(FRESH)::value ? NEWER_STORES : NEWER>();
        wait_lds<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // (A hi, B): the lower half of A and B of the next stage (behind the last one: what the ring holds, unused); copies of A
        int sb_next;
        static_for<0, 16>([&](auto X) {
            constexpr int x = decltype(X)::value;
            if constexpr (x % 2 == 0 && x < 8) faL[x / 2] = *(lds_v4i)(uintptr_t)(fa_at + x / 2 * FRAGMENT_BYTES);
            if constexpr (x == 1) copy_to(to, m0_a);
            if constexpr (x == 3) copy_a(std::integral_constant<int, 0>{});
            if constexpr (x == 5) saL = *(lds_int)(uintptr_t)sa_at;
            if constexpr (x == 7) sb_next = *(lds_int)(uintptr_t)sb_at;
            if constexpr (x == 9) copy_a(std::integral_constant<int, 1>{});
            if constexpr (x == 11) copy_a(std::integral_constant<int, 2>{});
            if constexpr (x == 13) copy_a(std::integral_constant<int, 3>{});
            if constexpr (x == 14) copy_a(std::integral_constant<int, 4>{});
            if constexpr (x == 8) fb[0] = *(lds_v4i)(uintptr_t)(fb_at + piece(0));
            if constexpr (x == 10) fb[1] = *(lds_v4i)(uintptr_t)(fb_at + piece(1));
            if constexpr (x == 12) fb[2] = *(lds_v4i)(uintptr_t)(fb_at + piece(2));
            math(faH, saH, N4{}, X);
            __builtin_amdgcn_sched_barrier(0);
        });
        fb[3] = *(lds_v4i)(uintptr_t)(fb_at + piece(3));
        sb = sb_next;
        off += TILE_BYTES;
        wait_lds<2>();
    };
    Order<4> order(TM, TP);
    int tm, tp;
    while (order.take(tm, tp)) {
        look_up();
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc[i][j] = v4f{0, 0, 0, 0};
                asm volatile("" : "+a"(acc[i][j]));
            }
        off = 0;
        while (off != fresh) stage(std::true_type{});
        uint32_t until = (uint32_t)(KT - HALF_RING) * TILE_BYTES;
#pragma clang loop unroll(disable)
        for (int part = 0; part < 3; ++part) {
            wait_lds<0>();  // (here and not at every stage: its last fetch, which is the last to be used, may be on its way then)
#pragma clang loop unroll(disable)
            while (off != until) stage(std::false_type{});
            if (part == 0) a.switch_over(KT - HALF_RING);
            if (part == 1) b.switch_over(KT - HALF_RING + 1);
            until = part == 0 ? (uint32_t)(KT - HALF_RING + 1) * TILE_BYTES : (uint32_t)operand_bytes;
        }
        a.move(operand_bytes);
        b.move(operand_bytes);
        fresh = put_tile<TYPE, 4>(g, acc, (int64_t)tm * TILE_R + wm * 128, (int64_t)tp * 128 + wn * 64,
                                  (int64_t)(tm + 1) * TILE_R <= g.m && (int64_t)(tp + 1) * 128 <= g.p, stream, lane)
                    ? (uint32_t)(KT - HALF_RING < HALF_RING - 2 ? KT - HALF_RING : HALF_RING - 2) * TILE_BYTES
                    : 0;
    }
    wait_vmcnt<0>();
}

template <int TYPE> void half(const Gemm& g, hipStream_t st)
{
    const int TM = (int)row_tiles(g.m), TP = (int)((g.p + 127) / 128);
    k_mx_half<TYPE><<<dim3(one_each((int64_t)TM * TP)), dim3(256), 0, st>>>(g, (int)inner_tiles(g.n), TM, TP, streams<TYPE>(g));
}

template <int TYPE> void product(const Gemm& g, int way, hipStream_t st)
{
    if (way == WAY_TILE)
        tile<TYPE>(g, st);
    else if (way == WAY_HALF)
        half<TYPE>(g, st);
    else
        direct(g, nullptr, st);
}

}  // namespace

namespace mxk {

// (32-bit offsets of a lane inside 28 rows of D, and 32-bit numbers of tiles)
bool way_fits(int way, int64_t m, int64_t n, int64_t p, int64_t ldd)
{
    if (way == WAY_TILE || way == WAY_HALF)
        return inner_tiles(n) >= (way == WAY_TILE ? RING : HALF_RING) && inner_tiles(n) < ((int64_t)1 << 31) / TILE_BYTES && ldd < (1 << 24) &&
               row_tiles(m) * row_tiles(p) < ((int64_t)1 << 28);
    return way == WAY_DIRECT;
}

// Microseconds that each way takes, roughly: the tiles by rounds of one for every compute unit, slower stages where more of those are at
// work (`fill`: clock and memory), k_mx_direct by its workgroups.  Fitted to
// (m x n x p: direct, half, tile)  256 x 4096 x 4096: 6.8, 15.4, 23.6;  1024 x 4096 x 4096: 17.0, 16.1, 23.5;  2048 x 4096 x 4096: 32.4, 20.0, 25.0;
// 4096 x 4096 x 4096: 63, 35.6, 33.7;  512 x 8192 x 8192: 29.2, 26.5, 40.3;  1024 x 8192 x 8192: 56, 32.9, 41.8;  2048 x 8192 x 8192: 112, 62, 56;
// 512 x 1024 x 8192: 9.6, 8.3, 11.4;  256 x 4096 x 14336: 17.8, 16.7, 24.4;  512 x 4096 x 14336: 33.0, 17.9, 25.0;  1024 x 4096 x 14336: 58, 32.5, 29.0;
// 768 x 4096 x 14336: 47, 31.2, 26.1;  2048 x 2048 x 2048: 11.9, 11.1, 15.7;  8192 x 2048 x 8192: 152, 74.5, 66.6;  4096 x 2051 x 1283: 19.8, 15.3, 24.1.
// Not in it, as it decides nothing at these: the writing of a large D of a short inner dimension (8192 x 512 x 8192: 110, -, 58, estimated 87, -, 29) and
// the length of the walk in few workgroups (64 x 8192 x 1024: 7.6, 23.6, 37.3, estimated 3.5, 26.2, 39.8).  beta != 0 takes longer in the tiles (2048 x 4096 x
// 4096: 20.4 us and 29.7) and in k_mx_direct (8192 x 128 x 8192: 88 and 160).
double estimate_us(int way, int64_t m, int64_t n, int64_t p)
{
    const double KT = (double)inner_tiles(n);
    if (way == WAY_DIRECT) return 3.0 + (double)(((m + 63) / 64) * ((p + 63) / 64)) * (0.0035 + 0.0004 * KT);
    const int64_t tiles = way == WAY_TILE ? row_tiles(m) * row_tiles(p) : row_tiles(m) * ((p + 127) / 128);
    const double rounds = (double)((tiles + COMPUTE_UNITS - 1) / COMPUTE_UNITS), fill = (double)tiles / (rounds * COMPUTE_UNITS);
    if (way == WAY_TILE) return 4.3 + rounds * (2.9 + KT * (0.51 + 0.28 * fill * fill));
    return 2.5 + rounds * (3.0 + KT * (0.32 + 0.10 * fill));
}

int choose(int64_t m, int64_t n, int64_t p, int64_t ldd)
{
    int best = WAY_DIRECT;
    for (int way : {WAY_TILE, WAY_HALF})
        if (way_fits(way, m, n, p, ldd) && estimate_us(way, m, n, p) < estimate_us(best, m, n, p)) best = way;
    return best;
}

bool few_rows(int64_t m, int64_t p) { return m <= FEW_ROWS || (m <= 4 * FEW_ROWS && few_units(m, p) <= COMPUTE_UNITS); }

hipError_t launch_few(const Gemm& g, int xtype, const void* X, int64_t ldx, hipStream_t st)
{
    if (xtype == F32) few<F32>(g, X, ldx, st);
    if (xtype == BF16) few<BF16>(g, X, ldx, st);
    if (xtype == F16) few<F16>(g, X, ldx, st);
    return hipGetLastError();
}

hipError_t launch_gemm(const Gemm& g, int way, hipStream_t st)
{
    if (way == WAY_AUTO) way = choose(g.m, g.n, g.p, g.ldd);
    if (g.dtype == F32) product<F32>(g, way, st);
    if (g.dtype == BF16) product<BF16>(g, way, st);
    if (g.dtype == F16) product<F16>(g, way, st);
    return hipGetLastError();
}

// Two products that do not depend on each other: in one launch where both are small
hipError_t launch_gemm2(const Gemm& a, const Gemm& b, hipStream_t st)
{
    if (choose(a.m, a.n, a.p, a.ldd) == WAY_DIRECT && choose(b.m, b.n, b.p, b.ldd) == WAY_DIRECT &&
        direct_units(a) + direct_units(b) <= 4 * COMPUTE_UNITS) {
        direct(a, &b, st);
        return hipGetLastError();
    }
    const hipError_t e = launch_gemm(a, WAY_AUTO, st);
    return e != hipSuccess ? e : launch_gemm(b, WAY_AUTO, st);
}

}  // namespace mxk
