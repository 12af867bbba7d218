// Weights in 4 bits with a scale per group (ozimmu_lm.h): quantisation, reading back, the plain layout, and the product of rows of 16 bits with
// them straight from the stored form.
#include "ozimmu_lm.h"
#include <type_traits>

namespace {

using namespace mxk;
using namespace lml;
using lmk::Linear;
using lmk::Weights;

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

constexpr int64_t COMPUTE_UNITS = 256;

template <int I, int N, class F> __device__ __attribute__((always_inline)) inline void static_for(F&& f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<I + 1, N>(f);
    }
}

// eight codes, element e at bits 4 e, and the order they are stored in
__device__ inline uint32_t stored_order(uint32_t w)
{
    uint32_t r = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) r |= (w >> (4 * e) & 15u) << (e % 2 * 16 + e / 2 * 4);
    return r;
}
__device__ inline uint32_t plain_order(uint32_t w)
{
    uint32_t r = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) r |= (w >> (e % 2 * 16 + e / 2 * 4) & 15u) << (4 * e);
    return r;
}
__device__ inline int code_at(uint32_t stored, int e) { return (int)(stored >> (e % 2 * 16 + e / 2 * 4) & 15u); }

__device__ inline float scale_float(int stype, uint16_t s) { return stype == BF16 ? to_float<BF16>(s) : to_float<F16>(s); }

// A row's record, as much of it as a block has
template <int GROUP> struct Record {
    static constexpr int GROUPS = INNER / GROUP, WORDS = (GROUPS * 3 + 3) / 4;
    uint32_t w[WORDS];
    __device__ inline void load(const uint8_t* p) { __builtin_memcpy(w, p, sizeof(w)); }
    __device__ inline uint16_t scale(int q) const { return (uint16_t)(w[q / 2] >> (q % 2 * 16)); }
    __device__ inline uint32_t zero(int q) const { return w[(2 * GROUPS + q) / 4] >> ((2 * GROUPS + q) % 4 * 8) & 255u; }
};

// A workgroup of 256 threads takes a block of 16 rows x 128 elements, thread t the eight elements t % 16 of row t / 16: 16 lanes read or write 128
// elements side by side, and a group lies in 4, 8 or 16 neighbouring lanes.
constexpr int64_t BLOCKS_Y = 32768;  // (there may be more blocks of rows than a grid has in its second dimension)
__device__ inline int64_t row_block() { return (int64_t)blockIdx.z * BLOCKS_Y + blockIdx.y; }
inline dim3 grid_of(int64_t inner_blocks, int64_t row_blocks)
{
    return dim3((unsigned)inner_blocks, (unsigned)(row_blocks < BLOCKS_Y ? row_blocks : BLOCKS_Y), (unsigned)((row_blocks + BLOCKS_Y - 1) / BLOCKS_Y));
}
struct Place {
    int64_t block, row, col;
    int place, chunk;  // of the row in the block, of the eight in the row
    __device__ inline Place(const Shape& s, int64_t row_block)
    {
        place = threadIdx.x >> 4;
        chunk = threadIdx.x & 15;
        block = row_block * s.inner_blocks() + blockIdx.x;
        row = row_block * ROWS + place;
        col = (int64_t)blockIdx.x * INNER + chunk * 8;
    }
    // where the word of the eight codes is, and the row's record
    __device__ inline int64_t word() const { return block * BLOCK_BYTES + ((chunk & 3) * 16 + place) * 16 + (chunk >> 2) * 4; }
    __device__ inline int64_t record(const Shape& s) const { return s.records_at() + (block * ROWS + place) * s.record(); }
};

// over neighbouring lanes: 4, 8 or 16 of them
template <int LANES, class T, class F> __device__ inline T over_lanes(T v, F&& f)
{
    auto moved = [&](auto CTRL) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(CTRL)::value, 0xf, 0xf, false));
    };
    v = f(v, moved(std::integral_constant<int, 0xb1>{}));                            // lane ^ 1
    v = f(v, moved(std::integral_constant<int, 0x4e>{}));                            // lane ^ 2
    if constexpr (LANES >= 8) v = f(v, moved(std::integral_constant<int, 0x141>{}));   // the other four of eight
    if constexpr (LANES >= 16) v = f(v, moved(std::integral_constant<int, 0x140>{}));  // the other eight of sixteen
    return v;
}

// ---- quantisation ----

// x / D, rounded once: with r the FP32 number nearest to 1 / D, q = x r and what q is short of, x - D q, exactly, q + (x - D q) r is the nearest
// number to the quotient (Markstein 1990).  Below 2^-100, where x - D q may not be a normal number, and for what is no number, by a division.
template <int D> __device__ inline float over(float x)
{
    constexpr float r = 1.0f / D;
    const float q = x * r;
    float y = __builtin_fmaf(__builtin_fmaf(-(float)D, q, x), r, q);
    if (__any((x < 0x1p-100f && x != 0.0f) || !(x < __builtin_inff()))) {
        asm volatile("");  // (a branch, and not both)
        y = x / (float)D;
    }
    return y;
}

// x / scale rounded to a whole number is x times the hardware's 1 / scale rounded, unless that lies so near to half way between two whole numbers that the
// quotient, as an FP32 number, may round the other way: the two differ by at most 2^-22 of them (1 / scale by 2^-23, the quotient by 2^-24), below
// 2^-17 up to 16, and what is beyond 16 becomes 0 or 15 in either form.  Where a lane has such a one the wave looks again: elements of 16 bits
// are half way then (quotients of two numbers of 11 bits are 2^-14 off it or not at all, and x = scale / 2 is no rare number), and the even
// neighbour is taken; those of 32 bits are divided.  The rounding is that of an addition to 1.5 x 2^23, whose last bits are the code then.
template <int TYPE, int GROUP, bool ZEROS>
__device__ inline void quantize_eight(const Shape& s, int stype, const typename Elem<TYPE>::Bits (&raw)[8], const Place& at, bool tail, uint8_t* out)
{
    constexpr int LANES = GROUP / 8;
    constexpr float WHOLE = 12582912.0f, NEAR = 0.5f - 0x1p-17f;
    const auto larger = [](auto a, auto b) { return a > b ? a : b; };
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = to_float<TYPE>(raw[e]);
    // (magnitudes as whole numbers: NaN above infinity above all others)
    const float amax = __uint_as_float(over_lanes<LANES>(f32_bits<TYPE>(max_magnitude<TYPE, 8>(raw)), larger));
    const bool finite = amax < __builtin_inff();
    float range, lo = 0.0f;
    if constexpr (ZEROS) {
        float hi = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            hi = fmaxf(hi, x[e]);
            lo = fminf(lo, x[e]);
        }
        hi = over_lanes<LANES>(hi, larger);
        lo = -over_lanes<LANES>(-lo, larger);
        range = over<15>(hi - lo);
    } else {
        range = over<7>(amax);
    }
    uint16_t bits;  // (a range that the type cannot hold: its largest number)
    if (stype == BF16) {
        bits = from_float<BF16>(range);
        if (bits == 0x7f80u) bits = 0x7f7fu;
        if (!finite) bits = 0x7fc0u;
    } else {
        bits = from_float<F16>(range);
        if (bits == 0x7c00u) bits = 0x7bffu;
        if (!finite) bits = 0x7e00u;
    }
    const float scale = scale_float(stype, bits);
    const bool some = scale > 0.0f;
    // (it overflows for the smallest scales in BF16, and is none of the hardware's numbers for the largest)
    const float inverse = some ? __builtin_amdgcn_rcpf(scale) : 0.0f;
    const auto short_of = [&](float v, float rounded) { return __builtin_fmaf(v, inverse, -rounded); };
    float zero = 8.0f, near = 0.0f;
    if constexpr (ZEROS) {
        zero = __builtin_fmaf(-lo, inverse, WHOLE) - WHOLE;
        near = fabsf(short_of(-lo, zero));
    }
    float q[8];  // the quotients rounded, + zero, + 1.5 x 2^23
    const float base = WHOLE + (ZEROS ? __builtin_amdgcn_fmed3f(zero, 0.0f, 15.0f) : 8.0f);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        q[e] = __builtin_fmaf(x[e], inverse, base);
        near = fmaxf(near, fabsf(short_of(x[e], q[e] - base)));
    }
    const bool close = !(near < NEAR), by_division = !finite || (some && !(scale > 0x1p-120f && scale < 0x1p+120f)) || (TYPE == F32 && close);
    if (__any(by_division)) {
        if constexpr (ZEROS) zero = some ? rintf(-lo / scale) : 0.0f;
        zero = __builtin_amdgcn_fmed3f(zero, 0.0f, 15.0f);
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = WHOLE + zero + (some ? __builtin_amdgcn_fmed3f(rintf(x[e] / scale), -16.0f, 16.0f) : 0.0f);
    } else if (TYPE != F32 && __any(close)) {
        // (half way: to the even neighbour)
        const auto even = [&](float v, float rounded) {
            const float e = short_of(v, rounded), half = 0.5f * rounded;
            return fabsf(e) >= NEAR && fabsf(e) <= 0.5f + 0x1p-17f && rintf(half) != half ? rounded + copysignf(1.0f, e) : rounded;
        };
        if constexpr (ZEROS) zero = even(-lo, zero);
        zero = __builtin_amdgcn_fmed3f(zero, 0.0f, 15.0f);
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = WHOLE + zero + even(x[e], __builtin_amdgcn_fmed3f(q[e] - base, -32.0f, 32.0f));
    }
    if constexpr (ZEROS) zero = __builtin_amdgcn_fmed3f(zero, 0.0f, 15.0f);
    uint32_t codes[2] = {0, 0};  // of even and of odd elements
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        uint32_t c = __float_as_uint(__builtin_amdgcn_fmed3f(q[e], WHOLE, WHOLE + 15.0f));
        if (tail && at.col + e >= s.n) c = __float_as_uint(WHOLE);
        codes[e % 2] += c << (e / 2 * 4);
    }
    constexpr uint32_t FOUR = 0x4b400000u * 0x1111u;
    if (at.row >= s.p) return;
    *(uint32_t*)(out + at.word()) = (codes[0] - FOUR) | (codes[1] - FOUR) << 16;
    if (at.chunk % LANES == 0) {
        if (tail && at.col >= s.n) bits = 0;
        uint8_t* const record = out + at.record(s);
        __builtin_memcpy(record + 2 * (at.chunk / LANES), &bits, 2);
        if (ZEROS) record[2 * s.groups() + at.chunk / LANES] = (uint8_t)zero;
    }
}

// A thread takes eight elements of each of two rows, whose loads are on their way together.  16384 x 8192 in BF16, groups of 128: 83 us, 337 MB at
// 4.1 TB/s (a copy 4.7), where vector instructions and memory take as long as each other: with a division for each element it was 118.
template <int TYPE, int GROUP, bool ZEROS>
__global__ __launch_bounds__(256) void k_lm_quantize(Shape s, int stype, const typename Elem<TYPE>::Bits* W, int64_t ldw, uint8_t* out)
{
    typename Elem<TYPE>::Bits raw[2][8];
    const int64_t pair = row_block();
    if (2 * pair >= s.row_blocks()) return;
    const bool tail = blockIdx.x == gridDim.x - 1;
    const Place at[2] = {Place(s, 2 * pair), Place(s, 2 * pair + 1)};
#pragma unroll
    for (int i = 0; i < 2; ++i) load_row<TYPE, 8>(W + at[i].row * ldw + at[i].col, at[i].row < s.p ? (tail ? s.n - at[i].col : 8) : 0, raw[i]);
#pragma unroll
    for (int i = 0; i < 2; ++i) quantize_eight<TYPE, GROUP, ZEROS>(s, stype, raw[i], at[i], tail, out);
}

// over a workgroup of 256 threads
template <class F> __device__ inline float over_workgroup(float v, F&& f)
{
    __shared__ float of_wave[4];
    for (int far = 1; far < 64; far *= 2) v = f(v, __shfl_xor(v, far));
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = v;
    __syncthreads();
    return f(f(of_wave[0], of_wave[1]), f(of_wave[2], of_wave[3]));
}

// The largest finite scale, in BF16, of rows row0 .. row0 + rows - 1 (row0: a multiple of 16), by parts of their records.  A launch: 4096 x 4096 4.2 us,
// 16384 x 4096 6.4.
__global__ __launch_bounds__(256) void k_scale_peaks(Weights w, int64_t row0, int64_t rows, float* peaks)
{
    const Shape& s = w.shape;
    const int64_t KB = s.inner_blocks(), first = row0 / ROWS * KB, records = (rows + ROWS - 1) / ROWS * KB * ROWS;
    const int groups = s.groups();
    const uint8_t* const at = w.data + s.records_at() + first * ROWS * s.record();
    int most = 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < records; i += (int64_t)gridDim.x * 256) {
        // (what stands in padding rows is no scale)
        if (i / (ROWS * KB) * ROWS + i % ROWS >= rows) continue;
        for (int q = 0; q < groups; ++q) {
            uint16_t bits;
            __builtin_memcpy(&bits, at + i * s.record() + 2 * q, 2);
            const int magnitude = bits & 0x7fff;
            most = max(most, magnitude < 0x7f80 ? magnitude : 0);
        }
    }
    const float peak = over_workgroup(to_float<BF16>((uint16_t)most), [](float a, float b) { return fmaxf(a, b); });
    if (threadIdx.x == 0) peaks[blockIdx.x] = peak;
}

// ---- reading back ----
// A thread takes eight elements of each of two rows.  Bound by its stores: 16384 x 8192 into BF16 48 us, 268 MB at 5.6 TB/s beside 70 MB of codes from the
// memory-side cache (a copy 4.7, stores alone 6.9).
// Where rows begin at multiples of 16 bytes they go PAST the caches (with one row a thread 58 us, else 98), or, where a product reads them next, THROUGH L2, which has nothing left to
// write back then when the kernel ends (4096 x 4096 with the product of 2048 rows: 2.5 of 68 us less).
//
// RAISED: into FP16 from scales in BF16, whose range is larger.  Weights are held times 2^up, which brings the largest scale to 2^11 .. 2^12 (fifteen of it are a
// number of FP16), so that those down to 2^-28 of the largest keep all digits; *factor is 2^-up.  `peaks`: the largest scales by parts of the matrix.
constexpr int PEAKS = lmk::SCALE_PEAKS;
enum Stores { PLAIN, PAST, THROUGH, RAISED };
template <int TYPE, int GROUP, int STORES>
__global__ __launch_bounds__(256) void k_lm_dequantize(Weights w, int64_t row0, int64_t rows, int64_t cols, typename Elem<TYPE>::Bits* X, int64_t ldx,
                                                       const float* peaks, float* factor)
{
    typedef typename Elem<TYPE>::Bits Bits;
    const Shape& s = w.shape;
    int up = 0;
    if constexpr (STORES == RAISED) {
        static_assert(PEAKS == 256, "a number a thread");
        const float most = over_workgroup(peaks[threadIdx.x], [](float a, float b) { return fmaxf(a, b); });
        // (no more than leaves a normal number as the factor)
        up = most > 0.0f ? min(12 - __builtin_amdgcn_frexp_expf(most), 120) : 0;
        if (threadIdx.x == 0 && blockIdx.x == 0 && row_block() == 0) *factor = ldexpf(1.0f, -up);
    }
    const int64_t pair = row0 / ROWS + 2 * row_block();  // (row0: a multiple of 16)
    const Place at[2] = {Place(s, pair), Place(s, pair + 1)};
    const int64_t left = cols - at[0].col;
    if (left <= 0) return;
    const int g = at[0].chunk / (GROUP / 8);
    uint32_t codes[2];
    uint16_t bits[2];
    int zero[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (at[i].row >= row0 + rows) break;
        codes[i] = *(const uint32_t*)(w.data + at[i].word());
        const uint8_t* const record = w.data + at[i].record(s);
        __builtin_memcpy(&bits[i], record + 2 * g, 2);
        zero[i] = s.zeros ? record[2 * s.groups() + g] : 8;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (at[i].row >= row0 + rows) break;
        const float scale = STORES == RAISED ? ldexpf(scale_float(w.stype, bits[i]), up) : scale_float(w.stype, bits[i]);
        Bits x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = at[i].col + e < s.n ? from_float<TYPE>((float)(code_at(codes[i], e) - zero[i]) * scale) : 0;
        Bits* const to = X + (at[i].row - row0) * ldx + at[i].col;
        if (STORES == PLAIN || left < 8) {
            store_row<TYPE, 8>(to, left, x);
            continue;
        }
        v4i y[sizeof(x) / 16];
        __builtin_memcpy(y, x, sizeof(x));
#pragma unroll
        for (int h = 0; h < (int)(sizeof(x) / 16); ++h) {
            if constexpr (STORES == PAST)
                __builtin_nontemporal_store(y[h], (v4i*)to + h);
            else
                asm volatile("global_store_dwordx4 %0, %1, off sc0 sc1\n\ts_nop 1" ::"v"((v4i*)to + h), "v"(y[h]) : "memory");
        }
    }
}

// ---- the plain layout: a word of eight codes a thread, changed over between the two orders; both ways once for a model that is loaded or stored.
// pack and unpack, us:  4096 x 4096 9.1, 9.2 (1.9 TB/s);  16384 x 8192 53, 52 (2.6);  131072 x 4096, groups of 64 with zero points, 333, 349 (1.7) ----
__global__ __launch_bounds__(256) void k_lm_pack(Shape s, const uint8_t* codes, int64_t ldc, const uint16_t* scales, int64_t lds, const uint8_t* zeros,
                                                 int64_t ldz, uint8_t* out)
{
    const Place at(s, row_block());
    if (at.row >= s.p) return;
    uint32_t w = 0;
    const uint8_t* const from = codes + at.row * ldc + at.col / 2;
    if (at.col + 8 <= s.n) {
        __builtin_memcpy(&w, from, 4);
    } else {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            if (at.col + 2 * b >= s.n) break;
            w |= (at.col + 2 * b + 1 >= s.n ? from[b] & 15u : (uint32_t)from[b]) << (8 * b);
        }
    }
    *(uint32_t*)(out + at.word()) = stored_order(w);
    const int per = s.group / 8;
    if (at.chunk % per == 0) {
        const int64_t g = at.col / s.group;
        const bool real = at.col < s.n;
        const uint16_t scale = real ? scales[at.row * lds + g] : 0;
        uint8_t* const record = out + at.record(s);
        __builtin_memcpy(record + 2 * (at.chunk / per), &scale, 2);
        if (s.zeros) record[2 * s.groups() + at.chunk / per] = real ? zeros[at.row * ldz + g] & 15 : 0;
    }
}

__global__ __launch_bounds__(256) void k_lm_unpack(Shape s, const uint8_t* in, uint8_t* codes, int64_t ldc, uint16_t* scales, int64_t lds, uint8_t* zeros,
                                                   int64_t ldz)
{
    const Place at(s, row_block());
    if (at.row >= s.p || at.col >= s.n) return;
    const uint32_t w = plain_order(*(const uint32_t*)(in + at.word()));
    uint8_t* const to = codes + at.row * ldc + at.col / 2;
    if (at.col + 8 <= s.n) {
        __builtin_memcpy(to, &w, 4);
    } else {
#pragma unroll
        for (int b = 0; b < 4; ++b)
            if (at.col + 2 * b < s.n) to[b] = (uint8_t)(w >> (8 * b));
    }
    const int per = s.group / 8;
    if (at.chunk % per == 0) {
        const int64_t g = at.col / s.group;
        const uint8_t* const record = in + at.record(s);
        uint16_t scale;
        __builtin_memcpy(&scale, record + 2 * (at.chunk / per), 2);
        scales[at.row * lds + g] = scale;
        if (s.zeros) zeros[at.row * ldz + g] = record[2 * s.groups() + at.chunk / per];
    }
}

// ---- D <- alpha X W^T + beta D from the stored form: 16 MF rows of X and 16 PF of W by a workgroup ----
//
// A code becomes a 16-bit number by one mask and one or: 128 + q as BF16, 1024 + q as FP16, both exact.  FP16 pairs then have 1024 + zero
// taken off, again exactly; BF16 has no such instruction, so its groups are summed with the 128 and (128 + zero) times the sum of X, which one more
// matrix instruction a step gives, is taken off the group's sum in FP32.  So no weight is rounded: a group's sum is multiplied by its scale in FP32.
// The waves share the blocks of 128 inner elements; their sums meet in LDS in a fixed order.
template <int XTYPE> __device__ inline v4f mfma(v4i x, v4i w, v4f c)
{
    if constexpr (XTYPE == BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, x), __builtin_bit_cast(v8bf, w), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, x), __builtin_bit_cast(v8h, w), c, 0, 0, 0);
}

template <int XTYPE> __device__ inline v4i numbers(uint32_t w, float zero)
{
    // (in a vector register: an instruction takes one scalar operand, and the mask is one)
    uint32_t one = XTYPE == BF16 ? 0x43004300u : 0x64006400u;
    asm("" : "+v"(one));
    const _Float16 off = (_Float16)(-1024.0f - zero);
    v4i r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t v = (w >> (4 * i) & 0x000f000fu) | one;
        r[i] = XTYPE == BF16 ? (int)v : __builtin_bit_cast(int, __builtin_bit_cast(v2h, v) + v2h{off, off});
    }
    return r;
}

// FOUR: at most four rows, row i at place 4 i of the fragment, so that a lane's first sum is the one that counts
//
// Bound by memory: what it takes is reading the codes once.  16 x 8192 x 16384 (70 MB) 18 us, 1 x 4096 x 131072 (293 MB) 57 us, 5.2 TB/s; 1 x 4096 x 4096
// (8.7 MB) 4.7 us and 4.3 from the caches, of which 2 are a launch's start and end.  A second block on its way beside the one that is multiplied gives
// nothing (20.8 and 20.7 us, 69 and 65: fewer waves); X in LDS is worth its barriers from more rows on (k_lm_shared).
//
// STREAM: codes past the caches, of weights that do not fit into the 256 MB of the memory-side cache (293 MB, one row: 57 us, else 61).  Smaller ones may
// stay there from one token to the next, and then it costs (8.7 MB, one row: 5.0 and 4.3 us; 70 MB, 16 rows, three such matrices in turn: 18.9 and 18.2; ten
// of them 19.1 and 20.7).
//
// ODD, for more than four rows: rows of X may begin at odd elements.  A load of 16 bytes takes twice as long where it does not begin at a whole word, and
// each of X is made by every workgroup; so whole words are loaded, one more where the elements begin in the middle of one, and shifted when they are
// multiplied (16 x 4099 x 4096, rows 4099 apart: 8.7 us, else 13.7; 4100 apart 6.8;  37 x 2051 x 1283: 11.3, else 14.1; 9.2).  (A word that is loaded holds an
// element of the row: what lies beside it in that word is shifted out.)
template <int XTYPE, int GROUP, int MF, int PF, int WAVES, bool FOUR, bool STREAM, bool ODD>
__global__ __launch_bounds__(64 * WAVES) void k_lm_direct(Linear g, Weights w)
{
    static_assert(!FOUR || MF == 1, "four rows are one fragment");
    typedef typename Elem<XTYPE>::Bits Bits;
    constexpr int STEPS = GROUP / 32, GROUPS = 4 / STEPS, R = FOUR ? 1 : 4;
    __shared__ __align__(16) float sums[WAVES][MF][PF][64][R];
    const Shape& s = w.shape;
    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int KB = (int)s.inner_blocks();
    const int64_t last_rows = s.row_blocks() - 1;
    const int64_t pb0 = (int64_t)blockIdx.x * PF, row0 = (int64_t)blockIdx.y * (16 * MF);
    const uint8_t* code_at[PF];
    const uint8_t* record_at[PF];
    const int record = s.record();
#pragma unroll
    for (int f = 0; f < PF; ++f) {
        // (blocks of rows behind the last one: the last one again, not stored)
        const int64_t block = (pb0 + f < last_rows ? pb0 + f : last_rows) * KB;
        code_at[f] = w.data + block * BLOCK_BYTES + lane * 16;
        record_at[f] = w.data + s.records_at() + (block * ROWS + (lane & 15)) * record;
    }
    const Bits* x_at[MF];
#pragma unroll
    for (int i = 0; i < MF; ++i) {
        const int64_t row = row0 + 16 * i + (FOUR ? (lane & 15) >> 2 : lane & 15);
        x_at[i] = (const Bits*)g.X + (row < g.m ? row : g.m - 1) * g.ldx + (lane >> 4) * 8;
    }
    // ODD: to the word that the row begins in, and the bits in front of it there
    uint32_t shift[MF];
    if constexpr (ODD)
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            shift[i] = (uint32_t)(uintptr_t)x_at[i] % 4 * 8;
            x_at[i] -= shift[i] / 16;
        }
    const int left = (int)s.n - (lane >> 4) * 8;  // elements of a row from this lane's first on

    float acc[MF][PF][R];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int f = 0; f < PF; ++f)
#pragma unroll
            for (int r = 0; r < R; ++r) acc[i][f][r] = 0.0f;

    struct Stored {
        v4i code;
        Record<GROUP> record;
    };
    struct Rows {
        v4i x[MF][4];
        uint32_t last[MF][4];  // ODD: the words behind them
    };
    auto load = [&](int kb, Stored (&o)[PF], Rows& rows) __attribute__((always_inline)) {
#pragma unroll
        for (int f = 0; f < PF; ++f) {
            const v4i* const from = (const v4i*)(code_at[f] + (int64_t)kb * BLOCK_BYTES);
            o[f].code = STREAM ? __builtin_nontemporal_load(from) : *from;
            o[f].record.load(record_at[f] + (int64_t)kb * (ROWS * record));
        }
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Bits* const from = x_at[i] + kb * INNER + 32 * j;
                rows.x[i][j] = v4i{0, 0, 0, 0};
                if constexpr (ODD) rows.last[i][j] = 0;
                if (left - kb * INNER - 32 * j >= 8) {
                    __builtin_memcpy(&rows.x[i][j], from, 16);
                    // (none where the eight end with the fourth)
                    if constexpr (ODD) __builtin_memcpy(&rows.last[i][j], from + (shift[i] ? 8 : 6), 4);
                }
            }
    };
    const v4i ones = {0x3f803f80, 0x3f803f80, 0x3f803f80, 0x3f803f80};
    auto multiply = [&](const Stored (&o)[PF], Rows& rows) __attribute__((always_inline)) {
        v4i(&x)[MF][4] = rows.x;
        if constexpr (ODD)
#pragma unroll
            for (int i = 0; i < MF; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[i][j][e] = (int)__builtin_amdgcn_alignbit(e < 3 ? (uint32_t)x[i][j][e + 1 & 3] : rows.last[i][j], (uint32_t)x[i][j][e], shift[i]);
        static_for<0, GROUPS>([&](auto Q) __attribute__((always_inline)) {
            constexpr int q = decltype(Q)::value;
            v4f xs[MF];
            if constexpr (XTYPE == BF16)
#pragma unroll
                for (int i = 0; i < MF; ++i) {
                    xs[i] = v4f{0, 0, 0, 0};
#pragma unroll
                    for (int j = q * STEPS; j < (q + 1) * STEPS; ++j) xs[i] = mfma<XTYPE>(x[i][j], ones, xs[i]);
                }
#pragma unroll
            for (int f = 0; f < PF; ++f) {
                const float scale = scale_float(w.stype, o[f].record.scale(q)), zero = s.zeros ? (float)o[f].record.zero(q) : 8.0f;
                v4f c[MF];
#pragma unroll
                for (int i = 0; i < MF; ++i) c[i] = v4f{0, 0, 0, 0};
#pragma unroll
                for (int j = q * STEPS; j < (q + 1) * STEPS; ++j) {
                    const v4i b = numbers<XTYPE>((uint32_t)o[f].code[j], zero);
#pragma unroll
                    for (int i = 0; i < MF; ++i) c[i] = mfma<XTYPE>(x[i][j], b, c[i]);
                }
#pragma unroll
                for (int i = 0; i < MF; ++i)
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const float sum = XTYPE == BF16 ? __builtin_fmaf(-128.0f - zero, xs[i][r], c[i][r]) : c[i][r];
                        acc[i][f][r] = __builtin_fmaf(scale, sum, acc[i][f][r]);
                    }
            }
        });
    };

    // one block on its way while the other is multiplied
    Stored o[2][PF];
    Rows x[2];
    if (wave < KB) load(wave, o[0], x[0]);
    for (int kb = wave; kb < KB; kb += 2 * WAVES) {
        if (kb + WAVES < KB) load(kb + WAVES, o[1], x[1]);
        multiply(o[0], x[0]);
        if (kb + WAVES < KB) {
            if (kb + 2 * WAVES < KB) load(kb + 2 * WAVES, o[0], x[0]);
            multiply(o[1], x[1]);
        }
    }
    // the eight elements that a row ends in, where they are not whole: zeros for the others
    if (s.n % 8 != 0 && wave == (KB - 1) % WAVES) {
        load(KB - 1, o[0], x[0]);
        if constexpr (ODD)  // (one by one, and nothing to shift)
#pragma unroll
            for (int i = 0; i < MF; ++i) {
                x_at[i] += shift[i] / 16;
                shift[i] = 0;
            }
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int here = left - (KB - 1) * INNER - 32 * j;
                Bits e[8];
#pragma unroll
                for (int n = 0; n < 8; ++n) e[n] = here < 8 && n < here ? x_at[i][(KB - 1) * INNER + 32 * j + n] : 0;
                __builtin_memcpy(&x[0].x[i][j], e, 16);
            }
        multiply(o[0], x[0]);
    }
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int f = 0; f < PF; ++f)
#pragma unroll
            for (int r = 0; r < R; ++r) sums[wave][i][f][lane][r] = acc[i][f][r];
    __syncthreads();
    // lane l: column l % 16 of fragment f, rows 4 (l / 16) + r (FOUR: row l / 16)
    for (int at = t; at < MF * PF * 64; at += 64 * WAVES) {
        const int l = at & 63, f = at / 64 % PF, i = at / (64 * PF);
        const int64_t col = (pb0 + f) * ROWS + (l & 15);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float v = sums[0][i][f][l][r];
#pragma unroll
            for (int u = 1; u < WAVES; ++u) v += sums[u][i][f][l][r];
            const int64_t row = row0 + 16 * i + (FOUR ? l >> 4 : (l >> 4) * 4 + r);
            if (row >= g.m || col >= s.p) continue;
            const int64_t to = row * g.ldd + col;
            auto out = [&](auto D) {
                constexpr int DTYPE = decltype(D)::value;
                typedef typename Elem<DTYPE>::Bits Out;
                Out* const d = (Out*)g.D + to;
                *d = from_float<DTYPE>(g.beta != 0.0f ? g.alpha * v + g.beta * to_float<DTYPE>(*d) : g.alpha * v);
            };
            if (g.dtype == F32) out(std::integral_constant<int, F32>{});
            if (g.dtype == BF16) out(std::integral_constant<int, BF16>{});
            if (g.dtype == F16) out(std::integral_constant<int, F16>{});
        }
    }
}

// ---- the same for more rows: X goes through LDS, 16 MF rows of it and 64 PF columns of the result by a workgroup ----
//
// Four waves take 16 PF columns each and share blocks of 16 MF rows x 128 of X, which come through registers (so that rows may begin anywhere)
// into two places in LDS: while one block is multiplied the next is on its way, and the codes as well.  In LDS the 16-byte pieces of a
// fragment's 16 rows are exchanged by their number in the row, so that neither the writes, of a row's 16 pieces, nor the reads, of a piece
// of 16 rows, fall on the same banks.  What a workgroup reads of X serves 64 PF columns (k_lm_direct: 16 PF), so for few rows the inner
// dimension is split over workgroups, whose sums meet in a second launch.
//
// Bound by vector instructions (seven for eight codes, beside the matrix instruction they feed) and, where there are few rows, by the start and end of two
// launches.  4096 x 4096, groups of 128, BF16: 32 rows 12.1 us, 128 17.7, 512 34 (0.5 PFLOP/s); beyond, weights are read back (choose).
struct Shared {
    Linear g;
    Weights w;
    int splits;
    float* parts;        // splits > 1: [split][row][column] of whole workgroups
    int64_t parts_ld, parts_stride;
};

// the sum of eight elements in BF16
__device__ inline float sum_of(v4i x)
{
    float even = 0.0f, odd = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        even += __uint_as_float((uint32_t)x[i] << 16);
        odd += __uint_as_float((uint32_t)x[i] & 0xffff0000u);
    }
    return even + odd;
}

template <int XTYPE, int GROUP, int MF, int PF> __global__ __launch_bounds__(256, MF * PF > 8 ? 2 : 3) void k_lm_shared(Shared a)
{
    typedef typename Elem<XTYPE>::Bits Bits;
    constexpr int STEPS = GROUP / 32, GROUPS = 4 / STEPS, ROWS_X = 16 * MF;
    constexpr bool SUMS = XTYPE == BF16;
    __shared__ __align__(16) uint8_t held[2][MF * 4096];
    __shared__ __align__(16) float sums[2][SUMS ? GROUPS : 1][ROWS_X];
    const Linear& g = a.g;
    const Weights& w = a.w;
    const Shape& s = w.shape;
    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int KB = (int)s.inner_blocks(), k0 = (int)((int64_t)KB * blockIdx.z / a.splits), k1 = (int)((int64_t)KB * (blockIdx.z + 1) / a.splits);
    const int64_t last_rows = s.row_blocks() - 1, pb0 = (int64_t)blockIdx.x * (4 * PF) + wave * PF, row0 = (int64_t)blockIdx.y * ROWS_X;
    const uint8_t* code_at[PF];
    const uint8_t* record_at[PF];
    const int record = s.record();
#pragma unroll
    for (int f = 0; f < PF; ++f) {
        // (blocks of rows behind the last one: the last one again, not stored)
        const int64_t block = (pb0 + f < last_rows ? pb0 + f : last_rows) * KB;
        code_at[f] = w.data + block * BLOCK_BYTES + lane * 16;
        record_at[f] = w.data + s.records_at() + (block * ROWS + (lane & 15)) * record;
    }
    // X: thread t has piece t % 16 of rows t / 16 + 16 i
    const int piece = t & 15, x_row = t >> 4;
    const Bits* x_at[MF];
#pragma unroll
    for (int i = 0; i < MF; ++i) {
        const int64_t row = row0 + 16 * i + x_row;
        x_at[i] = (const Bits*)g.X + (row < g.m ? row : g.m - 1) * g.ldx + piece * 8;
    }
    const int left = (int)s.n - piece * 8, to = (piece >> 2) * 1024 + (piece & 3) * 256 + ((x_row ^ piece) << 4);

    struct Stored {
        v4i code;
        Record<GROUP> record;
    };
    Stored o[2][PF];
    v4i x[MF];
    auto load = [&](int kb, Stored (&o)[PF]) __attribute__((always_inline)) {
#pragma unroll
        for (int f = 0; f < PF; ++f) {
            o[f].code = *(const v4i*)(code_at[f] + (int64_t)kb * BLOCK_BYTES);
            o[f].record.load(record_at[f] + (int64_t)kb * (ROWS * record));
        }
    };
    auto load_x = [&](int kb) __attribute__((always_inline)) {
        const int here = left - kb * INNER;
        if (here >= 8) {
#pragma unroll
            for (int i = 0; i < MF; ++i) __builtin_memcpy(&x[i], x_at[i] + kb * INNER, 16);
        } else {
#pragma unroll
            for (int i = 0; i < MF; ++i) {
                Bits e[8];
#pragma unroll
                for (int n = 0; n < 8; ++n) e[n] = n < here ? x_at[i][kb * INNER + n] : 0;
                __builtin_memcpy(&x[i], e, 16);
            }
        }
    };
    auto hold = [&](int place) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            *(v4i*)(held[place] + i * 4096 + to) = x[i];
            if constexpr (SUMS) {
                const float sum = over_lanes<GROUP / 8>(sum_of(x[i]), [](float p, float q) { return p + q; });
                if (piece % (GROUP / 8) == 0) sums[place][piece / (GROUP / 8)][16 * i + x_row] = sum;
            }
        }
    };

    float acc[MF][PF][4];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int f = 0; f < PF; ++f)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][f][r] = 0.0f;
    const int q = lane >> 4, place_x = lane & 15;
    auto multiply = [&](int place, const Stored (&o)[PF]) __attribute__((always_inline)) {
        static_for<0, GROUPS>([&](auto Q) __attribute__((always_inline)) {
            constexpr int n = decltype(Q)::value;
            v4f c[MF][PF];
#pragma unroll
            for (int i = 0; i < MF; ++i)
#pragma unroll
                for (int f = 0; f < PF; ++f) c[i][f] = v4f{0, 0, 0, 0};
#pragma unroll
            for (int j = n * STEPS; j < (n + 1) * STEPS; ++j) {
                v4i xf[MF];
#pragma unroll
                for (int i = 0; i < MF; ++i) xf[i] = *(const v4i*)(held[place] + i * 4096 + j * 1024 + q * 256 + ((place_x ^ (4 * j + q)) << 4));
#pragma unroll
                for (int f = 0; f < PF; ++f) {
                    const v4i b = numbers<XTYPE>((uint32_t)o[f].code[j], s.zeros ? (float)o[f].record.zero(n) : 8.0f);
#pragma unroll
                    for (int i = 0; i < MF; ++i) c[i][f] = mfma<XTYPE>(xf[i], b, c[i][f]);
                }
                __builtin_amdgcn_sched_barrier(0);  // (fetched one step ahead of all, X would fill the registers)
            }
#pragma unroll
            for (int i = 0; i < MF; ++i) {
                v4f xs = {0, 0, 0, 0};
                if constexpr (SUMS) xs = *(const v4f*)&sums[place][n][16 * i + 4 * q];
#pragma unroll
                for (int f = 0; f < PF; ++f) {
                    const float scale = scale_float(w.stype, o[f].record.scale(n)), zero = s.zeros ? (float)o[f].record.zero(n) : 8.0f;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        acc[i][f][r] = __builtin_fmaf(scale, SUMS ? __builtin_fmaf(-128.0f - zero, xs[r], c[i][f][r]) : c[i][f][r], acc[i][f][r]);
                }
            }
            // (added here and now: put off, the sums of all groups would fill the registers)
#pragma unroll
            for (int i = 0; i < MF; ++i)
#pragma unroll
                for (int f = 0; f < PF; ++f)
#pragma unroll
                    for (int r = 0; r < 4; ++r) asm volatile("" : "+v"(acc[i][f][r]));
            __builtin_amdgcn_sched_barrier(0);
        });
    };

    if (k0 < k1) {
        load(k0, o[0]);
        load_x(k0);
        hold(0);
    }
    __syncthreads();
    auto step = [&](int kb, auto PLACE) __attribute__((always_inline)) {
        constexpr int place = decltype(PLACE)::value;
        const bool more = kb + 1 < k1;
        if (more) {
            load(kb + 1, o[1 - place]);
            load_x(kb + 1);
        }
        multiply(place, o[place]);
        if (more) hold(1 - place);
        __syncthreads();
    };
    for (int kb = k0; kb < k1; kb += 2) {
        step(kb, std::integral_constant<int, 0>{});
        if (kb + 1 < k1) step(kb + 1, std::integral_constant<int, 1>{});
    }

    // lane l: column l % 16 of fragment f, rows 4 (l / 16) + r of fragment i
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int f = 0; f < PF; ++f)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t row = row0 + 16 * i + 4 * q + r, col = (pb0 + f) * ROWS + place_x;
                const float v = acc[i][f][r];
                if (a.splits > 1) {
                    a.parts[(int64_t)blockIdx.z * a.parts_stride + row * a.parts_ld + col] = v;
                    continue;
                }
                if (row >= g.m || col >= s.p) continue;
                auto out = [&](auto D) {
                    constexpr int DTYPE = decltype(D)::value;
                    auto* const d = (typename Elem<DTYPE>::Bits*)g.D + row * g.ldd + col;
                    *d = from_float<DTYPE>(g.beta != 0.0f ? g.alpha * v + g.beta * to_float<DTYPE>(*d) : g.alpha * v);
                };
                if (g.dtype == F32) out(std::integral_constant<int, F32>{});
                if (g.dtype == BF16) out(std::integral_constant<int, BF16>{});
                if (g.dtype == F16) out(std::integral_constant<int, F16>{});
            }
}

// The sums of the splits, in their order
template <int DTYPE> __global__ __launch_bounds__(256) void k_lm_meet(Shared a)
{
    typedef typename Elem<DTYPE>::Bits Bits;
    const Linear& g = a.g;
    const int64_t p = a.w.shape.p, fours = (p + 3) / 4;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < g.m * fours; at += (int64_t)gridDim.x * 256) {
        const int64_t row = at / fours, col = at % fours * 4;
        const float* const from = a.parts + row * a.parts_ld + col;
        v4f v = *(const v4f*)from;
        for (int s = 1; s < a.splits; ++s) v += *(const v4f*)(from + s * a.parts_stride);
        Bits* const d = (Bits*)g.D + row * g.ldd + col;
        Bits y[4];
        if (g.beta != 0.0f) load_row<DTYPE, 4>(d, p - col, y);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = from_float<DTYPE>(g.beta != 0.0f ? g.alpha * v[e] + g.beta * to_float<DTYPE>(y[e]) : g.alpha * v[e]);
        store_row<DTYPE, 4>(d, p - col, y);
    }
}

template <int XTYPE, int GROUP, int MF, int PF> void shared(const Shared& a, hipStream_t st)
{
    const dim3 grid((unsigned)((a.w.shape.row_blocks() + 4 * PF - 1) / (4 * PF)), (unsigned)((a.g.m + 16 * MF - 1) / (16 * MF)), (unsigned)a.splits);
    k_lm_shared<XTYPE, GROUP, MF, PF><<<grid, dim3(256), 0, st>>>(a);
}
template <int XTYPE, int GROUP> void shared(const Shared& a, const lmk::SharedPlan& plan, hipStream_t st)
{
    if (plan.rows == 32 && plan.columns == 128) shared<XTYPE, GROUP, 2, 2>(a, st);
    if (plan.rows == 32 && plan.columns == 256) shared<XTYPE, GROUP, 2, 4>(a, st);
    if (plan.rows == 64 && plan.columns == 128) shared<XTYPE, GROUP, 4, 2>(a, st);
    if (plan.rows == 64 && plan.columns == 256) shared<XTYPE, GROUP, 4, 4>(a, st);
}
template <int XTYPE> void shared(const Shared& a, const lmk::SharedPlan& plan, hipStream_t st)
{
    if (a.w.shape.group == 32) shared<XTYPE, 32>(a, plan, st);
    if (a.w.shape.group == 64) shared<XTYPE, 64>(a, plan, st);
    if (a.w.shape.group == 128) shared<XTYPE, 128>(a, plan, st);
}

template <int XTYPE, int GROUP, int MF, int PF, int WAVES, bool FOUR, bool STREAM = false> void direct(const Linear& g, const Weights& w, hipStream_t st)
{
    const dim3 grid((unsigned)((w.shape.row_blocks() + PF - 1) / PF), (unsigned)((g.m + 16 * MF - 1) / (16 * MF)));
    if constexpr (!FOUR)
        if ((uintptr_t)g.X % 4 != 0 || g.ldx % 2 != 0) {
            k_lm_direct<XTYPE, GROUP, MF, PF, WAVES, FOUR, STREAM, true><<<grid, dim3(64 * WAVES), 0, st>>>(g, w);
            return;
        }
    k_lm_direct<XTYPE, GROUP, MF, PF, WAVES, FOUR, STREAM, false><<<grid, dim3(64 * WAVES), 0, st>>>(g, w);
}

template <int XTYPE, int GROUP> void direct(const Linear& g, const Weights& w, hipStream_t st)
{
    const int64_t units = w.shape.row_blocks();
    const bool stream = w.shape.bytes() >= (int64_t)1 << 28;
    if (g.m <= 4) {
        if (units <= COMPUTE_UNITS) return direct<XTYPE, GROUP, 1, 1, 16, true>(g, w, st);
        if (units <= 4 * COMPUTE_UNITS) return direct<XTYPE, GROUP, 1, 2, 16, true>(g, w, st);
        if (units <= 16 * COMPUTE_UNITS) return direct<XTYPE, GROUP, 1, 2, 8, true>(g, w, st);
        return stream ? direct<XTYPE, GROUP, 1, 4, 4, true, true>(g, w, st) : direct<XTYPE, GROUP, 1, 4, 4, true>(g, w, st);
    }
    if (g.m <= 16) {
        if (units <= COMPUTE_UNITS) return direct<XTYPE, GROUP, 1, 1, 8, false>(g, w, st);
        if (units < 4 * COMPUTE_UNITS) return direct<XTYPE, GROUP, 1, 2, 8, false>(g, w, st);
        if (units <= 16 * COMPUTE_UNITS) return stream ? direct<XTYPE, GROUP, 1, 4, 8, false, true>(g, w, st) : direct<XTYPE, GROUP, 1, 4, 8, false>(g, w, st);
        return stream ? direct<XTYPE, GROUP, 1, 4, 4, false, true>(g, w, st) : direct<XTYPE, GROUP, 1, 4, 4, false>(g, w, st);
    }
    if (g.m <= 32) {
        if (units < 2 * COMPUTE_UNITS) return direct<XTYPE, GROUP, 2, 1, 8, false>(g, w, st);
        return direct<XTYPE, GROUP, 2, 2, 8, false>(g, w, st);
    }
    const int64_t all = units * ((g.m + 63) / 64);
    if (all < 2 * COMPUTE_UNITS) return direct<XTYPE, GROUP, 4, 1, 8, false>(g, w, st);
    if (all < 8 * COMPUTE_UNITS) return direct<XTYPE, GROUP, 4, 2, 8, false>(g, w, st);
    return direct<XTYPE, GROUP, 4, 4, 4, false>(g, w, st);
}
template <int XTYPE> void direct(const Linear& g, const Weights& w, hipStream_t st)
{
    if (w.shape.group == 32) direct<XTYPE, 32>(g, w, st);
    if (w.shape.group == 64) direct<XTYPE, 64>(g, w, st);
    if (w.shape.group == 128) direct<XTYPE, 128>(g, w, st);
}

inline dim3 grid_of(const Shape& s) { return grid_of(s.inner_blocks(), s.row_blocks()); }

template <int TYPE, int GROUP> void quantize(const void* W, int64_t ldw, const Shape& s, int stype, void* packed, hipStream_t st)
{
    const dim3 grid = grid_of(s.inner_blocks(), (s.row_blocks() + 1) / 2);
    const auto* w = (const typename Elem<TYPE>::Bits*)W;
    s.zeros ? k_lm_quantize<TYPE, GROUP, true><<<grid, dim3(256), 0, st>>>(s, stype, w, ldw, (uint8_t*)packed)
            : k_lm_quantize<TYPE, GROUP, false><<<grid, dim3(256), 0, st>>>(s, stype, w, ldw, (uint8_t*)packed);
}
template <int TYPE> void quantize(const void* W, int64_t ldw, const Shape& s, int stype, void* packed, hipStream_t st)
{
    if (s.group == 32) quantize<TYPE, 32>(W, ldw, s, stype, packed, st);
    if (s.group == 64) quantize<TYPE, 64>(W, ldw, s, stype, packed, st);
    if (s.group == 128) quantize<TYPE, 128>(W, ldw, s, stype, packed, st);
}

template <int TYPE, int GROUP>
void dequantize(const Weights& w, int64_t row0, int64_t rows, int64_t cols, void* X, int64_t ldx, bool through, float* peaks, hipStream_t st)
{
    const dim3 grid = grid_of((cols + INNER - 1) / INNER, (rows + 2 * ROWS - 1) / (2 * ROWS));
    auto* const x = (typename Elem<TYPE>::Bits*)X;
    auto kernel = (uintptr_t)X % 16 != 0 || ldx * sizeof(*x) % 16 != 0 ? k_lm_dequantize<TYPE, GROUP, PLAIN>
                                                                        : (through ? k_lm_dequantize<TYPE, GROUP, THROUGH> : k_lm_dequantize<TYPE, GROUP, PAST>);
    if constexpr (TYPE == F16)
        if (peaks) {
            k_scale_peaks<<<dim3(PEAKS), dim3(256), 0, st>>>(w, row0, rows, peaks);
            kernel = k_lm_dequantize<TYPE, GROUP, RAISED>;
        }
    kernel<<<grid, dim3(256), 0, st>>>(w, row0, rows, cols, x, ldx, peaks, peaks ? peaks + PEAKS : nullptr);
}
template <int TYPE> void dequantize(const Weights& w, int64_t row0, int64_t rows, int64_t cols, void* X, int64_t ldx, bool through, float* peaks, hipStream_t st)
{
    if (w.shape.group == 32) dequantize<TYPE, 32>(w, row0, rows, cols, X, ldx, through, peaks, st);
    if (w.shape.group == 64) dequantize<TYPE, 64>(w, row0, rows, cols, X, ldx, through, peaks, st);
    if (w.shape.group == 128) dequantize<TYPE, 128>(w, row0, rows, cols, X, ldx, through, peaks, st);
}

}  // namespace

namespace lmk {

hipError_t launch_quantize(int type, const void* W, int64_t ldw, const Shape& s, int stype, void* packed, hipStream_t st)
{
    if (type == F32) quantize<F32>(W, ldw, s, stype, packed, st);
    if (type == BF16) quantize<BF16>(W, ldw, s, stype, packed, st);
    if (type == F16) quantize<F16>(W, ldw, s, stype, packed, st);
    return hipGetLastError();
}

hipError_t launch_dequantize(int type, const Weights& w, int64_t row0, int64_t rows, int64_t cols, void* X, int64_t ldx, bool through, float* peaks, hipStream_t st)
{
    if (type == F32) dequantize<F32>(w, row0, rows, cols, X, ldx, through, peaks, st);
    if (type == BF16) dequantize<BF16>(w, row0, rows, cols, X, ldx, through, peaks, st);
    if (type == F16) dequantize<F16>(w, row0, rows, cols, X, ldx, through, peaks, st);
    return hipGetLastError();
}

hipError_t launch_pack(const Shape& s, const uint8_t* codes, int64_t ldc, const void* scales, int64_t lds, const uint8_t* zeros, int64_t ldz, void* packed,
                       hipStream_t st)
{
    k_lm_pack<<<grid_of(s), dim3(256), 0, st>>>(s, codes, ldc, (const uint16_t*)scales, lds, zeros, ldz, (uint8_t*)packed);
    return hipGetLastError();
}

hipError_t launch_unpack(const Shape& s, const void* packed, uint8_t* codes, int64_t ldc, void* scales, int64_t lds, uint8_t* zeros, int64_t ldz,
                         hipStream_t st)
{
    k_lm_unpack<<<grid_of(s), dim3(256), 0, st>>>(s, (const uint8_t*)packed, codes, ldc, (uint16_t*)scales, lds, zeros, ldz);
    return hipGetLastError();
}

hipError_t launch_shared(const Linear& l, const Weights& w, const SharedPlan& plan, float* parts, hipStream_t st)
{
    const int64_t rows = (l.m + plan.rows - 1) / plan.rows * plan.rows, columns = (w.shape.p + plan.columns - 1) / plan.columns * plan.columns;
    const Shared a{l, w, plan.splits, parts, columns, rows * columns};
    if (l.xtype == BF16) shared<BF16>(a, plan, st);
    if (l.xtype == F16) shared<F16>(a, plan, st);
    if (plan.splits > 1) {
        const int64_t blocks = (l.m * ((w.shape.p + 3) / 4) + 255) / 256;
        const dim3 grid((unsigned)(blocks < 8192 ? blocks : 8192));
        if (l.dtype == F32) k_lm_meet<F32><<<grid, dim3(256), 0, st>>>(a);
        if (l.dtype == BF16) k_lm_meet<BF16><<<grid, dim3(256), 0, st>>>(a);
        if (l.dtype == F16) k_lm_meet<F16><<<grid, dim3(256), 0, st>>>(a);
    }
    return hipGetLastError();
}

hipError_t launch_direct(const Linear& l, const Weights& w, hipStream_t st)
{
    if (l.xtype == BF16) direct<BF16>(l, w, st);
    if (l.xtype == F16) direct<F16>(l, w, st);
    return hipGetLastError();
}

}  // namespace lmk
