// C ABI of the operators around a model's output layer (declared in include/ozimmu_lm.h): argument checks, workspace carving and launches.
// No allocation, no host synchronisation, no state between calls.
#include "../../include/ozimmu.h"
#include "../../include/ozimmu_lm.h"
#include "ozimmu_lm.h"

namespace lmk {

constexpr int64_t COMPUTE_UNITS = 256;

// (32-bit offsets inside a panel, 30 bits where rows lie along the inner dimension: pieces behind a row's end are sent behind those)
bool tile_fits(const Tile& t)
{
    auto along = [](int64_t ld) { return ld * 2 < (1 << 22); };
    auto across = [&](int64_t ld) { return t.n * ld * 2 < ((int64_t)1 << 32) - (1 << 20); };
    const bool a = t.kind == WEIGHTS ? across(t.lda) : along(t.lda);
    const bool b = t.kind == WEIGHTS || t.kind == STATES ? across(t.ldb) : along(t.ldb);
    return a && b && t.n > 0 && (t.m + 127) / 128 * ((t.p + 255) / 256) * t.splits < ((int64_t)1 << 28);
}

// Microseconds of an output of that many tiles over KT stages each, roughly: rounds of one tile for every compute unit, of two with 128 x 128.
// Fitted to (loss alone, without its small launches; tokens x inner x words: 256 x 256, 128 x 256, 128 x 128)  133 x 1024 x 5003: 30, 18, 12;
// 777 x 1024 x 10007: 33, 38, 28;  2048 x 4096 x 4096: 85, 57, 59;  512 x 4096 x 4096: 78, 49, 36;  1024 x 1024 x 32768: 65, 75, 66;
// 4096 x 1024 x 32768: 255, 282, 275;  1 x 4096 x 32768: 77, 49, 42;  2048 x 4096 x 131072: 1570, 1820, -.
static double estimate_us(int shape, int64_t tiles, double KT)
{
    const double rounds = (double)((tiles + COMPUTE_UNITS - 1) / COMPUTE_UNITS);
    if (shape == TILE_256) return rounds * (13 + KT * (1.12 + 0.2 * (double)tiles / (rounds * COMPUTE_UNITS)));
    if (shape == TILE_128_256) return rounds * (5 + KT * 0.81);
    const int64_t pairs = tiles / (2 * COMPUTE_UNITS), rest = tiles % (2 * COMPUTE_UNITS);
    return (double)pairs * (3.5 + KT * 0.86) + (rest == 0 ? 0 : rest > COMPUTE_UNITS ? 3.5 + KT * 0.86 : 4 + KT * 0.5);
}

static int64_t tiles_of(int shape, int64_t m, int64_t p)
{
    const int64_t rows = shape == TILE_256 ? 256 : 128, columns = shape == TILE_128 ? 128 : 256;
    return (m + rows - 1) / rows * ((p + columns - 1) / columns);
}

int tile_shape(int64_t m, int64_t n, int64_t p, int splits)
{
    int best = TILE_256;
    for (int s : {TILE_128_256, TILE_128})
        if (estimate_us(s, tiles_of(s, m, p) * splits, (double)((n + 63) / 64) / splits) <
            estimate_us(best, tiles_of(best, m, p) * splits, (double)((n + 63) / 64) / splits))
            best = s;
    return best;
}

// The number of splits of n, four stages each at the least, that takes the least time; the sums of each are written and read again in FP32
int tile_splits(int64_t m, int64_t n, int64_t p)
{
    const int64_t KT = (n + 63) / 64;
    int best = 1;
    double least = 0;
    for (int64_t s = 1; s <= 256 && (s == 1 || s * 4 <= KT); s += s < 4 ? 1 : s / 4) {
        const int shape = tile_shape(m, n, p, (int)s);
        const double us = estimate_us(shape, tiles_of(shape, m, p) * s, (double)KT / (double)s) + (double)(s * m * p) * 8 / 4e6;
        if (s == 1 || us < least) {
            least = us;
            best = (int)s;
        }
    }
    return best;
}

hipError_t launch_tile(const Tile& t, hipStream_t st) { return t.type == BF16 ? launch_tile_1(t, st) : launch_tile_2(t, st); }

}  // namespace lmk

namespace {

using lmk::Tile;
using lml::Shape;

constexpr int64_t MAX_ROWS = ((int64_t)1 << 22) - 256, MAX_INNER = (int64_t)1 << 20, MAX_LD = ((int64_t)1 << 40) - 1;
constexpr int64_t MAX_SPAN = ((int64_t)1 << 60) - 1;   // rows x leading dimension: byte offsets stay within 64 bits
constexpr int64_t MAX_STATES = ((int64_t)1 << 31) - (1 << 20);

inline int64_t round_to(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
inline bool rows_ok(int64_t r) { return r >= 0 && r <= MAX_ROWS; }
inline bool sizes_ok(int64_t p, int64_t n) { return rows_ok(p) && n >= 0 && n <= MAX_INNER; }
inline bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }
inline bool type_ok(int type) { return type == OZIMMU_LM_F32 || type == OZIMMU_LM_BF16 || type == OZIMMU_LM_F16; }
inline bool type16_ok(int type) { return type == OZIMMU_LM_BF16 || type == OZIMMU_LM_F16; }
inline bool aligned(const void* p) { return ((uintptr_t)p & 255u) == 0; }

// a matrix in memory: given, aligned for its type, its rows apart
int matrix_status(int type, const void* p, int64_t rows, int64_t n, int64_t ld)
{
    if (!type_ok(type)) return OZIMMU_ERR_TYPE;
    if (ld < n || ld > MAX_LD || (rows > 0 && ld > MAX_SPAN / rows)) return OZIMMU_ERR_DIM;
    if (rows == 0 || n == 0) return OZIMMU_OK;
    if (!p) return OZIMMU_ERR_NULL;
    return ((uintptr_t)p & (type == OZIMMU_LM_F32 ? 3u : 1u)) == 0 ? OZIMMU_OK : OZIMMU_ERR_TYPE;
}
// numbers of `size` bytes, `stride` apart
int vector_status(const void* p, int64_t rows, int64_t stride, unsigned size)
{
    if (stride < 0 || stride > MAX_LD) return OZIMMU_ERR_DIM;
    if (rows == 0) return OZIMMU_OK;
    if (!p) return OZIMMU_ERR_NULL;
    return (uintptr_t)p % size == 0 ? OZIMMU_OK : OZIMMU_ERR_TYPE;
}
int packed_status(const void* p, int64_t rows, int64_t n, int group, int scale_type)
{
    if (!group_ok(group)) return OZIMMU_ERR_DIM;
    if (!type16_ok(scale_type)) return OZIMMU_ERR_TYPE;
    if (rows == 0 || n == 0) return OZIMMU_OK;
    if (!p) return OZIMMU_ERR_NULL;
    return aligned(p) ? OZIMMU_OK : OZIMMU_ERR_WORKSPACE;
}
int workspace_status(const void* p, size_t bytes, size_t need)
{
    if (need == 0) return OZIMMU_OK;
    if (!p) return OZIMMU_ERR_NULL;
    return bytes >= need && aligned(p) ? OZIMMU_OK : OZIMMU_ERR_WORKSPACE;
}
#define CHECK(x)                                  \
    do {                                          \
        const int status_ = (x);                  \
        if (status_ != OZIMMU_OK) return status_; \
    } while (0)

inline int launched(hipError_t e) { return e == hipSuccess ? OZIMMU_OK : OZIMMU_ERR_HIP; }

// Pieces of a workspace, one behind the other (without a workspace: their sizes)
struct Room {
    uint8_t* base;
    size_t used = 0;
    template <class T> T* take(int64_t count)
    {
        T* const at = base ? (T*)(base + used) : nullptr;
        used += (size_t)round_to(count * (int64_t)sizeof(T), 256);
        return at;
    }
};

// whether the tiles can take rows along the inner dimension as they are
bool as_it_is(const void* p, int64_t n, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && n % 8 == 0 && ld * 2 < (1 << 22); }

// ---- the linear layer from the stored form ----

struct LinearPlan {
    int64_t width, rows;   // of a piece of weights read back
    uint16_t *W, *X;
    size_t bytes;
    LinearPlan(int64_t m, int64_t n, int64_t p, void* workspace)
    {
        Room room{(uint8_t*)workspace};
        width = round_to(n, 64);
        // pieces of at most 128 MB, which stay in the memory-side cache until they are multiplied
        const int64_t most = ((int64_t)1 << 27) / (width * 2) / 256 * 256;
        rows = most < 256 ? 256 : most;
        if (rows > round_to(p, 256)) rows = round_to(p, 256);
        W = room.take<uint16_t>(rows * width);
        X = room.take<uint16_t>(m * width);
        bytes = room.used;
    }
};

// Two workgroups for every compute unit where the sizes give as many, by splits of four blocks of the inner dimension at the least (4096 x 4096, rows:
// splits and us  32: 4 12.3, 8 11.4, 16 13.8;  128: 2 19.4, 4 18.2;  512, of 64 rows a workgroup: 1 41, 2 34.3, 3 34.4;  1024: 1 53.5, 2 60).  32 rows a
// workgroup up to 128 (64 rows 13.6 and 15.7 us, 256 25.1 and 25.2, 512 35.6 and 34.3); 256 columns from 1024 workgroups on (2048 rows 90 and 102 us,
// 1024 rows 54 and 68).
lmk::SharedPlan shared_plan(int64_t m, int64_t n, int64_t p)
{
    const int rows = m <= 128 ? 32 : 64;
    const int64_t row_blocks = (m + rows - 1) / rows, most = (n + 511) / 512;
    const int columns = row_blocks * ((p + 127) / 128) >= 4 * lmk::COMPUTE_UNITS ? 256 : 128;
    const int64_t splits = 2 * lmk::COMPUTE_UNITS / (row_blocks * ((p + columns - 1) / columns));
    return {rows, columns, (int)(splits < 2 ? 1 : splits < most ? splits : most)};
}
size_t shared_bytes(int64_t m, int64_t n, int64_t p)
{
    const lmk::SharedPlan plan = shared_plan(m, n, p);
    return plan.splits < 2 ? 0 : (size_t)round_to(plan.splits * round_to(m, plan.rows) * round_to(p, plan.columns) * 4, 256);
}

// Up to 16 rows from the codes in one launch, in any case (callers need not ask for a workspace then), and more of them where there is little to do (128
// rows through 512 x 512: 5.6 us, with X in LDS 6.9; 37 rows through 2051 x 1283: 9.4, 11.1; 32 rows through 4096 x 4096: 10.6 and 12.1; 256 rows: 38 and 24).
// Beyond, weights are read back from one number of rows on, so that what is rounded does not change back and forth with them: behind 512, or where the outputs
// come to more than 128 tiles of 128 x 128, whichever is later.  (us, n x p, rows: X in LDS, weights read back)  4096 x 4096, 512: 36, 48;  640: 53, 48;  1024: 55,
// 48;  1200: 69, 62;  2048: 88, 68;  2100: 144, 87;  4096 x 16384, 384: 75, 80;  640: 146, 117;  8192 x 8192, 512: 99, 96;  640: 127, 119;  4096 x 1024, 1024: 26, 40;
// 2048: 38, 41;  2100: 54, 41;  2048 x 2048, 960: 24, 29;  1100: 31, 29;  2048 x 256, 6000: 24, 28;  8192: 26, 24.  It is the slower one right behind 512 rows where the
// inner dimension is short: 1024 x 4096, 1100: 25, 30;  512 x 8192, 640: 18, 21 (1100: 40, 32).
constexpr int64_t DIRECT_ROWS = 16, CODES_ROWS = 512, CODES_OUTPUTS = (int64_t)1 << 21;
int choose(int64_t m, int64_t n, int64_t p)
{
    if (m <= DIRECT_ROWS || (m <= 128 && (double)m * (double)p * (double)n < 1 << 27)) return OZIMMU_LM_WAY_DIRECT;
    return m <= CODES_ROWS || m * p <= CODES_OUTPUTS ? OZIMMU_LM_WAY_SHARED : OZIMMU_LM_WAY_TILE;
}

int linear_tile(int64_t m, int64_t n, int64_t p, float alpha, int xtype, const void* X, int64_t ldx, const lmk::Weights& w, float beta, int dtype, void* D,
                int64_t ldd, void* workspace, hipStream_t st)
{
    const LinearPlan plan(m, n, p, workspace);
    Tile t{lmk::LINEAR, xtype};
    t.m = m;
    t.n = n;
    t.A = X;
    t.lda = ldx;
    if (!as_it_is(X, n, ldx)) {
        t.n = plan.width;
        CHECK(launched(lmk::launch_lay_out(xtype, {m, n, X, ldx, plan.X, plan.width}, {}, st)));
        t.A = plan.X;
        t.lda = plan.width;
    }
    int64_t rows = plan.rows;
    float* peaks = nullptr;
    if (xtype == lmk::F16 && w.stype == lmk::BF16) {
        // room for the scales' peaks: where X would be laid out, or the last 16 rows of W's (2 KB at the least), which pieces leave free then
        constexpr int64_t ROOM = 16 * 64 * 2;
        static_assert((lmk::SCALE_PEAKS + 1) * sizeof(float) <= ROOM, "they fit");
        if (t.A == X && m * plan.width * 2 >= ROOM) {
            peaks = (float*)plan.X;
        } else {
            rows -= 16;
            peaks = (float*)(plan.W + rows * plan.width);
        }
        t.alpha_at = peaks + lmk::SCALE_PEAKS;
    }
    t.B = plan.W;
    t.ldb = plan.width;
    t.ldd = ldd;
    t.dtype = dtype;
    t.alpha = alpha;
    t.beta = beta;
    const int64_t size = dtype == OZIMMU_LM_F32 ? 4 : 2;
    for (int64_t at = 0; at < p; at += rows) {
        t.p = t.b_rows = p - at < rows ? p - at : rows;
        CHECK(launched(lmk::launch_dequantize(xtype, w, at, t.p, plan.width, plan.W, plan.width, true, peaks, st)));
        t.D = (uint8_t*)D + at * size;
        t.shape = lmk::tile_shape(t.m, t.n, t.p, t.splits);
        CHECK(launched(lmk::launch_tile(t, st)));
    }
    return OZIMMU_OK;
}

// ---- cross entropy ----

bool loss_sizes_ok(int64_t m, int64_t n, int64_t p)
{
    return rows_ok(m) && p >= 1 && p <= MAX_ROWS && n >= 1 && n <= MAX_INNER && round_to(m, 256) * round_to(n, 256) < MAX_STATES;
}

// W in pieces of rows that are laid out anew where the tiles cannot take it as it is: at most 256 MB (there are enough tiles in those)
int64_t laid_out_rows(int64_t width, int64_t p)
{
    int64_t rows = ((int64_t)1 << 28) / (width * 2) / 256 * 256;
    if (rows < 256) rows = 256;
    return rows < round_to(p, 256) ? rows : round_to(p, 256);
}

// How a loss is taken: straight from memory (rows of the plan > 0) for few tokens, more of them where W would have to be laid out for the tiles, and where
// there is little to do.  (us, straight and by tiles: 1 x 4096 x 32768 56 and 71, rows at odd elements 73 and 181;  32 rows 74 and 73;  40 rows 82 and 75;
// 64 rows at odd elements 123 and 194;  96 rows 201 and 196;  133 x 1001 x 5003 19 and 27, at odd elements 21 and 27;  64 x 1001 x 10007 at odd elements 23 and
// 29;  128 rows 38 and 30;  16 x 512 x 2048 7.0 and 13.8.)
lmk::FewPlan few_plan(int64_t m, int64_t n, int64_t p, bool aligned)
{
    if (m > (aligned ? 32 : 64) && (double)m * (double)n * (double)p >= 1e9) return {0, 0};
    const int rows = m <= 16 ? 16 : m <= 32 ? 32 : 64;
    return {rows, m > 4 && (m + rows - 1) / rows * ((p + 63) / 64) >= 128 ? 64 : 16};
}

struct LossPlan {
    lmk::FewPlan few;
    int64_t width, tokens, words;   // of a row laid out; tokens at a time; rows of W laid out at a time
    float* at_target;
    float2* parts;
    uint16_t *X, *W;
    size_t bytes;
    LossPlan(int64_t m, int64_t n, int64_t p, lmk::FewPlan few_, void* workspace) : few(few_)
    {
        Room room{(uint8_t*)workspace};
        width = round_to(n, 64);
        const int64_t blocks = few.rows ? (p + few.columns - 1) / few.columns : (p + 63) / 64;
        // tokens at a time, whole workgroups of them: parts of at most 256 MB (by tiles for 2^22 words, the most there are, 512 tokens)
        const int64_t unit = few.rows ? few.rows : 256;
        tokens = ((int64_t)1 << 25) / blocks / unit * unit;
        if (tokens < unit) tokens = unit;
        if (tokens > round_to(m, unit)) tokens = round_to(m, unit);
        words = laid_out_rows(width, p);
        at_target = room.take<float>(tokens);
        parts = room.take<float2>(blocks * tokens);
        X = room.take<uint16_t>(few.rows ? 0 : tokens * width);
        W = room.take<uint16_t>(few.rows ? 0 : words * width);
        bytes = room.used;
    }
};

struct GradientPlan {
    int64_t padded, width, states_ld, words;   // rows and columns of whole tiles; words at a time
    int splits;
    int *known, *far, *far_count;
    float *lse2, *largest, *peaks, *states;
    uint16_t *slopes, *X, *scaled, *W;
    size_t bytes;
    // lay_out: X and W are laid out anew
    GradientPlan(int64_t m, int64_t n, int64_t p, bool lay_out, void* workspace)
    {
        Room room{(uint8_t*)workspace};
        padded = round_to(m, 256);
        width = round_to(n, 64);
        states_ld = round_to(n, 256);
        // slopes of at most 128 MB, which stay in the memory-side cache for the two products that read them (of 256 words at the least: from 262144 tokens on
        // they take more), and pieces of W of at most 1 GB where it is, 256 MB where it is laid out
        words = ((int64_t)1 << 26) / padded / 256 * 256;
        const int64_t most = lay_out ? laid_out_rows(width, p) : ((int64_t)1 << 29) / width / 256 * 256;
        if (words > most) words = most;
        if (words < 256) words = 256;
        if (words > round_to(p, 256)) words = round_to(p, 256);
        splits = lmk::tile_splits(m, words, n);
        known = room.take<int>(padded);
        lse2 = room.take<float>(padded);
        largest = room.take<float>(1);
        peaks = room.take<float>(m);
        far = room.take<int>(m);
        far_count = room.take<int>(1);
        slopes = room.take<uint16_t>(padded * words);
        states = room.take<float>(splits * padded * states_ld);
        scaled = room.take<uint16_t>(m * width);
        X = room.take<uint16_t>(lay_out ? m * width : 0);
        W = room.take<uint16_t>(lay_out ? words * width : 0);
        bytes = room.used;
    }
};

}  // namespace

extern "C" {

size_t ozimmu_lm_bytes(int64_t p, int64_t n, int group, int zeros)
{
    return sizes_ok(p, n) && group_ok(group) ? (size_t)Shape{p, n, group, zeros != 0}.bytes() : 0;
}

int ozimmu_lm_quantize(int type, int64_t p, int64_t n, const void* W, int64_t ldw, int group, int zeros, int scale_type, void* packed, void* stream)
{
    if (!sizes_ok(p, n)) return OZIMMU_ERR_DIM;
    CHECK(matrix_status(type, W, p, n, ldw));
    CHECK(packed_status(packed, p, n, group, scale_type));
    if (p == 0 || n == 0) return OZIMMU_OK;
    return launched(lmk::launch_quantize(type, W, ldw, Shape{p, n, group, zeros != 0}, scale_type, packed, (hipStream_t)stream));
}

int ozimmu_lm_dequantize(int type, int64_t p, int64_t n, int group, int zeros, int scale_type, const void* packed, void* W, int64_t ldw, void* stream)
{
    if (!sizes_ok(p, n)) return OZIMMU_ERR_DIM;
    CHECK(matrix_status(type, W, p, n, ldw));
    CHECK(packed_status(packed, p, n, group, scale_type));
    if (p == 0 || n == 0) return OZIMMU_OK;
    const lmk::Weights w{Shape{p, n, group, zeros != 0}, scale_type, (const uint8_t*)packed};
    return launched(lmk::launch_dequantize(type, w, 0, p, n, W, ldw, false, nullptr, (hipStream_t)stream));
}

static int plain_status(int64_t p, int64_t n, int group, const void* codes, int64_t ldc, const void* scales, int64_t lds, const void* zeros, int64_t ldz,
                        const void* packed)
{
    if (!sizes_ok(p, n) || !group_ok(group)) return OZIMMU_ERR_DIM;
    const int64_t groups = (n + group - 1) / group;
    if (ldc < (n + 1) / 2 || ldc > MAX_LD || lds < groups || lds > MAX_LD || (zeros && (ldz < groups || ldz > MAX_LD))) return OZIMMU_ERR_DIM;
    if (p > 0 && n > 0 && (!codes || !scales)) return OZIMMU_ERR_NULL;
    if ((uintptr_t)scales & 1u) return OZIMMU_ERR_TYPE;
    return packed_status(packed, p, n, group, OZIMMU_LM_F16);
}

int ozimmu_lm_pack(int64_t p, int64_t n, int group, const uint8_t* codes, int64_t ldc, const void* scales, int64_t lds, const uint8_t* zeros, int64_t ldz,
                   void* packed, void* stream)
{
    CHECK(plain_status(p, n, group, codes, ldc, scales, lds, zeros, ldz, packed));
    if (p == 0 || n == 0) return OZIMMU_OK;
    return launched(lmk::launch_pack(Shape{p, n, group, zeros != nullptr}, codes, ldc, scales, lds, zeros, ldz, packed, (hipStream_t)stream));
}

int ozimmu_lm_unpack(int64_t p, int64_t n, int group, const void* packed, uint8_t* codes, int64_t ldc, void* scales, int64_t lds, uint8_t* zeros,
                     int64_t ldz, void* stream)
{
    CHECK(plain_status(p, n, group, codes, ldc, scales, lds, zeros, ldz, packed));
    if (p == 0 || n == 0) return OZIMMU_OK;
    return launched(lmk::launch_unpack(Shape{p, n, group, zeros != nullptr}, packed, codes, ldc, scales, lds, zeros, ldz, (hipStream_t)stream));
}

int ozimmu_lm_linear_choose(int64_t m, int64_t n, int64_t p) { return choose(m, n, p); }

size_t ozimmu_lm_linear_way_workspace_bytes(int way, int64_t m, int64_t n, int64_t p)
{
    if (!sizes_ok(p, n) || !rows_ok(m)) return 0;
    if (way == OZIMMU_LM_WAY_AUTO) way = choose(m, n, p);
    if (m == 0 || n == 0 || p == 0) return 0;
    if (way == OZIMMU_LM_WAY_SHARED) return shared_bytes(m, n, p);
    return way == OZIMMU_LM_WAY_TILE ? LinearPlan(m, n, p, nullptr).bytes : 0;
}
size_t ozimmu_lm_linear_workspace_bytes(int64_t m, int64_t n, int64_t p) { return ozimmu_lm_linear_way_workspace_bytes(OZIMMU_LM_WAY_AUTO, m, n, p); }

int ozimmu_lm_linear(int64_t m, int64_t n, int64_t p, float alpha, int xtype, const void* X, int64_t ldx, int group, int zeros, int scale_type,
                     const void* W, float beta, int dtype, void* D, int64_t ldd, void* workspace, size_t workspace_bytes, void* stream)
{
    return ozimmu_lm_linear_way(OZIMMU_LM_WAY_AUTO, m, n, p, alpha, xtype, X, ldx, group, zeros, scale_type, W, beta, dtype, D, ldd, workspace,
                                workspace_bytes, stream);
}

int ozimmu_lm_linear_way(int way, int64_t m, int64_t n, int64_t p, float alpha, int xtype, const void* X, int64_t ldx, int group, int zeros, int scale_type,
                         const void* W, float beta, int dtype, void* D, int64_t ldd, void* workspace, size_t workspace_bytes, void* stream)
{
    // (an empty inner dimension: the sum would be zero, but there is nothing stored to read it from)
    if (!sizes_ok(p, n) || !rows_ok(m) || n == 0) return OZIMMU_ERR_DIM;
    if (!type16_ok(xtype)) return OZIMMU_ERR_TYPE;
    CHECK(matrix_status(xtype, X, m, n, ldx));
    CHECK(matrix_status(dtype, D, m, p, ldd));
    if (way == OZIMMU_LM_WAY_AUTO) way = choose(m, n, p);
    if (way != OZIMMU_LM_WAY_DIRECT && way != OZIMMU_LM_WAY_TILE && way != OZIMMU_LM_WAY_SHARED) return OZIMMU_ERR_WAY;
    CHECK(packed_status(W, p, n, group, scale_type));
    if (m == 0 || p == 0) return OZIMMU_OK;
    CHECK(workspace_status(workspace, workspace_bytes, ozimmu_lm_linear_way_workspace_bytes(way, m, n, p)));
    const lmk::Weights w{Shape{p, n, group, zeros != 0}, scale_type, (const uint8_t*)W};
    const hipStream_t st = (hipStream_t)stream;
    if (way == OZIMMU_LM_WAY_TILE) return linear_tile(m, n, p, alpha, xtype, X, ldx, w, beta, dtype, D, ldd, workspace, st);
    const lmk::Linear l{m, X, ldx, xtype, D, ldd, dtype, alpha, beta};
    if (way == OZIMMU_LM_WAY_SHARED) return launched(lmk::launch_shared(l, w, shared_plan(m, n, p), (float*)workspace, st));
    return launched(lmk::launch_direct(l, w, st));
}

size_t ozimmu_lm_cross_entropy_workspace_bytes(int64_t m, int64_t n, int64_t p)
{
    if (!loss_sizes_ok(m, n, p) || m == 0) return 0;
    // (for rows that begin anywhere too)
    const size_t a = LossPlan(m, n, p, few_plan(m, n, p, true), nullptr).bytes, b = LossPlan(m, n, p, few_plan(m, n, p, false), nullptr).bytes;
    return a > b ? a : b;
}

int ozimmu_lm_cross_entropy(int type, int64_t m, int64_t n, int64_t p, const void* X, int64_t ldx, const void* W, int64_t ldw, const int64_t* y,
                            int64_t y_stride, int64_t ignore, float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!loss_sizes_ok(m, n, p)) return OZIMMU_ERR_DIM;
    if (!type16_ok(type)) return OZIMMU_ERR_TYPE;
    CHECK(matrix_status(type, X, m, n, ldx));
    CHECK(matrix_status(type, W, p, n, ldw));
    CHECK(vector_status(y, m, y_stride, 8));
    CHECK(vector_status(loss, m, 1, 4));
    CHECK(vector_status(lse, m, 1, 4));
    CHECK(workspace_status(workspace, workspace_bytes, ozimmu_lm_cross_entropy_workspace_bytes(m, n, p)));
    if (m == 0) return OZIMMU_OK;
    const LossPlan plan(m, n, p, few_plan(m, n, p, as_it_is(X, n, ldx) && as_it_is(W, n, ldw)), workspace);
    const hipStream_t st = (hipStream_t)stream;
    // (one that is laid out has zeros up to `width`; where that is beyond n the other may not be read so far, so both are)
    const bool x_as_it_is = as_it_is(X, n, ldx) && (n == plan.width || as_it_is(W, n, ldw));
    const bool w_as_it_is = as_it_is(W, n, ldw) && (n == plan.width || as_it_is(X, n, ldx));
    for (int64_t t0 = 0; t0 < m; t0 += plan.tokens) {
        const int64_t rows = m - t0 < plan.tokens ? m - t0 : plan.tokens, step = w_as_it_is ? p : plan.words;
        const lmk::Targets targets{y + t0 * y_stride, y_stride, ignore, p};
        if (plan.few.rows) {
            const int64_t blocks = (p + plan.few.columns - 1) / plan.few.columns;
            const lmk::FewLoss few{rows, n, p, (const uint16_t*)X + t0 * ldx, ldx, W, ldw, targets, plan.at_target, plan.parts, blocks};
            CHECK(launched(lmk::launch_few_loss(type, few, plan.few, st)));
            CHECK(launched(lmk::launch_join_rows(rows, blocks, plan.parts, blocks, targets, plan.at_target, loss + t0, lse + t0, st)));
            continue;
        }
        const lmk::LayOut x{rows, n, (const uint16_t*)X + t0 * ldx, ldx, plan.X, plan.width};
        Tile t{lmk::LOSS, type};
        t.m = rows;
        t.n = x_as_it_is && w_as_it_is ? n : plan.width;
        t.A = x_as_it_is ? x.X : plan.X;
        t.lda = x_as_it_is ? ldx : plan.width;
        t.targets = targets;
        t.at_target = plan.at_target;
        t.parts_ld = plan.tokens;
        t.shape = lmk::tile_shape(rows, t.n, step < p ? step : p, 1);
        const int64_t part = lmk::part_columns(t.shape);
        for (int64_t v0 = 0; v0 < p; v0 += step) {
            t.p = t.b_rows = p - v0 < step ? p - v0 : step;
            const lmk::LayOut w{t.p, n, (const uint16_t*)W + v0 * ldw, ldw, plan.W, plan.width}, none{};
            const bool lay_x = !x_as_it_is && v0 == 0;
            if (lay_x || !w_as_it_is) CHECK(launched(lmk::launch_lay_out(type, lay_x ? x : none, w_as_it_is ? none : w, st)));
            t.B = w_as_it_is ? w.X : plan.W;
            t.ldb = w_as_it_is ? ldw : plan.width;
            t.column0 = (int)v0;
            t.parts = plan.parts + v0 / part * plan.tokens;
            if (!lmk::tile_fits(t)) return OZIMMU_ERR_DIM;
            CHECK(launched(lmk::launch_tile(t, st)));
        }
        CHECK(launched(lmk::launch_join(rows, (p + part - 1) / part, plan.parts, plan.tokens, targets, plan.at_target, loss + t0, lse + t0, st)));
    }
    return OZIMMU_OK;
}

size_t ozimmu_lm_cross_entropy_backward_workspace_bytes(int64_t m, int64_t n, int64_t p)
{
    if (!loss_sizes_ok(m, n, p) || m == 0) return 0;
    // (for rows that begin anywhere too)
    const size_t a = GradientPlan(m, n, p, false, nullptr).bytes, b = GradientPlan(m, n, p, true, nullptr).bytes;
    return a > b ? a : b;
}

int ozimmu_lm_cross_entropy_backward(int type, int64_t m, int64_t n, int64_t p, const float* g, int64_t g_stride, const void* X, int64_t ldx, const void* W,
                                     int64_t ldw, const int64_t* y, int64_t y_stride, int64_t ignore, const float* lse, int dx_type, void* dX,
                                     int64_t lddx, float beta, int dw_type, void* dW, int64_t lddw, void* workspace, size_t workspace_bytes,
                                     void* stream)
{
    if (!loss_sizes_ok(m, n, p)) return OZIMMU_ERR_DIM;
    if (!type16_ok(type)) return OZIMMU_ERR_TYPE;
    CHECK(matrix_status(type, X, m, n, ldx));
    CHECK(matrix_status(type, W, p, n, ldw));
    if (dX) CHECK(matrix_status(dx_type, dX, m, n, lddx));
    if (dW) CHECK(matrix_status(dw_type, dW, p, n, lddw));
    CHECK(vector_status(y, m, y_stride, 8));
    CHECK(vector_status(g, m, g_stride, 4));
    CHECK(vector_status(lse, m, 1, 4));
    const hipStream_t st = (hipStream_t)stream;
    CHECK(workspace_status(workspace, workspace_bytes, ozimmu_lm_cross_entropy_backward_workspace_bytes(m, n, p)));
    if (!dX && !dW) return OZIMMU_OK;
    if (m == 0) {
        if (dW && beta != 1.0f) return launched(lmk::launch_scale(dw_type, p, n, beta, dW, lddw, st));
        return OZIMMU_OK;
    }
    // (W is read along its rows and across them, a piece of `words` rows at a time)
    const bool lay_out = !as_it_is(X, n, ldx) || !as_it_is(W, n, ldw) ||
                         GradientPlan(m, n, p, false, nullptr).words * ldw * 2 >= ((int64_t)1 << 32) - (1 << 20);
    const GradientPlan plan(m, n, p, lay_out, workspace);
    const float unscale = type == OZIMMU_LM_F16 ? 1.0f / lmk::SLOPE_SCALE_F16 : 1.0f;
    int splits = 0;
    for (int64_t v0 = 0; v0 < p; v0 += plan.words) {
        const int64_t words = p - v0 < plan.words ? p - v0 : plan.words, whole = round_to(words, 256);
        const lmk::LayOut w{words, n, (const uint16_t*)W + v0 * ldw, ldw, lay_out ? plan.W : nullptr, plan.width};
        const void* const W_at = lay_out ? (const void*)plan.W : w.X;
        const int64_t ldw_at = lay_out ? plan.width : ldw;
        if (v0 == 0) {
            const lmk::LayOut x{m, n, X, ldx, lay_out ? plan.X : nullptr, plan.width};
            if (dW && type == lmk::F16) CHECK(launched(lmk::launch_row_peaks(m, n, X, ldx, plan.peaks, st)));
            CHECK(launched(lmk::launch_prepare(type, {m, plan.padded, {y, y_stride, ignore, p}, g, g_stride, lse, plan.known, plan.lse2, plan.largest, plan.peaks,
                                                      plan.far, plan.far_count, x, dW ? plan.scaled : nullptr, w}, st)));
        } else if (lay_out) {
            CHECK(launched(lmk::launch_lay_out(type, w, {}, st)));
        }
        Tile t{lmk::SLOPE, type};
        t.m = m;
        t.n = lay_out ? plan.width : n;
        t.p = t.b_rows = words;
        t.A = lay_out ? (const void*)plan.X : X;
        t.lda = lay_out ? plan.width : ldx;
        t.B = W_at;
        t.ldb = ldw_at;
        t.D = plan.slopes;
        t.ldd = whole;
        t.known = plan.known;
        t.column0 = (int)v0;
        t.lse2 = plan.lse2;
        if (!lmk::tile_fits(t)) return OZIMMU_ERR_DIM;
        t.shape = lmk::tile_shape(t.m, t.n, t.p, t.splits);
        CHECK(launched(lmk::launch_tile(t, st)));
        if (dX) {
            Tile s{lmk::STATES, type};
            s.m = m;
            s.n = round_to(words, 64);  // (columns of slopes behind the words: zeros, as far as tiles reach, which is here at the least)
            s.p = round_to(n, 8);
            s.b_rows = words;
            s.A = plan.slopes;
            s.lda = whole;
            s.B = W_at;
            s.ldb = ldw_at;
            s.D = plan.states;
            s.ldd = plan.states_ld;
            s.split_stride = plan.padded * plan.states_ld;
            s.beta = v0 > 0 ? 1.0f : 0.0f;
            s.splits = plan.splits < (int)(s.n / 64) ? plan.splits : (int)(s.n / 64);
            if (v0 == 0) splits = s.splits;
            if (!lmk::tile_fits(s)) return OZIMMU_ERR_DIM;
            s.shape = lmk::tile_shape(s.m, s.n, s.p, s.splits);
            CHECK(launched(lmk::launch_tile(s, st)));
        }
        if (dW) {
            Tile s{lmk::WEIGHTS, type};
            s.m = words;
            s.n = s.b_rows = m;
            s.p = n;
            s.A = plan.slopes;
            s.lda = whole;
            s.B = plan.scaled;
            s.ldb = plan.width;
            s.D = (uint8_t*)dW + v0 * lddw * (dw_type == OZIMMU_LM_F32 ? 4 : 2);
            s.ldd = lddw;
            s.dtype = dw_type;
            s.alpha = unscale;
            s.alpha_at = plan.largest;
            s.beta = beta;
            if (!lmk::tile_fits(s)) return OZIMMU_ERR_DIM;
            s.shape = lmk::tile_shape(s.m, s.n, s.p, s.splits);
            CHECK(launched(lmk::launch_tile(s, st)));
            if (type == lmk::F16)
                CHECK(launched(lmk::launch_far(dw_type, words, n, plan.slopes, whole, X, ldx, g, g_stride, plan.far, plan.far_count, s.D, lddw, st)));
        }
    }
    if (dX)
        CHECK(launched(lmk::launch_states(dx_type, m, n, plan.states, plan.states_ld, splits, plan.padded * plan.states_ld, g, g_stride, plan.known, unscale, dX,
                                          lddx, st)));
    return OZIMMU_OK;
}

}  // extern "C"
