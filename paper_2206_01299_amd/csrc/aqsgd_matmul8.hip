// Products of 8-bit codes: which kernel a call takes.
#include "aqsgd_matmul8.h"

namespace aqsgd {

AQSGD_PRODUCT_DT(extern, AQSGD_F32)
AQSGD_PRODUCT_DT(extern, AQSGD_F16)
AQSGD_PRODUCT_DT(extern, AQSGD_BF16)

namespace {

template <template <int> class F, typename... Args>
hipError_t by_dtype(int dtype, Args&&... args) {
    switch (dtype) {
    case AQSGD_F32:  return F<AQSGD_F32>::go(args...);
    case AQSGD_F16:  return F<AQSGD_F16>::go(args...);
    default:         return F<AQSGD_BF16>::go(args...);
    }
}
template <int DT> struct Tiles256 {
    static hipError_t go(ProductKind k, const TilePlan& t, const ProductArgs& p, hipStream_t s) { return launch_tiles256_dt<DT>(k, t, p, s); }
};
template <int DT> struct Tiles128 {
    static hipError_t go(int cols, ProductKind k, const ProductArgs& p, hipStream_t s) { return launch_tiles128_dt<DT>(cols, k, p, s); }
};
template <int DT> struct Split {
    static hipError_t go(SplitTile t, ProductKind k, const ProductArgs& p, const Slices& l, hipStream_t s) { return launch_split_dt<DT>(t, k, p, l, s); }
};

uint32_t tiles(int64_t n, int64_t side) { return static_cast<uint32_t>((n + side - 1) / side); }

// What a call takes on an idle MI355X, in microseconds, for each kernel: a tile alone, and what every 256 tiles add, a
// part of it only with every full round of the CUs; both straight lines in k (thousands).  Fitted to 550 products with
// m, n up to 16384 and k from 16 to 16384, drawn evenly over their logarithms, and 98 whose sides are powers of two or
// the widths of models, each timed with every kernel in a captured graph: the mean distance is 7 to 10 %, and the
// kernel that the lines pick is 1 % slower on average than the best one (30 % at worst).  Sides measured (us):
// 512 x 512 x 4096 10.7 with 32 x 32, 17.9 with 16 x 16, 18.5 with 64 x 64; 1024 x 4096 x 1024 9.2 with 128 x 64, 10.7 with
// 128 x 128, 16.7 with 256 x 256, 27.0 with 64 x 64; 7373 x 7896 x 383 54.0 with 128 x 128, 77.9 with 128 x 64, whose rows
// of results are half as long, so it is left out from 1024 tiles on; one that the lines miss: 777 x 1001 x 1333 9.5 with
// 128 x 64, which they take, 8.3 with 64 x 64.
struct Line { int rows, cols; float alone, alone_k, more, more_k, rounds; };
constexpr Line kSplitLines[] = {            // by SplitTile
    {64, 64, 4.16f, 2.47f, 2.68f, 3.32f, 0.66f}, {64, 32, 3.56f, 1.61f, 1.62f, 2.54f, 0.61f}, {32, 32, 3.29f, 1.09f, 0.60f, 1.55f, 0.58f},
    {16, 16, 3.38f, 0.49f, 0.56f, 0.73f, 0.59f}, {16, 32, 3.33f, 0.86f, 0.54f, 1.13f, 0.56f}};
constexpr Line kTile128Line = {128, 128, 5.54f, 4.29f, 2.38f, 3.82f, 0.68f}, kTile128x64Line = {128, 64, 3.84f, 3.16f, 0.96f, 1.30f, 0.25f};

float cost(const Line& l, const ProductShape& p, int slices = 1) {
    const float k = 0.001f * static_cast<float>(p.k) / static_cast<float>(slices);
    const int64_t all = static_cast<int64_t>(tiles(p.m, l.rows)) * tiles(p.n, l.cols) * slices;
    const float many = l.rounds * static_cast<float>((all - 1) >> 8) + (1.0f - l.rounds) * static_cast<float>(all) * (1.0f / 256);
    return l.alone + l.alone_k * k + many * (l.more + l.more_k * k);
}

// Slices of k, where tiles are few and k is long: a second launch, and the sums once out and once in again, at a
// microsecond a megabyte (16 x 256 x 16384 8.3 us, in one piece 16.3; 204 x 340 x 10592 15.4 and 21.5; with more sums it
// soon costs more than it gives: 512 x 512 x 8192 24.2 and 17.8).
float join_cost(const ProductShape& p, int slices) {
    return 3.0f + static_cast<float>(slices) * static_cast<float>(p.m) * static_cast<float>(p.n) * 8e-6f;
}

// Where one tile spans all columns, every row of a comes from memory, and a tile of 128 rows has less of it on its way
// than its steps need: 14696 x 56 x 10448 52.8 us with 64 x 64, 71.9 with 128 x 64; 8794 x 64 x 8106 27.5 and 43.5.
float streams(const ProductShape& p, int cols) {
    return p.n <= cols && static_cast<int64_t>(p.m) * p.k > (int64_t{32} << 20) ? 1.6f : 1.0f;
}

// Tiles of 256 rows, one workgroup to a CU.  A tile of w columns takes 8 us and (0.45 + 0.0043 w) us for every 128
// of k, with all CUs at work.  Where whole tiles leave CUs idle in the last round, the last
// columns go as narrower ones, launched behind the others.  Measured with operands from memory: a message of 4096 x 1600
// times 6400, float16, 400 tiles of 256 columns 56.7 us, 256 of them and 240 of 160 columns 53.1, 192 of 192 columns 53.5;
// 4096 x 12800 x 1600 gated float16, 800 tiles 113.2, 768 of them and 128 of 64 columns 102.2, 64 of 128 columns 106.0;
// 6144 x 1536 x 8192 float32 added to, 144 tiles 111.5, 240 of 160 columns 98.0, 192 of 192 columns 103.0.  One that the lines
// miss: tiles of 96 and 160 columns have no whole number of rows to a wave's store and end row by row, which the line
// does not know; with the last product's sums in the caches already, 160 columns take 79.0 us, 192 columns 75.5.
constexpr uint32_t kCus = 256;
float tile256_time(int blocks, float steps) { return 8.0f + steps * (0.45f + 0.0043f * 32.0f * static_cast<float>(blocks)); }

// The longest of the CUs' times: `wide` tiles, then `narrow` ones to whichever CU is free first.
float makespan(uint32_t wide, uint32_t narrow, float t_wide, float t_narrow) {
    const uint32_t full = wide / kCus, ahead = wide % kCus;
    float t[2] = {static_cast<float>(full) * t_wide, static_cast<float>(full + 1) * t_wide};
    uint32_t cus[2] = {kCus - ahead, ahead};
    float end = ahead ? t[1] : t[0];
    while (narrow > 0) {
        const int g = cus[1] > 0 && t[1] < t[0] ? 1 : 0;
        const uint32_t taken = narrow < cus[g] ? narrow : cus[g];
        narrow -= taken;
        t[g] += t_narrow;
        if (t[g] > end) end = t[g];
    }
    return end;
}

TilePlan plan256(ProductKind kind, const ProductShape& p, float& best) {
    const float steps = static_cast<float>(tiles(p.k, 128)), t_wide = tile256_time(8, steps);
    TilePlan plan{tiles(p.m, 256), tiles(p.n, 256), 0, 0};
    best = 2.0f + makespan(plan.tiles_m * plan.wide_n, 0, t_wide, t_wide);
    const uint32_t rounds = plan.tiles_m * plan.wide_n / kCus;
    for (int blocks = 2; blocks < 8; ++blocks) {
        if (kind == kGated && blocks % 2) continue;               // the gate's columns come in pairs of sixteen
        const float t_narrow = tile256_time(blocks, steps);
        for (uint32_t r = rounds > 1 ? rounds - 1 : 0; r <= rounds; ++r) {        // rounds of whole tiles
            uint32_t wide_n = r * kCus / plan.tiles_m;
            if (wide_n >= tiles(p.n, 256)) wide_n = tiles(p.n, 256) - 1;
            const uint32_t narrow_n = tiles(p.n - static_cast<int64_t>(wide_n) * 256, 32 * blocks);
            const float t = 2.0f + makespan(plan.tiles_m * wide_n, plan.tiles_m * narrow_n, t_wide, t_narrow);
            if (t < 0.99f * best) {
                best = t;
                plan.wide_n = wide_n; plan.narrow_n = narrow_n; plan.narrow = blocks;
            }
        }
    }
    return plan;
}

constexpr int64_t kMostSplitTiles = (int64_t{1} << 23) - 1;       // of 512 lanes: a grid takes fewer than 2^32

// How a product goes: in slices of k or whole by tiles of the waves' registers, by tiles of 128 rows, or of 256.
struct Choice {
    int split = -1, slices = 1, cols = 128;
    bool large = false;
    TilePlan plan = {};
};

Choice choose(ProductKind kind, const ProductShape& p) {
    Choice c;
    float best = cost(kTile128Line, p) * streams(p, 128);
    if (static_cast<int64_t>(tiles(p.m, 128)) * tiles(p.n, 64) <= 1024) {
        const float now = cost(kTile128x64Line, p) * streams(p, 64);
        if (now < best) { best = now; c.cols = 64; }
    }
    const bool may_slice = (kind == kPlain || kind == kMessage) && p.k >= 4096 && static_cast<int64_t>(p.m) * p.n <= 1 << 20;
    for (int t = kSplit64; t <= kSplit16x32; ++t) {
        if (kind == kGated && t == kSplit16) continue;            // the gate's columns come in pairs of sixteen
        if (static_cast<int64_t>(tiles(p.m, kSplitLines[t].rows)) * tiles(p.n, kSplitLines[t].cols) > kMostSplitTiles) continue;
        float now = cost(kSplitLines[t], p);
        if (now < best) { best = now; c.split = t; c.slices = 1; }
        for (int slices = 2; may_slice && slices <= 16 && p.k >= 2048 * slices; slices *= 2) {
            now = cost(kSplitLines[t], p, slices) + join_cost(p, slices);
            if (now < 0.9f * best) { best = now; c.split = t; c.slices = slices; }
        }
    }
    if (c.split >= 0) return c;
    float large;
    c.plan = plan256(kind, p, large);
    c.large = large < best;
    return c;
}

bool whole_sectors(ProductKind kind, const ProductArgs& p) {
    const int64_t width = static_cast<int64_t>(kind == kGated ? p.n / 2 : p.n) * (p.dtype == AQSGD_F32 ? 4 : 2);
    return width % 32 == 0 && ((reinterpret_cast<uintptr_t>(p.out) | reinterpret_cast<uintptr_t>(p.pre)) & 31) == 0;
}

// The slices' sums in the workspace: rows of whole tiles.
Slices slices_of(const Choice& c, const ProductShape& p) {
    Slices s = {nullptr, 1, 0, 0};
    if (c.split < 0 || c.slices == 1) return s;
    const int32_t pieces = static_cast<int32_t>(tiles(p.k, 128));
    s.pieces = (pieces + c.slices - 1) / c.slices;
    s.count = (pieces + s.pieces - 1) / s.pieces;
    const int cols = kSplitLines[c.split].cols;
    s.pitch = static_cast<int32_t>(tiles(p.n, cols)) * cols;
    return s;
}

}  // namespace

int64_t product_workspace_bytes(ProductKind kind, const ProductShape& p) {
    if (p.m == 0 || p.n == 0 || p.k < 4096) return 0;
    const Slices s = slices_of(choose(kind, p), p);
    return s.count > 1 ? static_cast<int64_t>(s.count) * (p.m + 1) * s.pitch * 4 : 0;
}

hipError_t launch_product(ProductKind kind, const ProductArgs& q, void* workspace, hipStream_t stream) {
    ProductArgs p = q;
    p.stream = whole_sectors(kind, q);
    const ProductShape shape{p.m, p.n, p.k};
    const Choice c = choose(kind, shape);
    if (c.split >= 0) {
        Slices s = slices_of(c, shape);
        s.sums = static_cast<int32_t*>(workspace);
        return by_dtype<Split>(p.dtype, static_cast<SplitTile>(c.split), kind, p, s, stream);
    }
    if (c.large) return by_dtype<Tiles256>(p.dtype, kind, c.plan, p, stream);
    return by_dtype<Tiles128>(p.dtype, c.cols, kind, p, stream);
}

}  // namespace aqsgd
