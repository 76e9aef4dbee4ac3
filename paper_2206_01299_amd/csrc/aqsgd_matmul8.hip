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
    static hipError_t go(ProductKind k, const TilePlan& t, const ProductArgs& p, hipStream_t s) { return launch_tiles128_dt<DT>(k, t, p, s); }
};
template <int DT> struct Split {
    static hipError_t go(SplitTile t, ProductKind k, const ProductArgs& p, hipStream_t s) { return launch_split_dt<DT>(t, k, p, s); }
};

uint32_t tiles(int64_t n, int64_t side) { return static_cast<uint32_t>((n + side - 1) / side); }

// What a call takes on an idle MI355X, in microseconds, for each kernel: a tile alone, and what every 256 tiles add,
// both straight lines in k (thousands).  Fitted to 110 products with m, n up to 16384 and k from 16 to 16384, drawn
// evenly over their logarithms, each timed with every kernel in a captured graph: the mean distance is 8 to 11 %,
// and the kernel that the lines pick is 1.4 % slower on average than the best one.  Sides measured (us): 1 x 6400 x
// 1600 4.9 with 16 x 16, 6.6 with 64 x 64, 12.7 with 128 x 128; 512 x 512 x 4096 10.4 with 32 x 32, 17.9 with 16 x 16
// and with 64 x 64; 777 x 1001 x 1333 8.2 with 64 x 64, 9.8 with 32 x 32, 13.8 with 128 x 128; 1024 x 4096 x 1024 11.6
// with 128 x 128, 18.5 with 256 x 256, 27 with 64 x 64.
struct Line { int rows, cols; float alone, alone_k, more, more_k; };
constexpr Line kTile128Line = {128, 128, 5.2f, 4.36f, 2.4f, 3.68f};
constexpr Line kSplitLines[] = {            // by SplitTile
    {64, 64, 3.9f, 1.84f, 2.7f, 2.93f}, {64, 32, 3.4f, 1.43f, 1.8f, 2.16f}, {32, 32, 3.2f, 0.95f, 0.66f, 1.31f},
    {16, 16, 3.3f, 0.51f, 0.66f, 0.53f}, {16, 32, 3.3f, 0.73f, 0.64f, 0.90f}};

float cost(const Line& l, const ProductArgs& p) {
    const float k = 0.001f * static_cast<float>(p.k);
    const float many = static_cast<float>(tiles(p.m, l.rows)) * static_cast<float>(tiles(p.n, l.cols)) * (1.0f / 256);
    return l.alone + l.alone_k * k + many * (l.more + l.more_k * k);
}

// Tiles of 256 rows, one workgroup to a CU.  A tile of w columns takes 8 us and (0.45 + 0.0043 w) us for every 128
// of k, with all CUs at work (power bounds them then).  Where whole tiles leave CUs idle in the last round, the last
// columns go as narrower ones, launched behind the others: 4096 x 6400 x 1600, 400 tiles of 256 columns 54.2 us,
// 256 of them and 240 of 160 columns 52.5, 192 of 192 columns 50.8; 4096 x 12800 x 1600 gated, 800 tiles 114.9 us,
// 768 of them and 128 of 64 columns 102.7; 6144 x 1536 x 8192 added to, 144 tiles 110.7 us, 240 of 160 columns 98.0.
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

TilePlan plan256(ProductKind kind, const ProductArgs& p, float& best) {
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

}  // namespace

hipError_t launch_product(ProductKind kind, const ProductArgs& p, hipStream_t stream) {
    int split = -1;
    float best = cost(kTile128Line, p);
    for (int t = kSplit64; t <= kSplit16x32; ++t) {
        if (kind == kGated && t == kSplit16) continue;            // the gate's columns come in pairs of sixteen
        const float c = cost(kSplitLines[t], p);
        if (c < best) { best = c; split = t; }
    }
    if (split >= 0) return by_dtype<Split>(p.dtype, static_cast<SplitTile>(split), kind, p, stream);
    float large;
    const TilePlan plan = plan256(kind, p, large);
    if (large < best) return by_dtype<Tiles256>(p.dtype, kind, plan, p, stream);
    return by_dtype<Tiles128>(p.dtype, kind, TilePlan{tiles(p.m, 128), tiles(p.n, 128), 0, 0}, p, stream);
}

}  // namespace aqsgd
