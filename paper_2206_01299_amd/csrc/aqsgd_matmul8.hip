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
    static hipError_t go(SplitTile t, ProductKind k, const ProductArgs& p, hipStream_t s) { return launch_split_dt<DT>(t, k, p, s); }
};

uint32_t tiles(int64_t n, int64_t side) { return static_cast<uint32_t>((n + side - 1) / side); }

// What a call takes on an idle MI355X, in microseconds, for each kernel: a tile alone, and what every 256 tiles beyond
// the first few add, both straight lines in k (thousands).  Fitted to 160 products with m, n up to 16384 and k from 16
// to 16384, drawn evenly over their logarithms, each timed with every kernel in a captured graph: the mean distance is
// 7 to 10 %, and the kernel that the lines pick is 2 % slower on average than the best one.  Sides measured (us):
// 1 x 6400 x 1600 4.9 with 16 x 16, 6.6 with 64 x 64, 12.7 with 128 x 128; 512 x 512 x 4096 10.4 with 32 x 32, 17.9
// with 16 x 16 and with 64 x 64; 777 x 1001 x 1333 8.2 with 64 x 64, 9.8 with 32 x 32, 13.8 with 128 x 128; 4349 x 449 x
// 688 7.8 with 128 x 64, 10.2 with 128 x 128, 14.1 with 32 x 32; 1024 x 4096 x 1024 11.6 with 128 x 128, 18.5 with 256 x
// 256, 27 with 64 x 64; 7373 x 7896 x 383 55.8 with 128 x 128, 77.9 with 128 x 64, whose rows of results are half as
// long, so it is left out from 1024 tiles on.
struct Line { int rows, cols; float alone, alone_k, more, more_k, first; };
constexpr Line kSplitLines[] = {            // by SplitTile
    {64, 64, 4.06f, 2.16f, 2.56f, 3.44f, 0.32f}, {64, 32, 3.65f, 1.54f, 1.69f, 2.55f, 0.48f}, {32, 32, 3.41f, 1.13f, 0.77f, 1.48f, 0.62f},
    {16, 16, 3.46f, 0.61f, 0.72f, 0.59f, 0.57f}, {16, 32, 3.47f, 0.87f, 0.77f, 0.92f, 0.71f}};
constexpr Line kTile128Line = {128, 128, 4.81f, 4.44f, 2.74f, 3.67f, 0.16f}, kTile128x64Line = {128, 64, 4.08f, 2.61f, 0.92f, 2.43f, 0.0f};

float cost(const Line& l, const ProductArgs& p) {
    const float k = 0.001f * static_cast<float>(p.k);
    const float many = static_cast<float>(tiles(p.m, l.rows)) * static_cast<float>(tiles(p.n, l.cols)) * (1.0f / 256) - l.first;
    return l.alone + l.alone_k * k + (many > 0.0f ? many * (l.more + l.more_k * k) : 0.0f);
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

