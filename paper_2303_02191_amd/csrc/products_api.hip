// C entries of the 8-bit products and the gated feed-forward block: checks of the arguments (before any HIP call) and the choice of
// kernels.
#include <algorithm>
#include <cmath>

#include "product_tile.h"

namespace rtoss {

namespace {

bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) != 0; }
bool known(rtoss_dtype dt) { return dt == RTOSS_F32 || dt == RTOSS_F16 || dt == RTOSS_BF16; }
bool known(rtoss_act act) { return act == RTOSS_ACT_NONE || act == RTOSS_ACT_RELU || act == RTOSS_ACT_SILU; }

constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int kMaxWidth = 1 << 24;      // channels
constexpr int kMaxSumI8 = (1 << 17) - 1;  // 128 * 128 * R < 2^31
constexpr int64_t kMaxPitch = 0x7fffffff;

// A matrix of rows in memory: where its bytes are.
struct Span {
    int64_t from, rows, width, pitch;  // in bytes, one row of a matrix without gaps
};
Span span(const void* p, int64_t rows, int64_t width, int64_t ld, int eb)
{
    const Span s{(int64_t)(uintptr_t)p, p ? rows : 0, width * eb, ld * eb};
    return s.rows > 1 && ld == width ? Span{s.from, 1, s.rows * s.width, s.rows * s.width} : s;
}
// Whether rows i of a and j of b share a byte: -b.width < b.from - a.from + j b.pitch - i a.pitch < a.width.  (Of slices with different pitches: not looked for.)
bool overlap(const Span& a, const Span& b)
{
    if (!a.rows || !b.rows || (a.rows > 1 && b.rows > 1 && a.pitch != b.pitch)) return false;
    const auto below = [](int64_t n, int64_t by) { return n / by - (n % by < 0); };  // rounded down
    const int64_t pitch = a.rows > 1 ? a.pitch : b.pitch, apart = b.from - a.from;
    return std::max(below(-b.width - apart, pitch) + 1, 1 - a.rows) <= std::min(below(a.width - apart - 1, pitch), b.rows - 1);  // j - i
}

rtoss_status check_rows(int64_t M, const char* what)
{
    if (M < 0) return fail(RTOSS_EINVAL, "%s=%lld is negative", what, (long long)M);
    if (M > kMaxRows) return fail(RTOSS_ESHAPE, "%s=%lld: at most 2^31 - 1 rows", what, (long long)M);
    return RTOSS_OK;
}
rtoss_status check_width(int64_t n, const char* what)
{
    if (n < 1 || n > kMaxWidth) return fail(RTOSS_ESHAPE, "%s=%lld outside 1..2^24", what, (long long)n);
    return RTOSS_OK;
}
// ld: 0 means `width`
rtoss_status check_pitch(int64_t* ld, int64_t width, const char* what)
{
    if (*ld < 0) return fail(RTOSS_EINVAL, "%s=%lld is negative", what, (long long)*ld);
    if (*ld == 0) *ld = width;
    if (*ld < width || *ld > kMaxPitch) return fail(RTOSS_ESHAPE, "%s=%lld outside %lld..2^31 - 1", what, (long long)*ld, (long long)width);
    return RTOSS_OK;
}
rtoss_status check_pointer(const void* p, int align, const char* what)
{
    if (!p) return fail(RTOSS_EINVAL, "%s is NULL", what);
    if (misaligned(p, align)) return fail(RTOSS_EINVAL, "%s is not aligned to its element size", what);
    return RTOSS_OK;
}

#define RTOSS_TRY(call) \
    if (rtoss_status st_ = (call)) return st_

rtoss_status gated_desc(const rtoss_gated_desc* desc, rtoss_gated_desc* d)
{
    if (!desc) return fail(RTOSS_EINVAL, "descriptor is NULL");
    *d = *desc;
    if (!known(d->dt)) return fail(RTOSS_EDTYPE, "bad dtype %d", (int)d->dt);
    if (!known(d->act)) return fail(RTOSS_EINVAL, "unknown activation %d", (int)d->act);
    RTOSS_TRY(check_rows(d->M, "M"));
    RTOSS_TRY(check_width(d->K, "K"));
    RTOSS_TRY(check_width(d->F, "F"));
    RTOSS_TRY(check_pitch(&d->x_ld, d->K, "x_ld"));
    RTOSS_TRY(check_pitch(&d->w_ld, d->K, "w_ld"));
    RTOSS_TRY(check_pitch(&d->h_ld, d->F, "h_ld"));
    return RTOSS_OK;
}

// The kernel for a product: the one whose estimate is shortest.  All are bound by what a CU can copy in the small, by the matrix instructions
// in the large, and by whole rounds of workgroups.  Constants in us, for 256 CUs, fitted to 456 products of the forward pass in all tiles (measured again on
// 111 of such with the kernels as they are, the choice is 2.0 % longer than the best in the mean, 31 % at most); rows of whole 16-byte pieces, of words, of
// bytes:
//   slices of a x b: the launch 3.1, then for each round a little more the larger the tile, and the rows of both operands at 72, 41, 37 KB/us and CU
//     (fp32 also 0.77e6 products), or where the sum is short a workgroup's beginning and end.  8-bit 4096 x 4096, rows 1, 64, 128, 256: 5.2, 6.7,
//     7.6, 9.9 with the tile that this takes; 8.4, 9.4, 9.4, 9.9 with 64 x 64 for all.
//   slices of 64 x 64, one for every wave (fp32): 4.5, then for each round 4, 6 and 2.85, 3.6 a stage.  Gated fp32 16 -> 2801, rows 300, 1453, 6000:
//     8, 12, 44, a workgroup for each 11, 39, 146; 333 -> 2801 41, 48, 212 and 23, 84, 334; 2048 -> 2801 159, 186, 849 and 53, 210, 828.
//   tiles: for each round 6, 6, 7 and 0.85, 1.2, 1.8 a stage of 128 bytes; 0.77 and 0.65 of that with 128 rows, 8.9 and 1.26 with 256 channels.
//     Gated bf16 4096 -> 10944, rows 128, 256, 512, 1024, 2048: 49, 83, 118, 224, 420 with 128 x 128; 58, 62, 117, 184, 351 with 256 x 128; 80, 83,
//     88, 176, 287 with 256 x 256; slices of 64 x 64 63, 105, 183, 335, 635.
struct Choice {
    int kernel;   // slices by tile, those of a tile for every wave, tiles
    double time;  // us
};
Choice choose(ProductForm form, bool bits8, rtoss_dtype out, const Product& p, int cus)
{
    const int eb = bits8 ? 1 : elem_bytes(out);
    const bool gated = form == kGated, across = form == kBackRows || form == kBackWeights;
    const double row = (double)p.R * eb * (form == kBackRows ? 2 : 1);
    const auto up = [](int64_t n, int by) { return (double)((n + by - 1) / by); };
    const auto tiles = [&](int rows, int channels) { return up(p.M, rows) * up(p.N, channels) * (form == kBackWeights ? 2 : 1); };
    const Rows rows = product_rows(form, p, eb);
    Choice best{kSliceTiles - 1, 1e300};
    for (int t = across ? kSliceTiles - 1 : 0; t < kSliceTiles; ++t) {
        constexpr double kRound[kSliceTiles] = {0.17, 0.24, 0.57, 0.66, 1.57}, kShort[kSliceTiles] = {0.41, 0.58, 1.02, 1.03, 1.4};
        constexpr double kRate[] = {72e3, 41e3, 37e3}, kAligned[] = {1, 1.77, 2};
        const int a = kSlices[t].rows, n = gated ? kSlices[t].gated : kSlices[t].channels, b = gated ? 2 * n : n;
        if (tiles(a, n) > kMaxSliceTiles) continue;
        const double count = tiles(a, n) / cus;
        const int together = 160 / (a + b);  // workgroups whose LDS a CU holds
        const double rounds = together >= 2 ? std::max(1.0, count) : std::ceil(count);
        const double sum = kRound[t] + (a + b) * row / kRate[rows] + (eb == 4 ? a * b * row / eb / 0.77e6 : 0);
        const double time = 3.1 + rounds * std::max(sum, kShort[t] * kAligned[rows] * (gated ? 1.85 : 1) * (eb == 4 ? 1.24 : 1));
        if (time < best.time) best = Choice{t, time};
    }
    if (eb == 4 && gated) {
        const double rounds = std::ceil(tiles(64, 32) / (8 * cus)), stages = std::ceil(row / 128);
        const double time = 4.5 + rounds * (rows == kWhole ? 4 + stages * 2.85 : 6 + stages * 3.6);
        if (time < best.time) best = Choice{kSliceTiles, time};
    }
    if (product_tiles_ok(bits8, out, p)) {
        constexpr double kStageTime[] = {0.85, 1.2, 1.8}, kRoundTime[] = {6, 6, 7};
        const double stages = std::ceil(row / 128);
        for (int t = 0; t < (rows == kWhole ? 3 : 2); ++t) {
            const double rounds = std::ceil(tiles(kTiles[t].rows, kTiles[t].channels / (gated ? 2 : 1)) / cus);
            const double one = t == 2 ? 8.9 + stages * 1.26 : kRoundTime[rows] * (t ? 1 : 0.77) + stages * kStageTime[rows] * (t ? 1 : 0.65);
            const double time = rounds * one;
            if (time < best.time) best = Choice{kSliceTiles + 1 + t, time};
        }
    }
    return best;
}

rtoss_status launch_chosen(int kernel, ProductForm form, bool bits8, rtoss_dtype out, const Product& p, hipStream_t s)
{
    if (kernel <= kSliceTiles) return launch_product_slices(form, bits8, out, kernel, p, s);
    return launch_product_tiles(form, bits8, out, kernel - kSliceTiles - 1, p, s);
}

// Rows m .. m+rows-1 of the result, and channels n .. n+channels-1.
void* on(const void* base, int64_t bytes) { return base ? (void*)((char*)base + bytes) : nullptr; }
Product rows_of(ProductForm form, int eb, int out_eb, const Product& p, int64_t m, int64_t rows)
{
    Product part = p;
    const int64_t a_step = form == kBackWeights ? eb : p.lda * eb;  // (there the rows of the result are columns of its operand)
    part.M = (int)rows;
    part.a0 = on(p.a0, m * a_step);
    part.a1 = on(p.a1, m * a_step);
    part.sa = (const float*)on(p.sa, m * 4);
    part.residual = on(p.residual, m * p.ldr * out_eb);
    part.y = on(p.y, m * p.ldy * out_eb);
    part.y0 = on(p.y0, m * p.ldk * out_eb);
    part.y1 = on(p.y1, m * (form == kBackWeights ? p.ldy : p.ldk) * out_eb);
    return part;
}
Product channels_of(ProductForm form, int eb, int out_eb, const Product& p, int64_t n, int64_t channels)
{
    Product part = p;
    const int64_t b_step = form == kBackRows || form == kBackWeights ? eb : p.ldb * eb;
    part.N = (int)channels;
    part.b0 = on(p.b0, n * b_step);
    part.b1 = on(p.b1, n * b_step);
    part.s0 = (const float*)on(p.s0, n * 4);
    part.s1 = (const float*)on(p.s1, n * 4);
    part.bias = (const float*)on(p.bias, n * 4);
    part.residual = on(p.residual, n * out_eb);
    part.y = on(p.y, n * out_eb);
    part.y0 = on(p.y0, n * out_eb);
    part.y1 = on(p.y1, n * out_eb);
    return part;
}

// A product in one launch, or in two: as many rows or channels as fill whole rounds of tiles, and the rest with what suits it, where that is
// shorter.  Gated bf16 1000 x 4096 -> 10944: 344 tiles of 256 x 256, two rounds, 176 us; 256 of them, and the last 2752 channels in 172 of
// 256 x 128, 161.
struct ProductPlan {
    double time;
    int64_t rows, channels;  // of the first launch
};
ProductPlan plan_product(ProductForm form, bool bits8, rtoss_dtype out, const Product& p, int cus)
{
    const int eb = bits8 ? 1 : elem_bytes(out), out_eb = elem_bytes(out);
    const Choice whole = choose(form, bits8, out, p, cus);
    ProductPlan best{whole.time, p.M, p.N};
    if (whole.kernel <= kSliceTiles) return best;
    const auto& tile = kTiles[whole.kernel - kSliceTiles - 1];
    const int width = form == kGated ? tile.channels / 2 : tile.channels, both = form == kBackWeights ? 2 : 1;
    const int64_t high = ((int64_t)p.M + tile.rows - 1) / tile.rows, wide = ((int64_t)p.N + width - 1) / width, tiles = high * wide * both;
    const int64_t full = (tiles - 1) / cus * cus;  // tiles of whole rounds, without the last
    const auto try_split = [&](const Product& first, const Product& rest, int64_t rows, int64_t channels) {
        const double time = choose(form, bits8, out, first, cus).time + choose(form, bits8, out, rest, cus).time + 1.5;
        if (time < best.time * 0.97) best = ProductPlan{time, rows, channels};
    };
    const int64_t rows = full / (wide * both) * tile.rows, channels = full / (high * both) * width;
    if (rows > 0 && rows < p.M) try_split(rows_of(form, eb, out_eb, p, 0, rows), rows_of(form, eb, out_eb, p, rows, p.M - rows), rows, p.N);
    if (channels > 0 && channels < p.N)
        try_split(channels_of(form, eb, out_eb, p, 0, channels), channels_of(form, eb, out_eb, p, channels, p.N - channels), p.M, channels);
    return best;
}

// A launch has at most kMaxSliceTiles of the largest slices: more rows than that take several.
rtoss_status launch_product(ProductForm form, bool bits8, rtoss_dtype out, const Product& p, hipStream_t s)
{
    DeviceInfo dev;
    RTOSS_TRY(current_device(&dev));
    const int eb = bits8 ? 1 : elem_bytes(out), out_eb = elem_bytes(out);
    const auto launch = [&](const Product& part) { return launch_chosen(choose(form, bits8, out, part, dev.cus).kernel, form, bits8, out, part, s); };
    const int64_t across = ((int64_t)p.N + 31) / 32 * 2;
    const int64_t most = std::max<int64_t>(kMaxSliceTiles / across, 1) * 64;  // rows
    for (int64_t m = 0; m < p.M; m += most) {
        const Product part = rows_of(form, eb, out_eb, p, m, std::min<int64_t>(most, p.M - m));
        const ProductPlan plan = plan_product(form, bits8, out, part, dev.cus);
        if (plan.rows < part.M) {
            RTOSS_TRY(launch(rows_of(form, eb, out_eb, part, 0, plan.rows)));
            RTOSS_TRY(launch(rows_of(form, eb, out_eb, part, plan.rows, part.M - plan.rows)));
        } else if (plan.channels < part.N) {
            RTOSS_TRY(launch(channels_of(form, eb, out_eb, part, 0, plan.channels)));
            RTOSS_TRY(launch(channels_of(form, eb, out_eb, part, plan.channels, part.N - plan.channels)));
        } else {
            RTOSS_TRY(launch(part));
        }
    }
    return RTOSS_OK;
}

// Both gradients in one launch of slices, that of the rows in tiles of `high` ? 64 : 16 rows.  A sum that would take longer than all the copies is
// shared by several workgroups, which leave their parts in the workspace.  By the shape and type alone, so that the workspace's size is
// known without a device: 256 CUs, rows of whole pieces.
//   bytes   of both operands' rows, for all tiles        steps   of four stages, of the rows' sums and the weights'
struct Merged {
    double bytes, row_steps, weight_steps;
    int64_t row_tiles, weight_tiles;
    int row_parts, weight_parts;
    bool rows_each, weights_each;
    size_t counters() const { return ((row_parts > 1 ? row_tiles : 0) + (weight_parts > 1 ? weight_tiles : 0)) * 4; }
    size_t row_bytes(bool high) const { return row_parts > 1 ? (size_t)row_tiles * row_parts * (high ? 64 : 16) * 64 * 4 : 0; }
    size_t weight_bytes() const { return weight_parts > 1 ? (size_t)weight_tiles * weight_parts * 64 * 64 * 4 : 0; }
    size_t scratch(bool high) const { return align_up(counters(), 256) + row_bytes(high) + weight_bytes(); }
};
// us for four stages of tiles of 16 and 64 rows, bytes/us and CU, us for a tile and CU (half of it where every wave has one); rows of whole 16-byte pieces, of words, of bytes
struct MergedSpeed {
    double low, high, rate, low_tile, high_tile;
};
const MergedSpeed& merged_speed(rtoss_dtype dt, Rows rows)
{
    static const MergedSpeed speeds[2][3] = {{{0.4, 0.55, 95e3, 1.1, 1.6}, {0.9, 1.15, 73e3, 1.0, 2.4}, {1.1, 2.0, 52e3, 2.1, 2.85}},  // 16 bits
                                             {{0.6, 1.6, 56e3, 1.0, 1.85}, {1.08, 2.6, 56e3, 0.6, 3.0}, {}}};                         // fp32
    return speeds[dt == RTOSS_F32][rows];
}
Merged merged(rtoss_dtype dt, int64_t M, int K, int F, bool high)
{
    const int eb = elem_bytes(dt);
    const auto up = [](int64_t n, int64_t by) { return (n + by - 1) / by; };
    Merged g;
    g.row_tiles = up(M, high ? 64 : 16) * up(K, 64);
    g.weight_tiles = 2 * up(F, 64) * up(K, 64);
    g.bytes = (double)g.row_tiles * ((high ? 64 : 16) + 64) * 2 * F * eb + (double)g.weight_tiles * 128 * M * eb;
    g.row_steps = (double)up(2 * up((int64_t)F * eb, 128), 4);
    g.weight_steps = (double)up(M * eb, 512);
    // (joining takes 2.5 us, about as long as a part of 3 us is worth; four stages 0.6 and 0.75, fp32 0.78 and 1.5; 89 and 45 KB/us)
    const double copies = std::max(g.bytes / ((eb == 4 ? 45e3 : 89e3) * 256), 5.0), high_step = eb == 4 ? 1.5 : 0.75;
    const auto parts = [&](double steps, double step, int64_t tiles) {
        const double time = steps * step;
        return time < copies + 2.5 || tiles == 0 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>((int64_t)std::ceil(time / copies), 1024 / tiles));
    };
    g.row_parts = parts(g.row_steps, high ? high_step : eb == 4 ? 0.78 : 0.6, g.row_tiles);
    g.weight_parts = parts(g.weight_steps, high_step, g.weight_tiles);
    // Of many tiles with short sums every wave takes one, and nothing is joined: bf16 16 rows 1024 -> 2752 17 -> 14 us, 2 rows 990 -> 7682 62 -> 31; at
    // 1024 rows (16 stages) 54 either way, of 88 tiles with 512 rows 11 -> 14.
    g.rows_each = high && g.row_steps <= 2 && g.row_tiles >= 1024;
    g.weights_each = g.weight_steps <= 2 && g.weight_tiles >= 1024;
    return g;
}

// How the gradients are computed, of one (the other's y is NULL) by the same kernels as of both: in one launch of slices where that is shorter
// than two.  One launch: 4.3 us, then the copies and every tile's beginning and end, or the longest sum, or memory; constants fitted to 87 shapes, of
// which the choice is 0.9 % longer than the best in the mean.
//   bf16 1024 -> 2752, rows 16, 128, 512, 2048, both gradients with dg and du: 19, 21, 32, 78 us, in two launches 40, 44, 42, 83.
struct GradientPlan {
    bool one, high;
    Merged merged;
};
rtoss_status plan_gradients(rtoss_dtype dt, const Product& rows, const Product& weights, GradientPlan* plan)
{
    DeviceInfo dev;
    RTOSS_TRY(current_device(&dev));
    const int eb = elem_bytes(dt);
    double two = plan_product(kBackWeights, false, dt, weights, dev.cus).time;
    if (rows.M > 0) two += plan_product(kBackRows, false, dt, rows, dev.cus).time;
    const MergedSpeed& speed = merged_speed(dt, std::max(product_rows(kBackRows, rows, eb), product_rows(kBackWeights, weights, eb)));
    double best = 1e300;
    for (bool high : {false, true}) {
        const Merged g = merged(dt, rows.M, rows.N, weights.M, high);
        if (g.row_tiles + g.weight_tiles > kMaxSliceTiles) continue;
        const double longest = std::max(g.row_steps / g.row_parts * (high ? speed.high : speed.low), g.weight_steps / g.weight_parts * speed.high);
        const double tiles = g.row_tiles * g.row_parts * (high ? speed.high_tile : speed.low_tile) * (g.rows_each ? 0.5 : 1) +
                             g.weight_tiles * g.weight_parts * speed.high_tile * (g.weights_each ? 0.5 : 1);
        const double moved = (4.0 * weights.M * rows.N + 2.0 * rows.M * (rows.N + weights.M)) * eb / 5.9e6;
        const double time = 4.3 + (g.row_parts > 1 || g.weight_parts > 1 ? 1.5 : 0) + std::max({longest, g.bytes / (speed.rate * dev.cus) + tiles / dev.cus, moved});
        if (time < best) best = time, *plan = GradientPlan{true, high, g};
    }
    if (best >= two) *plan = GradientPlan{};
    return RTOSS_OK;
}

rtoss_status launch_gradients(rtoss_dtype dt, const GradientPlan& plan, const Product& rows, const Product& weights, void* scratch, hipStream_t s)
{
    if (plan.one) {
        const Merged& g = plan.merged;
        uint32_t* const arrived = (uint32_t*)scratch;
        float* const sums = (float*)((char*)scratch + align_up(g.counters(), 256));
        const SumParts row_parts{g.row_parts, g.rows_each, sums, arrived};
        const SumParts weight_parts{g.weight_parts, g.weights_each, (float*)((char*)sums + g.row_bytes(plan.high)), arrived + (g.row_parts > 1 ? g.row_tiles : 0)};
        return launch_product_slices_back(dt, plan.high, rows, weights, row_parts, weight_parts, s);
    }
    if (rows.y) RTOSS_TRY(launch_product(kBackRows, false, dt, rows, s));
    if (weights.y) RTOSS_TRY(launch_product(kBackWeights, false, dt, weights, s));
    return RTOSS_OK;
}

size_t slopes_bytes(const rtoss_gated_desc& d) { return align_up((size_t)d.M * slopes_pitch(d.F, d.dt) * elem_bytes(d.dt), 256); }
size_t gradient_scratch(const rtoss_gated_desc& d)
{
    return align_up(std::max(merged(d.dt, d.M, d.K, d.F, false).scratch(false), merged(d.dt, d.M, d.K, d.F, true).scratch(true)), 256);
}

}  // namespace

}  // namespace rtoss

using namespace rtoss;

extern "C" {

rtoss_status rtoss_quantize_rows(const void* x_dev, rtoss_dtype dt, int64_t M, int64_t K, int64_t x_ld, int8_t* q_dev, int64_t q_ld,
                                 float* scale_dev, void* hip_stream)
{
    if (!known(dt)) return fail(RTOSS_EDTYPE, "bad dtype %d", (int)dt);
    RTOSS_TRY(check_rows(M, "M"));
    RTOSS_TRY(check_width(K, "K"));
    RTOSS_TRY(check_pitch(&x_ld, K, "x_ld"));
    RTOSS_TRY(check_pitch(&q_ld, K, "q_ld"));
    if (M == 0) return RTOSS_OK;
    RTOSS_TRY(check_pointer(x_dev, elem_bytes(dt), "x_dev"));
    RTOSS_TRY(check_pointer(q_dev, 1, "q_dev"));
    RTOSS_TRY(check_pointer(scale_dev, 4, "scale_dev"));
    const Span x = span(x_dev, M, K, x_ld, elem_bytes(dt)), q = span(q_dev, M, K, q_ld, 1), sc = span(scale_dev, M, 1, 1, 4);
    if (overlap(x, q) || overlap(x, sc) || overlap(q, sc)) return fail(RTOSS_EINVAL, "x, q and scale overlap");
    return launch_quantize_rows(x_dev, dt, M, (int)K, x_ld, q_dev, q_ld, scale_dev, (hipStream_t)hip_stream);
}

rtoss_status rtoss_matmul_i8(const rtoss_matmul_desc* desc, const int8_t* a_dev, const float* a_scale_dev, const int8_t* w_dev,
                             const rtoss_epilogue* epilogue, void* y_dev, void* hip_stream)
{
    if (!desc) return fail(RTOSS_EINVAL, "descriptor is NULL");
    rtoss_matmul_desc d = *desc;
    const rtoss_epilogue e = epilogue ? *epilogue : rtoss_epilogue{};
    if (!known(d.out_dt)) return fail(RTOSS_EDTYPE, "bad result dtype %d", (int)d.out_dt);
    if (!known(e.act)) return fail(RTOSS_EINVAL, "unknown activation %d", (int)e.act);
    RTOSS_TRY(check_rows(d.M, "M"));
    RTOSS_TRY(check_width(d.N, "N"));
    RTOSS_TRY(check_width(d.K, "K"));
    if (d.K > kMaxSumI8) return fail(RTOSS_ESHAPE, "K=%d: sums of more than %d products may pass 32 bits", d.K, kMaxSumI8);
    int64_t y_ld = e.y_ld, residual_ld = e.residual_ld;
    RTOSS_TRY(check_pitch(&d.a_ld, d.K, "a_ld"));
    RTOSS_TRY(check_pitch(&d.w_ld, d.K, "w_ld"));
    RTOSS_TRY(check_pitch(&y_ld, d.N, "y_ld"));
    RTOSS_TRY(check_pitch(&residual_ld, d.N, "residual_ld"));
    if (misaligned(a_scale_dev, 4) || misaligned(e.scale_dev, 4) || misaligned(e.bias_dev, 4))
        return fail(RTOSS_EINVAL, "scales and bias must be 4-byte aligned");
    if (d.M == 0) return RTOSS_OK;
    const int eb = elem_bytes(d.out_dt);
    RTOSS_TRY(check_pointer(a_dev, 1, "a_dev"));
    RTOSS_TRY(check_pointer(w_dev, 1, "w_dev"));
    RTOSS_TRY(check_pointer(y_dev, eb, "y_dev"));
    if (misaligned(e.residual_dev, eb)) return fail(RTOSS_EINVAL, "residual_dev is not aligned to its element size");
    const Span y = span(y_dev, d.M, d.N, y_ld, eb);
    const Span in[] = {span(a_dev, d.M, d.K, d.a_ld, 1), span(w_dev, d.N, d.K, d.w_ld, 1), span(a_scale_dev, d.M, 1, 1, 4),
                       span(e.scale_dev, d.N, 1, 1, 4),  span(e.bias_dev, d.N, 1, 1, 4),   span(e.residual_dev, d.M, d.N, residual_ld, eb)};
    for (const Span& i : in)
        if (overlap(y, i)) return fail(RTOSS_EINVAL, "operands, scales, bias or residual and y overlap");
    Product p{};
    p.a0 = a_dev;
    p.b0 = w_dev;
    p.lda = d.a_ld;
    p.ldb = d.w_ld;
    p.M = (int)d.M;
    p.N = d.N;
    p.R = d.K;
    p.act = e.act;
    p.sa = a_scale_dev;
    p.s0 = e.scale_dev;
    p.bias = e.bias_dev;
    p.residual = e.residual_dev;
    p.y = y_dev;
    p.ldr = residual_ld;
    p.ldy = y_ld;
    return launch_product(kScaled, true, d.out_dt, p, (hipStream_t)hip_stream);
}

rtoss_status rtoss_gated_ff(const rtoss_gated_desc* desc, const void* x_dev, const void* w_gate_dev, const void* w_up_dev, void* h_dev,
                            void* gate_dev, void* up_dev, void* hip_stream)
{
    rtoss_gated_desc d;
    RTOSS_TRY(gated_desc(desc, &d));
    if (!gate_dev != !up_dev) return fail(RTOSS_EINVAL, "gate_dev and up_dev are kept both or not at all");
    if (d.M == 0) return RTOSS_OK;
    const int eb = elem_bytes(d.dt);
    RTOSS_TRY(check_pointer(x_dev, eb, "x_dev"));
    RTOSS_TRY(check_pointer(w_gate_dev, eb, "w_gate_dev"));
    RTOSS_TRY(check_pointer(w_up_dev, eb, "w_up_dev"));
    RTOSS_TRY(check_pointer(h_dev, eb, "h_dev"));
    if (misaligned(gate_dev, eb) || misaligned(up_dev, eb)) return fail(RTOSS_EINVAL, "gate_dev and up_dev are not aligned to their element size");
    const Span in[] = {span(x_dev, d.M, d.K, d.x_ld, eb), span(w_gate_dev, d.F, d.K, d.w_ld, eb), span(w_up_dev, d.F, d.K, d.w_ld, eb)};
    const Span out[] = {span(h_dev, d.M, d.F, d.h_ld, eb), span(gate_dev, d.M, d.F, d.F, eb), span(up_dev, d.M, d.F, d.F, eb)};
    for (const Span& o : out) {
        for (const Span& i : in)
            if (overlap(o, i)) return fail(RTOSS_EINVAL, "operands and results overlap");
        for (const Span& other : out)
            if (&o != &other && overlap(o, other)) return fail(RTOSS_EINVAL, "results overlap");
    }
    Product p{};
    p.a0 = x_dev;
    p.b0 = w_gate_dev;
    p.b1 = w_up_dev;
    p.lda = d.x_ld;
    p.ldb = d.w_ld;
    p.M = (int)d.M;
    p.N = d.F;
    p.R = d.K;
    p.act = d.act;
    p.y = h_dev;
    p.y0 = gate_dev;
    p.y1 = up_dev;
    p.ldk = p.N;
    p.ldy = d.h_ld;
    return launch_product(kGated, false, d.dt, p, (hipStream_t)hip_stream);
}

rtoss_status rtoss_gated_ff_i8(const rtoss_gated_desc* desc, const int8_t* a_dev, const float* a_scale_dev, const int8_t* w_gate_dev,
                               const float* gate_scale_dev, const int8_t* w_up_dev, const float* up_scale_dev, void* h_dev, void* hip_stream)
{
    rtoss_gated_desc d;
    RTOSS_TRY(gated_desc(desc, &d));
    if (d.K > kMaxSumI8) return fail(RTOSS_ESHAPE, "K=%d: sums of more than %d products may pass 32 bits", d.K, kMaxSumI8);
    if (misaligned(a_scale_dev, 4) || misaligned(gate_scale_dev, 4) || misaligned(up_scale_dev, 4))
        return fail(RTOSS_EINVAL, "scales must be 4-byte aligned");
    if (d.M == 0) return RTOSS_OK;
    const int eb = elem_bytes(d.dt);
    RTOSS_TRY(check_pointer(a_dev, 1, "a_dev"));
    RTOSS_TRY(check_pointer(w_gate_dev, 1, "w_gate_dev"));
    RTOSS_TRY(check_pointer(w_up_dev, 1, "w_up_dev"));
    RTOSS_TRY(check_pointer(h_dev, eb, "h_dev"));
    const Span h = span(h_dev, d.M, d.F, d.h_ld, eb);
    const Span in[] = {span(a_dev, d.M, d.K, d.x_ld, 1),      span(w_gate_dev, d.F, d.K, d.w_ld, 1), span(w_up_dev, d.F, d.K, d.w_ld, 1),
                       span(a_scale_dev, d.M, 1, 1, 4),       span(gate_scale_dev, d.F, 1, 1, 4),    span(up_scale_dev, d.F, 1, 1, 4)};
    for (const Span& i : in)
        if (overlap(h, i)) return fail(RTOSS_EINVAL, "operands or scales and h overlap");
    Product p{};
    p.a0 = a_dev;
    p.b0 = w_gate_dev;
    p.b1 = w_up_dev;
    p.lda = d.x_ld;
    p.ldb = d.w_ld;
    p.M = (int)d.M;
    p.N = d.F;
    p.R = d.K;
    p.act = d.act;
    p.sa = a_scale_dev;
    p.s0 = gate_scale_dev;
    p.s1 = up_scale_dev;
    p.y = h_dev;
    p.ldy = d.h_ld;
    return launch_product(kGated, true, d.dt, p, (hipStream_t)hip_stream);
}

rtoss_status rtoss_gated_ff_backward_size(const rtoss_gated_desc* desc, size_t* workspace_bytes)
{
    rtoss_gated_desc d;
    RTOSS_TRY(gated_desc(desc, &d));
    if (!workspace_bytes) return fail(RTOSS_EINVAL, "size output pointer is NULL");
    *workspace_bytes = 2 * slopes_bytes(d) + gradient_scratch(d);
    return RTOSS_OK;
}

rtoss_status rtoss_gated_ff_backward(const rtoss_gated_desc* desc, const void* dh_dev, const void* x_dev, const void* w_gate_dev,
                                     const void* w_up_dev, const void* gate_dev, const void* up_dev, void* dx_dev, void* dw_gate_dev,
                                     void* dw_up_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream)
{
    rtoss_gated_desc d;
    RTOSS_TRY(gated_desc(desc, &d));
    if (!dw_gate_dev != !dw_up_dev) return fail(RTOSS_EINVAL, "dw_gate_dev and dw_up_dev are computed both or not at all");
    const int eb = elem_bytes(d.dt);
    const bool rows = dx_dev && d.M > 0, weights = dw_gate_dev;
    if (!rows && !weights) return RTOSS_OK;
    if (misaligned(dx_dev, eb) || misaligned(dw_gate_dev, eb) || misaligned(dw_up_dev, eb))
        return fail(RTOSS_EINVAL, "results are not aligned to their element size");
    if (d.M > 0) {
        RTOSS_TRY(check_pointer(dh_dev, eb, "dh_dev"));
        RTOSS_TRY(check_pointer(gate_dev, eb, "gate_dev"));
        RTOSS_TRY(check_pointer(up_dev, eb, "up_dev"));
        if (weights) RTOSS_TRY(check_pointer(x_dev, eb, "x_dev"));
        if (rows) {
            RTOSS_TRY(check_pointer(w_gate_dev, eb, "w_gate_dev"));
            RTOSS_TRY(check_pointer(w_up_dev, eb, "w_up_dev"));
        }
    }
    const size_t need = 2 * slopes_bytes(d) + gradient_scratch(d);
    if (workspace_bytes < need) return fail(RTOSS_ENOSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
    if (need && !workspace_dev) return fail(RTOSS_EINVAL, "workspace_dev is NULL");
    if (misaligned(workspace_dev, 256)) return fail(RTOSS_EINVAL, "workspace_dev is not 256-byte aligned");
    const Span in[] = {span(dh_dev, d.M, d.F, d.h_ld, eb),        span(x_dev, weights ? d.M : 0, d.K, d.x_ld, eb),
                       span(w_gate_dev, rows ? d.F : 0, d.K, d.w_ld, eb), span(w_up_dev, rows ? d.F : 0, d.K, d.w_ld, eb),
                       span(gate_dev, d.M, d.F, d.F, eb),         span(up_dev, d.M, d.F, d.F, eb)};
    const Span out[] = {span(dx_dev, rows ? d.M : 0, d.K, d.K, eb), span(dw_gate_dev, weights ? d.F : 0, d.K, d.K, eb),
                        span(dw_up_dev, weights ? d.F : 0, d.K, d.K, eb), span(workspace_dev, need ? 1 : 0, (int64_t)need, (int64_t)need, 1)};
    for (const Span& o : out) {
        for (const Span& i : in)
            if (overlap(o, i)) return fail(RTOSS_EINVAL, "operands and results or workspace overlap");
        for (const Span& other : out)
            if (&o != &other && overlap(o, other)) return fail(RTOSS_EINVAL, "results or workspace overlap");
    }
    const hipStream_t s = (hipStream_t)hip_stream;
    void *dg = workspace_dev, *du = (char*)workspace_dev + slopes_bytes(d);
    Product p{};
    p.a0 = dg;
    p.a1 = du;
    p.lda = slopes_pitch(d.F, d.dt);
    p.N = d.K;
    p.ldy = d.K;
    Product to_rows = p, to_weights = p;
    to_rows.b0 = w_gate_dev;
    to_rows.b1 = w_up_dev;
    to_rows.ldb = d.w_ld;
    to_rows.M = (int)d.M;
    to_rows.R = d.F;
    to_rows.y = rows ? dx_dev : nullptr;
    to_weights.b0 = x_dev;
    to_weights.ldb = d.x_ld;
    to_weights.M = d.F;
    to_weights.R = (int)d.M;
    to_weights.y = dw_gate_dev;
    to_weights.y1 = dw_up_dev;
    void* const scratch = (char*)workspace_dev + 2 * slopes_bytes(d);
    GradientPlan plan;
    RTOSS_TRY(plan_gradients(d.dt, to_rows, to_weights, &plan));
    const int counts = plan.one ? (int)(plan.merged.counters() / 4) : 0;
    if (d.M > 0)
        RTOSS_TRY(launch_gated_slopes(d.dt, d.act, d.M, d.F, dh_dev, d.h_ld, gate_dev, up_dev, dg, du, (uint32_t*)scratch, counts, s));
    return launch_gradients(d.dt, plan, to_rows, to_weights, scratch, s);
}

}  // extern "C"
