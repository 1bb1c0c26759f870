// C entries of the 8-bit products and the gated feed-forward block: checks of the arguments (before any HIP call) and the choice of
// kernels.
#include <algorithm>
#include <cmath>

#include "products.h"

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
    const char *from, *to;
    bool plain;  // its rows without gaps (two slices of one wider buffer interleave without sharing an element)
};
Span span(const void* p, int64_t rows, int64_t width, int64_t ld, int eb)
{
    const char* c = (const char*)p;
    return Span{c, p && rows > 0 ? c + ((rows - 1) * ld + width) * eb : c, ld == width || rows <= 1};
}
bool overlap(const Span& a, const Span& b) { return a.plain && b.plain && a.from < b.to && b.from < a.to; }

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
// in the large, and by whole rounds of workgroups.  Constants as measured (us, 256 CUs; M x K x N):
//   slices of a x b: the launch 3.4 (64 x 64: 4.6), then 80 KB/us and CU for the rows of both operands.  8-bit 4096 x 4096, rows 1, 64, 128, 256, 512:
//     5.1, 6.8, 7.8, 10.2, 17.6 with the tile that this takes; 8.5, 9.6, 9.6, 10.2, 17.6 with 64 x 64 for all.
//   tiles: 6 and 8, then 0.95 and 1.3 a stage of 128 bytes (128 and 256 channels).  Gated bf16 4096 -> 10944, rows 256, 512, 1000, 2048: 62, 117,
//     183, 360 with 128, 83, 90, 173, 284 with 256 channels; slices of 64 x 64 104, 178, 352, 850.
struct Choice {
    int kernel;   // slices by tile, then the two widths of tiles
    double time;  // us
};
Choice choose(ProductForm form, bool bits8, rtoss_dtype out, const Product& p, int cus)
{
    const int eb = bits8 ? 1 : elem_bytes(out);
    const bool gated = form == kGated, across = form == kBackRows || form == kBackWeights;
    const double row = (double)p.R * eb * (form == kBackRows ? 2 : 1);
    const auto up = [](int64_t n, int by) { return (double)((n + by - 1) / by); };
    const auto tiles = [&](int rows, int channels) { return up(p.M, rows) * up(p.N, channels) * (form == kBackWeights ? 2 : 1); };
    Choice best{kSliceTiles - 1, 1e300};
    for (int t = across ? kSliceTiles - 1 : 0; t < kSliceTiles; ++t) {
        const int a = kSlices[t].rows, n = gated ? kSlices[t].gated : kSlices[t].channels, b = gated ? 2 * n : n;
        if (tiles(a, n) > kMaxSliceTiles) continue;
        const double count = tiles(a, n) / cus;
        const int together = 160 / (a + b);  // workgroups whose LDS a CU holds
        const double rounds = together >= 2 ? std::max(1.0, count) : std::ceil(count);
        const double one = std::max((a + b) * row / 80e3, eb == 4 ? a * b * row / eb / 500e3 : 0.0);
        const double time = (a + b >= 128 ? 4.6 : a + b >= 96 ? 3.8 : 3.4) + rounds * one;
        if (time < best.time) best = Choice{t, time};
    }
    if (product_tiles_ok(bits8, out, p)) {
        const double stages = std::ceil(row / 128);
        const int widths = product_pieces_ok(form, p, eb) ? 2 : 1;
        for (int wide = 0; wide < widths; ++wide) {
            const int n = (wide ? 256 : 128) / (gated ? 2 : 1);
            const double time = (wide ? 8 : 6) + std::ceil(tiles(256, n) / cus) * stages * (wide ? 1.3 : 0.95);
            if (time < best.time) best = Choice{kSliceTiles + wide, time};
        }
    }
    return best;
}

rtoss_status launch_chosen(int kernel, ProductForm form, bool bits8, rtoss_dtype out, const Product& p, hipStream_t s)
{
    if (kernel < kSliceTiles) return launch_product_slices(form, bits8, out, kernel, p, s);
    return launch_product_tiles(form, bits8, out, kernel > kSliceTiles, p, s);
}

// A launch has at most kMaxSliceTiles of the largest slices: more rows than that take several.
rtoss_status launch_product(ProductForm form, bool bits8, rtoss_dtype out, const Product& p, hipStream_t s)
{
    DeviceInfo dev;
    RTOSS_TRY(current_device(&dev));
    const int eb = bits8 ? 1 : elem_bytes(out), out_eb = elem_bytes(out);
    const int64_t across = ((int64_t)p.N + 31) / 32 * 2;
    const int64_t most = std::max<int64_t>(kMaxSliceTiles / across, 1) * 64;  // rows
    if (p.M <= most) return launch_chosen(choose(form, bits8, out, p, dev.cus).kernel, form, bits8, out, p, s);
    for (int64_t m = 0; m < p.M; m += most) {
        Product part = p;
        const auto on = [](const void* base, int64_t bytes) { return base ? (void*)((char*)base + bytes) : nullptr; };
        const int64_t a_step = form == kBackWeights ? eb : p.lda * eb;  // (there the rows of the result are columns of its operand)
        part.M = (int)std::min<int64_t>(most, p.M - m);
        part.a0 = on(p.a0, m * a_step);
        part.a1 = on(p.a1, m * a_step);
        part.sa = (const float*)on(p.sa, m * 4);
        part.residual = on(p.residual, m * p.ldr * out_eb);
        part.y = on(p.y, m * p.ldy * out_eb);
        part.y0 = on(p.y0, m * p.N * out_eb);
        part.y1 = on(p.y1, m * (form == kBackWeights ? p.ldy : p.N) * out_eb);
        RTOSS_TRY(launch_chosen(choose(form, bits8, out, part, dev.cus).kernel, form, bits8, out, part, s));
    }
    return RTOSS_OK;
}

// Both gradients, or one (the other's y is NULL), by the same kernels either way: in one launch of slices where that is shorter than two.
//   one launch: 3.5 us, then 65 KB/us and CU for the rows of both operands, or the longest sum, four stages at a time (0.6 and 0.75 us for tiles of
//   16 and 64 rows).  bf16 1024 -> 2752, rows 16, 128, 512, 2048, both gradients with dg and du: 18, 21, 32, 78 us, in two launches 40, 44, 42, 82.
rtoss_status launch_gradients(rtoss_dtype dt, Product rows, Product weights, hipStream_t s)
{
    DeviceInfo dev;
    RTOSS_TRY(current_device(&dev));
    const int eb = elem_bytes(dt);
    const auto up = [](int64_t n, int by) { return (double)((n + by - 1) / by); };
    double two = choose(kBackWeights, false, dt, weights, dev.cus).time;
    if (rows.M > 0) two += choose(kBackRows, false, dt, rows, dev.cus).time;
    const double weight_tiles = 2 * up(weights.M, 64) * up(weights.N, 64), stages = std::ceil(rows.R * eb / 128.0) * 2;
    bool high = false;
    double one = 1e300;
    for (int t = 0; t < 2; ++t) {
        const int a = t ? 64 : 16;
        const double row_tiles = up(rows.M, a) * up(rows.N, 64);
        if (row_tiles + weight_tiles > kMaxSliceTiles) continue;
        const double bytes = row_tiles * (a + 64) * 2.0 * rows.R * eb + weight_tiles * 128.0 * weights.R * eb;
        const double time = 3.5 + std::max(std::ceil(stages / 4) * (t ? 0.75 : 0.6), bytes / (65e3 * dev.cus));
        if (time < one) one = time, high = t;
    }
    if (one < two) return launch_product_slices_back(dt, high, rows, weights, s);
    if (rows.y) RTOSS_TRY(launch_product(kBackRows, false, dt, rows, s));
    if (weights.y) RTOSS_TRY(launch_product(kBackWeights, false, dt, weights, s));
    return RTOSS_OK;
}

size_t slopes_bytes(const rtoss_gated_desc& d) { return align_up((size_t)d.M * slopes_pitch(d.F, d.dt) * elem_bytes(d.dt), 256); }

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
    if (overlap(y, span(a_dev, d.M, d.K, d.a_ld, 1)) || overlap(y, span(w_dev, d.N, d.K, d.w_ld, 1))) return fail(RTOSS_EINVAL, "operands and y overlap");
    if (overlap(y, span(e.residual_dev, e.residual_dev ? d.M : 0, d.N, residual_ld, eb))) return fail(RTOSS_EINVAL, "residual and y overlap");
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
    const Span out[] = {span(h_dev, d.M, d.F, d.h_ld, eb), span(gate_dev, gate_dev ? d.M : 0, d.F, d.F, eb), span(up_dev, up_dev ? d.M : 0, d.F, d.F, eb)};
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
    if (overlap(h, span(a_dev, d.M, d.K, d.x_ld, 1)) || overlap(h, span(w_gate_dev, d.F, d.K, d.w_ld, 1)) || overlap(h, span(w_up_dev, d.F, d.K, d.w_ld, 1)))
        return fail(RTOSS_EINVAL, "operands and h overlap");
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
    *workspace_bytes = 2 * slopes_bytes(d);
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
    const size_t need = 2 * slopes_bytes(d);
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
    if (d.M > 0) RTOSS_TRY(launch_gated_slopes(d.dt, d.act, d.M, d.F, dh_dev, d.h_ld, gate_dev, up_dev, dg, du, s));
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
    return launch_gradients(d.dt, to_rows, to_weights, s);
}

}  // extern "C"
