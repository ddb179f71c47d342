// Host side of the C ABI declared in include/ptq_fp8.h: argument checks, the choice of a kernel and of its cut, launches.
#include "../../include/ptq_fp8.h"

#include <algorithm>
#include <numeric>

#include "ptq_block_host.h"
#include "ptq_fp8.cuh"
#include "ptq_tensor_map.h"

namespace ptq {
__device__ unsigned g_fp8_status;     // what a kernel of this file that gave up a wait leaves behind
}

namespace {

using namespace ptq_host;

int blocks_of(int cols) { return static_cast<int>(ceil_div(cols, ptq::kFp8Block)); }

ptq_status_t status_word(unsigned **word)
{
    void *p = nullptr;
    PTQ_CUDA(cudaGetSymbolAddress(&p, ptq::g_fp8_status));
    *word = static_cast<unsigned *>(p);
    return PTQ_OK;
}

ptq_status_t input_check(const ptq_fp8_input_t *in, int64_t most_rows)
{
    if (!in) return fail(PTQ_ERR_NULL, "the input's description is NULL");
    if (!in->x) return fail(PTQ_ERR_NULL, "x is NULL");
    if (!dtype_ok(in->dtype)) return fail(PTQ_ERR_VALUE, "unknown type %d", in->dtype);
    if (in->rows < 1 || in->rows > most_rows || in->cols < 1 || in->cols > PTQ_FP8_MAX_COLS || in->x_pitch < 0)
        return fail(PTQ_ERR_SHAPE, "rows %lld, cols %d, pitch %lld out of range", static_cast<long long>(in->rows), in->cols,
                    static_cast<long long>(in->x_pitch));
    if (!aligned({in->x}, elem_bytes(in->dtype))) return fail(PTQ_ERR_ALIGN, "x is not aligned to its type");
    return PTQ_OK;
}
ptq_status_t codes_check(const void *codes, int64_t pitch, int cols)
{
    if (!codes) return fail(PTQ_ERR_NULL, "the codes are NULL");
    if (!aligned({codes}, 16) || pitch % 16) return fail(PTQ_ERR_ALIGN, "rows of codes begin on multiples of 16 bytes");
    // a tensor map's pitch has 40 bits
    if (pitch < cols || pitch >= (1ll << 40)) return fail(PTQ_ERR_SHAPE, "pitch %lld of the codes out of range", static_cast<long long>(pitch));
    return PTQ_OK;
}
ptq_status_t weight_check(const ptq_fp8_weight_t *w)
{
    if (!w) return fail(PTQ_ERR_NULL, "the weight's description is NULL");
    if (!w->scales) return fail(PTQ_ERR_NULL, "the weight's scales are NULL");
    if (w->cols < 1 || w->cols > PTQ_FP8_MAX_COLS || w->outputs < 1 || w->outputs > PTQ_FP8_MAX_OUTPUTS)
        return fail(PTQ_ERR_SHAPE, "cols %d, outputs %d out of range", w->cols, w->outputs);
    PTQ_TRY(codes_check(w->codes, w->codes_pitch, w->cols));
    if (!aligned({w->scales, w->bias}, 4)) return fail(PTQ_ERR_ALIGN, "scales or bias are not aligned to their type");
    return PTQ_OK;
}
ptq_status_t output_check(const void *y, int dtype, int64_t pitch, int outputs)
{
    if (!y) return fail(PTQ_ERR_NULL, "y is NULL");
    if (!dtype_ok(dtype)) return fail(PTQ_ERR_VALUE, "unknown type %d", dtype);
    if (pitch < outputs) return fail(PTQ_ERR_SHAPE, "rows of y overlap");
    if (!aligned({y}, elem_bytes(dtype))) return fail(PTQ_ERR_ALIGN, "y is not aligned to its type");
    return PTQ_OK;
}

// Whether two of rows x blocks scales have the same place: i rows on are j blocks on, with the least such i and j (not both zero).
bool scales_overlap(int64_t rows, int64_t blocks, int64_t row, int64_t block)
{
    if (row == 0 && block == 0) return rows > 1 || blocks > 1;
    const int64_t both = std::gcd(row, block);
    return block / both < rows && row / both < blocks;
}

// Whether the rows of x can be read 16 bytes at a time.
bool input_whole(const ptq_fp8_input_t &in) { return aligned({in.x}, 16) && in.x_pitch % (16 / elem_bytes(in.dtype)) == 0 && in.cols % 8 == 0; }

ptq_status_t quantize(const ptq_fp8_input_t &in, void *codes, int64_t codes_pitch, float *scales, int64_t scale_row, int64_t scale_block, cudaStream_t stream)
{
    ptq::Fp8QuantizeParams p = {};
    p.x = in.x;
    p.x_pitch = in.x_pitch;
    p.rows = in.rows;
    p.cols = in.cols;
    p.blocks = blocks_of(in.cols);
    p.codes = static_cast<uint8_t *>(codes);
    p.codes_pitch = codes_pitch;
    p.scales = scales;
    p.scale_row = scale_row;
    p.scale_block = scale_block;
    // three blocks at a time where that leaves no more of them idle (768 and 1536 channels), else four (4096)
    const int set = ceil_div(p.blocks, 3) * 3 <= ceil_div(p.blocks, 4) * 4 ? 3 : 4;
    p.sets = ptq::make_fastdiv(static_cast<unsigned>(ceil_div(p.blocks, set)));
    const long long items = ceil_div(in.rows, ptq::kFp8QuantizeRows) * p.sets.d;
    if (items > kMaxGrid - 16 * kSms) return fail(PTQ_ERR_SHAPE, "the input is too large for one launch");
    p.items = static_cast<unsigned>(items);
    const unsigned ctas = static_cast<unsigned>(std::min<long long>(items, (set == 3 ? 5 : 4) * kSms));   // as many as an SM holds
    return with_type(in.dtype, [&](auto t) {
        using T = decltype(t);
        return with_flag(input_whole(in), [&](auto whole) {
            constexpr bool kWhole = decltype(whole)::value;
            if (set == 3)
                ptq::ptq_fp8_quantize_kernel<T, 3, kWhole><<<ctas, 256, 0, stream>>>(p);
            else
                ptq::ptq_fp8_quantize_kernel<T, 4, kWhole><<<ctas, 256, 0, stream>>>(p);
            return launched();
        });
    });
}

// Which kernel, and how a product is cut.  bn: columns of a tile; one: a tile or a part of one per CTA.
struct Fp8Plan {
    int bn, split;
    bool swap, one;
};
constexpr int kFp8Smem = 232448;
// The cost of a cut, in microseconds, fitted to 9 cuts each of 16 products (1 .. 50432 rows): a k-block of a tile, bound by its loads; a tile's
// start and stores; a split tile's barriers and sums.  Rows of y that begin anywhere cost a tile of many rows more (its lanes hold rows).
// The two forms with 16 and with 256 columns, say: 1 x 4096 -> 4096 6.6 and 17 us, 2048 x 2048 -> 2048 over 100 and 12.2.
Fp8Plan product_plan(int64_t rows, int blocks, int outputs, bool fused, bool whole)
{
    Fp8Plan best = {};
    double least = -1.0;
    const auto consider = [&](int bn, bool swap, bool one, int split) {
        const long long tiles = swap ? ceil_div(outputs, 128) * ceil_div(rows, bn) : ceil_div(rows, 128) * ceil_div(outputs, bn);
        const double step = bn == 256 ? 0.53 : bn == 128 ? 0.34 : bn == 64 ? 0.30 : bn == 32 ? 0.27 : 0.25;
        const double ragged = swap || whole ? 0.0 : bn / 50.0;
        double cost;
        if (one)
            cost = 3.8 + static_cast<double>(ceil_div(tiles * split, kSms)) *
                             (static_cast<double>(ceil_div(blocks, split)) * step + ragged / split + bn / 128.0 * (1.0 + 0.6 * split) + (split > 1 ? 0.6 : 0.0));
        else
            cost = 2.3 + static_cast<double>(ceil_div(tiles, kSms)) * (blocks * step + ragged + bn / 128.0);
        if (least < 0.0 || cost < least) {
            least = cost;
            best = {bn, split, swap, one};
        }
    };
    for (int split = 1; split <= 8 && split <= blocks; split *= 2) {
        const int part = static_cast<int>(ceil_div(blocks, split));
        if (fused) {
            if (part <= ptq::kFp8MaxFused) consider(ptq::kFp8FusedRows, true, true, split);
            continue;
        }
        for (int bn : {16, 32, 64})
            if (rows <= 4096 && part * bn <= ptq::kFp8MaxScales) consider(bn, true, true, split);
        for (int bn : {64, 128}) consider(bn, false, true, split);
    }
    if (!fused)
        for (int bn : {128, 256}) consider(bn, false, false, 1);
    return best;
}
// Few rows are quantized by the CTAs that multiply them, each for itself: one launch instead of two.
bool linear_fused(int64_t rows, int blocks) { return rows <= ptq::kFp8FusedRows && blocks <= 8 * ptq::kFp8MaxFused; }

template <typename Y, int BN, bool kSwap, bool kOneTile, bool kFused, bool kWhole>
ptq_status_t launch_product(const Fp8Plan &plan, const ptq::Fp8Params &params, const CUtensorMap &tmP, const CUtensorMap &tmQ, bool next, cudaStream_t stream)
{
    constexpr auto kKern = ptq::ptq_fp8_matmul_kernel<Y, BN, kSwap, kOneTile, kFused, kWhole>;
    PTQ_TRY(ensure_smem<kKern>(kFp8Smem));
    ptq::Fp8Params p = params;
    const int part = static_cast<int>(ceil_div(p.blocks, plan.split));
    p.stages = ptq::kFp8MaxStages;
    if (kOneTile) p.stages = std::min(p.stages, part);
    const auto bytes = [&] { return ptq::fp8_layout<BN, kSwap, kOneTile, kFused>(p.stages, part).bytes; };
    while (p.stages > 1 && bytes() > kFp8Smem) --p.stages;
    if (bytes() > kFp8Smem) return fail(PTQ_ERR_SHAPE, "internal: %d bytes of shared memory", bytes());
    const long long tiles = static_cast<long long>(p.p_tiles) * p.q_tiles;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(kOneTile ? tiles * plan.split : std::min<long long>(tiles, kSms)));
    cfg.blockDim = dim3(ptq::kFp8Threads);
    cfg.dynamicSmemBytes = bytes();
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    if (plan.split > 1) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim.x = static_cast<unsigned>(plan.split);
        attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    if (next) {                       // may begin while the quantize kernel of the same call drains
        attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
        ++cfg.numAttrs;
    }
    PTQ_CUDA(cudaLaunchKernelEx(&cfg, kKern, tmP, tmQ, p));
    return launched();
}

// The product of the codes at `a` or, where there are none, of p.x (x_whole: input_whole).
ptq_status_t product(const ptq_fp8_weight_t &w, ptq::Fp8Params p, const void *a, int64_t a_pitch, int y_dtype, bool x_whole, bool next, cudaStream_t stream)
{
    const bool fused = a == nullptr;
    p.whole = aligned({p.y}, 16) && p.y_pitch % (16 / elem_bytes(y_dtype)) == 0;
    const Fp8Plan plan = product_plan(p.rows, p.blocks, p.outputs, fused, p.whole);
    p.split = plan.split;
    p.p_tiles = static_cast<int>(ceil_div(plan.swap ? p.outputs : p.rows, 128));
    p.q_tiles = static_cast<int>(ceil_div(plan.swap ? p.rows : p.outputs, plan.bn));
    // the group of tiles that run together is counted in 32 bits
    if (static_cast<long long>(p.p_tiles + 12) * p.q_tiles * plan.split > 0x7fffffffll) return fail(PTQ_ERR_SHAPE, "the product is too large for one launch");
    PTQ_TRY(status_word(&p.status));
    CUtensorMap tmW, tmA = {};
    PTQ_TRY(make_map_2d(&tmW, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, w.codes, p.cols, p.outputs, w.codes_pitch, ptq::kFp8Block, plan.swap ? 128 : plan.bn));
    if (!fused) PTQ_TRY(make_map_2d(&tmA, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a, p.cols, p.rows, a_pitch, ptq::kFp8Block, plan.swap ? plan.bn : 128));
    return with_type(y_dtype, [&](auto t) -> ptq_status_t {
        using Y = decltype(t);
        if (fused)
            return with_flag(x_whole, [&](auto whole) {
                return launch_product<Y, ptq::kFp8FusedRows, true, true, true, decltype(whole)::value>(plan, p, tmW, tmW, next, stream);
            });
        if (plan.swap) {
            if (plan.bn == 16) return launch_product<Y, 16, true, true, false, false>(plan, p, tmW, tmA, next, stream);
            if (plan.bn == 32) return launch_product<Y, 32, true, true, false, false>(plan, p, tmW, tmA, next, stream);
            return launch_product<Y, 64, true, true, false, false>(plan, p, tmW, tmA, next, stream);
        }
        if (plan.one)
            return plan.bn == 64 ? launch_product<Y, 64, false, true, false, false>(plan, p, tmA, tmW, next, stream)
                                 : launch_product<Y, 128, false, true, false, false>(plan, p, tmA, tmW, next, stream);
        return plan.bn == 128 ? launch_product<Y, 128, false, false, false, false>(plan, p, tmA, tmW, next, stream)
                              : launch_product<Y, 256, false, false, false, false>(plan, p, tmA, tmW, next, stream);
    });
}

ptq::Fp8Params product_params(const ptq_fp8_weight_t &w, int64_t rows, void *y, int64_t y_pitch)
{
    ptq::Fp8Params p = {};
    p.w_scales = w.scales;
    p.bias = w.bias;
    p.y = y;
    p.y_pitch = y_pitch;
    p.rows = static_cast<int>(rows);
    p.cols = w.cols;
    p.outputs = w.outputs;
    p.blocks = blocks_of(w.cols);
    return p;
}

}  // namespace

extern "C" {

ptq_status_t ptq_fp8_quantize(const ptq_fp8_input_t *in, void *codes, int64_t codes_pitch, float *scales, const int64_t scales_pitch[2], void *stream)
{
    PTQ_TRY(input_check(in, PTQ_FP8_MAX_ROWS));
    PTQ_TRY(codes_check(codes, codes_pitch, in->cols));
    if (!scales || !scales_pitch) return fail(PTQ_ERR_NULL, "the scales or their pitches are NULL");
    if (!aligned({scales}, 4)) return fail(PTQ_ERR_ALIGN, "the scales are not aligned to their type");
    if (!not_negative({scales_pitch[0], scales_pitch[1]})) return fail(PTQ_ERR_SHAPE, "a pitch is negative");
    if (scales_overlap(in->rows, blocks_of(in->cols), scales_pitch[0], scales_pitch[1])) return fail(PTQ_ERR_SHAPE, "scales overlap");
    PTQ_TRY(check_arch());
    return quantize(*in, codes, codes_pitch, scales, scales_pitch[0], scales_pitch[1], static_cast<cudaStream_t>(stream));
}

ptq_status_t ptq_fp8_quantize_weight(const ptq_fp8_input_t *in, void *codes, int64_t codes_pitch, float *scales, void *stream)
{
    PTQ_TRY(input_check(in, PTQ_FP8_MAX_OUTPUTS));
    PTQ_TRY(codes_check(codes, codes_pitch, in->cols));
    if (!scales) return fail(PTQ_ERR_NULL, "the scales are NULL");
    if (!aligned({scales}, 4)) return fail(PTQ_ERR_ALIGN, "the scales are not aligned to their type");
    PTQ_TRY(check_arch());
    ptq::Fp8QuantizeParams p = {};
    p.x = in->x;
    p.x_pitch = in->x_pitch;
    p.rows = in->rows;
    p.cols = in->cols;
    p.blocks = blocks_of(in->cols);
    p.codes = static_cast<uint8_t *>(codes);
    p.codes_pitch = codes_pitch;
    p.scales = scales;
    const dim3 grid(static_cast<unsigned>(p.blocks), static_cast<unsigned>(ceil_div(in->rows, ptq::kFp8Block)));
    return with_type(in->dtype, [&](auto t) {
        ptq::ptq_fp8_quantize_weight_kernel<decltype(t)><<<grid, 256, 0, static_cast<cudaStream_t>(stream)>>>(p);
        return launched();
    });
}

ptq_status_t ptq_fp8_matmul(const ptq_fp8_weight_t *w, int64_t rows, const void *a, int64_t a_pitch, const float *a_scales, const int64_t a_scales_pitch[2],
                            void *y, int y_dtype, int64_t y_pitch, void *stream)
{
    PTQ_TRY(weight_check(w));
    if (rows < 1 || rows > PTQ_FP8_MAX_ROWS) return fail(PTQ_ERR_SHAPE, "rows %lld out of range", static_cast<long long>(rows));
    PTQ_TRY(codes_check(a, a_pitch, w->cols));
    if (!a_scales || !a_scales_pitch) return fail(PTQ_ERR_NULL, "the scales or their pitches are NULL");
    if (!aligned({a_scales}, 4)) return fail(PTQ_ERR_ALIGN, "the scales are not aligned to their type");
    if (!not_negative({a_scales_pitch[0], a_scales_pitch[1]})) return fail(PTQ_ERR_SHAPE, "a pitch is negative");
    PTQ_TRY(output_check(y, y_dtype, y_pitch, w->outputs));
    PTQ_TRY(check_arch());
    ptq::Fp8Params p = product_params(*w, rows, y, y_pitch);
    p.a_scales = a_scales;
    p.scale_row = a_scales_pitch[0];
    p.scale_block = a_scales_pitch[1];
    return product(*w, p, a, a_pitch, y_dtype, false, false, static_cast<cudaStream_t>(stream));
}

size_t ptq_fp8_linear_workspace_bytes(int64_t rows, int cols, int outputs)
{
    if (rows < 1 || rows > PTQ_FP8_MAX_ROWS || cols < 1 || cols > PTQ_FP8_MAX_COLS || outputs < 1 || outputs > PTQ_FP8_MAX_OUTPUTS) return 0;
    if (linear_fused(rows, blocks_of(cols))) return 0;
    return padded(static_cast<size_t>(rows) * (static_cast<size_t>(ceil_div(cols, 16)) * 16)) + padded(static_cast<size_t>(rows) * blocks_of(cols) * 4);
}

ptq_status_t ptq_fp8_linear(const ptq_fp8_weight_t *w, const ptq_fp8_input_t *in, void *y, int64_t y_pitch, void *workspace, size_t workspace_bytes, void *stream)
{
    PTQ_TRY(weight_check(w));
    PTQ_TRY(input_check(in, PTQ_FP8_MAX_ROWS));
    if (in->cols != w->cols) return fail(PTQ_ERR_SHAPE, "x has %d columns, the weight %d", in->cols, w->cols);
    PTQ_TRY(output_check(y, in->dtype, y_pitch, w->outputs));
    const size_t need = ptq_fp8_linear_workspace_bytes(in->rows, in->cols, w->outputs);
    PTQ_TRY(check_space(workspace, workspace_bytes, need));
    PTQ_TRY(check_arch());
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    ptq::Fp8Params p = product_params(*w, in->rows, y, y_pitch);
    if (need == 0) {
        p.x = in->x;
        p.x_pitch = in->x_pitch;
        return product(*w, p, nullptr, 0, in->dtype, input_whole(*in), false, st);
    }
    const int64_t pitch = ceil_div(in->cols, 16) * 16;
    float *scales = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + padded(static_cast<size_t>(in->rows) * pitch));
    PTQ_TRY(quantize(*in, workspace, pitch, scales, 1, in->rows, st));
    p.a_scales = scales;
    p.scale_row = 1;
    p.scale_block = in->rows;
    return product(*w, p, workspace, pitch, in->dtype, false, true, st);
}

ptq_status_t ptq_fp8_device_status(void)
{
    PTQ_TRY(check_arch());
    unsigned word = 0;
    PTQ_CUDA(cudaDeviceSynchronize());
    PTQ_CUDA(cudaMemcpyFromSymbol(&word, ptq::g_fp8_status, sizeof(word)));
    if (word == 0) return PTQ_OK;
    const unsigned zero = 0;
    PTQ_CUDA(cudaMemcpyToSymbol(ptq::g_fp8_status, &zero, sizeof(zero)));
    return fail(PTQ_ERR_TIMEOUT, "a kernel abandoned a bounded wait (status word 0x%x); its output is undefined", word);
}

}  // extern "C"
