// Host side of the C ABI declared in include/ptq_block.h: argument checks, how the work is cut, kernel launches.
#include "../../include/ptq_block.h"

#include <algorithm>
#include <cmath>

#include "ptq_block_host.h"
#include "ptq_conv.cuh"
#include "ptq_norm.cuh"
#include "ptq_scan_launch.cuh"

namespace {

using namespace ptq_host;

// ---------------------------------------------------------------------------------------------------- scan
// How a call is cut.
struct ScanPlan {
    ScanSplit split;                  // of the forward pass
    int group_warps, group_blocks, chunk_len, chunks;
    long long warps, ctas;            // of one chunk
    ScanCut cut(int n, bool whole) const { return {split, warps * n, ctas * n, whole}; }
};
// Chunks of a multiple of 32 steps.  The time goes as the steps of a chunk and as the sets of warps that the GPU holds at once: 12 to an
// SM, 16 where a lane has two states at most and, in the backward pass, rows of 16-bit values (binary32 rows fill the shared memory: 32 x 784
// x 384 with one state, 16 assumed: fp16 training 187 -> 167 us, fp32 192 -> 224).  Backward, shared memory leaves 8 warps in binary32 from N = 9
// on and 4 in every type from N = 17 on; such calls are cut as if there were 12.  More than one chunk: everything but the output is gone over twice,
// there is another launch (about 60 steps), and the last chunk folds the others' sums.
ScanPlan scan_plan(const ptq_scan_t &s, bool backward)
{
    const double resident = (s.states <= 2 && (!backward || s.dtype != PTQ_F32) ? 16.0 : 12.0) * kSms;
    const int per_group = s.channels / s.groups;
    const long long sequences = static_cast<long long>(s.batch) * s.groups;
    ScanPlan p;
    p.split = scan_split_forward(s.states, 0);
    long long warps = sequences * ceil_div(per_group, p.split.width());
    // A padded batch holds about half the tokens if its lengths are spread evenly.  One that is full after all may be cut into a chunk more than it
    // should: 64 x 197 x 384, N = 16, forward 72 us and 44 without lengths, backward 185 and 155; 16 x 784 x 768 the same with and without.
    const double filled = s.lengths ? 0.5 : 1.0;
    long long chunks = 1;
    double least = -1.0;
    for (long long n = 1; n <= ceil_div(s.length, 32) && n <= 512; n = n < 16 ? n + 1 : n + n / 8) {
        const double len = 32.0 * static_cast<double>(ceil_div(ceil_div(s.length, n), 32));
        const double load = std::max(1.0, std::ceil(filled * static_cast<double>(warps) * n / resident - 0.02));
        const double cost = n == 1 ? s.length * load : 1.8 * len * load + 60.0 + 2.0 * n;
        if (least < 0.0 || cost < least) {
            least = cost;
            chunks = n;
        }
    }
    if (warps * chunks < 9 * kSms) p.split = scan_split_forward(s.states, warps * chunks < 4 * kSms ? 2 : 1);
    p.chunk_len = static_cast<int>(ceil_div(ceil_div(s.length, chunks), 32) * 32);
    p.chunks = static_cast<int>(ceil_div(s.length, p.chunk_len));
    p.group_warps = static_cast<int>(ceil_div(per_group, p.split.width()));
    p.warps = sequences * p.group_warps;
    p.group_blocks = static_cast<int>(ceil_div(per_group, scan_split_backward(s.states).width() * ptq::kScanWarps));
    p.ctas = sequences * p.group_blocks;
    return p;
}

ptq_status_t scan_check(const ptq_scan_t *s)
{
    if (!s) return fail(PTQ_ERR_NULL, "the call's description is NULL");
    if (!s->u || !s->delta || !s->B || !s->C || !s->A) return fail(PTQ_ERR_NULL, "u, delta, A, B or C is NULL");
    if (!dtype_ok(s->dtype)) return fail(PTQ_ERR_VALUE, "unknown type %d", s->dtype);
    if (s->batch < 1 || s->length < 1 || s->length > PTQ_MAX_LENGTH || s->channels < 1 || s->channels > PTQ_MAX_CHANNELS || s->states < 1 ||
        s->states > PTQ_MAX_STATES || s->groups < 1)
        return fail(PTQ_ERR_SHAPE, "batch %d, length %d, channels %d, states %d, groups %d out of range", s->batch, s->length, s->channels, s->states,
                    s->groups);
    if (s->channels % s->groups) return fail(PTQ_ERR_SHAPE, "%d channels do not make %d groups", s->channels, s->groups);
    if (s->flags & ~(PTQ_SCAN_SOFTPLUS | PTQ_SEQ_REVERSE)) return fail(PTQ_ERR_VALUE, "unknown flags %u", s->flags);
    if (!not_negative({s->u_pitch[0], s->u_pitch[1], s->delta_pitch[0], s->delta_pitch[1], s->z ? s->z_pitch[0] : 0, s->z ? s->z_pitch[1] : 0,
                       s->B_pitch[0], s->B_pitch[1], s->B_pitch[2], s->C_pitch[0], s->C_pitch[1], s->C_pitch[2]}))
        return fail(PTQ_ERR_SHAPE, "a pitch is negative");
    if (!aligned({s->u, s->delta, s->z, s->B, s->C}, elem_bytes(s->dtype)) || !aligned({s->A, s->D, s->delta_bias, s->state, s->lengths}, 4))
        return fail(PTQ_ERR_ALIGN, "an input is not aligned to its type");
    return PTQ_OK;
}
ptq_status_t scan_check(const ScanPlan &plan)
{
    if (std::max(plan.warps, plan.ctas) * plan.chunks > kMaxGrid) return fail(PTQ_ERR_SHAPE, "the batch is too large for one launch");
    return PTQ_OK;
}

ptq::ScanParams scan_params(const ptq_scan_t &s, const ScanPlan &plan)
{
    ptq::ScanParams p = {};
    p.u = s.u;
    p.delta = s.delta;
    p.z = s.z;
    p.B = s.B;
    p.C = s.C;
    p.u_b = s.u_pitch[0];
    p.u_l = s.u_pitch[1];
    p.delta_b = s.delta_pitch[0];
    p.delta_l = s.delta_pitch[1];
    p.z_b = s.z ? s.z_pitch[0] : 0;
    p.z_l = s.z ? s.z_pitch[1] : 0;
    p.B_b = s.B_pitch[0];
    p.B_l = s.B_pitch[1];
    p.B_g = s.B_pitch[2];
    p.C_b = s.C_pitch[0];
    p.C_l = s.C_pitch[1];
    p.C_g = s.C_pitch[2];
    p.A = s.A;
    p.D = s.D;
    p.delta_bias = s.delta_bias;
    p.state = s.state;
    p.lengths = s.lengths;
    p.batch = s.batch;
    p.length = s.length;
    p.channels = s.channels;
    p.states = s.states;
    p.groups = s.groups;
    p.group_channels = s.channels / s.groups;
    p.group_warps = plan.group_warps;
    p.group_blocks = plan.group_blocks;
    p.chunk_len = plan.chunk_len;
    p.chunks = plan.chunks;
    p.flags = s.flags;
    p.unit = 1;
    for (int unit : {4, 2})
        if (p.unit == 1 && aligned({s.u, s.delta, s.z}, unit * elem_bytes(s.dtype)) &&
            multiples({p.u_b, p.u_l, p.delta_b, p.delta_l, p.z_b, p.z_l, p.group_channels}, unit))
            p.unit = unit;
    p.bc_unit = 1;
    for (int unit : {4, 2})
        if (p.bc_unit == 1 && s.states % unit == 0 && aligned({s.B, s.C}, unit * elem_bytes(s.dtype)) &&
            multiples({p.B_b, p.B_l, p.B_g, p.C_b, p.C_l, p.C_g}, unit))
            p.bc_unit = unit;
    return p;
}

// Whether a call's rows and states can be moved 16 bytes at a time, as far as its description goes.
bool scan_whole(const ptq_scan_t &s)
{
    const int unit = 16 / elem_bytes(s.dtype);
    return aligned({s.u, s.delta, s.z, s.A, s.D, s.delta_bias, s.state}, 16) &&
           multiples({s.u_pitch[0], s.u_pitch[1], s.delta_pitch[0], s.delta_pitch[1], s.z ? s.z_pitch[0] : 0, s.z ? s.z_pitch[1] : 0,
                      s.channels / s.groups}, unit) &&
           (s.states <= 2 || s.states % 4 == 0);
}

// Workspace: slots and sums of the chunks, and for the backward pass the shares of the CTAs.
struct ScanSpace {
    size_t slots, sums, part_A, part_D, part_bias, part_BC, bytes;
};
ScanSpace scan_space(const ptq_scan_t &s, const ScanPlan &plan, bool backward)
{
    ScanSpace w = {};
    size_t at = 0;
    const auto take = [&](size_t floats) {
        const size_t here = at;
        at += padded(floats * 4);
        return here;
    };
    const size_t rows = static_cast<size_t>(s.batch) * s.channels;
    if (plan.chunks > 1) {
        w.slots = take(rows * plan.chunks * s.states);
        w.sums = take(rows * plan.chunks);
    }
    if (backward) {
        w.part_A = take(rows * plan.chunks * s.states);
        w.part_D = take(rows * plan.chunks);
        w.part_bias = take(rows * plan.chunks);
        if (plan.group_blocks > 1) w.part_BC = take(static_cast<size_t>(s.groups) * plan.group_blocks * s.batch * s.length * 2 * s.states);
    }
    w.bytes = at;
    return w;
}

// ---------------------------------------------------------------------------------------------------- norm
ptq_status_t norm_check(const ptq_norm_t *n)
{
    if (!n) return fail(PTQ_ERR_NULL, "the call's description is NULL");
    if (!n->x) return fail(PTQ_ERR_NULL, "x is NULL");
    if (!dtype_ok(n->dtype) || !dtype_ok(n->residual_dtype)) return fail(PTQ_ERR_VALUE, "unknown type");
    if (n->residual_dtype != n->dtype && n->residual_dtype != PTQ_F32) return fail(PTQ_ERR_VALUE, "the residual has x's type or binary32");
    if (n->rows < 1 || n->cols < 1 || n->cols > PTQ_MAX_NORM_COLS || n->rows > (1ll << 40))
        return fail(PTQ_ERR_SHAPE, "rows %lld, cols %d out of range", static_cast<long long>(n->rows), n->cols);
    if (n->flags & ~(PTQ_NORM_LAYER | PTQ_NORM_GATE_OUT)) return fail(PTQ_ERR_VALUE, "unknown flags %u", n->flags);
    if (!(n->eps >= 0.0f) || std::isinf(n->eps)) return fail(PTQ_ERR_VALUE, "eps must be finite and not negative");
    if (!not_negative({n->x_pitch, n->residual ? n->residual_pitch : 0, n->gate ? n->gate_pitch : 0})) return fail(PTQ_ERR_SHAPE, "a pitch is negative");
    if (!aligned({n->x, n->gate}, elem_bytes(n->dtype)) || !aligned({n->residual}, elem_bytes(n->residual_dtype)) ||
        !aligned({n->weight, n->bias, n->scale}, 4))
        return fail(PTQ_ERR_ALIGN, "an input is not aligned to its type");
    return PTQ_OK;
}
ptq::NormParams norm_params(const ptq_norm_t &n)
{
    ptq::NormParams p = {};
    p.x = n.x;
    p.residual = n.residual;
    p.gate = n.gate;
    p.x_l = n.x_pitch;
    p.residual_l = n.residual_pitch;
    p.gate_l = n.gate_pitch;
    p.weight = n.weight;
    p.bias = n.bias;
    p.scale = n.scale;
    p.rows = n.rows;
    p.cols = n.cols;
    p.gate_at = !n.gate ? ptq::kGateNone : n.flags & PTQ_NORM_GATE_OUT ? ptq::kGateOut : ptq::kGateIn;
    p.eps = n.eps;
    p.inv_cols = static_cast<float>(1.0 / n.cols);
    p.layer = n.flags & PTQ_NORM_LAYER;
    return p;
}
bool norm_whole(const ptq_norm_t &n)
{
    const int unit = 16 / elem_bytes(n.dtype), residual_unit = 16 / elem_bytes(n.residual_dtype);
    return aligned({n.x, n.residual, n.gate, n.weight, n.bias, n.scale}, 16) && multiples({n.x_pitch, n.gate ? n.gate_pitch : 0, n.cols}, unit) &&
           (!n.residual || n.residual_pitch % residual_unit == 0);
}
// Threads of a CTA, rows that it takes at a time, sets of rows, their layout and bytes in shared memory, CTAs.  The number of CTAs goes by the
// description alone, since the workspace does: it takes a call with a residual to have a dresidual_out, and one without to have none.
struct NormPlan {
    int threads, rows, stages, bytes, ctas;
    ptq::NormStage stage;
};
NormPlan norm_plan(const ptq_norm_t &n, bool backward, bool has_dresidual)
{
    NormPlan p;
    p.threads = static_cast<int>(ceil_div(n.cols, 256)) * 32;
    p.rows = p.threads > 256 || n.rows <= 8 * kSms ? 1 : backward ? 2 : 4;
    const auto lay_out = [&](bool dresidual) {
        p.stage = ptq::norm_stage(n.residual, n.gate, backward, dresidual, elem_bytes(n.dtype) / 2, elem_bytes(n.residual_dtype) / 2, p.rows, p.threads);
        p.stages = 2 * 16 * p.stage.size <= 200 * 1024 ? 2 : 1;
        p.bytes = p.stages * 16 * p.stage.size;
    };
    lay_out(backward && n.residual);
    const int resident = std::max(1, std::min((backward ? 640 : 1024) / p.threads, 220 * 1024 / (p.bytes + 8 * 1024)));
    p.ctas = static_cast<int>(std::min<long long>(ceil_div(n.rows, p.rows), std::min(resident, 24) * kSms));
    lay_out(backward && has_dresidual);
    return p;
}
template <bool kBackward>
ptq_status_t launch_norm(const ptq_norm_t &n, const NormPlan &plan, const ptq::NormParams &p, bool whole_rows, cudaStream_t stream)
{
    return with_type(n.dtype, [&](auto t) {
        using T = decltype(t);
        const auto go = [&](auto r) {
            using R = decltype(r);
            return with_flag(whole_rows, [&](auto whole) {
                constexpr int kRB = kBackward ? 2 : 4;
                constexpr bool kWhole = decltype(whole)::value;
                const auto launch = [&](auto kern) {
                    constexpr auto kKern = decltype(kern)::value;
                    PTQ_TRY(ensure_smem<kKern>(200 * 1024));
                    kKern<<<plan.ctas, plan.threads, plan.bytes, stream>>>(p);
                    return launched();
                };
                using Kern = void (*)(const ptq::NormParams);
                if (plan.threads > 256) return launch(std::integral_constant<Kern, ptq::ptq_norm_kernel<T, R, 1, true, kBackward, kWhole>>());
                if (plan.rows > 1) return launch(std::integral_constant<Kern, ptq::ptq_norm_kernel<T, R, kRB, false, kBackward, kWhole>>());
                return launch(std::integral_constant<Kern, ptq::ptq_norm_kernel<T, R, 1, false, kBackward, kWhole>>());
            });
        };
        return n.residual_dtype == n.dtype ? go(T()) : go(0.0f);
    });
}

// ---------------------------------------------------------------------------------------------------- conv
ptq_status_t conv_check(const ptq_conv_t *c)
{
    if (!c) return fail(PTQ_ERR_NULL, "the call's description is NULL");
    if (!c->x || !c->weight) return fail(PTQ_ERR_NULL, "x or weight is NULL");
    if (!dtype_ok(c->dtype)) return fail(PTQ_ERR_VALUE, "unknown type %d", c->dtype);
    if (c->batch < 1 || c->length < 1 || c->length > PTQ_MAX_LENGTH || c->channels < 1 || c->channels > PTQ_MAX_CHANNELS || c->taps < 2 || c->taps > 4)
        return fail(PTQ_ERR_SHAPE, "batch %d, length %d, channels %d, taps %d out of range", c->batch, c->length, c->channels, c->taps);
    if (c->flags & ~(PTQ_CONV_SILU | PTQ_SEQ_REVERSE)) return fail(PTQ_ERR_VALUE, "unknown flags %u", c->flags);
    if (!not_negative({c->x_pitch[0], c->x_pitch[1]})) return fail(PTQ_ERR_SHAPE, "a pitch is negative");
    if (!aligned({c->x, c->state}, elem_bytes(c->dtype)) || !aligned({c->weight, c->bias, c->lengths}, 4))
        return fail(PTQ_ERR_ALIGN, "an input is not aligned to its type");
    return PTQ_OK;
}
ptq::ConvParams conv_params(const ptq_conv_t &c, long long segments)
{
    ptq::ConvParams p = {};
    p.x = c.x;
    p.state = c.state;
    p.x_b = c.x_pitch[0];
    p.x_l = c.x_pitch[1];
    p.weight = c.weight;
    p.bias = c.bias;
    p.lengths = c.lengths;
    p.batch = c.batch;
    p.length = c.length;
    p.channels = c.channels;
    p.flags = c.flags;
    p.pieces = static_cast<int>(ceil_div(c.channels, ptq::kConvE));
    p.segment = static_cast<int>(std::max<long long>(ceil_div(c.length, segments), 4));      // no shorter than the taps
    p.segments = static_cast<int>(ceil_div(c.length, p.segment));
    return p;
}
// Forward: segments until the GPU has about 120 thousand threads, but of 8 steps at least (each reads taps - 1 rows again).
ptq::ConvParams conv_forward_params(const ptq_conv_t &c)
{
    const long long threads = static_cast<long long>(c.batch) * ceil_div(c.channels, ptq::kConvE);
    return conv_params(c, std::max(1ll, std::min(ceil_div(kSms * 800, threads), ceil_div(c.length, 8))));
}
// Backward: one wave of CTAs of eight warps, two to an SM, that go over the segments; as many segments as make the longest walk of a warp
// shortest (a segment costs its steps and about 10 more for its start).
struct ConvBackPlan {
    ptq::ConvParams p;
    int blocks, rows;
};
ConvBackPlan conv_back_plan(const ptq_conv_t &c)
{
    ConvBackPlan plan;
    plan.blocks = static_cast<int>(ceil_div(ceil_div(c.channels, ptq::kConvE), 32));
    const long long rows = std::max(1, 2 * kSms / plan.blocks), warps = rows * 8;
    long long best = 1, least = -1;
    for (long long n = 1; n <= 256 && (n == 1 || c.length / n >= 8); ++n) {
        const long long cost = ceil_div(c.batch * n, warps) * (ceil_div(c.length, n) + 10);
        if (least < 0 || cost < least) {
            least = cost;
            best = n;
        }
    }
    plan.p = conv_params(c, best);
    plan.rows = static_cast<int>(std::min(rows, ceil_div(static_cast<long long>(c.batch) * plan.p.segments, 8)));
    return plan;
}
bool conv_whole(const ptq_conv_t &c)
{
    // a piece has kConvE channels: 8 bytes of 16-bit values, 16 of binary32 ones
    return aligned({c.x, c.state}, ptq::kConvE * elem_bytes(c.dtype)) && aligned({c.weight, c.bias}, 16) &&
           multiples({c.x_pitch[0], c.x_pitch[1], c.channels}, ptq::kConvE);
}
template <class Fn>
ptq_status_t with_taps(int taps, Fn fn)
{
    if (taps == 2) return fn(std::integral_constant<int, 2>());
    if (taps == 3) return fn(std::integral_constant<int, 3>());
    return fn(std::integral_constant<int, 4>());
}

}  // namespace

extern "C" {

size_t ptq_scan_workspace_bytes(const ptq_scan_t *s, int backward)
{
    if (!s || s->batch < 1 || s->length < 1 || s->length > PTQ_MAX_LENGTH || s->channels < 1 || s->channels > PTQ_MAX_CHANNELS || s->states < 1 ||
        s->states > PTQ_MAX_STATES || s->groups < 1 || s->channels % s->groups)
        return 0;
    return scan_space(*s, scan_plan(*s, backward != 0), backward != 0).bytes;
}

ptq_status_t ptq_scan_forward(const ptq_scan_t *s, void *y, float *final_state, float *history, void *workspace, size_t workspace_bytes, void *stream)
{
    PTQ_TRY(scan_check(s));
    if (!y) return fail(PTQ_ERR_NULL, "y is NULL");
    if (!aligned({y}, elem_bytes(s->dtype)) || !aligned({final_state, history}, 4)) return fail(PTQ_ERR_ALIGN, "an output is not aligned to its type");
    const ScanPlan plan = scan_plan(*s, false);
    PTQ_TRY(scan_check(plan));
    const ScanSpace space = scan_space(*s, plan, false);
    PTQ_TRY(check_space(workspace, workspace_bytes, space.bytes));
    PTQ_TRY(check_arch());
    ptq::ScanParams p = scan_params(*s, plan);
    p.y = y;
    p.final_state = final_state;
    p.history = history;
    const bool whole = scan_whole(*s) && aligned({y, final_state, history}, 16);
    if (!aligned({y}, 4 * elem_bytes(s->dtype))) p.unit = 1;
    unsigned char *w = static_cast<unsigned char *>(workspace);
    p.slots = reinterpret_cast<float *>(w + space.slots);
    p.sums = reinterpret_cast<float *>(w + space.sums);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return with_type(s->dtype, [&](auto t) {
        using Launch = ScanLaunch<decltype(t)>;
        if (s->length == 1 && !history)        // here only the states and B and C have to be whole
            return Launch::step(p, (s->states <= 2 || s->states % 4 == 0) && aligned({s->A, s->state, final_state}, 16) && p.bc_unit >= std::min(s->states, 4), st);
        if (plan.chunks > 1) PTQ_TRY(Launch::forward(ptq::kScanSum, p, plan.cut(plan.chunks - 1, whole), st));
        return Launch::forward(ptq::kScanForward, p, plan.cut(plan.chunks, whole), st);
    });
}

ptq_status_t ptq_scan_backward(const ptq_scan_t *s, const float *history, const void *dy, const float *dfinal, const ptq_scan_grads_t *g, void *workspace,
                               size_t workspace_bytes, void *stream)
{
    PTQ_TRY(scan_check(s));
    if (!history || !dy || !g) return fail(PTQ_ERR_NULL, "history, dy or grads is NULL");
    if (!g->du || !g->ddelta || !g->dB || !g->dC || !g->dA) return fail(PTQ_ERR_NULL, "du, ddelta, dA, dB or dC is NULL");
    if ((s->z != nullptr) != (g->dz != nullptr)) return fail(PTQ_ERR_NULL, "z and dz are given together");
    if (!aligned({dy, g->du, g->ddelta, g->dz, g->dB, g->dC}, elem_bytes(s->dtype)) ||
        !aligned({history, dfinal, g->dA, g->dD, g->ddelta_bias, g->dstate}, 4))
        return fail(PTQ_ERR_ALIGN, "an argument is not aligned to its type");
    const ScanPlan plan = scan_plan(*s, true);
    PTQ_TRY(scan_check(plan));
    const ScanSpace space = scan_space(*s, plan, true);
    PTQ_TRY(check_space(workspace, workspace_bytes, space.bytes));
    PTQ_TRY(check_arch());
    ptq::ScanParams p = scan_params(*s, plan);
    unsigned char *w = static_cast<unsigned char *>(workspace);
    const auto floats = [&](size_t at) { return reinterpret_cast<float *>(w + at); };
    p.slots = floats(space.slots);
    p.sums = floats(space.sums);
    p.part_A = floats(space.part_A);
    p.part_D = floats(space.part_D);
    p.part_bias = floats(space.part_bias);
    p.part_BC = plan.group_blocks > 1 ? floats(space.part_BC) : nullptr;
    p.dy = dy;
    p.dfinal = dfinal;
    p.kept = history;
    p.du = g->du;
    p.ddelta = g->ddelta;
    p.dz = g->dz;
    p.dB = g->dB;
    p.dC = g->dC;
    p.dstate = g->dstate;
    const bool whole = scan_whole(*s) && aligned({dy, g->du, g->ddelta, g->dz, history, dfinal, g->dstate}, 16);
    if (!aligned({dy, g->du, g->ddelta, g->dz}, 4 * elem_bytes(s->dtype))) p.unit = 1;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return with_type(s->dtype, [&](auto t) {
        using Launch = ScanLaunch<decltype(t)>;
        if (plan.chunks > 1) PTQ_TRY(Launch::forward(ptq::kScanGradSum, p, plan.cut(plan.chunks - 1, whole), st));
        PTQ_TRY(Launch::backward(p, plan.cut(plan.chunks, whole), st));
        return Launch::finish(p, g->dA, g->dD, g->ddelta_bias, st);
    });
}

ptq_status_t ptq_norm_forward(const ptq_norm_t *n, void *y, void *residual_out, void *stream)
{
    PTQ_TRY(norm_check(n));
    if (!y) return fail(PTQ_ERR_NULL, "y is NULL");
    if (!aligned({y}, elem_bytes(n->dtype)) || !aligned({residual_out}, elem_bytes(n->residual_dtype)))
        return fail(PTQ_ERR_ALIGN, "an output is not aligned to its type");
    PTQ_TRY(check_arch());
    ptq::NormParams p = norm_params(*n);
    p.y = y;
    p.residual_out = residual_out;
    const NormPlan plan = norm_plan(*n, false, false);
    p.stages = plan.stages;
    p.at = plan.stage;
    return launch_norm<false>(*n, plan, p, norm_whole(*n) && aligned({y, residual_out}, 16), static_cast<cudaStream_t>(stream));
}

size_t ptq_norm_workspace_bytes(const ptq_norm_t *n)
{
    if (!n || n->rows < 1 || n->cols < 1 || n->cols > PTQ_MAX_NORM_COLS) return 0;
    return padded(static_cast<size_t>(norm_plan(*n, true, n->residual).ctas) * 3 * n->cols * 4);
}

ptq_status_t ptq_norm_backward(const ptq_norm_t *n, const void *dy, const void *dresidual_out, const ptq_norm_grads_t *g, void *workspace,
                               size_t workspace_bytes, void *stream)
{
    PTQ_TRY(norm_check(n));
    if (!dy || !g || !g->dx) return fail(PTQ_ERR_NULL, "dy, grads or dx is NULL");
    if ((n->gate != nullptr) != (g->dgate != nullptr)) return fail(PTQ_ERR_NULL, "gate and dgate are given together");
    if (!aligned({dy, g->dx, g->dgate}, elem_bytes(n->dtype)) || !aligned({dresidual_out, g->dresidual}, elem_bytes(n->residual_dtype)) ||
        !aligned({g->dweight, g->dbias, g->dscale}, 4))
        return fail(PTQ_ERR_ALIGN, "an argument is not aligned to its type");
    PTQ_TRY(check_space(workspace, workspace_bytes, ptq_norm_workspace_bytes(n)));
    PTQ_TRY(check_arch());
    ptq::NormParams p = norm_params(*n);
    p.dy = dy;
    p.dresidual_out = dresidual_out;
    p.dx = g->dx;
    p.dresidual = g->dresidual;
    p.dgate = g->dgate;
    p.sum_scale = g->dscale != nullptr;
    p.part = static_cast<float *>(workspace);
    const NormPlan plan = norm_plan(*n, true, dresidual_out);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    p.stages = plan.stages;
    p.at = plan.stage;
    PTQ_TRY(launch_norm<true>(*n, plan, p, norm_whole(*n) && aligned({dy, dresidual_out, g->dx, g->dresidual, g->dgate}, 16), st));
    if (!g->dweight && !g->dbias && !g->dscale) return PTQ_OK;
    return launch_next(ptq::ptq_norm_finish_kernel, dim3(static_cast<unsigned>(ceil_div(n->cols, 32)), 3), 1024, 0, st, p.part, plan.ctas, n->cols, g->dweight,
                       g->dbias, g->dscale);
}

ptq_status_t ptq_conv_forward(const ptq_conv_t *c, void *y, void *final_state, void *stream)
{
    PTQ_TRY(conv_check(c));
    if (!y) return fail(PTQ_ERR_NULL, "y is NULL");
    if (!aligned({y, final_state}, elem_bytes(c->dtype))) return fail(PTQ_ERR_ALIGN, "an output is not aligned to its type");
    ptq::ConvParams p = conv_forward_params(*c);
    p.y = y;
    p.final_state = final_state;
    const long long ctas = ceil_div(static_cast<long long>(c->batch) * p.segments * p.pieces, 256);
    if (ctas > kMaxGrid) return fail(PTQ_ERR_SHAPE, "the batch is too large for one launch");
    PTQ_TRY(check_arch());
    return with_type(c->dtype, [&](auto t) {
        using T = decltype(t);
        return with_taps(c->taps, [&](auto w) {
            return with_flag(conv_whole(*c) && aligned({y, final_state}, ptq::kConvE * elem_bytes(c->dtype)), [&](auto whole) {
                ptq::ptq_conv_kernel<T, decltype(w)::value, decltype(whole)::value>
                    <<<static_cast<unsigned>(ctas), 256, 0, static_cast<cudaStream_t>(stream)>>>(p);
                return launched();
            });
        });
    });
}

size_t ptq_conv_workspace_bytes(const ptq_conv_t *c)
{
    if (!c || c->batch < 1 || c->length < 1 || c->length > PTQ_MAX_LENGTH || c->channels < 1 || c->channels > PTQ_MAX_CHANNELS || c->taps < 2 ||
        c->taps > 4)
        return 0;
    return padded(static_cast<size_t>(conv_back_plan(*c).rows) * (c->taps + 1) * c->channels * 4);
}

ptq_status_t ptq_conv_backward(const ptq_conv_t *c, const void *dy, const void *dfinal, const ptq_conv_grads_t *g, void *workspace,
                               size_t workspace_bytes, void *stream)
{
    PTQ_TRY(conv_check(c));
    if (!dy || !g || !g->dx || !g->dweight) return fail(PTQ_ERR_NULL, "dy, grads, dx or dweight is NULL");
    if (!aligned({dy, dfinal, g->dx, g->dstate}, elem_bytes(c->dtype)) || !aligned({g->dweight, g->dbias}, 4))
        return fail(PTQ_ERR_ALIGN, "an argument is not aligned to its type");
    PTQ_TRY(check_space(workspace, workspace_bytes, ptq_conv_workspace_bytes(c)));
    PTQ_TRY(check_arch());
    const ConvBackPlan plan = conv_back_plan(*c);
    ptq::ConvParams p = plan.p;
    p.dy = dy;
    p.dfinal = dfinal;
    p.dx = g->dx;
    p.dstate = g->dstate;
    p.part = static_cast<float *>(workspace);
    const int rows = plan.rows;
    const dim3 grid(static_cast<unsigned>(plan.blocks), static_cast<unsigned>(rows));
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    PTQ_TRY(with_type(c->dtype, [&](auto t) {
        using T = decltype(t);
        return with_taps(c->taps, [&](auto w) {
            return with_flag(conv_whole(*c) && aligned({dy, dfinal, g->dx, g->dstate}, ptq::kConvE * elem_bytes(c->dtype)), [&](auto whole) {
                ptq::ptq_conv_backward_kernel<T, decltype(w)::value, decltype(whole)::value><<<grid, 256, 0, st>>>(p);
                return launched();
            });
        });
    }));
    return launch_next(ptq::ptq_conv_finish_kernel, dim3(static_cast<unsigned>(ceil_div(c->channels, 32)), static_cast<unsigned>(c->taps + 1)), 1024, 0, st,
                       p.part, rows, c->channels, c->taps, g->dweight, g->dbias);
}

}  // extern "C"
