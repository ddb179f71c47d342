// Host side of the C ABI declared in include/ptq_heads.h: argument checks, how the sequences are cut, kernel launches.
#include "../../include/ptq_heads.h"

#include <algorithm>

#include "ptq_heads_finish.cuh"
#include "ptq_heads_launch.cuh"

namespace {

using namespace ptq_host;

static_assert(PTQ_HEADS_SOFTPLUS == ptq::kHeadsSoftplus && PTQ_SEQ_REVERSE == ptq::kHeadsReverse && PTQ_HEADS_UNSCALED == ptq::kHeadsUnscaled &&
              PTQ_HEADS_HISTORY == ptq::kHeadSteps, "the kernels' constants are the header's");

bool dims_ok(const ptq_heads_t &s)
{
    return s.batch >= 1 && s.length >= 1 && s.length <= PTQ_MAX_LENGTH && s.heads >= 1 && s.heads <= PTQ_MAX_HEADS && s.cols >= 1 &&
           s.cols <= PTQ_MAX_HEAD_COLS && s.states >= 1 && s.states <= PTQ_MAX_HEAD_STATES && s.groups >= 1 && s.heads % s.groups == 0;
}
ptq_status_t heads_check(const ptq_heads_t *s)
{
    if (!s) return fail(PTQ_ERR_NULL, "the call's description is NULL");
    if (!s->u || !s->B || !s->C || !s->A) return fail(PTQ_ERR_NULL, "u, B, C or A is NULL");
    if (!dtype_ok(s->dtype)) return fail(PTQ_ERR_VALUE, "unknown type %d", s->dtype);
    if (!dims_ok(*s))
        return fail(PTQ_ERR_SHAPE, "batch %d, length %d, heads %d, cols %d, states %d, groups %d out of range", s->batch, s->length, s->heads, s->cols,
                    s->states, s->groups);
    if (s->flags & ~(PTQ_HEADS_SOFTPLUS | PTQ_SEQ_REVERSE | PTQ_HEADS_UNSCALED)) return fail(PTQ_ERR_VALUE, "unknown flags %u", s->flags);
    if (!s->delta && s->delta_bias) return fail(PTQ_ERR_NULL, "delta_bias without delta");
    for (int k = 0; k < 3; ++k)
        if (!not_negative({s->u_pitch[k], s->B_pitch[k], s->C_pitch[k], s->delta ? s->delta_pitch[k] : 0})) return fail(PTQ_ERR_SHAPE, "a pitch is negative");
    if (!aligned({s->u, s->delta, s->B, s->C}, elem_bytes(s->dtype)) || !aligned({s->A, s->D, s->delta_bias, s->state, s->lengths}, 4))
        return fail(PTQ_ERR_ALIGN, "an input is not aligned to its type");
    return PTQ_OK;
}

int col_tiles(const ptq_heads_t &s) { return static_cast<int>(ceil_div(s.cols, ptq::kHeadCols)); }
int chunks_of(const ptq_heads_t &s) { return static_cast<int>(ceil_div(s.length, ptq::kHeadSteps)); }

// Sequences are cut into segments where there are too few heads to fill the GPU: the states of all segments but the last are summed first
// and joined.  A chunk of the forward pass costs 1.5 here, of the sums half of that, of the backward pass 8 (its sums 1), the join 6 and
// some per segment (in about two microseconds).  An SM has one CTA where activations are binary32 and of the backward pass with
// more than 64 states, else two; the last of several rounds is taken to be half full.  2 x 20011 x 16 heads (bfloat16, 128 states) in 4, 9
// and 18 segments: 554, 357, 373 us; training 8 x 784 x 6 heads (binary32, 16 states), the backward pass in 1, 3 and 13: 280, 212, 190;
// 1 x 197 x 6 heads (binary16, 64 states) in 1 and 4: 14.4 and 18.3.
struct HeadsPlan {
    int segments, segment_chunks;
};
HeadsPlan heads_plan(const ptq_heads_t &s, bool backward)
{
    const long long base = static_cast<long long>(s.batch) * s.heads * col_tiles(s), chunks = chunks_of(s);
    const bool two = s.dtype != PTQ_F32 && (!backward || s.states <= 64);
    const double resident = two ? 2 * kSms : kSms, unit = backward ? 8.0 : 1.5, sums = backward ? 1.0 : 0.75;
    // a padded batch holds about half the steps
    const double filled = s.lengths ? 0.5 : 1.0;
    long long best = 1;
    double least = -1.0;
    for (long long n = 1; n <= chunks && n <= 256 && base * n <= 16 * kSms; ++n) {
        const long long per = ceil_div(chunks, n);
        const double full = filled * static_cast<double>(base * n) / resident, waves = std::max(1.0, 0.5 * (full + std::ceil(full - 0.02)));
        const double cost = waves * per * unit + (n > 1 ? waves * per * sums + 6.0 + 0.1 * n : 0.0);
        if (least < 0.0 || cost < least) {
            least = cost;
            best = n;
        }
    }
    HeadsPlan p;
    p.segment_chunks = static_cast<int>(ceil_div(chunks, best));
    p.segments = static_cast<int>(ceil_div(chunks, p.segment_chunks));
    return p;
}

size_t times(std::initializer_list<size_t> v)          // SIZE_MAX / 4 where it is more
{
    size_t r = 1;
    for (size_t x : v)
        if (__builtin_mul_overflow(r, x, &r) || r > SIZE_MAX / 4) return SIZE_MAX / 4;
    return r;
}
struct HeadsSpace {
    size_t slots, logs, part_B, part_C, part_dt, part_D, shares, bytes;
};
HeadsSpace heads_space(const ptq_heads_t &s, const HeadsPlan &plan, bool backward)
{
    HeadsSpace w = {};
    size_t at = 0;
    const auto take = [&](size_t floats) {
        const size_t here = at;
        const size_t bytes = times({floats, 4});
        at = at + bytes > SIZE_MAX / 4 ? SIZE_MAX / 4 : at + padded(bytes);
        return here;
    };
    const size_t heads = times({static_cast<size_t>(s.batch), static_cast<size_t>(s.heads)}), tiles = col_tiles(s), segments = plan.segments;
    if (segments > 1) {
        w.slots = take(times({heads, segments, static_cast<size_t>(s.cols), static_cast<size_t>(s.states)}));
        w.logs = take(times({heads, segments}));
    }
    if (backward) {
        const size_t rows = times({heads, tiles, static_cast<size_t>(s.length)});
        w.part_B = take(times({rows, static_cast<size_t>(s.states)}));
        w.part_C = take(times({rows, static_cast<size_t>(s.states)}));
        w.part_dt = take(times({rows, 2}));
        w.part_D = take(times({heads, tiles, segments}));
        w.shares = take(times({heads, 2}));
    }
    w.bytes = at;
    return w;
}
ptq_status_t grid_check(const ptq_heads_t &s, const HeadsPlan &plan)
{
    if (static_cast<long long>(s.batch) * s.heads * col_tiles(s) * plan.segments > kMaxGrid) return fail(PTQ_ERR_SHAPE, "the batch is too large for one launch");
    return PTQ_OK;
}

ptq::HeadParams heads_params(const ptq_heads_t &s, const HeadsPlan &plan, const void *dy)
{
    ptq::HeadParams p = {};
    p.u = s.u;
    p.delta = s.delta;
    p.B = s.B;
    p.C = s.C;
    p.dy = dy;
    p.u_b = s.u_pitch[0];
    p.u_l = s.u_pitch[1];
    p.u_h = s.u_pitch[2];
    p.B_b = s.B_pitch[0];
    p.B_l = s.B_pitch[1];
    p.B_g = s.B_pitch[2];
    p.C_b = s.C_pitch[0];
    p.C_l = s.C_pitch[1];
    p.C_g = s.C_pitch[2];
    if (s.delta) {
        p.delta_b = s.delta_pitch[0];
        p.delta_l = s.delta_pitch[1];
        p.delta_h = s.delta_pitch[2];
    }
    p.A = s.A;
    p.D = s.D;
    p.delta_bias = s.delta_bias;
    p.state = s.state;
    p.lengths = s.lengths;
    p.batch = s.batch;
    p.length = s.length;
    p.heads = s.heads;
    p.cols = s.cols;
    p.states = s.states;
    p.groups = s.groups;
    p.group_heads = s.heads / s.groups;
    p.col_tiles = col_tiles(s);
    p.chunks = chunks_of(s);
    p.segments = plan.segments;
    p.segment_chunks = plan.segment_chunks;
    p.flags = s.flags;
    const int e = elem_bytes(s.dtype);
    p.unit = e;
    for (int bytes : {16, 8, 4})
        if (p.unit == e && bytes > e && aligned({s.u, s.B, s.C, dy}, bytes) &&
            multiples({p.u_b, p.u_l, p.u_h, p.B_b, p.B_l, p.B_g, p.C_b, p.C_l, p.C_g, s.cols, s.states}, bytes / e))
            p.unit = bytes;
    return p;
}

template <class Fn>
ptq_status_t with_launch(int dtype, Fn fn)
{
    return with_type(dtype, [&](auto t) { return fn(HeadsLaunch<decltype(t)>()); });
}

ptq_status_t fold(const ptq::HeadParams &p, const float *start, int grad, cudaStream_t stream)
{
    const int64_t heads = static_cast<int64_t>(p.batch) * p.heads, size = static_cast<int64_t>(p.cols) * p.states;
    const long long ctas = ceil_div(heads * size, 256);
    return launch_next(ptq::ptq_heads_fold_kernel, dim3(static_cast<unsigned>(ctas)), 256, 0, stream, p.slots, p.logs, start, heads, p.segments, size, grad);
}

}  // namespace

extern "C" {

size_t ptq_heads_workspace_bytes(const ptq_heads_t *s, int backward)
{
    if (!s || !dims_ok(*s)) return 0;
    return heads_space(*s, heads_plan(*s, backward != 0), backward != 0).bytes;
}

ptq_status_t ptq_heads_forward(const ptq_heads_t *s, void *y, float *final_state, float *history, void *workspace, size_t workspace_bytes, void *stream)
{
    PTQ_TRY(heads_check(s));
    if (!y) return fail(PTQ_ERR_NULL, "y is NULL");
    const int e = elem_bytes(s->dtype);
    if (!aligned({y}, e) || !aligned({final_state, history}, 4)) return fail(PTQ_ERR_ALIGN, "an output is not aligned to its type");
    const HeadsPlan plan = heads_plan(*s, false);
    PTQ_TRY(grid_check(*s, plan));
    const HeadsSpace space = heads_space(*s, plan, false);
    PTQ_TRY(check_space(workspace, workspace_bytes, space.bytes));
    PTQ_TRY(check_arch());
    ptq::HeadParams p = heads_params(*s, plan, nullptr);
    p.y = y;
    p.final_state = final_state;
    p.history = history;
    p.out_unit = aligned({y}, 2 * e) && s->cols % 2 == 0 ? 2 * e : e;
    unsigned char *w = static_cast<unsigned char *>(workspace);
    p.slots = reinterpret_cast<float *>(w + space.slots);
    p.logs = reinterpret_cast<float *>(w + space.logs);
    p.share = s->dtype == PTQ_F16 || static_cast<long long>(s->batch) * s->heads * p.col_tiles * p.segments <= kSms;
    const bool whole = p.unit == 16 && aligned({y}, 16) && aligned({s->state, final_state, history}, 8);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return with_launch(s->dtype, [&](auto launch) -> ptq_status_t {
        if (s->length == 1 && !history) return launch.step(p, s->states % 4 == 0 && aligned({s->state, final_state}, 16), st);
        if (plan.segments > 1) {
            PTQ_TRY(launch.chunks(ptq::kHeadSum, p, whole, false, st));
            PTQ_TRY(fold(p, s->state, 0, st));
        }
        return launch.chunks(ptq::kHeadForward, p, whole, plan.segments > 1, st);
    });
}

ptq_status_t ptq_heads_backward(const ptq_heads_t *s, const float *history, const void *dy, const float *dfinal, const ptq_heads_grads_t *g, void *workspace,
                                size_t workspace_bytes, void *stream)
{
    PTQ_TRY(heads_check(s));
    if (!history || !dy || !g) return fail(PTQ_ERR_NULL, "history, dy or grads is NULL");
    if (!g->du || !g->dB || !g->dC || !g->dA) return fail(PTQ_ERR_NULL, "du, dB, dC or dA is NULL");
    if ((s->delta != nullptr) != (g->ddelta != nullptr)) return fail(PTQ_ERR_NULL, "delta and ddelta are given together");
    const int e = elem_bytes(s->dtype);
    if (!aligned({dy, g->du, g->ddelta, g->dB, g->dC}, e) || !aligned({history, dfinal, g->dA, g->dD, g->ddelta_bias, g->dstate}, 4))
        return fail(PTQ_ERR_ALIGN, "an argument is not aligned to its type");
    const HeadsPlan plan = heads_plan(*s, true);
    PTQ_TRY(grid_check(*s, plan));
    const HeadsSpace space = heads_space(*s, plan, true);
    PTQ_TRY(check_space(workspace, workspace_bytes, space.bytes));
    const bool fours = s->states % 4 == 0 && aligned({g->dB, g->dC}, 4 * e);
    const int64_t sums = ceil_div(static_cast<int64_t>(s->batch) * s->length * s->groups * (s->states / (fours ? 4 : 1)), 256);
    const int64_t ctas = std::max(sums, static_cast<int64_t>(s->batch) * s->heads);
    if (ctas > kMaxGrid) return fail(PTQ_ERR_SHAPE, "the batch is too large for one launch");
    PTQ_TRY(check_arch());
    ptq::HeadParams p = heads_params(*s, plan, dy);
    unsigned char *w = static_cast<unsigned char *>(workspace);
    const auto floats = [&](size_t at) { return reinterpret_cast<float *>(w + at); };
    p.slots = floats(space.slots);
    p.logs = floats(space.logs);
    p.part_B = floats(space.part_B);
    p.part_C = floats(space.part_C);
    p.part_dt = reinterpret_cast<float2 *>(floats(space.part_dt));
    p.part_D = floats(space.part_D);
    float2 *shares = reinterpret_cast<float2 *>(floats(space.shares));
    p.kept = history;
    p.dfinal = dfinal;
    p.du = g->du;
    p.final_state = g->dstate;
    p.out_unit = aligned({g->du}, 2 * e) && s->cols % 2 == 0 ? 2 * e : e;
    const bool whole = p.unit == 16 && aligned({g->du}, 2 * e) && aligned({history, dfinal, g->dstate}, 8);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return with_type(s->dtype, [&](auto t) -> ptq_status_t {
        using T = decltype(t);
        using Launch = HeadsLaunch<T>;
        if (plan.segments > 1) {
            PTQ_TRY(Launch::chunks(ptq::kHeadGradSum, p, whole, false, st));
            PTQ_TRY(fold(p, dfinal, 1, st));
        }
        PTQ_TRY(Launch::backward(p, whole, plan.segments > 1, st));
        PTQ_TRY(launch_next(fours ? ptq::ptq_heads_finish_kernel<T, 4> : ptq::ptq_heads_finish_kernel<T, 1>, dim3(static_cast<unsigned>(ctas), 3), 256, 0, st, p,
                            static_cast<T *>(g->dB), static_cast<T *>(g->dC), static_cast<T *>(g->ddelta), shares));
        return launch_next(ptq::ptq_heads_finish_sums_kernel, dim3(static_cast<unsigned>(s->heads)), 128, 0, st, p, shares, g->dA, g->ddelta_bias, g->dD);
    });
}

}  // extern "C"
