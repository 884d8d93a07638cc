// Entry points of the block norm (see tdx.h).
#include "layer_host.cuh"

#include "norm_kernels.cuh"

namespace {

constexpr int64_t kNormMostChannels = 1 << 20;

struct NormPlan { int vec, nv, warps, sets; int64_t grid; size_t smem; };

// The widest access that every row and parameter of the call allows and that divides a group.
int norm_vector(const tdx_norm_args& a, bool back) {
    const int64_t el = elem_bytes(a.dtype);
    Widest w(16);
    auto rows = [&](const void* p, int64_t ld) { if (p) { w.ptr(p); w.stride(ld, el); } };
    w.stride(a.channels, el);
    if (a.norm_in && a.group) w.stride(a.group, el);
    rows(a.x, a.ld_x); rows(a.gate, a.ld_gate); rows(a.residual, a.ld_residual);
    if (back) {
        rows(a.dsum, a.ld_dsum); rows(a.dy, a.ld_dy); rows(a.dx, a.ld_dx); rows(a.dgate, a.ld_dgate); rows(a.dresidual, a.ld_dresidual);
    } else {
        rows(a.sum, a.ld_sum); rows(a.y, a.ld_y);
    }
    const int vec = static_cast<int>(std::max<int64_t>(1, w.bytes / el));
    const size_t align = 4 * static_cast<size_t>(std::min(vec, 4));
    if (misaligned(a.weight_in, align) || misaligned(a.scale, align) || misaligned(a.weight_out, align)) return 1;
    // kernels exist for 16-byte accesses, pairs of bf16, and single elements
    return vec * el == 16 ? vec : el == 2 && vec >= 2 ? 2 : 1;
}

// The most sets of rows (of one block of threads, or of one row's share of a block) that a backward pass is cut into, whatever the
// alignment is: 16 channels a thread at most, so so many warps a row at least, and two blocks of eight warps an SM at most.
int64_t norm_most_sets(int64_t rows, int64_t channels, int sm_count) {
    int64_t warps = 1;
    while (warps < 8 && warps * 32 * 16 < channels) warps *= 2;
    return std::min<int64_t>(rows + 7, 2 * sm_count * (8 / warps));
}

// Channels a thread: 8 (bf16) or 4 where 512 threads then hold a row, so that most loads are in flight at once; up to 16 for wider rows.
void plan_norm(const tdx_norm_args& a, int vec, int sm_count, bool back, tdx::NormParams* p, NormPlan* plan) {
    plan->vec = vec;
    p->vectors = static_cast<int>(a.channels / vec);
    int nv = vec == 8 ? 1 : vec == 4 ? 1 : vec == 2 ? 2 : 4;
    const int most = 16 / vec;
    while (nv < most && ceil_div(p->vectors, nv) > tdx::kNormThreads) nv *= 2;
    if (vec <= 2 && nv > (vec == 2 ? 2 : 4)) nv = most;
    plan->nv = ceil_div(p->vectors, nv) > tdx::kNormThreads ? 0 : nv;
    const int64_t group = a.norm_in && a.group ? a.group : a.channels;
    p->group = static_cast<int>(group);
    p->group_vectors = static_cast<int>(group / vec);
    const bool power = p->group_vectors <= 32 && (p->group_vectors & (p->group_vectors - 1)) == 0;
    p->group_lanes = group == a.channels ? 0 : power ? p->group_vectors : -1;
    if (plan->nv == 0) {
        plan->warps = tdx::kNormThreads / 32;
        plan->sets = 1;
        plan->smem = sizeof(float) * (tdx::kNormShared + 2 * (a.channels / group));
    } else {
        int warps = 1;
        while (warps * 32 * nv < p->vectors) warps *= 2;
        plan->warps = warps;
        plan->sets = std::max(1, 8 / warps);
        plan->smem = sizeof(float) * plan->sets * (tdx::kNormShared + (p->group_lanes < 0 ? p->vectors : 0));
    }
    p->warps = plan->warps;
    const int64_t blocks = std::max<int64_t>(1, ceil_div(a.rows, plan->sets));
    const int64_t resident = static_cast<int64_t>(sm_count) * (back ? std::max(1, 16 / (plan->warps * plan->sets)) : 64 / (plan->warps * plan->sets));
    plan->grid = std::min(blocks, std::max<int64_t>(1, resident));
}

int check_norm(const tdx_norm_args* args, bool back, tdx::NormParams* p) {
    if (args == nullptr) return fail(TDX_ERR_INVALID_ARG, "args is NULL");
    const tdx_norm_args& a = *args;
    if (a.rows < 0 || a.channels < 0 || a.group < 0) return fail(TDX_ERR_INVALID_ARG, "negative size");
    if (a.dtype != TDX_F32 && a.dtype != TDX_BF16) return fail(TDX_ERR_INVALID_ARG, "unknown dtype %d", a.dtype);
    if (a.norm_in != 0 && a.norm_in != 1) return fail(TDX_ERR_INVALID_ARG, "norm_in must be 0 or 1");
    if (a.channels > kNormMostChannels) return fail(TDX_ERR_UNSUPPORTED, "more than 2^20 channels");
    if (a.norm_in && a.group > 0 && a.channels % a.group) return fail(TDX_ERR_INVALID_ARG, "%lld channels do not divide into groups of %lld", (long long)a.channels, (long long)a.group);
    if (a.norm_in && a.group > 0 && a.group < a.channels && a.channels > tdx::kNormThreads * 16 && a.channels / a.group > 4096)
        return fail(TDX_ERR_UNSUPPORTED, "more than 4096 groups in rows of more than 8192 channels");
    if (!(a.eps >= 0.0f)) return fail(TDX_ERR_INVALID_ARG, "eps must not be negative");
    const size_t el = elem_bytes(a.dtype);
    const bool any = a.rows > 0 && a.channels > 0;
    TDX_TRY(check_tensor("x", a.x, any, el, a.ld_x, a.channels));
    TDX_TRY(check_tensor("gate", a.gate, false, el, a.ld_gate, a.channels));
    TDX_TRY(check_tensor("residual", a.residual, false, el, a.ld_residual, a.channels));
    TDX_TRY(check_tensor("weight_in", a.weight_in, false, 4));
    TDX_TRY(check_tensor("scale", a.scale, false, 4));
    TDX_TRY(check_tensor("weight_out", a.weight_out, false, 4));
    std::memset(p, 0, sizeof *p);
    if (back) {
        if (any && a.dsum == nullptr && a.dy == nullptr) return fail(TDX_ERR_INVALID_ARG, "neither dsum nor dy is given");
        TDX_TRY(check_tensor("dsum", a.dsum, false, el, a.ld_dsum, a.channels));
        TDX_TRY(check_tensor("dy", a.dy, false, el, a.ld_dy, a.channels));
        TDX_TRY(check_tensor("dx", a.dx, any, el, a.ld_dx, a.channels));
        TDX_TRY(check_tensor("dgate", a.dgate, any && a.gate, el, a.ld_dgate, a.channels));
        TDX_TRY(check_tensor("dresidual", a.dresidual, any && a.residual, el, a.ld_dresidual, a.channels));
        TDX_TRY(check_tensor("dweight_in", a.dweight_in, false, 4));
        TDX_TRY(check_tensor("dscale", a.dscale, false, 4));
        TDX_TRY(check_tensor("dweight_out", a.dweight_out, false, 4));
        if (a.dweight_in && !a.norm_in) return fail(TDX_ERR_INVALID_ARG, "dweight_in is given, but x has no norm");
        p->dsum = a.dsum; p->ld_dsum = a.ld_dsum; p->dy = a.dy; p->ld_dy = a.ld_dy;
        p->dx = a.dx; p->ld_dx = a.ld_dx; p->dgate = a.gate ? a.dgate : nullptr; p->ld_dgate = a.ld_dgate;
        p->dresidual = a.residual ? a.dresidual : nullptr; p->ld_dresidual = a.ld_dresidual;
        p->want_in = a.dweight_in != nullptr; p->want_scale = a.dscale != nullptr; p->want_out = a.dweight_out != nullptr;
    } else {
        if (any && a.sum == nullptr && a.y == nullptr) return fail(TDX_ERR_INVALID_ARG, "neither sum nor y is given");
        TDX_TRY(check_tensor("sum", a.sum, false, el, a.ld_sum, a.channels));
        TDX_TRY(check_tensor("y", a.y, false, el, a.ld_y, a.channels));
        p->sum = a.sum; p->ld_sum = a.ld_sum; p->y = a.y; p->ld_y = a.ld_y;
    }
    p->rows = a.rows; p->channels = static_cast<int>(a.channels); p->norm_in = a.norm_in; p->eps = a.eps;
    const int64_t group = a.norm_in && a.group ? a.group : std::max<int64_t>(1, a.channels);
    p->inv_group = 1.0f / static_cast<float>(group);
    p->inv_channels = 1.0f / static_cast<float>(std::max<int64_t>(1, a.channels));
    p->x = a.x; p->ld_x = a.ld_x; p->gate = a.gate; p->ld_gate = a.ld_gate; p->residual = a.residual; p->ld_residual = a.ld_residual;
    p->weight_in = a.weight_in; p->scale = a.scale; p->weight_out = a.weight_out;
    return TDX_OK;
}

template <typename T, int VEC, int NV, int HAS>
int launch_norm_has(bool back, const tdx::NormParams& p, const NormPlan& plan, cudaStream_t st) {
    const int threads = plan.warps * plan.sets * 32;
    return back ? launch_seq(tdx::norm_bwd_kernel<T, VEC, NV, HAS>, plan.grid, 1, threads, plan.smem, st, p)
                : launch_seq(tdx::norm_fwd_kernel<T, VEC, NV, HAS>, plan.grid, 1, threads, plan.smem, st, p);
}
// Kernels of their own for what calls usually have, where rows are 16-byte aligned and up to 512 threads hold them with one access each:
// heads' norm with gate; stream's sum and next norm, with and without the block's norm, its gate and its scale; a norm alone.
template <typename T, int VEC, int NV>
int launch_norm(bool back, const tdx::NormParams& p, const NormPlan& plan, cudaStream_t st) {
    if constexpr (VEC * sizeof(T) == 16 && NV == 1) {
        const int has = (p.norm_in ? tdx::kNormIn : 0) | (p.gate ? tdx::kNormGate : 0) | (p.scale ? tdx::kNormScale : 0) | (p.residual ? tdx::kNormResidual : 0) |
                        ((back ? p.dy : p.y) ? tdx::kNormY : 0) | ((back ? p.dsum : p.sum) ? tdx::kNormSum : 0);
        constexpr int kHeads = tdx::kNormIn | tdx::kNormGate | tdx::kNormSum, kStream = tdx::kNormResidual | tdx::kNormY | tdx::kNormSum;
        switch (has) {
            case kHeads: return launch_norm_has<T, VEC, NV, kHeads>(back, p, plan, st);
            case kStream: return launch_norm_has<T, VEC, NV, kStream>(back, p, plan, st);
            case kStream | tdx::kNormIn: return launch_norm_has<T, VEC, NV, kStream | tdx::kNormIn>(back, p, plan, st);
            case kStream | tdx::kNormIn | tdx::kNormScale: return launch_norm_has<T, VEC, NV, kStream | tdx::kNormIn | tdx::kNormScale>(back, p, plan, st);
            case kStream | kHeads | tdx::kNormScale: return launch_norm_has<T, VEC, NV, kStream | kHeads | tdx::kNormScale>(back, p, plan, st);
            case tdx::kNormY: return launch_norm_has<T, VEC, NV, static_cast<int>(tdx::kNormY)>(back, p, plan, st);
            default: break;
        }
    }
    return launch_norm_has<T, VEC, NV, -1>(back, p, plan, st);
}
template <typename T>
int launch_norm_wide(bool back, const tdx::NormParams& p, const NormPlan& plan, cudaStream_t st) {
    return back ? launch_seq(tdx::norm_bwd_wide_kernel<T>, plan.grid, 1, tdx::kNormThreads, plan.smem, st, p)
                : launch_seq(tdx::norm_fwd_wide_kernel<T>, plan.grid, 1, tdx::kNormThreads, plan.smem, st, p);
}
int run_norm(const tdx_norm_args& a, bool back, const tdx::NormParams& p, const NormPlan& plan, cudaStream_t st) {
    typedef __nv_bfloat16 bf16;
    if (plan.nv == 0) return a.dtype == TDX_F32 ? launch_norm_wide<float>(back, p, plan, st) : launch_norm_wide<bf16>(back, p, plan, st);
    switch (plan.vec * 100 + plan.nv) {
        case 801: return launch_norm<bf16, 8, 1>(back, p, plan, st);
        case 802: return launch_norm<bf16, 8, 2>(back, p, plan, st);
        case 202: return launch_norm<bf16, 2, 2>(back, p, plan, st);
        case 208: return launch_norm<bf16, 2, 8>(back, p, plan, st);
        case 401: return launch_norm<float, 4, 1>(back, p, plan, st);
        case 402: return launch_norm<float, 4, 2>(back, p, plan, st);
        case 404: return launch_norm<float, 4, 4>(back, p, plan, st);
        case 104: return a.dtype == TDX_F32 ? launch_norm<float, 1, 4>(back, p, plan, st) : launch_norm<bf16, 1, 4>(back, p, plan, st);
        default: return a.dtype == TDX_F32 ? launch_norm<float, 1, 16>(back, p, plan, st) : launch_norm<bf16, 1, 16>(back, p, plan, st);
    }
}

size_t norm_workspace_bytes(int64_t rows, int64_t channels, int sm_count) {
    return round_256(static_cast<size_t>(norm_most_sets(rows, channels, sm_count)) * 3 * channels * sizeof(float));
}

}  // namespace

extern "C" {

int tdx_block_norm(const tdx_norm_args* args, void* stream) {
    tdx::NormParams p;
    TDX_TRY(check_norm(args, false, &p));
    if (p.rows == 0 || p.channels == 0) return TDX_OK;
    tdx_host::Device dev;
    TDX_TRY(tdx_host::get_device(&dev));
    NormPlan plan;
    plan_norm(*args, norm_vector(*args, false), dev.sm_count, false, &p, &plan);
    return run_norm(*args, false, p, plan, static_cast<cudaStream_t>(stream));
}

int tdx_block_norm_bwd(const tdx_norm_args* args, void* stream) {
    tdx::NormParams p;
    TDX_TRY(check_norm(args, true, &p));
    if (p.channels == 0) return TDX_OK;
    const bool sums = p.want_in || p.want_scale || p.want_out;
    if (p.rows == 0 && !sums) return TDX_OK;
    tdx_host::Device dev;
    TDX_TRY(tdx_host::get_device(&dev));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (p.rows == 0) {
        for (float* out : {args->dweight_in, args->dscale, args->dweight_out})
            if (out) TDX_CUDA(cudaMemsetAsync(out, 0, p.channels * sizeof(float), st));
        return TDX_OK;
    }
    TDX_TRY(check_workspace(args->workspace, args->workspace_bytes, norm_workspace_bytes(p.rows, p.channels, dev.sm_count)));
    p.partial = static_cast<float*>(args->workspace);
    NormPlan plan;
    plan_norm(*args, norm_vector(*args, true), dev.sm_count, true, &p, &plan);
    TDX_TRY(run_norm(*args, true, p, plan, st));
    if (!sums) return TDX_OK;
    // sets behind the last row have written zeros
    return launch_seq(tdx::norm_join_kernel, ceil_div(p.channels, 32), 3, 256, 0, st, p.channels, static_cast<long long>(plan.grid * plan.sets),
                      static_cast<const float*>(p.partial), args->dweight_in, args->dscale, args->dweight_out);
}

int tdx_block_norm_workspace_size(const tdx_norm_args* args, size_t* bytes) {
    if (args == nullptr || bytes == nullptr) return fail(TDX_ERR_INVALID_ARG, "NULL argument");
    if (args->rows < 0 || args->channels < 0) return fail(TDX_ERR_INVALID_ARG, "negative size");
    if (args->channels > kNormMostChannels) return fail(TDX_ERR_UNSUPPORTED, "more than 2^20 channels");
    *bytes = norm_workspace_bytes(args->rows, args->channels, sm_count_or_default());
    return TDX_OK;
}

}  // extern "C"
