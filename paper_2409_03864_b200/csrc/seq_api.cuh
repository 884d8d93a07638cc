// Entry points of the sequence operators: causal convolution, selective scan and products with 4-bit weights (see tdx.h).
// Part of the translation unit tdx_api.cu.
#pragma once
#include "conv1d_kernels.cuh"
#include "scan_kernels.cuh"
#include "seq_host.cuh"
#include "w4_kernels.cuh"

namespace {

// ------------------------------------------------------------------ causal convolution
enum ConvPass { kConvForward, kConvBackward, kConvStep };

int64_t conv_dense_pieces(int64_t max_len, int64_t piece) { return std::max<int64_t>(1, ceil_div(max_len, piece)); }

int check_conv1d(const tdx_conv1d_args* a, ConvPass pass, tdx::Conv1dParams* p) {
    if (a == nullptr) return fail(TDX_ERR_INVALID_ARG, "args is NULL");
    const bool step = pass == kConvStep, back = pass == kConvBackward;
    TDX_TRY(check_sequences(a->batch, a->max_len, a->rows, a->channels, a->dtype, a->seq_offsets, step));
    if (a->width < 1 || a->width > 8) return fail(TDX_ERR_INVALID_ARG, "width %d is not in 1 .. 8", a->width);
    if (a->silu != 0 && a->silu != 1) return fail(TDX_ERR_INVALID_ARG, "silu must be 0 or 1");
    const bool stateful = a->width > 1;
    const int64_t per_slot = (a->width - 1) * a->channels;
    int64_t stride = a->state_stride;
    TDX_TRY(check_states(stateful && (a->state_in || a->state_out || (back && (a->dstate_in || a->dstate_out))), a->batch, per_slot, &stride,
                         a->slots, a->n_slots));
    if (step && misaligned(a->slots, 4)) return fail(TDX_ERR_ALIGNMENT, "slots is not aligned to its elements");
    const size_t el = elem_bytes(a->dtype);
    const bool any = a->channels > 0 && a->batch > 0, rows = any && (step || a->rows > 0);
    TDX_TRY(check_tensor("x", a->x, rows, el, a->ld_x, a->channels));
    TDX_TRY(check_tensor("weight", a->weight, any, 4));
    TDX_TRY(check_tensor("bias", a->bias, false, 4));
    TDX_TRY(check_tensor("state_in", a->state_in, step && any && stateful, el));
    if (back) {
        TDX_TRY(check_tensor("dy", a->dy, rows, el, a->ld_dy, a->channels));
        TDX_TRY(check_tensor("dx", a->dx, rows, el, a->ld_dx, a->channels));
        TDX_TRY(check_tensor("dweight", a->dweight, false, 4));
        TDX_TRY(check_tensor("dbias", a->dbias, false, 4));
        TDX_TRY(check_tensor("dstate_out", a->dstate_out, false, el));
        TDX_TRY(check_tensor("dstate_in", a->dstate_in, false, el));
    } else {
        TDX_TRY(check_tensor("y", a->y, rows, el, a->ld_y, a->channels));
        TDX_TRY(check_tensor("state_out", a->state_out, step && any && stateful, el));
    }
    std::memset(p, 0, sizeof *p);
    p->batch = a->batch; p->max_len = a->max_len; p->rows = a->rows; p->channels = a->channels;
    p->width = a->width; p->silu = a->silu;
    p->x = a->x; p->ld_x = a->ld_x; p->weight = a->weight; p->bias = a->bias; p->y = a->y; p->ld_y = a->ld_y;
    p->weight_aligned = !misaligned(a->weight, 16);
    // without states there are no slots to stay below: a step's slots then only tell which rows are padding
    p->offsets = a->seq_offsets; p->slots = a->slots; p->n_slots = stateful ? a->n_slots : INT64_MAX; p->state_stride = stride;
    p->state_in = stateful ? a->state_in : nullptr;
    p->state_out = stateful ? a->state_out : nullptr;
    if (back) {
        p->dy = a->dy; p->ld_dy = a->ld_dy; p->dx = a->dx; p->ld_dx = a->ld_dx; p->dweight = a->dweight; p->dbias = a->dbias;
        p->dstate_out = stateful ? a->dstate_out : nullptr;
        p->dstate_in = stateful ? a->dstate_in : nullptr;
    }
    return TDX_OK;
}

int64_t conv_bwd_numbers(const tdx::Conv1dParams& p) {
    const int64_t piece = tdx::kConvRuns * tdx::kConvBwdRows;
    return tdx::seq_pieces(p.offsets != nullptr, p.batch, p.rows, conv_dense_pieces(p.max_len, piece), piece);
}

int conv_vector(const tdx_conv1d_args* a, const tdx::Conv1dParams& p, int64_t most, bool back) {
    const int64_t el = elem_bytes(a->dtype);
    Widest w(most);
    w.stride(p.channels, el);                 // rows of a state, and the last vector of a row
    w.ptr(p.x); w.stride(p.ld_x, el);
    if (back) {
        w.ptr(p.dy); w.stride(p.ld_dy, el);
        w.ptr(p.dx); w.stride(p.ld_dx, el);
        w.ptr(p.dstate_in); w.ptr(p.dstate_out);
    } else {
        w.ptr(p.y); w.stride(p.ld_y, el);
        w.ptr(p.state_out);
    }
    w.ptr(p.state_in);
    if (p.state_in || p.state_out || p.dstate_in || p.dstate_out) w.stride(p.state_stride, el);
    return static_cast<int>(std::max<int64_t>(1, w.bytes / el));
}

template <typename T, int VEC, int KW>
int launch_conv1d(ConvPass pass, tdx::Conv1dParams& p, cudaStream_t st) {
    if (pass == kConvStep) {
        p.channel_tiles = static_cast<int>(ceil_div(p.channels, 128 * VEC));
        return launch_seq(tdx::conv1d_step_kernel<T, VEC, KW>, p.batch * p.channel_tiles, 1, 128, 0, st, p);
    }
    p.channel_tiles = static_cast<int>(ceil_div(p.channels, 32 * VEC));
    const int64_t piece = tdx::kConvRuns * (pass == kConvForward ? tdx::kConvRows : tdx::kConvBwdRows);
    p.dense = conv_dense_pieces(p.max_len, piece);
    const int64_t grid = tdx::seq_pieces(p.offsets != nullptr, p.batch, p.rows, p.dense, piece) * p.channel_tiles;
    if (pass == kConvForward) return launch_seq(tdx::conv1d_fwd_kernel<T, VEC, KW>, grid, 1, 128, 0, st, p);
    return launch_seq(tdx::conv1d_bwd_kernel<T, VEC, KW>, grid, 1, 128, 0, st, p);
}
template <typename T, int VEC>
int launch_conv1d_width(ConvPass pass, tdx::Conv1dParams& p, cudaStream_t st) {
    switch (p.width) {
        case 2: return launch_conv1d<T, VEC, 2>(pass, p, st);
        case 3: return launch_conv1d<T, VEC, 3>(pass, p, st);
        case 4: return launch_conv1d<T, VEC, 4>(pass, p, st);
        default: return launch_conv1d<T, VEC, 8>(pass, p, st);
    }
}
int run_conv1d(const tdx_conv1d_args* a, ConvPass pass, tdx::Conv1dParams& p, cudaStream_t st) {
    const bool back = pass == kConvBackward;
    if (a->dtype == TDX_F32) {
        return conv_vector(a, p, 16, back) == 4 ? launch_conv1d_width<float, 4>(pass, p, st) : launch_conv1d_width<float, 1>(pass, p, st);
    }
    // windows, weights and sums of eight channels a thread would leave too few warps
    const int vec = conv_vector(a, p, 8, back);
    return vec == 4 ? launch_conv1d_width<__nv_bfloat16, 4>(pass, p, st)
           : vec == 2 ? launch_conv1d_width<__nv_bfloat16, 2>(pass, p, st) : launch_conv1d_width<__nv_bfloat16, 1>(pass, p, st);
}

// ------------------------------------------------------------------ selective scan
enum ScanPass { kScanForwardPass, kScanBackwardPass, kScanStepPass };

int scan_padded_states(int states) {
    int n = 4;
    while (n < states) n *= 2;
    return n;
}

int check_scan(const tdx_scan_args* a, ScanPass pass, tdx::ScanParams* p, bool sizes_only = false) {
    if (a == nullptr) return fail(TDX_ERR_INVALID_ARG, "args is NULL");
    const bool step = pass == kScanStepPass, back = pass == kScanBackwardPass;
    TDX_TRY(check_sequences(a->batch, a->max_len, a->rows, a->channels, a->dtype, a->seq_offsets, step));
    if (a->states < 1) return fail(TDX_ERR_INVALID_ARG, "states = %d", a->states);
    if (a->states > 128) return fail(TDX_ERR_UNSUPPORTED, "more than 128 states per channel");
    if (a->groups < 1 || a->channels % a->groups) return fail(TDX_ERR_INVALID_ARG, "%lld channels do not divide into %d groups", (long long)a->channels, a->groups);
    if (a->dt_softplus != 0 && a->dt_softplus != 1) return fail(TDX_ERR_INVALID_ARG, "dt_softplus must be 0 or 1");
    int64_t stride = a->state_stride;
    if (!sizes_only) {
        TDX_TRY(check_states(a->state_in || a->state_out || (back && (a->dstate_in || a->dstate_out)), a->batch, a->channels * a->states, &stride,
                             a->slots, a->n_slots));
        const size_t el = elem_bytes(a->dtype);
        const bool any = a->channels > 0 && a->batch > 0, rows = any && (step || a->rows > 0);
        const int64_t bc = static_cast<int64_t>(a->groups) * a->states;
        TDX_TRY(check_tensor("x", a->x, rows, el, a->ld_x, a->channels));
        TDX_TRY(check_tensor("dt", a->dt, rows, el, a->ld_dt, a->channels));
        TDX_TRY(check_tensor("A", a->A, any, 4));
        TDX_TRY(check_tensor("B", a->B, rows, el, a->ld_B, bc));
        TDX_TRY(check_tensor("C", a->C, rows, el, a->ld_C, bc));
        TDX_TRY(check_tensor("D", a->D, false, 4));
        TDX_TRY(check_tensor("z", a->z, false, el, a->ld_z, a->channels));
        TDX_TRY(check_tensor("dt_bias", a->dt_bias, false, 4));
        TDX_TRY(check_tensor("state_in", a->state_in, step && any, 4));
        if (!back) {
            TDX_TRY(check_tensor("out", a->out, rows, el, a->ld_out, a->channels));
            TDX_TRY(check_tensor("state_out", a->state_out, step && any, 4));
        } else {
            TDX_TRY(check_tensor("dout", a->dout, rows, el, a->ld_dout, a->channels));
            TDX_TRY(check_tensor("dx", a->dx, rows, el, a->ld_dx, a->channels));
            TDX_TRY(check_tensor("ddt", a->ddt, rows, el, a->ld_ddt, a->channels));
            TDX_TRY(check_tensor("dB", a->dB, rows, el, a->ld_dB, bc));
            TDX_TRY(check_tensor("dC", a->dC, rows, el, a->ld_dC, bc));
            TDX_TRY(check_tensor("dz", a->dz, rows && a->z, el, a->ld_dz, a->channels));
            TDX_TRY(check_tensor("dA", a->dA, any, 4));
            TDX_TRY(check_tensor("dD", a->dD, false, 4));
            TDX_TRY(check_tensor("ddt_bias", a->ddt_bias, false, 4));
            TDX_TRY(check_tensor("dstate_out", a->dstate_out, false, 4));
            TDX_TRY(check_tensor("dstate_in", a->dstate_in, false, 4));
            TDX_TRY(check_tensor("saved", a->saved, rows, 16));
        }
    }
    std::memset(p, 0, sizeof *p);
    p->batch = a->batch; p->max_len = a->max_len; p->rows = a->rows; p->channels = a->channels;
    p->states = a->states; p->groups = a->groups; p->group_channels = static_cast<int>(a->channels / a->groups); p->softplus = a->dt_softplus;
    p->x = a->x; p->ld_x = a->ld_x; p->dt = a->dt; p->ld_dt = a->ld_dt; p->A = a->A; p->B = a->B; p->ld_b = a->ld_B; p->C = a->C; p->ld_c = a->ld_C;
    p->D = a->D; p->z = a->z; p->ld_z = a->ld_z; p->dt_bias = a->dt_bias; p->out = a->out; p->ld_out = a->ld_out;
    p->offsets = a->seq_offsets; p->state_in = a->state_in; p->state_out = a->state_out; p->state_stride = stride;
    p->slots = a->slots; p->n_slots = a->n_slots; p->saved = a->saved;
    if (back) {
        p->dout = a->dout; p->ld_dout = a->ld_dout; p->dx = a->dx; p->ld_dx = a->ld_dx; p->ddt = a->ddt; p->ld_ddt = a->ld_ddt;
        p->dB = a->dB; p->ld_db = a->ld_dB; p->dC = a->dC; p->ld_dc = a->ld_dC; p->dz = a->dz; p->ld_dz = a->ld_dz;
        p->dA = a->dA; p->dD = a->dD; p->ddt_bias = a->ddt_bias; p->dstate_out = a->dstate_out; p->dstate_in = a->dstate_in;
    }
    return TDX_OK;
}

size_t scan_saved_bytes(const tdx::ScanParams& p) {
    const int64_t n = tdx::seq_pieces(p.offsets != nullptr, p.batch, p.rows, ceil_div(p.max_len, tdx::kScanSave), tdx::kScanSave);
    return static_cast<size_t>(n) * p.channels * scan_padded_states(p.states) * sizeof(float);
}

// How a scan is spread over the SMs: sequences are cut into chunks when channels and sequences alone do not give every SM a
// block; a cut costs a second look at the inputs and a second exponential per state.  Blocks per SM asked for, 4096 x 4096 with 16
// states forward: two 255 us, three 240, although only two are resident (208 registers); backward two, as many as are resident.
void plan_scan(tdx::ScanParams* p, int sm_count, bool back) {
    const int n = scan_padded_states(p->states);
    // sequences that run side by side: packed ones of uneven length count by their rows
    const int64_t longest = std::max<int64_t>(1, std::min(p->max_len, p->rows));
    const int64_t side = p->offsets ? std::max<int64_t>(1, p->rows / longest) : std::max<int64_t>(1, p->batch);
    p->channel_tiles = static_cast<int>(ceil_div(p->group_channels, tdx::kScanThreads * 4 / n));
    const int64_t tiles = std::max<int64_t>(1, static_cast<int64_t>(p->channel_tiles) * p->groups);
    p->chunk = ceil_div(longest, 32) * 32;
    if (tiles * side < sm_count) {
        const int64_t want = ceil_div((back ? 2 : 3) * sm_count, tiles);                // chunks of all sequences together
        const int64_t chunk = std::max<int64_t>(64, ceil_div(ceil_div(p->offsets ? p->rows : longest * side, want), 32) * 32);
        if (chunk < p->chunk) p->chunk = chunk;
    }
    p->cut = longest > p->chunk;
    p->dense = std::max<int64_t>(1, ceil_div(p->max_len, p->chunk));
}
int64_t scan_numbers(const tdx::ScanParams& p) { return tdx::seq_pieces(p.offsets != nullptr, p.batch, p.rows, p.dense, p.chunk); }

int64_t scan_sum_tiles(const tdx::ScanParams& p) { return ceil_div(p.group_channels, 128) * 4; }

struct ScanWorkspace { size_t carry, carry_dt, part_bc, part_a, part_d, total; };
ScanWorkspace scan_workspace(const tdx::ScanParams& p, bool back) {
    const size_t numbers = static_cast<size_t>(scan_numbers(p)), channels = static_cast<size_t>(p.channels),
                 pad = static_cast<size_t>(scan_padded_states(p.states));
    ScanWorkspace w;
    size_t at = 0;
    auto take = [&](size_t floats) { const size_t here = at; at += round_256(floats * sizeof(float)); return here; };
    w.carry = take(p.cut ? numbers * channels * pad : 0);
    w.carry_dt = take(p.cut ? numbers * channels : 0);
    // blocks of more than 32 channels have sums per 32
    w.part_bc = take(back ? static_cast<size_t>(std::max<int64_t>(p.channel_tiles, scan_sum_tiles(p))) * p.rows * p.groups * 2 * pad : 0);
    w.part_a = take(back ? numbers * channels * pad : 0);
    w.part_d = take(back ? numbers * channels * 2 : 0);
    w.total = at;
    return w;
}
void place_scan(tdx::ScanParams* p, const ScanWorkspace& w, void* workspace) {
    char* base = static_cast<char*>(workspace);
    p->carry = reinterpret_cast<float*>(base + w.carry);
    p->carry_dt = reinterpret_cast<float*>(base + w.carry_dt);
    p->part_bc = reinterpret_cast<float*>(base + w.part_bc);
    p->part_a = reinterpret_cast<float*>(base + w.part_a);
    p->part_d = reinterpret_cast<float*>(base + w.part_d);
}

// Neighbouring channels per access: 2 where every row of every activation of the call starts at a multiple of two elements.
int scan_vector(const tdx_scan_args* a, const tdx::ScanParams& p, bool back) {
    const int64_t el = elem_bytes(a->dtype);
    Widest w(2 * el);
    w.stride(p.group_channels, el);
    w.ptr(p.x); w.stride(p.ld_x, el);
    w.ptr(p.dt); w.stride(p.ld_dt, el);
    if (p.z) { w.ptr(p.z); w.stride(p.ld_z, el); }
    if (back) {
        w.ptr(p.dout); w.stride(p.ld_dout, el);
        w.ptr(p.dx); w.stride(p.ld_dx, el);
        w.ptr(p.ddt); w.stride(p.ld_ddt, el);
        if (p.z) { w.ptr(p.dz); w.stride(p.ld_dz, el); }
    } else {
        w.ptr(p.out); w.stride(p.ld_out, el);
    }
    return w.bytes == 2 * el ? 2 : 1;
}

template <typename T, int N, int VEC>
int launch_scan_passes(ScanPass pass, tdx::ScanParams& p, cudaStream_t st) {
    typedef tdx::ScanShape<N> Shape;
    const int64_t numbers = scan_numbers(p), grid = numbers * p.channel_tiles * p.groups;
    constexpr int kThreads = tdx::kScanThreads;
    if (pass == kScanForwardPass) {
        if (p.cut) TDX_TRY(launch_seq(tdx::scan_fwd_kernel<T, N, tdx::kScanState, VEC>, grid, 1, kThreads, 0, st, p));
        return launch_seq(tdx::scan_fwd_kernel<T, N, tdx::kScanFull, VEC>, grid, 1, kThreads, 0, st, p);
    }
    p.sum_tiles = p.channel_tiles * (Shape::kChannels > 32 ? Shape::kChannels / 32 : 1);
    if (p.cut) TDX_TRY(launch_seq(tdx::scan_fwd_kernel<T, N, tdx::kScanAdjoint, VEC>, grid, 1, kThreads, 0, st, p));
    TDX_TRY(launch_seq(tdx::scan_bwd_kernel<T, N, VEC>, grid, 1, kThreads, 0, st, p));
    const int64_t bc_blocks = ceil_div(p.rows * p.groups * 2 * N / 4, 256), a_blocks = ceil_div(p.channels * N, 32), d_blocks = ceil_div(2 * p.channels, 32);
    return launch_seq(tdx::scan_bwd_join_kernel<T>, bc_blocks + a_blocks + d_blocks, 1, 256, 0, st, p, N, static_cast<long long>(bc_blocks),
                      static_cast<long long>(a_blocks), static_cast<long long>(numbers));
}
template <typename T, int N>
int launch_scan(ScanPass pass, int vec, tdx::ScanParams& p, int sm_count, cudaStream_t st) {
    if (pass == kScanStepPass) {
        p.channel_tiles = static_cast<int>(ceil_div(p.channels, 32));
        const bool vec4 = p.states == N && !misaligned(p.state_in, 16) && !misaligned(p.state_out, 16) && !misaligned(p.A, 16) && p.state_stride % 4 == 0;
        // several batch rows a warp, as long as every SM has 32 warps
        const int64_t blocks = ceil_div(p.channel_tiles, 4), rows = std::min<int64_t>(std::min<int64_t>(65535, p.batch), ceil_div(8 * sm_count, blocks));
        return vec4 ? launch_seq(tdx::scan_step_kernel<T, N / 4, true>, blocks, rows, 128, 0, st, p)
                    : launch_seq(tdx::scan_step_kernel<T, N / 4, false>, blocks, rows, 128, 0, st, p);
    }
    return vec == 2 ? launch_scan_passes<T, N, 2>(pass, p, st) : launch_scan_passes<T, N, 1>(pass, p, st);
}
template <typename T>
int launch_scan_states(ScanPass pass, int vec, tdx::ScanParams& p, int sm_count, cudaStream_t st) {
    switch (scan_padded_states(p.states)) {
        case 4: return launch_scan<T, 4>(pass, vec, p, sm_count, st);
        case 8: return launch_scan<T, 8>(pass, vec, p, sm_count, st);
        case 16: return launch_scan<T, 16>(pass, vec, p, sm_count, st);
        case 32: return launch_scan<T, 32>(pass, vec, p, sm_count, st);
        case 64: return launch_scan<T, 64>(pass, vec, p, sm_count, st);
        default: return launch_scan<T, 128>(pass, vec, p, sm_count, st);
    }
}
int run_scan(const tdx_scan_args* a, ScanPass pass, tdx::ScanParams& p, DeviceCtx* ctx, void* stream) {
    p.status = ctx->status_ptr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int vec = pass == kScanStepPass ? 1 : scan_vector(a, p, pass == kScanBackwardPass);
    return a->dtype == TDX_F32 ? launch_scan_states<float>(pass, vec, p, ctx->sm_count, st) : launch_scan_states<__nv_bfloat16>(pass, vec, p, ctx->sm_count, st);
}

// ------------------------------------------------------------------ 4-bit weights
constexpr int kW4Warps = 16;         // of a staged block (see launch_w4_tiles)
// What a block of w4_staged_kernel keeps in shared memory: the ring of weights, x, and `sets` times 16 rows of scales.
template <typename T>
size_t w4_staged_smem(const tdx::W4Params& p, int sets) {
    return tdx::kW4RingBytes * 32 * kW4Warps + tdx::w4_x_bytes<T>(p.steps, p.M) + sizeof(float2) * static_cast<size_t>(tdx::kW4Rows * sets) * tdx::w4_scale_pitch(p.groups);
}
template <typename T, int WORDS, int BLOCKS>
int launch_w4_staged(tdx::W4Params p, cudaStream_t st) {
    p.per = static_cast<int>(ceil_div(p.steps, kW4Warps));
    const size_t smem = w4_staged_smem<T>(p, BLOCKS);
    static std::atomic<bool> known[64];
    TDX_TRY(allow_smem(tdx::w4_staged_kernel<T, WORDS, BLOCKS>, known, smem));
    return launch_seq(tdx::w4_staged_kernel<T, WORDS, BLOCKS>, ceil_div(p.N, tdx::kW4Rows * BLOCKS), 1, 32 * kW4Warps, smem, st, p);
}
template <typename T, int WORDS, int TILES>
int launch_w4_direct(const tdx::W4Params& p, cudaStream_t st) {
    return launch_seq(tdx::w4_direct_kernel<T, WORDS, TILES>, ceil_div(p.N, 16), ceil_div(p.M, TILES * tdx::W4Columns<T>::kRows), 256, 0, st, p);
}
template <typename T, int WORDS>
int launch_w4_tiles(tdx::W4Params p, const DeviceCtx& ctx, cudaStream_t st) {
    constexpr int kRows = tdx::W4Columns<T>::kRows;
    p.steps = static_cast<int>(ceil_div(p.K, tdx::kW4Step));
    p.groups = static_cast<int>(p.K / p.group);
    // Sixteen warps a block: eight took 6.7 us instead of 4.7 for one token and 4096 x 4096 weights.  Two sets of 16 rows a block
    // save a layout of x, but halve the blocks: 13.5 instead of 15.4 us for 8192 x 8192 (512 sets), 7.0 instead of 4.7 for
    // 4096 x 4096 (256), so they are taken when one set each would need a second wave of two blocks per SM.  Scales grow with K /
    // group: where they and x leave no room for two sets a block has one, and where not even for one the direct kernel runs.
    if (p.M <= kRows && tdx::w4_x_bytes<T>(p.steps, p.M) <= 64 * 1024) {
        const size_t most = static_cast<size_t>(ctx.smem_optin);
        if (ceil_div(p.N, tdx::kW4Rows) > 2 * ctx.sm_count && w4_staged_smem<T>(p, 2) <= most) return launch_w4_staged<T, WORDS, 2>(p, st);
        if (w4_staged_smem<T>(p, 1) <= most) return launch_w4_staged<T, WORDS, 1>(p, st);
    }
    if (p.M <= kRows) return launch_w4_direct<T, WORDS, 1>(p, st);
    if (p.M <= 2 * kRows) return launch_w4_direct<T, WORDS, 2>(p, st);
    if (p.M <= 3 * kRows) return launch_w4_direct<T, WORDS, 3>(p, st);
    return launch_w4_direct<T, WORDS, 4>(p, st);
}
template <typename T>
int launch_w4(const tdx::W4Params& p, const DeviceCtx& ctx, cudaStream_t st) {
    // the tensor-core kernel reads 4, 8 or 16 bytes of a weight row and 16 bytes of a row of x at a time
    const bool fast = (p.group == 32 || p.group == 64 || p.group == 128) && p.K % p.group == 0 && !misaligned(p.weight, p.group / 8) &&
                      !misaligned(p.x, 16) && (p.M == 1 || p.ld_x * static_cast<int64_t>(sizeof(T)) % 16 == 0) && p.M <= 65535LL * 8;
    if (!fast) return launch_seq(tdx::w4_generic_kernel<T>, ceil_div(p.N, 4), std::min<int64_t>(ceil_div(p.M, 4), 1024), 128, 0, st, p);
    switch (p.group) {
        case 32: return launch_w4_tiles<T, 1>(p, ctx, st);
        case 64: return launch_w4_tiles<T, 2>(p, ctx, st);
        default: return launch_w4_tiles<T, 4>(p, ctx, st);
    }
}

}  // namespace

extern "C" {

int tdx_causal_conv1d(const tdx_conv1d_args* args, void* stream) {
    tdx::Conv1dParams p;
    TDX_TRY(check_conv1d(args, kConvForward, &p));
    if (p.batch == 0 || p.channels == 0 || (p.rows == 0 && p.state_out == nullptr)) return TDX_OK;
    DeviceCtx* ctx;
    TDX_TRY(get_ctx(&ctx));
    p.status = ctx->status_ptr;
    return run_conv1d(args, kConvForward, p, static_cast<cudaStream_t>(stream));
}

int tdx_causal_conv1d_step(const tdx_conv1d_args* args, void* stream) {
    tdx::Conv1dParams p;
    TDX_TRY(check_conv1d(args, kConvStep, &p));
    if (p.batch == 0 || p.channels == 0) return TDX_OK;
    DeviceCtx* ctx;
    TDX_TRY(get_ctx(&ctx));
    p.status = ctx->status_ptr;
    return run_conv1d(args, kConvStep, p, static_cast<cudaStream_t>(stream));
}

int tdx_causal_conv1d_workspace_size(const tdx_conv1d_args* args, size_t* bytes) {
    if (args == nullptr || bytes == nullptr) return fail(TDX_ERR_INVALID_ARG, "NULL argument");
    TDX_TRY(check_sequences(args->batch, args->max_len, args->rows, args->channels, args->dtype, args->seq_offsets, false));
    if (args->width < 1 || args->width > 8) return fail(TDX_ERR_INVALID_ARG, "width %d is not in 1 .. 8", args->width);
    tdx::Conv1dParams p;
    std::memset(&p, 0, sizeof p);
    p.batch = args->batch; p.max_len = args->max_len; p.rows = args->rows; p.offsets = args->seq_offsets;
    *bytes = round_256(static_cast<size_t>(conv_bwd_numbers(p)) * args->channels * (args->width + 1) * sizeof(float));
    return TDX_OK;
}

int tdx_causal_conv1d_bwd(const tdx_conv1d_args* args, void* stream) {
    tdx::Conv1dParams p;
    TDX_TRY(check_conv1d(args, kConvBackward, &p));
    if (p.channels == 0) return TDX_OK;
    const int64_t numbers = conv_bwd_numbers(p), elems = p.channels * (p.width + 1);
    TDX_TRY(check_workspace(args->workspace, args->workspace_bytes, static_cast<size_t>(numbers) * elems * sizeof(float)));
    if (numbers == 0 && p.dweight == nullptr && p.dbias == nullptr) return TDX_OK;
    DeviceCtx* ctx;
    TDX_TRY(get_ctx(&ctx));
    p.status = ctx->status_ptr;
    p.partial = static_cast<float*>(args->workspace);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (numbers > 0) TDX_TRY(run_conv1d(args, kConvBackward, p, st));
    if (p.dweight == nullptr && p.dbias == nullptr) return TDX_OK;
    return launch_seq(tdx::conv1d_dweight_kernel, ceil_div(elems, 32), 1, 256, 0, st, static_cast<long long>(elems), static_cast<long long>(numbers),
                      p.width, static_cast<const float*>(p.partial), p.dweight, p.dbias);
}

int tdx_selective_scan(const tdx_scan_args* args, void* stream) {
    tdx::ScanParams p;
    TDX_TRY(check_scan(args, kScanForwardPass, &p));
    if (p.batch == 0 || p.channels == 0 || (p.rows == 0 && p.state_out == nullptr)) return TDX_OK;
    if (p.saved) {
        if (misaligned(p.saved, 16)) return fail(TDX_ERR_ALIGNMENT, "saved is not 16-byte aligned");
        if (args->saved_bytes < scan_saved_bytes(p)) return fail(TDX_ERR_WORKSPACE, "saved needs %llu bytes", (unsigned long long)scan_saved_bytes(p));
    }
    DeviceCtx* ctx;
    TDX_TRY(get_ctx(&ctx));
    plan_scan(&p, ctx->sm_count, false);
    const ScanWorkspace w = scan_workspace(p, false);
    TDX_TRY(check_workspace(args->workspace, args->workspace_bytes, w.total));
    place_scan(&p, w, args->workspace);
    return run_scan(args, kScanForwardPass, p, ctx, stream);
}

int tdx_selective_scan_bwd(const tdx_scan_args* args, void* stream) {
    tdx::ScanParams p;
    TDX_TRY(check_scan(args, kScanBackwardPass, &p));
    if (p.channels == 0) return TDX_OK;
    if (p.rows > 0 && args->saved_bytes < scan_saved_bytes(p)) return fail(TDX_ERR_WORKSPACE, "saved needs %llu bytes", (unsigned long long)scan_saved_bytes(p));
    DeviceCtx* ctx;
    TDX_TRY(get_ctx(&ctx));
    if (p.batch == 0) {
        cudaStream_t st = static_cast<cudaStream_t>(stream);
        if (p.dA) TDX_CUDA(cudaMemsetAsync(p.dA, 0, p.channels * p.states * sizeof(float), st));
        if (p.dD) TDX_CUDA(cudaMemsetAsync(p.dD, 0, p.channels * sizeof(float), st));
        if (p.ddt_bias) TDX_CUDA(cudaMemsetAsync(p.ddt_bias, 0, p.channels * sizeof(float), st));
        return TDX_OK;
    }
    plan_scan(&p, ctx->sm_count, true);
    const ScanWorkspace w = scan_workspace(p, true);
    TDX_TRY(check_workspace(args->workspace, args->workspace_bytes, w.total));
    place_scan(&p, w, args->workspace);
    return run_scan(args, kScanBackwardPass, p, ctx, stream);
}

int tdx_selective_scan_step(const tdx_scan_args* args, void* stream) {
    tdx::ScanParams p;
    TDX_TRY(check_scan(args, kScanStepPass, &p));
    if (p.batch == 0 || p.channels == 0) return TDX_OK;
    DeviceCtx* ctx;
    TDX_TRY(get_ctx(&ctx));
    return run_scan(args, kScanStepPass, p, ctx, stream);
}

int tdx_selective_scan_saved_size(const tdx_scan_args* args, size_t* bytes) {
    if (bytes == nullptr) return fail(TDX_ERR_INVALID_ARG, "bytes is NULL");
    tdx::ScanParams p;
    TDX_TRY(check_scan(args, kScanForwardPass, &p, true));
    *bytes = scan_saved_bytes(p);
    return TDX_OK;
}

int tdx_selective_scan_workspace_size(const tdx_scan_args* args, size_t* bytes) {
    if (bytes == nullptr) return fail(TDX_ERR_INVALID_ARG, "bytes is NULL");
    tdx::ScanParams p;
    TDX_TRY(check_scan(args, kScanForwardPass, &p, true));
    const int sm_count = sm_count_or_default();
    plan_scan(&p, sm_count, false);
    *bytes = scan_workspace(p, false).total;
    if (args->saved != nullptr) {
        plan_scan(&p, sm_count, true);
        *bytes = std::max(*bytes, scan_workspace(p, true).total);
    }
    return TDX_OK;
}

int tdx_gemm_w4(const tdx_w4_args* args, void* stream) {
    if (args == nullptr) return fail(TDX_ERR_INVALID_ARG, "args is NULL");
    const tdx_w4_args& a = *args;
    if (a.M < 0 || a.N < 0 || a.K < 0) return fail(TDX_ERR_INVALID_ARG, "negative dimension");
    if (a.dtype != TDX_F32 && a.dtype != TDX_BF16) return fail(TDX_ERR_INVALID_ARG, "unknown dtype %d", a.dtype);
    if (a.group_size < 1) return fail(TDX_ERR_INVALID_ARG, "group_size must be >= 1");
    if (a.M == 0 || a.N == 0) return TDX_OK;
    if (a.K > (1LL << 31)) return fail(TDX_ERR_UNSUPPORTED, "K above 2^31");
    const size_t el = elem_bytes(a.dtype);
    TDX_TRY(check_tensor("x", a.x, a.K > 0, el, a.ld_x, a.K));
    TDX_TRY(check_tensor("weight", a.weight, a.K > 0, 1));
    TDX_TRY(check_tensor("scales", a.scales, a.K > 0, el));
    TDX_TRY(check_tensor("y", a.y, true, el, a.ld_y, a.N));
    DeviceCtx* ctx;
    TDX_TRY(get_ctx(&ctx));
    tdx::W4Params p;
    std::memset(&p, 0, sizeof p);
    p.M = a.M; p.N = a.N; p.K = a.K; p.group = a.group_size;
    p.x = a.x; p.ld_x = a.ld_x; p.weight = a.weight; p.scales = a.scales; p.zeros = a.zeros; p.y = a.y; p.ld_y = a.ld_y;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return a.dtype == TDX_F32 ? launch_w4<float>(p, *ctx, st) : launch_w4<__nv_bfloat16>(p, *ctx, st);
}

int tdx_w4_quantize(int64_t N, int64_t K, int group_size, int dtype, const void* w, int64_t ld_w, uint8_t* weight, void* scales,
                    uint8_t* zeros, void* stream) {
    if (N < 0 || K < 0) return fail(TDX_ERR_INVALID_ARG, "negative dimension");
    if (dtype != TDX_F32 && dtype != TDX_BF16) return fail(TDX_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (group_size < 1 || (group_size % 2 && group_size < K)) return fail(TDX_ERR_INVALID_ARG, "group_size %d is neither even nor >= K", group_size);
    if (N == 0 || K == 0) return TDX_OK;
    const size_t el = elem_bytes(dtype);
    TDX_TRY(check_tensor("w", w, true, el, ld_w, K));
    TDX_TRY(check_tensor("weight", weight, true, 1));
    TDX_TRY(check_tensor("scales", scales, true, el));
    DeviceCtx* ctx;
    TDX_TRY(get_ctx(&ctx));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t blocks = ceil_div(N * ceil_div(K, group_size), 4);
    if (dtype == TDX_F32)
        return launch_seq(tdx::w4_quantize_kernel<float>, blocks, 1, 128, 0, st, static_cast<long long>(N), static_cast<long long>(K), group_size,
                          static_cast<const float*>(w), static_cast<long long>(ld_w), weight, static_cast<float*>(scales), zeros);
    return launch_seq(tdx::w4_quantize_kernel<__nv_bfloat16>, blocks, 1, 128, 0, st, static_cast<long long>(N), static_cast<long long>(K), group_size,
                      static_cast<const __nv_bfloat16*>(w), static_cast<long long>(ld_w), weight, static_cast<__nv_bfloat16*>(scales), zeros);
}

}  // extern "C"
