// Entry points of the products grouped by expert (see tdx.h).
#include "layer_host.cuh"

#include "grouped_kernels.cuh"

namespace {

int check_grouped(const tdx_grouped_args* args, tdx::GroupedPass pass, tdx::GroupedParams* p) {
    if (args == nullptr) return fail(TDX_ERR_INVALID_ARG, "args is NULL");
    const tdx_grouped_args& a = *args;
    if (a.rows < 0 || a.experts < 0 || a.N < 0 || a.K < 0) return fail(TDX_ERR_INVALID_ARG, "negative size");
    if (a.dtype != TDX_F32 && a.dtype != TDX_BF16) return fail(TDX_ERR_INVALID_ARG, "unknown dtype %d", a.dtype);
    if (a.rows > INT_MAX || a.experts > (1 << 20)) return fail(TDX_ERR_UNSUPPORTED, "more than 2^31 - 1 rows or 2^20 experts");
    if (a.N > (1 << 24) || a.K > (1 << 24)) return fail(TDX_ERR_UNSUPPORTED, "N or K above 2^24");
    const size_t el = elem_bytes(a.dtype);
    const bool outs = pass == tdx::kGroupedForward ? a.rows > 0 && a.N > 0 : pass == tdx::kGroupedDx ? a.rows > 0 && a.K > 0 : a.N > 0 && a.K > 0;
    const bool any = a.experts > 0 && outs;
    const bool all = any && a.rows > 0 && a.N > 0 && a.K > 0;     // there are products
    if (any && a.offsets == nullptr) return fail(TDX_ERR_INVALID_ARG, "offsets is NULL");
    if (misaligned(a.offsets, 4)) return fail(TDX_ERR_ALIGNMENT, "offsets is not aligned to its elements");
    if (pass != tdx::kGroupedDw) TDX_TRY(check_tensor("weight", a.weight, all, el));
    if (pass != tdx::kGroupedDx) TDX_TRY(check_tensor("x", a.x, all, el, a.ld_x, a.K));
    if (pass != tdx::kGroupedForward) TDX_TRY(check_tensor("dy", a.dy, all, el, a.ld_dy, a.N));
    std::memset(p, 0, sizeof *p);
    p->rows = a.rows; p->experts = static_cast<int>(a.experts); p->N = static_cast<int>(a.N); p->K = static_cast<int>(a.K); p->offsets = a.offsets;
    switch (pass) {
        case tdx::kGroupedForward:
            TDX_TRY(check_tensor("y", a.y, any, el, a.ld_y, a.N));
            p->a = a.x; p->ld_a = a.ld_x; p->b = a.weight; p->out = a.y; p->ld_out = a.ld_y;
            break;
        case tdx::kGroupedDx:
            TDX_TRY(check_tensor("dx", a.dx, any, el, a.ld_dx, a.K));
            p->a = a.dy; p->ld_a = a.ld_dy; p->b = a.weight; p->out = a.dx; p->ld_out = a.ld_dx;
            break;
        default:
            TDX_TRY(check_tensor("dweight", a.dweight, any, el));
            p->a = a.dy; p->ld_a = a.ld_dy; p->b = a.x; p->ld_b = a.ld_x; p->out = a.dweight; p->ld_out = a.K;
    }
    return TDX_OK;
}

template <typename T, int PASS, int BM, int VEC>
int launch_grouped_simt(const tdx::GroupedParams& p, cudaStream_t st) {
    const int64_t tiles_m = PASS == tdx::kGroupedDw ? p.experts * ceil_div(p.N, BM) : tdx::seq_pieces(true, p.experts, p.rows, 0, BM);
    return launch_seq(tdx::grouped_simt_kernel<T, PASS, BM, VEC>, tiles_m * ceil_div(PASS == tdx::kGroupedForward ? p.N : p.K, tdx::kSimtColumns), 1, tdx::kSimtThreads, 0, st, p);
}
template <typename T, int PASS, int VEC>
int launch_grouped_rows(const tdx::GroupedParams& p, cudaStream_t st) {
    if constexpr (PASS != tdx::kGroupedDw)
        if (p.rows <= 16 * static_cast<int64_t>(p.experts)) return launch_grouped_simt<T, PASS, 16, VEC>(p, st);
    return launch_grouped_simt<T, PASS, 64, VEC>(p, st);
}

// Every row of every operand starts at 16 bytes and has a multiple of 16.
bool grouped_aligned(const tdx_grouped_args& a, const tdx::GroupedParams& p, int pass) {
    const int el = a.dtype == TDX_F32 ? 4 : 2;
    Widest w(16);
    w.stride(a.K, el);
    w.stride(a.N, el);
    w.ptr(p.a); w.stride(p.ld_a, el);
    w.ptr(p.b); w.ptr(p.out);
    if (pass == tdx::kGroupedDw) w.stride(p.ld_b, el);
    else w.stride(p.ld_out, el);
    return w.bytes == 16;
}
// The tensor-core kernel reads (aligned) operands by the copy engine and writes 16 bytes at a time; no rows, for dw, are zeros to write.
bool grouped_fast(const tdx_grouped_args& a) {
    return a.dtype == TDX_BF16 && a.rows != 0 && a.N != 0 && a.K != 0 && a.experts <= tdx::kGroupedMostExperts;
}

template <int PASS>
int launch_grouped_umma(tdx::GroupedParams p, const tdx_host::Device& dev, cudaStream_t st) {
    p.features = PASS == tdx::kGroupedDx ? p.K : p.N;
    const int depth = PASS == tdx::kGroupedForward ? p.K : p.N;
    const int64_t rows_each = ceil_div(p.rows, p.experts);
    if (PASS == tdx::kGroupedDw) {
        // Few rows are a short reduction, and the time is that of writing dw: tiles of 128 x 256, whose accumulators fit twice (40 rows an
        // expert, 32 x 2048 x 2048: 56 to 70 us instead of 70 to 87).  From about 500 rows on both take about the same: 512 rows, 16 x 4096 x
        // 2048: 134 instead of 130; 600, 8 x 2304 x 2048: 64 instead of 61; 1024: 81 instead of 76; 2048, 8 x 4096 x 4096: 434 instead of 431 to 448.
        p.bt = p.K > 128 ? 256 : 128;
        p.halves = p.N > 128 && rows_each > 512 ? 2 : 1;
    } else {
        // as wide as an expert's rows: 8 x 2048 rows, 4096 x 4096: 256 features x 256 rows 377 us, 128 x 256 444 to 470, 256 x 128 547 to 560, 128 x
        // 128 656 to 673; 16 x 100 rows, 4096 x 2048: 256 x 128 52, 128 x 128 and 256 x 256 55, 128 x 256 59; up to 16 rows 128 x 32
        p.bt = rows_each <= 16 ? 32 : rows_each <= 48 ? 64 : rows_each <= 128 ? 128 : 256;
        p.halves = p.bt >= 128 && p.features > 128 ? 2 : 1;
    }
    p.buffers = 2 * p.halves * p.bt <= 512 ? 2 : 1;
    p.box = std::min(p.bt, 64);
    p.feature_tiles = static_cast<int>(ceil_div(p.features, 128 * p.halves));
    p.column_tiles = static_cast<int>(ceil_div(p.K, p.bt));
    p.blocks = static_cast<int>(ceil_div(depth, 64));
    p.tmem_cols = 32;
    while (p.tmem_cols < p.buffers * p.halves * p.bt) p.tmem_cols *= 2;
    const int stage = p.halves * 16384 + p.bt * 128;
    const size_t fixed = 1024 + tdx::kGroupedStaging + sizeof(int) * 2 * (p.experts + 1);
    const int room = dev.smem_optin - 1024;                       // barriers are static
    p.stages = static_cast<int>(std::min<int64_t>(tdx::kGroupedMostStages, (room - static_cast<int64_t>(fixed)) / stage));
    const uint64_t K = p.K, N = p.N, rows = p.rows, E = p.experts;
    CUtensorMap a, b, out;
    if (PASS == tdx::kGroupedDw) {
        const uint64_t da[2] = {N, rows}, sa[1] = {static_cast<uint64_t>(p.ld_a) * 2}, db[2] = {K, rows}, sb[1] = {static_cast<uint64_t>(p.ld_b) * 2};
        const uint32_t box[2] = {64, 64};
        TDX_TRY(tdx_host::bf16_map(p.a, 2, da, sa, box, &a));
        TDX_TRY(tdx_host::bf16_map(p.b, 2, db, sb, box, &b));
        const uint64_t dw[3] = {K, N, E}, sw[2] = {K * 2, K * N * 2};
        const uint32_t box_out[3] = {32, 32, 1};
        TDX_TRY(tdx_host::bf16_map(p.out, 3, dw, sw, box_out, &out, 64));
    } else {
        const uint64_t dw[3] = {K, N, E}, sw[2] = {K * 2, K * N * 2}, dx[2] = {static_cast<uint64_t>(depth), rows}, sx[1] = {static_cast<uint64_t>(p.ld_a) * 2};
        const uint32_t box_w[3] = {64, PASS == tdx::kGroupedForward ? 128u : 64u, 1}, box_x[2] = {64, static_cast<uint32_t>(p.box)};
        TDX_TRY(tdx_host::bf16_map(p.b, 3, dw, sw, box_w, &a));
        TDX_TRY(tdx_host::bf16_map(p.a, 2, dx, sx, box_x, &b));
        const uint64_t dy[2] = {static_cast<uint64_t>(p.features), rows}, sy[1] = {static_cast<uint64_t>(p.ld_out) * 2};
        const uint32_t box_y[2] = {32, 16};
        TDX_TRY(tdx_host::bf16_map(p.out, 2, dy, sy, box_y, &out, 64));
    }
    const int64_t items = PASS == tdx::kGroupedDw ? E * p.feature_tiles * static_cast<int64_t>(p.column_tiles) : (p.rows / p.bt + p.experts) * static_cast<int64_t>(p.feature_tiles);
    const size_t smem = fixed + static_cast<size_t>(p.stages) * stage;
    static std::atomic<bool> known[64];
    TDX_TRY(allow_smem(tdx::grouped_umma_kernel<PASS>, known, smem, room));
    return launch_seq(tdx::grouped_umma_kernel<PASS>, std::min<int64_t>(items, dev.sm_count), 1, tdx::kGroupedThreads, smem, st, a, b, out, p);
}

template <int PASS>
int run_grouped(const tdx_grouped_args* args, void* stream) {
    tdx::GroupedParams p;
    TDX_TRY(check_grouped(args, static_cast<tdx::GroupedPass>(PASS), &p));
    if (p.experts == 0 || (PASS != tdx::kGroupedDw && p.rows == 0) || (PASS != tdx::kGroupedForward && p.K == 0) || (PASS != tdx::kGroupedDx && p.N == 0)) return TDX_OK;
    tdx_host::Device dev;
    TDX_TRY(tdx_host::get_device(&dev));
    p.status = dev.status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool aligned = grouped_aligned(*args, p, PASS);
    if (aligned && grouped_fast(*args)) return launch_grouped_umma<PASS>(p, dev, st);
    if (args->dtype != TDX_F32) return launch_grouped_rows<__nv_bfloat16, PASS, 1>(p, st);
    return aligned ? launch_grouped_rows<float, PASS, 4>(p, st) : launch_grouped_rows<float, PASS, 1>(p, st);
}

}  // namespace

extern "C" {

int tdx_gemm_grouped(const tdx_grouped_args* args, void* stream) { return run_grouped<tdx::kGroupedForward>(args, stream); }
int tdx_gemm_grouped_dx(const tdx_grouped_args* args, void* stream) { return run_grouped<tdx::kGroupedDx>(args, stream); }
int tdx_gemm_grouped_dw(const tdx_grouped_args* args, void* stream) { return run_grouped<tdx::kGroupedDw>(args, stream); }

int tdx_gemm_grouped_workspace_size(const tdx_grouped_args* args, size_t* bytes) {
    if (args == nullptr || bytes == nullptr) return fail(TDX_ERR_INVALID_ARG, "NULL argument");
    if (args->rows < 0 || args->experts < 0 || args->N < 0 || args->K < 0) return fail(TDX_ERR_INVALID_ARG, "negative size");
    *bytes = 0;
    return TDX_OK;
}

}  // extern "C"
