// Entry points of the linear attention with decay (see tdx.h).
#include "layer_host.cuh"

#include "attention_kernels.cuh"
#include "attention_umma.cuh"

namespace {

enum AttnPass { kAttnForward, kAttnBackward, kAttnStep };
// the four sums: which operand plays which role
enum AttnSum { kAttnOut, kAttnDq, kAttnDk, kAttnDv };

struct AttnShape { int q_heads, k_heads, v_heads; int64_t state_stride; };

int check_attention(const tdx_attention_args* args, AttnPass pass, AttnShape* shape, bool sizes_only = false) {
    if (args == nullptr) return fail(TDX_ERR_INVALID_ARG, "args is NULL");
    const tdx_attention_args& a = *args;
    const bool step = pass == kAttnStep, back = pass == kAttnBackward;
    if (a.heads < 0) return fail(TDX_ERR_INVALID_ARG, "heads = %d", a.heads);
    TDX_TRY(check_sequences(a.batch, a.max_len, a.rows, a.heads, a.dtype, a.seq_offsets, step));
    shape->q_heads = a.q_heads ? a.q_heads : a.heads;
    shape->k_heads = a.k_heads ? a.k_heads : a.heads;
    shape->v_heads = a.v_heads ? a.v_heads : a.heads;
    for (int h : {shape->q_heads, shape->k_heads, shape->v_heads})
        if (h < 0 || (a.heads > 0 && a.heads % h)) return fail(TDX_ERR_INVALID_ARG, "%d heads do not share %d", a.heads, h);
    if (a.dim_k < 1 || a.dim_v < 1) return fail(TDX_ERR_INVALID_ARG, "dim_k = %d, dim_v = %d", a.dim_k, a.dim_v);
    if (a.dim_k > 128 || a.dim_v > 128) return fail(TDX_ERR_UNSUPPORTED, "a head of more than 128");
    if (a.heads > (1 << 16)) return fail(TDX_ERR_UNSUPPORTED, "more than 2^16 heads");
    if (!(a.scale - a.scale == 0.0f)) return fail(TDX_ERR_INVALID_ARG, "scale is not finite");
    if (sizes_only) return TDX_OK;
    shape->state_stride = a.state_stride;
    TDX_TRY(check_states(a.state_in || a.state_out || step || (back && (a.dstate_in || a.dstate_out)), a.batch,
                         static_cast<int64_t>(a.heads) * a.dim_k * a.dim_v, &shape->state_stride, a.slots, a.n_slots));
    const size_t el = elem_bytes(a.dtype);
    const bool any = a.heads > 0 && a.batch > 0, rows = any && (step || a.rows > 0);
    const int64_t wq = static_cast<int64_t>(shape->q_heads) * a.dim_k, wk = static_cast<int64_t>(shape->k_heads) * a.dim_k,
                  wv = static_cast<int64_t>(shape->v_heads) * a.dim_v, wo = static_cast<int64_t>(a.heads) * a.dim_v;
    TDX_TRY(check_tensor("log_decay", a.log_decay, any, 4));
    TDX_TRY(check_tensor("q", a.q, rows, el, a.ld_q, wq));
    TDX_TRY(check_tensor("k", a.k, rows, el, a.ld_k, wk));
    TDX_TRY(check_tensor("v", a.v, rows, el, a.ld_v, wv));
    TDX_TRY(check_tensor("state_in", a.state_in, step && any, 4));
    if (back) {
        TDX_TRY(check_tensor("dout", a.dout, rows, el, a.ld_dout, wo));
        TDX_TRY(check_tensor("dq", a.dq, rows, el, a.ld_dq, wq));
        TDX_TRY(check_tensor("dk", a.dk, rows, el, a.ld_dk, wk));
        TDX_TRY(check_tensor("dv", a.dv, rows, el, a.ld_dv, wv));
        TDX_TRY(check_tensor("dstate_out", a.dstate_out, false, 4));
        TDX_TRY(check_tensor("dstate_in", a.dstate_in, false, 4));
    } else {
        TDX_TRY(check_tensor("out", a.out, rows, el, a.ld_out, wo));
        TDX_TRY(check_tensor("state_out", a.state_out, step && any, 4));
    }
    return TDX_OK;
}

int attention_padded(int d1) { return d1 > 64 ? 128 : 64; }
// Blocks of the kernel on mma.sync that an SM holds: two by their registers, one where fp32 operands take more than half the shared memory
// (a kilobyte of which goes with every block, next to what is static).
int attention_blocks(int dtype, int d1) {
    const bool wide = attention_padded(d1) == 128;
    const int bytes = dtype == TDX_F32 ? (wide ? tdx::AttnTiles<float, 128>::kBytes : tdx::AttnTiles<float, 64>::kBytes)
                                       : (wide ? tdx::AttnTiles<__nv_bfloat16, 128>::kBytes : tdx::AttnTiles<__nv_bfloat16, 64>::kBytes);
    return 2 * (bytes + 2048) <= kSmemLimitDefault + 1024 ? 2 : 1;
}

// How a sum is spread over the SMs: the rows of a segment.  Heads (and, in the kernel on mma.sync, slices of 64 columns) and sequences
// run side by side; where they do not fill the SMs evenly, sequences are cut into segments, which costs a look at k and v of all but the
// last one for what they add to the state (about half a segment's time) and two chunks' time a block for its start.  The number of segments
// with the least estimated time is taken, of two chunks at least (packed fp32 prompts, 2491 rows, 6 heads of 64 and 80: segments of 128
// rows 44 us, of 256 rows 72).
void plan_attention(const tdx_attention_args& a, int d1, int d2, bool umma, bool all_pieces, int sm_count, tdx::AttnParams* p) {
    const int64_t longest = std::max<int64_t>(1, std::min(a.max_len, a.rows));
    const int64_t side = a.seq_offsets ? std::max<int64_t>(1, a.rows / longest) : std::max<int64_t>(1, a.batch);
    const int64_t chunk = umma ? tdx::kAttnRows : tdx::kAttnC, slots = umma ? sm_count : attention_blocks(a.dtype, d1) * sm_count;
    p->slices = umma ? 1 : static_cast<int>(ceil_div(d2, tdx::kAttnV));
    const int64_t tiles = std::max<int64_t>(1, static_cast<int64_t>(p->slices) * a.heads) * side;
    double least = 0.0;
    p->seg = ceil_div(longest, chunk) * chunk;
    for (int64_t n = 1; n <= 64; ++n) {
        const int64_t seg = std::max<int64_t>(2 * chunk, ceil_div(ceil_div(longest, n), chunk) * chunk), cuts = ceil_div(longest, seg);
        if (n > 1 && cuts < n) continue;
        const double chunks = static_cast<double>(std::min(seg, longest)) / chunk;
        double cost = ceil_div(tiles * cuts, slots) * (chunks + 2.0);
        if (cuts > 1) cost += ceil_div(tiles * (cuts - 1), slots) * (0.5 * chunks + 2.0);
        if (n == 1 || cost < least) {
            least = cost;
            p->seg = seg;
        }
    }
    p->dense = std::max<int64_t>(1, ceil_div(a.max_len, p->seg));
    // the pass over the states has all segments but the last (with state_out that one too): pieces of them, as many as fill the SMs
    p->sub = p->seg;
    p->all_pieces = all_pieces;
    if (umma) {
        const int64_t busy = tiles * std::max<int64_t>(1, ceil_div(longest, p->seg) - (all_pieces ? 0 : 1)), most = p->seg / tdx::kAttnRows;
        int64_t k = std::min(most, std::max<int64_t>(1, sm_count / busy));
        while (most % k) --k;
        p->sub = p->seg / k;
    }
    p->sub_dense = std::max<int64_t>(1, ceil_div(a.max_len, p->sub));
    // Slots for all sequences as long as that is no more than a slot a segment: else sequences of one segment make their states on the way
    // to the outputs (lengths 3000, 700, 200 and 64, 16 heads of 128: 80 instead of 84 us; 8192 and 255 single rows, 32 heads: 2.0 instead of 1.1 ms
    // and 545 instead of 17 MB).
    p->every = a.seq_offsets == nullptr || a.batch <= a.rows / p->seg;
}
int64_t attention_numbers(const tdx_attention_args& a, const tdx::AttnParams& p) {
    return tdx::seq_pieces(a.seq_offsets != nullptr, a.batch, a.rows, p.dense, p.seg);
}
int64_t attention_slots(const tdx_attention_args& a, const tdx::AttnParams& p) {
    return a.seq_offsets ? tdx::attn_slots_before(static_cast<int>(a.rows), a.batch, static_cast<int>(p.sub), static_cast<int>(p.seg), p.every) : a.batch * p.sub_dense;
}
bool attention_cut(const tdx_attention_args& a, const tdx::AttnParams& p) { return std::min(a.max_len, a.rows) > p.seg; }

struct AttnWorkspace { size_t carry, each, total; };
AttnWorkspace attention_workspace(const tdx_attention_args& a, const AttnShape& shape, int sm_count, bool back) {
    AttnWorkspace w = {0, 0, 0};
    tdx::AttnParams p;
    for (int sum = 0; sum < (back ? 4 : 1); ++sum) {
        const int d1 = sum == kAttnOut || sum == kAttnDv ? a.dim_k : a.dim_v, d2 = sum == kAttnOut || sum == kAttnDv ? a.dim_v : a.dim_k;
        for (int way = 0; way < 3; ++way) {                      // whichever the alignment allows, with and without state_out
            const bool umma = way > 0;
            plan_attention(a, d1, d2, umma, way == 2, sm_count, &p);
            const size_t each = umma ? tdx::kAttnRows * tdx::kAttnRows : p.slices * attention_padded(d1) * tdx::kAttnV;
            if (attention_cut(a, p)) w.carry = std::max(w.carry, static_cast<size_t>(attention_slots(a, p)) * a.heads * each * sizeof(float));
        }
    }
    w.carry = round_256(w.carry);
    if (back && (shape.q_heads < a.heads || shape.k_heads < a.heads || shape.v_heads < a.heads))
        w.each = round_256(static_cast<size_t>(a.rows) * a.heads * std::max(a.dim_k, a.dim_v) * sizeof(float));
    w.total = w.carry + w.each;
    return w;
}

template <typename T, int KD, bool STATE, int UP>
int launch_attention(const tdx::AttnParams& p, int64_t numbers, cudaStream_t st) {
    static std::atomic<bool> known[64];
    constexpr size_t kBytes = tdx::AttnTiles<T, KD>::kBytes;
    TDX_TRY(allow_smem(tdx::attn_kernel<T, KD, STATE, UP>, known, kBytes, static_cast<int>(kBytes)));
    return launch_seq(tdx::attn_kernel<T, KD, STATE, UP>, numbers * p.heads * p.slices, 1, tdx::kAttnThreads, kBytes, st, p);
}
template <typename T, int KD, int UP>
int launch_attention_passes(const tdx::AttnParams& p, int64_t numbers, int64_t slots, cudaStream_t st) {
    if (slots > 0) TDX_TRY((launch_attention<T, KD, true, UP>(p, slots, st)));
    return launch_attention<T, KD, false, UP>(p, numbers, st);
}
template <typename T, int KD>
int launch_attention_pieces(const tdx::AttnParams& p, int64_t numbers, int64_t slots, cudaStream_t st) {
    if (sizeof(T) == 4 || p.state_out != nullptr) return launch_attention_passes<T, KD, 3>(p, numbers, slots, st);
    return launch_attention_passes<T, KD, sizeof(T) == 4 ? 3 : 2>(p, numbers, slots, st);
}

template <bool STATE, bool BACK, int UP>
int launch_attention_umma(const CUtensorMap (&maps)[3], const tdx::AttnParams& p, int64_t numbers, cudaStream_t st) {
    static std::atomic<bool> known[64];
    constexpr size_t kBytes = tdx::AttnUmma<STATE, UP>::kBytes + 1024;
    TDX_TRY(allow_smem(tdx::attn_umma_kernel<STATE, BACK, UP>, known, kBytes, static_cast<int>(kBytes)));
    return launch_seq(tdx::attn_umma_kernel<STATE, BACK, UP>, numbers * p.heads, 1, tdx::kAttnUmmaThreads, kBytes, st, maps[0], maps[1], maps[2], p);
}
// slots: of the pass over the states, 0 where there is none to make.  States that are handed on come from three bf16 pieces of the
// keys: out of the pass over the states where a sequence has slots, else (which leaves one tile of v) on the way.
template <bool BACK>
int launch_attention_umma_passes(const CUtensorMap (&maps)[3], const tdx::AttnParams& p, int64_t numbers, int64_t slots, bool cut, cudaStream_t st) {
    if (p.state_out && cut) {
        TDX_TRY((launch_attention_umma<true, BACK, 3>(maps, p, slots, st)));
        if (p.every) TDX_TRY((launch_attention_umma<false, BACK, 2>(maps, p, numbers, st)));
        else TDX_TRY((launch_attention_umma<false, BACK, 3>(maps, p, numbers, st)));
        // last, since state_out may be state_in, which all segments start from
        return launch_seq(tdx::attn_state_kernel, (p.every ? p.batch : p.rows / p.seg) * p.heads * 16, 1, 256, 0, st, p);
    }
    if (slots > 0) TDX_TRY((launch_attention_umma<true, BACK, 2>(maps, p, slots, st)));
    return p.state_out ? launch_attention_umma<false, BACK, 3>(maps, p, numbers, st) : launch_attention_umma<false, BACK, 2>(maps, p, numbers, st);
}

template <typename T>
int run_attention(const tdx_attention_args& a, const AttnShape& shape, AttnSum sum, const tdx_host::Device& dev, const AttnWorkspace& w, cudaStream_t st) {
    tdx::AttnParams p;
    std::memset(&p, 0, sizeof p);
    const int64_t el = sizeof(T);
    struct Role { const void* at; int64_t ld; int heads, dim; };
    const Role q = {a.q, a.ld_q, shape.q_heads, a.dim_k}, k = {a.k, a.ld_k, shape.k_heads, a.dim_k}, v = {a.v, a.ld_v, shape.v_heads, a.dim_v},
               g = {a.dout, a.ld_dout, a.heads, a.dim_v};
    const Role first = sum == kAttnOut ? q : sum == kAttnDq ? g : sum == kAttnDk ? v : k;
    const Role second = sum == kAttnOut ? k : sum == kAttnDq ? v : sum == kAttnDk ? g : q;
    const Role third = sum == kAttnOut ? v : sum == kAttnDq ? k : sum == kAttnDk ? q : g;
    struct Out { void* at; int64_t ld; int heads; };
    const Out out = sum == kAttnOut ? Out{a.out, a.ld_out, a.heads} : sum == kAttnDq ? Out{a.dq, a.ld_dq, shape.q_heads}
                    : sum == kAttnDk ? Out{a.dk, a.ld_dk, shape.k_heads} : Out{a.dv, a.ld_dv, shape.v_heads};
    p.batch = a.batch; p.max_len = a.max_len; p.rows = a.rows; p.heads = a.heads;
    p.q = first.at; p.ld_q = first.ld; p.q_share = a.heads / first.heads; p.d1 = first.dim;
    p.k = second.at; p.ld_k = second.ld; p.k_share = a.heads / second.heads;
    p.v = third.at; p.ld_v = third.ld; p.v_share = a.heads / third.heads; p.d2 = third.dim;
    const bool shared = out.heads < a.heads;
    p.out = out.at; p.ld_out = out.ld;
    if (shared) {
        p.out = static_cast<char*>(a.workspace) + w.carry;
        p.ld_out = static_cast<int64_t>(a.heads) * p.d2;
        p.out_f32 = 1;
    }
    // one answer for all sums of a pass: those of the backward pass share what a segment adds to the state
    Widest widest(16);
    auto rows = [&](const void* at, int64_t ld) { widest.ptr(at); widest.stride(ld, el); };
    widest.stride(a.dim_k, el);
    widest.stride(a.dim_v, el);
    rows(a.q, a.ld_q); rows(a.k, a.ld_k); rows(a.v, a.ld_v);
    if (sum == kAttnOut) {
        rows(a.out, a.ld_out);
    } else {
        rows(a.dout, a.ld_dout); rows(a.dq, a.ld_dq); rows(a.dk, a.ld_dk); rows(a.dv, a.ld_dv);
    }
    p.vec = widest.bytes == 16;
    Widest wide(32);
    wide.ptr(p.out); wide.stride(p.ld_out, el); wide.stride(p.d2, el);
    p.wide = wide.bytes == 32;
    const bool late = sum == kAttnDk || sum == kAttnDv;
    p.scale_in = late ? a.scale : 1.0f;
    p.scale_out = late ? 1.0f : a.scale;
    p.back = late;
    p.log_decay = a.log_decay; p.offsets = a.seq_offsets; p.slots = a.slots; p.n_slots = a.n_slots; p.state_stride = shape.state_stride;
    p.state_in = late ? a.dstate_out : a.state_in;
    p.state_out = sum == kAttnOut ? a.state_out : sum == kAttnDv ? a.dstate_in : nullptr;
    const bool turned = sum == kAttnDq || sum == kAttnDk;        // the state's columns are this sum's first dimension
    p.s1 = turned ? 1 : a.dim_v;
    p.s2 = turned ? a.dim_v : 1;
    p.state_vec = !turned && a.dim_v % 4 == 0 && p.state_stride % 4 == 0 && !misaligned(p.state_in, 16) && !misaligned(p.state_out, 16);
    p.status = dev.status;
    p.carry = static_cast<float*>(a.workspace);
    const bool umma = sizeof(T) == 2 && p.vec && a.rows > 0 && a.rows <= INT_MAX;   // (rows are coordinates of the copy engine)
    const bool all_pieces = (sum == kAttnOut ? a.state_out : late ? a.dstate_in : nullptr) != nullptr;
    plan_attention(a, p.d1, p.d2, umma, all_pieces, dev.sm_count, &p);
    // A segment on the other kernel may end, and write the state, before one in front of it has started from the state that it replaces: so
    // sequences are not cut, which costs what the cuts gain (fp32, 4096 rows, 8 heads of 128: 944 us in place, 183 apart).
    if (!umma && p.state_out != nullptr && p.state_out == p.state_in) {
        p.seg = ceil_div(std::max<int64_t>(1, a.max_len), tdx::kAttnC) * tdx::kAttnC;
        p.dense = 1;
    }
    const int64_t numbers = attention_numbers(a, p);
    const bool cut = attention_cut(a, p);
    if (umma) {
        CUtensorMap maps[3];
        const Role roles[3] = {first, second, third};
        for (int i = 0; i < 3; ++i) {
            const uint64_t dims[3] = {static_cast<uint64_t>(roles[i].dim), static_cast<uint64_t>(roles[i].heads), static_cast<uint64_t>(a.rows)};
            const uint64_t strides[2] = {static_cast<uint64_t>(roles[i].dim) * 2, static_cast<uint64_t>(roles[i].ld) * 2};
            const uint32_t box[3] = {64, 1, tdx::kAttnRows};
            TDX_TRY(tdx_host::bf16_map(roles[i].at, 3, dims, strides, box, &maps[i]));
        }
        // the state's gradient is the same for dk, which comes behind dv, with its dimensions exchanged
        p.carry_turned = sum == kAttnDk;
        const int64_t slots = cut && sum != kAttnDk ? attention_slots(a, p) : 0;
        TDX_TRY(p.back ? launch_attention_umma_passes<true>(maps, p, numbers, slots, cut, st) : launch_attention_umma_passes<false>(maps, p, numbers, slots, cut, st));
    } else {
        const int64_t slots = cut ? attention_slots(a, p) : 0;
        TDX_TRY(attention_padded(p.d1) == 64 ? (launch_attention_pieces<T, 64>(p, numbers, slots, st)) : (launch_attention_pieces<T, 128>(p, numbers, slots, st)));
    }
    if (!shared || a.rows == 0) return TDX_OK;
    const int64_t blocks = std::min<int64_t>(ceil_div(a.rows * out.heads * p.d2, 256), 16 * dev.sm_count);
    return launch_seq(tdx::attn_share_kernel<T>, blocks, 1, 256, 0, st, p.batch, p.max_len, p.rows, p.offsets, out.heads, a.heads / out.heads, p.d2,
                      static_cast<const float*>(p.out), static_cast<T*>(out.at), static_cast<long long>(out.ld));
}

int run_attention_pass(const tdx_attention_args* args, AttnPass pass, void* stream) {
    AttnShape shape;
    TDX_TRY(check_attention(args, pass, &shape));
    const tdx_attention_args& a = *args;
    if (a.batch == 0 || a.heads == 0) return TDX_OK;
    const bool back = pass == kAttnBackward;
    if (a.rows == 0 && !(back ? a.dstate_in : a.state_out)) return TDX_OK;
    tdx_host::Device dev;
    TDX_TRY(tdx_host::get_device(&dev));
    const AttnWorkspace w = attention_workspace(a, shape, dev.sm_count, back);
    TDX_TRY(check_workspace(a.workspace, a.workspace_bytes, w.total));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto run = [&](AttnSum sum) { return a.dtype == TDX_F32 ? run_attention<float>(a, shape, sum, dev, w, st) : run_attention<__nv_bfloat16>(a, shape, sum, dev, w, st); };
    if (!back) return run(kAttnOut);
    TDX_TRY(run(kAttnDq));
    TDX_TRY(run(kAttnDv));
    return run(kAttnDk);
}

}  // namespace

extern "C" {

int tdx_decay_attention(const tdx_attention_args* args, void* stream) { return run_attention_pass(args, kAttnForward, stream); }
int tdx_decay_attention_bwd(const tdx_attention_args* args, void* stream) { return run_attention_pass(args, kAttnBackward, stream); }

int tdx_decay_attention_step(const tdx_attention_args* args, void* stream) {
    AttnShape shape;
    TDX_TRY(check_attention(args, kAttnStep, &shape));
    const tdx_attention_args& a = *args;
    if (a.batch == 0 || a.heads == 0) return TDX_OK;
    tdx_host::Device dev;
    TDX_TRY(tdx_host::get_device(&dev));
    tdx::AttnParams p;
    std::memset(&p, 0, sizeof p);
    p.batch = a.batch; p.heads = a.heads; p.d1 = a.dim_k; p.d2 = a.dim_v;
    p.q = a.q; p.ld_q = a.ld_q; p.q_share = a.heads / shape.q_heads;
    p.k = a.k; p.ld_k = a.ld_k; p.k_share = a.heads / shape.k_heads;
    p.v = a.v; p.ld_v = a.ld_v; p.v_share = a.heads / shape.v_heads;
    p.out = a.out; p.ld_out = a.ld_out; p.scale_out = a.scale; p.log_decay = a.log_decay;
    p.slots = a.slots; p.n_slots = a.n_slots; p.state_stride = shape.state_stride; p.state_in = a.state_in; p.state_out = a.state_out;
    p.status = dev.status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool vec = a.dim_v % 4 == 0 && p.state_stride % 4 == 0 && !misaligned(a.state_in, 16) && !misaligned(a.state_out, 16);
    const int64_t blocks = a.batch * a.heads;
    if (a.dtype == TDX_F32)
        return vec ? launch_seq(tdx::attn_step_kernel<float, 4>, blocks, 1, tdx::kAttnStepThreads, 0, st, p) : launch_seq(tdx::attn_step_kernel<float, 1>, blocks, 1, tdx::kAttnStepThreads, 0, st, p);
    return vec ? launch_seq(tdx::attn_step_kernel<__nv_bfloat16, 4>, blocks, 1, tdx::kAttnStepThreads, 0, st, p)
               : launch_seq(tdx::attn_step_kernel<__nv_bfloat16, 1>, blocks, 1, tdx::kAttnStepThreads, 0, st, p);
}

int tdx_decay_attention_workspace_size(const tdx_attention_args* args, size_t* bytes) {
    if (bytes == nullptr) return fail(TDX_ERR_INVALID_ARG, "bytes is NULL");
    AttnShape shape;
    TDX_TRY(check_attention(args, kAttnForward, &shape, true));
    const int sm_count = sm_count_or_default();
    *bytes = attention_workspace(*args, shape, sm_count, false).total;
    if (args->dout != nullptr) *bytes = std::max(*bytes, attention_workspace(*args, shape, sm_count, true).total);
    return TDX_OK;
}

}  // extern "C"
