// Cross entropy of a linear layer over a vocabulary, without the logits: for every row
//     z = x W^T,   lse = log sum_v exp z_v,   loss = lse - z_target        (W: [V][D]; loss 0 where there is no target)
// and its gradient, with P = (softmax z - [v is the target]) dloss,
//     dx = P W,   dW = P^T x.
//
// Forward: pair_gemm_kernel makes 256 (128) columns of logits at a time and keeps of each row and half of them a reference value and the
// sum of exponentials over it; a second kernel joins them.  Gradient: pieces of the vocabulary, each one launch that computes the
// piece's logits again and writes its columns of P in bf16 (they are an operand of two products whose results are bf16), and one
// that computes the piece's rows of dW and adds its part of dx, kept in fp32 until the last piece.
#pragma once
#include "gated_linear.cuh"

namespace gf {
namespace vl {

using namespace pg;
using gl::choose_cg;

constexpr int JOIN_THREADS = 512;

// stats [tiles][rows] -> lse, loss.  A block takes ROWS rows, JOIN_THREADS / ROWS threads sharing the tiles of each out between them: 32
// rows read whole lines; a call with fewer has more threads on each (7 rows, 626 half tiles: 10 us with 32 rows to a block).
template <int ROWS>
__global__ void __launch_bounds__(JOIN_THREADS) join_kernel(const float2* __restrict__ stats, const float* __restrict__ target_logit,
                                                            const long long* __restrict__ targets, long long vocab, int tiles, int rows,
                                                            float* __restrict__ loss, float* __restrict__ lse)
{
    constexpr int SHARES = JOIN_THREADS / ROWS;
    __shared__ float2 part[SHARES][ROWS];
    asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
    const int share = threadIdx.x / ROWS, r = threadIdx.x % ROWS, row = blockIdx.x * ROWS + r;
    float ref = -INFINITY, sum = 0.f;
    // (references are finite, so a first one's factor below is exp(-inf) = 0; an infinite sum's is FLT_MAX, so its own factor is 1)
    auto join = [&](float2 o) {
        const float top = fmaxf(ref, o.x);
        sum = sum * __expf(ref - top) + o.y * __expf(o.x - top);
        ref = top;
    };
    if (row < rows) {
        int t = share;
        for (; t + 3 * SHARES < tiles; t += 4 * SHARES) {
            float2 o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = stats[(size_t)(t + q * SHARES) * rows + row];
#pragma unroll
            for (int q = 0; q < 4; ++q) join(o[q]);
        }
        for (; t < tiles; t += SHARES) join(stats[(size_t)t * rows + row]);
    }
    part[share][r] = make_float2(ref, sum);
#pragma unroll
    for (int h = SHARES / 2; h > 0; h /= 2) {         // (a share without tiles has -inf and joins nothing)
        __syncthreads();
        if (share < h && part[share + h][r].x > -INFINITY) {
            join(part[share + h][r]);
            part[share][r] = make_float2(ref, sum);
        }
    }
    if (share == 0 && row < rows) {
        const float l = ref + logf(sum);
        const long long t = targets[row];
        lse[row] = l;
        loss[row] = t >= 0 && t < vocab ? l - target_logit[row] : 0.f;
    }
}

inline int forward_cg(long long rows, long long cols, int n_sm)
{
    return choose_cg(ceil_div(rows, 256) * ceil_div(cols, 256), ceil_div(rows, 128) * ceil_div(cols, 128), n_sm);
}

// The launch's one group: logits of rows x cols (maps 0: x, 1: the columns' rows of W).
inline void logits(GemmParams& p, int cg, long long rows, int D, long long cols)
{
    Group g = make_group(cg, rows, cols, 128 * cg);
    add_segment(g, segment(0, false, 1, false, D));
    p.n_groups = p.n_tiles = 0;
    add_group(p, g);
}

// Columns of P that the gradient holds at a time: 256 MB of them, between 1024 and the vocabulary, in equal pieces.
inline long long piece_cols(long long rows, long long V)
{
    long long most = (128LL << 20) / rows / 256 * 256;
    if (most < 1024) most = 1024;
    const long long n = ceil_div(V, most);
    return ceil_div(ceil_div(V, n), 256) * 256;
}

}  // namespace vl

inline size_t round_256(size_t n) { return (n + 255) & ~(size_t)255; }
// Forward: the statistics of every half tile of columns (64 at least), and the targets' logits.
inline size_t vocab_stats_bytes(long long rows, long long V) { return round_256((size_t)rows * 2 * pg::ceil_div(V, 128) * sizeof(float2)); }
inline size_t vocab_loss_bytes(long long rows, long long V) { return vocab_stats_bytes(rows, V) + (size_t)rows * 4; }
namespace vl {
// A piece's products: its part of dx (map 0: P, 1: the piece's rows of W) and its rows of dW (2: x); 3: what rounding left of P (keep_rests()).
inline void gradient_products(Product (&q)[2], long long rows, int D, long long cols, __nv_bfloat16* dx, __nv_bfloat16* dw)
{
    const int n = keep_rests(rows) ? 2 : 1;
    q[0] = Product{rows, D, n, {segment(0, false, 1, true, cols), segment(3, false, 1, true, cols)}, dx};
    q[1] = Product{cols, D, n, {segment(0, true, 2, true, rows), segment(3, true, 2, true, rows)}, dw};
}
// (all pieces are cut like the first, the largest)
inline Plan gradient_plan(long long rows, int D, long long V)
{
    const long long step = piece_cols(rows, V);
    Product q[2];
    gradient_products(q, rows, D, step < V ? step : V, nullptr, nullptr);
    return plan_products(q, 2, plan_sms(), step < V);
}
inline size_t one_piece(long long rows, long long V) { return ((size_t)rows * piece_cols(rows, V) * 2 + 255) & ~(size_t)255; }
inline size_t piece_bytes(long long rows, long long V) { return one_piece(rows, V) * (keep_rests(rows) ? 2 : 1); }
}  // namespace vl

// Gradient: a piece of P (of few rows what rounding left of it too), and fp32 sums of dx over the pieces and of products that are cut.
inline size_t vocab_loss_backward_bytes(long long rows, int D, long long V) { return vl::piece_bytes(rows, V) + vl::gradient_plan(rows, D, V).bytes; }

inline gf_status_t vocab_loss(const __nv_bfloat16* x, const __nv_bfloat16* w, const long long* targets, float* loss, float* lse, long long rows,
                              int D, long long V, void* ws, cudaStream_t st, std::atomic<uint64_t>* launches)
{
    using namespace vl;
    const int n_sm = sm_count();
    if (n_sm < 2) return GF_ERR_CUDA;
    GemmParams p = {};
    if (!in_map(p, 0, x, rows, D) || !in_map(p, 1, w, V, D)) return GF_ERR_CUDA;
    p.targets = targets;
    p.vocab = V;
    p.stats = static_cast<float2*>(ws);
    p.target_logit = reinterpret_cast<float*>(static_cast<char*>(ws) + vocab_stats_bytes(rows, V));
    int cg = forward_cg(rows, V, n_sm);
    logits(p, cg, rows, D, V);
    if (!launch<EPI_LSE>(Launch{cg, TILES, cg}, p, st, launches)) {
        if (cg == 1) return GF_ERR_CUDA;
        logits(p, cg = 1, rows, D, V);
        if (!launch<EPI_LSE>(SINGLE, p, st, launches)) return GF_ERR_CUDA;
    }
    auto join = rows >= 1024 ? join_kernel<32> : rows >= 256 ? join_kernel<8> : join_kernel<1>;
    const int block_rows = rows >= 1024 ? 32 : rows >= 256 ? 8 : 1;
    const cudaError_t e = launch_pdl(join, (unsigned)ceil_div(rows, block_rows), JOIN_THREADS, 0, st, (const float2*)p.stats, (const float*)p.target_logit, targets, V,
                                     2 * p.g[0].tiles_n, (int)rows, loss, lse);
    launches->fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? GF_OK : GF_ERR_CUDA;
}

inline gf_status_t vocab_loss_backward(const __nv_bfloat16* x, const __nv_bfloat16* w, const long long* targets, const float* lse, const float* dloss,
                                       __nv_bfloat16* dx, __nv_bfloat16* dw, long long rows, int D, long long V, void* ws, cudaStream_t st,
                                       std::atomic<uint64_t>* launches)
{
    using namespace vl;
    const int n_sm = sm_count();
    if (n_sm < 2) return GF_ERR_CUDA;
    const long long step = piece_cols(rows, V);
    Plan plan = gradient_plan(rows, D, V);
    __nv_bfloat16 *P = static_cast<__nv_bfloat16*>(ws), *P_rest = P + one_piece(rows, V) / 2;
    const bool rests = keep_rests(rows);
    for (long long v0 = 0; v0 < V; v0 += step) {
        const long long cols = V - v0 < step ? V - v0 : step;
        const long long pitch = (cols + 7) / 8 * 8;               // (a row of a tensor map is a multiple of 16 bytes; the last columns are zero)
        const __nv_bfloat16* wp = w + (size_t)v0 * D;
        {
            GemmParams p = {};
            if (!in_map(p, 0, x, rows, D) || !in_map(p, 1, wp, cols, D) || !out_map(&p.out[0], P, rows, pitch) || (rests && !out_map(&p.out[1], P_rest, rows, pitch)))
                return GF_ERR_CUDA;
            p.targets = targets;
            p.vocab = V;
            p.first_col = (int)v0;
            p.lse = lse;
            p.dloss = dloss;
            const int cg = rests ? 1 : forward_cg(rows, cols, n_sm);
            logits(p, cg, rows, D, cols);
            if (!(rests ? launch<EPI_PROB_RESTS>(SINGLE, p, st, launches) : launch<EPI_PROB>(Launch{cg, TILES, cg}, p, st, launches))) {
                if (cg == 1) return GF_ERR_CUDA;
                logits(p, 1, rows, D, cols);
                if (!launch<EPI_PROB>(SINGLE, p, st, launches)) return GF_ERR_CUDA;
            }
        }
        GemmParams p = {};
        const bool first = v0 == 0, last = v0 + step >= V;
        if (!in_map(p, 0, P, rows, pitch) || !in_map(p, 1, wp, cols, D) || !in_map(p, 2, x, rows, D) || (rests && !in_map(p, 3, P_rest, rows, pitch))) return GF_ERR_CUDA;
        Product q[2];
        gradient_products(q, rows, D, cols, dx, dw + (size_t)v0 * D);
        const gf_status_t s = run_products(p, q, 2, plan, first ? (last ? PART_ONLY : PART_FIRST) : last ? PART_LAST : PART_MIDDLE,
                                           static_cast<char*>(ws) + piece_bytes(rows, V), st, launches);
        if (s != GF_OK) return s;
    }
    return GF_OK;
}

}  // namespace gf
