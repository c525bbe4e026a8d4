// The gated linear block and its gradient: y = act(x W) * (x2 W2), elementwise over the columns, with the second factor left out
// where there is no W2.  The paper's channel mix is two of these, h = relu(x_k W_k)^2 and o = sigmoid(x_r W_r) * (h W_v)
// (channel-mix equations); x2 = x is the usual gated hidden layer.
//
// Forward: one launch of pair_gemm_kernel; a tile's left half holds columns of x W, its right half the same columns of x2 W2, so
// neither product leaves the SM.  Gradient: one launch recomputes both products and writes, rounded to bf16 (they are operands of
// the products that follow, whose results are rounded to bf16 too),
//     da = dy * b * act'(a),   db = dy * act(a)        (a = x W, b = x2 W2)
// and a second one computes dx = da W^T, dx2 = db W2^T (x2 = x: their sum, in one accumulator), dW = x^T da, dW2 = x2^T db.
#pragma once
#include "pair_gemm.cuh"

namespace gf {
namespace gl {

using namespace pg;

struct Shape {
    long long rows;
    int K1, K2, F;                  // K2 = 0: no second product
    bool same;                      // x2 is x
};

// Pairs of CTAs on 256 x 256 accumulators or single ones on 128 x 128 (see pair_gemm.cuh): `large` and `small` count the tiles.
inline int choose_cg(long long large, long long small, int n_sm)
{
    return ceil_div(large, n_sm / 2) * STEP_TIME[2] <= ceil_div(small, n_sm) * STEP_TIME[1] ? 2 : 1;
}

// Both products of every column (maps 0: x, 1: w, 2: w2, 3: x2; all as they lie in memory, weights [K][F]).
inline bool products(GemmParams& p, const Launch& l, const Shape& s, const __nv_bfloat16* x, const __nv_bfloat16* w, const __nv_bfloat16* x2, const __nv_bfloat16* w2)
{
    const bool gated = s.K2 > 0;
    if (!in_map(p, 0, x, s.rows, s.K1) || !in_map(p, 1, w, s.K1, s.F)) return false;
    if (gated && (!in_map(p, 2, w2, s.K2, s.F) || !in_map(p, 3, x2, s.rows, s.K2))) return false;
    const bool whole = l.mode != TILES;               // an accumulator of a whole tile's columns for each product
    Group g = make_group(l.cg, s.rows, s.F, gated && !whole ? 64 * l.cg : 128 * l.cg);
    if (!gated || (s.same && !whole)) {
        add_segment(g, segment(0, false, 1, true, s.K1, gated ? B_DUAL : B_WHOLE));
    } else {
        add_segment(g, segment(0, false, 1, true, s.K1, whole ? B_WHOLE : B_HALF, false));
        add_segment(g, segment(3, false, 2, true, s.K2, whole ? B_WHOLE : B_HALF, true));
    }
    p.gated = gated;
    p.n_groups = p.n_tiles = 0;
    add_group(p, g);
    return true;
}
// How both products are launched: rounds of tiles times the time of one, in units of 1/30 us (STEP_TIME's).
//  - Products of half a tile's columns take 0.64 of a whole tile's step (16384 rows, 2048 and 7168 deep -> 2048: 520 us, wide 408; 8192
//    rows, twice 512 -> 8192: 149, wide 126), a wide tile about two steps more for what its epilogue leaves (8192 rows, twice 256
//    -> 8192: 103 and 101); where wide tiles are too few, half ones win (2048 rows, 768 and 2688 -> 768: 20 us, wide 25).
//  - A tile that a cluster divides costs the joining, 2 us; all clusters have to run at one time.
inline Launch forward_launch(const Shape& s, int n_sm, bool clusters, bool split)
{
    const long long m2 = ceil_div(s.rows, 256), m1 = ceil_div(s.rows, 128), s1 = ceil_div(s.K1, 64), s2 = ceil_div(s.K2, 64), both = s1 + s2;
    auto rounds = [&](long long tiles, int units) { return ceil_div(tiles, units); };
    if (!clusters) return SINGLE;
    Launch best = {2, TILES, 2};
    long long time;
    auto offer = [&](int cg, Mode mode, int cluster, long long t) {
        if (t < time) {
            time = t;
            best = Launch{cg, mode, cluster};
        }
    };
    if (s.K2 == 0 || s.same) {
        const int w = s.K2 > 0 ? 64 : 128;
        time = rounds(m2 * ceil_div(s.F, 2 * w), n_sm / 2) * s1 * STEP_TIME[2];
        offer(1, TILES, 1, rounds(m1 * ceil_div(s.F, w), n_sm) * s1 * STEP_TIME[1]);
    } else {
        time = rounds(m2 * ceil_div(s.F, 128), n_sm / 2) * both * 5;
        offer(2, WIDE_TILES, 2, rounds(m2 * ceil_div(s.F, 256), n_sm / 2) * (both + 2) * STEP_TIME[2]);
        offer(1, TILES, 1, rounds(m1 * ceil_div(s.F, 64), n_sm) * both * 6);
    }
    const long long tiles = m1 * ceil_div(s.F, 128);
    for (int c = 8; split && c >= 2; --c)          // (two steps at least for each CTA)
        if (tiles * c <= n_sm && both >= 2 * c && tiles <= clusters_at_once(c, n_sm)) offer(1, SPLIT_TILES, c, ceil_div(both, c) * STEP_TIME[1] + 60);
    return best;
}

}  // namespace gl

inline gf_status_t gated_linear(const __nv_bfloat16* x, const __nv_bfloat16* w, const __nv_bfloat16* x2, const __nv_bfloat16* w2, int act,
                                __nv_bfloat16* y, const gl::Shape& s, cudaStream_t st, std::atomic<uint64_t>* launches)
{
    const int n_sm = sm_count();
    if (n_sm < 2) return GF_ERR_CUDA;
    pg::GemmParams p = {};
    p.act = act;
    p.y = y;
    if (!pg::out_map(&p.out[0], y, s.rows, s.F)) return GF_ERR_CUDA;
    for (const bool clusters : {true, false}) {       // (without any where the device refuses them)
        const pg::Launch l = gl::forward_launch(s, n_sm, clusters, true);
        if (!gl::products(p, l, s, x, w, x2, w2)) return GF_ERR_CUDA;
        if (pg::launch<pg::EPI_GATE>(l, p, st, launches)) return GF_OK;
    }
    return GF_ERR_CUDA;
}

namespace gl {
// The gradient's products.  Maps 0: da, 1: db, 2: w, 3: w2, 4: x, 5: x2, 6, 7: what rounding left of da, db (keep_rests()).
inline int gradient_products(const Shape& s, Product (&q)[MAX_GROUPS], __nv_bfloat16* dx, __nv_bfloat16* dw, __nv_bfloat16* dx2, __nv_bfloat16* dw2)
{
    const bool gated = s.K2 > 0, rests = keep_rests(s.rows);
    int n = 0;
    auto add = [](Product& p, const Segment& g) { p.seg[p.n_seg++] = g; };
    auto by_weights = [&](Product& p, int d, int w) {            // d w^T
        add(p, segment(d, false, w, false, s.F));
        if (rests) add(p, segment(d + 6, false, w, false, s.F));
    };
    auto by_inputs = [&](Product& p, int x, int d) {             // x^T d
        add(p, segment(x, true, d, true, s.rows));
        if (rests) add(p, segment(x, true, d + 6, true, s.rows));
    };
    Product& px = q[n++] = Product{s.rows, s.K1, 0, {}, dx};
    by_weights(px, 0, 2);
    if (gated && s.same) by_weights(px, 1, 3);
    by_inputs(q[n++] = Product{s.K1, s.F, 0, {}, dw}, 4, 0);
    if (gated) {
        by_inputs(q[n++] = Product{s.K2, s.F, 0, {}, dw2}, 5, 1);
        if (!s.same) by_weights(q[n++] = Product{s.rows, s.K2, 0, {}, dx2}, 1, 3);
    }
    return n;
}
inline size_t one_operand(const Shape& s) { return ((size_t)s.rows * s.F * 2 + 255) & ~(size_t)255; }
inline size_t operand_bytes(const Shape& s) { return one_operand(s) * (s.K2 > 0 ? 2 : 1) * (keep_rests(s.rows) ? 2 : 1); }
}  // namespace gl

// Workspace of the gradient: da and, where there is a second product, db, [rows][F] bf16 each (and of few rows what rounding left of them), and the sums of
// products that are cut.
inline size_t gated_linear_backward_bytes(const gl::Shape& s)
{
    pg::Product q[pg::MAX_GROUPS];
    const int n = gl::gradient_products(s, q, nullptr, nullptr, nullptr, nullptr);
    return gl::operand_bytes(s) + pg::plan_products(q, n, pg::plan_sms(), false).bytes;
}

inline gf_status_t gated_linear_backward(const __nv_bfloat16* x, const __nv_bfloat16* w, const __nv_bfloat16* x2, const __nv_bfloat16* w2, int act,
                                         const __nv_bfloat16* dy, __nv_bfloat16* dx, __nv_bfloat16* dw, __nv_bfloat16* dx2, __nv_bfloat16* dw2,
                                         const gl::Shape& s, __nv_bfloat16* ws, cudaStream_t st, std::atomic<uint64_t>* launches)
{
    using namespace gl;
    const int n_sm = sm_count();
    if (n_sm < 2) return GF_ERR_CUDA;
    const bool gated = s.K2 > 0, rests = keep_rests(s.rows);
    __nv_bfloat16* d[4];                              // da, db, and what rounding left of them
    for (int i = 0; i < 4; ++i) d[i] = ws + one_operand(s) / 2 * (gated ? i : i / 2);
    bool done = false;
    for (const bool clusters : {true, false}) {
        GemmParams p = {};
        p.act = act;
        p.dy = dy;
        const Launch l = rests ? SINGLE : forward_launch(s, n_sm, clusters, false);
        if (!products(p, l, s, x, w, x2, w2)) return GF_ERR_CUDA;
        for (int i = 0; i < 4; ++i)
            if ((i % 2 == 0 || gated) && (i < 2 || rests) && !out_map(&p.out[i], d[i], s.rows, s.F)) return GF_ERR_CUDA;
        if ((done = rests ? launch<EPI_GATE_GRAD_RESTS>(l, p, st, launches) : launch<EPI_GATE_GRAD>(l, p, st, launches))) break;
    }
    if (!done) return GF_ERR_CUDA;
    GemmParams p = {};
    if (!in_map(p, 0, d[0], s.rows, s.F) || !in_map(p, 2, w, s.K1, s.F) || !in_map(p, 4, x, s.rows, s.K1) || (rests && !in_map(p, 6, d[2], s.rows, s.F))) return GF_ERR_CUDA;
    if (gated && (!in_map(p, 1, d[1], s.rows, s.F) || !in_map(p, 3, w2, s.K2, s.F) || !in_map(p, 5, x2, s.rows, s.K2) || (rests && !in_map(p, 7, d[3], s.rows, s.F))))
        return GF_ERR_CUDA;
    Product q[MAX_GROUPS];
    const int n = gradient_products(s, q, dx, dw, dx2, dw2);
    Plan plan = plan_products(q, n, plan_sms(), false);
    return run_products(p, q, n, plan, PART_ONLY, reinterpret_cast<char*>(ws) + operand_bytes(s), st, launches);
}

}  // namespace gf
