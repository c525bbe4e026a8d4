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

inline Segment segment(int a, bool a_mn, int b, bool b_mn, long long depth, bool fresh = true, BCols cols = B_WHOLE, bool right = false)
{
    Segment s = {};
    s.a = (unsigned char)a; s.b = (unsigned char)b;
    s.a_mn = a_mn; s.b_mn = b_mn;
    s.cols = cols; s.right = right; s.fresh = fresh;
    s.steps = (int)ceil_div(depth, 64);
    return s;
}

// Pairs of CTAs on 256 x 256 accumulators or single ones on 128 x 128 (see pair_gemm.cuh): `small` and `large` count the tiles.
inline int choose_cg(long long large, long long small, int n_sm)
{
    const long long t2 = 2 * ceil_div(large, n_sm / 2) * 4, t1 = ceil_div(small, n_sm) * 5;
    return t2 <= t1 ? 2 : 1;
}

// Both products of every column (maps 0: x, 1: w, 2: w2, 3: x2; all as they lie in memory, weights [K][F]).
inline bool products(GemmParams& p, int cg, bool wide, const Shape& s, const __nv_bfloat16* x, const __nv_bfloat16* w, const __nv_bfloat16* x2, const __nv_bfloat16* w2)
{
    const bool gated = s.K2 > 0;
    if (!in_map(&p.in[0], x, s.rows, s.K1) || !in_map(&p.in[1], w, s.K1, s.F)) return false;
    if (gated && (!in_map(&p.in[2], w2, s.K2, s.F) || !in_map(&p.in[3], x2, s.rows, s.K2))) return false;
    Group g = make_group(cg, s.rows, s.F, gated && !wide ? 64 * cg : 128 * cg);
    if (!gated) {
        g.n_seg = 1;
        g.seg[0] = segment(0, false, 1, true, s.K1);
    } else if (s.same) {
        g.n_seg = 1;
        g.seg[0] = segment(0, false, 1, true, s.K1, true, B_DUAL);
    } else {
        g.n_seg = 2;
        g.seg[0] = segment(0, false, 1, true, s.K1, true, wide ? B_WHOLE : B_HALF, false);
        g.seg[1] = segment(3, false, 2, true, s.K2, true, wide ? B_WHOLE : B_HALF, true);
    }
    p.gated = gated;
    add_group(p, g);
    return true;
}
// The launch of both products: pairs of CTAs or single ones; *wide: a whole accumulator for each product (see pair_gemm.cuh).
// Rounds of tiles times the time of one, in steps of a pair on 256 x 256: half tiles take 0.64 of one (16384 rows, 2048 and 7168 deep
// -> 2048: 520 us, wide 408; 8192 rows, twice 512 -> 8192: 149, wide 126), a wide tile about two more for what its epilogue leaves
// (8192 rows, twice 256 -> 8192: 103 and 101); where wide tiles are too few, half ones win (2048 rows, 768 and 2688 -> 768:
// 20 us, wide 25).
inline int forward_cg(const Shape& s, int n_sm, bool* wide)
{
    const long long m2 = ceil_div(s.rows, 256), m1 = ceil_div(s.rows, 128);
    *wide = false;
    if (s.K2 == 0 || s.same) {
        const int w = s.K2 > 0 ? 64 : 128;
        return choose_cg(m2 * ceil_div(s.F, 2 * w), m1 * ceil_div(s.F, w), n_sm);
    }
    const long long steps = ceil_div(s.K1, 64) + ceil_div(s.K2, 64);
    const long long t_wide = ceil_div(m2 * ceil_div(s.F, 256), n_sm / 2) * (steps + 2) * 100;
    const long long t_half = ceil_div(m2 * ceil_div(s.F, 128), n_sm / 2) * steps * 64, t_one = ceil_div(m1 * ceil_div(s.F, 64), n_sm) * steps * 45;
    *wide = t_wide <= t_half && t_wide <= t_one;
    return *wide || t_half <= t_one ? 2 : 1;
}

}  // namespace gl

inline gf_status_t gated_linear(const __nv_bfloat16* x, const __nv_bfloat16* w, const __nv_bfloat16* x2, const __nv_bfloat16* w2, int act,
                                __nv_bfloat16* y, const gl::Shape& s, cudaStream_t st, std::atomic<uint64_t>* launches)
{
    const int n_sm = sm_count();
    if (n_sm < 2) return GF_ERR_CUDA;
    pg::GemmParams p = {};
    p.act = act;
    bool wide;
    const int cg = gl::forward_cg(s, n_sm, &wide);
    if (!gl::products(p, cg, wide, s, x, w, x2, w2) || !pg::out_map(&p.out[0], y, s.rows, s.F)) return GF_ERR_CUDA;
    return pg::launch<pg::EPI_GATE>(cg, p, st, launches, wide);
}

// Workspace of the gradient: da and, where there is a second product, db, [rows][F] bf16 each.
inline size_t gated_linear_backward_bytes(long long rows, int F, bool gated) { return (size_t)rows * F * 2 * (gated ? 2 : 1); }

inline gf_status_t gated_linear_backward(const __nv_bfloat16* x, const __nv_bfloat16* w, const __nv_bfloat16* x2, const __nv_bfloat16* w2, int act,
                                         const __nv_bfloat16* dy, __nv_bfloat16* dx, __nv_bfloat16* dw, __nv_bfloat16* dx2, __nv_bfloat16* dw2,
                                         const gl::Shape& s, __nv_bfloat16* ws, cudaStream_t st, std::atomic<uint64_t>* launches)
{
    using namespace gl;
    const int n_sm = sm_count();
    if (n_sm < 2) return GF_ERR_CUDA;
    const bool gated = s.K2 > 0;
    __nv_bfloat16 *da = ws, *db = ws + (size_t)s.rows * s.F;
    {
        GemmParams p = {};
        p.act = act;
        p.dy = dy;
        bool wide;
        const int cg = forward_cg(s, n_sm, &wide);
        if (!products(p, cg, wide, s, x, w, x2, w2) || !out_map(&p.out[0], da, s.rows, s.F) || (gated && !out_map(&p.out[1], db, s.rows, s.F))) return GF_ERR_CUDA;
        const gf_status_t e = launch<EPI_GATE_GRAD>(cg, p, st, launches, wide);
        if (e != GF_OK) return e;
    }
    GemmParams p = {};
    // maps 0: da, 1: db, 2: w, 3: w2, 4: x, 5: x2
    if (!in_map(&p.in[0], da, s.rows, s.F) || !in_map(&p.in[2], w, s.K1, s.F) || !in_map(&p.in[4], x, s.rows, s.K1) || !out_map(&p.out[0], dx, s.rows, s.K1) ||
        !out_map(&p.out[1], dw, s.K1, s.F))
        return GF_ERR_CUDA;
    if (gated && (!in_map(&p.in[1], db, s.rows, s.F) || !in_map(&p.in[3], w2, s.K2, s.F) || !in_map(&p.in[5], x2, s.rows, s.K2) || !out_map(&p.out[3], dw2, s.K2, s.F) ||
                  (!s.same && !out_map(&p.out[2], dx2, s.rows, s.K2))))
        return GF_ERR_CUDA;
    auto tiles = [&](int c) {
        long long n = ceil_div(s.rows, 128 * c) * ceil_div(s.K1, 128 * c) + ceil_div(s.K1, 128 * c) * ceil_div(s.F, 128 * c);
        if (gated) n += (s.same ? 0 : ceil_div(s.rows, 128 * c) * ceil_div(s.K2, 128 * c)) + ceil_div(s.K2, 128 * c) * ceil_div(s.F, 128 * c);
        return n;
    };
    const int cg = choose_cg(tiles(2), tiles(1), n_sm);
    auto group = [&](long long m, long long n, int out, Segment a) {
        Group g = make_group(cg, m, n, 128 * cg);
        g.n_seg = 1;
        g.seg[0] = a;
        g.out = (unsigned char)out;
        g.mode = OUT_BF16;
        return g;
    };
    Group gx = group(s.rows, s.K1, 0, segment(0, false, 2, false, s.F));
    if (gated && s.same) {
        gx.seg[gx.n_seg++] = segment(1, false, 3, false, s.F, false);
    }
    const Group gw = group(s.K1, s.F, 1, segment(4, true, 0, true, s.rows));
    add_group(p, gx);
    if (gated && !s.same) add_group(p, group(s.rows, s.K2, 2, segment(1, false, 3, false, s.F)));
    add_group(p, gw);
    if (gated) add_group(p, group(s.K2, s.F, 3, segment(5, true, 1, true, s.rows)));
    return launch<EPI_STORE>(cg, p, st, launches);
}

}  // namespace gf
