// Gradient of the LayerNorm across all heads (ln_heads.cuh): with mu, rstd the row's statistics, xhat = (y - mu) rstd and
// g = dout * gamma,
//     dy = rstd (g - mean(g) - xhat mean(g xhat)),   dgamma = sum over rows of dout * xhat,   dbeta = sum over rows of dout.
// The statistics are taken from y again (it is read anyway), so the forward call keeps nothing.
//
// Bound by HBM (2 D elements in, D out per token).  As in the forward kernel a team of W warps owns whole rows and a lane the
// 8-channel slices l + 32*W*j of them, raw slices of the next group being loaded while the current one is worked on; here a
// lane also carries the sums of dgamma and dbeta over all its rows in registers (so at most four bf16 or two fp32 slices per lane:
// y, dout, their prefetch and the sums fill the register file).  One exchange per row: each warp's mean, squared
// deviations, sum of g and sum of g (y - its mean), joined by the pairwise formulae.  At the end a CTA adds its teams' sums up in
// shared memory in a fixed order and leaves one row of each in the workspace; a second kernel adds those over the CTAs.
#pragma once
#include "ln_heads.cuh"

namespace gf {
namespace lng {

using ln::Raw;
using ln::add2;
using ln::fma2;
using ln::mul2;
using ln::warp_sum;

// bf16: eight warps with up to 255 registers a thread; fp32: sixteen with up to 128
template <typename IO> constexpr int cta_threads() { return sizeof(IO) == 2 ? 256 : 512; }
template <typename IO> constexpr int max_slices() { return sizeof(IO) == 2 ? 4 : 2; }
constexpr int rows_per_group(int max_vpl, int vpl) { return max_vpl / vpl; }

template <typename IO, int VPL, int W>
constexpr int smem_bytes() { return VPL * 2 * 32 * W * 16 * 3; }      // gamma, and the sums of dgamma and dbeta, as float4 [VPL][2][32 W]

template <typename IO, int VPL, int W>
__global__ void __launch_bounds__(cta_threads<IO>(), 1)
layernorm_heads_grad_kernel(const IO* __restrict__ y, const IO* __restrict__ dout, const float* __restrict__ gamma, float eps, IO* __restrict__ dy,
                            float* __restrict__ sums, long long rows, int D)
{
    constexpr int R = rows_per_group(max_slices<IO>(), VPL);
    constexpr int THREADS = cta_threads<IO>();
    constexpr int TEAMS = THREADS / 32 / W;
    constexpr int TL = 32 * W;
    extern __shared__ float4 sh[];                  // gamma [VPL][2][TL], dgamma, dbeta
    __shared__ float4 part[TEAMS][2][R][W];         // per warp: mean, squared deviations, sum of g, sum of g (y - mean); by group parity
    __shared__ float cnt[THREADS / 32];             // channels that each warp holds
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int team = warp / W, wt = warp % W, tl = wt * 32 + lane;
    asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");

    for (int idx = tid; idx < VPL * 2 * TL; idx += THREADS) {
        const int j = idx / (2 * TL), half = (idx / TL) & 1, l = idx % TL;
        const int c = 8 * (l + TL * j) + 4 * half;
        float4 gv = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < D) gv = gamma ? *reinterpret_cast<const float4*>(gamma + c) : make_float4(1.f, 1.f, 1.f, 1.f);
        sh[idx] = gv;
        sh[VPL * 2 * TL + idx] = sh[2 * VPL * 2 * TL + idx] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    int col[VPL];
    bool on[VPL];
    float mine = 0.f;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
        col[j] = 8 * (tl + TL * j);
        on[j] = col[j] < D;
        mine += on[j] ? 8.f : 0.f;
    }
    const float n_w = warp_sum(mine), inv_nw = 1.f / n_w;   // every warp holds at least one slice (host picks W, VPL)
    if (lane == 0) cnt[warp] = n_w;
    __syncthreads();
    const float inv_d = 1.f / (float)D;

    auto load_group = [&](Raw<IO> (&ry)[R][VPL], Raw<IO> (&rd)[R][VPL], long long r0) {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                if (on[j] && r0 + i < rows) {
                    ln::load_raw(y + (size_t)(r0 + i) * D + col[j], ry[i][j]);
                    ln::load_raw(dout + (size_t)(r0 + i) * D + col[j], rd[i][j]);
                } else {
                    ln::zero_raw(ry[i][j]);
                    ln::zero_raw(rd[i][j]);
                }
            }
    };

    float2 dg[VPL][4], db[VPL][4];                  // this lane's sums over its rows
#pragma unroll
    for (int j = 0; j < VPL; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) dg[j][e] = db[j][e] = make_float2(0.f, 0.f);

    const long long stride = (long long)gridDim.x * TEAMS * R;
    long long r0 = ((long long)blockIdx.x * TEAMS + team) * R;
    Raw<IO> ny[R][VPL], nd[R][VPL];
    if (r0 < rows) load_group(ny, nd, r0);
    int par = 0;
    for (; r0 < rows; r0 += stride, par ^= 1) {
        float2 x[R][VPL][4], d[R][VPL][4];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                ln::unpack(ny[i][j], x[i][j]);
                ln::unpack(nd[i][j], d[i][j]);
            }
        if (r0 + stride < rows) load_group(ny, nd, r0 + stride);

        float mu[R], m2[R], sg[R], sgx[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float2 s2 = make_float2(0.f, 0.f), g2 = s2;
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                const float4 g0 = sh[(2 * j) * TL + tl], g1 = sh[(2 * j + 1) * TL + tl];
                const float2 gm[4] = {make_float2(g0.x, g0.y), make_float2(g0.z, g0.w), make_float2(g1.x, g1.y), make_float2(g1.z, g1.w)};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s2 = add2(s2, x[i][j][e]);
                    g2 = fma2(d[i][j][e], gm[e], g2);
                }
            }
            mu[i] = s2.x + s2.y;
            sg[i] = g2.x + g2.y;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < R; ++i) {
                mu[i] += __shfl_xor_sync(0xffffffffu, mu[i], o);
                sg[i] += __shfl_xor_sync(0xffffffffu, sg[i], o);
            }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            mu[i] *= inv_nw;
            const float2 neg_m = make_float2(-mu[i], -mu[i]);
            float2 q2 = make_float2(0.f, 0.f), p2 = q2;
#pragma unroll
            for (int j = 0; j < VPL; ++j)
                if (on[j]) {
                    const float4 g0 = sh[(2 * j) * TL + tl], g1 = sh[(2 * j + 1) * TL + tl];
                    const float2 gm[4] = {make_float2(g0.x, g0.y), make_float2(g0.z, g0.w), make_float2(g1.x, g1.y), make_float2(g1.z, g1.w)};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 c = add2(x[i][j][e], neg_m);
                        q2 = fma2(c, c, q2);
                        p2 = fma2(mul2(d[i][j][e], gm[e]), c, p2);
                    }
                }
            m2[i] = q2.x + q2.y;
            sgx[i] = p2.x + p2.y;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < R; ++i) {
                m2[i] += __shfl_xor_sync(0xffffffffu, m2[i], o);
                sgx[i] += __shfl_xor_sync(0xffffffffu, sgx[i], o);
            }
        if (W > 1) {
            // ---- merge the team's warps: deviations from the common mean m are those from the warp's plus (its mean - m)
            if (lane == 0) {
#pragma unroll
                for (int i = 0; i < R; ++i) part[team][par][i][wt] = make_float4(mu[i], m2[i], sg[i], sgx[i]);
            }
            asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(TL) : "memory");
#pragma unroll
            for (int i = 0; i < R; ++i) {
                float m = 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) m = fmaf(cnt[team * W + w], part[team][par][i][w].x, m);
                m *= inv_d;
                float q = 0.f, s = 0.f, p = 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const float4 pw = part[team][par][i][w];
                    const float dm = pw.x - m;
                    q += fmaf(cnt[team * W + w] * dm, dm, pw.y);
                    s += pw.z;
                    p += fmaf(pw.z, dm, pw.w);
                }
                mu[i] = m;
                m2[i] = q;
                sg[i] = s;
                sgx[i] = p;
            }
            // part[team][par] is next written two groups on, after the barrier of the group between
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (r0 + i >= rows) break;
            const float rstd = rsqrtf(fmaf(m2[i], inv_d, eps));
            const float mg = sg[i] * inv_d, mgx = sgx[i] * rstd * inv_d;
            const float2 neg_mu = make_float2(-mu[i], -mu[i]), r2 = make_float2(rstd, rstd);
            const float2 neg_mg = make_float2(-mg, -mg), neg_mgx = make_float2(-mgx, -mgx);
#pragma unroll
            for (int j = 0; j < VPL; ++j)
                if (on[j]) {
                    const float4 g0 = sh[(2 * j) * TL + tl], g1 = sh[(2 * j + 1) * TL + tl];
                    const float2 gm[4] = {make_float2(g0.x, g0.y), make_float2(g0.z, g0.w), make_float2(g1.x, g1.y), make_float2(g1.z, g1.w)};
                    float2 o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 xh = mul2(add2(x[i][j][e], neg_mu), r2);
                        dg[j][e] = fma2(d[i][j][e], xh, dg[j][e]);
                        db[j][e] = add2(db[j][e], d[i][j][e]);
                        o[e] = mul2(fma2(xh, neg_mgx, fma2(d[i][j][e], gm[e], neg_mg)), r2);
                    }
                    ln::store8(dy + (size_t)(r0 + i) * D + col[j], o);
                }
        }
    }

    if (!sums) return;
    // ---- the CTA's sums: the teams one after another, each into its own lanes' places
    float4* sg4 = sh + VPL * 2 * TL;
    float4* sb4 = sg4 + VPL * 2 * TL;
    for (int t = 0; t < TEAMS; ++t) {
        __syncthreads();
        if (team == t) {
#pragma unroll
            for (int j = 0; j < VPL; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int at = (2 * j + h) * TL + tl;
                    float4 a = sg4[at], b = sb4[at];
                    a.x += dg[j][2 * h].x; a.y += dg[j][2 * h].y; a.z += dg[j][2 * h + 1].x; a.w += dg[j][2 * h + 1].y;
                    b.x += db[j][2 * h].x; b.y += db[j][2 * h].y; b.z += db[j][2 * h + 1].x; b.w += db[j][2 * h + 1].y;
                    sg4[at] = a;
                    sb4[at] = b;
                }
        }
    }
    __syncthreads();
    float* mine_g = sums + (size_t)blockIdx.x * 2 * D;
    for (int idx = tid; idx < VPL * 2 * TL; idx += THREADS) {
        const int j = idx / (2 * TL), half = (idx / TL) & 1, l = idx % TL;
        const int c = 8 * (l + TL * j) + 4 * half;
        if (c < D) {
            *reinterpret_cast<float4*>(mine_g + c) = sg4[idx];
            *reinterpret_cast<float4*>(mine_g + D + c) = sb4[idx];
        }
    }
}

// sums [n][2 D] -> dgamma, dbeta (either may be nullptr).  A block takes 32 columns, its warps every eighth row.
__global__ void __launch_bounds__(256) layernorm_heads_sum_kernel(const float* __restrict__ sums, int n, int D, float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ float part[8][32];
    asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < 2 * D) {
#pragma unroll 4
        for (int i = warp; i < n; i += 8) s += sums[(size_t)i * 2 * D + c];
    }
    part[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < 2 * D) {
#pragma unroll
        for (int w = 1; w < 8; ++w) s += part[w][lane];
        if (c < D) {
            if (dgamma) dgamma[c] = s;
        } else if (dbeta) dbeta[c - D] = s;
    }
}

template <typename IO, int VPL, int W>
inline cudaError_t launch(const IO* y, const IO* dout, const float* gamma, float eps, IO* dy, float* sums, long long rows, int D, int n_sm, unsigned* ctas, cudaStream_t st)
{
    constexpr int R = rows_per_group(max_slices<IO>(), VPL), TEAMS = cta_threads<IO>() / 32 / W, SMEM = smem_bytes<IO, VPL, W>();
    if (SMEM + 4096 > 48 * 1024) {
        static PerDeviceFlag attr_set;
        const int dev = current_device();
        if (dev < 0) return cudaErrorInvalidDevice;
        if (!attr_set.is_set(dev)) {
            const cudaError_t e = cudaFuncSetAttribute(layernorm_heads_grad_kernel<IO, VPL, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
            if (e != cudaSuccess) return e;
            attr_set.set(dev);
        }
    }
    const long long groups = (rows + (long long)R * TEAMS - 1) / ((long long)R * TEAMS);
    *ctas = (unsigned)(groups < n_sm ? groups : n_sm);
    return launch_pdl(layernorm_heads_grad_kernel<IO, VPL, W>, *ctas, cta_threads<IO>(), SMEM, st, y, dout, gamma, eps, dy, sums, rows, D);
}

}  // namespace lng

// Workspace: one row of partial sums per CTA (at most one CTA per SM).
inline size_t layernorm_heads_grad_bytes(int D, int n_sm) { return (size_t)n_sm * 2 * D * sizeof(float); }

// D a multiple of 8, at most ln::MAX_D.  The team is the narrowest that keeps to the slices a lane can hold.
template <typename IO>
inline gf_status_t layernorm_heads_grad(const IO* y, const IO* dout, const float* gamma, float eps, IO* dy, float* dgamma, float* dbeta, long long rows,
                                        int D, float* ws, int n_sm, cudaStream_t st, std::atomic<uint64_t>* launches)
{
    constexpr int MAX_VPL = lng::max_slices<IO>();
    const int nvec = D / 8;
    int w = 1;
    while (32 * w * MAX_VPL < nvec) w *= 2;
    const int vpl = (nvec + 32 * w - 1) / (32 * w);
    float* sums = dgamma || dbeta ? ws : nullptr;
    cudaError_t e = cudaErrorInvalidValue;
    unsigned ctas = 0;
#define GF_LNG_CASE(V, W_) \
    if (vpl == V && w == W_) e = lng::launch<IO, V, W_>(y, dout, gamma, eps, dy, sums, rows, D, n_sm, &ctas, st);
    if constexpr (MAX_VPL == 4) {
        GF_LNG_CASE(1, 1) GF_LNG_CASE(2, 1) GF_LNG_CASE(3, 1) GF_LNG_CASE(4, 1)
        GF_LNG_CASE(3, 2) GF_LNG_CASE(4, 2) GF_LNG_CASE(3, 4) GF_LNG_CASE(4, 4) GF_LNG_CASE(3, 8) GF_LNG_CASE(4, 8)
    } else {
        GF_LNG_CASE(1, 1) GF_LNG_CASE(2, 1) GF_LNG_CASE(2, 2) GF_LNG_CASE(2, 4) GF_LNG_CASE(2, 8) GF_LNG_CASE(2, 16)
    }
#undef GF_LNG_CASE
    launches->fetch_add(1, std::memory_order_relaxed);
    if (e != cudaSuccess) return GF_ERR_CUDA;
    if (!sums) return GF_OK;
    e = launch_pdl(lng::layernorm_heads_sum_kernel, (unsigned)((2 * D + 31) / 32), 256, 0, st, (const float*)sums, (int)ctas, D, dgamma, dbeta);
    launches->fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? GF_OK : GF_ERR_CUDA;
}

}  // namespace gf
