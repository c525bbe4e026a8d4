// Gradient of the LayerNorm across all heads (ln_heads.cuh): with mu, rstd the row's statistics, xhat = (y - mu) rstd and
// g = dout * gamma,
//     dy = rstd (g - mean(g) - xhat mean(g xhat)),   dgamma = sum over rows of dout * xhat,   dbeta = sum over rows of dout.
// The statistics are taken from y again (it is read anyway), so the forward call keeps nothing.
//
// Bound by HBM (2 D elements in, D out per token).  A row's statistics want its elements side by side, the sums over rows want a column's
// one below the other.  So rows come through a ring of three stages in shared memory (bulk copies of consecutive rows, up to 64 KB a
// stage), and a stage is gone through twice:
//  - along its rows: a warp (W warps for rows of more than 4 KB) takes one row's mean, squared deviations, sum of g and sum of
//    g (y - mean) in registers, two true passes with a butterfly of shuffles after each; several warps' shares are joined by the
//    pairwise formulae by the readers;
//  - down its columns: a thread owns UPT units of 16 bytes of every row, writes their dy and carries the sums of dgamma and dbeta.
// One barrier per stage between the two; behind it the stage before is refilled.  At the end a CTA leaves one row of sums in the
// workspace; a second kernel adds those over the CTAs.
// Measured: 10007 x 4096 fp32 77 us, 98 % of the copy rate; 16384 x 2048 bf16 43 us (71 %), 65536 rows 146 (84 %): half the bytes for the same
// arithmetic, so bf16 rows wait on latency, and the launch, the ring's first fill and the sums (4 us) weigh more.  (A team of warps
// that keeps whole rows and all column sums in registers, with a barrier for each row: the fp32 case 121 us with prefetches in
// registers and 91 through a ring.)
// Waits for copies are bounded (ck::mbar_wait): where one runs out, the status is raised and the CTA goes through its rows without
// further waits, so that the warps that meet at barriers all come to them.
#pragma once
#include "ln_heads.cuh"
#include "wkv6_chunked.cuh"

namespace gf {
namespace lng {

using ln::add2;
using ln::fma2;
using ln::mul2;

constexpr int STAGES = 3;
constexpr int RING_STAGE_BYTES = 64 * 1024;             // of both tensors, at most, of all CTAs of an SM
constexpr int MAX_CTAS = 2;                             // per SM
constexpr int MAX_STAGE_ROWS = 64;
constexpr int gamma_bytes(int D) { return 4 * (D < ln::MAX_D ? D : ln::MAX_D); }       // at most
template <typename IO> constexpr int per_unit() { return 16 / (int)sizeof(IO); }

// eight bf16 or four fp32 values of shared memory
template <typename IO> __device__ __forceinline__ void load_unit(uint32_t a, float2 (&f)[per_unit<IO>() / 2])
{
    uint32_t w[4];
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(a));
    if constexpr (sizeof(IO) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    } else {
        f[0] = make_float2(__uint_as_float(w[0]), __uint_as_float(w[1]));
        f[1] = make_float2(__uint_as_float(w[2]), __uint_as_float(w[3]));
    }
}
__device__ __forceinline__ void store_unit(__nv_bfloat16* p, const float2 (&f)[4]) { ln::store8(p, f); }
__device__ __forceinline__ void store_unit(float* p, const float2 (&f)[2]) { __stcs(reinterpret_cast<float4*>(p), make_float4(f[0].x, f[0].y, f[1].x, f[1].y)); }

// n bytes (a multiple of 16) of global memory into shared memory
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t n, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(n), "r"(bar) : "memory");
}
// WARPS per CTA, CTAS per SM.  Along rows W warps share a row, a lane holds LU units of it, RB rows at a time; down columns a thread owns UPT units.
// dynamic shared memory: gamma [D] as float4, then the ring [STAGES][y, dout][stage_rows][D], which the sums take over at the end
template <typename IO, int WARPS, int CTAS, int LU, int W, int UPT, int RB>
__global__ void __launch_bounds__(32 * WARPS, CTAS)
layernorm_heads_grad_kernel(const IO* __restrict__ y, const IO* __restrict__ dout, const float* __restrict__ gamma, float eps, IO* __restrict__ dy,
                            float* __restrict__ sums, long long rows, int D, int stage_rows, int row_lanes)
{
    constexpr int E = per_unit<IO>(), EH = E / 2, Q = E / 4;       // values, pairs and quads of a unit
    constexpr int THREADS = 32 * WARPS;
    static_assert(gamma_bytes(E * THREADS * UPT) + STAGES * RING_STAGE_BYTES / CTAS + 2 * MAX_STAGE_ROWS * 16 + (W > 1 ? WARPS * (WARPS / W) * 16 : 16) + 256 <= 232448 / CTAS, "shared memory of an SM");
    extern __shared__ float4 sh[];
    // by the stages' parity: per row its statistics (mean, rstd, mean g, mean g xhat), or per row and warp what they come from
    // (mean, squared deviations, sum of g, sum of g (y - mean))
    __shared__ float4 part[2][MAX_STAGE_ROWS];
    __shared__ float4 joined[W > 1 ? WARPS : 1][W > 1 ? WARPS / W : 1];       // a row's statistics as each warp has joined them
    __shared__ uint4 zero;                          // what a lane reads where the row has no unit for it
    __shared__ float cnt[W];                        // channels of a row that each of its warps holds
    __shared__ uint64_t full[STAGES];
    __shared__ uint32_t misc[2];                    // abort word, wait limit
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int units = D / E;
    const uint32_t abort_flag = ck::smem_u32(misc), row_bytes = (uint32_t)D * sizeof(IO), tensor_bytes = stage_rows * row_bytes;
    const uint32_t ring = ck::smem_u32(sh + D / 4), gammas = ck::smem_u32(sh);
    auto bar = [&](int s) { return ck::smem_u32(&full[s]); };
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) ck::mbar_init(bar(s), 1);
        zero = make_uint4(0u, 0u, 0u, 0u);
        ck::sts32(abort_flag, 0u);
        ck::sts32(abort_flag + 4, ck::WAIT_LIMIT_US);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        ck::fence_proxy_async();
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // the CTA's blocks of stage_rows rows: every gridDim.x-th
    const long long n_blocks = (rows + stage_rows - 1) / stage_rows;
    auto fetch = [&](long long b, int s) {          // by one thread
        const long long r = b * stage_rows;
        const uint32_t n = (uint32_t)min((long long)stage_rows, rows - r) * row_bytes, dst = ring + s * 2 * tensor_bytes;
        ck::mbar_expect_tx(bar(s), 2 * n);
        bulk_load(dst, y + (size_t)r * D, n, bar(s));
        bulk_load(dst + tensor_bytes, dout + (size_t)r * D, n, bar(s));
    };
    if (tid == 0)
        for (int s = 0; s < STAGES && blockIdx.x + (long long)s * gridDim.x < n_blocks; ++s) fetch(blockIdx.x + (long long)s * gridDim.x, s);
    for (int i = tid; i < D / 4; i += THREADS) sh[i] = gamma ? reinterpret_cast<const float4*>(gamma)[i] : make_float4(1.f, 1.f, 1.f, 1.f);
    auto gamma_of = [&](int unit, float2 (&g)[EH]) {
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const float4 v = ck::ldsf4(gammas + (unit * Q + q) * 16);
            g[2 * q] = make_float2(v.x, v.y);
            g[2 * q + 1] = make_float2(v.z, v.w);
        }
    };

    // along rows: this lane's units
    const int piece = warp % W, per_warp = 32 / row_lanes, row_step = W > 1 ? WARPS / W : WARPS * per_warp;        // (W > 1: row_lanes is 32)
    const int unit0 = W > 1 ? 32 * piece + lane : lane % row_lanes, unit_step = W > 1 ? 32 * W : row_lanes;
    if (W > 1 && warp < W && lane == 0) {
        int n = 0;
        for (int u = 32 * warp; u < units; u += 32 * W) n += min(32, units - u);
        cnt[warp] = (float)(n * E);
    }
    __syncthreads();
    uint32_t offset[LU];                            // of this lane's units in a row; past its end: none
    bool has[LU];
#pragma unroll
    for (int j = 0; j < LU; ++j) {
        const int u = unit0 + unit_step * j;
        has[j] = u < units;
        offset[j] = u * 16;
    }
    const uint32_t nothing = ck::smem_u32(&zero);
    const float inv_d = 1.f / (float)D, inv_n = W > 1 ? 1.f / cnt[piece] : inv_d;

    // down columns: this thread's units, and of every how many rows
    const int groups = UPT > 1 ? 1 : THREADS / units, group = UPT > 1 ? 0 : tid / units;
    int unit[UPT];
    bool on[UPT];
    float2 gm[UPT][EH], dg[UPT][EH], db[UPT][EH];
#pragma unroll
    for (int u = 0; u < UPT; ++u) {
        unit[u] = UPT > 1 ? tid + THREADS * u : tid % units;
        on[u] = UPT > 1 ? unit[u] < units : group < groups;
        if (!on[u]) unit[u] = 0;
        gamma_of(unit[u], gm[u]);
#pragma unroll
        for (int e = 0; e < EH; ++e) dg[u][e] = db[u][e] = make_float2(0.f, 0.f);
    }

    int s = 0, ph = 0, par = 0, prev = STAGES - 1;
    bool alive = true;
    for (long long b = blockIdx.x; b < n_blocks; b += gridDim.x, par ^= 1) {
        alive = ck::mbar_wait_warp(bar(s), ph, abort_flag) && alive;
        const int here = (int)min((long long)stage_rows, rows - b * stage_rows);
        const uint32_t st = ring + s * 2 * tensor_bytes;
        // ---- along rows
        // (RB rows at a time where they are short: their loads and shuffles hide one another's latency)
        for (int r0 = W > 1 ? warp / W : warp * per_warp; r0 < here; r0 += RB * row_step) {
            float2 x[RB][LU][EH];
            float mu[RB], m2[RB], sg[RB], sgx[RB];
            bool in[RB];
            uint32_t at[RB];
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                const int r = r0 + i * row_step + (W > 1 ? 0 : lane / row_lanes);
                in[i] = r < here;
                at[i] = st + r * row_bytes;
                float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
                for (int j = 0; j < LU; ++j) {
                    load_unit<IO>(in[i] && has[j] ? at[i] + offset[j] : nothing, x[i][j]);
#pragma unroll
                    for (int e = 0; e < EH; ++e) s2 = add2(s2, x[i][j][e]);
                }
                mu[i] = s2.x + s2.y;
            }
            for (int o = row_lanes / 2; o > 0; o >>= 1)
#pragma unroll
                for (int i = 0; i < RB; ++i) mu[i] += __shfl_xor_sync(0xffffffffu, mu[i], o);
            float2 q2[RB], g2[RB], p2[RB];
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                mu[i] *= inv_n;
                q2[i] = g2[i] = p2[i] = make_float2(0.f, 0.f);
            }
#pragma unroll
            for (int j = 0; j < LU; ++j) {
                float2 gj[EH];
                gamma_of(has[j] ? unit0 + unit_step * j : 0, gj);
#pragma unroll
                for (int i = 0; i < RB; ++i) {
                    float2 d[EH];
                    load_unit<IO>(in[i] && has[j] ? at[i] + tensor_bytes + offset[j] : nothing, d);
                    const float neg = has[j] ? -mu[i] : 0.f;
                    const float2 neg_m = make_float2(neg, neg);
#pragma unroll
                    for (int e = 0; e < EH; ++e) {
                        const float2 c = add2(x[i][j][e], neg_m), g = mul2(d[e], gj[e]);
                        q2[i] = fma2(c, c, q2[i]);
                        g2[i] = add2(g2[i], g);
                        p2[i] = fma2(g, c, p2[i]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                m2[i] = q2[i].x + q2[i].y;
                sg[i] = g2[i].x + g2[i].y;
                sgx[i] = p2[i].x + p2[i].y;
            }
            for (int o = row_lanes / 2; o > 0; o >>= 1)
#pragma unroll
                for (int i = 0; i < RB; ++i) {
                    m2[i] += __shfl_xor_sync(0xffffffffu, m2[i], o);
                    sg[i] += __shfl_xor_sync(0xffffffffu, sg[i], o);
                    sgx[i] += __shfl_xor_sync(0xffffffffu, sgx[i], o);
                }
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                const int r = r0 + i * row_step + (W > 1 ? 0 : lane / row_lanes);
                if (W > 1) {
                    if (in[i] && lane == 0) part[par][r * W + piece] = make_float4(mu[i], m2[i], sg[i], sgx[i]);
                } else if (in[i] && lane % row_lanes == 0) {
                    const float rstd = rsqrtf(fmaf(m2[i], inv_d, eps));
                    part[par][r] = make_float4(mu[i], rstd, sg[i] * inv_d, sgx[i] * rstd * inv_d);
                }
            }
        }
        __syncthreads();
        // every warp has left the stage before
        if (tid == 0 && alive && b != blockIdx.x && b + (long long)(STAGES - 1) * gridDim.x < n_blocks) fetch(b + (long long)(STAGES - 1) * gridDim.x, prev);
        if (W > 1 && lane < here) {
            // ---- a row's warps, joined: deviations from the common mean m are those from the warp's plus (its mean - m)
            float m = 0.f, q = 0.f, sg = 0.f, p = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) m = fmaf(cnt[w], part[par][lane * W + w].x, m);
            m *= inv_d;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float4 pw = part[par][lane * W + w];
                const float dm = pw.x - m;
                q += fmaf(cnt[w] * dm, dm, pw.y);
                sg += pw.z;
                p += fmaf(pw.z, dm, pw.w);
            }
            const float rstd = rsqrtf(fmaf(q, inv_d, eps));
            joined[warp][lane] = make_float4(m, rstd, sg * inv_d, p * rstd * inv_d);
        }
        __syncwarp();
        // ---- down columns
#pragma unroll 2
        for (int r0 = 0; r0 < here; r0 += groups) {
            const int r = min(r0 + group, here - 1);
            const bool mine_too = r0 + group < here;
            const float4 v = W > 1 ? joined[warp][r] : part[par][r];
            const float2 neg_mu = make_float2(-v.x, -v.x), r2 = make_float2(v.y, v.y), neg_mg = make_float2(-v.z, -v.z), neg_mgx = make_float2(-v.w, -v.w);
            IO* out = dy + (size_t)(b * stage_rows + r) * D;
#pragma unroll
            for (int u = 0; u < UPT; ++u)
                if (on[u] && mine_too) {
                    float2 x[EH], d[EH], o[EH];
                    const uint32_t at = st + r * row_bytes + unit[u] * 16;
                    load_unit<IO>(at, x);
                    load_unit<IO>(at + tensor_bytes, d);
#pragma unroll
                    for (int e = 0; e < EH; ++e) {
                        const float2 xh = mul2(add2(x[e], neg_mu), r2);
                        dg[u][e] = fma2(d[e], xh, dg[u][e]);
                        db[u][e] = add2(db[u][e], d[e]);
                        o[e] = mul2(fma2(xh, neg_mgx, fma2(d[e], gm[u][e], neg_mg)), r2);
                    }
                    store_unit(out + unit[u] * E, o);
                }
        }
        prev = s;
        if (++s == STAGES) { s = 0; ph ^= 1; }
    }
    if (ck::lds32(abort_flag))                      // copies that are still under way land before the CTA leaves
        for (int k = 0; k < STAGES; ++k)
            if (blockIdx.x + (long long)k * gridDim.x < n_blocks) ck::mbar_wait_warp(bar(k), k < s ? ph ^ 1 : ph, abort_flag, false);

    if (!sums) return;
    float* mine_g = sums + (size_t)blockIdx.x * 2 * D;
    if (groups == 1) {
#pragma unroll
        for (int u = 0; u < UPT; ++u)
            if (on[u]) {
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    *reinterpret_cast<float4*>(mine_g + unit[u] * E + 4 * q) = make_float4(dg[u][2 * q].x, dg[u][2 * q].y, dg[u][2 * q + 1].x, dg[u][2 * q + 1].y);
                    *reinterpret_cast<float4*>(mine_g + D + unit[u] * E + 4 * q) = make_float4(db[u][2 * q].x, db[u][2 * q].y, db[u][2 * q + 1].x, db[u][2 * q + 1].y);
                }
            }
        return;
    }
    // ---- the groups' sums through shared memory: [value][thread], added up by the first group in order
    __syncthreads();
    float* hold = reinterpret_cast<float*>(sh + D / 4);
#pragma unroll
    for (int e = 0; e < EH; ++e) {
        hold[(4 * e + 0) * THREADS + tid] = dg[0][e].x;
        hold[(4 * e + 1) * THREADS + tid] = dg[0][e].y;
        hold[(4 * e + 2) * THREADS + tid] = db[0][e].x;
        hold[(4 * e + 3) * THREADS + tid] = db[0][e].y;
    }
    __syncthreads();
    for (int i = tid; i < 2 * D; i += THREADS) {
        const int c = i < D ? i : i - D, u = c / E, e = c % E;
        const float* v = hold + (4 * (e / 2) + (i < D ? 0 : 2) + (e & 1)) * THREADS + u;
        float t = 0.f;
        for (int k = 0; k < groups; ++k) t += v[k * units];
        mine_g[i] = t;
    }
}

// sums [n][2 D] -> dgamma, dbeta (either may be nullptr).  A block takes 32 columns, eight lanes of four each; its 64 groups of lanes take every
// 64th row, and the first adds the groups' sums up in order.
constexpr int SUM_GROUPS = 64;
__global__ void __launch_bounds__(8 * SUM_GROUPS) layernorm_heads_sum_kernel(const float* __restrict__ sums, int n, int D, float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ float4 part[SUM_GROUPS][8];
    asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
    const int group = threadIdx.x / 8, lane = threadIdx.x % 8, c = blockIdx.x * 32 + 4 * lane;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < 2 * D) {                                  // (D a multiple of 8: the four columns are all inside)
#pragma unroll 5
        for (int i = group; i < n; i += SUM_GROUPS) {
            const float4 v = __ldcs(reinterpret_cast<const float4*>(sums + (size_t)i * 2 * D + c));
            t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
        }
    }
    part[group][lane] = t;
    __syncthreads();
    if (threadIdx.x < 32 && blockIdx.x * 32 + threadIdx.x < 2 * D) {
        const int k = blockIdx.x * 32 + threadIdx.x;
        const float* v = reinterpret_cast<const float*>(part) + threadIdx.x;
        float a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int g = 0; g < SUM_GROUPS; ++g) a[g & 3] += v[g * 32];
        const float sum = (a[0] + a[1]) + (a[2] + a[3]);
        if (k < D) {
            if (dgamma) dgamma[k] = sum;
        } else if (dbeta) dbeta[k - D] = sum;
    }
}

template <typename IO, int WARPS, int CTAS, int LU, int W, int UPT, int RB>
inline cudaError_t launch(const IO* y, const IO* dout, const float* gamma, float eps, IO* dy, float* sums, long long rows, int D, int n_sm, unsigned* ctas, cudaStream_t st)
{
    const int row_bytes = D * (int)sizeof(IO), units = row_bytes / 16;
    int row_lanes = 32;
    while (row_lanes / 2 >= units) row_lanes /= 2;
    // As many rows to a stage as it holds, but a pass of all warps along rows where few rows leave a CTA less than three stages; whole
    // passes where it is several.
    constexpr int STAGE_BYTES = RING_STAGE_BYTES / CTAS;
    const int pass = RB * (W > 1 ? WARPS / W : WARPS * (32 / row_lanes));
    int most = STAGE_BYTES / (2 * row_bytes);
    if (most > MAX_STAGE_ROWS / W) most = MAX_STAGE_ROWS / W;
    if (W > 1 && most > WARPS / W) most = WARPS / W;
    if (most > pass) most = most / pass * pass;
    const long long share = rows / (3LL * CTAS * n_sm);
    int stage_rows = share >= most ? most : share < pass ? pass : (int)(share / pass * pass);
    if (stage_rows > most) stage_rows = most;
    n_sm *= CTAS;
    const int ring = STAGES * 2 * stage_rows * row_bytes, hold = 4 * (per_unit<IO>() / 2) * 32 * WARPS * 4, smem = D * 4 + (ring > hold ? ring : hold);
    static PerDeviceFlag attr_set;
    const int dev = current_device();
    if (dev < 0) return cudaErrorInvalidDevice;
    if (!attr_set.is_set(dev)) {
        const cudaError_t e = cudaFuncSetAttribute(layernorm_heads_grad_kernel<IO, WARPS, CTAS, LU, W, UPT, RB>, cudaFuncAttributeMaxDynamicSharedMemorySize, gamma_bytes(per_unit<IO>() * 32 * WARPS * UPT) + STAGES * STAGE_BYTES);
        if (e != cudaSuccess) return e;
        attr_set.set(dev);
    }
    const long long blocks = (rows + stage_rows - 1) / stage_rows;
    *ctas = (unsigned)(blocks < n_sm ? blocks : n_sm);
    return launch_pdl(layernorm_heads_grad_kernel<IO, WARPS, CTAS, LU, W, UPT, RB>, *ctas, 32 * WARPS, smem, st, y, dout, gamma, eps, dy, sums, rows, D, stage_rows, row_lanes);
}

}  // namespace lng

// Workspace: one row of partial sums per CTA.
inline size_t layernorm_heads_grad_bytes(int D, int n_sm) { return (size_t)n_sm * lng::MAX_CTAS * 2 * D * sizeof(float); }

// D a multiple of 8, at most ln::MAX_D: up to 2048 units of 16 bytes.
template <typename IO>
inline gf_status_t layernorm_heads_grad(const IO* y, const IO* dout, const float* gamma, float eps, IO* dy, float* dgamma, float* dbeta, long long rows,
                                        int D, float* ws, int n_sm, cudaStream_t st, std::atomic<uint64_t>* launches)
{
    const int units = D / lng::per_unit<IO>();
    float* sums = dgamma || dbeta ? ws : nullptr;
    cudaError_t e = cudaErrorInvalidValue;
    unsigned ctas = 0;
    // Two small CTAs per SM where their columns' sums fit: one's barrier and shuffles pass while the other computes (65536 x 2048 bf16: one of
    // sixteen warps 150 us, two of eight 150, two of four 146; 65536 x 768: 72, 72, 75).  Rows of more than 4 KB: one CTA, whose threads
    // own more columns (16384 x 4096 bf16 81 us, two of eight warps 112).  Short rows two at a time (200000 x 64: 26.6 us, one 34).
#define GF_LNG_CASE(most, WARPS, CTAS, LU, W, UPT, RB) \
    else if (units <= most) e = lng::launch<IO, WARPS, CTAS, LU, W, UPT, RB>(y, dout, gamma, eps, dy, sums, rows, D, n_sm, &ctas, st);
    if (units <= 0) return GF_ERR_INVALID_ARG;
    GF_LNG_CASE(32, 8, 2, 1, 1, 1, 2) GF_LNG_CASE(64, 8, 2, 2, 1, 1, 2) GF_LNG_CASE(96, 16, 1, 3, 1, 1, 1) GF_LNG_CASE(128, 8, 2, 4, 1, 1, 1)
    if constexpr (sizeof(IO) == 2) {
        if (units <= 128) {}
        GF_LNG_CASE(256, 4, 2, 8, 1, 2, 1) GF_LNG_CASE(512, 8, 1, 8, 2, 2, 1) GF_LNG_CASE(1024, 16, 1, 4, 8, 2, 1)
    } else {
        if (units <= 128) {}
        GF_LNG_CASE(256, 8, 2, 4, 2, 1, 1) GF_LNG_CASE(512, 16, 1, 4, 4, 1, 1) GF_LNG_CASE(1024, 8, 1, 8, 4, 4, 1) GF_LNG_CASE(2048, 8, 1, 8, 8, 8, 1)
    }
#undef GF_LNG_CASE
    launches->fetch_add(1, std::memory_order_relaxed);
    if (e != cudaSuccess) return GF_ERR_CUDA;
    if (!sums) return GF_OK;
    e = launch_pdl(lng::layernorm_heads_sum_kernel, (unsigned)((2 * D + 31) / 32), 8 * lng::SUM_GROUPS, 0, st, (const float*)sums, (int)ctas, D, dgamma, dbeta);
    launches->fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? GF_OK : GF_ERR_CUDA;
}

}  // namespace gf
