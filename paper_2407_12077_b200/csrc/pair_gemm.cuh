// Matrix products with the elementwise work of an operator in their epilogue, for sm_100a (tcgen05 + TMEM + TMA): what the
// gated linear block and the vocabulary loss, and the gradients of both, are built from.
//
//     C[m][n] = sum_k A(m, k) B(k, n)        bf16 operands, fp32 accumulators
//
// Either operand may lie with its contraction index or its other index contiguous in memory (K-major, MN-major); both are read by
// TMA as they are, in 64 x 64 tiles, so a gradient's products (dy W^T, x^T dy) need no transposed copies.  A launch computes one
// or more groups of output tiles (two gradients of one call), whose tiles are handed out in order to persistent units: a unit
// is a pair of CTAs on neighbouring SMs that works on 256 x 256 accumulators with cta_group::2 instructions (each CTA holds 128 rows
// of A and of the result, and half the columns of B; one instruction of the leading CTA feeds both tensor cores, and every byte of
// an operand enters shared memory once), or, where a call has too few such tiles to fill the GPU, one CTA with 128 x 128 ones.
// Two accumulator sets fill tensor memory: the products of a tile run while the epilogue drains the one before.
//
// A tile's columns can be shared out in halves (B_DUAL, B_HALF): the left half holds columns of a first product, the right half the
// same columns of a second one, so that an epilogue sees both values of an element (the gated linear block).  B_DUAL: both
// products have the same A and run as one; B_HALF: each has its own A and depth, and they run one after the other.  As products of half a
// tile's columns keep the tensor cores at 3/4 of their rate (an instruction reads as much of A for half the work), WIDE gives each of two
// deep products a whole 256 x 256 accumulator; these fill tensor memory, so there is one set, and what the epilogue can do with the
// first product alone it does while the second one runs.  SPLIT, for results of few tiles (decoding): a cluster of up to eight CTAs divides a tile's
// contraction indices, leaves its sums in shared memory and adds them up there, each CTA a share of the tile's places.
//
//   warp 0      TMA producer: 64 contraction indices of A and B (16 KB each per CTA) per stage of a five-stage ring
//   warp 1      tensor-memory allocation; an elected lane of the leading CTA issues the four products of a stage
//   warps 2-9   epilogue: a lane owns a row of the tile, 32 columns at a time, two warps sharing a row's columns out in blocks of 64
// Every wait is bounded (status flag and abort as in the prefill kernel); a pair's CTAs meet before either leaves.
#pragma once
#include "key_compress.cuh"
#include "wkv6_chunked.cuh"

#include <float.h>
#include <type_traits>

namespace gf {
namespace pg {

using namespace ck;                                   // PTX wrappers, descriptors, TILE, bounded waits
using kc::cluster_sync;

constexpr int N_EPI = 8;                              // epilogue warps: two per tensor-memory sub-partition
constexpr int THREADS = 64 + 32 * N_EPI;
constexpr int NSTAGE = 5;
constexpr int STAGE_BYTES = 4 * TILE;                 // 128 x 64 of A, 128 x 64 of B
constexpr int OFF_SLAB = NSTAGE * STAGE_BYTES;        // [N_EPI warps][2][32 rows x 128 B]
constexpr int OFF_MISC = OFF_SLAB + N_EPI * 2 * 4096;     // abort word, wait limit, tensor-memory address, barriers
constexpr int SUMS_PITCH = (2 * 128 + 4) * 4;          // SPLIT_TILES: a row of both products' sums, fp32, in place of the ring
static_assert(128 * SUMS_PITCH <= OFF_SLAB, "partial sums");
constexpr int SMEM = OFF_MISC + 256 + 1024;           // + slack for manual 1024-byte alignment
static_assert(SMEM <= 232448, "shared memory budget of one sm_100 CTA");
enum { BAR_FULL = 0, BAR_EMPTY = NSTAGE, BAR_ACC_FULL = 2 * NSTAGE, BAR_ACC_EMPTY = BAR_ACC_FULL + 2, BAR_LEFT_FULL = BAR_ACC_EMPTY + 2, BAR_DRAIN, N_BARS };
static_assert(16 + 8 * N_BARS <= 256, "barrier block");

// what the epilogue makes of an accumulator
enum Epilogue {
    EPI_STORE,          // the product itself (Group::mode)
    EPI_GATE,           // act(a) * b of the two halves, or act(a) of a whole tile
    EPI_GATE_GRAD,      // dy b act'(a) and dy act(a)
    EPI_LSE,            // per row and tile of columns: maximum and sum of exponentials, and the target's logit
    EPI_PROB,           // (exp(z - lse) - [column is the target]) * dloss
    // the same two, and what rounding an output to bf16 leaves of it in a tensor of its own (maps out[2], out[3]; out[1])
    EPI_GATE_GRAD_RESTS,
    EPI_PROB_RESTS
};
constexpr bool is_gate_grad(Epilogue e) { return e == EPI_GATE_GRAD || e == EPI_GATE_GRAD_RESTS; }
constexpr bool is_prob(Epilogue e) { return e == EPI_PROB || e == EPI_PROB_RESTS; }
constexpr bool has_rests(Epilogue e) { return e == EPI_GATE_GRAD_RESTS || e == EPI_PROB_RESTS; }
enum Mode { TILES, WIDE_TILES, SPLIT_TILES };
enum BCols : unsigned char { B_WHOLE, B_DUAL, B_HALF };
enum OutMode : unsigned char { OUT_BF16, OUT_F32, OUT_F32_ADD, OUT_BF16_ADD };   // (_ADD: onto, resp. with, the fp32 sums of earlier launches; F32: [slices][rows][cols])
enum Act { ACT_SIGMOID = 0, ACT_RELU2 = 1, ACT_SILU = 2, ACT_GELU = 3 };

constexpr int MAX_IN = 8, MAX_OUT = 4, MAX_GROUPS = 4, MAX_SEGMENTS = 4;
// A run of contraction indices of a group's products: 64 * steps of them (the last may reach past the tensors, where TMA reads zeros).
struct Segment {
    unsigned char a, b;             // tensor maps (B_DUAL: b and b + 1)
    bool a_mn, b_mn;                // the operand's non-contraction index is the contiguous one
    BCols cols;
    bool right;                     // B_HALF: accumulates in the tile's right half
    int steps;
};
struct Group {
    int tiles_m, tiles_n, first;    // first: number of the group's first tile in the launch
    uint32_t per_mul, per_shift;    // division by the tiles of a band (see tile_at): (mulhi(i, per_mul) + i) >> per_shift
    int slices;                     // tiles per place of the result, each with its share of the contraction indices (all segments' in a row)
    int steps;                      // of all segments
    int n_seg;
    Segment seg[MAX_SEGMENTS];
    unsigned char out;              // tensor map of the result
    OutMode mode;
    int rows, cols;                 // extent of the result (of each half's columns where a tile is halved)
    float* part;                    // OUT_BF16_ADD: fp32 sums [rows][cols]
};
struct GemmParams {
    CUtensorMap in[MAX_IN], out[MAX_OUT];
    Group g[MAX_GROUPS];
    int n_groups, n_tiles;
    uint32_t in_used;               // bit per map of `in`
    // EPI_GATE, EPI_GATE_GRAD
    int act;
    bool gated;
    const __nv_bfloat16* dy;
    __nv_bfloat16* y;               // SPLIT_TILES
    // EPI_LSE, EPI_PROB
    const long long* targets;
    long long vocab;                // a target outside [0, vocab) is none
    int first_col;                  // the vocabulary's index of this launch's first column
    float2* stats;                  // [2 tiles_n][rows] (reference value, sum of exponentials over it) of each half of a tile's columns
    float* target_logit;
    const float* lse;
    const float* dloss;             // or nullptr: ones
};

// ---------------------------------------------------------------- PTX of CTA pairs
__device__ __forceinline__ uint32_t map_to_leader(uint32_t saddr)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(saddr));
    return a;
}
// Says that accumulators have been read (tcgen05.wait::ld, fence::before_thread_sync); no memory has to become visible with it: a release at
// cluster scope would wait for the tile's stores on their way to global memory, 1700 cycles of the 6000 that a tile of shallow products takes.
__device__ __forceinline__ void arrive_cluster_if(uint32_t addr, bool pred)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\t@p mbarrier.arrive.shared::cluster.b64 _, [%0];\n\t}"
                 ::"r"(addr), "r"((uint32_t)pred) : "memory");
}
// A tile into this CTA's shared memory; its bytes are counted by the barrier at a shared::cluster address, the leading CTA's.
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* tm, int c0, int c1, uint32_t bar_cluster)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(dst), "l"(tm), "r"(c0), "r"(c1), "r"(bar_cluster) : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t smem_dst, uint32_t cols)      // one full warp of either CTA
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t cols)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
__device__ __forceinline__ void tc_mma_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// One arrival at the barrier of both CTAs of the pair once the products issued so far are complete.
__device__ __forceinline__ void tc_commit_pair(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((unsigned short)3) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* tm, int c0, int c1, int c2, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];"
                 ::"l"(tm), "r"(c0), "r"(c1), "r"(c2), "r"(src) : "memory");
}
__device__ __forceinline__ void tma_reduce_add_3d(const CUtensorMap* tm, int c0, int c1, int c2, uint32_t src)
{
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2, %3}], [%4];"
                 ::"l"(tm), "r"(c0), "r"(c1), "r"(c2), "r"(src) : "memory");
}

// K-major: 8-row groups 1024 bytes apart.  MN-major: blocks of 64 indices a tile apart.
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr, bool mn) { return mn ? kc::kc_desc_w(saddr) : smem_desc(saddr); }
// fp32 accumulator, bf16 A and B
__device__ __forceinline__ uint32_t instr_desc(int m, int n, bool a_mn, bool b_mn)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// ---------------------------------------------------------------- activations
// The normal distribution Phi(a) by the Chebyshev fit of the complementary error function in Press et al., Numerical Recipes (erfcc): a relative error
// of 1.2e-7 on the whole axis, and of 4e-6 (|a| < 8) with the exponential's argument in fp32, far below a bf16 rounding.  Fourteen
// instructions where erfcf takes some forty (8192 rows, twice 512 deep -> 8192, with gelu: 220 us -> 164).
__device__ __forceinline__ float normal_cdf(float a)
{
    const float x = fabsf(a) * 0.70710678f, t = __fdividef(1.f, fmaf(0.5f, x, 1.f));
    float p = fmaf(0.17087277f, t, -0.82215223f);
    p = fmaf(p, t, 1.48851587f);
    p = fmaf(p, t, -1.13520398f);
    p = fmaf(p, t, 0.27886807f);
    p = fmaf(p, t, -0.18628806f);
    p = fmaf(p, t, 0.09678418f);
    p = fmaf(p, t, 0.37409196f);
    p = fmaf(p, t, 1.00002368f);
    p = fmaf(p, t, -1.26551223f);
    const float q = 0.5f * t * ex2(fmaf(-x, x, p) * LOG2E);
    return a < 0.f ? q : 1.f - q;
}
__device__ __forceinline__ float relu(float a)        // (a NaN stays one)
{
    float r;
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(a));
    return r;
}
template <int ACT> __device__ __forceinline__ float act_value(float a)
{
    if constexpr (ACT == ACT_RELU2) {
        const float r = relu(a);
        return r * r;
    } else if constexpr (ACT == ACT_GELU) {
        return a * normal_cdf(a);
    } else {
        const float s = __fdividef(1.f, 1.f + __expf(-a));
        return ACT == ACT_SIGMOID ? s : a * s;
    }
}
// value and derivative; the sigmoid and one minus it from an exponential that cannot overflow, without cancellation
template <int ACT> __device__ __forceinline__ void act_grad(float a, float& f, float& df)
{
    if constexpr (ACT == ACT_RELU2) {
        const float r = relu(a);
        f = r * r;
        df = 2.f * r;
    } else if constexpr (ACT == ACT_GELU) {
        const float phi = normal_cdf(a);
        f = a * phi;
        df = fmaf(a * 0.39894228f, __expf(-0.5f * a * a), phi);
    } else {
        const float e = __expf(-fabsf(a)), r = __fdividef(1.f, 1.f + e), er = e * r;
        const float s = a >= 0.f ? r : er, t = a >= 0.f ? er : r;
        f = ACT == ACT_SIGMOID ? s : a * s;
        df = ACT == ACT_SIGMOID ? s * t : s * fmaf(a, t, 1.f);
    }
}
// f(std::integral_constant<int, act>): one branch for all values of a lane
template <typename F> __device__ __forceinline__ void by_act(int act, F&& f)
{
    if (act == ACT_SIGMOID) f(std::integral_constant<int, ACT_SIGMOID>());
    else if (act == ACT_RELU2) f(std::integral_constant<int, ACT_RELU2>());
    else if (act == ACT_SILU) f(std::integral_constant<int, ACT_SILU>());
    else f(std::integral_constant<int, ACT_GELU>());
}

__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
// 32 values of the lane's row, rounded to bf16, into columns 32*half .. of a 64-column slab
__device__ __forceinline__ void put_bf16(uint32_t slab, int lane, int half, const float (&o)[32])
{
#pragma unroll
    for (int q = 0; q < 4; ++q)
        sts128(slab + swz(lane, (4 * half + q) << 4), pack_bf16(o[8 * q], o[8 * q + 1]), pack_bf16(o[8 * q + 2], o[8 * q + 3]),
               pack_bf16(o[8 * q + 4], o[8 * q + 5]), pack_bf16(o[8 * q + 6], o[8 * q + 7]));
}
// 32 columns of the lane's accumulator row
__device__ __forceinline__ void ld_acc(uint32_t taddr, float (&o)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, "
        "%8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, "
        "%24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(o[0]), "=f"(o[1]), "=f"(o[2]), "=f"(o[3]), "=f"(o[4]), "=f"(o[5]), "=f"(o[6]), "=f"(o[7]),
          "=f"(o[8]), "=f"(o[9]), "=f"(o[10]), "=f"(o[11]), "=f"(o[12]), "=f"(o[13]), "=f"(o[14]), "=f"(o[15]),
          "=f"(o[16]), "=f"(o[17]), "=f"(o[18]), "=f"(o[19]), "=f"(o[20]), "=f"(o[21]), "=f"(o[22]), "=f"(o[23]),
          "=f"(o[24]), "=f"(o[25]), "=f"(o[26]), "=f"(o[27]), "=f"(o[28]), "=f"(o[29]), "=f"(o[30]), "=f"(o[31])
        : "r"(taddr) : "memory");
}
// two runs of 32 columns with one wait
__device__ __forceinline__ void ld_acc2(uint32_t t0, float (&a)[32], uint32_t t1, float (&b)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, "
        "%8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, "
        "%24, %25, %26, %27, %28, %29, %30, %31}, [%64];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%32, %33, %34, %35, %36, %37, %38, %39, "
        "%40, %41, %42, %43, %44, %45, %46, %47, "
        "%48, %49, %50, %51, %52, %53, %54, %55, "
        "%56, %57, %58, %59, %60, %61, %62, %63}, [%65];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(a[0]), "=f"(a[1]), "=f"(a[2]), "=f"(a[3]), "=f"(a[4]), "=f"(a[5]), "=f"(a[6]), "=f"(a[7]),
          "=f"(a[8]), "=f"(a[9]), "=f"(a[10]), "=f"(a[11]), "=f"(a[12]), "=f"(a[13]), "=f"(a[14]), "=f"(a[15]),
          "=f"(a[16]), "=f"(a[17]), "=f"(a[18]), "=f"(a[19]), "=f"(a[20]), "=f"(a[21]), "=f"(a[22]), "=f"(a[23]),
          "=f"(a[24]), "=f"(a[25]), "=f"(a[26]), "=f"(a[27]), "=f"(a[28]), "=f"(a[29]), "=f"(a[30]), "=f"(a[31]),
          "=f"(b[0]), "=f"(b[1]), "=f"(b[2]), "=f"(b[3]), "=f"(b[4]), "=f"(b[5]), "=f"(b[6]), "=f"(b[7]),
          "=f"(b[8]), "=f"(b[9]), "=f"(b[10]), "=f"(b[11]), "=f"(b[12]), "=f"(b[13]), "=f"(b[14]), "=f"(b[15]),
          "=f"(b[16]), "=f"(b[17]), "=f"(b[18]), "=f"(b[19]), "=f"(b[20]), "=f"(b[21]), "=f"(b[22]), "=f"(b[23]),
          "=f"(b[24]), "=f"(b[25]), "=f"(b[26]), "=f"(b[27]), "=f"(b[28]), "=f"(b[29]), "=f"(b[30]), "=f"(b[31])
        : "r"(t0), "r"(t1) : "memory");
}

// v <- v minus its rounding to bf16 (nothing of an infinity or a NaN: the rounded value carries it)
__device__ __forceinline__ void leave_rest(float (&v)[32])
{
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const float r = v[j] - __bfloat162float(__float2bfloat16_rn(v[j]));
        v[j] = fabsf(r) < INFINITY ? r : 0.f;
    }
}
struct Tile {
    int g, m, n;                    // group, place in it
    int slice, lo, hi;              // the steps it takes
};
// share, shares: of a tile that a cluster of CTAs divides (a group is cut into slices or divided, not both)
__device__ __forceinline__ Tile tile_at(const GemmParams& p, int tile, int share, int shares)
{
    Tile t;
    t.g = 0;
    while (t.g + 1 < p.n_groups && tile >= p.g[t.g + 1].first) ++t.g;
    const Group& g = p.g[t.g];
    const int places = g.tiles_m * g.tiles_n;
    int i = tile - g.first;
    t.slice = 0;
    if (g.slices > 1) {
        t.slice = i / places;
        i -= t.slice * places;
    }
    const uint32_t of = g.slices * shares, nth = t.slice + share;
    t.lo = (int)((uint32_t)g.steps * nth / of);       // (steps <= 2^27 - 16, four segments of a tensor's longest side; of <= 32)
    t.hi = (int)((uint32_t)g.steps * (nth + 1) / of);
    // bands of eight tiles along m, column by column: the tiles that run at one time share few rows of A and of B
    const int per = 8 * g.tiles_n, band = (int)((__umulhi((uint32_t)i, g.per_mul) + (uint32_t)i) >> g.per_shift), rest = i - band * per;
    const int h = min(8, g.tiles_m - 8 * band);
    t.n = h == 8 ? rest >> 3 : rest / h;
    t.m = 8 * band + rest - t.n * h;
    return t;
}

__device__ __forceinline__ void st_acc(uint32_t taddr, const float (&o)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};\n\t"
        "tcgen05.wait::st.sync.aligned;"
        ::"r"(taddr), "f"(o[0]), "f"(o[1]), "f"(o[2]), "f"(o[3]), "f"(o[4]), "f"(o[5]), "f"(o[6]), "f"(o[7]), "f"(o[8]), "f"(o[9]), "f"(o[10]), "f"(o[11]),
          "f"(o[12]), "f"(o[13]), "f"(o[14]), "f"(o[15]), "f"(o[16]), "f"(o[17]), "f"(o[18]), "f"(o[19]), "f"(o[20]), "f"(o[21]), "f"(o[22]), "f"(o[23]),
          "f"(o[24]), "f"(o[25]), "f"(o[26]), "f"(o[27]), "f"(o[28]), "f"(o[29]), "f"(o[30]), "f"(o[31])
        : "memory");
}
// 32 bf16 values of a row that has `left` more of them (a multiple of 8); zeros past its end and where the row is none
__device__ __forceinline__ void load_row32(const __nv_bfloat16* src, bool in, int left, uint32_t (&d)[16])
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint4 u = in && 8 * q < left ? __ldg(reinterpret_cast<const uint4*>(src) + q) : make_uint4(0u, 0u, 0u, 0u);
        d[4 * q] = u.x; d[4 * q + 1] = u.y; d[4 * q + 2] = u.z; d[4 * q + 3] = u.w;
    }
}
// blocks of 64 among `left` indices, at most the two of a CTA's operand
__device__ __forceinline__ int tiles_of(int left) { return left <= 0 ? 0 : left <= 64 ? 1 : 2; }
// bit i where 0 <= i < 32, else nothing
__device__ __forceinline__ uint32_t one_of_32(long long i) { return i >= 0 && i < 32 ? 1u << (int)i : 0u; }
// v <- exp(v - r); the difference first: of logits far from zero it is exact where it matters
__device__ __forceinline__ void exp_of_difference(float (&v)[32], float r)
{
    const float2 neg = make_float2(-r, -r), l2e = make_float2(LOG2E, LOG2E);
#pragma unroll
    for (int j = 0; j < 32; j += 2) {
        const float2 d = mul2(add2(make_float2(v[j], v[j + 1]), neg), l2e);
        v[j] = ex2(d.x);
        v[j + 1] = ex2(d.y);
    }
}
__device__ __forceinline__ float bf16_at(const uint32_t (&d)[16], int j) { return __uint_as_float(j & 1 ? d[j / 2] & 0xffff0000u : d[j / 2] << 16); }

template <int CG, Epilogue EPI, Mode MODE>
__global__ void __launch_bounds__(THREADS, 1) pair_gemm_kernel(const __grid_constant__ GemmParams p)
{
    constexpr int BN = 128 * CG;                      // columns of a tile
    constexpr bool WIDE = MODE == WIDE_TILES, SPLIT = MODE == SPLIT_TILES;
    static_assert(!WIDE || CG == 2, "pairs of CTAs");
    static_assert(!SPLIT || (CG == 1 && EPI == EPI_GATE), "single CTAs, forward block");
    constexpr int HW = MODE == TILES ? BN / 2 : BN;   // columns of a half
    constexpr int SETS = MODE == TILES ? 2 : 1, ACC_COLS = 256;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t sbase = smem_u32(smem);
    const uint32_t abort_flag = sbase + OFF_MISC;
    auto bar = [&](int i) { return sbase + OFF_MISC + 16 + 8 * i; };
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint32_t rank = 0;
    if constexpr (CG == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    uint32_t share = 0, shares = 1;                   // SPLIT: of a tile's contraction indices
    if constexpr (SPLIT) {
        asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(share));
        asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(shares));
    }
    const int unit = blockIdx.x / (SPLIT ? shares : CG), units = gridDim.x / (SPLIT ? shares : CG);

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (warp == 2 && (p.in_used >> lane & 1)) asm volatile("prefetch.tensormap [%0];" ::"l"(&p.in[lane]) : "memory");      // (of the launch's parameters)
    if (tid == 0) {
        for (int i = 0; i < NSTAGE; ++i) {
            mbar_init(bar(BAR_FULL + i), 1);
            mbar_init(bar(BAR_EMPTY + i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(BAR_ACC_FULL + i), 1);
            mbar_init(bar(BAR_ACC_EMPTY + i), N_EPI * CG);
        }
        mbar_init(bar(BAR_LEFT_FULL), 1);
        mbar_init(bar(BAR_DRAIN), 1);
        sts32(abort_flag, 0u);
        sts32(abort_flag + 4, ck::WAIT_LIMIT_US);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    if (warp == 1) {
        if constexpr (CG == 2) tmem_alloc_pair(sbase + OFF_MISC + 8, 512);
        else tmem_alloc(sbase + OFF_MISC + 8, 512);
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();            // the other CTA's barriers are there before anything arrives at them
    tc_fence_after();
    const uint32_t tmem = lds32(sbase + OFF_MISC + 8);
    const Tile first = tile_at(p, unit, share, shares);       // (a unit has a tile at least)

    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 0) {
        // ============================== TMA producer ==============================
        int s = 0, ph = 0, issued = 0;
        bool alive = true;
        for (int tile = unit; tile < p.n_tiles && alive; tile += units) {
            const Tile t = tile == unit ? first : tile_at(p, tile, share, shares);
            const Group& g = p.g[t.g];
            const int m0 = t.m * 128 * CG + 128 * (int)rank, tn = t.n;
            for (int q = 0, at = 0; q < g.n_seg && alive; at += g.seg[q++].steps) {
                const Segment sg = g.seg[q];
                const int end = min(sg.steps, t.hi - at);
                // this CTA's columns of B: 128 of the tile's (one block of 64 where the tile's halves have products of their own)
                const int n0 = sg.cols == B_WHOLE ? tn * BN + 128 * (int)rank : sg.cols == B_DUAL ? tn * HW : tn * HW + 64 * (int)rank;
                const int n1 = sg.cols == B_DUAL && CG == 1 ? n0 : n0 + 64;
                // tiles past the result's last row or column are not loaded: what multiplies them is not stored
                const int a_here = tiles_of(g.rows - m0), b_here = sg.cols == B_DUAL && CG == 1 ? 2 : min(tiles_of(g.cols - n0), sg.cols == B_HALF ? 1 : 2);
                int bytes = (a_here + b_here) * TILE;
                if constexpr (CG == 2) {
                    const int n_there = sg.cols == B_WHOLE ? n0 + 128 : sg.cols == B_DUAL ? n0 : n0 + 64;        // (of the other CTA; the leading one counts)
                    bytes += (tiles_of(g.rows - m0 - 128) + min(tiles_of(g.cols - n_there), sg.cols == B_HALF ? 1 : 2)) * TILE;
                }
                const CUtensorMap* ma = &p.in[sg.a];
                const CUtensorMap* mb0 = &p.in[sg.b + (sg.cols == B_DUAL && CG == 2 ? rank : 0)];
                const CUtensorMap* mb1 = sg.cols == B_DUAL && CG == 1 ? &p.in[sg.b + 1] : mb0;
                for (int ks = max(0, t.lo - at); ks < end; ++ks) {
                    if (issued >= NSTAGE && !mbar_wait_warp(bar(BAR_EMPTY + s), ph ^ 1, abort_flag)) { alive = false; break; }
                    const uint32_t st = sbase + s * STAGE_BYTES;
                    if (elect_one()) {
                        const int k = ks * 64;
                        const uint32_t full = CG == 2 ? map_to_leader(bar(BAR_FULL + s)) : bar(BAR_FULL + s);
                        auto load = [&](uint32_t dst, const CUtensorMap* m, int c0, int c1) {
                            if constexpr (CG == 2) tma_load_pair(dst, m, c0, c1, full);
                            else tma_load_2d(dst, m, c0, c1, full);
                        };
                        if (rank == 0) mbar_expect_tx(bar(BAR_FULL + s), bytes);
                        if (a_here > 0) load(st, ma, sg.a_mn ? m0 : k, sg.a_mn ? k : m0);
                        if (a_here > 1) load(st + TILE, ma, sg.a_mn ? m0 + 64 : k, sg.a_mn ? k : m0 + 64);
                        if (b_here > 0) load(st + 2 * TILE, mb0, sg.b_mn ? n0 : k, sg.b_mn ? k : n0);
                        if (b_here > 1) load(st + 3 * TILE, mb1, sg.b_mn ? n1 : k, sg.b_mn ? k : n1);
                    }
                    __syncwarp();
                    ++issued;
                    if (++s == NSTAGE) { s = 0; ph ^= 1; }
                }
            }
        }
        // do not leave while copies may still be in flight (a pair's are counted by the leading CTA, and its CTAs leave together)
        if (rank == 0) {
            for (int c = min(issued, NSTAGE); c > 0; --c) {
                // stages s - c .. s - 1, each in the phase of its last use
                const int st = s - c < 0 ? s - c + NSTAGE : s - c, sp = s - c < 0 ? ph ^ 1 : ph;
                if (!mbar_wait_warp(bar(BAR_FULL + st), sp, abort_flag, false)) break;
            }
        }
    } else if (warp == 1) {
        // ============================== MMA issuer (leading CTA) ==============================
        if (rank == 0) {
            int s = 0, ph = 0, ti = 0;
            bool alive = true;
            for (int tile = unit; tile < p.n_tiles && alive; tile += units, ++ti) {
                const Tile t = tile == unit ? first : tile_at(p, tile, share, shares);
                const Group& g = p.g[t.g];
                const int set = SETS == 2 ? ti & 1 : 0, use = SETS == 2 ? ti >> 1 : ti;
                // the epilogue has read this set's previous tile out of tensor memory
                if (use >= 1 && !mbar_wait_warp(bar(BAR_ACC_EMPTY + set), (use + 1) & 1, abort_flag)) { alive = false; break; }
                tc_fence_after();
                uint32_t begun = 0;                   // bits 0, 1: the left, the right accumulators hold products of this tile
                for (int q = 0, at = 0; q < g.n_seg && alive; at += g.seg[q++].steps) {
                    const Segment sg = g.seg[q];
                    const int end = min(sg.steps, t.hi - at);
                    const uint32_t idesc = instr_desc(128 * CG, sg.cols == B_HALF ? HW : BN, sg.a_mn, sg.b_mn);
                    const uint32_t acc = tmem + ACC_COLS * set + (sg.right ? HW : 0);
                    const uint64_t a_step = sg.a_mn ? 128 : 2, b_step = sg.b_mn ? 128 : 2;      // 16 contraction indices
                    for (int ks = max(0, t.lo - at); ks < end; ++ks) {
                        if (!mbar_wait_warp(bar(BAR_FULL + s), ph, abort_flag)) { alive = false; break; }
                        tc_fence_after();
                        if (elect_one()) {
                            const uint32_t st = sbase + s * STAGE_BYTES;
                            const uint64_t da = operand_desc(st, sg.a_mn), db = operand_desc(st + 2 * TILE, sg.b_mn);
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk) {
                                const uint32_t on = (begun >> sg.right & 1) || kk > 0;
                                if constexpr (CG == 2) tc_mma_pair(acc, da + a_step * kk, db + b_step * kk, idesc, on);
                                else tc_mma(acc, da + a_step * kk, db + b_step * kk, idesc, on);
                            }
                            const bool last = at + ks == t.hi - 1, left = WIDE && ks == sg.steps - 1 && q == 0;
                            if constexpr (CG == 2) {
                                tc_commit_pair(bar(BAR_EMPTY + s));
                                if (left) tc_commit_pair(bar(BAR_LEFT_FULL));
                                if (last) tc_commit_pair(bar(BAR_ACC_FULL + set));
                            } else {
                                tc_commit(bar(BAR_EMPTY + s));
                                if (last) tc_commit(bar(BAR_ACC_FULL + set));
                            }
                        }
                        __syncwarp();
                        begun |= 1u << sg.right;
                        if (++s == NSTAGE) { s = 0; ph ^= 1; }
                    }
                }
            }
            if (!alive) {                             // products in flight end before tensor memory is given back
                if (elect_one()) {
                    if constexpr (CG == 2) tc_commit_pair(bar(BAR_DRAIN));
                    else tc_commit(bar(BAR_DRAIN));
                }
                __syncwarp();
                mbar_wait_warp(bar(BAR_DRAIN), 0, abort_flag, false);
            }
        }
    } else {
        // ============================== epilogue warps ==============================
        const int sp = warp & 3;                      // tensor-memory sub-partition: accumulator rows 32*sp .. 32*sp+31
        const int part = (warp - 2) >> 2;             // takes the row's blocks of 64 columns part, part + 2, ..
        const uint32_t slabs = sbase + OFF_SLAB + (warp - 2) * 2 * 4096;
        uint32_t sl = slabs;                          // the slab that was filled last
        // a row's target (-1: none), normaliser and weight, read a tile ahead
        struct RowValues { long long target; float lse, weight; };
        auto row_values = [&](const Tile& t) {
            RowValues v = {-1, 0.f, 0.f};
            if constexpr (EPI == EPI_LSE || is_prob(EPI)) {
                const int r = t.m * 128 * CG + 128 * (int)rank + 32 * sp + lane;
                if (r < p.g[t.g].rows) {
                    v.target = p.targets[r];
                    if (v.target < 0 || v.target >= p.vocab) v.target = -1;
                    if constexpr (is_prob(EPI)) {
                        v.lse = p.lse[r];
                        v.weight = v.target < 0 ? 0.f : p.dloss ? p.dloss[r] : 1.f;
                    }
                }
            }
            return v;
        };
        Tile next = first;
        RowValues ahead = row_values(first);
        int ti = 0;
        for (int tile = unit; tile < p.n_tiles; tile += units, ++ti) {
            const Tile place = next;
            const Group& g = p.g[place.g];
            const int tm = place.m, tn = place.n;
            const int row0 = tm * 128 * CG + 128 * (int)rank + 32 * sp, row = row0 + lane;
            const bool in = row < g.rows;
            // what the epilogue reads from memory is under way while the products run
            const int width = EPI == EPI_GATE || is_gate_grad(EPI) ? (WIDE || p.gated ? HW : BN) : BN;
            uint32_t dy[2][16];                       // of the warp's first block of 64 columns
            auto load_dy = [&](int c) {
                if constexpr (is_gate_grad(EPI)) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int col = tn * width + c + 32 * half;
                        load_row32(p.dy + (size_t)row * g.cols + col, in && c < width, g.cols - col, dy[half]);
                    }
                }
            };
            load_dy(64 * part);
            const long long target = ahead.target;
            const float lse = ahead.lse, weight = ahead.weight;
            const int set = SETS == 2 ? ti & 1 : 0;
            if (!mbar_wait_warp(bar(WIDE ? BAR_LEFT_FULL : BAR_ACC_FULL + set), (SETS == 2 ? ti >> 1 : ti) & 1, abort_flag)) break;
            tc_fence_after();
            const uint32_t acc = tmem + ((uint32_t)(32 * sp) << 16) + ACC_COLS * set;
            if (tile + units < p.n_tiles) {           // the next tile's place, and what it reads of its rows
                next = tile_at(p, tile + units, share, shares);
                ahead = row_values(next);
            }
            // the warp's other slab, once no store is reading it any more (the one before may be under way)
            auto take_slab = [&]() {
                sl ^= slabs ^ (slabs + 4096);
                if (lane == 0) bulk_wait_read<1>();
                __syncwarp();
            };
            auto send = [&](const CUtensorMap* m, int col) {
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) {                      // (a group each time, if an empty one: take_slab() counts them)
                    if (row0 < g.rows) tma_store_2d(m, col, row0, sl);
                    bulk_commit();
                }
            };
            if constexpr (EPI == EPI_STORE) {
                for (int c = 64 * part; c < BN; c += 128) {
                    const int col = tn * BN + c;
                    if (col >= g.cols) break;
                    if (g.mode == OUT_F32 || g.mode == OUT_F32_ADD) {
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            float v[32];
                            ld_acc(acc + c + 32 * half, v);
                            take_slab();
#pragma unroll
                            for (int q = 0; q < 8; ++q)
                                sts128(sl + swz(lane, q << 4), __float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]), __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3]));
                            fence_proxy_async();
                            __syncwarp();
                            if (lane == 0) {
                                if (row0 < g.rows && col + 32 * half < g.cols) {
                                    if (g.mode == OUT_F32) tma_store_3d(&p.out[g.out], col + 32 * half, row0, place.slice, sl);
                                    else tma_reduce_add_3d(&p.out[g.out], col + 32 * half, row0, place.slice, sl);
                                }
                                bulk_commit();
                            }
                        }
                    } else {
                        float w[2][32];
                        ld_acc2(acc + c, w[0], acc + c + 32, w[1]);
                        take_slab();
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            float(&v)[32] = w[half];
                            if (g.mode == OUT_BF16_ADD && in) {
                                const float* src = g.part + (size_t)row * g.cols + col + 32 * half;
#pragma unroll
                                for (int q = 0; q < 8; ++q)
                                    if (col + 32 * half + 4 * q < g.cols) {          // (a multiple of 8)
                                        const float4 f = __ldcs(reinterpret_cast<const float4*>(src) + q);
                                        v[4 * q] += f.x; v[4 * q + 1] += f.y; v[4 * q + 2] += f.z; v[4 * q + 3] += f.w;
                                    }
                            }
                            put_bf16(sl, lane, half, v);
                        }
                        send(&p.out[g.out], col);
                    }
                }
            } else if constexpr (SPLIT) {
                // this CTA's sums to shared memory (the ring is free: every slice that was loaded has been multiplied)
                for (int c = 64 * part; c < 2 * BN; c += 128) {
                    if (c < BN ? place.lo >= g.seg[0].steps : place.hi <= g.seg[0].steps) continue;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float v[32];
                        ld_acc(acc + c + 32 * half, v);
                        if (in) {
#pragma unroll
                            for (int q = 0; q < 8; ++q)
                                sts128(sbase + (32 * sp + lane) * SUMS_PITCH + (c + 32 * half + 4 * q) * 4, __float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]),
                                       __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3]));
                        }
                    }
                }
            } else if constexpr (EPI == EPI_GATE && WIDE) {
                // the activation goes back where its argument was while the second product runs
                for (int c = 64 * part; c < HW && tn * HW + c < g.cols; c += 128)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float a[32];
                        ld_acc(acc + c + 32 * half, a);
                        by_act(p.act, [&](auto k) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) a[j] = act_value<decltype(k)::value>(a[j]);
                        });
                        st_acc(acc + c + 32 * half, a);
                    }
                if (!mbar_wait_warp(bar(BAR_ACC_FULL), ti & 1, abort_flag)) break;
                tc_fence_after();
                for (int c = 64 * part; c < HW; c += 128) {
                    const int col = tn * HW + c;
                    if (col >= g.cols) break;
                    take_slab();
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float a[32], b[32];
                        ld_acc2(acc + c + 32 * half, a, acc + HW + c + 32 * half, b);
#pragma unroll
                        for (int j = 0; j < 32; ++j) a[j] *= b[j];
                        put_bf16(sl, lane, half, a);
                    }
                    send(&p.out[0], col);
                }
            } else if constexpr (EPI == EPI_GATE_GRAD && WIDE) {
                // db needs the first product alone: it leaves, and dy act'(a) takes the first product's place, while the second one runs
                for (int c = 64 * part; c < HW; c += 128) {
                    const int col = tn * HW + c;
                    if (col >= g.cols) break;
                    if (c >= 128) load_dy(c);
                    take_slab();
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t(&d)[16] = dy[half];
                        float a[32], b[32];
                        ld_acc(acc + c + 32 * half, a);
                        by_act(p.act, [&](auto k) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) {
                                float f, df;
                                act_grad<decltype(k)::value>(a[j], f, df);
                                a[j] = bf16_at(d, j) * df;
                                b[j] = bf16_at(d, j) * f;
                            }
                        });
                        st_acc(acc + c + 32 * half, a);
                        put_bf16(sl, lane, half, b);
                    }
                    send(&p.out[1], col);
                }
                if (!mbar_wait_warp(bar(BAR_ACC_FULL), ti & 1, abort_flag)) break;
                tc_fence_after();
                for (int c = 64 * part; c < HW; c += 128) {
                    const int col = tn * HW + c;
                    if (col >= g.cols) break;
                    take_slab();
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float a[32], b[32];
                        ld_acc2(acc + c + 32 * half, a, acc + HW + c + 32 * half, b);
#pragma unroll
                        for (int j = 0; j < 32; ++j) a[j] *= b[j];
                        put_bf16(sl, lane, half, a);
                    }
                    send(&p.out[0], col);
                }
            } else if constexpr (EPI == EPI_GATE) {
                for (int c = 64 * part; c < width; c += 128) {
                    const int col = tn * width + c;
                    if (col >= g.cols) break;
                    take_slab();
#pragma unroll 1                                      // (a small call runs this code once: what it fetches of it counts)
                    for (int half = 0; half < 2; ++half) {
                        float a[32], b[32];
                        if (p.gated) ld_acc2(acc + c + 32 * half, a, acc + HW + c + 32 * half, b);
                        else ld_acc(acc + c + 32 * half, a);
                        by_act(p.act, [&](auto k) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) a[j] = act_value<decltype(k)::value>(a[j]);
                        });
                        if (p.gated) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) a[j] *= b[j];
                        }
                        put_bf16(sl, lane, half, a);
                    }
                    send(&p.out[0], col);
                }
            } else if constexpr (is_gate_grad(EPI)) {
                for (int rest = 0; rest <= (int)has_rests(EPI); ++rest)
                for (int c = 64 * part; c < width; c += 128) {
                    const int col = tn * width + c;
                    if (col >= g.cols) break;
                    if (c >= 128 || rest) load_dy(c);
                    take_slab();
                    uint32_t later[2][16];            // db, in bf16, until da has left the slab
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t(&d)[16] = dy[half];
                        float a[32];
                        if (p.gated) {
                            float b[32];
                            ld_acc2(acc + c + 32 * half, a, acc + HW + c + 32 * half, b);
                            by_act(p.act, [&](auto k) {
#pragma unroll
                                for (int j = 0; j < 32; ++j) {
                                    float f, df;
                                    act_grad<decltype(k)::value>(a[j], f, df);
                                    a[j] = bf16_at(d, j) * b[j] * df;
                                    b[j] = bf16_at(d, j) * f;
                                }
                            });
                            if (rest) leave_rest(b);
#pragma unroll
                            for (int j = 0; j < 16; ++j) later[half][j] = pack_bf16(b[2 * j], b[2 * j + 1]);
                        } else {
                            ld_acc(acc + c + 32 * half, a);
                            by_act(p.act, [&](auto k) {
#pragma unroll
                                for (int j = 0; j < 32; ++j) {
                                    float f, df;
                                    act_grad<decltype(k)::value>(a[j], f, df);
                                    a[j] = bf16_at(d, j) * df;
                                }
                            });
                        }
                        if (rest) leave_rest(a);
                        put_bf16(sl, lane, half, a);
                    }
                    send(&p.out[2 * rest], col);
                    if (p.gated) {
                        take_slab();
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            sts128(sl + swz(lane, q << 4), later[q / 4][4 * (q % 4)], later[q / 4][4 * (q % 4) + 1], later[q / 4][4 * (q % 4) + 2], later[q / 4][4 * (q % 4) + 3]);
                        send(&p.out[2 * rest + 1], col);
                    }
                }
            } else if constexpr (EPI == EPI_LSE) {
                // a warp takes half of the tile's columns.  exp is taken of differences to a reference, the largest value so far, which stays
                // finite: FLT_MAX for +inf (the sum is infinite by itself, and no later reference scales it down), -FLT_MAX where all are
                // -inf (the sum is zero, and any other reference is larger); a NaN reaches the sum through its own exponential
                float ref = -FLT_MAX, sum = 0.f;
                for (int c = HW * part; c < HW * part + HW; c += 64) {
                    const int col = tn * BN + c;
                    if (col >= g.cols) break;
                    float v[2][32];
                    ld_acc2(acc + c, v[0], acc + c + 32, v[1]);
                    float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        if (col + 32 * half + 32 > g.cols) {
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (col + 32 * half + j >= g.cols) v[half][j] = -INFINITY;
                        }
                        const uint32_t hit = one_of_32(target - (col + 32 * half));
                        if (__any_sync(0xffffffffu, hit)) {
                            float z = 0.f;
#pragma unroll
                            for (int j = 0; j < 32; ++j) z = hit >> j & 1 ? v[half][j] : z;
                            if (hit) p.target_logit[row] = z;
                        }
#pragma unroll
                        for (int j = 0; j < 32; ++j) t4[j & 3] = fmaxf(t4[j & 3], v[half][j]);
                    }
                    const float top = fminf(fmaxf(fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])), ref), FLT_MAX);
                    float2 s2[4] = {make_float2(sum * ex2((ref - top) * LOG2E), 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        exp_of_difference(v[half], top);
#pragma unroll
                        for (int j = 0; j < 16; ++j) s2[j & 3] = add2(s2[j & 3], make_float2(v[half][2 * j], v[half][2 * j + 1]));
                    }
                    s2[0] = add2(add2(s2[0], s2[1]), add2(s2[2], s2[3]));
                    sum = s2[0].x + s2[0].y;
                    ref = top;
                }
                if (in) p.stats[(size_t)(2 * tn + part) * g.rows + row] = make_float2(ref, sum);
            } else {
                const long long at = target < 0 ? -1 : target - p.first_col;
                for (int rest = 0; rest <= (int)has_rests(EPI); ++rest)
                for (int c = 64 * part; c < BN; c += 128) {
                    const int col = tn * BN + c;
                    if (col >= g.cols) break;
                    float e[2][32];
                    ld_acc2(acc + c, e[0], acc + c + 32, e[1]);
                    take_slab();
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float(&v)[32] = e[half];
                        exp_of_difference(v, lse);
                        const uint32_t hit = one_of_32(at - (col + 32 * half));
                        if (__any_sync(0xffffffffu, hit)) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] -= hit >> j & 1 ? 1.f : 0.f;
                        }
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const float2 o = mul2(make_float2(v[j], v[j + 1]), make_float2(weight, weight));
                            v[j] = o.x;
                            v[j + 1] = o.y;
                        }
                        if (__any_sync(0xffffffffu, target < 0)) {    // (zero, whatever the logits of a row without a target are)
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = target < 0 ? 0.f : v[j];
                        }
                        if (col + 32 * half + 32 > g.cols) {          // (columns that fill up a row of the tensor: an operand, so zero)
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (col + 32 * half + j >= g.cols) v[j] = 0.f;
                        }
                        if (rest) leave_rest(v);
                        put_bf16(sl, lane, half, v);
                    }
                    send(&p.out[rest], col);
                }
            }
            tc_fence_before();
            __syncwarp();
            if constexpr (CG == 2) arrive_cluster_if(map_to_leader(bar(BAR_ACC_EMPTY + set)), lane == 0);
            else mbar_arrive_if(bar(BAR_ACC_EMPTY + set), lane == 0);
        }
        if (lane == 0) bulk_wait_read<0>();           // (shared memory may go; the grid's end completes the stores)
        __syncwarp();
    }

    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();            // neither CTA's memory goes while the other's products or arrivals may reach it
    if constexpr (SPLIT) {
        cluster_sync();
        // the cluster's sums of a place, in the order of the contraction indices; the CTAs share the tile's places out
        const Group& g = p.g[0];
        const int rows = min(128, g.rows - 128 * first.m), items = rows * (BN / 4), steps0 = g.seg[0].steps;
        int left_end = 0, right_begin = 0;            // shares 0 .. left_end-1 have products of the left, right_begin .. of the right
        for (int q = 0; q < (int)shares; ++q) {
            if (g.steps * q / (int)shares < steps0) left_end = q + 1;
            if (g.steps * (q + 1) / (int)shares <= steps0) right_begin = q + 1;
        }
        const int end = items * (int)(share + 1) / (int)shares;
        for (int i = items * (int)share / (int)shares + tid; i < end; i += THREADS) {
            const int r = i / (BN / 4), c = i % (BN / 4) * 4;
            float4 a[8], b[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                a[q] = b[q] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (q < left_end) a[q] = kc::ld_cluster(sbase + r * SUMS_PITCH + c * 4, q);
                if (q >= right_begin && q < (int)shares) b[q] = kc::ld_cluster(sbase + r * SUMS_PITCH + (BN + c) * 4, q);
            }
#pragma unroll
            for (int q = 1; q < 8; ++q) {
                a[0].x += a[q].x; a[0].y += a[q].y; a[0].z += a[q].z; a[0].w += a[q].w;
                b[0].x += b[q].x; b[0].y += b[q].y; b[0].z += b[q].z; b[0].w += b[q].w;
            }
            float o[4] = {a[0].x, a[0].y, a[0].z, a[0].w};
            by_act(p.act, [&](auto k) {
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = act_value<decltype(k)::value>(o[j]);
            });
            if (p.gated) { o[0] *= b[0].x; o[1] *= b[0].y; o[2] *= b[0].z; o[3] *= b[0].w; }
            const int col = first.n * BN + c;
            if (col < g.cols)                         // (a multiple of 8)
                *reinterpret_cast<uint2*>(p.y + (size_t)(128 * first.m + r) * g.cols + col) = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
        }
        __syncwarp();
        cluster_sync();                               // no CTA leaves while another reads its sums
    }
    if (warp == 1) {
        tc_fence_after();
        if constexpr (CG == 2) tmem_dealloc_pair(tmem, 512);
        else tmem_dealloc(tmem, 512);
    }
}

// [slices][rows][C] fp32 tensor, box = 32 rows x 32 columns (128 bytes), 128-byte swizzle
inline bool make_map_f32(CUtensorMap* tm, const void* base, int slices, long long rows, long long C)
{
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    cuuint64_t dims[3] = {(cuuint64_t)C, (cuuint64_t)rows, (cuuint64_t)slices};
    cuuint64_t strides[2] = {(cuuint64_t)C * 4, (cuuint64_t)C * rows * 4};
    cuuint32_t box[3] = {32, 32, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// operand in 64 x 64 tiles; result in 32-row slabs of 64 columns.  (A row is 2 C bytes: C a multiple of 8.)
inline bool in_map(GemmParams& p, int i, const void* base, long long rows, long long C)
{
    p.in_used |= 1u << i;
    return make_map(&p.in[i], base, rows, C, 64);
}
inline bool out_map(CUtensorMap* tm, const void* base, long long rows, long long C) { return make_map(tm, base, rows, C, 32); }

inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// A group whose result is rows x cols, in tiles of 128*cg rows and `width` columns.
inline Group make_group(int cg, long long rows, long long cols, int width)
{
    Group g = {};
    g.tiles_m = (int)ceil_div(rows, 128 * cg);
    g.tiles_n = (int)ceil_div(cols, width);
    g.rows = (int)rows;
    g.cols = (int)cols;
    g.slices = 1;
    // i / d for i < 2^30, d = 8 tiles_n: with s = ceil(log2 d), floor(2^32 (2^s - d) / d) + 1 and one addition (Granlund, Montgomery)
    const uint64_t d = 8ull * g.tiles_n;
    while ((1ull << g.per_shift) < d) ++g.per_shift;
    g.per_mul = (uint32_t)((((1ull << g.per_shift) - d) << 32) / d + 1);
    return g;
}
inline Segment segment(int a, bool a_mn, int b, bool b_mn, long long depth, BCols cols = B_WHOLE, bool right = false)
{
    Segment s = {};
    s.a = (unsigned char)a; s.b = (unsigned char)b;
    s.a_mn = a_mn; s.b_mn = b_mn;
    s.cols = cols; s.right = right;
    s.steps = (int)ceil_div(depth, 64);
    return s;
}
inline void add_segment(Group& g, const Segment& s)
{
    g.seg[g.n_seg++] = s;
    g.steps += s.steps;
}
inline void add_group(GemmParams& p, const Group& g)
{
    p.g[p.n_groups] = g;
    p.g[p.n_groups].first = p.n_tiles;
    p.n_tiles += g.tiles_m * g.tiles_n * g.slices;
    ++p.n_groups;
}

template <int CG, Epilogue EPI, Mode MODE>
inline cudaError_t launch_one(const GemmParams& p, int n_sm, int dev, cudaStream_t st, int cluster = CG)
{
    static PerDeviceFlag attr_set;
    if (!attr_set.is_set(dev)) {
        const cudaError_t e = cudaFuncSetAttribute(pair_gemm_kernel<CG, EPI, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
        if (e != cudaSuccess) return e;
        attr_set.set(dev);
    }
    const int units = MODE == SPLIT_TILES ? p.n_tiles : n_sm / CG;
    const unsigned grid = (unsigned)(cluster * (p.n_tiles < units ? p.n_tiles : units));
    return launch_pdl_cluster(pair_gemm_kernel<CG, EPI, MODE>, grid, THREADS, SMEM, cluster, st, p);
}
// Clusters of c CTAs (2 .. 8), one CTA per SM, that are counted on to run at one time: a cluster must lie within one GPC, so it is fewer than the
// SMs would hold.  cudaOccupancyMaxActiveClusters says 74, 45, 33, 26, 22, 15, 15 on a GPU of 148 SMs (key_compress.cuh saw 14 of 8 on
// another); one less is counted on, as GPUs differ in which SMs they have.  Where they do not all fit, the call takes a second round.
inline int clusters_at_once(int c, int n_sm)
{
    constexpr int of_148[9] = {0, 0, 73, 44, 32, 25, 21, 14, 14};
    return of_148[c] * n_sm / 148;
}

struct Launch {
    int cg;                         // 1 or 2
    Mode mode;
    int cluster;                    // CTAs per cluster (SPLIT_TILES; otherwise cg)
};
constexpr Launch SINGLE = {1, TILES, 1};              // what needs no cluster
// false, and nothing enqueued, where the device refuses it (no cluster can be placed on a partitioned one: the caller goes on with SINGLE)
template <Epilogue EPI>
inline bool launch(const Launch& l, const GemmParams& p, cudaStream_t st, std::atomic<uint64_t>* launches)
{
    const int n_sm = sm_count(), dev = current_device();
    if (n_sm < 2 || dev < 0) return false;
    cudaError_t e = cudaErrorInvalidValue;
    if (l.mode == TILES && l.cg == 1) e = launch_one<1, EPI, TILES>(p, n_sm, dev, st);
    if constexpr (!has_rests(EPI))                    // (few rows: SINGLE)
        if (l.mode == TILES && l.cg == 2) e = launch_one<2, EPI, TILES>(p, n_sm, dev, st);
    if constexpr (EPI == EPI_GATE || EPI == EPI_GATE_GRAD)
        if (l.mode == WIDE_TILES) e = launch_one<2, EPI, WIDE_TILES>(p, n_sm, dev, st);
    if constexpr (EPI == EPI_GATE)
        if (l.mode == SPLIT_TILES) e = launch_one<1, EPI, SPLIT_TILES>(p, n_sm, dev, st, l.cluster);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    launches->fetch_add(1, std::memory_order_relaxed);
    return true;
}

// ---------------------------------------------------------------- several products in one launch (a gradient's)
// A gradient's first operand (da, db, P) is rounded to bf16: 2.2e-3 to 2.4e-3 of the result's norm in all, whatever the number of rows (1 to 1024
// measured), the result's own rounding being 1.7e-3 of it.  That is what many roundings average to; where one row or two carry a result,
// a few of them decide (1.5e-3 to 3.2e-3 measured).  Up to REST_ROWS rows what the rounding leaves is kept too, in a second bf16 tensor, and
// multiplied as well: 1.6e-3 to 1.8e-3.  Such a call is one tile of rows and waits for launches and weights; it pays 6 to 20 us (us without
// and with, 16 and 128 rows: gated 424 -> 2072 19, 28 and 23, 35; 768 -> 2688 27, 32 and 29, 36; the loss, 768 deep over 40011 entries, 55, 67 and
// 61, 81).  With more rows the products count, and the price grows with them (512 and 1024 rows: 768 -> 2688 31, 49 and 40, 69; the loss
// 111, 173 and 163, 279).  The rule goes by the tensors' rows: how many of them have a target is known on the device alone, so a
// batch of more rows that is masked but for a few has the error of one rounding (1024 rows, one target: up to 3.2e-3).
constexpr long long REST_ROWS = 128;
inline bool keep_rests(long long rows) { return rows <= REST_ROWS; }
// Time of 64 contraction indices, in units of 1/30 us.  An SM takes in 64 bytes per cycle: the 32 KB of its share of a pair's 256 x 256 products
// take as long as these do, and the 32 KB of a 128 x 128 tile of its own hardly less (8192 deep, one tile: 0.264 us a step), for a
// half of the work per SM.
constexpr int STEP_TIME[3] = {0, 7, 8};

struct Product {
    long long m, n;
    int n_seg;
    Segment seg[MAX_SEGMENTS];
    __nv_bfloat16* out;             // [m][n]
    int steps() const
    {
        int n = 0;
        for (int i = 0; i < n_seg; ++i) n += seg[i].steps;
        return n;
    }
};
// Of a sum that several launches contribute to (pieces of the vocabulary)
enum Part { PART_ONLY, PART_FIRST, PART_MIDDLE, PART_LAST };
struct Plan {
    int cg;
    int slices[MAX_GROUPS];
    size_t sums_at[MAX_GROUPS], bytes;            // fp32 sums [slices][m][n] of products that are not stored at once, from the workspace's start
};

// Tiles go to the units in turn, so the busiest unit's load can be counted.  A few tiles of a deep product (rows of few tokens times a large
// vocabulary) leave most units idle: such a product is cut into slices of its contraction indices, whose fp32 sums a further kernel
// adds up in order.  That costs its launch and the sums' way through memory.
inline long long plan_time(const Product* q, int n, int cg, const int* slices, int n_sm, long long sum_bytes)
{
    const int units = n_sm / cg;
    long long all = 0, worst = 0, one[MAX_GROUPS], more[MAX_GROUPS], from[MAX_GROUPS], at = 0;
    for (int i = 0; i < n; ++i) {
        const long long tiles = ceil_div(q[i].m, 128 * cg) * ceil_div(q[i].n, 128 * cg) * slices[i];
        one[i] = (ceil_div(q[i].steps(), slices[i]) + 2) * STEP_TIME[cg];
        all += tiles / units * one[i];
        more[i] = tiles % units;                      // units that take one tile more, from this one on
        from[i] = at;
        at = (at + tiles) % units;
    }
    for (int i = 0; i < n; ++i) {                     // the busiest unit is the first of one of these runs
        long long t = 0;
        for (int j = 0; j < n; ++j)
            if ((from[i] - from[j] + units) % units < more[j]) t += one[j];
        worst = t > worst ? t : worst;
    }
    worst += all;
    // a step of a pair is 0.25 us: a further launch, with its set-up and its wait, about 5 us, the sums' bytes at 6 TB/s
    return worst + (sum_bytes ? 150 + sum_bytes / 220000 : 0);
}
inline Plan plan_products(const Product* q, int n, int n_sm, bool kept)
{
    Plan best = {};
    long long best_time = -1;
    int deepest = 0;
    for (int i = 0; i < n; ++i) deepest = q[i].steps() > deepest ? q[i].steps() : deepest;
    for (int cg = 2; cg >= 1; --cg)
        for (int cut = 1; cut <= 32 && (cut == 1 || deepest / cut >= 4); cut += cut < 4 ? 1 : cut / 2) {
            const int most = (int)ceil_div(deepest, cut);      // steps of a slice
            Plan p = {};
            p.cg = cg;
            long long sums = 0;
            for (int i = 0; i < n; ++i) {
                p.slices[i] = (int)ceil_div(q[i].steps(), most);
                if (p.slices[i] > 1) sums += (long long)p.slices[i] * q[i].m * q[i].n * 4;
            }
            if (sums > 256LL << 20) continue;
            const long long t = plan_time(q, n, cg, p.slices, n_sm, sums);
            if (best_time < 0 || t < best_time) {
                best_time = t;
                best = p;
            }
        }
    for (int i = 0; i < n; ++i)
        if (best.slices[i] > 1 || (kept && i == 0)) {
            best.sums_at[i] = best.bytes;
            best.bytes += ((size_t)best.slices[i] * q[i].m * q[i].n * 4 + 255) & ~(size_t)255;
        }
    return best;
}

// out = the slices' sums, in order, rounded once
struct SumJob {
    const float* sums;
    __nv_bfloat16* out;
    long long n;                    // elements of the result (a multiple of 8)
    int slices;
};
struct SumJobs {
    SumJob job[MAX_GROUPS];
    int n;
};
__global__ void __launch_bounds__(256) sum_slices_kernel(const SumJobs jobs)
{
    asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
    for (int k = 0; k < jobs.n; ++k) {
        const SumJob& j = jobs.job[k];
        for (long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 8; i < j.n; i += (long long)gridDim.x * 2048) {
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
#pragma unroll 4
            for (int s = 0; s < j.slices; ++s) {
                const float4* src = reinterpret_cast<const float4*>(j.sums + (size_t)s * j.n + i);
                const float4 u = __ldcs(src), v = __ldcs(src + 1);
                a.x += u.x; a.y += u.y; a.z += u.z; a.w += u.w;
                b.x += v.x; b.y += v.y; b.z += v.z; b.w += v.w;
            }
            *reinterpret_cast<uint4*>(j.out + i) = make_uint4(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(b.x, b.y), pack_bf16(b.z, b.w));
        }
    }
}

inline void whole_tiles(Plan& plan)
{
    const Plan was = plan;
    plan = Plan{1, {1, 1, 1, 1}, {}, was.bytes};      // (sums that are kept over several launches lie at the workspace's start in every plan)
}
// The products' launch and, where any is cut, the one that adds its slices up.  p.in holds the segments' maps; the first product may be a part
// of a sum over several calls (its slices stay in the workspace between them).  Where the device places no pairs of CTAs, the plan becomes
// one of single CTAs.
inline gf_status_t run_products(GemmParams& p, const Product* q, int n, Plan& plan, Part part, void* ws, cudaStream_t st, std::atomic<uint64_t>* launches)
{
    SumJobs jobs = {};
    for (;;) {
        int order[MAX_GROUPS], depth[MAX_GROUPS];
        for (int i = 0; i < n; ++i) {                 // the deepest tiles first: the round that ends unevenly is the shorter ones'
            depth[i] = (int)ceil_div(q[i].steps(), plan.slices[i]);
            int at = i;
            while (at > 0 && depth[order[at - 1]] < depth[i]) { order[at] = order[at - 1]; --at; }
            order[at] = i;
        }
        p.n_groups = p.n_tiles = jobs.n = 0;
        for (int k = 0; k < n; ++k) {
            const int i = order[k];
            const Product& r = q[i];
            const Part role = i == 0 ? part : PART_ONLY;
            const bool cut = plan.slices[i] > 1;
            Group g = make_group(plan.cg, r.m, r.n, 128 * plan.cg);
            for (int j = 0; j < r.n_seg; ++j) add_segment(g, r.seg[j]);
            g.slices = plan.slices[i] < g.steps ? plan.slices[i] : g.steps;      // (a last piece may have fewer steps than slices: the rest keep their sums)
            g.out = (unsigned char)i;
            float* sums = reinterpret_cast<float*>(static_cast<char*>(ws) + plan.sums_at[i]);
            g.part = sums;
            g.mode = role == PART_ONLY ? (cut ? OUT_F32 : OUT_BF16) : role == PART_FIRST ? OUT_F32 : role == PART_MIDDLE || cut ? OUT_F32_ADD : OUT_BF16_ADD;
            const bool f32 = g.mode == OUT_F32 || g.mode == OUT_F32_ADD;
            if (!(f32 ? make_map_f32(&p.out[i], sums, plan.slices[i], r.m, r.n) : out_map(&p.out[i], r.out, r.m, r.n))) return GF_ERR_CUDA;
            if (cut && (role == PART_ONLY || role == PART_LAST)) jobs.job[jobs.n++] = SumJob{sums, r.out, r.m * r.n, plan.slices[i]};
            add_group(p, g);
        }
        if (launch<EPI_STORE>(Launch{plan.cg, TILES, plan.cg}, p, st, launches)) break;
        if (plan.cg == 1 || part == PART_MIDDLE || part == PART_LAST) return GF_ERR_CUDA;
        whole_tiles(plan);
    }
    if (jobs.n == 0) return GF_OK;
    long long most = 0;
    for (int i = 0; i < jobs.n; ++i) most = jobs.job[i].n > most ? jobs.job[i].n : most;
    const long long blocks = ceil_div(most, 2048), cap = 8LL * sm_count();
    const cudaError_t e = launch_pdl(sum_slices_kernel, (unsigned)(blocks < cap ? blocks : cap), 256, 0, st, jobs);
    launches->fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? GF_OK : GF_ERR_CUDA;
}
// The SM count that plans are made for: the current device's, or a B200's where there is none to ask.
inline int plan_sms()
{
    const int n = sm_count();
    return n >= 2 ? n : 148;
}

}  // namespace pg
}  // namespace gf
