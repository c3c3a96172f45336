// Orthogonalising an update by Newton-Schulz products.  X = G / (|G|_F + eps), taken transposed if G is taller than wide, so that
// X is M x N with M <= N; then `steps` times
//     A = X X^T,   B = b A + c A A,   X <- a X + B X
// and the result is X.  The three products run on the tensor cores (tcgen05, binary16 operands, binary32 sums in tensor memory).
//
// Number formats.  A gradient has a few strong directions and many weak ones; the weak ones grow by a factor of up to a in every
// step, and so does every rounding of the strong ones that falls on them.  So X is held as hi + lo, two binary16 numbers (22 bits).
// On chip (k_ns_small: a side of at most 128, the other up to 4096) all three products take both halves of both operands, hi lo +
// lo hi + hi hi; B includes a I.  The result is then within 0.05 % of the 64-bit one for every spectrum measured
// and for steep coefficients, 0.01 % mostly.
// In the tiled kernels hi is the operand and the carried term a X uses both.  A and B are nearly diagonal once the singular
// values are near 1, so their diagonals are kept apart, in binary32, and only the rest is rounded to binary16:
//     A = D + O,  B = E + P:  P = b O + c (O O + (D_i + D_j) O) off the diagonal, E = b D + c (O O + D D) on it,
//     X <- (a + E_i) X + P X,
// which takes the diagonal's products out of the rounded operands.  X's low half is multiplied with P too in the steps whose
// rounding would still grow (kNsLowFrom), and for few rows O and P have low halves (kNsFine).  The result is then within 0.05 -
// 0.1 % of the 64-bit one for noise, 0.04 % for one strong direction over weak ones, 0.02 - 0.4 % for a constant level over small
// noise, whose equal entries are all rounded the same way (diagonals inside A and B: 0.15 - 0.2 % for noise; X's hi alone: 0.3 % at 129
// rows for one strong direction, and 2 - 7 % at low rank if the carried term has no more).
// Scaling by powers of two keeps everything in binary16's normal range: X times sx ~ sqrt(N), A and B times 256, lo times 2^11.
//
// Products with 128 x 128 tiles, one CTA each (k_ns_tile); the sum over K may be split over a cluster of 2 or 4 CTAs, which add
// their parts through distributed shared memory in a fixed order.  Large products with 256 x 256 tiles, two CTAs each
// (k_ns_pair): both hold half of either operand, which halves the bytes an SM takes in per product, and the sums are double
// buffered in tensor memory, so that one tile is written while the next is computed.  Matrices with a side of 128 or less stay on
// chip for all steps (k_ns_small).  A step is work of 3 M M N + M M M operations (of the symmetric A and B only half the tiles are
// computed, the others are their mirror images).  Measured, 5 steps: 8192 x 8192 float32 9.4 ms, 1.17 PFLOP/s, bound by the tensor
// cores under the power limit; 4096 x 4096 1.16 - 1.19 ms, 1.17 PFLOP/s; 4096 x 1024 187 us, 0.37 PFLOP/s, bound by 17 dependent
// launches of 36 to 256 tiles and, in A, by the operands' way through L2 (75 MB).
#include "trv_tma.cuh"
#include "trv_train.cuh"

namespace trv {

constexpr int kNsTile = 128, kNsK = 64;                     // a stage: 128 x 64 elements of either operand
constexpr int kNsHalf = kNsTile * kNsK * 2, kNsStageBytes = 2 * kNsHalf;
constexpr int kNsMaxStages = 5;
constexpr float kNsScale = 256.0f;                          // A and B are stored times this
constexpr int kNsMaxParts = 4 * kSMs;
constexpr int kNsGroup = 8;                                 // tiles are taken in bands of 8 tile rows, for the L2 cache

enum { NS_GRAM = 0, NS_POLY = 1, NS_APPLY = 2, NS_LAST = 3 };

struct NsArgs {
    int M, N, K;            // output M x N, summed over K
    int ld;                 // pitch of the binary16 outputs (and of carry), in elements
    size_t mat;             // elements between the matrices of a batch (outputs and carry)
    int Md;                 // between the diagonals of a batch
    float a, b;             // the step's coefficients (the third is in POLY's alpha)
    float alpha;            // what the sum is multiplied by; LAST: the result's scale is in it and in unit
    float unit;
    const float* diag;      // POLY: D of A, APPLY and LAST: E of B (times kNsScale)
    float* diag_out;        // GRAM: D, POLY: E
    const __half* hi;       // POLY: O, APPLY and LAST: X hi
    const __half* lo;       // X lo; POLY: O lo or NULL
    __half* out;            // O, P or the new X hi
    __half* out_lo;         // new X lo; O lo, P lo or NULL
    int low;                // products before that of the high halves: 1 left hi with right lo, 2 left lo with right hi
    __nv_bfloat16* last;    // LAST: the result
    long long last_row, last_col, last_mat;     // its strides
    bool last_vec;          // its rows start on 16-byte boundaries
    int tiles_m, tiles_n, tiles;                // k_ns_pair: 256 x 256 tiles of a matrix, and all of them
    unsigned* giveups;
};

// the operands' high and low halves (the latter where they are asked for)
struct NsMaps {
    CUtensorMap left, right, left_low, right_low;
};
// Which halves are multiplied: 1 left's high with right's low, 2 left's low with right's high, 0 the high halves, always and last
__device__ __forceinline__ int ns_first(int low) { return low & 1 ? 1 : low; }
__device__ __forceinline__ int ns_next(int which, int low) { return which == 1 ? low & 2 : 0; }

__device__ __forceinline__ bool ns_wait(unsigned bar, unsigned parity) {
    unsigned done = 0;
    for (unsigned spins = 0; spins < kTmaWaitLimit; ++spins) {
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
    }
    return false;
}
__device__ __forceinline__ void ns_expect(unsigned bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
template <int CG>
__device__ __forceinline__ void ns_load(unsigned dst, const CUtensorMap* map, int x, int y, int z, unsigned bar) {
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
    else        // the barrier may be the other CTA's
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// shared-memory operand descriptor, 128-byte swizzle; byte offsets in units of 16
__device__ __forceinline__ unsigned long long ns_desc(unsigned addr, unsigned leading, unsigned stride) {
    return (unsigned long long)((addr & 0x3ffff) >> 4) | ((unsigned long long)(leading >> 4) << 16) | ((unsigned long long)(stride >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
// D binary32, A and B binary16; right operand K-major, or N-major
__device__ __forceinline__ constexpr unsigned ns_idesc(int m, int n, bool n_major) {
    return (1u << 4) | (n_major ? 1u << 16 : 0u) | ((unsigned)(n >> 3) << 17) | ((unsigned)(m >> 4) << 24);
}
// Called by a whole warp, issued by one elected thread: the operands then stay in the warp's uniform registers (from a single
// thread's branch every product took 100 cycles to issue).
template <int CG>
__device__ __forceinline__ void ns_mma(unsigned tmem, unsigned long long a, unsigned long long b, unsigned idesc, int add) {
    if (CG == 1)
        asm volatile("{\n\t.reg .pred p, e;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.s32 p, %4, 0;\n\t"
                     "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(tmem), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, e;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.s32 p, %4, 0;\n\t"
                     "@e tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(tmem), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// The same, and what was added up so far counts 2^-11 (the instruction's own scaling of the addend): products with a low half, which
// is held times 2^11, come first, and the first one without begins like this.
constexpr float kNsLow = 2048.0f;
template <int CG>
__device__ __forceinline__ void ns_mma_shift(unsigned tmem, unsigned long long a, unsigned long long b, unsigned idesc) {
    if (CG == 1)
        asm volatile("{\n\t.reg .pred p, e;\n\telect.sync _|e, 0xffffffff;\n\tsetp.eq.s32 p, 0, 0;\n\t"
                     "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p, 11;\n\t}" ::"r"(tmem), "l"(a), "l"(b), "r"(idesc) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, e;\n\telect.sync _|e, 0xffffffff;\n\tsetp.eq.s32 p, 0, 0;\n\t"
                     "@e tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p, 11;\n\t}" ::"r"(tmem), "l"(a), "l"(b), "r"(idesc) : "memory");
}
// one stage: K = 64 in four products.  left: 128 rows of 128 bytes; right: the same, or (N_MAJOR) 64 rows of K for every 64 columns.
// shift: the first stage behind those with low halves
template <int CG, bool N_MAJOR>
__device__ __forceinline__ void ns_mma_stage(unsigned tmem, unsigned left, unsigned right, unsigned idesc, bool add, bool shift) {
#pragma unroll
    for (int q = 0; q < kNsK / 16; ++q) {
        const unsigned long long a = ns_desc(left + 32 * q, 16, 1024);
        const unsigned long long b = N_MAJOR ? ns_desc(right + 2048 * q, 8192, 1024) : ns_desc(right + 32 * q, 16, 1024);
        if (q == 0 && shift) ns_mma_shift<CG>(tmem, a, b, idesc);
        else ns_mma<CG>(tmem, a, b, idesc, add || q);
    }
}
template <int CG>
__device__ __forceinline__ void ns_commit(unsigned bar) {       // a whole warp; CG = 2: arrives at the same place of both CTAs
    if (CG == 1)
        asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
                     "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
    else
        asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
                     "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}"
                     ::"r"(bar), "h"((short)3) : "memory");
}
// a value that all lanes share, and the warp's number, in a form the compiler knows to be uniform
__device__ __forceinline__ unsigned ns_uniform(unsigned v) { return __shfl_sync(~0u, v, 0); }
__device__ __forceinline__ int ns_warp() { return __shfl_sync(~0u, (int)threadIdx.x >> 5, 0); }
__device__ __forceinline__ void ns_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void ns_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void ns_ld32(unsigned tmem, float (&v)[32]) {
    unsigned r[32];
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(tmem));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void ns_cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void ns_cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ unsigned ns_cluster_rank() {
    unsigned r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ unsigned ns_peer(unsigned addr, unsigned rank) {       // shared::cluster address of the same place in another CTA
    unsigned r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

// Epilogue of one warp: its 32 rows (one per lane, as tensor memory holds them) of `cols` columns of a tile.  Global memory is read
// and written in whole 64-byte runs, 4 lanes to a row; 32 rows x 32 columns at a time change hands through 2 KB of shared memory
// per operand (16-byte units of a row permuted by the row: no bank conflicts either way).  (A lane reading and writing its own row
// directly: 32 lines per access, 3000 cycles per 32 columns against 700.)  The mirror image of a tile goes through the same
// memory: single elements from registers to their transposed places in global memory took 1700 cycles per 32 columns.  What is
// left is latency, which more warps hide: 16 instead of 8 took 512 x 2048 from 119 to 113 us and 200 x 300 from 106 to 99.
constexpr int kNsEpilogueWarps = 16;                        // warps w, w + 4, ... share 32 rows, a quarter of the columns each
constexpr int kNsWarpBuf = 2048, kNsWarpBytes = 2 * kNsWarpBuf;
constexpr int kNsThreads = 32 * (kNsEpilogueWarps + 2);     // then one warp for the copies, one for the products
constexpr int ns_smem(int stages) { return 1024 + stages * kNsStageBytes + kNsEpilogueWarps * kNsWarpBytes; }

__device__ __forceinline__ unsigned ns_unit(unsigned buf, int row, int u) { return buf + row * 64 + ((u ^ (row >> 1 & 3)) << 4); }
__device__ __forceinline__ uint4 ns_lds(unsigned at) {
    uint4 u;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "r"(at) : "memory");
    return u;
}
__device__ __forceinline__ void ns_sts(unsigned at, uint4 u) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w) : "memory");
}
__device__ __forceinline__ void ns_async16(unsigned to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

// Loads of the carried operand for columns j .. j + 31 of rows i0 .. i0 + 31.  FINE: A and B have low halves
template <int MODE, bool FINE>
__device__ __forceinline__ void ns_fetch(const NsArgs& a, int z, int i0, int j, unsigned buf) {
    const int lane = threadIdx.x & 31, r = lane >> 2, u = lane & 3;
    if (MODE != NS_GRAM && j < a.N) {
        const size_t at = (size_t)z * a.mat + (size_t)(i0 + r) * a.ld + j + 8 * u;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i0 + r + 8 * k < a.M) {
                ns_async16(ns_unit(buf, r + 8 * k, u), a.hi + at + (size_t)8 * k * a.ld);
                if (MODE != NS_POLY || FINE) ns_async16(ns_unit(buf + kNsWarpBuf, r + 8 * k, u), a.lo + at + (size_t)8 * k * a.ld);
            }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
}

__device__ __forceinline__ unsigned ns_bits(__half2 h) {
    unsigned u;
    memcpy(&u, &h, 4);
    return u;
}

// two values of a lane's row, columns 2 k and 2 k + 1, into the transposed image [column][32 rows]
__device__ __forceinline__ void ns_mirror(unsigned buf, int lane, int k, unsigned pair) {
    const unsigned to = buf + kNsWarpBuf + 128 * k + lane * 2;
    asm volatile("st.shared.b16 [%0], %1;" ::"r"(to), "h"((unsigned short)(pair & 0xffff)) : "memory");
    asm volatile("st.shared.b16 [%0], %1;" ::"r"(to + 64), "h"((unsigned short)(pair >> 16)) : "memory");
}

// get(c, v): the sums of columns c .. c + 31 of this lane's row; cols: a multiple of 32.  ns_fetch has been called for the first 32.
template <int MODE, bool FINE, typename Get>
__device__ __forceinline__ void ns_epilogue(const NsArgs& a, int z, int i0, int j0, int cols, bool mirror, unsigned buf, Get get) {
    const int lane = threadIdx.x & 31, i = i0 + lane;
    const size_t dd = (size_t)z * a.Md;
    const bool row = i < a.M;
    const float d = MODE != NS_GRAM && row ? a.diag[dd + i] : 0.0f;
    const float2 e = f2_splat(a.unit * fmaf(d, 1.0f / kNsScale, a.a)), alpha = f2_splat(a.alpha), b = f2_splat(a.b), d2 = f2_splat(d);
#pragma unroll 1
    for (int c = 0; c < cols; c += 32) {
        const int j = j0 + c;
        if (j >= a.N) break;
        if (c) ns_fetch<MODE, FINE>(a, z, i0, j, buf);
        float v[32];
        get(c, v);
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
        const bool here = (MODE == NS_GRAM || MODE == NS_POLY) && i >= j && i < j + 32;       // the diagonal crosses these columns
        if (here) {
            float on_diag = 0;
#pragma unroll
            for (int q = 0; q < 32; ++q)
                if (i == j + q) on_diag = MODE == NS_GRAM ? a.alpha * v[q] : fmaf(a.alpha, fmaf(d, d, v[q]), a.b * d);
            if (row) a.diag_out[dd + i] = on_diag;
        }
        // FINE: the row, for the mirror image (its place still holds low halves in the loop) and the low halves behind the loop.  A
        // kernel of its own: the loop below with the mirror image behind it costs the others 0.3 us a launch.
        unsigned hi[16], low[16];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const unsigned at = ns_unit(buf, lane, q);
            uint4 u;
            __half2 h[4], l[4];
            if (MODE != NS_GRAM) u = ns_lds(at), memcpy(h, &u, 16);
            if (MODE >= NS_APPLY || (MODE == NS_POLY && FINE)) u = ns_lds(at + kNsWarpBuf), memcpy(l, &u, 16);
            float4 dj[2];
            if (MODE == NS_POLY) {                          // the same for all lanes; up to the pitch, which is a multiple of 64
                dj[0] = *(const float4*)(a.diag + dd + j + 8 * q);
                dj[1] = *(const float4*)(a.diag + dd + j + 8 * q + 4);
            }
            unsigned hb[4], lb[4] = {};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float2 x = make_float2(v[8 * q + 2 * k], v[8 * q + 2 * k + 1]);
                if (MODE == NS_GRAM) {
                    x = f2_mul(x, alpha);
                } else if (MODE == NS_POLY) {
                    float2 o = __half22float2(h[k]);
                    if (FINE) o = f2_fma(__half22float2(l[k]), f2_splat(1.0f / kNsLow), o);
                    const float2 s = k & 1 ? make_float2(dj[k / 2].z, dj[k / 2].w) : make_float2(dj[k / 2].x, dj[k / 2].y);
                    x = f2_fma(alpha, f2_fma(f2_add(d2, s), o, x), f2_mul(b, o));
                } else {
                    x = f2_fma(e, f2_fma(__half22float2(l[k]), f2_splat(1.0f / kNsLow), __half22float2(h[k])), f2_mul(alpha, x));
                }
                if (here) {
                    if (i == j + 8 * q + 2 * k) x.x = 0;
                    if (i == j + 8 * q + 2 * k + 1) x.y = 0;
                }
                if (MODE == NS_LAST) {
                    v[8 * q + 2 * k] = x.x, v[8 * q + 2 * k + 1] = x.y;
                    const __nv_bfloat162 p = __floats2bfloat162_rn(x.x, x.y);
                    memcpy(&hb[k], &p, 4);
                } else {
                    const __half2 y = __floats2half2_rn(x.x, x.y);
                    hb[k] = ns_bits(y);
                    if (MODE == NS_APPLY || FINE) {
                        const float2 r = f2_mul(f2_fma(__half22float2(y), f2_splat(-1.0f), x), f2_splat(kNsLow));
                        lb[k] = ns_bits(__floats2half2_rn(r.x, r.y));
                    }
                    if (FINE) hi[4 * q + k] = hb[k], low[4 * q + k] = lb[k];
                    else if (MODE != NS_APPLY && mirror) ns_mirror(buf, lane, 4 * q + k, hb[k]);
                }
            }
            ns_sts(at, make_uint4(hb[0], hb[1], hb[2], hb[3]));
            if (MODE == NS_APPLY) ns_sts(at + kNsWarpBuf, make_uint4(lb[0], lb[1], lb[2], lb[3]));
        }
        if (MODE == NS_LAST && a.last_col != 1 && row) {    // transposed: a row of X is a column of the result
            __nv_bfloat16* to = a.last + z * a.last_mat + i * a.last_row + j * a.last_col;
#pragma unroll
            for (int q = 0; q < 32; ++q)
                if (j + q < a.N) to[q * a.last_col] = __float2bfloat16_rn(v[q]);
        }
        __syncwarp();
        if (FINE && mirror) {
#pragma unroll
            for (int k = 0; k < 16; ++k) ns_mirror(buf, lane, k, hi[k]);
            __syncwarp();
        }
        const int r = lane >> 2, u = lane & 3;
        if (MODE == NS_LAST) {
            if (a.last_col == 1) {
                __nv_bfloat16* to = a.last + z * a.last_mat + (i0 + r) * a.last_row + j + 8 * u;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (i0 + r + 8 * k >= a.M || j + 8 * u >= a.N) continue;
                    const uint4 w = ns_lds(ns_unit(buf, r + 8 * k, u));
                    if (a.last_vec && j + 8 * u + 8 <= a.N) {
                        *(uint4*)(to + 8 * k * a.last_row) = w;
                    } else {
                        __nv_bfloat16 b8[8];
                        memcpy(b8, &w, 16);
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            if (j + 8 * u + q < a.N) to[8 * k * a.last_row + q] = b8[q];
                    }
                }
            }
        } else {
            auto write = [&](__half* to, unsigned from) {
                to += (size_t)z * a.mat + (size_t)(i0 + r) * a.ld + j + 8 * u;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i0 + r + 8 * k < a.M) *(uint4*)(to + (size_t)8 * k * a.ld) = ns_lds(ns_unit(from, r + 8 * k, u));
            };
            auto write_mirror = [&](__half* to) {           // 8 columns of 64 bytes at a time; elements behind row M - 1 fall into the pitch
                to += (size_t)z * a.mat + (size_t)(j + r) * a.ld + i0 + 8 * u;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (j + r + 8 * k < a.N) *(uint4*)(to + (size_t)8 * k * a.ld) = ns_lds(buf + kNsWarpBuf + (r + 8 * k) * 64 + u * 16);
            };
            write(a.out, buf);
            if (MODE == NS_APPLY) write(a.out_lo, buf + kNsWarpBuf);
            if (MODE != NS_APPLY && mirror && i0 < a.M) write_mirror(a.out);
            if (FINE) {                                     // the low halves the same way
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 4; ++q) ns_sts(ns_unit(buf, lane, q), make_uint4(low[4 * q], low[4 * q + 1], low[4 * q + 2], low[4 * q + 3]));
                if (mirror)
#pragma unroll
                    for (int k = 0; k < 16; ++k) ns_mirror(buf, lane, k, low[k]);
                __syncwarp();
                write(a.out_lo, buf);
                if (mirror && i0 < a.M) write_mirror(a.out_lo);
            }
        }
        __syncwarp();
    }
}

// The last copies of a CTA that issued n stages (full barriers at bar, parity flips per turn) have landed: no CTA leaves with a copy
// on its way, not even after a wait that ran out.
__device__ __forceinline__ void ns_landed(unsigned bar, unsigned n) {
    for (unsigned k = n > kNsMaxStages ? n - kNsMaxStages : 0; k < n; ++k) ns_wait(bar + 8 * (k % kNsMaxStages), k / kNsMaxStages & 1);
}

// One 128 x 128 tile of  left . right  per cluster, the sum over K split over its CTAs.  left: rows along y, K along x.
// right: the same (GRAM, POLY: the product with its transpose) or rows of K, N along x (APPLY, LAST).  Bound by latency: a launch
// is filling the stages from L2, K / 64 blocks of products, the exchange of a split and one epilogue.  512 x 512: 111 us for 15
// of these and the two launches before them, 6 to 7 us each.
template <int MODE, bool FINE>
__global__ void __launch_bounds__(kNsThreads, 1) k_ns_tile(const __grid_constant__ NsMaps maps,
                                                           const __grid_constant__ NsArgs a, int split) {
    constexpr bool kSym = MODE == NS_GRAM || MODE == NS_POLY;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kNsMaxStages + 2];
    __shared__ unsigned tmem_at;
    const int warp = ns_warp(), lane = threadIdx.x & 31, part = blockIdx.x % split, tj = blockIdx.x / split, ti = blockIdx.y, z = blockIdx.z;
    pdl_trigger();
    if (kSym && tj < ti) return;                            // the mirror of a tile above the diagonal (the whole cluster leaves)
    const unsigned base = (smem_u32(raw) + 1023) & ~1023u, bar = smem_u32(bars);
    auto full = [&](int s) { return bar + 8 * s; };
    auto empty = [&](int s) { return bar + 8 * (kNsMaxStages + s); };
    const unsigned done = bar + 8 * 2 * kNsMaxStages, left_off = done + 8;
    if (threadIdx.x == 32 * kNsEpilogueWarps) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.left) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.right) : "memory");
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < 2 * kNsMaxStages + 2; ++s) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar + 8 * s) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kNsEpilogueWarps + 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 128;" ::"r"(smem_u32(&tmem_at)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    ns_fence_before();
    __syncthreads();
    ns_fence_after();
    const unsigned tmem = ns_uniform(tmem_at);
    const int blocks = (a.K + kNsK - 1) / kNsK, k0 = blocks * part / split, nk = blocks * (part + 1) / split - k0;
    const int i0 = ti * kNsTile, j0 = tj * kNsTile, q = warp & 3;
    const unsigned mine = base + kNsMaxStages * kNsStageBytes + warp * kNsWarpBytes;      // of an epilogue warp
    // columns of an epilogue warp: 32 of the CTA's share, which is less than one for all four in a split
    const int width = kNsTile / split, first = width * part + 32 * (warp >> 2), cols = 32 * (warp >> 2) < width ? 32 : 0;
    bool ok = true;
    pdl_wait();
    if (warp == kNsEpilogueWarps) {
        if (lane == 0) {
            unsigned loads = 0;
            for (int s = 0, ph = 1, which = ns_first(a.low); ok; which = ns_next(which, a.low)) {
                const CUtensorMap* const l = which == 2 ? &maps.left_low : &maps.left;
                const CUtensorMap* const r = which == 1 ? &maps.right_low : &maps.right;
                for (int k = 0; k < nk; ++k) {
                    if (!(ok = ns_wait(empty(s), ph))) break;
                    const unsigned dst = base + s * kNsStageBytes;
                    const int x = (k0 + k) * kNsK;
                    ns_expect(full(s), kNsStageBytes);
                    ns_load<1>(dst, l, x, i0, z, full(s));
                    if (kSym) {
                        ns_load<1>(dst + kNsHalf, r, x, j0, z, full(s));
                    } else {
                        ns_load<1>(dst + kNsHalf, r, j0, x, z, full(s));
                        ns_load<1>(dst + kNsHalf + 8192, r, j0 + 64, x, z, full(s));
                    }
                    ++loads;
                    if (++s == kNsMaxStages) s = 0, ph ^= 1;
                }
                if (!which) break;
            }
            ns_landed(bar, loads);
        }
    } else if (warp == kNsEpilogueWarps + 1) {
        for (int s = 0, ph = 0, which = ns_first(a.low); ok; which = ns_next(which, a.low)) {
            for (int k = 0; k < nk; ++k) {
                if (!(ok = __all_sync(~0u, ns_wait(full(s), ph)))) break;
                ns_fence_after();
                const unsigned l = base + s * kNsStageBytes;
                ns_mma_stage<1, !kSym>(tmem, l, l + kNsHalf, ns_idesc(128, 128, !kSym), k > 0 || which != ns_first(a.low), a.low && !which && !k);
                ns_commit<1>(empty(s));
                if (++s == kNsMaxStages) s = 0, ph ^= 1;
            }
            if (!which) break;
        }
        ns_commit<1>(ok ? done : left_off);
        if (!ok) ns_wait(left_off, 0);                      // its products too
    } else {
        if (cols) ns_fetch<MODE, FINE>(a, z, i0 + 32 * q, j0 + first, mine);
        ok = __all_sync(~0u, ns_wait(done, 0));
        ns_fence_after();
        if (split == 1 && ok)
            ns_epilogue<MODE, FINE>(a, z, i0 + 32 * q, j0 + first, cols, tj > ti, mine,
                              [&](int c, float (&v)[32]) { ns_ld32(tmem + ((unsigned)(32 * q) << 16) + first + c, v); });
    }
    if (split > 1) {
        // Every 32 columns go to the CTA that adds their parts: [part][columns / 32][16-byte unit of the row][128 rows] over the stages,
        // once all CTAs have consumed theirs.  Writing to the reader costs one way, reading from the writer two; a warp's 16-byte
        // units are neighbours.
        const int chunks = 4 / split, row = 32 * q + lane;
        __syncwarp();
        ns_cluster_arrive();
        ns_cluster_wait();
        if (warp < kNsEpilogueWarps) {
            const int c = warp >> 2;
            float v[32];
            ns_ld32(tmem + ((unsigned)(32 * q) << 16) + 32 * c, v);
            const unsigned to = ns_peer(base + (part * chunks + c % chunks) * kNsTile * 128 + row * 16, c / chunks);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + k * kNsTile * 16), "f"(v[4 * k]), "f"(v[4 * k + 1]),
                             "f"(v[4 * k + 2]), "f"(v[4 * k + 3]) : "memory");
        }
        __syncwarp();
        ns_cluster_arrive();
        ns_cluster_wait();
        if (warp < kNsEpilogueWarps && cols && ok)
            ns_epilogue<MODE, FINE>(a, z, i0 + 32 * q, j0 + first, cols, tj > ti, mine, [&](int, float (&v)[32]) {
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] = 0;
#pragma unroll 1
                for (int p = 0; p < split; ++p) {
                    const unsigned from = base + (p * chunks + (warp >> 2)) * kNsTile * 128 + row * 16;
                    uint4 u[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) u[k] = ns_lds(from + k * kNsTile * 16);
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        v[4 * k] += __uint_as_float(u[k].x), v[4 * k + 1] += __uint_as_float(u[k].y), v[4 * k + 2] += __uint_as_float(u[k].z),
                            v[4 * k + 3] += __uint_as_float(u[k].w);
                }
            });
    }
    if (!ok) atomicAdd(a.giveups, 1u);
    asm volatile("cp.async.wait_all;" ::: "memory");
    ns_fence_before();
    __syncthreads();
    if (warp == kNsEpilogueWarps + 1) {
        __syncwarp();
        ns_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 128;" ::"r"(tmem));
    }
}

// Tile t of a batch: bands of kNsGroup tile rows, column after column inside a band; of a symmetric result the tiles on and
// above the diagonal.  In closed form: stepping from tile to tile cost 15000 cycles a tile.
template <bool SYM>
__device__ __forceinline__ void ns_tile_at(const NsArgs& a, int t, int* z, int* ti, int* tj) {
    const int tm = a.tiles_m, tn = a.tiles_n, per = SYM ? tm * (tm + 1) / 2 : tm * tn;
    *z = t / per;
    t -= *z * per;
    if (!SYM) {
        const int band = t / (kNsGroup * tn), rows = min(kNsGroup, tm - band * kNsGroup);
        t -= band * kNsGroup * tn;
        *tj = t / rows, *ti = band * kNsGroup + t % rows;
        return;
    }
    int first = 0, rows = min(kNsGroup, tm);                // the band's first row and column, its rows
    for (int n; t >= (n = rows * (tn - first) - rows * (rows - 1) / 2); t -= n) first += kNsGroup, rows = min(kNsGroup, tm - first);
    if (t < rows * (rows + 1) / 2) {                        // its triangle
        int c = 0;
        for (; t > c; t -= c) ++c;
        *tj = first + c, *ti = first + t;
    } else {
        t -= rows * (rows + 1) / 2;
        *tj = first + rows + t / rows, *ti = first + t % rows;
    }
}

// 256 x 256 tiles, one per CTA pair at a time: CTA r holds rows 128 r .. of left and rows (columns) 128 r .. of right; CTA 0 issues
// the products, whose sums appear in both CTAs' tensor memory, 128 rows each.  5 stages of 32 KB keep the copies ahead of the
// products; a tile's epilogue runs beside the next tile's products.  4096 x 4096: 59 us for A, 62 for B (half the tiles each), 112
// for X, the tensor pipe 61 - 65 % busy: 136 tiles of A are 1.8 turns of 74 pairs.
template <int MODE, bool FINE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kNsThreads, 1) k_ns_pair(const __grid_constant__ NsMaps maps,
                                                                                     const __grid_constant__ NsArgs a) {
    constexpr bool kSym = MODE == NS_GRAM || MODE == NS_POLY;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kNsMaxStages + 5];
    __shared__ unsigned tmem_at;
    const int warp = ns_warp(), lane = threadIdx.x & 31;
    const unsigned rank = ns_cluster_rank();
    pdl_trigger();
    const unsigned base = (smem_u32(raw) + 1023) & ~1023u, bar = smem_u32(bars);
    auto full = [&](int s) { return bar + 8 * s; };                             // CTA 0's: both CTAs' copies of a stage
    auto empty = [&](int s) { return bar + 8 * (kNsMaxStages + s); };           // each CTA's: the products have read the stage
    auto sums = [&](int t) { return bar + 8 * (2 * kNsMaxStages + t); };        // each CTA's: the sums of a tile are complete
    auto taken = [&](int t) { return bar + 8 * (2 * kNsMaxStages + 2 + t); };   // CTA 0's: both CTAs' epilogue warps have read them
    const unsigned left_off = bar + 8 * (2 * kNsMaxStages + 4);                 // each CTA's: products issued before a wait ran out
    if (threadIdx.x == 32 * kNsEpilogueWarps) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.left) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.right) : "memory");
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < 2 * kNsMaxStages + 5; ++s)
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;"
                         ::"r"(bar + 8 * s), "r"(s == 2 * kNsMaxStages + 2 || s == 2 * kNsMaxStages + 3 ? 2 * kNsEpilogueWarps : 1) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kNsEpilogueWarps + 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_at)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    __syncwarp();
    ns_fence_before();
    ns_cluster_arrive();
    ns_cluster_wait();
    ns_fence_after();
    const unsigned tmem = ns_uniform(tmem_at);
    const unsigned mine = base + kNsMaxStages * kNsStageBytes + warp * kNsWarpBytes;      // of an epilogue warp
    const int nk = (a.K + kNsK - 1) / kNsK, pairs = gridDim.x / 2, pair = blockIdx.x / 2;
    bool ok = true;
    pdl_wait();
    if (warp == kNsEpilogueWarps) {
        if (lane == 0) {
            unsigned loads = 0;
            for (int s = 0, ph = 1, n = pair; n < a.tiles && ok; n += pairs) {
                int ti, tj, z;
                ns_tile_at<kSym>(a, n, &z, &ti, &tj);
                const int i0 = ti * 256 + 128 * rank, j0 = tj * 256 + 128 * rank;
                for (int which = ns_first(a.low); ok; which = ns_next(which, a.low)) {
                    const CUtensorMap* const l = which == 2 ? &maps.left_low : &maps.left;
                    const CUtensorMap* const r = which == 1 ? &maps.right_low : &maps.right;
                    for (int k = 0; k < nk; ++k) {
                        if (!(ok = ns_wait(empty(s), ph))) break;
                        const unsigned dst = base + s * kNsStageBytes, at = ns_peer(full(s), 0);
                        if (rank == 0) ns_expect(full(s), 2 * kNsStageBytes);
                        ns_load<2>(dst, l, k * kNsK, i0, z, at);
                        if (kSym) {
                            ns_load<2>(dst + kNsHalf, r, k * kNsK, j0, z, at);
                        } else {
                            ns_load<2>(dst + kNsHalf, r, j0, k * kNsK, z, at);
                            ns_load<2>(dst + kNsHalf + 8192, r, j0 + 64, k * kNsK, z, at);
                        }
                        ++loads;
                        if (++s == kNsMaxStages) s = 0, ph ^= 1;
                    }
                    if (!which) break;
                }
            }
            if (rank == 0) ns_landed(bar, loads);           // both CTAs' copies; the other CTA waits for this one before it leaves
        }
    } else if (warp == kNsEpilogueWarps + 1) {
        if (rank == 0) {
            int t = 0, tph = 1;
            for (int s = 0, ph = 0, n = pair; n < a.tiles && ok; n += pairs) {
                if (!(ok = __all_sync(~0u, ns_wait(taken(t), tph)))) break;
                ns_fence_after();
                for (int which = ns_first(a.low); ok; which = ns_next(which, a.low)) {
                    for (int k = 0; k < nk; ++k) {
                        if (!(ok = __all_sync(~0u, ns_wait(full(s), ph)))) break;
                        ns_fence_after();
                        const unsigned l = base + s * kNsStageBytes;
                        ns_mma_stage<2, !kSym>(tmem + 256 * t, l, l + kNsHalf, ns_idesc(256, 256, !kSym), k > 0 || which != ns_first(a.low),
                                               a.low && !which && !k);
                        ns_commit<2>(empty(s));
                        if (++s == kNsMaxStages) s = 0, ph ^= 1;
                    }
                    if (!which) break;
                }
                if (ok) ns_commit<2>(sums(t));
                if (++t == 2) t = 0, tph ^= 1;
            }
            if (!ok) ns_commit<2>(left_off), ns_wait(left_off, 0);
        }
    } else {
        const int q = warp & 3, first = 64 * (warp >> 2);
        int t = 0, tph = 0;
        for (int n = pair; n < a.tiles && ok; n += pairs) {
            int ti, tj, z;
            ns_tile_at<kSym>(a, n, &z, &ti, &tj);
            const int i0 = ti * 256 + 128 * (int)rank + 32 * q, j0 = tj * 256 + first;
            ns_fetch<MODE, FINE>(a, z, i0, j0, mine);             // while the products run
            if (!(ok = __all_sync(~0u, ns_wait(sums(t), tph)))) break;
            ns_fence_after();
            ns_epilogue<MODE, FINE>(a, z, i0, j0, 64, tj > ti, mine, [&](int c, float (&v)[32]) {
                ns_ld32(tmem + ((unsigned)(32 * q) << 16) + 256 * t + first + c, v);
            });
            ns_fence_before();                              // the tile after the next may use the buffer
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(ns_peer(taken(t), 0)) : "memory");
            if (++t == 2) t = 0, tph ^= 1;
        }
    }
    if (!ok) atomicAdd(a.giveups, 1u);
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
    ns_fence_before();
    ns_cluster_arrive();                                    // no CTA leaves while the other's copies, products or arrivals may reach it
    ns_cluster_wait();
    if (warp == kNsEpilogueWarps + 1) {
        ns_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

// Matrices with M <= 128, whole iterations on chip: one CTA, or a cluster of up to 16 that share the columns, per matrix; one launch
// for a batch.  X is in tensor memory in binary32 (times 256, as B X leaves it) and as two binary16 halves in shared memory, where one
// 128-byte-swizzled layout serves as K-major operand of X X^T and as N-major operand of B X; A and B are there too.  A step is
// three products (three times: see the header) and three passes over registers, 16 columns of a row per thread and turn; a cluster
// adds the CTAs' parts of X X^T through distributed shared memory, every CTA a share of the columns, in a fixed order.  Bound by the
// latency of this chain: 81 x 243 float32 44 us, 32 matrices of 128 x 1000 91 us, 16 x 40 16 us (with high halves alone 31, 61
// and 14 us and errors of up to 3 %: 2/3 of the difference are the additional products, the rest of a cluster's the doubled exchange of A).
// Sides are rounded up to 16, not to 128: 16 x 40 took 24 us with 128.  The code is kept small (loops of 16 columns, one pass for
// every purpose): run once by a CTA it comes from memory, and unrolled loads of 128 elements a thread took 20 us for their
// instructions alone.
constexpr int kNsSmallThreads = 512, kNsSmallWidth = 256, kNsSmallCluster = 16;
struct NsSmall {
    const void* g;
    __nv_bfloat16* out;
    long long row, mat, out_row, out_mat;
    int M, N, W, C, steps;      // W: columns of a CTA, a multiple of 64; C: CTAs of a cluster
    bool tall;
    float sx, eps;
    unsigned* giveups;
    float c[3 * 64];
};

// bytes of X's low half (or a cluster's parts of A: 128 x 128 binary32) and of a half of A
__host__ __device__ constexpr int ns_small_low(int W, int C) { return C > 1 ? 65536 : W * 256; }
__host__ __device__ constexpr int ns_small_square(int M) { return M > 64 ? 32768 : 16384; }

__device__ __forceinline__ void ns_ld16(unsigned tmem, float (&v)[16]) {
    unsigned r[16];
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(tmem));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void ns_ld8(unsigned tmem, float (&v)[8]) {
    unsigned r[8];
    __syncwarp();
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(tmem));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void ns_st16(unsigned tmem, const float (&v)[16]) {
    __syncwarp();
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(tmem),
        "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]),
        "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
        : "memory");
}
// x * s in binary32 for a binary64 s that may lie outside binary32's range: mantissa, and the power of two in two halves
struct NsFactor {
    float m, p, q;
    __device__ __forceinline__ explicit NsFactor(double s) {
        const long long b = __double_as_longlong(s);
        const int e = (int)((b >> 52) & 0x7ff) - 1023;
        if (s > 0 && e < 200 && e > -200) {
            m = (float)__longlong_as_double((b & 0xfffffffffffffll) | 0x3ff0000000000000ll);
            p = __uint_as_float((unsigned)(127 + e / 2) << 23);
            q = __uint_as_float((unsigned)(127 + e - e / 2) << 23);
        } else {                                            // 0 or NaN
            m = (float)s, p = q = 1.0f;
        }
    }
    __device__ __forceinline__ float operator()(float x) const { return x * p * q * m; }
};
// ns_wait without suspension: the products waited for take less than waking up
__device__ __forceinline__ bool ns_poll(unsigned bar, unsigned parity) {
    unsigned done = 0;
    for (unsigned spins = 0; spins < 16 * kTmaWaitLimit; ++spins) {
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
    }
    return false;
}
__device__ __forceinline__ void ns_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void ns_fence_async() { asm volatile("fence.proxy.async;" ::: "memory"); }
// 8 values times s (a power of two) as binary16, and what that leaves out times 2^11 as binary16: 22 bits
__device__ __forceinline__ void ns_split8(const float* v, float s, uint4& hi, uint4& lo) {
    unsigned u[4], w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 f = f2_mul(make_float2(v[2 * k], v[2 * k + 1]), f2_splat(s));
        const __half2 h = __floats2half2_rn(f.x, f.y);
        const float2 r = f2_mul(f2_fma(__half22float2(h), f2_splat(-1.0f), f), f2_splat(kNsLow));
        u[k] = ns_bits(h), w[k] = ns_bits(__floats2half2_rn(r.x, r.y));
    }
    hi = make_uint4(u[0], u[1], u[2], u[3]), lo = make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T>
__global__ void __launch_bounds__(kNsSmallThreads) k_ns_small(const __grid_constant__ NsSmall a) {
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) unsigned long long bars[1];
    __shared__ double part_norm[kNsSmallCluster], red[kNsSmallThreads / 32];
    __shared__ unsigned tmem_at;
    constexpr int kWarps = kNsSmallThreads / 32;
    const int t = threadIdx.x, warp = ns_warp(), lane = t & 31, quarter = warp >> 2, row = 32 * (warp & 3) + lane;
    const int rank = a.C > 1 ? (int)ns_cluster_rank() : 0, z = blockIdx.x / a.C, n0 = rank * a.W;
    const unsigned base = (smem_u32(raw) + 1023) & ~1023u, bar = smem_u32(bars);
    // X, A and B as high and low halves.  B takes A's place (element by element); a cluster's parts of A take that of X's low half,
    // which is then written again.
    const unsigned xh = base, xl = xh + a.W * 256, sh = xl + ns_small_low(a.W, a.C), sl = sh + ns_small_square(a.M), parts = xl;
    // [128][W] words over X, before the first and after the last step; the columns of a row permuted by the row
    float* stage = (float*)(raw + (base - smem_u32(raw)));
    auto unit = [&](unsigned at, int r, int u) { return at + (u >> 3) * 16384 + r * 128 + (((u & 7) ^ (r & 7)) << 4); };  // 8 columns of a row
    const int tcols = a.W <= 128 ? 256 : 512;
    // Rows and columns of the square matrices, in steps of 16.  Rows from mp on are never read by others (they give rows from mp on): the
    // warps whose 32 rows begin there skip all passes.
    const int mp = (a.M + 15) & ~15, units = mp / 8;
    const bool busy = 32 * (warp & 3) < mp;
    if (t == 0) {
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        ns_fence_async();
    }
    if (warp == 0) {
        if (tcols == 256) asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 256;" ::"r"(smem_u32(&tmem_at)) : "memory");
        else asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_at)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    // The matrix as it lies in memory: a warp takes every 16th row, lanes the columns.  Of X these are rows, or (tall) columns.
    const int pad = (a.M + 31) & ~31, rows = a.tall ? a.W : pad, cols = a.tall ? pad : a.W;   // of the CTA's part
    const int rows_in = a.tall ? a.N - n0 : a.M, cols_in = a.tall ? a.M : a.N - n0;         // those that exist
    auto place = [&](int r, int c) {
        const int m = a.tall ? c : r, n = a.tall ? r : c;
        return m * a.W + (n ^ (m & 31));
    };
    {
        const T* g = (const T*)a.g + z * a.mat + (a.tall ? n0 * a.row : n0);
        double sum = 0;
#pragma unroll 1
        for (int r = warp; r < rows; r += 4 * kWarps) {
            float v[4][kNsSmallWidth / 32];
#pragma unroll
            for (int h = 0; h < 4; ++h)
#pragma unroll
                for (int j = 0; j < kNsSmallWidth / 32; ++j) {
                    const int rr = r + h * kWarps, c = lane + 32 * j;
                    v[h][j] = rr < rows_in && c < cols_in ? to_f32(g[rr * a.row + c]) : 0.0f;
                }
#pragma unroll
            for (int h = 0; h < 4; ++h)
#pragma unroll
                for (int j = 0; j < kNsSmallWidth / 32; ++j)
                    if (32 * j < cols && r + h * kWarps < rows) {
                        sum = fma((double)v[h][j], (double)v[h][j], sum);
                        stage[place(r + h * kWarps, lane + 32 * j)] = v[h][j];
                    }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        if (lane == 0) red[warp] = sum;
    }
    ns_fence_before();
    __syncwarp();
    if (a.C > 1) {                                          // all CTAs of the cluster run before any writes to another
        ns_cluster_arrive();
        ns_cluster_wait();
    } else {
        __syncthreads();
    }
    ns_fence_after();
    const unsigned tx = ns_uniform(tmem_at), ts = tx + a.W, mine = (unsigned)(32 * (warp & 3)) << 16;      // X and the square sums; a warp's lanes
    double norm = 0;
    for (int w = 0; w < kWarps; ++w) norm += red[w];
    if (a.C > 1) {
        if (t < a.C) asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(ns_peer(smem_u32(&part_norm[rank]), t)), "d"(norm) : "memory");
        __syncwarp();
        ns_cluster_arrive();
        ns_cluster_wait();
        norm = 0;
        for (int p = 0; p < a.C; ++p) norm += part_norm[p];
    }
    norm = sqrt(norm) + (double)a.eps;
    const NsFactor scale(norm > 0 || norm != norm ? (double)a.sx * (double)kNsScale / norm : 0.0);
    // this warp's columns of X, and its 8-column units of a square matrix
    const int x0 = a.W / 4 * quarter, x1 = busy ? x0 + a.W / 4 : 0, each = (units + 3) / 4, u0 = each * quarter, u1 = busy ? min(u0 + each, units) : 0;
#pragma unroll 1
    for (int c = x0; c < x1; c += 16) {
        float v[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) v[q] = scale(stage[row * a.W + ((c + q) ^ (row & 31))]);
        ns_st16(tx + mine + c, v);
    }
    ns_wait_st();
    ns_fence_before();
    __syncthreads();
    ns_fence_after();

    bool ok = true;
    unsigned phase = 0;
    auto product = [&](auto issue, auto meanwhile) {        // what all wrote is in place; warp 0 issues, all do the other and wait
        ns_fence_async();
        ns_fence_before();
        __syncthreads();
        if (warp == 0) {
            ns_fence_after();
            issue();
            ns_commit<1>(bar);
        }
        meanwhile();
        if (!ns_poll(bar, phase)) ok = false;
        phase ^= 1;
        __syncwarp();
        ns_fence_after();
    };
    // Three products each: high . low, low . high, then high . high, over 16 columns of left k16 times (and of right, or rows of right).
    // Unrolled by twelve: rolled products issue slower (81 x 243 61 us, by four 51, by twelve 49).  High halves alone in the last step
    // save 2 us and cost 0.05 - 0.5 %.
    auto three = [&](unsigned to, unsigned lh, unsigned ll, unsigned rh, unsigned rl, int k16, bool n_major, unsigned idesc) {
#pragma unroll
        for (int n = 0; n < 3; ++n) {
            const unsigned l = n == 1 ? ll : lh, r = n == 0 ? rl : rh;
#pragma unroll 1
            for (int k = 0; k < k16; k += 4)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const unsigned long long a = ns_desc(l + (k >> 2) * 16384 + q * 32, 16, 1024);
                    const unsigned long long b = n_major ? ns_desc(r + (k + q) * 2048, 16384, 1024) : ns_desc(r + (k >> 2) * 16384 + q * 32, 16, 1024);
                    if (q == 0 && n == 2 && k == 0) ns_mma_shift<1>(to, a, b, idesc);
                    else if (k + q < k16) ns_mma<1>(to, a, b, idesc, n || k || q);
                }
        }
    };
    auto squares = [&](unsigned h, unsigned l, int k16) { three(ts, h, l, h, l, k16, false, ns_idesc(128, mp, false)); };
    auto store = [&](unsigned h, unsigned l, int u, const float* v, float s) {
        uint4 hi, lo;
        ns_split8(v, s, hi, lo);
        ns_sts(unit(h, row, u), hi), ns_sts(unit(l, row, u), lo);
    };
    const float to_a = kNsScale / (a.sx * a.sx);
#pragma unroll 1
    for (int s = 0; s < a.steps; ++s) {
#pragma unroll 1
        for (int c = x0; c < x1; c += 16) {
            float v[16];
            ns_ld16(tx + mine + c, v);
            store(xh, xl, c / 8, v, 1.0f / kNsScale);
            store(xh, xl, c / 8 + 1, v + 8, 1.0f / kNsScale);
        }
        product([&] { squares(xh, xl, a.W / 16); }, [] {});
        if (a.C == 1) {
#pragma unroll 1
            for (int u = u0; u < u1; ++u) {
                float v[8];
                ns_ld8(ts + mine + 8 * u, v);
                store(sh, sl, u, v, to_a);
            }
        } else {
            ns_cluster_arrive();                            // all CTAs have read their low halves of X
            ns_cluster_wait();
            // 8 columns of a row at a time to the CTA that adds them: [part][its units][half][128 rows] of 16 bytes
            const int own = (units + a.C - 1) / a.C;        // units of a CTA
#pragma unroll 1
            for (int u = u0; u < u1; ++u) {
                float v[8];
                ns_ld8(ts + mine + 8 * u, v);
                const unsigned to = ns_peer(parts + (rank * own + u % own) * 4096 + row * 16, u / own);
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + q * 2048), "f"(v[4 * q]), "f"(v[4 * q + 1]),
                                 "f"(v[4 * q + 2]), "f"(v[4 * q + 3]) : "memory");
            }
            ns_fence_before();
            __syncwarp();
            ns_cluster_arrive();
            ns_cluster_wait();
#pragma unroll 1
            for (int k = t; k < own * 128; k += kNsSmallThreads) {
                const int r = k & 127, lu = k >> 7, u = rank * own + lu;
                if (r >= mp || u >= units) continue;
                float v[8] = {};
#pragma unroll 4
                for (int p = 0; p < a.C; ++p) {
                    const unsigned from = parts + (p * own + lu) * 4096 + r * 16;
                    const uint4 x = ns_lds(from), y = ns_lds(from + 2048);
                    const float f[8] = {__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w),
                                        __uint_as_float(y.x), __uint_as_float(y.y), __uint_as_float(y.z), __uint_as_float(y.w)};
#pragma unroll
                    for (int q = 0; q < 8; ++q) v[q] += f[q];
                }
                uint4 w[2];
                ns_split8(v, to_a, w[0], w[1]);
#pragma unroll 1
                for (int p = 0; p < a.C; ++p) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(ns_peer(unit(h ? sl : sh, r, u), p)), "r"(w[h].x),
                                     "r"(w[h].y), "r"(w[h].z), "r"(w[h].w) : "memory");
                }
            }
            ns_fence_async();
            __syncwarp();
            ns_cluster_arrive();
            ns_cluster_wait();
        }
        product([&] { squares(sh, sl, mp / 16); }, [&] {
            if (a.C > 1)                                    // X's low half, where the parts were
#pragma unroll 1
                for (int c = x0; c < x1; c += 16) {
                    float v[16];
                    ns_ld16(tx + mine + c, v);
                    uint4 h, l;
                    ns_split8(v, 1.0f / kNsScale, h, l), ns_sts(unit(xl, row, c / 8), l);
                    ns_split8(v + 8, 1.0f / kNsScale, h, l), ns_sts(unit(xl, row, c / 8 + 1), l);
                }
        });
        const float ca = a.c[3 * s] * kNsScale, cb = a.c[3 * s + 1], cc = a.c[3 * s + 2] * (1.0f / kNsScale);
#pragma unroll 1
        for (int u = u0; u < u1; ++u) {
            float v[8];
            ns_ld8(ts + mine + 8 * u, v);
            const uint4 h8 = ns_lds(unit(sh, row, u)), l8 = ns_lds(unit(sl, row, u));
            __half2 h4[4], l4[4];
            memcpy(h4, &h8, 16), memcpy(l4, &l8, 16);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 o = f2_fma(__half22float2(l4[k]), f2_splat(1.0f / kNsLow), __half22float2(h4[k]));
                const float2 f = f2_fma(f2_splat(cc), make_float2(v[2 * k], v[2 * k + 1]), f2_mul(f2_splat(cb), o));
                v[2 * k] = f.x, v[2 * k + 1] = f.y;
            }
            if (row >> 3 == u) {
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    if (row == 8 * u + q) v[q] += ca;
            }
            store(sh, sl, u, v, 1.0f);
        }
        product([&] { three(tx, sh, sl, xh, xl, mp / 16, true, ns_idesc(128, a.W, true)); }, [] {});
    }
    if (!ok) atomicAdd(a.giveups, 1u);
    const float unit_out = 1.0f / (kNsScale * a.sx);
#pragma unroll 1
    for (int c = x0; c < x1; c += 16) {
        float v[16];
        ns_ld16(tx + mine + c, v);
#pragma unroll
        for (int q = 0; q < 16; ++q) stage[row * a.W + ((c + q) ^ (row & 31))] = v[q] * unit_out;
    }
    ns_fence_before();
    __syncthreads();
    __nv_bfloat16* out = a.out + z * a.out_mat + (a.tall ? n0 * a.out_row : n0);
#pragma unroll 2
    for (int r = warp; r < rows; r += kWarps) {
        float v[kNsSmallWidth / 32];
#pragma unroll
        for (int j = 0; j < kNsSmallWidth / 32; ++j)
            if (32 * j < cols) v[j] = stage[place(r, lane + 32 * j)];
#pragma unroll
        for (int j = 0; j < kNsSmallWidth / 32; ++j)
            if (ok && r < rows_in && lane + 32 * j < cols_in && 32 * j < cols) out[r * a.out_row + lane + 32 * j] = __float2bfloat16_rn(v[j]);
    }
    if (warp == 0) {
        __syncwarp();
        ns_fence_after();
        if (tcols == 256) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 256;" ::"r"(tx));
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tx));
    }
}

// sum of squares of every matrix, in binary64 (no overflow, no order effects worth mentioning): a warp takes whole rows, eight
// elements a lane at a time where rows are 16-byte aligned; one partial per block
template <typename T>
__global__ void __launch_bounds__(256) k_ns_norm(const T* __restrict__ g, int rows, int cols, long long row, long long mat, bool vec,
                                                 double* __restrict__ part) {
    __shared__ double red[8];
    constexpr int V = 16 / sizeof(T);
    const T* m = g + blockIdx.y * mat;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, chunks = (cols + 32 * V - 1) / (32 * V);
    double s = 0;
    // a warp's unit: up to 32 * V columns of a row
    for (long long w = (long long)blockIdx.x * 8 + warp; w < (long long)rows * chunks; w += (long long)gridDim.x * 8) {
        const int r = (int)(w / chunks), c = (int)(w - (long long)r * chunks) * 32 * V;
        const T* p = m + r * row + c;
        if (vec && c + lane * V + V <= cols) {
            T t[V];
            const uint4 u = *(const uint4*)(p + lane * V);
            memcpy(t, &u, 16);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const double v = (double)to_f32(t[i]);
                s = fma(v, v, s);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int k = vec ? lane * V + i : lane + 32 * i;
                if (c + k < cols) {
                    const double v = (double)to_f32(p[k]);
                    s = fma(v, v, s);
                }
            }
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    if (lane == 0) red[warp] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0;
        for (int w = 0; w < 8; ++w) s += red[w];
        part[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
    }
}

// X = G * sx / (|G| + eps) as hi + lo, transposed if tall; 64 x 64 tiles through shared memory, pairs of neighbours written at once
template <typename T>
__global__ void __launch_bounds__(256) k_ns_prepare(const T* __restrict__ g, int rows, int cols, long long row, long long mat,
                                                    const double* __restrict__ part, int parts, float eps, float sx, int tall, __half* __restrict__ hi,
                                                    __half* __restrict__ lo, int ld, size_t xmat) {
    __shared__ float tile[64][65];
    __shared__ double factor;
    const int z = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
    pdl_trigger();
    float in[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) {          // loads first: the partial sums are added while they are on their way
        const int r = r0 + warp + 8 * (k >> 1), c = c0 + lane + 32 * (k & 1);
        in[k] = r < rows && c < cols ? to_f32(g[z * mat + (long long)r * row + c]) : 0.0f;
    }
    pdl_wait();
    if (warp == 0) {
        double s = 0;
        for (int k = lane; k < parts; k += 32) s += part[(size_t)z * parts + k];
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
        s = sqrt(s) + (double)eps;
        if (lane == 0) factor = s > 0 || s != s ? (double)sx / s : 0.0;
    }
    __syncthreads();
    const NsFactor scale(factor);
#pragma unroll
    for (int k = 0; k < 16; ++k) tile[warp + 8 * (k >> 1)][lane + 32 * (k & 1)] = scale(in[k]);
    __syncthreads();
    const int i0 = tall ? c0 : r0, j0 = tall ? r0 : c0, M = tall ? cols : rows, N = tall ? rows : cols;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int r = warp + 8 * k, j = j0 + 2 * lane;
        if (i0 + r < M && j < N) {          // the pitch is a multiple of 64: the second of a pair may lie behind the row
            const float v0 = tall ? tile[2 * lane][r] : tile[r][2 * lane], v1 = tall ? tile[2 * lane + 1][r] : tile[r][2 * lane + 1];
            const __half2 h = __floats2half2_rn(v0, v1);
            const float2 f = __half22float2(h);
            const size_t at = z * xmat + (size_t)(i0 + r) * ld + j;
            *(__half2*)(hi + at) = h;
            *(__half2*)(lo + at) = __floats2half2_rn((v0 - f.x) * 2048.0f, (v1 - f.y) * 2048.0f);
        }
    }
}

// Tiled kernels: up to this M the square matrices have low halves too.  That takes the roundings of P away, which fall on few rows
// there (16 x 8192, one direction over 1e-5: 0.12 -> 0.004 %, 3 x 9000, a level over noise 0.10 -> 0.04 %), for a tenth more time;
// 200 x 300 would go from 0.08 to 0.06 % and take a quarter more.
constexpr int kNsFine = 128;
struct NsLayout {
    int M, N, ldm, ldn, parts;
    size_t xmat, amat, part_off, x0, x1, l0, l1, a_off, b_off, al, bl, da, db, bytes;
    bool fine;              // A and B have low halves too
};
static NsLayout ns_layout(size_t batch, size_t rows, size_t cols) {
    NsLayout L;
    L.M = (int)(rows < cols ? rows : cols);
    L.N = (int)(rows < cols ? cols : rows);
    L.ldm = (L.M + 63) / 64 * 64;
    L.ldn = (L.N + 63) / 64 * 64;
    const size_t want = ((size_t)L.M * L.N + 16383) / 16384;
    L.parts = (int)(want < 1 ? 1 : want > kNsMaxParts ? kNsMaxParts : want);
    L.xmat = (size_t)L.M * L.ldn;
    L.amat = (size_t)L.M * L.ldm;
    auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
    L.part_off = 0;
    L.x0 = up(batch * L.parts * sizeof(double));
    L.x1 = L.x0 + up(batch * L.xmat * 2);
    L.l0 = L.x1 + up(batch * L.xmat * 2);
    L.l1 = L.l0 + up(batch * L.xmat * 2);
    L.a_off = L.l1 + up(batch * L.xmat * 2);
    L.b_off = L.a_off + up(batch * L.amat * 2);
    L.fine = L.M <= kNsFine;
    L.al = L.b_off + up(batch * L.amat * 2);
    L.bl = L.al + (L.fine ? up(batch * L.amat * 2) : 0);
    L.da = L.bl + (L.fine ? up(batch * L.amat * 2) : 0);
    L.db = L.da + up(batch * (size_t)L.ldm * 4);
    L.bytes = L.db + up(batch * (size_t)L.ldm * 4);
    return L;
}

static bool ns_map(CUtensorMap* out, void* base, int inner, int rows, size_t batch, int ld, size_t mat, int box_rows) {
    const cuuint64_t dim[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)batch};
    const cuuint64_t stride[2] = {(cuuint64_t)ld * 2, (cuuint64_t)mat * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
    return tma_encode_half(out, 3, base, dim, stride, box);
}

// Which kernel: 256 x 256 tiles by CTA pairs if there are more of them than half the pairs (below that, 128 x 128 tiles fill more
// SMs), else 128 x 128 tiles.  Their sums over K are split in 2 or 4 as long as all clusters of 4 run at once (an SM takes one CTA,
// and 32 clusters fit whichever SMs of a GPC are left) and every part keeps eight blocks of K.  Measured, all steps: up to 148 CTAs
// instead of 128 4096 x 1024 210 us against 182, up to 74 1024 x 1024 126 us against 123; parts of four blocks instead of eight
// 1024 x 1024 210 us against 142; one part alone 512 x 2048 154 us against 132 (the last two with slower epilogues).
constexpr int kNsSplitMax = 128;
template <int MODE, bool FINE = false>
static bool ns_product(const NsMaps& maps, NsArgs a, int batch, cudaStream_t st) {
    constexpr bool kSym = MODE == NS_GRAM || MODE == NS_POLY;
    auto count = [&](int t) {
        const long long m = (a.M + t - 1) / t, n = (a.N + t - 1) / t;
        return batch * (kSym ? m * (m + 1) / 2 : m * n);
    };
    const long long big = count(256), small = count(128);
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr, cfg.numAttrs = 1, cfg.stream = st, cfg.blockDim = dim3(kNsThreads);
    static std::atomic<uint64_t> done[2];
    constexpr int smem = ns_smem(kNsMaxStages);
    cfg.dynamicSmemBytes = smem;
    cudaError_t e;
    if (big > kSMs / 4) {
        a.tiles_m = (a.M + 255) / 256, a.tiles_n = (a.N + 255) / 256, a.tiles = (int)big;
        cfg.gridDim = dim3((unsigned)(2 * (big < kSMs / 2 ? big : kSMs / 2)));
        if (!allow_big_smem_once(k_ns_pair<MODE, FINE>, smem, done[0])) return false;
        e = cudaLaunchKernelEx(&cfg, k_ns_pair<MODE, FINE>, maps, a);
    } else {
        int split = 1;
        while (split < 4 && small * split * 2 <= kNsSplitMax && a.K / kNsK >= split * 16) split *= 2;
        cfg.gridDim = dim3((a.N + kNsTile - 1) / kNsTile * split, (a.M + kNsTile - 1) / kNsTile, batch);
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim = {(unsigned)split, 1, 1};
        cfg.numAttrs = 2;
        if (!allow_big_smem_once(k_ns_tile<MODE, FINE>, smem, done[1])) return false;
        e = cudaLaunchKernelEx(&cfg, k_ns_tile<MODE, FINE>, maps, a, split);
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess;
}

template <typename T>
static void ns_start(const void* g, size_t batch, size_t rows, size_t cols, size_t row, size_t mat, float eps, float sx, const NsLayout& L,
                     unsigned char* ws, cudaStream_t st) {
    double* part = (double*)(ws + L.part_off);
    const bool vec = !misaligned(g, 16) && row * sizeof(T) % 16 == 0 && (batch == 1 || mat * sizeof(T) % 16 == 0);
    TRV_LAUNCH(k_ns_norm<T>, dim3(L.parts, (unsigned)batch), 256, 0, st, (const T*)g, (int)rows, (int)cols, (long long)row, (long long)mat, vec, part);
    launch_pdl(k_ns_prepare<T>, dim3((unsigned)(cols + 63) / 64, (unsigned)(rows + 63) / 64, (unsigned)batch), dim3(256), 0, st, (const T*)g,
               (int)rows, (int)cols, (long long)row, (long long)mat, (const double*)part, L.parts, eps, sx, (int)(rows > cols), (__half*)(ws + L.x0),
               (__half*)(ws + L.l0), L.ldn, L.xmat);
}

// Matrices that k_ns_small takes: M <= 128 and columns for at most a cluster of 16
static bool ns_is_small(const NsLayout& L) { return L.M <= 128 && L.N <= kNsSmallCluster * kNsSmallWidth; }
template <typename T>
static bool ns_small(NsSmall a, size_t batch, cudaStream_t st) {
    a.C = 1;
    while (a.C * kNsSmallWidth < a.N) a.C *= 2;
    a.W = ((a.N + a.C - 1) / a.C + 63) / 64 * 64;
    const int smem = 1024 + a.W * 256 + ns_small_low(a.W, a.C) + 2 * ns_small_square(a.M);
    static std::atomic<uint64_t> done;
    if (!allow_big_smem_once(k_ns_small<T>, 1024 + kNsSmallWidth * 256 + 65536 + 2 * 32768, done)) return false;
    if (a.C > 8 && cudaFuncSetAttribute(k_ns_small<T>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return false;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)a.C, 1, 1};
    cfg.attrs = attr, cfg.numAttrs = 1, cfg.stream = st, cfg.blockDim = dim3(kNsSmallThreads), cfg.gridDim = dim3((unsigned)(batch * a.C));
    cfg.dynamicSmemBytes = smem;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k_ns_small<T>, a);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess;
}

constexpr size_t kNsMaxSide = (size_t)1 << 20, kNsMaxBatch = 65535;
constexpr float kNsDefault[3] = {3.4445f, -4.7750f, 2.0315f};
constexpr int kNsMaxSteps = 64;
// Tiled kernels: in which steps P is multiplied with X's low half too.  What it rounds off a strong direction falls, through P's
// part outside the diagonal, on all the others, 2^-12 / M times about 10 of the strong one, and grows with them in later steps:
// with X's high half alone one strong direction over weak ones ended 2.9 % off at 16 rows, 0.3 % at 129, 0.08 % at 512, 0.04 % at
// 2048.  A step's share is kept below 1e-4, where it drowns in the other roundings: low half if 24 times the growth still to
// come exceeds M.  Default coefficients: three steps of five at M = 200, the first at 1024, none from 3379 on.
constexpr double kNsLowFrom = 24;

}  // namespace trv

using namespace trv;

extern "C" trv_status_t trv_orthogonalize_workspace_bytes(size_t batch, size_t rows, size_t cols, size_t* bytes) {
    if (!bytes) return TRV_ERR_INVALID_ARG;
    *bytes = 0;
    if (rows > kNsMaxSide || cols > kNsMaxSide || batch > kNsMaxBatch) return TRV_ERR_UNSUPPORTED;
    if (batch && rows && cols) {
        const NsLayout L = ns_layout(batch, rows, cols);
        *bytes = ns_is_small(L) ? 0 : L.bytes;
    }
    return TRV_OK;
}

extern "C" trv_status_t trv_orthogonalize(const void* g, void* out, size_t batch, size_t rows, size_t cols, size_t g_stride, size_t g_batch_stride,
                                          size_t out_stride, size_t out_batch_stride, int32_t steps, const float* coefficients, float eps,
                                          trv_dtype_t dtype, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!float_dtype(dtype) || steps < 1 || steps > kNsMaxSteps || !(eps >= 0)) return TRV_ERR_INVALID_ARG;
    if (rows > kNsMaxSide || cols > kNsMaxSide || batch > kNsMaxBatch) return TRV_ERR_UNSUPPORTED;
    const size_t most = (size_t)1 << 40;
    if (g_stride < cols || out_stride < cols || g_stride > most || out_stride > most || g_batch_stride > most || out_batch_stride > most)
        return TRV_ERR_INVALID_ARG;
    if (!batch || !rows || !cols) return TRV_OK;
    const size_t es = dtype_bytes(dtype);
    if (!g || !out || misaligned(g, es) || misaligned(out, 2)) return TRV_ERR_INVALID_ARG;
    // the matrices of the result must not overlap one another
    if (batch > 1 && out_batch_stride < (rows - 1) * out_stride + cols) return TRV_ERR_INVALID_ARG;
    const NsLayout L = ns_layout(batch, rows, cols);
    const size_t need = ns_is_small(L) ? 0 : L.bytes;
    if (need && (!workspace || misaligned(workspace, 256) || workspace_bytes < need)) return TRV_ERR_SCRATCH;
    // a batch of matrices is one matrix of their rows if the distance between them is a whole number of rows
    auto span = [&](const void* p, size_t stride, size_t batch_stride, size_t size) {
        const bool whole = batch == 1 || batch_stride % stride == 0;
        return Span{p, ((batch - 1) * batch_stride + (rows - 1) * stride + cols) * size, cols * size, whole ? stride * size : 0};
    };
    const Span in[1] = {span(g, g_stride, g_batch_stride, es)};
    const Span outs[2] = {span(out, out_stride, out_batch_stride, 2), {workspace, need}};
    if (!disjoint(in, outs)) return TRV_ERR_INVALID_ARG;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    unsigned char* ws = (unsigned char*)workspace;
    __half* X[2] = {(__half*)(ws + L.x0), (__half*)(ws + L.x1)};
    __half* lo[2] = {(__half*)(ws + L.l0), (__half*)(ws + L.l1)};
    __half *A = (__half*)(ws + L.a_off), *B = (__half*)(ws + L.b_off);
    float *DA = (float*)(ws + L.da), *DB = (float*)(ws + L.db);
    int e = 0;                                              // sx = 2^e, nearest to sqrt(N)
    while (((size_t)2 << (2 * e)) <= (size_t)L.N) ++e;
    const float sx = (float)(1 << e);
    unsigned* giveups = tma_giveup_counter();
    if (!giveups) return TRV_ERR_CUDA;
    bool ok = true;
    if (ns_is_small(L)) {
        NsSmall k = {g, (__nv_bfloat16*)out, (long long)g_stride, (long long)g_batch_stride, (long long)out_stride, (long long)out_batch_stride,
                     L.M, L.N, 0, 0, steps, rows > cols, sx, eps, giveups, {}};
        for (int i = 0; i < 3 * steps; ++i) k.c[i] = coefficients ? coefficients[i] : kNsDefault[i % 3];
        ok = dtype == TRV_FLOAT32 ? ns_small<float>(k, batch, st) : dtype == TRV_BFLOAT16 ? ns_small<__nv_bfloat16>(k, batch, st) : ns_small<__half>(k, batch, st);
        g_last_kernel = "orthogonalize_small";
        return ok && cudaGetLastError() == cudaSuccess ? TRV_OK : TRV_ERR_CUDA;
    }
    CUtensorMap xk[2], xn[2], ln[2], ak, bk, akl = {}, bkl = {};
    __half *al = L.fine ? (__half*)(ws + L.al) : nullptr, *bl = L.fine ? (__half*)(ws + L.bl) : nullptr;
    for (int p = 0; p < 2 && ok; ++p)
        ok = ns_map(&xk[p], X[p], L.N, L.M, batch, L.ldn, L.xmat, kNsTile) && ns_map(&xn[p], X[p], L.N, L.M, batch, L.ldn, L.xmat, kNsK) &&
             ns_map(&ln[p], lo[p], L.N, L.M, batch, L.ldn, L.xmat, kNsK);
    ok = ok && ns_map(&ak, A, L.M, L.M, batch, L.ldm, L.amat, kNsTile) && ns_map(&bk, B, L.M, L.M, batch, L.ldm, L.amat, kNsTile);
    if (L.fine) ok = ok && ns_map(&akl, al, L.M, L.M, batch, L.ldm, L.amat, kNsTile) && ns_map(&bkl, bl, L.M, L.M, batch, L.ldm, L.amat, kNsTile);
    if (!ok) return TRV_ERR_CUDA;
    if (dtype == TRV_FLOAT32) ns_start<float>(g, batch, rows, cols, g_stride, g_batch_stride, eps, sx, L, ws, st);
    else if (dtype == TRV_BFLOAT16) ns_start<__nv_bfloat16>(g, batch, rows, cols, g_stride, g_batch_stride, eps, sx, L, ws, st);
    else ns_start<__half>(g, batch, rows, cols, g_stride, g_batch_stride, eps, sx, L, ws, st);
    const bool tall = rows > cols;
    for (int s = 0; s < steps && ok; ++s) {
        auto step = [&](int t) { return coefficients ? coefficients + 3 * t : kNsDefault; };
        const float* c = step(s);
        const int p = s & 1;
        double grows = 1;                                   // by this factor in the later steps, if weak enough
        for (int t = s + 1; t < steps; ++t) grows *= fabs((double)step(t)[0]);
        NsArgs k = {};
        k.Md = L.ldm, k.a = c[0], k.b = c[1], k.giveups = giveups;
        NsArgs gram = k, poly = k, apply = k;
        gram.M = gram.N = poly.M = poly.N = poly.K = apply.M = apply.K = L.M;
        gram.K = apply.N = L.N;
        gram.ld = poly.ld = L.ldm, gram.mat = poly.mat = L.amat, apply.ld = L.ldn, apply.mat = L.xmat;
        gram.alpha = kNsScale / (sx * sx), gram.out = A, gram.out_lo = al, gram.diag_out = DA;
        poly.alpha = c[2] / kNsScale, poly.hi = A, poly.diag = DA, poly.out = B, poly.diag_out = DB;
        poly.lo = al, poly.out_lo = bl, poly.low = L.fine ? 3 : 0;
        const bool last = s + 1 == steps;
        apply.unit = last ? 1.0f / sx : 1.0f, apply.alpha = apply.unit / kNsScale, apply.hi = X[p], apply.lo = lo[p], apply.diag = DB;
        apply.low = (kNsLowFrom * grows > L.M ? 1 : 0) | (L.fine ? 2 : 0);
        apply.out = X[1 - p], apply.out_lo = lo[1 - p], apply.last = (__nv_bfloat16*)out;
        apply.last_row = (long long)(tall ? 1 : out_stride), apply.last_col = (long long)(tall ? out_stride : 1);
        apply.last_mat = (long long)out_batch_stride;
        apply.last_vec = !misaligned(out, 16) && out_stride % 8 == 0 && (batch == 1 || out_batch_stride % 8 == 0);
        const NsMaps xx = {xk[p], xk[p], xk[p], xk[p]}, aa = {ak, ak, akl, akl}, bx = {bk, xn[p], bkl, ln[p]};
        ok = (L.fine ? ns_product<NS_GRAM, true>(xx, gram, (int)batch, st) && ns_product<NS_POLY, true>(aa, poly, (int)batch, st)
                     : ns_product<NS_GRAM>(xx, gram, (int)batch, st) && ns_product<NS_POLY>(aa, poly, (int)batch, st)) &&
             (last ? ns_product<NS_LAST>(bx, apply, (int)batch, st) : ns_product<NS_APPLY>(bx, apply, (int)batch, st));
    }
    g_last_kernel = "orthogonalize";
    return ok && cudaGetLastError() == cudaSuccess ? TRV_OK : TRV_ERR_CUDA;
}
