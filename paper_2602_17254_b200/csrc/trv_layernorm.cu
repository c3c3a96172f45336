// Layer norm, forward and backward.  Row x of C values: mu = sum x / C, v = sum (x - mu)^2 / C, r = 1 / sqrt(v + eps),
// h = (x - mu) r, y = h gamma + beta.  Backward, with g = dy gamma:  dx = r (g - mean(g) - h mean(g h)),
// dgamma = sum over rows of dy h, dbeta = sum over rows of dy.
//
// Every matrix is read or written once: a row lives in registers between its one read and its one write (the variance is of the
// differences from the mean, a second pass over registers).  CTAs are persistent, so that gamma and beta (and, backward, the sums
// of the parameters' gradients) stay in registers, and each keeps its next rows on their way into shared memory by asynchronous
// copies while it reduces the present one.  Short rows take a warp each, longer ones a CTA or a part of one, the longest of the
// backward pass a cluster of two CTAs.
//
// Bound by memory; behind it by the chain of a row's sums and by issue slots (half busy on 16-bit rows: unpacking, three passes over
// the row, packing; hence the packed binary32 arithmetic, and forward as many elements a thread as registers allow, since a row's
// sums cost every thread the same; backward the parameters' gradients take the registers).  Measured:
// forward 16384 x 4096 bfloat16 45 us, 6.0 TB/s, 32768 x 8192 168 us, 6.4 TB/s; backward 32768 x 8192 bfloat16 288 us, 5.6 TB/s;
// 6561 x 2187 float32, rows that start off 16-byte boundaries, forward 24.5 us, 4.7 TB/s, backward 37 us, 4.6 TB/s.  Further from
// memory's rate: short rows (65536 x 512 bfloat16 backward 43 us, 200000 x 100 float32 33 us forward, 52 backward: 80 - 127 registers,
// 2 to 3 CTAs of a warp per row); rows off 16-byte boundaries (122 - 146 registers, 1 or 2 CTAs per SM); pairs of CTAs (8192 x 16384
// bfloat16 backward 220 us: a cluster barrier per row with nothing to do meanwhile).  Operands that start at different places of a
// 16-byte vector are read element by element, nothing ahead; so are rows above 16384 columns, in three passes.  Spills: pairs with loose
// ends 32 (16-bit) and 64 bytes (float32), forward float32 rows above 8192 columns with loose ends 60.
#include <atomic>

#include "trv_train.cuh"

namespace trv {

constexpr int kLnThreads = 256;
constexpr int kLnMaxThreads = 512;          // of a CTA that holds a row: leaves 128 registers a thread
constexpr int kLnMaxParts = 4 * kSMs;       // most CTAs, so most partial sums of dgamma and dbeta

// VEC elements of a row as loaded: 16 bytes, or one element where the matrices' rows have no common 16-byte alignment
template <typename T, int VEC> struct LnRaw { uint4 u; };
template <typename T> struct LnRaw<T, 1> { T u; };

__device__ __forceinline__ void ln_unpack(const LnRaw<float, 4>& r, float* f) {
    f[0] = __uint_as_float(r.u.x), f[1] = __uint_as_float(r.u.y), f[2] = __uint_as_float(r.u.z), f[3] = __uint_as_float(r.u.w);
}
__device__ __forceinline__ void ln_unpack(const LnRaw<__nv_bfloat16, 8>& r, float* f) {
    const unsigned u[4] = {r.u.x, r.u.y, r.u.z, r.u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(u[i] << 16), f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
}
__device__ __forceinline__ void ln_unpack(const LnRaw<__half, 8>& r, float* f) {
    const unsigned u[4] = {r.u.x, r.u.y, r.u.z, r.u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __half2 h;
        memcpy(&h, &u[i], 4);
        const float2 p = __half22float2(h);
        f[2 * i] = p.x, f[2 * i + 1] = p.y;
    }
}
template <typename T> __device__ __forceinline__ void ln_unpack(const LnRaw<T, 1>& r, float* f) { f[0] = to_f32(r.u); }

__device__ __forceinline__ void ln_pack(const float* f, LnRaw<float, 4>* r) {
    r->u = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
__device__ __forceinline__ unsigned ln_pair(float a, float b, __nv_bfloat16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    unsigned u;
    memcpy(&u, &h, 4);
    return u;
}
__device__ __forceinline__ unsigned ln_pair(float a, float b, __half) {
    const __half2 h = __floats2half2_rn(a, b);
    unsigned u;
    memcpy(&u, &h, 4);
    return u;
}
template <typename T>
__device__ __forceinline__ void ln_pack(const float* f, LnRaw<T, 8>* r) {
    r->u = make_uint4(ln_pair(f[0], f[1], T()), ln_pair(f[2], f[3], T()), ln_pair(f[4], f[5], T()), ln_pair(f[6], f[7], T()));
}
template <typename T> __device__ __forceinline__ void ln_pack(const float* f, LnRaw<T, 1>* r) { r->u = from_f32<T>(f[0]); }

__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// one parameter; NULL gives `none`
template <typename T>
__device__ __forceinline__ float ln_param(const void* p, bool p32, int c, float none) {
    return !p ? none : p32 ? ((const float*)p)[c] : to_f32(((const T*)p)[c]);
}

// How the threads t of a group of G share a row: NV vectors each, t, t + G, ... of the `nvec` whole 16-byte vectors that start at
// column `head`; with EDGE (rows that start or end inside a vector) threads t < `edges` also take one of the elements before or
// behind them.  All rows of a thread have the same alignment (the row step of a grid is a multiple of 8 rows, so of 16
// bytes), so its columns are the same in every row.
template <typename T, int VEC, int NV, bool EDGE, int AHEAD>
struct LnRow {
    static constexpr int P = VEC * NV / 2;      // elements in pairs, for the packed arithmetic
    static constexpr int VP = VEC > 1 ? VEC / 2 : 1, NP = P / VP;       // pairs that are valid together, and how many such groups
    static constexpr int D = VEC == 1 ? 1 : AHEAD + 1;      // rows in shared memory: the present one and those on their way
    struct Raw {
        LnRaw<T, VEC> v[NV];
        T e;
    };
    int t, G, head, nvec, edges, edge;
    __device__ __forceinline__ LnRow(int t_, int G_, const T* row, int cols) : t(t_), G(G_), head(0), nvec(cols / VEC), edges(0), edge(0) {
        if (EDGE) {
            head = (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T);
            if (head > cols) head = cols;
            nvec = (cols - head) / VEC;
            edges = cols - nvec * VEC;
            edge = t < head ? t : nvec * VEC + t;
        }
    }
    // column of element i < 2 P, valid only where has(i)
    __device__ __forceinline__ int col(int i) const { return head + (t + i / VEC * G) * VEC + i % VEC; }
    __device__ __forceinline__ bool has(int i) const { return t + i / VEC * G < nvec; }
    __device__ __forceinline__ bool has_edge() const { return EDGE && t < edges; }
    // Shared-memory slots of this thread, [D][NV] of 16 bytes, `stride` bytes apart: filled by asynchronous copies, read by the same
    // thread alone, so no barrier is involved.  VEC == 1: no slots, rows are loaded when they are needed.
    __device__ __forceinline__ void clear(unsigned slots, unsigned stride) const {
        if (VEC > 1)
            for (int i = 0; i < D * NV; ++i) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(slots + i * stride), "r"(0) : "memory");
    }
    __device__ __forceinline__ void fetch(const T* row, unsigned slots, unsigned stride, int d) const {
        if (VEC > 1) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (t + v * G < nvec)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(slots + (d * NV + v) * stride),
                                 "l"(row + head + (size_t)(t + v * G) * VEC) : "memory");
        }
    }
    __device__ __forceinline__ T fetch_edge(const T* row) const { return has_edge() ? row[edge] : from_f32<T>(0.0f); }
    __device__ __forceinline__ void take(const T* row, unsigned slots, unsigned stride, int d, Raw& r) const {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (VEC > 1) {
                uint4& u = r.v[v].u;
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "r"(slots + (d * NV + v) * stride) : "memory");
            } else {
                r.v[v].u = from_f32<T>(0.0f);
                if (t + v * G < nvec) r.v[v].u = row[head + (size_t)(t + v * G)];
            }
        }
    }
    __device__ __forceinline__ static void unpack(const Raw& r, float2 (&f)[P], float& e) {
        float g[2 * P];
#pragma unroll
        for (int v = 0; v < NV; ++v) ln_unpack(r.v[v], g + v * VEC);
#pragma unroll
        for (int i = 0; i < P; ++i) f[i] = make_float2(g[2 * i], g[2 * i + 1]);
        e = EDGE ? to_f32(r.e) : 0.0f;
    }
    __device__ __forceinline__ void store(T* row, const float2 (&f)[P], float e) const {
        float g[2 * P];
#pragma unroll
        for (int i = 0; i < P; ++i) g[2 * i] = f[i].x, g[2 * i + 1] = f[i].y;
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (t + v * G < nvec) {
                LnRaw<T, VEC> r;
                ln_pack(g + v * VEC, &r);
                *(decltype(r.u)*)(row + head + (size_t)(t + v * G) * VEC) = r.u;
            }
        if (has_edge()) row[edge] = from_f32<T>(e);
    }
    // a parameter of every element (the row starts at parameter c0), 0 outside the row; one by one they were half of a small call
    // (17 x 1000 bfloat16 5.3 us, now 2.3) and 4 us of 16384 x 4096
    __device__ __forceinline__ void params(const void* p, bool p32, int c0, float none, float2 (&f)[P], float& e) const {
        if constexpr (!EDGE && VEC > 1) if (p && !((uintptr_t)p & 15)) {            // 16 bytes at a time (c0 is a multiple of VEC)
            float g[2 * P];
            e = 0;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float* to = g + v * VEC;
#pragma unroll
                for (int i = 0; i < VEC; ++i) to[i] = 0;
                const int c = c0 + (t + v * G) * VEC;
                if (t + v * G >= nvec) continue;
                if (p32) {
#pragma unroll
                    for (int i = 0; i < VEC; i += 4) {
                        const float4 u = *(const float4*)((const float*)p + c + i);
                        to[i] = u.x, to[i + 1] = u.y, to[i + 2] = u.z, to[i + 3] = u.w;
                    }
                } else {
                    LnRaw<T, VEC> r;
                    r.u = *(const decltype(r.u)*)((const T*)p + c);
                    ln_unpack(r, to);
                }
            }
#pragma unroll
            for (int i = 0; i < P; ++i) f[i] = make_float2(g[2 * i], g[2 * i + 1]);
            return;
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            f[i].x = has(2 * i) ? ln_param<T>(p, p32, c0 + col(2 * i), none) : 0.0f;
            f[i].y = has(2 * i + 1) ? ln_param<T>(p, p32, c0 + col(2 * i + 1), none) : 0.0f;
        }
        e = has_edge() ? ln_param<T>(p, p32, c0 + edge, none) : 0.0f;
    }
};

// Sum over the threads that share a row: the warp, or the CTA through shared memory (cleared before).  Consecutive calls alternate
// between two buffers, so one barrier per call is enough.  Behind it every thread adds up to 8 warps' sums itself (6561 x 2187
// float32 24.6 us, with shuffles 30); MANY: more of them by shuffles (8192 x 16384 bfloat16 95 us, without 101).  A loop, although
// it turns once: as straight code the rows off 16-byte boundaries spill (6561 x 2187 31 us).
template <bool WARP, bool MANY>
__device__ __forceinline__ float ln_row_sum(float v, float* red) {
    v = warp_sum(v);
    if (WARP) return v;
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    if (MANY) return warp_sum(red[threadIdx.x & 31]);
    float2 s = make_float2(0, 0);
    for (int i = 0; i < (int)blockDim.x >> 5; i += 8) {
        const float4 u = *(const float4*)(red + i), w = *(const float4*)(red + i + 4);
        s = f2_add(s, f2_add(f2_add(make_float2(u.x, u.y), make_float2(u.z, u.w)), f2_add(make_float2(w.x, w.y), make_float2(w.z, w.w))));
    }
    return s.x + s.y;
}
__device__ __forceinline__ void ln_clear(float* red, int n) {
    for (int i = threadIdx.x; i < n; i += blockDim.x) red[i] = 0;
    __syncthreads();
}
// 1 / sqrt(v) to 1 ulp: an approximation and a Newton step; for v = 0, infinite or NaN the approximation itself
__device__ __forceinline__ float ln_rsqrt(float v) {
    const float r = rsqrtf(v), e = fmaf(-v * r, r, 1.0f);
    return fabsf(e) < 1.0f ? fmaf(0.5f * r, e, r) : r;
}

template <typename T>
struct LnFwd {
    const T* x;
    const void *gamma, *beta;
    T* y;
    float *mean, *rstd;
    long long rows, xs, ys;
    int cols;
    bool p32;
    float eps;
};

template <typename T, int VEC, int NV, bool EDGE, bool WARP, int AHEAD, bool MANY = false>
__global__ void __launch_bounds__(WARP ? kLnThreads : kLnMaxThreads) k_ln_fwd(const LnFwd<T> a) {
    using Row = LnRow<T, VEC, NV, EDGE, AHEAD>;
    constexpr int P = Row::P;
    __shared__ __align__(16) float red[2][32];
    const int per = WARP ? blockDim.x >> 5 : 1;
    const long long step = (long long)gridDim.x * per;
    long long r = (long long)blockIdx.x * per + (WARP ? threadIdx.x >> 5 : 0);
    if (r >= a.rows) return;
    const Row k(WARP ? threadIdx.x & 31 : threadIdx.x, WARP ? 32 : blockDim.x, a.x + r * a.xs, a.cols);
    extern __shared__ __align__(16) unsigned char ring[];
    const unsigned stride = blockDim.x * 16, slots = (unsigned)__cvta_generic_to_shared(ring) + threadIdx.x * 16;
    k.clear(slots, stride);
    if (!WARP) ln_clear(red[0], 64);
    for (int d = 0; d < Row::D - 1; ++d) {
        if (r + d * step < a.rows) k.fetch(a.x + (r + d * step) * a.xs, slots, stride, d);
        cp_commit();
    }
    T edge = k.fetch_edge(a.x + r * a.xs);
    float2 gm[P], bt[P];
    float gme, bte;
    k.params(a.gamma, a.p32, 0, 1.0f, gm, gme);
    k.params(a.beta, a.p32, 0, 0.0f, bt, bte);
    const float inv = 1.0f / a.cols;
    for (int d = 0; r < a.rows; r += step, d = (d + 1) % Row::D) {
        float2 x[P], s2 = make_float2(0, 0);
        float xe;
        const long long ahead = r + (Row::D - 1) * step;
        if (ahead < a.rows) k.fetch(a.x + ahead * a.xs, slots, stride, (d + Row::D - 1) % Row::D);
        cp_commit();
        cp_wait<Row::D - 1>();
        typename Row::Raw raw;
        k.take(a.x + r * a.xs, slots, stride, d, raw);
        raw.e = edge;
        if (r + step < a.rows) edge = k.fetch_edge(a.x + (r + step) * a.xs);
        Row::unpack(raw, x, xe);
#pragma unroll
        for (int i = 0; i < P; ++i) s2 = f2_add(s2, x[i]);
        const float mu = ln_row_sum<WARP, MANY>(s2.x + s2.y + xe, red[0]) * inv;
        float s = 0;
#pragma unroll
        for (int v = 0; v < Row::NP; ++v) {
            s2 = make_float2(0, 0);
#pragma unroll
            for (int i = v * Row::VP; i < (v + 1) * Row::VP; ++i) {
                x[i] = f2_add(x[i], f2_splat(-mu));
                s2 = f2_fma(x[i], x[i], s2);
            }
            s += VEC > 1 ? (k.has(2 * Row::VP * v) ? s2.x + s2.y : 0.0f) : (k.has(2 * v) ? s2.x : 0.0f) + (k.has(2 * v + 1) ? s2.y : 0.0f);
        }
        xe -= mu;
        if (k.has_edge()) s = fmaf(xe, xe, s);
        const float rs = ln_rsqrt(ln_row_sum<WARP, MANY>(s, red[1]) * inv + a.eps);
        if (k.t == 0) {
            if (a.mean) a.mean[r] = mu;
            if (a.rstd) a.rstd[r] = rs;
        }
#pragma unroll
        for (int i = 0; i < P; ++i) x[i] = f2_fma(f2_mul(x[i], f2_splat(rs)), gm[i], bt[i]);
        k.store(a.y + r * a.ys, x, fmaf(xe * rs, gme, bte));
    }
}

// Rows beyond what a CTA's registers hold: three passes over the row, the later two from L2
template <typename T>
__global__ void __launch_bounds__(1024) k_ln_fwd_long(const LnFwd<T> a) {
    __shared__ __align__(16) float red[2][32];
    ln_clear(red[0], 64);
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = a.x + r * a.xs;
        float s = 0;
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) s += to_f32(x[c]);
        const float mu = ln_row_sum<false, true>(s, red[0]) / a.cols;
        s = 0;
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
            const float d = to_f32(x[c]) - mu;
            s = fmaf(d, d, s);
        }
        const float rs = 1.0f / sqrtf(ln_row_sum<false, true>(s, red[1]) / a.cols + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[r] = mu;
            if (a.rstd) a.rstd[r] = rs;
        }
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x)
            a.y[r * a.ys + c] = from_f32<T>(fmaf((to_f32(x[c]) - mu) * rs, ln_param<T>(a.gamma, a.p32, c, 1.0f), ln_param<T>(a.beta, a.p32, c, 0.0f)));
    }
}

template <typename T>
struct LnBwd {
    const T *dy, *x;
    const void* gamma;
    const float *mean, *rstd;
    T* dx;
    float* part;            // [CTA][2][cols], NULL if no parameter's gradient is wanted
    long long rows, dys, xs, dxs;
    int cols;
    bool p32;
    int group;              // LN_GROUP: threads that share a row
    int cols0;              // LN_PAIR: columns of the first CTA
};

// Who shares a row in the backward pass: a warp; a group of a.group threads, one or several to a CTA; the CTAs of a cluster of two,
// each a half of the columns (rows too long for one CTA's registers), which exchange their warps' sums through distributed
// shared memory: one cluster barrier per row in the place of the CTA's.
template <typename T> constexpr int kLnBwdAhead = sizeof(T) == 4 ? 1 : 3;       // rows on their way: 32 bytes a thread and row
enum LnShare { LN_WARP, LN_GROUP, LN_PAIR };

template <typename T, int VEC, int NV, bool EDGE, LnShare SHARE>
__global__ void __launch_bounds__(SHARE == LN_WARP ? kLnThreads : kLnMaxThreads) k_ln_bwd(const LnBwd<T> a) {
    using Row = LnRow<T, VEC, NV, EDGE, kLnBwdAhead<T>>;
    constexpr int P = Row::P;
    constexpr bool WARP = SHARE == LN_WARP, PAIR = SHARE == LN_PAIR;
    // the row sums' [groups][2][2][32], the groups' sums over rows [groups][2][cols] if there are several, rows on their way
    extern __shared__ __align__(16) float sums[];
    const int lane = threadIdx.x & 31, G = WARP ? 32 : PAIR ? blockDim.x : a.group, per = blockDim.x / G, group = threadIdx.x / G;
    unsigned rank = 0;
    if (PAIR) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int c0 = PAIR && rank ? a.cols0 : 0, ccols = PAIR ? (rank ? a.cols - a.cols0 : a.cols0) : a.cols;     // this CTA's columns
    const int block = PAIR ? blockIdx.x / 2 : blockIdx.x;
    const long long step = (long long)(PAIR ? gridDim.x / 2 : gridDim.x) * per;
    long long r = (long long)block * per + group;
    const T *x = a.x + c0, *dy = a.dy + c0;
    const Row k(threadIdx.x % G, G, x + r * a.xs, ccols);
    float* red = sums + 128 * group;
    float* combine = sums + (WARP ? 0 : 128 * per);
    const unsigned stride = blockDim.x * 16;
    const unsigned slots = (unsigned)__cvta_generic_to_shared(combine) + (per > 1 ? per * 8 * ((a.cols + 1) & ~1) : 0) + threadIdx.x * 16;
    const unsigned slots_dy = slots + Row::D * NV * stride;
    if (PAIR) {                                             // both CTAs run before either writes to the other
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    k.clear(slots, stride);
    k.clear(slots_dy, stride);
    for (int d = 0; d < Row::D - 1; ++d) {
        const long long q = r + d * step;
        if (q < a.rows) {
            k.fetch(x + q * a.xs, slots, stride, d);
            k.fetch(dy + q * a.dys, slots_dy, stride, d);
        }
        cp_commit();
    }
    T ex = from_f32<T>(0.0f), ed = ex;
    float nmu = 0, nrs = 0;
    auto small = [&](long long q) {
        if (q >= a.rows) return;
        ex = k.fetch_edge(x + q * a.xs);
        ed = k.fetch_edge(dy + q * a.dys);
        nmu = a.mean[q], nrs = a.rstd[q];
    };
    small(r);
    float2 gm[P], dg[P], db[P];
    float gme, dge = 0, dbe = 0;
    k.params(a.gamma, a.p32, c0, 1.0f, gm, gme);
#pragma unroll
    for (int i = 0; i < P; ++i) dg[i] = db[i] = make_float2(0, 0);
    const float inv = 1.0f / a.cols;
    int flip = 0;
    for (int slot = 0; r < a.rows; r += step, slot = (slot + 1) % Row::D) {
        float2 h[P], d[P], t0 = make_float2(0, 0), t1 = make_float2(0, 0);
        float he, de;
        const float mu = nmu, rs = nrs;
        const long long ahead = r + (Row::D - 1) * step;
        if (ahead < a.rows) {
            k.fetch(x + ahead * a.xs, slots, stride, (slot + Row::D - 1) % Row::D);
            k.fetch(dy + ahead * a.dys, slots_dy, stride, (slot + Row::D - 1) % Row::D);
        }
        cp_commit();
        cp_wait<Row::D - 1>();
        typename Row::Raw raw;
        k.take(x + r * a.xs, slots, stride, slot, raw);
        raw.e = ex;
        Row::unpack(raw, h, he);
        k.take(dy + r * a.dys, slots_dy, stride, slot, raw);
        raw.e = ed;
        Row::unpack(raw, d, de);
        small(r + step);
#pragma unroll
        for (int v = 0; v < Row::NP; ++v) {
            // places outside the row have x = dy = gamma = 0 and add nothing: h = 0 there, for -mean rstd may overflow and 0 inf is NaN
            const float2 m = VEC > 1 ? f2_splat(k.has(2 * Row::VP * v) ? -mu : 0.0f) : make_float2(k.has(2 * v) ? -mu : 0.0f, k.has(2 * v + 1) ? -mu : 0.0f);
#pragma unroll
            for (int i = v * Row::VP; i < (v + 1) * Row::VP; ++i) h[i] = f2_mul(f2_add(h[i], m), f2_splat(rs));
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            dg[i] = f2_fma(d[i], h[i], dg[i]);
            db[i] = f2_add(db[i], d[i]);
            d[i] = f2_mul(d[i], gm[i]);
            t0 = f2_add(t0, d[i]);
            t1 = f2_fma(d[i], h[i], t1);
        }
        float s0 = t0.x + t0.y, s1 = t1.x + t1.y;
        if (EDGE) {
            he = k.has_edge() ? (he - mu) * rs : 0.0f;
            dge = fmaf(de, he, dge);
            dbe += de;
            de *= gme;
            s0 += de;
            s1 = fmaf(de, he, s1);
        }
        // both sums at once: the lower half of a warp goes on with s0, the upper with s1
        const bool upper = lane & 16;
        float sum = (upper ? s1 : s0) + __shfl_xor_sync(~0u, upper ? s0 : s1, 16);
#pragma unroll
        for (int o = 8; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        if (!WARP) {
            float* buf = red + 64 * flip + 2 * (lane & 16);  // [sum][warp], PAIR: [sum][rank][warp]
            flip ^= 1;
            const int w = (int)(threadIdx.x % G) >> 5, at = PAIR ? rank * 16 + w : w;
            if ((lane & 15) == 0) buf[at] = sum;
            if (PAIR) {
                if ((lane & 15) == 0) {
                    unsigned to;
                    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((unsigned)__cvta_generic_to_shared(buf + at)), "r"(rank ^ 1));
                    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(sum) : "memory");
                }
                __syncwarp();
                asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
                asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            } else if (per == 1) {
                __syncthreads();
            } else {
                asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(G) : "memory");
            }
            const int v = lane & 15;                        // at most 16 warps
            sum = v < G >> 5 ? PAIR ? buf[v] + buf[16 + v] : buf[v] : 0.0f;
#pragma unroll
            for (int o = 8; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        }
        s0 = __shfl_sync(~0u, sum, 0), s1 = __shfl_sync(~0u, sum, 16);
        s0 *= inv, s1 *= inv;
#pragma unroll
        for (int i = 0; i < P; ++i) d[i] = f2_mul(f2_splat(rs), f2_fma(h[i], f2_splat(-s1), f2_add(d[i], f2_splat(-s0))));
        k.store(a.dx + c0 + r * a.dxs, d, rs * fmaf(he, -s1, de - s0));
    }
    if (!a.part) return;
    float* part = a.part + (size_t)block * 2 * a.cols;
    float* to = per > 1 ? combine + (size_t)group * 2 * a.cols : part + c0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        if (k.has(2 * i)) to[k.col(2 * i)] = dg[i].x, to[a.cols + k.col(2 * i)] = db[i].x;
        if (k.has(2 * i + 1)) to[k.col(2 * i + 1)] = dg[i].y, to[a.cols + k.col(2 * i + 1)] = db[i].y;
    }
    if (k.has_edge()) to[k.edge] = dge, to[a.cols + k.edge] = dbe;
    if (per > 1) {
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * a.cols; c += blockDim.x) {
            float s = 0;
            for (int w = 0; w < per; ++w) s += combine[(size_t)w * 2 * a.cols + c];
            part[c] = s;
        }
    }
}

// Longer rows: dx alone, two passes over the row (the second from L2) ...
template <typename T>
__global__ void __launch_bounds__(1024) k_ln_bwd_long(const LnBwd<T> a) {
    __shared__ __align__(16) float red[2][32];
    ln_clear(red[0], 64);
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *dy = a.dy + r * a.dys, *x = a.x + r * a.xs;
        const float mu = a.mean[r], rs = a.rstd[r];
        float s0 = 0, s1 = 0;
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
            const float g = to_f32(dy[c]) * ln_param<T>(a.gamma, a.p32, c, 1.0f);
            s0 += g;
            s1 = fmaf(g, (to_f32(x[c]) - mu) * rs, s1);
        }
        const float m0 = ln_row_sum<false, true>(s0, red[0]) / a.cols, m1 = ln_row_sum<false, true>(s1, red[1]) / a.cols;
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
            const float g = to_f32(dy[c]) * ln_param<T>(a.gamma, a.p32, c, 1.0f);
            a.dx[r * a.dxs + c] = from_f32<T>(rs * (g - m0 - (to_f32(x[c]) - mu) * rs * m1));
        }
    }
}
// ... and the partial sums of the parameters' gradients, a column per thread, a chunk of rows per blockIdx.y
template <typename T>
__global__ void __launch_bounds__(kLnThreads) k_ln_bwd_long_part(const LnBwd<T> a) {
    const int c = blockIdx.x * kLnThreads + threadIdx.x;
    if (c >= a.cols) return;
    const long long r0 = a.rows * blockIdx.y / gridDim.y, r1 = a.rows * (blockIdx.y + 1) / gridDim.y;
    float g = 0, b = 0;
    for (long long r = r0; r < r1; ++r) {
        const float d = to_f32(a.dy[r * a.dys + c]);
        g = fmaf(d, (to_f32(a.x[r * a.xs + c]) - a.mean[r]) * a.rstd[r], g);
        b += d;
    }
    a.part[(size_t)blockIdx.y * 2 * a.cols + c] = g;
    a.part[((size_t)blockIdx.y * 2 + 1) * a.cols + c] = b;
}

// dgamma and dbeta from the partial sums [parts][2 cols]: 32 columns per CTA, 32 warps over the parts, a fixed order
__global__ void __launch_bounds__(1024) k_ln_bwd_sum(const float* __restrict__ part, int parts, int cols, float* __restrict__ dgamma,
                                                     float* __restrict__ dbeta) {
    __shared__ float red[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;
    pdl_wait();
    float s = 0;
    if (c < 2ll * cols)
        for (int p = warp; p < parts; p += 32) s += part[(size_t)p * 2 * cols + c];
    red[warp][lane] = s;
    __syncthreads();
    s = warp_sum(red[lane][warp]);
    const long long o = (long long)blockIdx.x * 32 + warp;
    if (lane == 0 && o < 2ll * cols) {
        float* to = o < cols ? dgamma : dbeta;
        if (to) to[o < cols ? o : o - cols] = s;
    }
}

// CTAs of a kernel that an SM holds; the last answer for a CTA size is kept with the shared memory it was given for (which goes by the
// columns as well), so that grid and order of sums never depend on the widths of earlier calls
template <typename K>
static int ln_resident(K kernel, int threads, int smem, std::atomic<uint64_t>* cache) {
    // 48 KB are allowed without asking, the static arrays included; one size for all calls, so that none takes back another's
    if (smem > 32 << 10) allow_big_smem(kernel, 200 << 10);
    const uint64_t kept = cache[threads / 32].load(std::memory_order_relaxed);
    if (kept && (int)(kept >> 32) == smem) return (int)(unsigned)kept;
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) != cudaSuccess || n < 1) n = 1;
    cache[threads / 32].store((uint64_t)smem << 32 | (unsigned)n, std::memory_order_relaxed);
    return n;
}

// threads that hold a row
template <int VEC, int NV, bool WARP>
static int ln_threads(int cols) { return WARP ? kLnThreads : ((cols / VEC + NV - 1) / NV + 31) / 32 * 32; }
// CTAs: one per row (or eight), or as many as are resident; with EDGE then a multiple of 8 (see LnRow)
template <bool EDGE, bool WARP>
static int ln_grid(long long rows, int resident) {
    const long long want = WARP ? (rows + kLnThreads / 32 - 1) / (kLnThreads / 32) : rows;
    const long long most = EDGE ? (long long)kSMs * resident / 8 * 8 : (long long)kSMs * resident;
    return (int)(want < most ? want : most);
}

template <typename T, int VEC, int NV, bool EDGE, bool WARP, int AHEAD, bool MANY = false>
static void ln_fwd_launch(const LnFwd<T>& a, cudaStream_t st) {
    static std::atomic<uint64_t> cache[33];
    const int threads = ln_threads<VEC, NV, WARP>(a.cols);
    const int smem = VEC > 1 ? LnRow<T, VEC, NV, EDGE, AHEAD>::D * NV * 16 * threads : 0;
    const int resident = ln_resident(k_ln_fwd<T, VEC, NV, EDGE, WARP, AHEAD, MANY>, threads, smem, cache);
    const int grid = ln_grid<EDGE, WARP>(a.rows, resident);
    TRV_LAUNCH((k_ln_fwd<T, VEC, NV, EDGE, WARP, AHEAD, MANY>), grid, threads, smem, st, a);
}
template <typename T, bool EDGE>
static bool ln_forward_vec(const LnFwd<T>& a, cudaStream_t st) {
    // A warp's rows: as few elements a thread as hold them.  Longer rows: 32 elements a thread (16: 16384 x 4096 bfloat16 50 us
    // against 49, 8192 x 8190 72 us against 54).  Rows on their way, FAR in a warp's rows and the longest, else one (bfloat16, two
    // instead of one: 16384 x 5120 61 us against 56, 32768 x 8192 191 us against 168; 8192 x 16384 86 us against 95, 65536 x 400
    // 21 us against 23; float32 4096 x 12288 78 us against 72).
    constexpr int VEC = 16 / sizeof(T), NV = 32 / VEC, FAR = sizeof(T) == 4 ? 1 : 2;
    if (a.cols < VEC) return false;
    if (a.cols <= 32 * VEC) ln_fwd_launch<T, VEC, 1, EDGE, true, FAR>(a, st);
    else if (a.cols <= 64 * VEC) ln_fwd_launch<T, VEC, 2, EDGE, true, FAR>(a, st);
    else if (a.cols <= 32 * 16) ln_fwd_launch<T, VEC, NV / 2, EDGE, true, FAR>(a, st);
    else if (a.cols <= kLnThreads * 32) ln_fwd_launch<T, VEC, NV, EDGE, false, 1>(a, st);
    else if (a.cols <= kLnMaxThreads * 32) ln_fwd_launch<T, VEC, NV, EDGE, false, FAR, true>(a, st);
    else return false;
    return true;
}
template <typename T>
static void ln_forward(const LnFwd<T>& a, cudaStream_t st) {
    constexpr int VEC = 16 / sizeof(T);
    // 16-byte accesses need rows of x and y that start at the same place of a 16-byte vector
    const bool vec = !(((uintptr_t)a.x ^ (uintptr_t)a.y) & 15) && (a.rows == 1 || (a.xs - a.ys) % VEC == 0);
    const bool edge = ((uintptr_t)a.x & 15) || a.xs % VEC || a.cols % VEC;
    if (vec && (edge ? ln_forward_vec<T, true>(a, st) : ln_forward_vec<T, false>(a, st))) return;
    if (a.cols <= kLnMaxThreads * 8) ln_fwd_launch<T, 1, 8, false, false, 1, true>(a, st);
    else TRV_LAUNCH(k_ln_fwd_long<T>, (unsigned)(a.rows < 65536 ? a.rows : 65536), 1024, 0, st, a);
}

template <typename T, int VEC, int NV, bool EDGE, LnShare SHARE>
static int ln_bwd_launch(LnBwd<T> a, cudaStream_t st) {
    static std::atomic<uint64_t> cache[33];
    constexpr bool WARP = SHARE == LN_WARP, PAIR = SHARE == LN_PAIR;
    int cols = a.cols;
    if (PAIR) cols = a.cols0 = (a.cols + 2 * VEC - 1) / (2 * VEC) * VEC;        // the larger half
    const int group = ln_threads<VEC, NV, false>(cols);
    const int per = WARP ? kLnThreads / 32 : PAIR || group > kLnThreads / 2 ? 1 : kLnThreads / group;   // rows at a time
    const int threads = WARP ? kLnThreads : per * group;
    a.group = group;
    const int smem = (WARP ? 0 : 512 * per) + (per > 1 ? per * 8 * ((a.cols + 1) & ~1) : 0) + (VEC > 1 ? 2 * LnRow<T, VEC, NV, EDGE, kLnBwdAhead<T>>::D * NV * 16 * threads : 0);
    int resident = ln_resident(k_ln_bwd<T, VEC, NV, EDGE, SHARE>, threads, smem, cache);
    if (resident > kLnMaxParts / kSMs) resident = kLnMaxParts / kSMs;
    const long long want = (a.rows + per - 1) / per;
    long long most = (long long)kSMs * resident / (PAIR ? 2 : 1);
    if (EDGE) most = most / 8 * 8;                          // see LnRow
    const int grid = (int)(want < most ? want : most);
    if (!grid) return 0;
    if (!PAIR) {
        TRV_LAUNCH((k_ln_bwd<T, VEC, NV, EDGE, SHARE>), grid, threads, smem, st, a);
    } else {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim = {2, 1, 1};
        cfg.attrs = attr, cfg.numAttrs = 1, cfg.stream = st, cfg.gridDim = dim3(2 * grid), cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = smem;
        (void)cudaLaunchKernelEx(&cfg, k_ln_bwd<T, VEC, NV, EDGE, SHARE>, a);       // the caller asks for the last error
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    return grid;
}
template <typename T, bool EDGE>
static int ln_backward_vec(const LnBwd<T>& a, cudaStream_t st) {
    constexpr int VEC = 16 / sizeof(T), NV = 16 / VEC;      // 16 elements a thread: their sums, gamma and two rows' values fit 128 registers
    if (a.cols < VEC) return -1;
    if (a.cols <= 32 * VEC) return ln_bwd_launch<T, VEC, 1, EDGE, LN_WARP>(a, st);
    if (a.cols <= 64 * VEC) return ln_bwd_launch<T, VEC, 2, EDGE, LN_WARP>(a, st);
    if (a.cols <= kLnMaxThreads * 16) return ln_bwd_launch<T, VEC, NV, EDGE, LN_GROUP>(a, st);
    if (a.cols <= 2 * kLnMaxThreads * 16) return ln_bwd_launch<T, VEC, NV, EDGE, LN_PAIR>(a, st);
    return -1;
}
static int ln_parts(size_t rows) { return (int)(rows < kLnMaxParts ? (rows ? rows : 1) : kLnMaxParts); }

template <typename T>
static void ln_backward(const LnBwd<T>& a, float* dgamma, float* dbeta, cudaStream_t st) {
    constexpr int VEC = 16 / sizeof(T);
    const bool vec = !((((uintptr_t)a.x ^ (uintptr_t)a.dy) | ((uintptr_t)a.x ^ (uintptr_t)a.dx)) & 15) &&
                     (a.rows <= 1 || ((a.xs - a.dys) % VEC == 0 && (a.xs - a.dxs) % VEC == 0));
    const bool edge = ((uintptr_t)a.x & 15) || a.xs % VEC || a.cols % VEC;
    int parts = !vec ? -1 : edge ? ln_backward_vec<T, true>(a, st) : ln_backward_vec<T, false>(a, st);
    if (parts < 0 && a.cols <= kLnMaxThreads * 8) parts = ln_bwd_launch<T, 1, 8, false, LN_GROUP>(a, st);
    if (parts < 0) {
        if (a.rows) TRV_LAUNCH(k_ln_bwd_long<T>, (unsigned)(a.rows < 65536 ? a.rows : 65536), 1024, 0, st, a);
        parts = a.rows ? ln_parts((size_t)a.rows) : 0;
        if (a.part && parts) TRV_LAUNCH(k_ln_bwd_long_part<T>, dim3((a.cols + kLnThreads - 1) / kLnThreads, parts), kLnThreads, 0, st, a);
    }
    if (a.part) launch_pdl(k_ln_bwd_sum, dim3((unsigned)((2ll * a.cols + 31) / 32)), dim3(1024), 0, st, (const float*)a.part, parts, a.cols, dgamma, dbeta);
}

static trv_status_t ln_check(size_t rows, size_t cols, trv_dtype_t dtype, trv_dtype_t param_dtype) {
    if (!float_dtype(dtype) || (param_dtype != TRV_FLOAT32 && param_dtype != dtype)) return TRV_ERR_INVALID_ARG;
    if (rows >= ((size_t)1 << 40) || cols >= ((size_t)1 << 30)) return TRV_ERR_UNSUPPORTED;
    return TRV_OK;
}
static bool ln_stride_ok(size_t rows, size_t cols, size_t stride) {
    return stride >= cols && (rows <= 1 || stride <= ((size_t)1 << 60) / rows / 4);
}

}  // namespace trv

using namespace trv;

extern "C" trv_status_t trv_layernorm_forward(const void* x, const void* gamma, const void* beta, void* y, float* mean, float* rstd,
                                              size_t rows, size_t cols, size_t x_stride, size_t y_stride, float eps, trv_dtype_t dtype,
                                              trv_dtype_t param_dtype, void* cuda_stream) {
    const trv_status_t bad = ln_check(rows, cols, dtype, param_dtype);
    if (bad != TRV_OK) return bad;
    if (!ln_stride_ok(rows, cols, x_stride) || !ln_stride_ok(rows, cols, y_stride) || !(eps >= 0)) return TRV_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return TRV_OK;
    if (!x || !y) return TRV_ERR_INVALID_ARG;
    const size_t es = dtype_bytes(dtype), ps = dtype_bytes(param_dtype);
    if (misaligned(x, es) || misaligned(y, es) || misaligned(gamma, ps) || misaligned(beta, ps) || misaligned(mean, 4) || misaligned(rstd, 4))
        return TRV_ERR_INVALID_ARG;
    const Span in[3] = {matrix_span(x, rows, cols, x_stride, es), {gamma, cols * ps}, {beta, cols * ps}};
    const Span out[3] = {matrix_span(y, rows, cols, y_stride, es), {mean, rows * 4}, {rstd, rows * 4}};
    if (!disjoint(in, out)) return TRV_ERR_INVALID_ARG;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    auto run = [&](auto zero) {
        using T = decltype(zero);
        ln_forward<T>({(const T*)x, gamma, beta, (T*)y, mean, rstd, (long long)rows, (long long)x_stride, (long long)y_stride, (int)cols,
                       param_dtype == TRV_FLOAT32, eps}, st);
    };
    if (dtype == TRV_FLOAT32) run(0.0f);
    else if (dtype == TRV_BFLOAT16) run(__nv_bfloat16());
    else run(__half());
    g_last_kernel = "layernorm_forward";
    return cudaGetLastError() == cudaSuccess ? TRV_OK : TRV_ERR_CUDA;
}

extern "C" trv_status_t trv_layernorm_workspace_bytes(size_t rows, size_t cols, size_t* bytes) {
    if (!bytes) return TRV_ERR_INVALID_ARG;
    *bytes = 0;
    if (rows >= ((size_t)1 << 40) || cols >= ((size_t)1 << 30)) return TRV_ERR_UNSUPPORTED;
    *bytes = (size_t)ln_parts(rows) * 2 * cols * 4;
    return TRV_OK;
}

extern "C" trv_status_t trv_layernorm_backward(const void* dy, const void* x, const void* gamma, const float* mean, const float* rstd,
                                               void* dx, float* dgamma, float* dbeta, size_t rows, size_t cols, size_t dy_stride,
                                               size_t x_stride, size_t dx_stride, trv_dtype_t dtype, trv_dtype_t param_dtype,
                                               void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const trv_status_t bad = ln_check(rows, cols, dtype, param_dtype);
    if (bad != TRV_OK) return bad;
    if (!ln_stride_ok(rows, cols, dy_stride) || !ln_stride_ok(rows, cols, x_stride) || !ln_stride_ok(rows, cols, dx_stride))
        return TRV_ERR_INVALID_ARG;
    if (cols == 0) return TRV_OK;
    if (rows && (!dy || !x || !mean || !rstd || !dx)) return TRV_ERR_INVALID_ARG;
    const size_t es = dtype_bytes(dtype), ps = dtype_bytes(param_dtype);
    if (misaligned(dy, es) || misaligned(x, es) || misaligned(dx, es) || misaligned(gamma, ps) || misaligned(mean, 4) || misaligned(rstd, 4) ||
        misaligned(dgamma, 4) || misaligned(dbeta, 4))
        return TRV_ERR_INVALID_ARG;
    size_t need = 0;
    if (dgamma || dbeta) {
        trv_layernorm_workspace_bytes(rows, cols, &need);
        if (!workspace || misaligned(workspace, 256) || workspace_bytes < need) return TRV_ERR_SCRATCH;
    }
    const Span in[5] = {matrix_span(dy, rows, cols, dy_stride, es), matrix_span(x, rows, cols, x_stride, es), {gamma, cols * ps},
                        {mean, rows * 4}, {rstd, rows * 4}};
    const Span out[4] = {matrix_span(dx, rows, cols, dx_stride, es), {dgamma, cols * 4}, {dbeta, cols * 4}, {workspace, need}};
    if (!disjoint(in, out)) return TRV_ERR_INVALID_ARG;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    auto run = [&](auto zero) {
        using T = decltype(zero);
        ln_backward<T>({(const T*)dy, (const T*)x, gamma, mean, rstd, (T*)dx, need ? (float*)workspace : nullptr, (long long)rows,
                        (long long)dy_stride, (long long)x_stride, (long long)dx_stride, (int)cols, param_dtype == TRV_FLOAT32, 0, 0}, dgamma, dbeta, st);
    };
    if (dtype == TRV_FLOAT32) run(0.0f);
    else if (dtype == TRV_BFLOAT16) run(__nv_bfloat16());
    else run(__half());
    g_last_kernel = "layernorm_backward";
    return cudaGetLastError() == cudaSuccess ? TRV_OK : TRV_ERR_CUDA;
}
