// Expert router with balance loss.  Token t with logits l over E experts: p = softmax(l); ids = the k largest logits, ties to
// the lowest index; gates = p at the ids, or that over its sum.  Over all counted tokens (mask on, some logit not -inf):
// c_e = tokens that chose e, S_e = sum of p_te, N = their number;  loss = coef E / (k N^2) sum_e c_e S_e, c held constant.
// Gradient: with q_e = coef E c_e / (k N^2) and G_e = the gate's incoming gradient at a chosen e, else 0,
//   gates = p          : dl_e = p_e (q_e + G_e - sum_j p_j (q_j + G_j))
//   gates = p / sum = w: dl_e = p_e (q_e - sum_j p_j q_j) + w_e (G_e - sum_j w_j G_j)
//
// A token belongs to a group of G = 1 .. 32 lanes, 8 neighbouring experts to a lane (16 or 32 above 256 and 512 experts), so one
// 16-byte access brings a lane's share of a 16-bit row, and a warp works on 32 / G tokens at once.  Selection: logits become
// order-preserving integers with the index below, so that all differ and ties sort themselves; a lane sorts its 8 once, and
// each of the k rounds is one reduction over the lanes' heads and a shift in the lane that lost its head.  The first round's
// value is the softmax's maximum.  Probability sums stay in registers, counts in shared memory; the CTAs' parts are added by a
// second kernel in a fixed order.
//
// Bound by issue slots and the integer pipe, not by memory: compares and selects of the selection run at half rate, and with 8
// choices of 256 experts most of a token's steps leave no lane idle.  What only the choices need (a gate's exponential, its store, the
// count) is done for several turns at once, so that every lane has a choice.  65536 x 256 bfloat16, k = 8: forward 36 us (41 with
// the choices of each token apart), backward 28 us; the logits alone would pass in 5 us.  3 to 6 CTAs per SM: no difference.
#include "trv_train.cuh"

namespace trv {

constexpr int kRtThreads = 256, kRtWarps = kRtThreads / 32;
constexpr int kRtMaxExperts = 1024, kRtMaxK = 32, kRtMaxBlocks = 4 * kSMs;

// Keys.  High part: the value as an unsigned number of the same order; low part: the index counted down from the end, so that of
// equal values the lower index has the larger key.  Adding +0 first makes -0 equal to +0 and every NaN the canonical one, which
// ranks above every number.  Keys up to kNone are those of -inf (closed experts, places behind the last expert, tokens left out).
// 16-bit types: both parts in 32 bits, two values at a time.
template <typename T> struct RtKey { using type = unsigned; };
template <> struct RtKey<float> { using type = unsigned long long; };
template <typename T> __device__ __forceinline__ constexpr typename RtKey<T>::type rt_none();
template <> __device__ __forceinline__ constexpr unsigned rt_none<__nv_bfloat16>() { return 0x007fffffu; }
template <> __device__ __forceinline__ constexpr unsigned rt_none<__half>() { return 0x03ffffffu; }
template <> __device__ __forceinline__ constexpr unsigned long long rt_none<float>() { return 0x007fffffffffffffull; }
template <typename T> __device__ __forceinline__ constexpr unsigned rt_closed();        // the bits of -inf, twice for 16-bit types
template <> __device__ __forceinline__ constexpr unsigned rt_closed<__nv_bfloat16>() { return 0xff80ff80u; }
template <> __device__ __forceinline__ constexpr unsigned rt_closed<__half>() { return 0xfc00fc00u; }
template <> __device__ __forceinline__ constexpr unsigned rt_closed<float>() { return 0xff800000u; }

__device__ __forceinline__ unsigned rt_plus_zero(unsigned u, __nv_bfloat16) {
    __nv_bfloat162 h;
    memcpy(&h, &u, 4);
    h = __hadd2(h, __nv_bfloat162(__ushort_as_bfloat16(0), __ushort_as_bfloat16(0)));
    memcpy(&u, &h, 4);
    return u;
}
__device__ __forceinline__ unsigned rt_plus_zero(unsigned u, __half) {
    __half2 h;
    memcpy(&h, &u, 4);
    h = __hadd2(h, __half2(__ushort_as_half(0), __ushort_as_half(0)));
    memcpy(&u, &h, 4);
    return u;
}
__device__ __forceinline__ int rt_index(unsigned key) { return 0xffff - (int)(key & 0xffffu); }
__device__ __forceinline__ int rt_index(unsigned long long key) { return (int)(0xffffffffu - (unsigned)key); }
__device__ __forceinline__ float rt_value(unsigned key, __nv_bfloat16) {
    const unsigned o = key & 0xffff0000u;
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o & 0xffff0000u);
}
__device__ __forceinline__ float rt_value(unsigned key, __half) {
    const unsigned o = key >> 16, b = o & 0x8000u ? o ^ 0x8000u : ~o & 0xffffu;
    return __half2float(__ushort_as_half((unsigned short)b));
}
__device__ __forceinline__ float rt_value(unsigned long long key, float) {
    const unsigned o = (unsigned)(key >> 32);
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

// a lane's V logits, experts e0 .. e0 + V - 1 of a row, as 32-bit words of one or two; -inf behind the last expert
template <typename T, int V> struct RtRow {
    static constexpr int W = V * sizeof(T) / 4, PER = 4 / sizeof(T);
    unsigned w[W];
    __device__ __forceinline__ void load(const T* row, int e0, int E, bool vec) {
        if (vec && e0 + V <= E) {
#pragma unroll
            for (int i = 0; i < W; i += 4) {
                const uint4 u = *(const uint4*)(row + e0 + i * PER);
                w[i] = u.x, w[i + 1] = u.y, w[i + 2] = u.z, w[i + 3] = u.w;
            }
        } else {
            T x[V];
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = e0 + i < E ? row[e0 + i] : from_f32<T>(-INFINITY);
            memcpy(w, x, sizeof(w));
        }
    }
    __device__ __forceinline__ void close() {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = rt_closed<T>();
    }
    __device__ __forceinline__ void values(float2 (&f)[V / 2]) const {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            if constexpr (sizeof(T) == 4) {
                f[i] = make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
            } else {
                T t[2];
                memcpy(t, &w[i], 4);
                f[i] = make_float2(to_f32(t[0]), to_f32(t[1]));
            }
        }
    }
    __device__ __forceinline__ void keys(int e0, typename RtKey<T>::type (&k)[V]) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const unsigned u = __float_as_uint(__fadd_rn(__uint_as_float(w[i]), 0.0f));
                k[i] = (unsigned long long)(u ^ ((unsigned)((int)u >> 31) | 0x80000000u)) << 32 | (0xffffffffu - (unsigned)(e0 + i));
            }
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const unsigned u = rt_plus_zero(w[i], T()), s = u ^ (((u >> 15) & 0x00010001u) * 0x7fffu | 0x80008000u);
                k[2 * i] = s << 16 | (0xffffu - (unsigned)(e0 + 2 * i));
                k[2 * i + 1] = (s & 0xffff0000u) | (0xffffu - (unsigned)(e0 + 2 * i + 1));
            }
        }
    }
};

// over the G lanes of a group
template <int G>
__device__ __forceinline__ unsigned rt_max(unsigned v) {
    if (G == 32) return __reduce_max_sync(~0u, v);
#pragma unroll
    for (int o = G / 2; o; o >>= 1) v = max(v, __shfl_xor_sync(~0u, v, o));
    return v;
}
template <int G>
__device__ __forceinline__ unsigned long long rt_max(unsigned long long v) {
    if (G == 32) {
        const unsigned hi = __reduce_max_sync(~0u, (unsigned)(v >> 32));
        const unsigned lo = __reduce_max_sync(~0u, (unsigned)(v >> 32) == hi ? (unsigned)v : 0u);
        return (unsigned long long)hi << 32 | lo;
    }
#pragma unroll
    for (int o = G / 2; o; o >>= 1) v = max(v, __shfl_xor_sync(~0u, v, o));
    return v;
}
template <int G>
__device__ __forceinline__ float rt_sum(float v) {
#pragma unroll
    for (int o = G / 2; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

// two sums at once: the halves of a group go on with one each
template <int G>
__device__ __forceinline__ float2 rt_sum2(float2 v) {
    if (G < 8) return make_float2(rt_sum<G>(v.x), rt_sum<G>(v.y));
    const bool upper = threadIdx.x & (G / 2);
    float mine = upper ? v.y : v.x;
    mine += __shfl_xor_sync(~0u, upper ? v.x : v.y, G / 2);
#pragma unroll
    for (int o = G / 4; o; o >>= 1) mine += __shfl_xor_sync(~0u, mine, o);
    return make_float2(__shfl_sync(~0u, mine, 0, G), __shfl_sync(~0u, mine, G / 2, G));
}
// maximum of the numbers among them
template <int G>
__device__ __forceinline__ float rt_fmax(float v) {
    if (G == 32) {
        float r;
        asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
        return r;
    }
#pragma unroll
    for (int o = G / 2; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    return v;
}

// descending, Batcher's odd-even merge network
template <int V, typename K>
__device__ __forceinline__ void rt_sort(K (&k)[V]) {
#pragma unroll
    for (int p = 1; p < V; p *= 2)
#pragma unroll
        for (int q = p; q; q /= 2)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int at = i - q % p;                   // pairs (i, i + q), blocks of 2 q from q mod p on, within blocks of 2 p
                if (at >= 0 && at / q % 2 == 0 && i + q < V && i / (2 * p) == (i + q) / (2 * p)) {
                    const K a = k[i], b = k[i + q];
                    k[i] = max(a, b);
                    k[i + q] = min(a, b);
                }
            }
}

// e^x for x <= 0 (or NaN), relative error up to (1.3 |x| + 4) 2^-24: x log2 e is rounded once, as x = l - top was before it, and the
// instruction adds its 2 ulp; below 2^-126 zero
__device__ __forceinline__ float rt_exp(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.4426950408889634f));
    return r;
}

// 1 / x to 1 ulp; x is a sum of exponentials, which are normal numbers (see rt_exp)
__device__ __forceinline__ float rt_inverse(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// e^(l - top) of a lane's values in place, and their sum; a row of -inf gives zeros
template <int V>
__device__ __forceinline__ float rt_exps(float2 (&l)[V / 2], float top) {
    float2 z = make_float2(0, 0);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        l[i] = f2_mul(f2_add(l[i], f2_splat(-top)), f2_splat(1.4426950408889634f));
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(l[i].x));
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(l[i].y));
        z = f2_add(z, l[i]);
    }
    return z.x + z.y;
}

template <typename T>
struct RouterArgs {
    const T* logits;
    const uint8_t* mask;
    long long tokens, ls, ds;
    int E, k, normalize;
    bool vec;               // rows of logits (and dlogits) start on 16-byte boundaries
    int *ids, *part_c;
    float *gates, *part_p;
    const int* counts;
    const float* dgates;
    T* dlogits;
    float coef;
};

template <typename T, int V, int G>
__global__ void __launch_bounds__(kRtThreads) k_router_fwd(const RouterArgs<T> a) {
    using K = typename RtKey<T>::type;
    constexpr int PER = 32 / G, KMAX = V * G < kRtMaxK ? V * G : kRtMaxK;       // tokens of a warp, most choices of a token
    __shared__ int cnt[V * G + 1];
    __shared__ float ps[kRtWarps][V * G];
    __shared__ K chosen[kRtWarps][PER * KMAX < 32 ? 32 : PER * KMAX];
    __shared__ float2 found[kRtWarps][32];                  // of a token: top and 1 / sum of the exponentials
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, in = lane % G, group = lane / G, e0 = in * V, E = a.E, k = a.k;
    // The choices of `turns` turns are written together, 1 << ks places to a token, so that every lane has one
    const int ks = k > 1 ? 32 - __clz(k - 1) : 0, turns = max(1, 32 / PER >> ks);
    for (int e = threadIdx.x; e <= E; e += kRtThreads) cnt[e] = 0;
    __syncthreads();
    float2 sum[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) sum[i] = make_float2(0, 0);
    int live_tokens = 0;
    const long long step = (long long)gridDim.x * kRtWarps * PER;
    long long t0 = ((long long)blockIdx.x * kRtWarps + warp) * PER;
    RtRow<T, V> next;
    bool next_on = false;
    auto fetch = [&](long long t) {
        next_on = t < a.tokens && (!a.mask || a.mask[t]);
        if (next_on) next.load(a.logits + t * a.ls, e0, E, a.vec);
    };
    fetch(t0 + group);
    long long first = t0;
    int turn = 0;
    auto write = [&] {
        __syncwarp();
        const int places = turn * PER << ks;                // at most 32, or a multiple of it
        for (int i = lane; i - lane < places; i += 32) {
            const int b = i >> ks, j = i & ((1 << ks) - 1);
            const long long t = first + b / PER * step + b % PER;
            const K c = i < places && j < k ? chosen[warp][i] : K(0);
            const bool is = c > rt_none<T>();
            const float2 f = found[warp][b];
            const float e = is ? rt_exp(rt_value(c, T()) - f.x) : 0.0f;
            float scale = f.y;
            if (a.normalize) {
                float s = e;
                for (int o = 1 << ks >> 1; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
                scale = s == 0.0f ? 0.0f : rt_inverse(s);
            }
            if (is) atomicAdd(&cnt[rt_index(c)], 1);
            live_tokens += is && j == 0;
            if (i < places && j < k && t < a.tokens) {
                a.ids[t * k + j] = is ? rt_index(c) : -1;
                a.gates[t * k + j] = is ? e * scale : 0.0f;
            }
        }
        __syncwarp();
    };
    for (; t0 < a.tokens; t0 += step) {
        const long long t = t0 + group;
        const int b = turn * PER + group;
        K* const mine = &chosen[warp][b << ks];
        if (!next_on) next.close();
        float2 l[V / 2];
        K key[V];
        next.values(l);
        next.keys(e0, key);
        fetch(t + step);
        rt_sort<V>(key);
        K best = rt_max<G>(key[0]);
        const bool live = best > rt_none<T>();
        const float top = live ? rt_value(best, T()) : 0.0f;
        const float z = rt_sum<G>(rt_exps<V>(l, top)), inv = live ? rt_inverse(z) : 0.0f;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) sum[i] = f2_fma(l[i], f2_splat(inv), sum[i]);
        // Round j: the group's largest head, and a shift in the lane that lost it (selects, not a branch that one lane takes every
        // time).  Up to 8 rounds unrolled: behind round j only the next 7 - j keys of a lane can still be asked for.
        auto shift = [&](auto keep) {
            const bool lost = key[0] == best;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < decltype(keep)::value) key[i] = !lost ? key[i] : i + 1 < V ? key[i + 1 < V ? i + 1 : i] : K(0);
            best = rt_max<G>(key[0]);
        };
        if (k <= 8) {
            auto round = [&](auto j) {
                constexpr int J = decltype(j)::value;
                if (in == 0 && J < k) mine[J] = best;
                if constexpr (J < 7)
                    if (J + 1 < k) shift(std::integral_constant<int, 7 - J>());
            };
            round(std::integral_constant<int, 0>()), round(std::integral_constant<int, 1>()), round(std::integral_constant<int, 2>());
            round(std::integral_constant<int, 3>()), round(std::integral_constant<int, 4>()), round(std::integral_constant<int, 5>());
            round(std::integral_constant<int, 6>()), round(std::integral_constant<int, 7>());
        } else {
            for (int j = 0;;) {
                if (in == 0) mine[j] = best;
                if (++j >= k) break;
                shift(std::integral_constant<int, V>());
            }
        }
        if (in == 0) found[warp][b] = make_float2(top, inv);
        if (++turn == turns) {
            write();
            turn = 0, first = t0 + step;
        }
    }
    if (turn) write();
    if (live_tokens) atomicAdd(&cnt[E], live_tokens);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
#pragma unroll
        for (int o = G; o < 32; o *= 2) {
            sum[i].x += __shfl_xor_sync(~0u, sum[i].x, o);
            sum[i].y += __shfl_xor_sync(~0u, sum[i].y, o);
        }
        if (group == 0) ps[warp][e0 + 2 * i] = sum[i].x, ps[warp][e0 + 2 * i + 1] = sum[i].y;
    }
    __syncthreads();
    // a lone CTA's parts are the sums (part_p and part_c are then the caller's arrays)
    for (int e = threadIdx.x; e < E; e += kRtThreads) {
        float s = 0;
#pragma unroll
        for (int w = 0; w < kRtWarps; ++w) s += ps[w][e];
        a.part_p[(size_t)blockIdx.x * E + e] = s;
    }
    for (int e = threadIdx.x; e <= E; e += kRtThreads) a.part_c[(size_t)blockIdx.x * (E + 1) + e] = cnt[e];
}

// sums the parts of all CTAs in a fixed order: 8 columns per CTA, 128 threads to a column
constexpr int kRtSumThreads = 1024;
__global__ void __launch_bounds__(kRtSumThreads) k_router_sum(const float* __restrict__ part_p, const int* __restrict__ part_c, int parts, int E,
                                                              float* __restrict__ prob_sum, int* __restrict__ counts) {
    __shared__ float sp[8][kRtSumThreads / 8 + 1];
    __shared__ int sc[8][kRtSumThreads / 8 + 1];
    const int col = threadIdx.x & 7, row = threadIdx.x >> 3, e = blockIdx.x * 8 + col;
    float p = 0;
    int c = 0;
    pdl_wait();
#pragma unroll
    for (int i = 0; i < (kRtMaxBlocks + kRtSumThreads / 8 - 1) / (kRtSumThreads / 8); ++i) {
        const int b = row + i * (kRtSumThreads / 8);
        if (b < parts && e < E) p += part_p[(size_t)b * E + e];
        if (b < parts && e <= E) c += part_c[(size_t)b * (E + 1) + e];
    }
    sp[col][row] = p;
    sc[col][row] = c;
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, o = blockIdx.x * 8 + warp;
    if (warp >= 8) return;
    p = 0, c = 0;
#pragma unroll
    for (int i = 0; i < kRtSumThreads / 8; i += 32) p += sp[warp][lane + i], c += sc[warp][lane + i];
    p = warp_sum(p);
    c = __reduce_add_sync(~0u, c);
    if (lane == 0 && o < E) prob_sum[o] = p;
    if (lane == 0 && o <= E) counts[o] = c;
}

__global__ void __launch_bounds__(kRtThreads) k_balance_loss(const int* __restrict__ counts, const float* __restrict__ prob_sum, int E, int k,
                                                             float coef, float* __restrict__ loss) {
    __shared__ float red[kRtWarps];
    const float n = fmaxf((float)counts[E], 1.0f);
    float s = 0;
    for (int e = threadIdx.x; e < E; e += kRtThreads) s += ((float)counts[e] / n) * (prob_sum[e] / n);
    s = warp_sum(s);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0;
        for (int w = 0; w < kRtWarps; ++w) s += red[w];
        *loss = coef * (float)E / (float)k * s;
    }
}

// The gates' gradients reach their experts' lanes through a row of shared memory per token, zero but for the chosen places.  Four CTAs
// per SM (64 registers) from 8 lanes to a token on, although that spills 80 to 104 bytes with 8 lanes and 16 with 16 of them:
// 65536 x 64 12.5 -> 11.9 us; with fewer lanes it does not pay, 131072 x 16 float32 13.0 -> 14.4 us.
template <typename T, int V, int G>
__global__ void __launch_bounds__(kRtThreads, V == 8 && G >= 8 ? 4 : 1) k_router_bwd(const RouterArgs<T> a) {
    constexpr int PER = 32 / G, KMAX = V * G < kRtMaxK ? V * G : kRtMaxK, TURNS = (KMAX + G - 1) / G;     // choices of a token: TURNS per lane
    __shared__ __align__(16) float place[kRtWarps][32 * V];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, in = lane % G, group = lane / G, e0 = in * V, E = a.E, k = a.k;
    const float n = fmaxf((float)a.counts[E], 1.0f), scale = a.coef * (float)E / (float)k / n;
    float* mine = &place[warp][lane * V];                   // this lane's experts
    float* token = &place[warp][group * G * V];             // this token's
    float2 q[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        q[i].x = e0 + 2 * i < E ? scale * ((float)a.counts[e0 + 2 * i] / n) : 0.0f;
        q[i].y = e0 + 2 * i + 1 < E ? scale * ((float)a.counts[e0 + 2 * i + 1] / n) : 0.0f;
        mine[2 * i] = mine[2 * i + 1] = 0;
    }
    __syncwarp();
    const long long step = (long long)gridDim.x * kRtWarps * PER;
    long long t0 = ((long long)blockIdx.x * kRtWarps + warp) * PER;
    RtRow<T, V> next;
    bool next_on = false;
    int next_id[TURNS];
    float next_g[TURNS];
    auto fetch = [&](long long t) {
        next_on = t < a.tokens && (!a.mask || a.mask[t]);
        if (next_on) next.load(a.logits + t * a.ls, e0, E, a.vec);
        if (a.dgates)
#pragma unroll
            for (int i = 0; i < TURNS; ++i) {
                const int j = in + i * G;
                next_id[i] = -1, next_g[i] = 0;
                if (next_on && j < k) next_id[i] = a.ids[t * k + j], next_g[i] = a.dgates[t * k + j];
            }
    };
    fetch(t0 + group);
    for (; t0 < a.tokens; t0 += step) {
        const long long t = t0 + group;
        const bool there = t < a.tokens;
        if (!next_on) next.close();
        float2 p[V / 2], up[V / 2];
        next.values(p);
        int id[TURNS];
        float g[TURNS], w[TURNS];
        if (a.dgates)
#pragma unroll
            for (int i = 0; i < TURNS; ++i) {
                id[i] = (unsigned)next_id[i] < (unsigned)E ? next_id[i] : -1;
                g[i] = id[i] >= 0 ? next_g[i] : 0.0f;       // what stands at a place that is not an expert may be NaN or infinite
                w[i] = a.normalize && id[i] >= 0 ? to_f32(a.logits[t * a.ls + id[i]]) : -INFINITY;
            }
        fetch(t + step);
        auto put = [&](bool zero) {
#pragma unroll
            for (int i = 0; i < TURNS; ++i)
                if (id[i] >= 0) token[id[i]] = zero ? 0.0f : g[i];
            __syncwarp();
        };
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) top = fmaxf(top, fmaxf(p[i].x, p[i].y)), up[i] = q[i];
        top = rt_fmax<G>(top);
        if (top == -INFINITY) top = 0;                      // a row left out: exponentials of 0 (or NaN: fmax passes over it)
        if (a.dgates) {
            if (a.normalize) {
                float2 s = make_float2(0, 0);               // of the weights, and with their gradients
#pragma unroll
                for (int i = 0; i < TURNS; ++i) {
                    w[i] = rt_exp(w[i] - top);
                    s.x += w[i];
                    s.y = fmaf(w[i], g[i], s.y);
                }
                // only the lanes with choices, the first k of a group, need the sums
                s = k <= 8 ? rt_sum2<G < 8 ? G : 8>(s) : rt_sum2<G>(s);
                const float r = s.x == 0.0f ? 0.0f : rt_inverse(s.x);
                s.y *= r;
#pragma unroll
                for (int i = 0; i < TURNS; ++i) g[i] = w[i] * r * (g[i] - s.y);
            }
            put(false);
            if (!a.normalize)
#pragma unroll
                for (int i = 0; i < V / 2; i += 2) {
                    const float4 f = *(const float4*)(mine + 2 * i);
                    up[i] = f2_add(up[i], make_float2(f.x, f.y)), up[i + 1] = f2_add(up[i + 1], make_float2(f.z, f.w));
                }
        }
        float2 zs = make_float2(rt_exps<V>(p, top), 0), s2 = make_float2(0, 0);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) s2 = f2_fma(p[i], up[i], s2);
        zs.y = s2.x + s2.y;
        zs = rt_sum2<G>(zs);
        const float inv = zs.x == 0.0f ? 0.0f : rt_inverse(zs.x), s = zs.y * inv;
        T out[V];
#pragma unroll
        for (int i = 0; i < V / 2; i += 2) {
            // normalised gates: a term of its own, outside q's sum
            const float4 x = a.dgates && a.normalize ? *(const float4*)(mine + 2 * i) : make_float4(0, 0, 0, 0);
            const float2 f = f2_fma(f2_mul(p[i], f2_splat(inv)), f2_add(up[i], f2_splat(-s)), make_float2(x.x, x.y));
            const float2 h = f2_fma(f2_mul(p[i + 1], f2_splat(inv)), f2_add(up[i + 1], f2_splat(-s)), make_float2(x.z, x.w));
            out[2 * i] = from_f32<T>(f.x), out[2 * i + 1] = from_f32<T>(f.y), out[2 * i + 2] = from_f32<T>(h.x), out[2 * i + 3] = from_f32<T>(h.y);
        }
        if (a.dgates) {
            __syncwarp();
            put(true);
        }
        if (!there) continue;
        T* row = a.dlogits + t * a.ds + e0;
        if (a.vec && e0 + V <= E) {
#pragma unroll
            for (int i = 0; i < V; i += 16 / (int)sizeof(T)) {
                uint4 u;
                memcpy(&u, &out[i], 16);
                *(uint4*)(row + i) = u;
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (e0 + i < E) row[i] = out[i];
        }
    }
}

// lanes of a token's group, experts of a lane
static int rt_group(int E) {
    int g = 1;
    while (g < 32 && g * 8 < E) g *= 2;
    return g;
}
static int rt_blocks(size_t tokens, int E) {
    const size_t per = (size_t)kRtWarps * (32 / rt_group(E)), b = (tokens + per - 1) / per;
    return (int)(b < 1 ? 1 : b > kRtMaxBlocks ? kRtMaxBlocks : b);
}

template <typename T, int V, int G>
static void router_launch(const RouterArgs<T>& a, bool forward, cudaStream_t st) {
    const int blocks = rt_blocks((size_t)a.tokens, a.E);
    if (forward) TRV_LAUNCH((k_router_fwd<T, V, G>), blocks, kRtThreads, 0, st, a);
    else TRV_LAUNCH((k_router_bwd<T, V, G>), blocks, kRtThreads, 0, st, a);
}
template <typename T>
static void router_run(RouterArgs<T> a, bool forward, cudaStream_t st) {
    constexpr int W = 16 / sizeof(T);
    a.vec = !misaligned(a.logits, 16) && a.ls % W == 0 && (forward || (!misaligned(a.dlogits, 16) && a.ds % W == 0));
    switch (rt_group(a.E)) {
        case 1: return router_launch<T, 8, 1>(a, forward, st);
        case 2: return router_launch<T, 8, 2>(a, forward, st);
        case 4: return router_launch<T, 8, 4>(a, forward, st);
        case 8: return router_launch<T, 8, 8>(a, forward, st);
        case 16: return router_launch<T, 8, 16>(a, forward, st);
        default:
            if (a.E <= 256) router_launch<T, 8, 32>(a, forward, st);
            else if (a.E <= 512) router_launch<T, 16, 32>(a, forward, st);
            else router_launch<T, 32, 32>(a, forward, st);
    }
}

static trv_status_t router_check(size_t tokens, int32_t experts, int32_t top_k, size_t stride, trv_dtype_t dtype) {
    if (!float_dtype(dtype) || experts < 1 || top_k < 1 || top_k > experts || stride < (size_t)experts) return TRV_ERR_INVALID_ARG;
    if (experts > kRtMaxExperts || top_k > kRtMaxK || tokens > 0x7fffffff || stride >= ((size_t)1 << 28)) return TRV_ERR_UNSUPPORTED;
    return TRV_OK;
}

}  // namespace trv

using namespace trv;

extern "C" trv_status_t trv_router_workspace_bytes(size_t tokens, int32_t experts, size_t* bytes) {
    if (!bytes || experts < 1) return TRV_ERR_INVALID_ARG;
    *bytes = 0;
    if (experts > kRtMaxExperts || tokens > 0x7fffffff) return TRV_ERR_UNSUPPORTED;
    const size_t blocks = (size_t)rt_blocks(tokens, experts);
    *bytes = blocks == 1 ? 0 : blocks * (2 * (size_t)experts + 1) * 4;
    return TRV_OK;
}

extern "C" trv_status_t trv_router_forward(const void* logits, const uint8_t* mask, int32_t* ids, float* gates, int32_t* counts,
                                           float* prob_sum, size_t tokens, int32_t experts, int32_t top_k, size_t logits_stride,
                                           int32_t normalize, trv_dtype_t dtype, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const trv_status_t bad = router_check(tokens, experts, top_k, logits_stride, dtype);
    if (bad != TRV_OK) return bad;
    const size_t es = dtype_bytes(dtype), E = (size_t)experts, picks = tokens * (size_t)top_k * 4;
    if (!counts || !prob_sum || (tokens && (!logits || !ids || !gates))) return TRV_ERR_INVALID_ARG;
    if (misaligned(logits, es) || misaligned(ids, 4) || misaligned(gates, 4) || misaligned(counts, 4) || misaligned(prob_sum, 4))
        return TRV_ERR_INVALID_ARG;
    size_t need = 0;
    trv_router_workspace_bytes(tokens, experts, &need);
    if (need && (!workspace || misaligned(workspace, 256) || workspace_bytes < need)) return TRV_ERR_SCRATCH;
    const Span in[2] = {matrix_span(logits, tokens, E, logits_stride, es), {mask, tokens}};
    const Span out[5] = {{ids, picks}, {gates, picks}, {counts, (E + 1) * 4}, {prob_sum, E * 4}, {workspace, need}};
    if (!disjoint(in, out)) return TRV_ERR_INVALID_ARG;
    const int blocks = rt_blocks(tokens, experts);
    float* part_p = blocks == 1 ? prob_sum : (float*)workspace;
    int* part_c = blocks == 1 ? (int*)counts : (int*)workspace + (size_t)blocks * E;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    auto run = [&](auto zero) {
        RouterArgs<decltype(zero)> a = {};
        a.logits = (const decltype(zero)*)logits, a.mask = mask, a.tokens = (long long)tokens, a.ls = (long long)logits_stride, a.E = experts;
        a.k = top_k, a.normalize = normalize != 0, a.ids = ids, a.gates = gates, a.part_p = part_p, a.part_c = part_c;
        router_run(a, true, st);
    };
    if (dtype == TRV_FLOAT32) run(0.0f);
    else if (dtype == TRV_BFLOAT16) run(__nv_bfloat16());
    else run(__half());
    if (blocks > 1)
        launch_pdl(k_router_sum, dim3(experts / 8 + 1), dim3(kRtSumThreads), 0, st, (const float*)part_p, (const int*)part_c, blocks, (int)experts,
                   prob_sum, (int*)counts);
    g_last_kernel = "router_forward";
    return cudaGetLastError() == cudaSuccess ? TRV_OK : TRV_ERR_CUDA;
}

extern "C" trv_status_t trv_balance_loss(const int32_t* counts, const float* prob_sum, int32_t experts, int32_t top_k, float coef, float* loss,
                                         void* cuda_stream) {
    if (!counts || !prob_sum || !loss || experts < 1 || top_k < 1 || top_k > experts) return TRV_ERR_INVALID_ARG;
    if (misaligned(counts, 4) || misaligned(prob_sum, 4) || misaligned(loss, 4)) return TRV_ERR_INVALID_ARG;
    if (experts > kRtMaxExperts) return TRV_ERR_UNSUPPORTED;
    const Span in[2] = {{counts, ((size_t)experts + 1) * 4}, {prob_sum, (size_t)experts * 4}};
    const Span out[1] = {{loss, 4}};
    if (!disjoint(in, out)) return TRV_ERR_INVALID_ARG;
    TRV_LAUNCH(k_balance_loss, 1, kRtThreads, 0, (cudaStream_t)cuda_stream, counts, prob_sum, (int)experts, (int)top_k, coef, loss);
    g_last_kernel = "balance_loss";
    return cudaGetLastError() == cudaSuccess ? TRV_OK : TRV_ERR_CUDA;
}

extern "C" trv_status_t trv_router_backward(const void* logits, const uint8_t* mask, const int32_t* ids, const float* dgates,
                                            const int32_t* counts, void* dlogits, size_t tokens, int32_t experts, int32_t top_k,
                                            size_t logits_stride, size_t dlogits_stride, int32_t normalize, float coef, trv_dtype_t dtype,
                                            void* cuda_stream) {
    trv_status_t bad = router_check(tokens, experts, top_k, logits_stride, dtype);
    if (bad == TRV_OK) bad = router_check(tokens, experts, top_k, dlogits_stride, dtype);
    if (bad != TRV_OK) return bad;
    if (tokens == 0) return TRV_OK;
    if (!logits || !counts || !dlogits || (dgates && !ids)) return TRV_ERR_INVALID_ARG;
    const size_t es = dtype_bytes(dtype), E = (size_t)experts, picks = tokens * (size_t)top_k * 4;
    if (misaligned(logits, es) || misaligned(dlogits, es) || misaligned(ids, 4) || misaligned(dgates, 4) || misaligned(counts, 4))
        return TRV_ERR_INVALID_ARG;
    const Span in[5] = {matrix_span(logits, tokens, E, logits_stride, es), {mask, tokens}, {ids, dgates ? picks : 0}, {dgates, picks},
                        {counts, (E + 1) * 4}};
    const Span out[1] = {matrix_span(dlogits, tokens, E, dlogits_stride, es)};
    if (!disjoint(in, out)) return TRV_ERR_INVALID_ARG;
    auto run = [&](auto zero) {
        RouterArgs<decltype(zero)> a = {};
        a.logits = (const decltype(zero)*)logits, a.mask = mask, a.tokens = (long long)tokens, a.ls = (long long)logits_stride;
        a.ds = (long long)dlogits_stride, a.E = experts, a.k = top_k, a.normalize = normalize != 0, a.ids = (int*)ids, a.dgates = dgates;
        a.counts = counts, a.dlogits = (decltype(zero)*)dlogits, a.coef = coef;
        router_run(a, false, (cudaStream_t)cuda_stream);
    };
    if (dtype == TRV_FLOAT32) run(0.0f);
    else if (dtype == TRV_BFLOAT16) run(__nv_bfloat16());
    else run(__half());
    g_last_kernel = "router_backward";
    return cudaGetLastError() == cudaSuccess ? TRV_OK : TRV_ERR_CUDA;
}
