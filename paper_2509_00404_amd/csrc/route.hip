// Routing to experts: scores, selection, weights, their gradient, and the plan that sorts the choices into slots.
#include <type_traits>
#include "elementwise.h"

#define ROUTE_LANES 16                    // lanes that share a token: one row of the wave, inside which data moves without LDS
#define ROUTE_TOKENS 16                   // tokens of a workgroup
#define ROUTE_MAX_E 512
#define ROUTE_MAX_K 16

namespace {

// v of the lane N places on, around the row of 16
template <int N>
__device__ __forceinline__ uint32_t row_rotate(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N, 0xF, 0xF, true);
}
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
    uint32_t o;
    o = row_rotate<8>(v); v = v > o ? v : o;
    o = row_rotate<4>(v); v = v > o ? v : o;
    o = row_rotate<2>(v); v = v > o ? v : o;
    o = row_rotate<1>(v); return v > o ? v : o;
}
__device__ __forceinline__ float row_maxf(float v) {
    v = fmaxf(v, __uint_as_float(row_rotate<8>(__float_as_uint(v))));
    v = fmaxf(v, __uint_as_float(row_rotate<4>(__float_as_uint(v))));
    v = fmaxf(v, __uint_as_float(row_rotate<2>(__float_as_uint(v))));
    return fmaxf(v, __uint_as_float(row_rotate<1>(__float_as_uint(v))));
}
// every lane adds the same pairs in the same tree, so that all hold the same bits
__device__ __forceinline__ float row_sum(float v) {
    v += __uint_as_float(row_rotate<8>(__float_as_uint(v)));
    v += __uint_as_float(row_rotate<4>(__float_as_uint(v)));
    v += __uint_as_float(row_rotate<2>(__float_as_uint(v)));
    return v + __uint_as_float(row_rotate<1>(__float_as_uint(v)));
}

// Keys as unsigned numbers of the same order, all of them above 0, which stands for an expert that is not available.  -0 and +0 are one key.
__device__ __forceinline__ uint32_t order_key(float f) {
    const uint32_t u = __float_as_uint(f + 0.0f);
    return u ^ ((int32_t)u < 0 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t u) {
    return __uint_as_float(u ^ ((int32_t)u < 0 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ float sigmoid_f32(float x) { return 1.0f / (1.0f + expf(-x)); }

struct RouteArgs {
    int64_t T, ld;
    const float* bias;
    const uint8_t* valid;
    int32_t* idx;
    float* weights;
    int E, k, groups, top_groups, renorm;
    float scale;
    bool vec;                             // a lane's experts are all there or none, and their logits whole 16-byte units
};

// One row of 16 lanes per token; a lane has the keys of V neighbouring experts, in the experts' order.  A round of the selection is the
// highest key of the row and its lowest lane, which then looks for its next one.  With V > 4 the lane holds the highest of every four keys, and
// the keys themselves are in LDS, so that a round looks at four keys and V / 4 maxima instead of V keys.
// What bounds it: vector issue, two thirds of the clocks with the four waves a SIMD that 16384 tokens make, and between them the rounds' steps,
// which depend on one another.  16384 tokens, 256 experts in 8 groups, 8 choices: 14.4 us, of which the logits' 16.8 MB would take 3.3.  (All of a lane's keys looked at in every round, and every key's group by itself: 39.)
template <typename T, int V, bool SIGMOID>
__global__ void __launch_bounds__(ROUTE_LANES * ROUTE_TOKENS)
k_route(const T* __restrict__ logits, RouteArgs a) {
    constexpr int Q = V < 4 ? V : 4, NQ = V / Q;                           // keys of a quad, quads of a lane
    __shared__ __attribute__((aligned(16))) uint32_t s_key[ROUTE_TOKENS][ROUTE_LANES * V];
    __shared__ uint32_t s_group[ROUTE_TOKENS][ROUTE_LANES * V];
    __shared__ int s_idx[ROUTE_TOKENS][ROUTE_MAX_K];
    const int lane = threadIdx.x & (ROUTE_LANES - 1), tok = threadIdx.x / ROUTE_LANES;
    const int64_t t = (int64_t)blockIdx.x * ROUTE_TOKENS + tok;
    const bool row_there = t < a.T;
    const bool ok = row_there && (!a.valid || a.valid[t]);
    const T* row = logits + (row_there ? t : 0) * a.ld;
    uint32_t key[V];
    float x[V];
    const int e0 = lane * V;
    // (every lane has a line of its own, so that a load costs the same whether it takes 4 bytes or 16: 16384 x 256 fp32 with a bias 23 us by 4
    // bytes)
    bool loaded = false;
    if constexpr (V * sizeof(T) >= 16) {
        if (a.vec) {
            loaded = true;
            constexpr int N = 16 / (int)sizeof(T);
#pragma unroll
            for (int u = 0; u < V / N; ++u) {
                ew_u4 w = {0u, 0u, 0u, 0u};
                if (e0 < a.E) w = *reinterpret_cast<const ew_u4*>(row + e0 + N * u);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    x[N * u + i] = e0 >= a.E ? -INFINITY : N == 4 ? __uint_as_float(w[i & 3]) : i & 1 ? bf16hi_to_f32(w[i >> 1 & 3]) : bf16lo_to_f32(w[i >> 1 & 3]);
            }
        }
    }
    if (!loaded) {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = e0 + v < a.E ? load_one(row + e0 + v) : -INFINITY;
    }
    float add[V];
#pragma unroll
    for (int v = 0; v < V; ++v) add[v] = 0.0f;
    if (a.bias) {
        if (V >= 4 && a.vec) {
            if constexpr (V >= 4)
#pragma unroll
                for (int u = 0; u < V / 4; ++u) {
                    const ew_f4 w = *reinterpret_cast<const ew_f4*>(a.bias + (e0 < a.E ? e0 : 0) + 4 * u);
#pragma unroll
                    for (int i = 0; i < 4; ++i) add[4 * u + i] = w[i];
                }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) add[v] = a.bias[e0 + v < a.E ? e0 + v : 0];
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (!ok || !(x[v] > -INFINITY)) x[v] = -INFINITY;
        const float f = (SIGMOID ? sigmoid_f32(x[v]) : x[v]) + add[v];
        key[v] = x[v] > -INFINITY && f > -INFINITY ? order_key(f) : 0u;
    }
    // groups: the best of them by score, ties to the lowest; the keys of the others go
    if (a.top_groups < a.groups) {
        const int size = a.E / a.groups;
        const bool own = size % V == 0;                                    // a lane's keys are of one group
        uint32_t first = 0u, second = 0u;
        auto take = [&](uint32_t u) {
            const uint32_t low = u < first ? u : first;
            first = u > first ? u : first;
            second = low > second ? low : second;
        };
        if (own) {
#pragma unroll
            for (int v = 0; v < V; ++v) take(key[v]);
            s_key[tok][lane] = first;                                      // the lanes' best two
            if constexpr (V > 1) s_key[tok][ROUTE_LANES * V / 2 + lane] = second;
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) s_key[tok][e0 + v] = key[v];
        }
        __syncthreads();
        for (int g = lane; g < a.groups; g += ROUTE_LANES) {
            first = second = 0u;
            if (own) {
                for (int i = 0; i < size / V; ++i) {
                    take(s_key[tok][g * (size / V) + i]);
                    if constexpr (V > 1) take(s_key[tok][ROUTE_LANES * V / 2 + g * (size / V) + i]);
                }
            } else {
                for (int i = 0; i < size; ++i) take(s_key[tok][g * size + i]);
            }
            s_group[tok][g] = SIGMOID && second ? order_key(key_value(first) + key_value(second)) : first;
        }
        __syncthreads();
        // a group stays if fewer than top_groups come before it
        auto stays = [&](int g) {
            const uint32_t mine = s_group[tok][g];
            int before = 0;
            for (int h = 0; h < a.groups; ++h) {
                const uint32_t o = s_group[tok][h];
                before += o > mine || (o == mine && h < g);
            }
            return before < a.top_groups;
        };
        if (own) {
            if (e0 < a.E && !stays(e0 / size)) {
#pragma unroll
                for (int v = 0; v < V; ++v) key[v] = 0u;
            }
        } else {
            int g = e0 / size, left = size - (e0 - g * size);              // the keys' group, and how many of them are still of it
            bool keep = e0 < a.E && stays(g);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (left == 0) {
                    ++g;
                    left = size;
                    keep = e0 + v < a.E && stays(g);
                }
                key[v] = keep ? key[v] : 0u;
                --left;
            }
        }
        __syncthreads();
    }
    uint32_t high[NQ];                                                     // the highest of every quad
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        high[q] = key[Q * q];
#pragma unroll
        for (int i = 1; i < Q; ++i) high[q] = high[q] > key[Q * q + i] ? high[q] : key[Q * q + i];
        if constexpr (NQ > 1) *reinterpret_cast<ew_u4*>(&s_key[tok][e0 + Q * q]) = ew_u4{key[Q * q], key[Q * q + 1], key[Q * q + 2], key[Q * q + 3]};
    }
    const int shift = threadIdx.x & 48;
    for (int j = 0; j < a.k; ++j) {
        uint32_t best = high[0];
        int quad = 0;
#pragma unroll
        for (int q = 1; q < NQ; ++q) {
            quad = high[q] > best ? q : quad;
            best = high[q] > best ? high[q] : best;
        }
        const uint32_t top = row_max(best);
        const uint32_t mask = (uint32_t)(__ballot(best == top) >> shift) & 0xFFFFu;
        if (lane == __ffs(mask) - 1) {
            ew_u4 k4 = {0u, 0u, 0u, 0u};
            if constexpr (NQ > 1) {
                k4 = *reinterpret_cast<const ew_u4*>(&s_key[tok][e0 + Q * quad]);
            } else {
#pragma unroll
                for (int i = 0; i < Q; ++i) k4[i] = key[i];
            }
            int at = 0;
#pragma unroll
            for (int i = Q - 1; i >= 0; --i) at = k4[i] == top ? i : at;
            s_idx[tok][j] = top ? e0 + Q * quad + at : -1;
            uint32_t next = 0u;
#pragma unroll
            for (int i = 0; i < Q; ++i) {
                k4[i] = i == at ? 0u : k4[i];
                next = next > k4[i] ? next : k4[i];
            }
            if constexpr (NQ > 1) {
                s_key[tok][e0 + Q * quad + at] = 0u;
            } else {
#pragma unroll
                for (int i = 0; i < Q; ++i) key[i] = k4[i];
            }
#pragma unroll
            for (int q = 0; q < NQ; ++q) high[q] = q == quad ? next : high[q];
        }
    }
    __syncthreads();
    // one lane per choice from here on
    const int e = lane < a.k ? s_idx[tok][lane] : -1;
    const float xe = e >= 0 ? load_one(row + e) : -INFINITY;
    float w;
    if (SIGMOID) {
        w = e >= 0 ? sigmoid_f32(xe) : 0.0f;
        if (a.renorm) {
            const float sum = row_sum(w);
            w = sum > 0.0f ? w / sum : 0.0f;
        }
    } else {
        float top = xe, sum;
        if (a.renorm) {
            top = row_maxf(top);
            sum = row_sum(e >= 0 ? expf(xe - top) : 0.0f);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) top = fmaxf(top, x[v]);
            top = row_maxf(top);
            float part = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) part += x[v] > -INFINITY ? expf(x[v] - top) : 0.0f;
            sum = row_sum(part);
        }
        w = e >= 0 ? expf(xe - top) / sum : 0.0f;
    }
    if (row_there && lane < a.k) {
        a.idx[t * a.k + lane] = e;
        a.weights[t * a.k + lane] = e >= 0 ? a.scale * w : 0.0f;
    }
}

// ---- gradient of the logits ----
// As above, but a lane's experts are 16 apart: whole lines in and out.  A choice's part goes to its expert by way of LDS.  16384 x 64 fp32, dense:
// 4.8 us, of which the 8.9 MB would take 1.7; a launch's latency.
template <typename T, typename O, int V, bool SIGMOID>
__global__ void __launch_bounds__(ROUTE_LANES * ROUTE_TOKENS)
k_route_grads(const T* __restrict__ logits, int64_t ld, int64_t tokens, const int32_t* __restrict__ idx,
              const float* __restrict__ dweights, O* __restrict__ dlogits, int64_t ldd, int E, int k, int renorm, float scale) {
    __shared__ float s_dx[ROUTE_TOKENS][ROUTE_LANES * V];
    const int lane = threadIdx.x & (ROUTE_LANES - 1), tok = threadIdx.x / ROUTE_LANES;
    const int64_t t = (int64_t)blockIdx.x * ROUTE_TOKENS + tok;
    const bool there = t < tokens;
    const T* row = logits + (there ? t : 0) * ld;
    int e = there && lane < k ? idx[t * k + lane] : -1;
    const float xe = (uint32_t)e < (uint32_t)E ? load_one(row + e) : -INFINITY;
    if (!(xe > -INFINITY)) e = -1;
    const float v = e >= 0 ? scale * dweights[t * k + lane] : 0.0f;
    float x[V], p[V], d = 0.0f, inner = 0.0f;
    const bool dense = !SIGMOID && !renorm;
    if (SIGMOID) {
        const float s = e >= 0 ? sigmoid_f32(xe) : 0.0f;
        d = v;
        if (renorm) {
            const float z = row_sum(s), dot = row_sum(v * s);
            d = z > 0.0f ? (v - dot / z) / z : 0.0f;
        }
        d *= s * (1.0f - s);
    } else if (renorm) {
        const float top = row_maxf(xe);
        const float q0 = e >= 0 ? expf(xe - top) : 0.0f, sum = row_sum(q0);
        const float q = e >= 0 ? q0 / sum : 0.0f;
        d = q * (v - row_sum(v * q));
    } else {
        float top = -INFINITY, part = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int n = lane + ROUTE_LANES * i;
            x[i] = there && n < E ? load_one(row + n) : -INFINITY;
            top = fmaxf(top, x[i]);
        }
        top = row_maxf(top);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            p[i] = x[i] > -INFINITY ? expf(x[i] - top) : 0.0f;
            part += p[i];
        }
        const float sum = row_sum(part), inv = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] *= inv;
        inner = row_sum(e >= 0 ? v * (expf(xe - top) * inv) : 0.0f);
        d = v;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) s_dx[tok][lane + ROUTE_LANES * i] = 0.0f;
    __syncthreads();
    // the choices of a token one after the other: an expert that a caller lists twice gets both, in one order
    for (int j = 0; j < k; ++j) {
        if (lane == j && e >= 0) s_dx[tok][e] += d;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    if (!there) return;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int n = lane + ROUTE_LANES * i;
        if (n >= E) continue;
        const float g = s_dx[tok][n];
        store_one(dlogits + t * ldd + n, dense ? p[i] * (g - inner) : g);
    }
}

// ---- the plan: a stable counting sort of the choices by expert ----
// The choices are cut into chunks.  With several chunks a first launch counts each chunk's choices of every expert; then every workgroup
// adds up the counts of the chunks before its own, so that no launch is spent on a scan.  Up to PLAN_ALONE choices one workgroup does all of
// it, which costs it about a microsecond per 1024 and saves a launch of four.
// 131072 choices of 256 experts: 2.8 us for the counts and 7.8 for the rest, latency of its steps (waves wait 0.63 of their time; one thread per expert adding up the
// counts, and chunks of 2048: 21).
#define PLAN_THREADS 1024
#define PLAN_WAVES (PLAN_THREADS / METIS_WAVE)
#define PLAN_MAX_CHUNKS 128
#define PLAN_ALONE 4096

int64_t plan_chunk(int64_t S) {
    if (S <= PLAN_ALONE) return PLAN_ALONE;
    return (S + PLAN_MAX_CHUNKS * PLAN_THREADS - 1) / (PLAN_MAX_CHUNKS * PLAN_THREADS) * PLAN_THREADS;
}

__global__ void __launch_bounds__(PLAN_THREADS)
k_plan_count(const int32_t* __restrict__ idx, int64_t S, int64_t chunk, int E, int32_t* __restrict__ counts) {
    __shared__ int32_t s_count[ROUTE_MAX_E];
    for (int e = threadIdx.x; e < E; e += PLAN_THREADS) s_count[e] = 0;
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * chunk, to = from + chunk < S ? from + chunk : S;
    for (int64_t i = from + threadIdx.x; i < to; i += PLAN_THREADS) {
        const int e = idx[i];
        if ((uint32_t)e < (uint32_t)E) atomicAdd(&s_count[e], 1);         // whole numbers: the order does not matter
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += PLAN_THREADS) counts[(int64_t)blockIdx.x * E + e] = s_count[e];
}

__global__ void __launch_bounds__(PLAN_THREADS)
k_plan(const int32_t* __restrict__ idx, int64_t S, FastDiv by_k, int64_t chunk, int E, const int32_t* __restrict__ counts,
       int32_t* __restrict__ offsets, int32_t* __restrict__ token, int32_t* __restrict__ slot) {
    __shared__ int32_t s_next[ROUTE_MAX_E];                               // the next slot of every expert
    __shared__ int32_t s_wave[PLAN_WAVES][ROUTE_MAX_E];                   // counts of a wave's 64 choices, then their first slots
    __shared__ int32_t s_before[ROUTE_MAX_E], s_all[ROUTE_MAX_E];
    __shared__ int32_t s_sum[PLAN_WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nchunks = (int)gridDim.x;
    const int64_t from = (int64_t)blockIdx.x * chunk, to = from + chunk < S ? from + chunk : S;
    if (tid < E) s_before[tid] = s_all[tid] = 0;
    __syncthreads();
    if (counts) {
        // the threads share an expert's chunks: as many parts as there are threads for
        const int parts = PLAN_THREADS / E, e = tid % E, part = tid / E;
        if (part < parts) {
            int32_t before = 0, all = 0;
#pragma unroll 8
            for (int c = part; c < nchunks; c += parts) {
                const int32_t n = counts[(int64_t)c * E + e];
                before += c < (int)blockIdx.x ? n : 0;
                all += n;
            }
            atomicAdd(&s_before[e], before);
            atomicAdd(&s_all[e], all);
        }
    } else {
        for (int64_t i = from + tid; i < to; i += PLAN_THREADS) {
            const int e = idx[i];
            if ((uint32_t)e < (uint32_t)E) atomicAdd(&s_all[e], 1);
        }
    }
    __syncthreads();
    const int32_t mine = tid < E ? s_all[tid] : 0;
    int32_t upto = mine;                                                   // inclusive scan over the experts
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 63) s_sum[wave] = upto;
    __syncthreads();
    int32_t total = 0;
    for (int w = 0; w < ROUTE_MAX_E / 64; ++w) {
        upto += w < wave ? s_sum[w] : 0;
        total += s_sum[w];
    }
    if (tid < E) {
        s_next[tid] = upto - mine + s_before[tid];
        if (blockIdx.x == 0) offsets[tid + 1] = upto;
    }
    if (blockIdx.x == 0 && tid == 0) offsets[0] = 0;
    // slots that serve no choice
    for (int64_t i = total + (int64_t)blockIdx.x * PLAN_THREADS + tid; i < S; i += (int64_t)nchunks * PLAN_THREADS) token[i] = -1;
    for (int64_t base = from; base < to; base += PLAN_THREADS) {
        const int64_t i = base + tid;
        const int e = i < to ? idx[i] : -1;
        const bool there = (uint32_t)e < (uint32_t)E;
        for (int n = lane; n < E; n += 64) s_wave[wave][n] = 0;
        // the lanes of the wave that chose the same expert
        uint64_t same = __ballot(there);
        for (int b = 1; b < E; b *= 2) {
            const uint64_t m = __ballot(there && (e & b));
            same &= e & b ? m : ~m;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        if (there && rank == 0) s_wave[wave][e] = __popcll(same);
        __syncthreads();
        if (tid < E) {
            int32_t n = s_next[tid], c[PLAN_WAVES];
#pragma unroll
            for (int w = 0; w < PLAN_WAVES; ++w) c[w] = s_wave[w][tid];
#pragma unroll
            for (int w = 0; w < PLAN_WAVES; ++w) {
                s_wave[w][tid] = n;
                n += c[w];
            }
            s_next[tid] = n;
        }
        __syncthreads();
        if (i < to) {
            const int32_t at = there ? s_wave[wave][e] + rank : -1;
            slot[i] = at;
            if (there) token[at] = (int32_t)div_by(by_k, (uint64_t)i);
        }
    }
}

int router_status(const metis_mat* logits, const metis_router* r) {
    if (!logits || !r || (!logits->ptr && logits->rows > 0)) return METIS_INVALID_ARG;
    if (logits->dtype != METIS_BF16 && logits->dtype != METIS_F32) return METIS_INVALID_ARG;
    if (r->scores != METIS_SCORES_SOFTMAX && r->scores != METIS_SCORES_SIGMOID) return METIS_INVALID_ARG;
    if (r->experts < 1 || r->k < 1) return METIS_INVALID_ARG;
    if (r->experts > ROUTE_MAX_E || r->k > ROUTE_MAX_K) return METIS_UNSUPPORTED;
    if (logits->rows < 0 || logits->cols != r->experts || logits->ld < logits->cols) return METIS_BAD_SHAPE;
    if (logits->rows > 0x7FFFFFFFll / r->k) return METIS_BAD_SHAPE;
    if (!grid_fits(ceil_div64(logits->rows, ROUTE_TOKENS), ROUTE_LANES * ROUTE_TOKENS)) return METIS_UNSUPPORTED;
    return METIS_OK;
}

// f(integral constant of the keys a lane holds)
template <typename F>
int by_keys(int E, const F& f) {
    const int v = (E + ROUTE_LANES - 1) / ROUTE_LANES;
    if (v <= 1) return f(std::integral_constant<int, 1>{});
    if (v <= 2) return f(std::integral_constant<int, 2>{});
    if (v <= 4) return f(std::integral_constant<int, 4>{});
    if (v <= 8) return f(std::integral_constant<int, 8>{});
    if (v <= 16) return f(std::integral_constant<int, 16>{});
    return f(std::integral_constant<int, 32>{});
}

template <typename T>
int launch_route(hipStream_t s, const metis_mat* logits, const metis_router* r, const RouteArgs& a) {
    return by_keys(r->experts, [&](auto v) -> int {
        constexpr int V = decltype(v)::value;
        const dim3 grid((unsigned)ceil_div64(a.T, ROUTE_TOKENS)), block(ROUTE_LANES * ROUTE_TOKENS);
        if (r->scores == METIS_SCORES_SIGMOID) hipLaunchKernelGGL((k_route<T, V, true>), grid, block, 0, s, (const T*)logits->ptr, a);
        else hipLaunchKernelGGL((k_route<T, V, false>), grid, block, 0, s, (const T*)logits->ptr, a);
        METIS_LAUNCH_CHECK();
        return METIS_OK;
    });
}

template <typename T, typename O>
int launch_route_grads(hipStream_t s, const metis_mat* logits, const metis_router* r, const int32_t* idx, const float* dw, metis_mat* d) {
    return by_keys(r->experts, [&](auto v) -> int {
        constexpr int V = decltype(v)::value;
        const dim3 grid((unsigned)ceil_div64(logits->rows, ROUTE_TOKENS)), block(ROUTE_LANES * ROUTE_TOKENS);
        auto kern = r->scores == METIS_SCORES_SIGMOID ? k_route_grads<T, O, V, true> : k_route_grads<T, O, V, false>;
        hipLaunchKernelGGL(kern, grid, block, 0, s, (const T*)logits->ptr, logits->ld, logits->rows, idx, dw, (O*)d->ptr, d->ld,
                           r->experts, r->k, r->renorm, r->scale);
        METIS_LAUNCH_CHECK();
        return METIS_OK;
    });
}

}  // namespace

extern "C" int metis_route(void* stream, const metis_mat* logits, const metis_router* r, const float* bias, const uint8_t* valid,
                           int32_t* idx, float* weights) {
    const int st = router_status(logits, r);
    if (st != METIS_OK) return st;
    if (r->groups < 1 || r->experts % r->groups || r->top_groups < 1 || r->top_groups > r->groups ||
        r->k > r->top_groups * (r->experts / r->groups))
        return METIS_INVALID_ARG;
    if (logits->rows == 0) return METIS_OK;
    if (!idx || !weights) return METIS_INVALID_ARG;
    int held = 1;                                                          // experts a lane has
    while (held * ROUTE_LANES < r->experts) held *= 2;
    const RouteArgs a = {logits->rows, logits->ld, bias, valid, idx, weights, r->experts, r->k, r->groups, r->top_groups, r->renorm, r->scale,
                         r->experts % held == 0 && mat_aligned16(logits) && (uintptr_t)bias % 16 == 0};
    return logits->dtype == METIS_BF16 ? launch_route<bf16_t>((hipStream_t)stream, logits, r, a)
                                       : launch_route<float>((hipStream_t)stream, logits, r, a);
}

extern "C" int metis_route_grads(void* stream, const metis_mat* logits, const metis_router* r, const int32_t* idx, const float* dweights,
                                 metis_mat* dlogits) {
    const int st = router_status(logits, r);
    if (st != METIS_OK) return st;
    if (!dlogits || (dlogits->dtype != METIS_BF16 && dlogits->dtype != METIS_F32)) return METIS_INVALID_ARG;
    if (dlogits->rows != logits->rows || dlogits->cols != logits->cols || dlogits->ld < dlogits->cols) return METIS_BAD_SHAPE;
    if (logits->rows == 0) return METIS_OK;
    if (!dlogits->ptr || !idx || !dweights) return METIS_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    const bool bf_in = logits->dtype == METIS_BF16, bf_out = dlogits->dtype == METIS_BF16;
    if (bf_in) return bf_out ? launch_route_grads<bf16_t, bf16_t>(s, logits, r, idx, dweights, dlogits)
                             : launch_route_grads<bf16_t, float>(s, logits, r, idx, dweights, dlogits);
    return bf_out ? launch_route_grads<float, bf16_t>(s, logits, r, idx, dweights, dlogits)
                  : launch_route_grads<float, float>(s, logits, r, idx, dweights, dlogits);
}

extern "C" size_t metis_dispatch_workspace_bytes(int64_t tokens, int experts, int k) {
    if (tokens < 1 || experts < 1 || k < 1 || experts > ROUTE_MAX_E || k > ROUTE_MAX_K || tokens > 0x7FFFFFFFll / k) return 0;
    const int64_t S = tokens * k, chunks = ceil_div64(S, plan_chunk(S));
    return chunks > 1 ? (size_t)chunks * experts * sizeof(int32_t) : 0;
}

extern "C" int metis_dispatch(void* stream, const int32_t* idx, metis_expert_plan* plan, void* workspace, size_t workspace_bytes) {
    if (!plan || !plan->offsets || plan->tokens < 0 || plan->experts < 1 || plan->k < 1) return METIS_INVALID_ARG;
    if (plan->experts > ROUTE_MAX_E || plan->k > ROUTE_MAX_K) return METIS_UNSUPPORTED;
    if (plan->tokens > 0x7FFFFFFFll / plan->k) return METIS_BAD_SHAPE;
    const int64_t S = plan->tokens * plan->k;
    if (S > 0 && (!idx || !plan->token || !plan->slot)) return METIS_INVALID_ARG;
    const int64_t chunk = plan_chunk(S), chunks = S > 0 ? ceil_div64(S, chunk) : 1;
    const size_t need = metis_dispatch_workspace_bytes(plan->tokens, plan->experts, plan->k);
    if (workspace_bytes < need || (need && !workspace)) return METIS_WORKSPACE_TOO_SMALL;
    if (need && (uintptr_t)workspace % 16) return METIS_INVALID_ARG;
    int32_t* counts = need ? (int32_t*)workspace : nullptr;
    hipStream_t s = (hipStream_t)stream;
    if (counts) {
        hipLaunchKernelGGL(k_plan_count, dim3((unsigned)chunks), dim3(PLAN_THREADS), 0, s, idx, S, chunk, plan->experts, counts);
        METIS_LAUNCH_CHECK();
    }
    hipLaunchKernelGGL(k_plan, dim3((unsigned)chunks), dim3(PLAN_THREADS), 0, s, idx, S, fast_div((uint32_t)plan->k), chunk, plan->experts, counts,
                       plan->offsets, plan->token, plan->slot);
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}
