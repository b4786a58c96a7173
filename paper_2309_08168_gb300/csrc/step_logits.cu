// step_logits.cu - penalties, biases and masks on logits, and the choice of the
// best tokens of every row (ssd_logits_adjust, ssd_logits_choose of ssd_step.h).
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <mutex>
#include <type_traits>

#include "step_ops.cuh"

namespace ssd {
namespace step {

constexpr int kLogitThreads = 256, kLogitWarps = kLogitThreads / 32;
constexpr int kMaxVocab = 262144;
constexpr int kMaxSlice = 131136;  // tokens of a CTA: at most 65 chunks of 8 in each of its threads
constexpr int kFew = 8;            // a mask that leaves one token of so many is taken as a list
constexpr int kMaxListed = 65472;  // tokens of a CTA whose places a list can hold in 16 bits
constexpr int kMaxSplit = 8;      // CTAs of a row: one portable cluster
constexpr int kMaxBest = 16;
constexpr int kJoinWarps = kMaxSplit * kMaxBest / 32;
constexpr uint32_t kPrompt = 0x80000000u;  // a token's count: times that the model said it, and this bit if the prompt holds it

struct LogitArgs {
    ssd_logit_rules r;
    const void* logits;
    void* out;  // adjust
    int64_t stride, out_stride;
    int32_t* tokens;  // choose
    float *logprob, *total;
    int k, slice, rows;  // tokens of a CTA (a multiple of 64), rows of a cluster
    int counted;         // whether anything is penalised
    // dynamic shared memory: candidates of the k best, words of the row's mask from at_show on, the
    // tokens that a mask of few leaves from at_list on, and from at_bits on what has been
    // said: n_words words of bits, the bits before each four of them, counts
    int at_show, at_list, at_bits, n_words;
};

// what a float sorts by; 0 is below all of them (-inf gives 0x007fffff)
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t u = __float_as_uint(v);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_order(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
// (logit, token) as one number: larger logits first, of equal ones the lower token; 0 is none
__device__ __forceinline__ uint64_t key_of(float v, int x) { return (uint64_t)order_of(v) << 32 | (uint32_t)~x; }

__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f;
// exp(v - m) for v <= m, 1 for v = m = inf
__device__ __forceinline__ float weight(float v, float m) { return v == m ? 1.f : exp2_of((v - m) * kLog2e); }
__device__ __forceinline__ void copy4(void* to, const void* from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;\n" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;\n" ::: "memory"); }
// what the CTAs of a row hand to the one that joins them
struct Partial {
    uint64_t sum;  // (maximum, sum of weights) as floats
    uint64_t best[kMaxBest];
};

// 8 tokens' logits as they lie in memory
template <typename T>
struct Chunk {
    static constexpr int V = Vec<T>::N;
    uint4 u[8 / V];
    __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
        for (int i = 0; i < 8 / V; ++i) {
            float g[V];
            Vec<T>::get(u[i], g);
#pragma unroll
            for (int j = 0; j < V; ++j) f[V * i + j] = g[j];
        }
    }
    __device__ __forceinline__ void put(const float (&f)[8]) {
#pragma unroll
        for (int i = 0; i < 8 / V; ++i) {
            float g[V];
#pragma unroll
            for (int j = 0; j < V; ++j) g[j] = f[V * i + j];
            u[i] = Vec<T>::put(g);
        }
    }
};

// A row's tokens are cut into slices of a CTA each (a cluster joins them), those into chunks of 8 that start on
// 16 bytes of the logits (how far the row's first one lies before its first token depends on the row), chunk j in thread j mod 256.
//
// What a text has said is worked out once for the rows of one request that a cluster takes, for the CTA's
// slice alone: a bit for every token that the history or some node of the round says, and a count for each of these bits
// (found by the number of bits before it).  A row's nodes are added to the counts before the row and taken off after it.
//
// The k best: each thread keeps its own best; the k-th largest of these is a bound that at least k tokens reach, and only
// tokens of the k threads above it can be among the k best.  Their chunks are read once more (from L2), what reaches the bound is
// ranked by counting, and ranks below k are the answer.  All keys differ (the token is part of them), so ties need no care.
//
// The pass is bound by the instructions it issues (8 fp16 tokens: 8 conversions, 8 exponentials, a maximum, and two in one where the
// chip has it), so a thread keeps its best chunk rather than its best token, and sums weights relative to a whole number above its
// best, which seldom changes.
//
// kRules: 0: the rules have no part; 1: no biases; 2: biases; 3: biases that do not lie on 16 bytes where the logits do.  (With the code for biases in it, though none are added, 456 rows of 128256 take
// 55 us instead of 42 where texts are penalised.  207 bf16 rows of 50257 with biases, eight best: 28.0 us; biases as eight floats each through L1
// 29.0; in 3 with two chunks under way, which spills, 30.0.)
//
// kCtas of an SM at most.  With biases three of them leave 80 registers, which spills; where two are enough for all of the work, they are faster
// (64 rows of 128256, all rules: 28.5 us, two 21.6; 512 rows 90, two 92; 200 rows 47, two 56).
constexpr int ctas_of(bool choose, int rules) { return choose && rules ? 3 : 4; }
template <typename T, bool kChoose, int kRules, int kCtas = ctas_of(kChoose, kRules)>
__global__ void __launch_bounds__(kLogitThreads, kCtas) logits_kernel(const __grid_constant__ LogitArgs a) {
    constexpr int V = Vec<T>::N;  // tokens in 16 bytes
    constexpr int kParts = 8 / V, kAdds = kRules == 3 ? 3 : 2;
    // chunks under way in a thread, as many as registers hold (adjusting 294 bf16 rows of 151936, penalised and masked: 2 43.0 us, 3 41.0, 4 41.5; fp32 rows
    // 59.7, 61.5, 64.1; with biases 51.7, 51.8, 55.7)
    constexpr int kAhead = kRules == 3 && kCtas > 2 ? 1 : kRules >= 2 ? 2 : kRules && !kChoose ? V == 8 ? 3 : 2 : V / 2;
    extern __shared__ __align__(16) unsigned char s_dyn[];
    __shared__ int s_request, s_rows[2], s_n, s_scan[kLogitWarps];
    __shared__ float s_m[kLogitWarps], s_s[kLogitWarps];
    __shared__ uint64_t s_first[kLogitWarps * kMaxBest], s_bound;
    __shared__ int s_from[kMaxBest], s_found;
    __shared__ Partial s_part[2];
    uint64_t* s_cand = reinterpret_cast<uint64_t*>(s_dyn);
    uint32_t* s_show = reinterpret_cast<uint32_t*>(s_dyn + a.at_show);
    uint16_t* s_list = reinterpret_cast<uint16_t*>(s_dyn + a.at_list);
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, split = gridDim.x, vocab = a.r.vocab;
    const int lo = blockIdx.x * a.slice, deep = (a.slice / 8 + kLogitThreads - 1) / kLogitThreads;  // chunks of a thread
    const int row0 = blockIdx.y * a.rows, row1 = min(row0 + a.rows, a.r.n_rows);

    // -- what has been said of tokens lo - 8 .. lo + slice - 1 (chunks may start up to 7 tokens before the slice)
    const int n_words = a.n_words;
    uint32_t *s_bits = reinterpret_cast<uint32_t*>(s_dyn + a.at_bits), *s_before = s_bits + n_words, *s_count = s_before + n_words / 4;
    auto place = [&](int x) { return x >= 0 && x < vocab && x >= lo - 8 && x < lo + a.slice ? x - lo + 8 : -1; };
    const uint4* fours = reinterpret_cast<const uint4*>(s_bits);
    auto count_of = [&](int i) {  // bits before bit i
        const uint4 u = fours[i / 128];
        const int r = i / 32 % 4;
        const uint32_t below = (1u << i % 32) - 1u;
        return s_before[i / 128] + __popc(r > 0 ? u.x : u.x & below) + (r > 0 ? __popc(r > 1 ? u.y : u.y & below) : 0) +
               (r > 1 ? __popc(r > 2 ? u.z : u.z & below) : 0) + (r > 2 ? __popc(u.w & below) : 0);
    };
    int said = 0, prompt = 0;  // tokens of the request's history, those of them that are the prompt's
    // history tokens, several loads at once; f(token's place, whether it is the prompt's)
    auto history = [&](int b, auto&& f) {
        const int n = min(max(said, 0), a.r.max_history);
        const int32_t* h = a.r.history + (int64_t)b * a.r.history_stride;
        for (int j = tid; j < n; j += 8 * kLogitThreads) {
            int x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = j + i * kLogitThreads < n ? __ldcg(h + j + i * kLogitThreads) : -1;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int p = place(x[i]);
                if (p >= 0) f(p, j + i * kLogitThreads < prompt);
            }
        }
    };
    int request = -1, start = 0, end = 0;  // of the row before
    int old = -1;                          // the row whose nodes are in the counts
    auto reach = [&]() { return a.r.masks ? min(end - start, 64 * a.r.mask_words) : end - start; };
    auto nodes = [&](int row, uint32_t more) {  // more to the counts of the nodes that a row's mask shows
        const int n = a.r.masks ? reach() : row - start + 1;
        for (int j = tid; j < n; j += kLogitThreads) {
            const bool seen = !a.r.masks || (__ldcg(reinterpret_cast<const unsigned long long*>(a.r.masks) + (int64_t)row * a.r.mask_words + j / 64) >> (j % 64) & 1);
            const int p = seen ? place(__ldcg(a.r.tokens + start + j)) : -1;
            if (p >= 0) atomicAdd(s_count + count_of(p), more);
        }
    };
    float again = 1.f, often = 0.f, once = 0.f;
    const float* bias = nullptr;  // of the row's request

    int turn = 0;  // which of the two parts
    for (int row = row0; row < row1; ++row) {
        // the request that owns the row
        if (!a.r.row_start) start = row, end = row + 1;
        const bool fresh = !a.r.row_start || row >= end;
        int owner = request;
        if (a.r.row_start && fresh && !a.counted && !a.r.bias_of) {  // (whose it is does not matter)
            const int s0 = __ldcg(a.r.row_start), s1 = __ldcg(a.r.row_start + a.r.n_requests);
            owner = s0 <= row && row < s1 ? 0 : a.r.n_requests;
            end = row + 1;
        } else if (a.r.row_start && fresh && a.r.n_requests == a.r.n_rows && __ldcg(a.r.row_start + row) == row && __ldcg(a.r.row_start + row + 1) == row + 1) {
            owner = start = row, end = row + 1;  // (a row a request: no search)
        } else if (a.r.row_start && fresh) {
            if (tid == 0) s_request = a.r.n_requests;
            __syncthreads();
            for (int b = tid; b < a.r.n_requests; b += kLogitThreads) {
                const Rows r = rows_of(a.r.row_start, b, a.r.n_rows);
                if (r.r0 <= row && row < r.r0 + r.n) atomicMin(&s_request, b);
            }
            __syncthreads();
            owner = s_request;
            if (owner < a.r.n_requests && tid == owner % kLogitThreads) {
                const Rows r = rows_of(a.r.row_start, owner, a.r.n_rows);
                s_rows[0] = r.r0, s_rows[1] = r.r0 + r.n;
            }
            __syncthreads();
            start = owner < a.r.n_requests ? s_rows[0] : row;  // (else no one's)
            end = owner < a.r.n_requests ? s_rows[1] : row + 1;
        } else if (fresh) {
            owner = row;
        }
        request = owner;
        if (owner >= a.r.n_requests) {  // (uniform over the cluster: its CTAs have the same rows)
            continue;
        }
        const T* src = (const T*)a.logits + (int64_t)row * a.stride;
        const int first = lo - (int)(((uintptr_t)src & 15u) / sizeof(T)), stop = min(first + a.slice, vocab);  // this CTA's tokens: [max(first, 0), stop)
        auto inside = [&](int x) { return x >= 0 && x < vocab; };
        auto whole = [&](int x) { return x >= 0 && x + 8 <= vocab; };
        auto load = [&](int x0, Chunk<T>& c) {  // (what is outside the row is -inf)
            if (whole(x0)) {
#pragma unroll
                for (int i = 0; i < kParts; ++i) c.u[i] = __ldcg(reinterpret_cast<const uint4*>(src + x0) + i);
            } else {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = inside(x0 + i) ? (float)src[x0 + i] : -INFINITY;
                c.put(f);
            }
        };
        // what the row and its request have, asked for at once
        if (kRules && fresh) {
            const int b = a.r.bias_of ? __ldcg(a.r.bias_of + owner) : 0;
            if (a.counted) {
                again = a.r.repetition ? __ldcg(a.r.repetition + owner) : 1.f;
                often = a.r.frequency ? __ldcg(a.r.frequency + owner) : 0.f;
                once = a.r.presence ? __ldcg(a.r.presence + owner) : 0.f;
                said = a.r.history ? __ldcg(a.r.history_len + owner) : 0;
                prompt = a.r.prompt_len ? __ldcg(a.r.prompt_len + owner) : 0;
            }
            bias = a.r.bias && b >= 0 && b < a.r.n_bias ? a.r.bias + (int64_t)b * a.r.bias_stride : nullptr;
        }
        const uint32_t* allowed = nullptr;
        if (kRules && a.r.allowed) {
            const int m = a.r.allowed_of ? __ldcg(a.r.allowed_of + row) : row;
            if (m >= 0 && m < a.r.n_allowed) allowed = a.r.allowed + (int64_t)m * a.r.allowed_stride;
        }
        // (from the word on that holds token lo - 8; what lies before the row's first word is not there)
        const int word0 = (lo - 8) >> 5;
        if (allowed) {
            for (int i = max(word0, 0) + tid; i <= (stop - 1) / 32; i += kLogitThreads) copy4(s_show + i - word0, allowed + i);
        }
        if (kRules && a.counted && fresh) {
            __syncthreads();  // (the counts of the row before are no longer read)
            for (int i = tid; i < n_words; i += kLogitThreads) s_bits[i] = 0u;
            old = -1;
            __syncthreads();
            if (a.r.history) history(owner, [&](int p, bool) { atomicOr(s_bits + p / 32, 1u << p % 32); });
            if (a.r.tokens)
                for (int j = tid; j < reach(); j += kLogitThreads) {
                    const int p = place(__ldcg(a.r.tokens + start + j));
                    if (p >= 0) atomicOr(s_bits + p / 32, 1u << p % 32);
                }
            __syncthreads();
            // bits before each four words: each thread's words, then the threads'
            const int n_fours = n_words / 4, each = (n_fours + kLogitThreads - 1) / kLogitThreads, w0 = min(tid * each, n_fours), w1 = min(w0 + each, n_fours);
            auto bits_of = [&](int w) {
                const uint4 u = fours[w];
                return __popc(u.x) + __popc(u.y) + __popc(u.z) + __popc(u.w);
            };
            int mine = 0;
            for (int w = w0; w < w1; ++w) mine += bits_of(w);
            int upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int v = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += v;
            }
            if (lane == 31) s_scan[warp] = upto;
            __syncthreads();
            int at = upto - mine, all = 0;
            for (int w = 0; w < kLogitWarps; ++w) {
                if (w < warp) at += s_scan[w];
                all += s_scan[w];
            }
            for (int w = w0; w < w1; ++w) {
                s_before[w] = (uint32_t)at;
                at += bits_of(w);
            }
            for (int i = tid; i < all; i += kLogitThreads) s_count[i] = 0u;
            __syncthreads();
            if (a.r.history)
                history(owner, [&](int p, bool prompt) {
                    if (prompt) atomicOr(s_count + count_of(p), kPrompt);
                    else atomicAdd(s_count + count_of(p), 1u);
                });
        }
        if (kRules && a.counted && a.r.tokens) {
            __syncthreads();  // (history counted; the row before read)
            if (old >= 0) nodes(old, ~0u);
            nodes(row, 1u);
            old = row;
        }
        if (allowed) copies_wait();
        if (a.counted || allowed) __syncthreads();
        auto bits8 = [&](const uint32_t* w, int x) -> uint32_t {  // bits x .. x + 7 (of the next word, too, which is always there)
            return __funnelshift_r(w[x / 32u], w[x / 32u + 1], x % 32u) & 255u;
        };
        // the 8 bits of a chunk's tokens in the row's mask; 0: nothing of it is left
        auto shown = [&](int x0) -> uint32_t { return allowed ? bits8(s_show, x0 - 32 * word0) : 255u; };
        // A chunk's biases are the 8 floats from number `shift` on of the 12 in add (rules 3: aligned loads, and the same shift for all of the row)
        const int shift = kRules == 3 && bias ? (int)(((uintptr_t)bias / 4 + (uintptr_t)(intptr_t)first) & 3u) : 0;
        auto load_bias = [&](int x, float4 (&add)[kAdds]) {
            if (kRules < 2 || !bias) return;
            if (kRules == 2 ? whole(x) && ((uintptr_t)(bias + x) & 15u) == 0 : x >= shift && x - shift + 12 <= vocab) {
#pragma unroll
                for (int i = 0; i < kAdds; ++i) add[i] = __ldcg(reinterpret_cast<const float4*>(bias + x - shift) + i);
            } else {
                float v[4 * kAdds];
#pragma unroll
                for (int j = 0; j < 4 * kAdds; ++j) {
                    const bool there = j >= shift && j < shift + 8 && inside(x + j - shift);
                    v[j] = there ? bias[x + j - shift] : 0.f;
                }
#pragma unroll
                for (int i = 0; i < kAdds; ++i) add[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            }
        };
        auto penalised = [&](float l, uint32_t n) {
            const uint32_t c = n & ~kPrompt;
            l = __fsub_rn(l > 0.f ? __fdiv_rn(l, again) : __fmul_rn(l, again), __fmul_rn(often, (float)c));
            return c ? __fsub_rn(l, once) : l;
        };
        auto rules = [&](int x0, uint32_t show, const float4 (&add)[kAdds], float (&f)[8]) {
            if (a.counted) {
                const int at = x0 - lo + 8;  // >= 0
                const uint32_t m = bits8(s_bits, at);
                if (m) {
                    const uint32_t* counts = s_count + count_of(at);  // of the chunk's said tokens, one behind the other
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t n = m >> j & 1u ? counts[__popc(m & ((1u << j) - 1u))] : 0u;
                        if (n) f[j] = penalised(f[j], n);  // (0: not said, or by another node only)
                    }
                }
            }
            if (kRules >= 2 && bias) {
                float v[4 * kAdds];
#pragma unroll
                for (int i = 0; i < kAdds; ++i) v[4 * i] = add[i].x, v[4 * i + 1] = add[i].y, v[4 * i + 2] = add[i].z, v[4 * i + 3] = add[i].w;
                auto plus = [&](auto from) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] += v[(j + decltype(from)::value) % (4 * kAdds)];
                };
                if (kRules == 2 || shift == 0) plus(std::integral_constant<int, 0>());
                else if (shift == 1) plus(std::integral_constant<int, 1>());
                else if (shift == 2) plus(std::integral_constant<int, 2>());
                else plus(std::integral_constant<int, 3>());
            }
            if (show != 255u) {
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = show >> j & 1u ? f[j] : -INFINITY;
            }
        };
        // A mask that leaves at most 1 / kFew of the slice: its tokens in order, so that only they are read (`few` of them; -1: more).  512 rows
        // of 128256 with penalties and biases, 64 masks, one of ten in [1/16, 1/8]: 90.0 us; at 1/16 93.8, at 1/4 97.7, for five best 130 (a list of 32 KB takes a CTA's place).
        int few = -1;
        if (kChoose && kRules && allowed) {
            const int low = max(first, 0), n = (stop - 1) / 32 - word0 + 1;
            const int each = (n + kLogitThreads - 1) / kLogitThreads | 1;  // (odd: threads meet different banks)
            const int w0 = min(tid * each, n), w1 = min(w0 + each, n);
            auto word = [&](int w) {  // bits of [low, stop)
                const int x = 32 * (word0 + w);
                uint32_t u = s_show[w];
                if (x < low) u = x + 32 <= low ? 0u : u & ~0u << (low - x);
                return x + 32 > stop ? u & ~0u >> (x + 32 - stop) : u;
            };
            int mine = 0;
            for (int w = w0; w < w1; ++w) mine += __popc(word(w));
            int upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int v = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += v;
            }
            if (lane == 31) s_scan[warp] = upto;
            __syncthreads();
            int to = upto - mine, all = 0;
            for (int w = 0; w < kLogitWarps; ++w) {
                if (w < warp) to += s_scan[w];
                all += s_scan[w];
            }
            if (all * kFew <= a.slice) {
                few = all;
                for (int w = w0; w < w1; ++w)
                    for (uint32_t u = word(w); u; u &= u - 1) s_list[to++] = (uint16_t)(32 * (word0 + w) + __ffs((int)u) - 1 - (lo - 8));
            }
            __syncthreads();
        }
        // the logit l of a token that the mask leaves after the other rules
        auto value = [&](int x, float l, float add) {
            if (a.counted) {
                const int i = x - lo + 8;
                const uint32_t n = s_bits[i / 32] >> i % 32 & 1u ? s_count[count_of(i)] : 0u;
                if (n) l = penalised(l, n);
            }
            return kRules >= 2 && bias ? l + add : l;
        };
        // choose: the largest logit of the thread, its chunk (of few: its number among them), and the sum of exp(logit - ref)
        float best = -INFINITY, ref = -FLT_MAX, sum = 0.f;
        int at = 0x7fffffff;
        Chunk<T> kept;
        T* out = kChoose ? nullptr : (T*)a.out + (int64_t)row * a.out_stride;
        // sum and reference with 8 more logits, the largest of them top
        auto weigh = [&](const float (&f)[8], float top) {
            if (top > ref) {
                const float up = ceilf(top);
                sum *= exp2_of((ref - up) * kLog2e);
                ref = up;
            }
            uint64_t e2 = 0ull;
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float2 d = of_pair(mul_pair(add_pair(pair_of(f[j], f[j + 1]), pair_of(-ref, -ref)), pair_of(kLog2e, kLog2e)));
                e2 = add_pair(e2, pair_of(exp2_of(d.x), exp2_of(d.y)));
            }
            const float2 e = of_pair(e2);
            float s = e.x + e.y;
            if (!(s < 16.f)) {  // (infinite or NaN among them)
                s = 0.f;
                for (int j = 0; j < 8; ++j)
                    if (f[j] == f[j]) s += weight(f[j], ref);
            }
            sum += s;
        };
        // (fmaxf passes NaN over)
        auto largest = [](const float (&f)[8]) { return fmaxf(fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])), fmaxf(fmaxf(f[4], f[5]), fmaxf(f[6], f[7]))); };
        for (int e = tid; kChoose && kRules && e < few; e += 8 * kLogitThreads) {
            int x[8];  // places
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = e + i * kLogitThreads < few ? (int)s_list[e + i * kLogitThreads] : -1;
                f[i] = x[i] >= 0 ? (float)src[lo - 8 + x[i]] : -INFINITY;
            }
            if (a.counted) {
                uint32_t m = 0u;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (x[i] >= 0) m |= (s_bits[x[i] / 32] >> x[i] % 32 & 1u) << i;
                if (m) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t n = m >> i & 1u ? s_count[count_of(x[i])] : 0u;
                        if (n) f[i] = penalised(f[i], n);
                    }
                }
            }
            if (kRules >= 2 && bias) {
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] += x[i] >= 0 ? __ldcg(bias + lo - 8 + x[i]) : 0.f;  // (asked for with the logits: registers, the same time)
            }
            const float top = largest(f);
            if (top > best) {
                best = top;
#pragma unroll
                for (int i = 7; i >= 0; --i) at = f[i] == top ? e + i * kLogitThreads : at;
            }
            weigh(f, top);
        }
        for (int x = few < 0 ? first + 8 * tid : stop; x < stop; x += 8 * kLogitThreads * kAhead) {
            Chunk<T> c[kAhead];
            float4 add[kAdds];
            uint32_t show[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int x0 = x + 8 * kLogitThreads * i;
                show[i] = x0 < stop ? kRules ? shown(x0) : 255u : 0u;
                if (show[i]) {
                    load(x0, c[i]);
                    if (kRules && i == 0) load_bias(x0, add);
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int x0 = x + 8 * kLogitThreads * i;
                float f[8];
                if constexpr (kChoose) {
                    if (show[i]) {
                        c[i].get(f);
                        if (kRules) rules(x0, show[i], add, f);
                    }
                    if (kRules && i + 1 < kAhead && show[(i + 1) % kAhead]) load_bias(x0 + 8 * kLogitThreads, add);
                    if (!show[i]) continue;
                    const float top = largest(f);
                    if (top > best) {
                        best = top, at = x0;
                        if (!kRules) kept = c[i];
                    }
                    weigh(f, top);
                } else {
                    if (x0 >= stop) break;
                    if (show[i]) {
                        c[i].get(f);
                        rules(x0, show[i], add, f);
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[j] = -INFINITY;
                    }
                    if (i + 1 < kAhead && show[(i + 1) % kAhead]) load_bias(x0 + 8 * kLogitThreads, add);
                    if (whole(x0) && ((uintptr_t)(out + x0) & 15u) == 0) {
                        c[i].put(f);
#pragma unroll
                        for (int j = 0; j < kParts; ++j) reinterpret_cast<uint4*>(out + x0)[j] = c[i].u[j];
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (inside(x0 + j)) out[x0 + j] = (T)f[j];
                    }
                }
            }
        }
        if constexpr (!kChoose) {
            if (a.counted || a.r.allowed) __syncthreads();  // (masks and counts are read)
        } else {
            // the CTA's reference and sum of weights
            const float m_w = warp_max(ref);
            const float s_w = warp_sum(sum * weight(ref, m_w));
            if (lane == 0) s_m[warp] = m_w, s_s[warp] = s_w;
            // each warp's k best of its threads, largest first, of equal ones the lowest chunk
            uint32_t mine = best > -INFINITY ? order_of(best + 0.f) : 0u;
            for (int i = 0; i < a.k; ++i) {
                const uint32_t o = __reduce_max_sync(0xffffffffu, mine);
                const int x = __reduce_min_sync(0xffffffffu, mine == o ? at : 0x7fffffff);
                if (lane == 0) s_first[warp * a.k + i] = o ? (uint64_t)o << 32 | (uint32_t)~(x + 8) : 0ull;
                if (mine == o && at == x) mine = 0u;
            }
            Partial& part = s_part[turn];
            turn ^= 1;
            if (tid < kMaxBest) part.best[tid] = 0ull, s_from[tid] = -1;
            if (tid == 0) s_n = 0, s_found = 0, s_bound = 1ull;
            __syncthreads();
            const int lists = kLogitWarps * a.k;
            if (a.k == 1) {
                uint64_t key = 0ull;
#pragma unroll
                for (int i = 0; i < kLogitWarps; ++i) key = max(key, s_first[i]);
                if (key && at == (int)~(uint32_t)key - 8) {  // (this thread's chunk)
                    int token = at + 7;
                    if (kRules && few >= 0) {
                        token = lo - 8 + (int)s_list[at];
                    } else {
                        float f[8];
                        float4 add[kAdds];
                        if (kRules) {
                            load(at, kept);
                            load_bias(at, add);
                        }
                        kept.get(f);
                        if (kRules) rules(at, shown(at), add, f);
#pragma unroll
                        for (int j = 6; j >= 0; --j) token = f[j] == best ? at + j : token;
                    }
                    part.best[0] = key_of(best + 0.f, token);
                }
            } else if (tid < lists) {  // the k best threads, and the last of them as the bound
                const uint64_t key = s_first[tid];
                int rank = 0;
                for (int i = 0; i < lists; ++i) rank += s_first[i] > key;
                if (key && rank < a.k) {
                    const int x = (int)~(uint32_t)key - 8;
                    s_from[rank] = (kRules && few >= 0 ? x : (x - first) / 8) % kLogitThreads;
                    if (rank == a.k - 1) s_bound = key & ~0xffffffffull;  // (by the logit alone: the token lies somewhere in the chunk)
                    atomicAdd(&s_found, 1);
                }
            }
            if (warp == kLogitWarps - 1) {
                const float m = lane < kLogitWarps ? s_m[lane] : -INFINITY, s = lane < kLogitWarps ? s_s[lane] : 0.f;
                const float m_c = warp_max(m), s_c = warp_sum(s * weight(m, m_c));
                if (lane == 0) part.sum = (uint64_t)__float_as_uint(m_c) << 32 | __float_as_uint(s_c);
            }
            if (a.k > 1) {
                __syncthreads();
                const int n_from = s_found;
                const uint64_t bound = s_bound;
                const bool listed = kRules && few >= 0;
                if (listed) {
                    for (int i = tid; i < n_from * ((few + kLogitThreads - 1) / kLogitThreads); i += kLogitThreads) {
                        const int e = s_from[i % n_from] + i / n_from * kLogitThreads;
                        if (e >= few) continue;
                        const int x = lo - 8 + (int)s_list[e];
                        const float l = value(x, (float)src[x], kRules >= 2 && bias ? __ldcg(bias + x) : 0.f);
                        const uint64_t key = key_of(l + 0.f, x);
                        if (l > -INFINITY && key >= bound) s_cand[atomicAdd(&s_n, 1)] = key;
                    }
                }
                for (int i = listed ? n_from * deep : tid; i < n_from * deep; i += kLogitThreads) {
                    const int x0 = first + 8 * (s_from[i % n_from] + i / n_from * kLogitThreads);
                    if (x0 >= stop) continue;
                    Chunk<T> c;
                    float f[8];
                    float4 add[kAdds];
                    load(x0, c);
                    if (kRules) load_bias(x0, add);
                    c.get(f);
                    if (kRules) rules(x0, shown(x0), add, f);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (f[j] > -INFINITY) {
                            const uint64_t key = key_of(f[j] + 0.f, x0 + j);  // (0 and -0 are equal)
                            if (key >= bound) s_cand[atomicAdd(&s_n, 1)] = key;
                        }
                }
                __syncthreads();
                const int n = s_n;
                for (int i = tid; i < n; i += kLogitThreads) {
                    const uint64_t key = s_cand[i];
                    int rank = 0;
                    for (int j = 0; j < n; ++j) rank += s_cand[j] > key;
                    if (rank < a.k) part.best[rank] = key;
                }
            }
            // the CTAs of the row are joined by one of them, in turn.  (Two parts alternate: the one of this row is written
            // again after the next row's barrier, which its reader reaches when it has read.)
            if (split > 1) cluster_sync();
            else __syncthreads();
            if (row % split == (int)blockIdx.x && warp < kJoinWarps) {
                uint64_t* all = s_first;  // (its readers are behind a barrier)
                const int n = split * a.k;
                for (int i = tid; i < n; i += 32 * kJoinWarps) all[i] = split > 1 ? peer_load(&part.best[i % a.k], i / a.k) : part.best[i % a.k];
                float m = -INFINITY, s = 0.f;
                if (lane < split) {
                    const uint64_t u = split > 1 ? peer_load(&part.sum, lane) : part.sum;
                    m = __uint_as_float((uint32_t)(u >> 32)), s = __uint_as_float((uint32_t)u);
                }
                const float top = warp_max(m);
                const float log_sum = logf(warp_sum(s * weight(m, top)));
                asm volatile("bar.sync 1, %0;\n" ::"n"(32 * kJoinWarps) : "memory");
                for (int i = tid; i < n; i += 32 * kJoinWarps) {
                    const uint64_t key = all[i];
                    int rank = 0;
                    for (int j = 0; j < n; ++j) rank += all[j] > key || (all[j] == key && j < i);  // (only keys of 0 are equal)
                    if (rank < a.k) {
                        const float v = of_order((uint32_t)(key >> 32));
                        a.tokens[(int64_t)row * a.k + rank] = key ? (int)~(uint32_t)key : -1;
                        a.logprob[(int64_t)row * a.k + rank] = key ? (v == top ? 0.f : v - top) - log_sum : -INFINITY;
                    }
                }
                if (tid == 0 && a.total) a.total[row] = top + log_sum;
            }
            __syncthreads();
        }
    }
    if (kChoose && split > 1) cluster_sync();  // (no CTA leaves while another may read its part)
}

// lays dynamic shared memory out; returns its bytes.  Counts are kept for as many tokens as can be said in a slice.
size_t lay_out(LogitArgs& a) {
    const ssd_logit_rules& r = a.r;
    const int deep = (a.slice / 8 + kLogitThreads - 1) / kLogitThreads;
    a.at_show = a.k > 1 ? a.k * deep * 8 * 8 : 0;
    a.at_list = a.at_show + (r.allowed ? (a.slice / 32 + 3) * 4 : 0);
    a.at_bits = a.at_list + (r.allowed && a.k ? (a.slice / kFew + 1) / 2 * 4 : 0);
    a.at_bits = (a.at_bits + 15) / 16 * 16;
    a.n_words = (a.slice + 8 + 127) / 128 * 4;
    if (!a.counted) return a.at_bits;
    const long long said = (r.history ? r.max_history : 0ll) + (r.tokens ? r.n_rows : 0ll);
    return a.at_bits + 4 * (a.n_words + a.n_words / 4 + 1 + (size_t)std::min<long long>(a.slice + 8, said));
}
constexpr int kMostShared = 180 * 1024;  // (a slice of 32832 tokens, all of them said: 18 + 4 + 140 KB)

template <typename T>
int set_up() {
    void (*const k[])(LogitArgs) = {logits_kernel<T, true, 0>, logits_kernel<T, true, 1>, logits_kernel<T, true, 2>, logits_kernel<T, true, 3>, logits_kernel<T, true, 2, 2>, logits_kernel<T, true, 3, 2>, logits_kernel<T, false, 1>, logits_kernel<T, false, 2>,
                                      logits_kernel<T, false, 3>};
    cudaError_t e = cudaSuccess;
    for (auto f : k)
        if (e == cudaSuccess) e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
    return (int)e;
}

template <typename T>
cudaError_t start(const cudaLaunchConfig_t& cfg, const LogitArgs& a, bool choose, int rules, int ctas) {
    if (choose && ctas == 2) return cudaLaunchKernelEx(&cfg, rules == 3 ? logits_kernel<T, true, 3, 2> : logits_kernel<T, true, 2, 2>, a);
    if (!choose) return cudaLaunchKernelEx(&cfg, rules == 3 ? logits_kernel<T, false, 3> : rules == 2 ? logits_kernel<T, false, 2> : logits_kernel<T, false, 1>, a);
    return cudaLaunchKernelEx(&cfg, rules == 3 ? logits_kernel<T, true, 3> : rules == 2 ? logits_kernel<T, true, 2> : rules ? logits_kernel<T, true, 1> : logits_kernel<T, true, 0>, a);
}

int check_rules(const char* call, const ssd_logit_rules* r, int dtype, const void* logits, int64_t stride) {
    if (!r) return refuse_arg(call, "NULL rules");
    if (dtype != SSD_F32 && dtype != SSD_F16 && dtype != SSD_BF16) return refuse_arg(call, "logits are fp32, fp16 or bf16");
    if (r->vocab < 1 || r->vocab > kMaxVocab) return refuse_arg(call, "need 1 <= vocab <= 262144");
    if (r->n_rows < 0 || r->max_rows < 1) return refuse_arg(call, "need n_rows >= 0 and max_rows >= 1");
    if (r->n_rows == 0) return SSD_OK;
    if (r->row_start ? r->n_requests < 1 || r->n_requests > kMaxRequests : r->n_requests != r->n_rows)
        return refuse_arg(call, "need 1 <= n_requests <= 4096, or without row_start n_requests = n_rows");
    if (!aligned(4, {r->row_start, r->history, r->history_len, r->prompt_len, r->tokens, r->repetition, r->presence, r->frequency, r->bias, r->bias_of, r->allowed, r->allowed_of}) ||
        !aligned(8, {r->masks}))
        return refuse_arg(call, "what the rules read must be aligned to its type");
    const int64_t most = int64_t(1) << 37;
    if (!logits) return refuse_arg(call, "NULL logits");
    if (stride < r->vocab || stride > most || (uintptr_t)logits % (dtype == SSD_F32 ? 4 : 2)) return refuse_arg(call, "logits: rows must not overlap, aligned to their type");
    if (r->history && (!r->history_len || r->max_history < 0 || r->history_stride < r->max_history || r->history_stride > most))
        return refuse_arg(call, "history needs history_len and history_stride >= max_history >= 0");
    if (r->masks && (!r->tokens || r->mask_words < 1 || r->mask_words > 4)) return refuse_arg(call, "masks need tokens and 1 .. 4 words a row");
    if (!r->masks && r->mask_words != 0) return refuse_arg(call, "mask_words must be 0 without masks");
    if (r->bias && (r->n_bias < 1 || r->bias_stride < r->vocab || r->bias_stride > most)) return refuse_arg(call, "bias: need n_bias >= 1 rows of at least vocab floats");
    if (r->allowed && (r->n_allowed < 1 || r->allowed_stride < (r->vocab + 31) / 32 || r->allowed_stride > most || (!r->allowed_of && r->n_allowed < r->n_rows)))
        return refuse_arg(call, "allowed: need n_allowed >= 1 sets (n_rows without allowed_of) of at least vocab bits");
    return SSD_OK;
}

// whether a result lies where the rules are read
bool meets_rules(const Range (&out)[1], const ssd_logit_rules& r) {
    const size_t b = 4 * (size_t)r.n_requests, n = 4 * (size_t)r.n_rows, words = (size_t)(r.vocab + 31) / 32;
    const Range in[14] = {{r.row_start, b + 4},
                          {r.history, 4 * ((size_t)(r.n_requests - 1) * (size_t)r.history_stride + (size_t)r.max_history)},
                          {r.history_len, b},
                          {r.prompt_len, b},
                          {r.tokens, n},
                          {r.masks, 2 * n * (size_t)r.mask_words},
                          {r.repetition, b},
                          {r.presence, b},
                          {r.frequency, b},
                          {r.bias, r.bias ? 4 * ((size_t)(r.n_bias - 1) * (size_t)r.bias_stride + (size_t)r.vocab) : 0},
                          {r.bias_of, b},
                          {r.allowed, r.allowed ? 4 * ((size_t)(r.n_allowed - 1) * (size_t)r.allowed_stride + words) : 0},
                          {r.allowed_of, n},
                          {nullptr, 0}};
    return meet(out, in);
}

int launch_logits(const char* call, LogitArgs& a, int dtype, bool choose, void* stream) {
    const ssd_logit_rules& r = a.r;
    int dev = 0;
    if (int rc = check_device(call, a.logits)) return rc;
    if (int rc = device_of(call, &dev)) return rc;
    {
        static std::mutex mu;
        static bool ready[kMaxDevices] = {};
        std::lock_guard<std::mutex> lock(mu);
        if (!ready[dev]) {  // (for all types, so that a first use with one of them prepares captures with any)
            int e = set_up<float>();
            if (!e) e = set_up<f16>();
            if (!e) e = set_up<bf16>();
            if (e) return refuse(SSD_ERR_CUDA, call, "%s", cudaGetErrorString((cudaError_t)e));
            ready[dev] = true;
        }
    }
    a.counted = (r.repetition || r.presence || r.frequency) && (r.history || r.tokens);
    int sms = 0;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return refuse(SSD_ERR_CUDA, call, "no device");
    // (chunks start on 16 bytes of the logits: those of the biases too in every row and set, or not)
    const size_t size = dtype == SSD_F32 ? 4 : 2;
    const bool even = ((uintptr_t)r.bias & 15u) == 0 && r.bias_stride % 4 == 0 && (uintptr_t)a.logits % (4 * size) == 0 && a.stride % 4 == 0;
    const int rules = r.bias ? even ? 2 : 3 : a.counted || r.allowed ? 1 : 0;
    // A row's slices: 1 to 8, whichever is done first if a wave of CTAs takes as long as its slice and 20000 tokens more for its start
    // and end, or 30000 with counts to make.  (512 rows of 128256, penalised and masked: whole 68 us, in two 70, in four 94; 207
    // rows of 50257, penalised and with biases: whole 39, in two 29, in four 44.)
    // With biases two CTAs an SM are taken to need three quarters of the time of three.
    int split = 0, ctas = 0;
    long long least = 0;
    for (int n = ctas_of(choose, rules); n >= (choose && rules >= 2 ? 2 : ctas_of(choose, rules)); --n)
        for (int parts = 1; parts <= kMaxSplit; parts *= 2) {
            a.slice = ((r.vocab + 7 + parts - 1) / parts + 63) / 64 * 64;
            if (a.slice > (choose && r.allowed ? kMaxListed : kMaxSlice) || (parts > 1 && a.slice < 1024)) continue;
            const size_t bytes = lay_out(a);
            if (bytes > kMostShared) continue;
            const int fit = (int)std::min<size_t>(n, (222 * 1024) / (bytes + 4096));
            const long long waves = ((long long)r.n_rows * parts + sms * fit - 1) / (sms * fit);
            const long long cost = waves * (a.slice + (a.counted ? 30000 : 20000)) * (n == 2 ? 3 : 4);
            if (!split || cost < least) split = parts, ctas = n, least = cost;
        }
    a.slice = ((r.vocab + 7 + split - 1) / split + 63) / 64 * 64;
    // rows of a request share its counts, as many as leave two waves of CTAs
    a.rows = a.counted ? (int)std::min<long long>(r.max_rows, std::max(1ll, (long long)r.n_rows * split / 912)) : 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)split, (unsigned)((r.n_rows + a.rows - 1) / a.rows), 1);
    if (cfg.gridDim.y > 65535u) {
        a.rows = (r.n_rows + 65534) / 65535;
        cfg.gridDim.y = (unsigned)((r.n_rows + a.rows - 1) / a.rows);
    }
    cfg.blockDim = dim3(kLogitThreads, 1, 1);
    cfg.dynamicSmemBytes = lay_out(a);
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)split, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = choose && split > 1 ? 2 : 1;
    const cudaError_t e = dtype == SSD_F32 ? start<float>(cfg, a, choose, rules, ctas) : dtype == SSD_F16 ? start<f16>(cfg, a, choose, rules, ctas) : start<bf16>(cfg, a, choose, rules, ctas);
    return e == cudaSuccess ? SSD_OK : refuse(SSD_ERR_CUDA, call, "%s", cudaGetErrorString(e));
}

}  // namespace step
}  // namespace ssd

using namespace ssd;
using namespace ssd::step;

extern "C" int ssd_logits_adjust(const ssd_logit_rules* rules, int dtype, const void* logits, int64_t stride, void* out,
                                 int64_t out_stride, void* cuda_stream) {
    static const char call[] = "ssd_logits_adjust";
    if (int rc = check_rules(call, rules, dtype, logits, stride)) return rc;
    if (rules->n_rows == 0) return SSD_OK;
    if (!out) return refuse_arg(call, "NULL out");
    if (out_stride < rules->vocab || out_stride > (int64_t(1) << 37) || (uintptr_t)out % (dtype == SSD_F32 ? 4 : 2))
        return refuse_arg(call, "out: rows must not overlap, aligned to their type");
    if (out == logits ? out_stride != stride : meet(out, span(rules->n_rows, out_stride, rules->vocab, dtype), logits, span(rules->n_rows, stride, rules->vocab, dtype)))
        return refuse_arg(call, "out must be the logits with their stride, or not overlap them");
    const Range all[1] = {{out, span(rules->n_rows, out_stride, rules->vocab, dtype)}};
    if (meets_rules(all, *rules)) return refuse_arg(call, "out must not overlap what the rules read");
    LogitArgs a{};
    a.r = *rules;
    a.logits = logits;
    a.stride = stride;
    a.out = out;
    a.out_stride = out_stride;
    return launch_logits(call, a, dtype, false, cuda_stream);
}

extern "C" int ssd_logits_choose(const ssd_logit_rules* rules, int dtype, const void* logits, int64_t stride, int k,
                                 int32_t* tokens, float* logprob, float* total, void* cuda_stream) {
    static const char call[] = "ssd_logits_choose";
    if (int rc = check_rules(call, rules, dtype, logits, stride)) return rc;
    if (k < 1 || k > kMaxBest) return refuse_arg(call, "need 1 <= k <= 16");
    if (rules->n_rows == 0) return SSD_OK;
    if (!tokens || !logprob) return refuse_arg(call, "NULL pointer");
    if (!aligned(4, {tokens, logprob, total})) return refuse_arg(call, "the results must be aligned to their type");
    const size_t n = 4 * (size_t)rules->n_rows;
    const Range a1[1] = {{tokens, n * k}}, a2[1] = {{logprob, n * k}}, a3[1] = {{total, n}}, in[1] = {{logits, span(rules->n_rows, stride, rules->vocab, dtype)}};
    if (meet(a1, a2) || meet(a1, a3) || meet(a2, a3) || meet(a1, in) || meet(a2, in) || meet(a3, in) || meets_rules(a1, *rules) || meets_rules(a2, *rules) ||
        meets_rules(a3, *rules))
        return refuse_arg(call, "the results must overlap neither each other, nor the logits or what the rules read");
    LogitArgs a{};
    a.r = *rules;
    a.logits = logits;
    a.stride = stride;
    a.k = k;
    a.tokens = tokens;
    a.logprob = logprob;
    a.total = total;
    return launch_logits(call, a, dtype, true, cuda_stream);
}
