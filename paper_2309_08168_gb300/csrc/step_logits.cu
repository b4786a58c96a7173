// step_logits.cu - penalties, biases and masks on logits, and the choice of the
// best tokens of every row (ssd_logits_adjust, ssd_logits_choose of ssd_step.h).
#include <algorithm>
#include <cmath>

#include "step_ops.cuh"

namespace ssd {
namespace step {

constexpr int kLogitThreads = 512, kLogitWarps = kLogitThreads / 32;
constexpr int kMaxVocab = 262144;
constexpr int kMaxSlice = 32832;  // tokens of a CTA: at most 9 chunks of 8 in each of its threads
constexpr int kMaxSplit = 8;      // CTAs of a row: one portable cluster
constexpr int kMaxBest = 16;
constexpr int kCandidates = kMaxBest * ((kMaxSlice / 8 + kLogitThreads - 1) / kLogitThreads) * 8;
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
};

// what a float sorts by; 0 is below all of them (-inf gives 0x007fffff)
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t u = __float_as_uint(v);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_order(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
// (logit, token) as one number: larger logits first, of equal ones the lower token; 0 is none
__device__ __forceinline__ uint64_t key_of(float v, int x) { return (uint64_t)order_of(v) << 32 | (uint32_t)~x; }

// exp(v - m) for v <= m, 1 for v = m = inf
__device__ __forceinline__ float weight(float v, float m) { return v == m ? 1.f : exp2f((v - m) * 1.4426950408889634f); }

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
// 16 bytes of the logits (a: how far the row's first one lies before its first token), chunk j in thread j mod 512.
//
// The counts of what a text has said are made once for the rows of one request that a cluster takes, in shared memory, for the CTA's
// slice alone: history tokens are added by all threads, a row's nodes before the row and taken off after it.  A bit for each
// token tells whether there is anything to look up, so that the pass over the logits asks two words per 8 tokens.
//
// The k best: each thread keeps its own best; the k-th largest of these is a bound that at least k tokens reach, and only
// tokens of the k threads above it can be among the k best.  Their chunks are read once more (from L2), what reaches the bound is
// ranked by counting, and ranks below k are the answer.  All keys differ (the token is part of them), so ties need no care.
template <typename T, bool kChoose>
__global__ void __launch_bounds__(kLogitThreads, 2) logits_kernel(const __grid_constant__ LogitArgs a) {
    constexpr int V = Vec<T>::N;  // tokens in 16 bytes
    constexpr int kAhead = 2;     // chunks of 8 tokens under way in a thread
    extern __shared__ __align__(16) uint32_t s_dyn[];
    __shared__ int s_request[2], s_n;
    __shared__ float s_m[kLogitWarps], s_s[kLogitWarps];
    __shared__ uint64_t s_first[kLogitWarps * kMaxBest], s_bound;
    __shared__ int s_from[kMaxBest], s_found;
    __shared__ uint64_t s_cand[kChoose ? kCandidates : 1];
    __shared__ Partial s_part[2];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, split = gridDim.x, vocab = a.r.vocab;
    const int lo = blockIdx.x * a.slice;
    const int row0 = blockIdx.y * a.rows, row1 = min(row0 + a.rows, a.r.n_rows);
    // counts of tokens lo - 8 .. lo + slice - 1 (chunks may start up to 7 tokens before the slice)
    const int width = a.slice + 8;
    uint32_t *s_said = s_dyn, *s_count = s_dyn + (width + 31) / 32;
    // adds (or takes off) one token that the model has said
    auto say_token = [&](int x, bool off) {
        const int i = x - lo + 8;
        if (x < 0 || x >= vocab || i < 0 || i >= width) return;
        if (!off) {
            atomicAdd(s_count + i, 1u);
            atomicOr(s_said + i / 32, 1u << i % 32);
        } else if (atomicSub(s_count + i, 1u) == 1u) {
            atomicAnd(s_said + i / 32, ~(1u << i % 32));
        }
    };
    int request = -1, start = 0, end = 0;  // of the row before
    int old = -1;                          // the row whose nodes are in the counts
    auto nodes = [&](int row, bool off) {  // the nodes that a row's mask shows
        const int n = a.r.masks ? min(end - start, 64 * a.r.mask_words) : row - start + 1;
        for (int j = tid; j < n; j += kLogitThreads) {
            const bool seen = !a.r.masks || (__ldcg(reinterpret_cast<const unsigned long long*>(a.r.masks) + (int64_t)row * a.r.mask_words + j / 64) >> (j % 64) & 1);
            if (seen) say_token(__ldcg(a.r.tokens + start + j), off);
        }
    };
    float again = 1.f, often = 0.f, once = 0.f;
    const float* bias = nullptr;
    int turn = 0;  // which of the two parts
    for (int row = row0; row < row1; ++row) {
        // the request that owns the row
        if (!a.r.row_start) {
            start = row, end = row + 1;
        }
        const bool fresh = !a.r.row_start || row >= end;
        int owner = request;
        if (a.r.row_start && fresh && !a.counted && !a.r.bias_of) {  // (whose it is does not matter)
            const int s0 = __ldcg(a.r.row_start), s1 = __ldcg(a.r.row_start + a.r.n_requests);
            owner = s0 <= row && row < s1 ? 0 : a.r.n_requests;
            end = row + 1;
        } else if (a.r.row_start && fresh) {
            if (tid == 0) s_request[0] = a.r.n_requests;
            __syncthreads();
            for (int b = tid; b < a.r.n_requests; b += kLogitThreads) {
                const Rows r = rows_of(a.r.row_start, b, a.r.n_rows);
                if (r.r0 <= row && row < r.r0 + r.n) atomicMin(&s_request[0], b);
            }
            __syncthreads();
            owner = s_request[0];
            if (owner < a.r.n_requests) {
                const Rows r = rows_of(a.r.row_start, owner, a.r.n_rows);
                start = r.r0, end = r.r0 + r.n;
            } else {
                start = row, end = row + 1;  // (no one's)
            }
            __syncthreads();  // (s_request is read before the next search)
        } else if (fresh) {
            owner = row;
        }
        const bool owned = owner < a.r.n_requests;
        if (owned && fresh) {
            if (a.counted) {
                __syncthreads();  // (the counts of the row before are no longer read)
                for (int i = tid; i < (width + 31) / 32 + width; i += kLogitThreads) s_dyn[i] = 0u;
                old = -1;
                again = a.r.repetition ? __ldcg(a.r.repetition + owner) : 1.f;
                often = a.r.frequency ? __ldcg(a.r.frequency + owner) : 0.f;
                once = a.r.presence ? __ldcg(a.r.presence + owner) : 0.f;
                __syncthreads();
                if (a.r.history) {
                    const int n = min(max(__ldcg(a.r.history_len + owner), 0), a.r.max_history);
                    const int prompt = a.r.prompt_len ? __ldcg(a.r.prompt_len + owner) : 0;
                    const int32_t* h = a.r.history + (int64_t)owner * a.r.history_stride;
                    for (int j = tid; j < n; j += kLogitThreads) {
                        const int x = __ldcg(h + j), i = x - lo + 8;
                        if (j >= prompt) {
                            say_token(x, false);
                        } else if (x >= 0 && x < vocab && i >= 0 && i < width) {
                            atomicOr(s_count + i, kPrompt);
                            atomicOr(s_said + i / 32, 1u << i % 32);
                        }
                    }
                }
            }
            bias = nullptr;
            if (a.r.bias) {
                const int b = a.r.bias_of ? __ldcg(a.r.bias_of + owner) : 0;
                if (b >= 0 && b < a.r.n_bias) bias = a.r.bias + (int64_t)b * a.r.bias_stride;
            }
        }
        request = owner;
        if (!owned) continue;  // (uniform over the cluster: its CTAs have the same rows)
        if (a.counted && a.r.tokens) {
            __syncthreads();  // (history counted; the row before read)
            if (old >= 0) {
                nodes(old, true);
                __syncthreads();
            }
            nodes(row, false);
            old = row;
        }
        if (a.counted) __syncthreads();
        const uint32_t* allowed = nullptr;
        if (a.r.allowed) {
            const int m = a.r.allowed_of ? __ldcg(a.r.allowed_of + row) : row;
            if (m >= 0 && m < a.r.n_allowed) allowed = a.r.allowed + (int64_t)m * a.r.allowed_stride;
        }
        const T* src = (const T*)a.logits + (int64_t)row * a.stride;
        const int before = (int)(((uintptr_t)src & 15u) / sizeof(T));
        const int first = lo - before, stop = min(lo + a.slice - before, vocab);  // this CTA's tokens: [max(first, 0), stop)
        const int words = (vocab + 31) / 32;
        // token x0 + i of a chunk is there
        auto inside = [&](int x) { return x >= 0 && x < vocab; };
        auto load = [&](int x0, Chunk<T>& c) {
            if (x0 >= 0 && x0 + 8 <= vocab) {
#pragma unroll
                for (int i = 0; i < 8 / V; ++i) c.u[i] = __ldcg(reinterpret_cast<const uint4*>(src + x0) + i);
            } else {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = inside(x0 + i) ? (float)src[x0 + i] : -INFINITY;
                c.put(f);
            }
        };
        auto bits8 = [&](const uint32_t* w, int n_words, int x) -> uint32_t {  // bits x .. x + 7, x >= 0
            const int i = x / 32, s = x % 32;
            uint32_t u = i < n_words ? w[i] : 0u;
            if (s > 24 && i + 1 < n_words) return __funnelshift_r(u, w[i + 1], s) & 255u;
            return (u >> s) & 255u;
        };
        auto rules = [&](int x0, float (&f)[8]) {
            if (a.counted) {
                const int at = x0 - lo + 8;  // >= 0
                uint32_t m = bits8(s_said, (width + 31) / 32, at);
                while (m) {
                    const int i = __ffs((int)m) - 1;
                    m &= m - 1;
                    const uint32_t n = s_count[at + i], c = n & ~kPrompt;
                    float l = f[0];
#pragma unroll
                    for (int j = 1; j < 8; ++j) l = i == j ? f[j] : l;
                    l = l > 0.f ? __fdiv_rn(l, again) : __fmul_rn(l, again);
                    l = __fsub_rn(l, __fmul_rn(often, (float)c));
                    if (c) l = __fsub_rn(l, once);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] = i == j ? l : f[j];
                }
            }
            if (bias) {
                if (x0 >= 0 && x0 + 8 <= vocab && ((uintptr_t)(bias + x0) & 15u) == 0) {
                    const float4 u = __ldcg(reinterpret_cast<const float4*>(bias + x0)), w = __ldcg(reinterpret_cast<const float4*>(bias + x0 + 4));
                    f[0] += u.x, f[1] += u.y, f[2] += u.z, f[3] += u.w, f[4] += w.x, f[5] += w.y, f[6] += w.z, f[7] += w.w;
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (inside(x0 + i)) f[i] += __ldcg(bias + x0 + i);
                }
            }
            if (allowed) {
                const int x = max(x0, 0);
                const int i = x / 32, s = x % 32;
                uint32_t u = __ldcg(allowed + i) >> s;
                if (s > 24 && i + 1 < words) u |= __ldcg(allowed + i + 1) << (32 - s);
                u <<= x - x0;
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = u >> j & 1u ? f[j] : -INFINITY;
            }
        };
        if constexpr (!kChoose) {
            T* out = (T*)a.out + (int64_t)row * a.out_stride;
            for (int x = first + 8 * tid; x < stop; x += 8 * kLogitThreads * kAhead) {
                Chunk<T> c[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
                    if (x + 8 * kLogitThreads * i < stop) load(x + 8 * kLogitThreads * i, c[i]);
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int x0 = x + 8 * kLogitThreads * i;
                    if (x0 >= stop) break;
                    float f[8];
                    c[i].get(f);
                    rules(x0, f);
                    if (x0 >= 0 && x0 + 8 <= vocab && ((uintptr_t)(out + x0) & 15u) == 0) {
                        c[i].put(f);
#pragma unroll
                        for (int j = 0; j < 8 / V; ++j) reinterpret_cast<uint4*>(out + x0)[j] = c[i].u[j];
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (inside(x0 + j)) out[x0 + j] = (T)f[j];
                    }
                }
            }
        } else {
            // NaN and what is not there count as -inf
            auto taken = [&](int x0, float (&f)[8]) {
                rules(x0, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = (inside(x0 + j) && f[j] == f[j]) ? f[j] + 0.f : -INFINITY;
            };
            float best = -INFINITY, sum = 0.f;
            int token = 0x7fffffff;
            for (int x = first + 8 * tid; x < stop; x += 8 * kLogitThreads * kAhead) {
                Chunk<T> c[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
                    if (x + 8 * kLogitThreads * i < stop) load(x + 8 * kLogitThreads * i, c[i]);
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int x0 = x + 8 * kLogitThreads * i;
                    if (x0 >= stop) break;
                    float f[8];
                    c[i].get(f);
                    taken(x0, f);
                    const float was = best;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (f[j] > best) best = f[j], token = x0 + j;
                    if (best > -INFINITY) {
                        sum *= weight(was, best);
#pragma unroll
                        for (int j = 0; j < 8; ++j) sum += weight(f[j], best);
                    }
                }
            }
            // the CTA's maximum and sum of weights
            const float m_w = warp_max(best);
            const float s_w = warp_sum(best > -INFINITY ? sum * weight(best, m_w) : 0.f);
            if (lane == 0) s_m[warp] = m_w, s_s[warp] = s_w;
            // each warp's k best of its threads, largest first
            uint32_t mine = best > -INFINITY ? order_of(best) : 0u;
            for (int i = 0; i < a.k; ++i) {
                const uint32_t o = __reduce_max_sync(0xffffffffu, mine);
                const uint32_t t = __reduce_min_sync(0xffffffffu, mine == o ? (uint32_t)token : 0xffffffffu);
                if (lane == 0) s_first[warp * a.k + i] = o ? (uint64_t)o << 32 | (uint32_t)~t : 0ull;
                if (mine == o && (uint32_t)token == t) mine = 0u;
            }
            Partial& part = s_part[turn];
            turn ^= 1;
            if (tid < kMaxBest) part.best[tid] = 0ull, s_from[tid] = -1;
            if (tid == 0) s_n = 0, s_found = 0, s_bound = 1ull;
            __syncthreads();
            const int lists = kLogitWarps * a.k;
            if (tid < lists) {  // the k best threads, and the last of them as the bound
                const uint64_t key = s_first[tid];
                int rank = 0;
                for (int i = 0; i < lists; ++i) rank += s_first[i] > key;
                if (key && rank < a.k) {
                    if (a.k == 1) {
                        part.best[0] = key;
                    } else {
                        const int x = (int)~(uint32_t)key;
                        s_from[rank] = (x - first) / 8 % kLogitThreads;
                        if (rank == a.k - 1) s_bound = key;
                        atomicAdd(&s_found, 1);
                    }
                }
            }
            if (warp == kLogitWarps - 1) {
                const float m = lane < kLogitWarps ? s_m[lane] : -INFINITY, s = lane < kLogitWarps ? s_s[lane] : 0.f;
                const float m_c = warp_max(m), s_c = warp_sum(m > -INFINITY ? s * weight(m, m_c) : 0.f);
                if (lane == 0) part.sum = (uint64_t)__float_as_uint(m_c) << 32 | __float_as_uint(s_c);
            }
            if (a.k > 1) {
                __syncthreads();
                const int chunks = a.slice / 8, deep = (chunks + kLogitThreads - 1) / kLogitThreads, n_from = s_found;
                const uint64_t bound = s_bound;
                for (int i = tid; i < n_from * deep; i += kLogitThreads) {
                    const int x0 = first + 8 * (s_from[i % n_from] + i / n_from * kLogitThreads);
                    if (x0 >= stop) continue;
                    Chunk<T> c;
                    float f[8];
                    load(x0, c);
                    c.get(f);
                    taken(x0, f);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (f[j] > -INFINITY) {
                            const uint64_t key = key_of(f[j], x0 + j);
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
            if (row % split == (int)blockIdx.x && warp < 1 + (kMaxSplit * kMaxBest) / 32) {
                uint64_t* all = s_first;  // (its readers are behind a barrier)
                const int n = split * a.k;
                for (int i = tid; i < n; i += 32 * (1 + (kMaxSplit * kMaxBest) / 32))
                    all[i] = split > 1 ? peer_load(&part.best[i % a.k], i / a.k) : part.best[i % a.k];
                float m = -INFINITY, s = 0.f;
                if (lane < split) {
                    const uint64_t u = split > 1 ? peer_load(&part.sum, lane) : part.sum;
                    m = __uint_as_float((uint32_t)(u >> 32)), s = __uint_as_float((uint32_t)u);
                }
                const float top = warp_max(m);
                const float log_sum = logf(warp_sum(m > -INFINITY ? s * weight(m, top) : 0.f));
                asm volatile("bar.sync 1, %0;\n" ::"n"(32 * (1 + (kMaxSplit * kMaxBest) / 32)) : "memory");
                for (int i = tid; i < n; i += 32 * (1 + (kMaxSplit * kMaxBest) / 32)) {
                    const uint64_t key = all[i];
                    int rank = 0;
                    for (int j = 0; j < n; ++j) rank += all[j] > key || (all[j] == key && j < i);  // (only keys of 0 are equal)
                    if (rank < a.k) {
                        const float v = of_order((uint32_t)(key >> 32));
                        a.tokens[(int64_t)row * a.k + rank] = key ? (int)~(uint32_t)key : -1;
                        a.logprob[(int64_t)row * a.k + rank] = key ? (v == top ? 0.f : v - top) - log_sum : -INFINITY;
                    }
                }
                if (tid == 0 && a.total) a.total[row] = top > -INFINITY ? top + log_sum : -INFINITY;
            }
            __syncthreads();
        }
    }
    if (kChoose && split > 1) cluster_sync();  // (no CTA leaves while another may read its part)
}

int smem_of(int slice) { return 4 * ((slice + 8 + 31) / 32 + slice + 8); }

template <typename T>
int set_up() {
    const int most = smem_of(kMaxSlice);
    cudaError_t e = cudaFuncSetAttribute(logits_kernel<T, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(logits_kernel<T, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    return (int)e;
}

int check_rules(const char* call, const ssd_logit_rules* r, int dtype, const void* logits, int64_t stride) {
    if (!r) return refuse_arg(call, "NULL rules");
    if (dtype != SSD_F32 && dtype != SSD_F16 && dtype != SSD_BF16) return refuse_arg(call, "logits are fp32, fp16 or bf16");
    if (r->vocab < 1 || r->vocab > kMaxVocab) return refuse_arg(call, "need 1 <= vocab <= 262144");
    if (r->n_rows < 0 || r->max_rows < 1) return refuse_arg(call, "need n_rows >= 0 and max_rows >= 1");
    if (r->n_rows == 0) return SSD_OK;
    if (r->row_start ? r->n_requests < 1 || r->n_requests > kMaxRequests : r->n_requests != r->n_rows)
        return refuse_arg(call, "need 1 <= n_requests <= 4096, or without row_start n_requests = n_rows");
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

int launch_logits(const char* call, LogitArgs& a, int dtype, bool choose, void* stream) {
    const ssd_logit_rules& r = a.r;
    int dev = 0;
    if (int rc = check_device(call, a.logits)) return rc;
    if (cudaGetDevice(&dev) != cudaSuccess) return refuse(SSD_ERR_CUDA, call, "no device");
    static int ready[64][3] = {};  // (set once a device and type; setting it twice is harmless)
    if (dev < 64 && !ready[dev][dtype]) {
        const int e = dtype == SSD_F32 ? set_up<float>() : dtype == SSD_F16 ? set_up<f16>() : set_up<bf16>();
        if (e) return refuse(SSD_ERR_CUDA, call, "%s", cudaGetErrorString((cudaError_t)e));
        ready[dev][dtype] = 1;
    }
    a.counted = (r.repetition || r.presence || r.frequency) && (r.history || r.tokens);
    // slices of at most 32768 tokens, and until there are two CTAs for an SM, of at least 2048
    auto slice_of = [&](int split) { return ((r.vocab + 7 + split - 1) / split + 63) / 64 * 64; };
    int split = 1;
    while (slice_of(split) > kMaxSlice) split *= 2;
    while (split < kMaxSplit && (long long)r.n_rows * split < 304 && r.vocab > 2048 * split) split *= 2;
    a.slice = slice_of(split);
    if (a.slice > kMaxSlice) a.slice = kMaxSlice;
    // rows of a request share their counts: as many to a cluster as leaves two CTAs for an SM
    a.rows = a.counted ? (int)std::min<long long>(r.max_rows, std::max(1ll, (long long)r.n_rows * split / 304)) : 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)split, (unsigned)((r.n_rows + a.rows - 1) / a.rows), 1);
    if (cfg.gridDim.y > 65535u) {
        a.rows = (r.n_rows + 65534) / 65535;
        cfg.gridDim.y = (unsigned)((r.n_rows + a.rows - 1) / a.rows);
    }
    cfg.blockDim = dim3(kLogitThreads, 1, 1);
    cfg.dynamicSmemBytes = a.counted ? (size_t)smem_of(a.slice) : 0;
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)split, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = choose && split > 1 ? 2 : 1;
    cudaError_t e;
    if (choose) {
        e = dtype == SSD_F32 ? cudaLaunchKernelEx(&cfg, logits_kernel<float, true>, a) : dtype == SSD_F16 ? cudaLaunchKernelEx(&cfg, logits_kernel<f16, true>, a)
                                                                                                          : cudaLaunchKernelEx(&cfg, logits_kernel<bf16, true>, a);
    } else {
        e = dtype == SSD_F32 ? cudaLaunchKernelEx(&cfg, logits_kernel<float, false>, a) : dtype == SSD_F16 ? cudaLaunchKernelEx(&cfg, logits_kernel<f16, false>, a)
                                                                                                           : cudaLaunchKernelEx(&cfg, logits_kernel<bf16, false>, a);
    }
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
    const size_t n = 4 * (size_t)rules->n_rows, rows = span(rules->n_rows, stride, rules->vocab, dtype);
    if (meet(tokens, n * k, logprob, n * k) || meet(tokens, n * k, total, n) || meet(logprob, n * k, total, n) || meet(tokens, n * k, logits, rows) ||
        meet(logprob, n * k, logits, rows) || meet(total, n, logits, rows) || meet(tokens, n * k, rules->tokens, n))
        return refuse_arg(call, "the results must overlap neither each other, nor the logits or the nodes' tokens");
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
