// step_heads.cu - per-head norms and rotary positions on several axes with the
// write of keys and values (ssd_norm_rope_kv of ssd_step.h).
#include <algorithm>
#include <cmath>

#include "step_ops.cuh"

namespace ssd {
namespace step {

constexpr int kHeadAhead = 4, kValueAhead = 4;  // heads under way in a lane

struct HeadArgs {
    const void *q, *k, *v;
    void* q_out;
    int64_t q_stride, k_stride, v_stride, q_out_stride;  // elements
    const int32_t *positions, *slots;
    void *kc, *vc;  // the layer's cache
    int64_t page_stride, head_stride, pos_stride;
    const float *q_gain, *k_gain;  // nullptr: no norm
    float eps;
    int n_rows, n_heads, n_kv_heads, hd, page_size, n_pages;
    ssd_rope rope;
    uint8_t axis[64];
};

// A CTA takes a row (blockIdx.x), or with gridDim.y > 1 a share of its heads; hd / V lanes hold a
// head, 16 bytes each, so that the sum of squares is a few shuffles and every byte is read once.
// Rotated dim e with partner p becomes r (x_e g_e cos +- x_p g_p sin), r = 1 / sqrt(mean x^2 + eps): the
// products of gains and angles are formed once a row in shared memory (a, b; pair p's by thread p, so that one barrier does), and the
// partner's 16 bytes come from the lane that holds them.  Bound by HBM, for 16-bit rows of few heads by instructions (16000 fp16 rows: issue slots 73 %, then the table's
// reads from shared memory), for few rows by the chain position - angle - table - store.  Measured: 4095 fp32 rows of 32 + 2 x 32 heads of 128 60.7 us (335 MB, 5.5 TB/s, 82 % of the copy rate); 16000 fp16
// rows of 32 + 2 x 8 heads 84.4 us (394 MB, 4.7 TB/s); 403 fp16 rows 6.0; one row 2.8.  (Angles first, then each dim's products behind a second
// barrier: 63.8, 90.0, 7.1, 3.5.  CTAs that stay for several rows, the next one's table and loads under way: 77, 106.)
//
// T: rows, C: cache
template <typename T, typename C, int kHeadThreads>
__global__ void __launch_bounds__(kHeadThreads, 1024 / kHeadThreads) heads_kernel(const __grid_constant__ HeadArgs a) {
    constexpr int V = Vec<T>::N;
    __shared__ __align__(16) float s_a[2][128], s_b[2][128];  // [q, k][dim]
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x, rot = a.rope.rot_dim, half = rot / 2, tid = threadIdx.x;
    const int per = a.hd / V, c = tid % per, e = c * V;  // lanes of a head (8, 16 or 32), this one's place
    const int line = (blockIdx.y * kHeadThreads + tid) / per, step = kHeadThreads * gridDim.y / per;
    const int heads = a.n_heads + a.n_kv_heads;
    auto source = [&](int h) {
        return h < a.n_heads ? (const T*)a.q + (int64_t)row * a.q_stride + (int64_t)h * a.hd + e
                             : (const T*)a.k + (int64_t)row * a.k_stride + (int64_t)(h - a.n_heads) * a.hd + e;
    };
    uint4 x[kHeadAhead], y[kValueAhead];
    auto load = [&](int h0) {
#pragma unroll
        for (int i = 0; i < kHeadAhead; ++i)
            if (h0 + i * step < heads) x[i] = __ldcg(reinterpret_cast<const uint4*>(source(h0 + i * step)));
    };
    auto load_values = [&](int h0) {
        const T* v = (const T*)a.v + (int64_t)row * a.v_stride + e;
#pragma unroll
        for (int i = 0; i < kValueAhead; ++i)
            if (h0 + i * step < a.n_kv_heads) y[i] = __ldcg(reinterpret_cast<const uint4*>(v + (int64_t)(h0 + i * step) * a.hd));
    };
    // the first heads and values are on their way while the row's position becomes angles
    const int slot = __ldcg(a.slots + row);
    const int64_t position = tid < half ? __ldcg(a.positions + (int64_t)a.axis[tid] * a.n_rows + row) : 0;
    load(line);
    load_values(line);
    // thread p has pair p, in both of its dims
    if (tid < half) {
        const int d0 = a.rope.interleaved ? 2 * tid : tid, d1 = a.rope.interleaved ? 2 * tid + 1 : tid + half;
        float g[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float* gain = i ? a.k_gain : a.q_gain;
            g[i][0] = gain ? __ldcg(gain + d0) : 1.f, g[i][1] = gain ? __ldcg(gain + d1) : 1.f;
        }
        const uint64_t turn = (uint64_t)position * a.rope.turns[tid];
        float s, c;
        sincospif((float)((int64_t)turn >> 32) * 0x1p-31f, &s, &c);
        s *= a.rope.amplitude, c *= a.rope.amplitude;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s_a[i][d0] = c * g[i][0], s_a[i][d1] = c * g[i][1];
            s_b[i][d0] = -s * g[i][1], s_b[i][d1] = s * g[i][0];
        }
    }
    for (int d = rot + (kHeadThreads - 1 - tid); d < a.hd; d += kHeadThreads) {
        s_a[0][d] = a.q_gain ? __ldcg(a.q_gain + d) : 1.f, s_a[1][d] = a.k_gain ? __ldcg(a.k_gain + d) : 1.f;
        s_b[0][d] = s_b[1][d] = 0.f;
    }
    const bool cached = slot >= 0 && slot < a.n_pages * a.page_size;
    const int64_t at = cached ? (int64_t)(slot / a.page_size) * a.page_stride + (int64_t)(slot % a.page_size) * a.pos_stride : 0;
    auto to_cache = [&](void* base, int head, int e, const float (&f)[V]) {
        if (!cached) return;
        C* p = (C*)base + at + (int64_t)head * a.head_stride + e;
        if constexpr (V == 8) *reinterpret_cast<uint4*>(p) = Vec<C>::put(f);
        else *reinterpret_cast<uint2*>(p) = make_uint2(pack2(f[0], f[1], C()), pack2(f[2], f[3], C()));
    };
    for (int h = line; h < a.n_kv_heads; h += kValueAhead * step) {
        if (h != line) load_values(h);
#pragma unroll
        for (int i = 0; i < kValueAhead; ++i)
            if (h + i * step < a.n_kv_heads) {
                float f[V];
                Vec<T>::get(y[i], f);
                to_cache(a.vc, h + i * step, e, f);
            }
    }
    __syncthreads();
    // where the partners of this lane's dims are: its own 16 bytes (neighbours), or another lane's
    const bool rotated = e < rot;
    const int lane = tid % 32, other = a.rope.interleaved || !rotated ? lane : e < half ? lane + half / V : lane - half / V;
    const float inv_hd = 1.f / (float)a.hd;
    const int first_line = (blockIdx.y * kHeadThreads + tid / 32 * 32) / per;  // of the warp
    for (int h0 = line, w0 = first_line; w0 < heads; h0 += kHeadAhead * step, w0 += kHeadAhead * step) {
        if (h0 != line) load(h0);
        // (all lanes of a warp take part in the shuffles; those without a head shuffle what they hold)
        float r[kHeadAhead];
#pragma unroll
        for (int i = 0; i < kHeadAhead; ++i) {
            r[i] = 0.f;
            if (w0 + i * step >= heads) break;
            if (h0 + i * step >= heads) x[i] = make_uint4(0u, 0u, 0u, 0u);
            float f[V];
            Vec<T>::get(x[i], f);
            uint64_t s = 0ull;
#pragma unroll
            for (int j = 0; j < V; j += 2) {
                const uint64_t v = pair_of(f[j], f[j + 1]);
                s = fma_pair(v, v, s);
            }
            const float2 both = of_pair(s);
            r[i] = both.x + both.y;
        }
        if (a.q_gain || a.k_gain) {
            for (int o = per / 2; o > 0; o >>= 1)
#pragma unroll
                for (int i = 0; i < kHeadAhead; ++i) r[i] += __shfl_xor_sync(0xffffffffu, r[i], o);
        }
#pragma unroll
        for (int i = 0; i < kHeadAhead; ++i) {
            const int h = h0 + i * step;
            if (w0 + i * step >= heads) break;
            uint4 y;
            y.x = __shfl_sync(0xffffffffu, x[i].x, other);
            y.y = __shfl_sync(0xffffffffu, x[i].y, other);
            y.z = __shfl_sync(0xffffffffu, x[i].z, other);
            y.w = __shfl_sync(0xffffffffu, x[i].w, other);
            if (h >= heads) continue;
            const int kind = h < a.n_heads ? 0 : 1;
            const float scale = (kind ? a.k_gain : a.q_gain) ? rsqrtf(fmaf(r[i], inv_hd, a.eps)) : 1.f;
            float f[V], g[V], o[V];
            Vec<T>::get(x[i], f);
            Vec<T>::get(y, g);
            const uint64_t both = pair_of(scale, scale);
#pragma unroll
            for (int j = 0; j < V; j += 4) {
                const ulonglong2 A = *reinterpret_cast<const ulonglong2*>(&s_a[kind][e + j]);
                uint64_t u = mul_pair(pair_of(f[j], f[j + 1]), A.x), w = mul_pair(pair_of(f[j + 2], f[j + 3]), A.y);
                if (rotated) {
                    const ulonglong2 B = *reinterpret_cast<const ulonglong2*>(&s_b[kind][e + j]);
                    u = fma_pair(a.rope.interleaved ? pair_of(f[j + 1], f[j]) : pair_of(g[j], g[j + 1]), B.x, u);
                    w = fma_pair(a.rope.interleaved ? pair_of(f[j + 3], f[j + 2]) : pair_of(g[j + 2], g[j + 3]), B.y, w);
                }
                const float2 p = of_pair(mul_pair(u, both)), q = of_pair(mul_pair(w, both));
                o[j] = p.x, o[j + 1] = p.y, o[j + 2] = q.x, o[j + 3] = q.y;
            }
            if (kind) to_cache(a.kc, h - a.n_heads, e, o);
            else *reinterpret_cast<uint4*>((T*)a.q_out + (int64_t)row * a.q_out_stride + (int64_t)h * a.hd + e) = Vec<T>::put(o);
        }
    }
}

}  // namespace step
}  // namespace ssd

using namespace ssd;
using namespace ssd::step;

template <int kThreads>
static int start(const char* call, const HeadArgs& a, int dtype, int split, void* stream) {
    const dim3 grid((unsigned)a.n_rows, (unsigned)split);
    if (dtype == SSD_F32) return launch(call, heads_kernel<float, f16, kThreads>, grid, kThreads, 0, stream, a);
    if (dtype == SSD_F16) return launch(call, heads_kernel<f16, f16, kThreads>, grid, kThreads, 0, stream, a);
    return launch(call, heads_kernel<bf16, bf16, kThreads>, grid, kThreads, 0, stream, a);
}

static bool rope_ok(const ssd_rope* rope, int most) {
    return rope && rope->rot_dim >= 16 && rope->rot_dim % 16 == 0 && rope->rot_dim <= most;
}

extern "C" int ssd_rope_axes_init(const ssd_rope* rope, int layout, int n_axes, const int* pairs, ssd_rope_axes* out) {
    static const char call[] = "ssd_rope_axes_init";
    if (!out || !pairs) return refuse_arg(call, "NULL pointer");
    if (!rope_ok(rope, 128)) return refuse_arg(call, "rope must come from ssd_rope_init");
    if (layout != SSD_AXES_SECTIONS && layout != SSD_AXES_IN_TURNS) return refuse_arg(call, "unknown layout");
    if (n_axes < 1 || n_axes > 4) return refuse_arg(call, "need 1 .. 4 axes");
    const int half = rope->rot_dim / 2;
    int left = half;
    for (int i = 0; i < n_axes; ++i) {
        if (pairs[i] < 0 || pairs[i] > left) return refuse_arg(call, "pairs must be counts that add up to rot_dim / 2");
        left -= pairs[i];
    }
    if (left) return refuse_arg(call, "pairs must be counts that add up to rot_dim / 2");
    ssd_rope_axes r{};
    r.n_axes = n_axes;
    if (layout == SSD_AXES_SECTIONS) {
        for (int a = 0, i = 0; a < n_axes; ++a)
            for (int j = 0; j < pairs[a]; ++j) r.axis[i++] = (uint8_t)a;
    } else {
        for (int i = 0; i < half; ++i) r.axis[i] = (uint8_t)(i / n_axes < pairs[i % n_axes] ? i % n_axes : 0);
    }
    *out = r;
    return SSD_OK;
}

extern "C" int ssd_norm_rope_kv(const ssd_pages* cache, int layer, const ssd_rope* rope, const ssd_rope_axes* axes,
                                const ssd_head_norm* norm, int dtype, int n_rows, int n_heads, const void* q, int64_t q_stride,
                                const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* positions,
                                const int32_t* slots, void* q_out, int64_t q_out_stride, void* cuda_stream) {
    static const char call[] = "ssd_norm_rope_kv";
    if (int rc = check_pages(call, cache)) return rc;
    if (layer < 0 || layer >= cache->n_layers) return refuse_arg(call, "no such layer");
    if (int rc = check_rows_type(call, dtype, cache)) return rc;
    if (!rope_ok(rope, cache->head_dim)) return refuse_arg(call, "rope must come from ssd_rope_init, with rot_dim <= head_dim");
    HeadArgs a{};
    if (axes) {
        if (axes->n_axes < 1 || axes->n_axes > 4) return refuse_arg(call, "axes must come from ssd_rope_axes_init");
        for (int i = 0; i < rope->rot_dim / 2; ++i) {
            if (axes->axis[i] >= axes->n_axes) return refuse_arg(call, "axes must come from ssd_rope_axes_init");
            a.axis[i] = axes->axis[i];
        }
    }
    if (norm && (norm->q_gain || norm->k_gain)) {
        if (!(norm->eps > 0.f) || !std::isfinite(norm->eps)) return refuse_arg(call, "need eps > 0, finite");
        if (((uintptr_t)norm->q_gain | (uintptr_t)norm->k_gain) & 15u) return refuse_arg(call, "gains must be 16-byte aligned");
        a.q_gain = norm->q_gain;
        a.k_gain = norm->k_gain;
        a.eps = norm->eps;
    }
    if (n_rows < 0 || n_heads < 1 || n_heads > 65536) return refuse_arg(call, "need n_rows >= 0 and 1 <= n_heads <= 65536");
    if (n_rows == 0) return SSD_OK;
    if (!q || !k || !v || !positions || !slots || !q_out) return refuse_arg(call, "NULL pointer");
    if (!aligned(4, {positions, slots})) return refuse_arg(call, "positions and slots must be aligned to their type");
    const int hd = cache->head_dim;
    if (int rc = check_rows(call, "q", q, q_stride, dtype, (int64_t)n_heads * hd)) return rc;
    if (int rc = check_rows(call, "q_out", q_out, q_out_stride, dtype, (int64_t)n_heads * hd)) return rc;
    if (int rc = check_rows(call, "k", k, k_stride, dtype, (int64_t)cache->n_kv_heads * hd)) return rc;
    if (int rc = check_rows(call, "v", v, v_stride, dtype, (int64_t)cache->n_kv_heads * hd)) return rc;
    if (q == q_out && q_stride != q_out_stride) return refuse_arg(call, "q_out in q's place needs its stride");
    const size_t row_bytes = dtype == SSD_F32 ? 4 : 2, n = 4 * (size_t)n_rows;
    const Range o[1] = {{q_out, span(n_rows, q_out_stride, (int64_t)n_heads * hd, dtype)}};
    const Range in[4] = {{positions, n * (axes ? axes->n_axes : 1)}, {slots, n}, {a.q_gain, 4 * (size_t)hd}, {a.k_gain, 4 * (size_t)hd}};
    // (k and v may lie between the rows of q in one tensor: the first row tells)
    if (meet(o, in) || meet(q_out, row_bytes * n_heads * hd, k, row_bytes * cache->n_kv_heads * hd) || meet(q_out, row_bytes * n_heads * hd, v, row_bytes * cache->n_kv_heads * hd) ||
        (q_out != q && meet(q_out, row_bytes * n_heads * hd, q, row_bytes * n_heads * hd)))
        return refuse_arg(call, "q_out must be q with its stride or overlap no input");
    if (int rc = check_device(call, cache->k)) return rc;
    if (int rc = set_up_once<heads_kernel<float, f16, 64>, heads_kernel<f16, f16, 64>, heads_kernel<bf16, bf16, 64>, heads_kernel<float, f16, 128>, heads_kernel<f16, f16, 128>,
                             heads_kernel<bf16, bf16, 128>>(call))
        return rc;
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_out = q_out;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.q_out_stride = q_out_stride;
    a.positions = positions;
    a.slots = slots;
    a.kc = (char*)cache->k + 2 * layer * cache->layer_stride;
    a.vc = (char*)cache->v + 2 * layer * cache->layer_stride;
    a.page_stride = cache->page_stride;
    a.head_stride = cache->head_stride;
    a.pos_stride = cache->pos_stride;
    a.n_rows = n_rows;
    a.n_heads = n_heads;
    a.n_kv_heads = cache->n_kv_heads;
    a.hd = hd;
    a.page_size = cache->page_size;
    a.n_pages = cache->n_pages;
    a.rope = *rope;
    // few rows: a row's heads over several CTAs, until there are four per SM.  Many rows of few heads: half as many threads each, since what
    // a warp does once a row is half of its instructions (16000 bf16 rows of 32 + 8 heads of 128 84.5 us, 128 threads 96; 4095 of them 26.3,
    // 128 threads 28.7; of 32 + 32 heads, with a longer start of a row, 42, 128 threads 41).
    const int per16 = dtype == SSD_F32 ? 4 : 8;
    const long long units = (long long)(n_heads + cache->n_kv_heads) * hd / per16;
    if (n_rows >= 2432 && units < 1024) return start<64>(call, a, dtype, 1, cuda_stream);
    int split = 1;
    while (split < 64 && (long long)n_rows * split < 608 && units > 128ll * split) split *= 2;
    return start<128>(call, a, dtype, split, cuda_stream);
}
