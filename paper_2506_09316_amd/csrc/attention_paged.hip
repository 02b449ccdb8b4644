// Softmax attention of the last tokens of every sequence over a paged cache (include/dsla.h: dsla_attention_paged).
#include <cfloat>

#include "paged_common.h"

namespace dsla {
namespace {

// One query of one head: a workgroup.  A lane holds one key at a time: its score is a sum over the features; scores of 256 keys
// go to LDS, and the workgroup's threads then take features of the values.
template <int D, class TIO>
__global__ __launch_bounds__(256) void attention_paged_plain_kernel(CacheArgs c, BatchArgs x, int H, int max_n, float scale_log2e, const TIO *q,
                                                                    const TIO *k_pages, const TIO *v_pages, const uint64_t *tree, TIO *o)
{
    __shared__ float s_q[D], s_p[256], s_red[256], s_acc[256];
    __shared__ int s_page[256];
    const int h = blockIdx.x % H, j = (blockIdx.x / H) % max_n, b = blockIdx.x / H / max_n, tid = threadIdx.x;
    const Entry e = read_entry(x, c, b);
    const int start = x.start[b];
    if (!e.ok || e.n > max_n || static_cast<long long>(start) + e.n > row_room(c)) {
        if (tid == 0 && (!e.ok || start >= 0)) report(c.status, DSLA_STATUS_CACHE_ENTRY);
        return;
    }
    if (start < 0 || j >= e.n) return;
    const int kv = h / (H / c.H_kv), L = start + e.n, page = 1 << c.page_log2;
    const size_t at = (static_cast<size_t>(e.cu + j) * H + h) * D;
    for (int f = tid; f < D; f += 256) s_q[f] = to_f32(q[at + f]) * scale_log2e;
    const uint64_t mask = tree ? tree[e.cu + j] : ~0ull >> (63 - j);
    constexpr int SPLIT = 256 / D;
    float m = -FLT_MAX, z = 0.f, acc = 0.f;
    for (int t0 = 0; t0 < L; t0 += 256) {
        __syncthreads();
        const int t = t0 + tid;
        float s = -INFINITY;
        int p = -1;
        if (t < L && (t < start || (mask >> (t - start) & 1))) {
            p = page_of(c, e.row, t);
            if (p < 0) {
                report(c.status, DSLA_STATUS_CACHE_ENTRY);
            } else {
                const TIO *kp = k_pages + (((static_cast<size_t>(p) * c.H_kv + kv) << c.page_log2) + (t & (page - 1))) * D;
                s = 0.f;
                for (int f = 0; f < D; ++f) s = fmaf(s_q[f], to_f32(kp[f]), s);
            }
        }
        s_red[tid] = s;
        s_page[tid] = p;
        __syncthreads();
        for (int n = 128; n > 0; n >>= 1) {
            if (tid < n) s_red[tid] = fmaxf(s_red[tid], s_red[tid + n]);
            __syncthreads();
        }
        const float top = fmaxf(m, s_red[0]), c0 = exp2f(m - top);
        m = top;
        s_p[tid] = p >= 0 ? exp2f(s - m) : 0.f;
        __syncthreads();
        z *= c0;
        acc *= c0;
        const int f = tid % D;
        for (int i = tid / D; i < 256; i += SPLIT)
            if (s_page[i] >= 0) {
                const int u = t0 + i;
                z += s_p[i];
                acc = fmaf(s_p[i], to_f32(v_pages[(((static_cast<size_t>(s_page[i]) * c.H_kv + kv) << c.page_log2) + (u & (page - 1))) * D + f]), acc);
            }
    }
    __syncthreads();
    s_red[tid] = z;
    s_acc[tid] = acc;
    __syncthreads();
    if (tid < D) {
        for (int i = 1; i < SPLIT; ++i) {
            z += s_red[tid + i * D];
            acc += s_acc[tid + i * D];
        }
        o[at + tid] = from_f32<TIO>(z > 0.f || z != z ? acc / z : 0.f);
    }
}

}  // namespace

size_t attention_paged_workspace_bytes(const dsla_cache &, const dsla_batch &, int, int64_t) { return 0; }

template <int D, class TIO>
hipError_t launch_t(const dsla_cache &c, const dsla_batch &x, int H, float scale, const void *q, const void *k_pages, const void *v_pages,
                    const uint64_t *tree, void *o, hipStream_t stream)
{
    ProfileScope ps(DSLA_KERNEL_ATTENTION_PAGED, stream);
    DSLA_LAUNCH(ps, (attention_paged_plain_kernel<D, TIO>), dim3(static_cast<unsigned>(x.B) * x.max_n * H), dim3(256), 0, stream, args_of(c), args_of(x),
                H, static_cast<int>(x.max_n), scale * 1.44269504088896341f, static_cast<const TIO *>(q), static_cast<const TIO *>(k_pages),
                static_cast<const TIO *>(v_pages), tree, static_cast<TIO *>(o));
    return hipGetLastError();
}

hipError_t launch_attention_paged(const dsla_cache &c, const dsla_batch &x, int H, int64_t, float scale, const void *q, const void *k_pages,
                                  const void *v_pages, const uint64_t *tree, void *o, void *, hipStream_t stream)
{
    if (c.dtype == DSLA_BF16)
        return c.d == 128 ? launch_t<128, bf16_t>(c, x, H, scale, q, k_pages, v_pages, tree, o, stream)
                          : launch_t<64, bf16_t>(c, x, H, scale, q, k_pages, v_pages, tree, o, stream);
    return c.d == 128 ? launch_t<128, float>(c, x, H, scale, q, k_pages, v_pages, tree, o, stream)
                      : launch_t<64, float>(c, x, H, scale, q, k_pages, v_pages, tree, o, stream);
}

}  // namespace dsla
