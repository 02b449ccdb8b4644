// Norm and rotation of q and k for every head, keys and values written into the pages of a cache (include/dsla.h:
// dsla_qk_rope).  A lane holds 8 + 8 features of a head: with pairs (i, i + rot/2) piece p of 8 features goes with piece p +
// rot/16, with pairs (2i, 2i + 1) with its neighbour, so that both halves of every pair and the cosines of pairs 8 c .. 8 c + 7
// are the lane's own, c = 0 .. d/16 - 1; the d/16 lanes of a head exchange only its sum of squares.
#include "paged_common.h"

namespace dsla {
namespace {

struct RopeArgs {
    const void *q, *k, *v;
    void *q_out, *k_out, *k_pages, *v_pages;
    const float *inv_freq, *q_weight, *k_weight;
    const int32_t *offsets;
    int H, H_kv, rot, first;
    float eps;
    bool cached, interleaved;
    CacheArgs c;
    BatchArgs x;
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Everything is read once and written once, whole rows at a time: with the non-temporal hint on both 16000 tokens take 70 to 74 us (5.3 to 5.6 TB/s; a
// plain copy of as many bytes 5.5, one with the same hints 6.1), on the stores only 77, on the loads only 81, without 80.
__device__ __forceinline__ void load8(const bf16_t *p, float (&f)[8])
{
    const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float *p, float (&f)[8])
{
    const f32x4 a = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(p)), b = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(p + 4));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i] = a[i];
        f[4 + i] = b[i];
    }
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&f)[8])
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = f32_to_bf16_bits(f[2 * i]) | static_cast<uint32_t>(f32_to_bf16_bits(f[2 * i + 1])) << 16;
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(p));
}
__device__ __forceinline__ void store8(float *p, const float (&f)[8])
{
    __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, reinterpret_cast<f32x4 *>(p));
    __builtin_nontemporal_store(f32x4{f[4], f[5], f[6], f[7]}, reinterpret_cast<f32x4 *>(p + 4));
}

// Cosine and sine of position * freq: the turns and their fraction in 64 bits (a far position in 32 bits has no fraction left).
__device__ __forceinline__ void angle_of(long long position, float freq, float *cos, float *sin)
{
    const double turns = static_cast<double>(position) * static_cast<double>(freq) * 0.15915494309189533577;   // 1 / (2 pi)
    sincospif(static_cast<float>(2.0 * (turns - rint(turns))), sin, cos);
}

template <int D, class TIO>
__global__ __launch_bounds__(256) void qk_rope_kernel(RopeArgs a)
{
    constexpr int LPR = D / 16, ROWS = 256 / LPR;   // lanes of a head; heads at a time
    __shared__ float s_cos[D / 2], s_sin[D / 2];
    const int m = a.first + blockIdx.x;
    // the token's entry, its place in the sequence and its page
    long long place = 0, position = a.offsets ? a.offsets[m] : m;
    int page = -1;
    if (a.cached) {
        int b = m;
        if (a.x.cu) {   // the last entry that begins at m or before
            int lo = 0, hi = a.x.B;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (a.x.cu[mid] <= m) lo = mid;
                else hi = mid;
            }
            b = lo;
        }
        const Entry e = read_entry(a.x, a.c, b);
        const int start = a.x.start[b], j = m - e.cu;
        if (!e.ok) {
            if (threadIdx.x == 0 && blockIdx.y == 0) report(a.c.status, DSLA_STATUS_CACHE_ENTRY);
            return;
        }
        if (start < 0 || j < 0 || j >= e.n) return;
        place = static_cast<long long>(start) + j;
        position = static_cast<long long>(start) + (a.offsets ? a.offsets[m] : j);
        page = place < row_room(a.c) ? page_of(a.c, e.row, static_cast<int>(place)) : -1;
        if (page < 0 && threadIdx.x == 0 && blockIdx.y == 0) report(a.c.status, DSLA_STATUS_CACHE_ENTRY);
    }
    for (int i = threadIdx.x; i < a.rot / 2; i += 256) angle_of(position, a.inv_freq[i], &s_cos[i], &s_sin[i]);
    __syncthreads();

    const int c = threadIdx.x % LPR, in_page = static_cast<int>(place & ((1 << a.c.page_log2) - 1));
    // the lane's two pieces: with halves the first rot/16 lanes hold what is rotated
    const int rotated = a.rot / 16;
    const bool turns = c < rotated;
    const int p0 = a.interleaved || !turns ? 2 * c : c, p1 = a.interleaved || !turns ? 2 * c + 1 : c + rotated;
    const int heads = a.H + a.H_kv + (a.cached ? a.H_kv : 0);
    for (int r = blockIdx.y * ROWS + threadIdx.x / LPR; r < heads; r += gridDim.y * ROWS) {   // (the lanes of a head stay together)
        const bool is_q = r < a.H, is_v = r >= a.H + a.H_kv;
        const int h = is_q ? r : is_v ? r - a.H - a.H_kv : r - a.H;
        const TIO *src = static_cast<const TIO *>(is_q ? a.q : is_v ? a.v : a.k) + (static_cast<size_t>(m) * (is_q ? a.H : a.H_kv) + h) * D;
        float u[8], w[8];
        load8(src + 8 * p0, u);
        load8(src + 8 * p1, w);
        if (!is_v) {
            const float *weight = is_q ? a.q_weight : a.k_weight;
            if (weight) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fmaf(u[i], u[i], fmaf(w[i], w[i], sum));
#pragma unroll
                for (int off = 1; off < LPR; off <<= 1) sum += __shfl_xor(sum, off);
                const float inv = 1.0f / sqrtf(sum * (1.0f / D) + a.eps);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    u[i] *= inv * weight[8 * p0 + i];
                    w[i] *= inv * weight[8 * p1 + i];
                }
            }
            if (turns) {
                if (a.interleaved) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float c0 = s_cos[8 * c + i], s0 = s_sin[8 * c + i], c1 = s_cos[8 * c + 4 + i], s1 = s_sin[8 * c + 4 + i];
                        const float x0 = u[2 * i], x1 = w[2 * i];
                        u[2 * i] = x0 * c0 - u[2 * i + 1] * s0;
                        u[2 * i + 1] = x0 * s0 + u[2 * i + 1] * c0;
                        w[2 * i] = x1 * c1 - w[2 * i + 1] * s1;
                        w[2 * i + 1] = x1 * s1 + w[2 * i + 1] * c1;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float cs = s_cos[8 * c + i], sn = s_sin[8 * c + i], x0 = u[i];
                        u[i] = x0 * cs - w[i] * sn;
                        w[i] = x0 * sn + w[i] * cs;
                    }
                }
            }
        }
        if (is_q) {
            TIO *to = static_cast<TIO *>(a.q_out) + (static_cast<size_t>(m) * a.H + h) * D;
            store8(to + 8 * p0, u);
            store8(to + 8 * p1, w);
        } else {
            if (page >= 0) {
                TIO *to = static_cast<TIO *>(is_v ? a.v_pages : a.k_pages) +
                          (((static_cast<size_t>(page) * a.H_kv + h) << a.c.page_log2) + in_page) * D;
                store8(to + 8 * p0, u);
                store8(to + 8 * p1, w);
            }
            if (!is_v && a.k_out) {
                TIO *to = static_cast<TIO *>(a.k_out) + (static_cast<size_t>(m) * a.H_kv + h) * D;
                store8(to + 8 * p0, u);
                store8(to + 8 * p1, w);
            }
        }
    }
}

}  // namespace

hipError_t launch_qk_rope(const dsla_rope &r, int64_t rows, const void *q, const void *k, const void *v, void *q_out, void *k_out,
                          const dsla_cache *c, const dsla_batch *x, void *k_pages, void *v_pages, hipStream_t stream)
{
    RopeArgs a = {};
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_out = q_out;
    a.k_out = k_out;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.inv_freq = r.inv_freq;
    a.q_weight = r.q_weight;
    a.k_weight = r.k_weight;
    a.offsets = r.offsets;
    a.H = r.H;
    a.H_kv = r.H_kv;
    a.rot = r.rot_dim;
    a.eps = r.eps;
    a.cached = c != nullptr;
    a.interleaved = r.interleaved != 0;
    if (c) {
        a.c = args_of(*c);
        a.x = args_of(*x);
    }
    const bool bf16 = r.io_dtype == DSLA_BF16;
    auto kernel = bf16 ? (r.d == 128 ? qk_rope_kernel<128, bf16_t> : qk_rope_kernel<64, bf16_t>)
                       : (r.d == 128 ? qk_rope_kernel<128, float> : qk_rope_kernel<64, float>);
    // A workgroup to a token: what it reads of the token is uniform and read before anything is written, by scalar loads (in a loop over
    // tokens these are vector loads: 16000 tokens 94 us instead of 78).  Where there are few, one to every chunk of a token's heads (48 heads of
    // 128, with chunks / without: 1 token 3.5 / 4.0 us, 64 4.3 / 5.1, 512 5.4 / 5.8, 1024 9.1 / 8.2).
    const int heads = r.H + r.H_kv + (c ? r.H_kv : 0), at_a_time = 256 / (r.d / 16);
    const unsigned chunks = rows <= 512 ? (heads + at_a_time - 1) / at_a_time : 1;
    constexpr int64_t kMost = 1 << 23;   // threads of a launch are a 32-bit number
    for (int64_t first = 0; first < rows; first += kMost) {
        a.first = static_cast<int>(first);
        const int64_t n = rows - first < kMost ? rows - first : kMost;
        ProfileScope ps(DSLA_KERNEL_QK_ROPE, stream);
        DSLA_LAUNCH(ps, kernel, dim3(static_cast<unsigned>(n), chunks), dim3(256), 0, stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace dsla
