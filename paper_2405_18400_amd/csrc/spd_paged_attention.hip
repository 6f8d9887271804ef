// Causal attention of every sequence's new tokens over a paged cache.
//
// One wave per (token, query head): 64 keys at a time, one per lane, with a running maximum and sum; then the lanes share out the
// features.  Sums in 64 bits.
#include "spd_device.h"

#include <algorithm>

using namespace spdd;

namespace {

struct q8_t { int8_t b; };

template <typename KT> __device__ __forceinline__ float element(const void *p, size_t i) {
    if constexpr (sizeof(KT) == 1) return (float)as_global((const int8_t *)p)[i];
    else return Store<KT>::load1(p, i);
}

// The sequence that token t belongs to: behind all that end before it.  (Bounded whatever `first` holds.)
__device__ __forceinline__ int sequence_of(const int32_t *first, int n_seq, int t, int lane) {
    int before = 0;
    for (int i = lane; i < n_seq; i += WAVE) before += as_global(first)[i + 1] <= t;
    for (int o = 1; o < WAVE; o <<= 1) before += __shfl_xor(before, o, WAVE);
    return before;
}

template <typename KT, typename IO>
__global__ __launch_bounds__(WAVE) void paged_attn_kernel(const PagedAttnArgs p) {
    __shared__ float q[256];
    const int lane = threadIdx.x, t = blockIdx.x / p.n_heads, h = blockIdx.x % p.n_heads, d = p.c.d_head, kvh = h / p.group;
    if (blockIdx.x == 0)                         // what no token may show
        for (int i = lane; i < p.c.n_seq; i += WAVE)
            if ((as_global(p.first)[i] < 0 || as_global(p.first)[i] > as_global(p.first)[i + 1] || as_global(p.first)[i + 1] > p.n_tokens) && p.err) *as_global(p.err) = 1;
    const int s = sequence_of(p.first, p.c.n_seq, t, lane);
    if (s >= p.c.n_seq) return;
    const int a = as_global(p.first)[s], b = as_global(p.first)[s + 1], len = as_global(p.len)[s];
    if (t < a || t >= b) return;
    const size_t row = ((size_t)t * p.n_heads + h) * d;
    const bool fits = a >= 0 && b <= p.n_tokens && len >= b - a && len <= p.max_len && (long long)len <= (long long)p.c.table_stride << p.c.page_shift;
    if (!fits && p.err && lane == 0) *as_global(p.err) = 1;
    const int n = fits ? len - (b - a) + (t - a) + 1 : 0;
    for (int i = lane; i < d; i += WAVE) q[i] = Store<IO>::load1(p.q, (size_t)t * p.q_stride + (size_t)h * d + i);
    __syncthreads();
    float m = -INFINITY;
    double l = 0.0, o[4] = {0.0, 0.0, 0.0, 0.0};
    const float scale = 1.4426950408889634f / sqrtf((float)d);
    const int page_size = 1 << p.c.page_shift;
    for (int k0 = 0; k0 < n; k0 += WAVE) {
        const int pos = k0 + lane;
        size_t place = 0;
        bool in = pos < n;
        if (in) {
            const int page = as_global(p.c.table)[(size_t)s * p.c.table_stride + (pos >> p.c.page_shift)];
            in = (unsigned)page < (unsigned)p.c.n_pages;
            if (!in && p.err) *as_global(p.err) = 1;
            else place = ((size_t)page * p.c.n_kv_heads + kvh) * page_size + (pos & (page_size - 1));
        }
        float z = -INFINITY, vs = 1.f;
        if (in) {
            z = 0.f;
            for (int i = 0; i < d; ++i) z = fmaf(q[i], element<KT>(p.c.K, place * d + i), z);
            if constexpr (sizeof(KT) == 1) {
                z *= as_global(p.k_scale)[place];
                vs = as_global(p.v_scale)[place];
            }
            z *= scale;
        }
        const float mx = fmaxf(m, wave_max(z));
        if (mx == -INFINITY && !__any(z != z)) continue;
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mx), e = __builtin_amdgcn_exp2f(z - mx);
        m = mx;
        l = l * f + e;
        for (int i = 0; i < 4; ++i) o[i] *= f;
        for (int k = 0; k < WAVE; ++k) {
            const float w = __shfl(e, k, WAVE) * __shfl(vs, k, WAVE);
            const size_t from = (size_t)__shfl((unsigned long long)place, k, WAVE) * d;
            if (w == 0.f) continue;
            for (int i = 0; i < 4; ++i)
                if (lane + i * WAVE < d) o[i] += (double)w * element<KT>(p.c.V, from + lane + i * WAVE);
        }
    }
    for (int i = 1; i < WAVE; i <<= 1) l += __shfl_xor(l, i, WAVE);
    for (int i = 0; i < 4; ++i)
        if (lane + i * WAVE < d) Store<IO>::store1(p.out, row + lane + i * WAVE, l == 0.0 ? 0.f : (float)(o[i] / l));
}

template <typename KT, typename IO>
hipError_t launch(hipStream_t s, const PagedAttnArgs &a) {
    hipLaunchKernelGGL((paged_attn_kernel<KT, IO>), dim3((unsigned)(a.n_tokens * a.n_heads)), dim3(WAVE), 0, s, a);
    return hipGetLastError();
}

bool io_fits(int dtype, int io) {
    if (io == SPD_DTYPE_FP32) return true;
    return dtype == SPD_DTYPE_INT8 ? io == SPD_DTYPE_FP16 || io == SPD_DTYPE_BF16 : dtype == io;
}

}  // namespace

extern "C" size_t spd_op_attention_paged_scratch_bytes(int32_t dtype, int32_t io_dtype, int32_t n_seq, int32_t n_tokens, int32_t n_heads, int32_t n_kv_heads, int32_t d_head,
                                                       int32_t max_new, int32_t max_len) {
    (void)dtype; (void)io_dtype; (void)n_seq; (void)n_tokens; (void)n_heads; (void)n_kv_heads; (void)d_head; (void)max_new; (void)max_len;
    return 0;
}

extern "C" int spd_op_attention_paged(int32_t dtype, int32_t io_dtype, const void *q, int64_t q_stride, const void *K, const void *V, const float *K_scale, const float *V_scale,
                                      const int32_t *table, int32_t n_pages, int32_t n_kv_heads, int32_t page_size, int32_t d_head, int32_t n_seq, int32_t table_stride, const int32_t *first,
                                      const int32_t *len, int32_t n_tokens, int32_t n_heads, int32_t max_new, int32_t max_len, void *out, void *scratch, size_t scratch_bytes,
                                      int32_t *err, void *hip_stream) {
    const PagedCache c = spdk::paged_cache((void *)K, (void *)V, table, n_pages, n_kv_heads, page_size, d_head, n_seq, table_stride);
    const int rc = spdk::paged_cache_status(dtype, c, page_size, K_scale, V_scale);
    if (rc != SPD_OK) return rc;
    if (!io_fits(dtype, io_dtype) || n_tokens < 0 || n_heads < 1 || n_heads % n_kv_heads || max_new < 0 || max_len < 0 || max_len > (long long)table_stride * page_size || max_len > INT32_MAX / 2)
        return SPD_EINVAL;
    if (n_tokens == 0 || n_seq == 0) return SPD_OK;
    if ((long long)n_tokens * n_heads > (1 << 24) || n_seq > (1 << 20)) return SPD_EINVAL;
    const int io_bytes = io_dtype == SPD_DTYPE_FP32 ? 4 : 2;
    if (!q || !first || !len || !out || ((uintptr_t)q | (uintptr_t)out) % 16 || q_stride < (int64_t)n_heads * d_head || q_stride % 8) return SPD_EINVAL;
    const size_t need = spd_op_attention_paged_scratch_bytes(dtype, io_dtype, n_seq, n_tokens, n_heads, n_kv_heads, d_head, max_new, max_len);
    if (need && (!scratch || (uintptr_t)scratch % 256)) return SPD_EINVAL;
    if (scratch_bytes < need) return SPD_EWORKSPACE;
    const size_t rows = (size_t)n_tokens * n_heads * d_head * io_bytes, q_bytes = ((size_t)(n_tokens - 1) * q_stride + (size_t)n_heads * d_head) * io_bytes, pool = spdk::pool_bytes(dtype, c),
                 scales = spdk::scale_bytes(c);
    const spdk::Span sq{q, q_bytes}, so{out, rows}, sK{K, pool}, sV{V, pool}, sk{K_scale, scales}, sv{V_scale, scales}, st{table, (size_t)n_seq * table_stride * 4},
        sf{first, (size_t)(n_seq + 1) * 4}, sl{len, (size_t)n_seq * 4}, se{err, 4}, sw{scratch, need};
    if (spdk::over_any(so, {sq, sK, sV, sk, sv, st, sf, sl, se, sw}) || spdk::over_any(sw, {sq, sK, sV, sk, sv, st, sf, sl, se})) return SPD_EINVAL;
    PagedAttnArgs a{c, K_scale, V_scale, q, q_stride, out, first, len, err, n_tokens, n_heads, n_heads / n_kv_heads, max_len};
    hipStream_t s = (hipStream_t)hip_stream;
    hipError_t e = hipErrorInvalidValue;
    if (dtype == SPD_DTYPE_FP32) e = launch<float, float>(s, a);
    else if (dtype == SPD_DTYPE_FP16) e = io_dtype == SPD_DTYPE_FP32 ? launch<half_t, float>(s, a) : launch<half_t, half_t>(s, a);
    else if (dtype == SPD_DTYPE_BF16) e = io_dtype == SPD_DTYPE_FP32 ? launch<bf16_t, float>(s, a) : launch<bf16_t, bf16_t>(s, a);
    else e = io_dtype == SPD_DTYPE_FP32 ? launch<q8_t, float>(s, a) : io_dtype == SPD_DTYPE_FP16 ? launch<q8_t, half_t>(s, a) : launch<q8_t, bf16_t>(s, a);
    return e == hipSuccess ? SPD_OK : SPD_EHIP;
}
