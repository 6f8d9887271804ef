// Attention of one query per sequence and head over a paged cache, for groups of sequences that
// share their first positions.
//
// A block per (sequence, query head): groups of lanes that hold a position's row side by side walk
// through the positions with a running maximum and sum of their own, and meet in LDS at the end.
#include "spd_device.h"

using namespace spdd;

namespace {

constexpr int NTS = 256, NWS = NTS / WAVE;

// exp(a - b) with exp(-inf - anything) = 0, also where b is -inf (nothing seen yet).
__device__ __forceinline__ float exp_below(float a, float b) { return expf(a - (b == -INFINITY ? 0.f : b)); }

template <typename KT>
__global__ __launch_bounds__(NTS) void shared_attn_kernel(const SharedAttnArgs a) {
    constexpr int VEC = Store<KT>::VEC;
    __shared__ float acc_s[NTS * VEC], m_s[NTS], l_s[NTS];
    const int tid = threadIdx.x, d = a.c.d_head, lpp = d / VEC, groups = NTS / lpp, gi = tid / lpp, li = tid % lpp;
    const int s = blockIdx.x / a.n_heads, hq = blockIdx.x % a.n_heads, lead = s - s % a.width, kvh = hq / (a.n_heads / a.c.n_kv_heads);
    const int shift = a.c.page_shift, page_size = 1 << shift;
    const int shared = as_global(a.shared)[s / a.width], len = as_global(a.len)[s];
    const long long room = (long long)a.c.table_stride << shift;
    const bool fits = shared >= 0 && len >= 0 && shared <= a.max_shared && (len <= shared || len - shared <= a.max_own) && len <= room;
    if (!fits && a.err && tid == 0) *as_global(a.err) = 1;
    const int n = fits ? len : 0;
    const float scale = 1.0f / sqrtf((float)d);
    float qv[VEC], acc[VEC], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int v = 0; v < VEC; ++v) { qv[v] = as_global(a.q)[((size_t)s * a.n_heads + hq) * d + li * VEC + v]; acc[v] = 0.f; }
    for (int p0 = 0; p0 < n; p0 += groups) {
        const int p = p0 + gi;
        const int page = p < n ? as_global(a.c.table)[(size_t)(p < shared ? lead : s) * a.c.table_stride + (p >> shift)] : 0;
        const bool good = (unsigned)page < (unsigned)a.c.n_pages, there = p < n && good;
        if (!good && a.err) *as_global(a.err) = 1;
        float kf[VEC], vf[VEC], x = 0.f;
#pragma unroll
        for (int v = 0; v < VEC; ++v) kf[v] = vf[v] = 0.f;
        if (there) {
            const size_t at = (((size_t)page * a.c.n_kv_heads + kvh) * page_size + (p & (page_size - 1))) * d + li * VEC;
            Store<KT>::unpack(global_load16((const char *)a.c.K + at * sizeof(KT)), kf);
            Store<KT>::unpack(global_load16((const char *)a.c.V + at * sizeof(KT)), vf);
        }
#pragma unroll
        for (int v = 0; v < VEC; ++v) x = fmaf(kf[v], qv[v], x);
        for (int o = 1; o < lpp; o <<= 1) x += __shfl_xor(x, o, WAVE);
        x = there ? x * scale : -INFINITY;
        const float mx = fmaxf(m, x), corr = exp_below(m, mx), w = there ? exp_below(x, mx) : 0.f;
        m = mx;
        l = l * corr + w;
#pragma unroll
        for (int v = 0; v < VEC; ++v) acc[v] = fmaf(w, vf[v], acc[v] * corr);
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) acc_s[gi * d + li * VEC + v] = acc[v];
    if (li == 0) { m_s[gi] = m; l_s[gi] = l; }
    __syncthreads();
    for (int c = tid; c < d; c += NTS) {
        float M = -INFINITY, L = 0.f, O = 0.f;
        for (int g = 0; g < groups; ++g) M = fmaxf(M, m_s[g]);
        for (int g = 0; g < groups; ++g) {
            const float f = exp_below(m_s[g], M);
            L += f * l_s[g];
            O += f * acc_s[g * d + c];
        }
        as_global(a.out)[((size_t)s * a.n_heads + hq) * d + c] = L == 0.f ? 0.f : O / L;   // a row that sees nothing: zeros
    }
}

}  // namespace

extern "C" size_t spd_op_attention_shared_scratch_bytes(int32_t n_seq, int32_t width, int32_t n_heads, int32_t n_kv_heads, int32_t d_head, int32_t max_shared,
                                                        int32_t max_own) {
    if (n_seq <= 0 || width <= 0 || n_heads <= 0 || n_kv_heads <= 0 || d_head <= 0 || max_shared < 0 || max_own < 0) return 0;
    return 256;
}

extern "C" int spd_op_attention_shared(int32_t dtype, const float *q, const void *K, const void *V, const int32_t *table, int32_t n_pages, int32_t n_kv_heads,
                                       int32_t page_size, int32_t d_head, int32_t n_seq, int32_t table_stride, const int32_t *shared, const int32_t *len,
                                       int32_t width, int32_t n_heads, int32_t max_shared, int32_t max_own, float *out, void *scratch, size_t scratch_bytes,
                                       int32_t *err, void *hip_stream) {
    const PagedCache c = spdk::paged_cache((void *)K, (void *)V, table, n_pages, n_kv_heads, page_size, d_head, n_seq, table_stride);
    const int rc = spdk::paged_cache_status(dtype, c, page_size);
    if (rc != SPD_OK) return rc;
    if (width < 1 || n_seq % width || n_heads < 1 || n_heads % n_kv_heads || max_shared < 0 || max_own < 0) return SPD_EINVAL;
    const long long room = (long long)table_stride * page_size;      // (the longest shared and the longest own part may be different sequences')
    if (max_shared > room || max_own > room || (long long)max_shared + max_own > INT32_MAX - 65536) return SPD_EINVAL;
    if (n_seq == 0) return SPD_OK;
    if (!q || !shared || !len || !out || ((uintptr_t)q | (uintptr_t)out) % 16) return SPD_EINVAL;
    if (!scratch || (uintptr_t)scratch % 256) return SPD_EINVAL;
    if (scratch_bytes < spd_op_attention_shared_scratch_bytes(n_seq, width, n_heads, n_kv_heads, d_head, max_shared, max_own)) return SPD_EWORKSPACE;
    const long long blocks = (long long)n_seq * n_heads;
    if (blocks > INT32_MAX) return SPD_EINVAL;
    const SharedAttnArgs a{c, q, out, shared, len, err, width, n_heads, max_shared, max_own};
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == SPD_DTYPE_FP32) hipLaunchKernelGGL(shared_attn_kernel<float>, dim3((unsigned)blocks), dim3(NTS), 0, s, a);
    else if (dtype == SPD_DTYPE_FP16) hipLaunchKernelGGL(shared_attn_kernel<half_t>, dim3((unsigned)blocks), dim3(NTS), 0, s, a);
    else hipLaunchKernelGGL(shared_attn_kernel<bf16_t>, dim3((unsigned)blocks), dim3(NTS), 0, s, a);
    return hipGetLastError() == hipSuccess ? SPD_OK : SPD_EHIP;
}
