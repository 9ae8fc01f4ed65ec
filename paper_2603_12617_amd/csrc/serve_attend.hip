// Attention of a chunk of new tokens over a paged cache (sd_attend).
//
// One wavefront per (new token, query head).  Keys in blocks of 64, a key to a lane for the scores (float32 products
// and sums over D), one pass with a running maximum and sum, then a share of D to a lane for the weighted values.
#include "../../include/specdec.h"

#include <hip/hip_runtime.h>

#include <math.h>

namespace {

struct bf16 { uint16_t u; };
__device__ __forceinline__ float to_float(bf16 v) { return __uint_as_float((unsigned)v.u << 16); }
__device__ __forceinline__ float to_float(_Float16 v) { return (float)v; }
__device__ __forceinline__ void from_float(float f, _Float16 &o) { o = (_Float16)f; }
__device__ __forceinline__ void from_float(float f, bf16 &o)
{
    const unsigned u = __float_as_uint(f);
    o.u = f == f ? (uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16) : (uint16_t)0x7fc0;
}

template <typename T> __global__ void __launch_bounds__(64) sd_attend_kernel(const sd_attention a)
{
    const int lane = threadIdx.x;
    const int t = blockIdx.x, h = blockIdx.y, kh = h / (int)(a.Hq / a.cache.heads);
    const int D = (int)a.cache.D, page = (int)a.cache.page;
    int b = 0;
    for (int n = (int)a.B; n > 1;) {
        const int step = (n + 63) / 64;
        const u_int64_t mask = __ballot(lane * step < n && a.cu[b + lane * step] <= t);
        const int last = mask ? 63 - __builtin_clzll(mask) : 0;
        n = min(step, n - last * step);
        b += last * step;
    }
    const int m = a.cu[b + 1] - a.cu[b];
    const int64_t kv = min((int64_t)a.kv[b], a.width * page);
    const int64_t pos = kv - m + (t - a.cu[b]);
    const int64_t lo = a.window > 0 ? max((int64_t)0, pos - a.window + 1) : 0, hi = min(pos + 1, kv);
    const T *q = static_cast<const T *>(a.q) + t * a.q_tok_stride + h * a.q_head_stride;
    float top = -INFINITY, sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t j0 = lo; j0 < hi; j0 += 64) {
        const int64_t j = j0 + lane;
        float s = -INFINITY;
        int P = 0, at = 0;
        if (j < hi) {
            P = min(max(a.table[b * a.table_stride + j / page], 0), (int)a.cache.pages - 1);
            at = (int)(j % page);
            const T *k = static_cast<const T *>(a.cache.k) + P * a.cache.k_page_stride + at * a.cache.k_tok_stride + kh * a.cache.k_head_stride;
            float d = 0.f;
            for (int e = 0; e < D; ++e) d += to_float(q[e]) * to_float(k[e]);
            s = d * (float)a.scale;
        }
        float most = s;
        for (int sh = 32; sh >= 1; sh >>= 1) most = fmaxf(most, __shfl_xor(most, sh));
        const float now = fmaxf(top, most), back = top == now ? 1.f : expf(top - now);
        float w = j < hi && now > -INFINITY ? expf(s - now) : 0.f, all = w;
        for (int sh = 32; sh >= 1; sh >>= 1) all += __shfl_xor(all, sh);
        sum = sum * back + all;
        top = now;
        for (int c = 0; c < 4; ++c) o[c] *= back;
        const int n = (int)min((int64_t)64, hi - j0);
        for (int i = 0; i < n; ++i) {
            const float wi = __shfl(w, i);
            const T *v = static_cast<const T *>(a.cache.v) + __shfl(P, i) * a.cache.v_page_stride + __shfl(at, i) * a.cache.v_tok_stride + kh * a.cache.v_head_stride;
            for (int c = 0; c < 4; ++c)
                if (c * 64 + lane < D) o[c] += wi * to_float(v[c * 64 + lane]);
        }
    }
    T *out = static_cast<T *>(a.out) + t * a.out_tok_stride + h * a.out_head_stride;
    for (int c = 0; c < 4; ++c)
        if (c * 64 + lane < D) from_float(sum > 0.f ? o[c] / sum : lo < hi ? o[c] : 0.f, out[c * 64 + lane]);
    if (lane == 0 && a.lse) a.lse[t * a.Hq + h] = lo < hi ? top + logf(sum) : -INFINITY;
}

bool misaligned(const void *p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

int check(const sd_attention &a)
{
    const sd_cache &c = a.cache;
    if (a.B <= 0 || a.tokens < 0 || a.Hq <= 0 || a.width <= 0 || a.table_stride < a.width || a.window < 0) return SD_EINVAL;
    if (c.pages <= 0 || c.page <= 0 || c.heads <= 0 || c.D <= 0 || a.Hq % c.heads != 0) return SD_EINVAL;
    if (!(a.scale > 0.0) || !(a.scale <= 3e38)) return SD_EINVAL;
    if (c.dtype != SD_F32 && c.dtype != SD_BF16 && c.dtype != SD_F16) return SD_EINVAL;
    const int64_t strides[] = {c.k_page_stride, c.k_tok_stride, c.k_head_stride, c.v_page_stride, c.v_tok_stride, c.v_head_stride,
                               a.q_tok_stride, a.q_head_stride, a.out_tok_stride, a.out_head_stride};
    for (int64_t s : strides) {
        if (s < 0) return SD_EINVAL;
        if (s % 8 != 0) return SD_EINVAL;
    }
    const int64_t most = 0x7fffffff;
    if (c.dtype == SD_F32 || c.D % 8 != 0 || c.D > SD_MAX_HEAD_DIM || a.B > SD_MAX_REQUESTS) return SD_EUNSUPPORTED;
    if (c.pages > most || c.page > most || c.pages * c.page > most || a.width > most || a.width * c.page > most || a.Hq > 65535 || a.tokens * a.Hq > most)
        return SD_EUNSUPPORTED;
    return SD_OK;
}

}  // namespace

extern "C" {

size_t sd_attend_workspace_bytes(const sd_attention *a)
{
    if (!a || check(*a) != SD_OK) return 0;
    return 16;
}

int sd_attend(const sd_attention *args, void *ws, size_t ws_bytes, void *hip_stream)
{
    if (!args) return SD_EINVAL;
    const sd_attention &a = *args;
    const int rc = check(a);
    if (rc != SD_OK) return rc;
    if (!a.cache.k || !a.cache.v || !a.cu || !a.kv || !a.table || !ws) return SD_EINVAL;
    if (a.tokens > 0 && (!a.q || !a.out)) return SD_EINVAL;
    if (misaligned(a.cache.k, 16) || misaligned(a.cache.v, 16) || misaligned(a.q, 16) || misaligned(a.out, 16) || misaligned(a.lse, 4) ||
        misaligned(a.cu, 4) || misaligned(a.kv, 4) || misaligned(a.table, 4) || misaligned(ws, 16))
        return SD_EINVAL;
    if (ws_bytes < sd_attend_workspace_bytes(args)) return SD_ENOMEM;
    if (a.tokens == 0) return SD_OK;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const dim3 grid((unsigned)a.tokens, (unsigned)a.Hq);
    if (a.cache.dtype == SD_BF16) hipLaunchKernelGGL(sd_attend_kernel<bf16>, grid, dim3(64), 0, st, a);
    else hipLaunchKernelGGL(sd_attend_kernel<_Float16>, grid, dim3(64), 0, st, a);
    return hipGetLastError() == hipSuccess ? SD_OK : SD_EHIP;
}

}  // extern "C"
