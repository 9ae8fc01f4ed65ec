// Keys and values of new tokens into the pages of a cache: a copy with one level of indirection, bound by HBM.
// A thread moves W bytes (16 where pointers, strides and D allow, an element otherwise) of the keys and of the
// values of a token at a time; a token's heads lie one behind the other along the threads of a workgroup.  16384 tokens of 8 heads, D = 128,
// 16 bits: 26.3 us, 5.1 TB/s read and written together, what a large copy reaches; 160 tokens 2.8 us, the launch.
#include "../../include/specdec.h"

#include <hip/hip_runtime.h>

namespace {

struct Store {
    const char *k, *v;
    char *kc, *vc;
    int64_t k_tok, k_head, v_tok, v_head;                                  // all in bytes
    int64_t kc_page, kc_tok, kc_head, vc_page, vc_tok, vc_head;
    const int32_t *slot;
    int64_t slots;
    int tokens, page, per_head, per_tok;                                   // pieces of W bytes
};

template <typename P>
__global__ void __launch_bounds__(256) sd_store_kernel(const Store s)
{
    const int64_t all = (int64_t)s.tokens * s.per_tok;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int t = (int)(i / s.per_tok), e = (int)(i % s.per_tok);
        const int slot = s.slot[t];
        if (slot < 0 || slot >= s.slots) continue;
        const int h = e / s.per_head, c = e % s.per_head;
        const int64_t page = slot / s.page, at = slot % s.page;
        const P a = *reinterpret_cast<const P *>(s.k + t * s.k_tok + h * s.k_head + c * (int64_t)sizeof(P));
        const P b = *reinterpret_cast<const P *>(s.v + t * s.v_tok + h * s.v_head + c * (int64_t)sizeof(P));
        *reinterpret_cast<P *>(s.kc + page * s.kc_page + at * s.kc_tok + h * s.kc_head + c * (int64_t)sizeof(P)) = a;
        *reinterpret_cast<P *>(s.vc + page * s.vc_page + at * s.vc_tok + h * s.vc_head + c * (int64_t)sizeof(P)) = b;
    }
}

}  // namespace

extern "C" int sd_cache_store(const sd_cache *cache, const void *k, int64_t k_tok_stride, int64_t k_head_stride, const void *v,
                              int64_t v_tok_stride, int64_t v_head_stride, const int32_t *slot, int64_t tokens, void *hip_stream)
{
    if (!cache || tokens < 0) return SD_EINVAL;
    const sd_cache &c = *cache;
    if (!c.k || !c.v || c.pages <= 0 || c.page <= 0 || c.heads <= 0 || c.D <= 0) return SD_EINVAL;
    if (c.dtype != SD_F32 && c.dtype != SD_BF16 && c.dtype != SD_F16) return SD_EINVAL;
    if (tokens == 0) return SD_OK;
    if (!k || !v || !slot) return SD_EINVAL;
    const int es = c.dtype == SD_F32 ? 4 : 2;
    const int64_t strides[] = {k_tok_stride, k_head_stride, v_tok_stride, v_head_stride, c.k_page_stride, c.k_tok_stride, c.k_head_stride,
                               c.v_page_stride, c.v_tok_stride, c.v_head_stride, c.D};
    const uintptr_t ptrs = reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | reinterpret_cast<uintptr_t>(c.k) | reinterpret_cast<uintptr_t>(c.v);
    if (ptrs % es || reinterpret_cast<uintptr_t>(slot) % 4) return SD_EINVAL;
    bool wide = ptrs % 16 == 0;
    for (int64_t x : strides) {
        if (x < 0) return SD_EINVAL;
        wide = wide && x * es % 16 == 0;
    }
    const int64_t most = 0x7fffffff;
    if (tokens > most || c.page > most || c.pages > most || c.pages * c.page > most || c.heads > most || c.D > most || c.heads * c.D > most) return SD_EUNSUPPORTED;
    const int w = wide ? 16 : es;
    Store s;
    s.k = static_cast<const char *>(k); s.v = static_cast<const char *>(v);
    s.kc = static_cast<char *>(c.k); s.vc = static_cast<char *>(c.v);
    s.k_tok = k_tok_stride * es; s.k_head = k_head_stride * es; s.v_tok = v_tok_stride * es; s.v_head = v_head_stride * es;
    s.kc_page = c.k_page_stride * es; s.kc_tok = c.k_tok_stride * es; s.kc_head = c.k_head_stride * es;
    s.vc_page = c.v_page_stride * es; s.vc_tok = c.v_tok_stride * es; s.vc_head = c.v_head_stride * es;
    s.slot = slot; s.slots = c.pages * c.page; s.tokens = (int)tokens; s.page = (int)c.page;
    s.per_head = (int)(c.D * es / w); s.per_tok = (int)(c.heads * s.per_head);
    const int64_t all = tokens * s.per_tok;
    const unsigned grid = (unsigned)((all + 255) / 256 < 16384 ? (all + 255) / 256 : 16384);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (w == 16) hipLaunchKernelGGL(sd_store_kernel<uint4>, dim3(grid), dim3(256), 0, st, s);
    else if (w == 4) hipLaunchKernelGGL(sd_store_kernel<uint32_t>, dim3(grid), dim3(256), 0, st, s);
    else hipLaunchKernelGGL(sd_store_kernel<uint16_t>, dim3(grid), dim3(256), 0, st, s);
    return hipGetLastError() == hipSuccess ? SD_OK : SD_EHIP;
}
