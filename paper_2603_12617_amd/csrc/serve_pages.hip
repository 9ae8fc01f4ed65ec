// Block tables and slot maps of a served step, and the write of new keys and values into a paged cache.
//
// sd_pages is integer bookkeeping: per request the pages it needs and the pages it gives back, three
// exclusive sums over the requests (new tokens, pages given back, pages taken), and then items that are
// independent of each other: one per new token, per page taken, per page pushed.  There is nothing to
// stream (a decoding step of 64 requests touches 5 KB), so what counts is the number of launches and of dependent trips
// to memory: one launch, in which every workgroup sums over all requests by itself (16 KB per input from L2 at
// most) into LDS and then works its share of the items, finding an item's request by bisection there.  No workgroup
// waits for another: what one reads (entries held before, the stack below its old top) none writes.
#include "../../include/specdec.h"

#include <hip/hip_runtime.h>

namespace {

constexpr int kMaxB = SD_MAX_REQUESTS;

struct Need { int add, back, need, keep, held, want; };

// what request b has, needs and gives back; numbers out of range are clamped
__device__ __forceinline__ Need need_of(const sd_page_step &s, int b)
{
    Need r;
    r.held = min(max(s.pages[b], 0), (int)s.width);
    const int64_t cap = (int64_t)r.held * s.page;
    const int64_t more = s.accepted ? (int64_t)max(s.accepted[b], 0) + 1 : 0;
    r.keep = (int)min((int64_t)max(s.length[b], 0) + more, cap);
    r.add = min(max(s.add[b], 0), 0x7fffffff / (int)s.B);
    const int64_t want = ((int64_t)r.keep + r.add + s.page - 1) / s.page;
    r.want = (int)min(want, s.width + 1);
    r.back = max(r.held - r.want, 0);
    r.need = r.want <= s.width ? max(r.want - r.held, 0) : 0;
    return r;
}

__device__ __forceinline__ int wave_scan(int v, int lane)
{
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) {
        const int o = __shfl_up(v, sh);
        if (lane >= sh) v += o;
    }
    return v;
}

// the last request whose sum before it is <= x: sums are ascending, sum[0] = 0
__device__ __forceinline__ int find(const int *sum, int B, int x)
{
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (sum[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__global__ void __launch_bounds__(256) sd_pages_kernel(const sd_page_step s)
{
    constexpr int kWaves = 4;
    __shared__ int cu[kMaxB], back[kMaxB], taken[kMaxB];      // sums over the requests before
    __shared__ int part[3][kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int B = (int)s.B;
    const int per = (B + 255) / 256;

    int a = 0, f = 0, t = 0;
    for (int e = 0; e < per; ++e) {
        const int b = tid * per + e;
        if (b < B) { const Need r = need_of(s, b); a += r.add; f += r.back; t += r.need; }
    }
    const int ia = wave_scan(a, lane), iff = wave_scan(f, lane), it = wave_scan(t, lane);
    if (lane == 63) { part[0][wave] = ia; part[1][wave] = iff; part[2][wave] = it; }
    __syncthreads();
    int ea = ia - a, ef = iff - f, et = it - t, total_back = 0;
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) { ea += part[0][w]; ef += part[1][w]; et += part[2][w]; }
        total_back += part[1][w];
    }
    const int pool = (int)s.pool;
    const int nfree = min(max(s.nfree[0], 0), pool);
    const int top = min(nfree + total_back, pool);            // of the stack once the surplus pages are on it
    for (int e = 0; e < per; ++e) {
        const int b = tid * per + e;
        if (b >= B) break;
        const Need r = need_of(s, b);
        cu[b] = ea; back[b] = ef; taken[b] = et;
        const bool served = r.want <= s.width && (r.need == 0 || et + r.need <= top);
        if (blockIdx.x == 0) {
            s.cu_out[b] = ea;
            if (b == B - 1) s.cu_out[B] = ea + r.add;
            s.length_out[b] = r.keep;
            s.kv_out[b] = served ? r.keep + r.add : r.keep;
            s.pages_out[b] = served ? r.want : r.held;
        }
        ea += r.add; ef += r.back; et += r.need;
    }
    __syncthreads();

    // what was taken: up to the first request that found too few pages
    int all_taken;
    {
        const Need r = need_of(s, B - 1);
        all_taken = taken[B - 1] + r.need;
        if (all_taken > top) {
            int lo = 0, hi = B - 1;                           // the first request whose sum passes the top
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if ((mid + 1 < B ? taken[mid + 1] : all_taken) > top) hi = mid; else lo = mid + 1;
            }
            all_taken = taken[lo];
        }
    }
    const int left = top - all_taken;
    if (blockIdx.x == 0 && tid == 0) s.nfree_out[0] = left;

    const int step = gridDim.x * 256, first = blockIdx.x * 256 + tid;
    // entry i of the stack with the surplus pages on it
    auto stack = [&](int i) {
        if (i < nfree) return s.free[i];
        const int b = find(back, B, i - nfree);
        const int at = need_of(s, b).want + (i - nfree - back[b]);
        return at >= 0 && at < s.width ? s.table[b * s.table_stride + at] : -1;
    };
    for (int i = first; i < all_taken; i += step) {
        const int b = find(taken, B, i);
        const int at = need_of(s, b).held + i - taken[b];
        if (at < s.width) s.table[b * s.table_stride + at] = stack(top - 1 - i);
    }
    for (int i = nfree + first; i < left; i += step) s.free[i] = stack(i);
    for (int i = first; i < s.tokens; i += step) {
        const int b = find(cu, B, i);
        const Need r = need_of(s, b);
        const bool served = r.want <= s.width && (r.need == 0 || taken[b] + r.need <= top);
        int slot = -1, pos = -1;
        if (served && i - cu[b] < r.add) {
            pos = r.keep + i - cu[b];
            const int at = pos / (int)s.page;
            const int page = at < r.held ? s.table[b * s.table_stride + at] : stack(top - 1 - (taken[b] + at - r.held));
            slot = page * (int)s.page + pos % (int)s.page;
        }
        s.slot_out[i] = slot;
        s.pos_out[i] = pos;
    }
}

bool misaligned(const void *p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

}  // namespace

extern "C" int sd_pages(const sd_page_step *step, void *hip_stream)
{
    if (!step) return SD_EINVAL;
    const sd_page_step &s = *step;
    if (s.B <= 0 || s.page <= 0 || s.width <= 0 || s.table_stride < s.width || s.pool <= 0 || s.tokens < 0) return SD_EINVAL;
    const void *in[] = {s.pages, s.length, s.accepted, s.add, s.nfree};
    const void *out[] = {s.table, s.free, s.pages_out, s.length_out, s.kv_out, s.nfree_out, s.cu_out, s.slot_out, s.pos_out};
    for (int i = 0; i < 5; ++i)
        if ((!in[i] && i != 2) || misaligned(in[i], 4)) return SD_EINVAL;
    for (int o = 0; o < 9; ++o) {
        if ((!out[o] && (o < 7 || s.tokens > 0)) || misaligned(out[o], 4)) return SD_EINVAL;
        for (int i = 0; i < 5; ++i)
            if (out[o] && out[o] == in[i]) return SD_EINVAL;
    }
    const int64_t most = 0x7fffffff;
    if (s.B > SD_MAX_REQUESTS || s.page > most || s.width >= most || s.pool > most || s.tokens > most) return SD_EUNSUPPORTED;
    if (s.width * s.page > most || s.pool * s.page > most || s.width * s.B > most) return SD_EUNSUPPORTED;   // (sums are 32 bits)
    // a workgroup per 1024 tokens, four to a thread; they also share out the pages
    int64_t grid = (s.tokens + 1023) / 1024;
    grid = grid < 1 ? 1 : grid > 1024 ? 1024 : grid;
    hipLaunchKernelGGL(sd_pages_kernel, dim3((unsigned)grid), dim3(256), 0, static_cast<hipStream_t>(hip_stream), s);
    return hipGetLastError() == hipSuccess ? SD_OK : SD_EHIP;
}
