// Block tables and slot maps of a served step.
//
// sd_pages is integer bookkeeping: per request the pages it needs and the pages it gives back, three
// exclusive sums over the requests (new tokens, pages given back, pages taken), and then items that are
// independent of each other: one per four new tokens, per page taken, per page pushed.  There is nothing to
// stream (a decoding step of 64 requests touches 5 KB), so what counts is the number of launches and of dependent trips
// to memory: one launch, in which every workgroup sums over all requests by itself (16 KB per input from L2 at
// most) and keeps what it found of each in LDS, then works its share of the items, finding an item's request by bisection
// there.  No workgroup waits for another: what one reads (entries held before, the stack below its old top) none writes.
// 64 requests of 5 tokens 5.4 us; 1024 requests, a million new tokens 12 us, of which the sums are the larger part (its 8.9 MB would take 2).
#include "../../include/specdec.h"

#include <hip/hip_runtime.h>

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

struct Step {
    sd_page_step s;
    int page_shift;                // x / page = mulhi(2 x, page_mul) >> page_shift for x < 2^31
    unsigned page_mul;
};
__device__ __forceinline__ int page_of(const Step &p, int x) { return (int)(__umulhi(2u * (unsigned)x, p.page_mul) >> p.page_shift); }

struct Need { int add, back, need, keep, held, want; };

// what request b has, needs and gives back; numbers out of range are clamped
__device__ __forceinline__ Need need_of(const Step &p, int b)
{
    const sd_page_step &s = p.s;
    Need r;
    const int pages = s.pages[b], length = s.length[b], accepted = s.accepted ? max(s.accepted[b], -1) : -1, add = s.add[b];
    r.held = min(max(pages, 0), (int)s.width);
    r.keep = (int)min((unsigned)max(length, 0) + (unsigned)accepted + 1u, (unsigned)(r.held * (int)s.page));
    r.add = max(add, 0);
    const unsigned x = (unsigned)r.keep + (unsigned)r.add;
    r.want = x > (unsigned)(s.width * s.page) ? (int)s.width + 1 : x ? page_of(p, (int)(x - 1)) + 1 : 0;
    r.back = max(r.held - r.want, 0);
    r.need = r.want <= s.width ? max(r.want - r.held, 0) : 0;
    return r;
}

// sums over the lanes up to this one
template <typename F> __device__ __forceinline__ int wave_scan(int v, int lane, F f)
{
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) {
        const int o = __shfl_up(v, sh);
        if (lane >= sh) v = f(v, o);
    }
    return v;
}
// of tokens: sums that would pass 31 bits end there (pages are no more than the tables hold)
constexpr auto kTokens = [](int a, int b) { return (int)min((unsigned)a + (unsigned)b, 0x7fffffffu); };
constexpr auto kPages = [](int a, int b) { return a + b; };

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

__global__ void __launch_bounds__(kThreads) sd_pages_kernel(const Step p)
{
    extern __shared__ int lds[];
    __shared__ int part[3][kWaves];
    const sd_page_step &s = p.s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int B = (int)s.B, page = (int)s.page;
    int *const cu = lds, *const back = cu + B, *const taken = back + B;      // sums over the requests before
    int *const keep = taken + B, *const pages = keep + B;                    // tokens kept; pages held, ~pages if refused
    const int per = (B + kThreads - 1) / kThreads;

    const Need first_need = tid * per < B ? need_of(p, tid * per) : Need{0, 0, 0, 0, 0, 0};
    int a = first_need.add, f = first_need.back, t = first_need.need;
    for (int e = 1; e < per; ++e) {
        const int b = tid * per + e;
        if (b < B) { const Need r = need_of(p, b); a = kTokens(a, r.add); f += r.back; t += r.need; }
    }
    const int nfree = min(max(s.nfree[0], 0), (int)s.pool);
    const int ia = wave_scan(a, lane, kTokens), iff = wave_scan(f, lane, kPages), it = wave_scan(t, lane, kPages);
    if (lane == 63) { part[0][wave] = ia; part[1][wave] = iff; part[2][wave] = it; }
    int ea = __shfl_up(ia, 1);                               // (a sum that has ended cannot be taken back)
    if (lane == 0) ea = 0;
    __syncthreads();
    int ef = iff - f, et = it - t, all_add = 0, all_back = 0, all_need = 0;
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) { ea = kTokens(ea, part[0][w]); ef += part[1][w]; et += part[2][w]; }
        all_add = kTokens(all_add, part[0][w]);
        all_back += part[1][w];
        all_need += part[2][w];
    }
    const int top = min(nfree + all_back, (int)s.pool);       // of the stack once the surplus pages are on it
    for (int e = 0; e < per; ++e) {
        const int b = tid * per + e;
        if (b >= B) break;
        const Need r = e ? need_of(p, b) : first_need;
        const bool served = r.want <= s.width && (r.need == 0 || et + r.need <= top);
        cu[b] = ea; back[b] = ef; taken[b] = et; keep[b] = r.keep; pages[b] = served ? r.held : ~r.held;
        if (blockIdx.x == 0) {
            s.cu_out[b] = ea;
            if (b == B - 1) s.cu_out[B] = kTokens(ea, r.add);
            s.length_out[b] = r.keep;
            s.kv_out[b] = served ? r.keep + r.add : r.keep;
            s.pages_out[b] = served ? r.want : r.held;
        }
        ea = kTokens(ea, r.add); ef += r.back; et += r.need;
    }
    __syncthreads();

    // what was taken: all, or up to the first request that found too few pages
    int all_taken = all_need;
    if (all_need > top) {
        int lo = 0, hi = B - 1;                               // the first request whose sum passes the top
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if ((mid + 1 < B ? taken[mid + 1] : all_need) > top) hi = mid; else lo = mid + 1;
        }
        all_taken = taken[lo];
    }
    const int left = top - all_taken;
    if (blockIdx.x == 0 && tid == 0) s.nfree_out[0] = left;

    const int step = gridDim.x * kThreads, first = blockIdx.x * kThreads + tid;
    // entry i of the stack with the surplus pages on it
    auto stack = [&](int i) {
        if (i < nfree) return s.free[i];
        const int b = find(back, B, i - nfree);
        const int held = pages[b] < 0 ? ~pages[b] : pages[b], given = (b + 1 < B ? back[b + 1] : all_back) - back[b];
        const int at = held - given + (i - nfree - back[b]);
        return at >= 0 && at < s.width ? s.table[b * s.table_stride + at] : -1;
    };
    for (int i = first; i < all_taken; i += step) {
        const int b = find(taken, B, i), at = pages[b] + i - taken[b];
        if (at >= 0 && at < s.width) s.table[b * s.table_stride + at] = stack(top - 1 - i);
    }
    for (int i = nfree + first; i < left; i += step) s.free[i] = stack(i);
    for (int64_t i0 = 4ll * first; i0 < s.tokens; i0 += 4ll * step) {
        int b = find(cu, B, (int)i0), place = -1, id = -1;
        int slot[4], pos[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = (int)i0 + e, was = b;
            while (b + 1 < B && cu[b + 1] <= i) ++b;
            const int held = pages[b];
            const int x = (int)((unsigned)keep[b] + (unsigned)(i - cu[b])), at = page_of(p, x);
            slot[e] = pos[e] = -1;
            if (held >= 0 && i < all_add && at < s.width) {
                if (at != place || b != was) {
                    place = at;
                    const int k = top - 1 - (taken[b] + at - held);
                    id = at < held ? s.table[b * s.table_stride + at] : k >= 0 ? stack(k) : -1;
                }
                slot[e] = id * page + (x - at * page);
                pos[e] = x;
            }
        }
        if (i0 + 4 <= s.tokens && p.s.tokens % 4 == 0 && ((reinterpret_cast<uintptr_t>(s.slot_out) | reinterpret_cast<uintptr_t>(s.pos_out)) & 15) == 0) {
            *reinterpret_cast<int4 *>(s.slot_out + i0) = int4{slot[0], slot[1], slot[2], slot[3]};
            *reinterpret_cast<int4 *>(s.pos_out + i0) = int4{pos[0], pos[1], pos[2], pos[3]};
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i0 + e < s.tokens) { s.slot_out[i0 + e] = slot[e]; s.pos_out[i0 + e] = pos[e]; }
        }
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
    Step p;
    p.s = s;
    // x / page for x < 2^31: with h = ceil(log2(page)), floor(x m / 2^(31 + h)), m = floor(2^(31 + h) / page) + 1 <= 2^32 - 1
    int h = 0;
    while ((1ll << h) < s.page) ++h;
    p.page_mul = (unsigned)((1ull << (31 + h)) / (unsigned long long)s.page + 1);
    p.page_shift = h;
    // a workgroup per 1024 tokens, four to a thread; they also share out the pages
    int64_t grid = (s.tokens + 1023) / 1024;
    grid = grid < 1 ? 1 : grid > 1024 ? 1024 : grid;
    const unsigned bytes = (unsigned)s.B * 5 * sizeof(int);
    if (bytes > 64 * 1024 &&                                  // (each call: it is the current device's)
        hipFuncSetAttribute(reinterpret_cast<const void *>(sd_pages_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess)
        return SD_EHIP;
    hipLaunchKernelGGL(sd_pages_kernel, dim3((unsigned)grid), dim3(kThreads), bytes, static_cast<hipStream_t>(hip_stream), p);
    return hipGetLastError() == hipSuccess ? SD_OK : SD_EHIP;
}
