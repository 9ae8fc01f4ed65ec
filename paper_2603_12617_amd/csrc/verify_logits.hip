// Verification of drafted tokens from logits (sd_verify_logits): two launches.
//
//   stats   every row of V logits in segments of kSeg, a workgroup each: the largest logit and, of the rows of requests with a
//           temperature, sum 2^((l - top) c), c = log2(e) / tau, of greedy ones the largest's first place.  All segments are independent,
//           so a batch of one request fills V / kSeg workgroups a row and a large one the chip; each logit is read once.
//   draw    per request and kRace places: the rows' partial sums are joined (again by every workgroup of the request: a few
//           hundred numbers from L2, in a fixed order, half a wavefront to a row), the drafts tested, and these places of row n
//           raced: score(x) = weight(x) / noise(x).  Workgroups of a request meet in a 64-bit maximum of
//           (score's bits, lowest place), whose order does not matter; the last one writes n and next.
//
// Bound by the logits' way from HBM: 2 k + 1 rows a request in `stats`, two rows and the noise again in `draw`; beside it `stats` has 11 vector
// instructions a logit (counted: 58 million of a wavefront for 350 million logits), one of them the power of two.  256 requests of 4 drafts, V = 151936,
// bfloat16: 127 us for 700 MB, 5.5 TB/s of the 6.1 that a pure read reaches, and 62 us for the draw's 289 MB, 4.7 TB/s behind a chain of dependent reads.  8 of 4,
// V = 32000, float: 4.8 and 7.8 us, the launch and such chains.
//
// The difference is taken before it is multiplied: of l c - top c each part would be rounded in units of its own size, which for masks of -1e10
// or temperatures of 1e-8 are powers of two of 1 and more.  So the largest logit's weight is 1 whatever its size, no sum is more than its
// number of places, and weights of all segments are relative to the same exact number.  c is kept as a sum of two floats: its own rounding would move
// all weights of a row together, by |l - top| c 6e-8.  The low part is positive, so that l = -inf gives a weight of 0 without a test.  What these few
// instructions cannot do (NaN, +inf, rows of -inf) shows in a workgroup's maximum and sum, and is done again one by one.
#include "../../include/specdec.h"

#include <hip/hip_runtime.h>

namespace {

typedef unsigned long long u64;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kPer = 32;                       // logits of a thread
constexpr int kSeg = kThreads * kPer;          // of a workgroup
// Places of a thread of the draw: half as many as a segment has, so that a few requests spread over twice the workgroups (8, 16, 32 of them, us a
// call: 8 requests of 4 drafts, V = 32000, float: 11.9, 12.2, 13.1; 256 of 4, V = 151936, bfloat16: 208, 189.6, 188.4; 100 of up to 8 without
// a distribution, V = 50257, float16: 24.1, 22.8, 23.8).
constexpr int kRacePer = 16;
constexpr int kRace = kThreads * kRacePer;
constexpr int kMaxSegs = (SD_MAX_V + kSeg - 1) / kSeg;
constexpr float kNone = -__builtin_inff(), kLargest = 3.4028234663852886e38f;
static_assert(kMaxSegs <= 32, "half a wavefront joins a row");

struct Stat { float top, sum; int at; };       // of a row's segment
struct Race { u64 best; unsigned met, pad; };  // of a request, cleared by `stats`

// ---- element types: 16 bytes of logits, at any alignment that the type has ----
struct bf16 { uint16_t u; };
typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned u4h __attribute__((ext_vector_type(4), aligned(2)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float one(const float *p) { return *p; }
__device__ __forceinline__ float one(const bf16 *p) { return __uint_as_float((unsigned)p->u << 16); }
__device__ __forceinline__ float one(const _Float16 *p) { return (float)*p; }
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int kVec = 4;
    typedef f4u Raw;
    static __device__ __forceinline__ float get(const Raw &v, int e) { return v[e]; }
    static __device__ __forceinline__ Raw none() { return Raw{kNone, kNone, kNone, kNone}; }
};
template <> struct Vec<bf16> {
    static constexpr int kVec = 8;
    typedef u4h Raw;
    static __device__ __forceinline__ float get(const Raw &v, int e) { return __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16); }
    static __device__ __forceinline__ Raw none() { return Raw{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}; }
};
template <> struct Vec<_Float16> {
    static constexpr int kVec = 8;
    typedef u4h Raw;
    static __device__ __forceinline__ float get(const Raw &v, int e) { return (float)__builtin_bit_cast(h2, (unsigned)v[e / 2])[e & 1]; }
    static __device__ __forceinline__ Raw none() { return Raw{0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u}; }
};
// kVec logits from place x of a row of V; those past its end are -inf
template <typename T> __device__ __forceinline__ typename Vec<T>::Raw load(const T *row, int x, int V)
{
    typedef Vec<T> E;
    if (x + E::kVec <= V) return *reinterpret_cast<const typename E::Raw *>(row + x);
    typename E::Raw v = E::none();
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (x + e < V) v[e] = row[x + e];
    } else {
        const uint16_t *const h = reinterpret_cast<const uint16_t *>(row) + x;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned lo = x + 2 * e < V ? h[2 * e] : v[e] & 0xffffu, hi = x + 2 * e + 1 < V ? h[2 * e + 1] : v[e] >> 16;
            v[e] = hi << 16 | lo;
        }
    }
    return v;
}
// a thread's logits of segment `seg` of `size`: raw[c] from place place(seg, c) on
template <typename T, int size> __device__ __forceinline__ int place(int seg, int c) { return seg * size + (c * kThreads + (int)threadIdx.x) * Vec<T>::kVec; }

// NaN counts as -inf, +inf as the largest float
__device__ __forceinline__ float clean(float l) { return l == l ? fminf(l, kLargest) : kNone; }

// ---- temperature ----
struct Heat { float hi, lo; };                 // log2(e) / tau as a sum, lo > 0
__device__ __forceinline__ Heat heat(float tau)
{
    const double c = fmax(fmin(1.4426950408889634 / (double)tau, 1e38), 1e-30);
    Heat h;
    h.hi = (float)c;
    if ((double)h.hi > c) h.hi = __uint_as_float(__float_as_uint(h.hi) - 1);
    h.lo = fmaxf((float)(c - (double)h.hi), 1e-37f);
    return h;
}
// the weight of a logit in a row whose largest is `top`, both finite, or l = -inf
__device__ __forceinline__ float power(float l, float top, Heat h)
{
    const float d = l - top;
    return __builtin_amdgcn_exp2f(__builtin_fmaf(d, h.lo, d * h.hi));
}
// the same of any clean logits
__device__ __forceinline__ float power_any(float l, float top, Heat h) { return l > kNone ? power(l, top, h) : 0.f; }

// ---- reductions by lane moves within the wavefront's registers (a trip through LDS per step would be the larger part of a small call) ----
// lanes without a source, and rows outside ROWS, get `none`
template <int CTRL, int ROWS> __device__ __forceinline__ int moved(int v, int none) { return __builtin_amdgcn_update_dpp(none, v, CTRL, ROWS, 0xF, false); }
template <int CTRL, int ROWS> __device__ __forceinline__ float moved(float v, float none) { return __int_as_float(moved<CTRL, ROWS>(__float_as_int(v), __float_as_int(none))); }
template <int CTRL, int ROWS> __device__ __forceinline__ double moved(double v, double none)
{
    const long long u = __double_as_longlong(v), n = __double_as_longlong(none);
    const unsigned lo = (unsigned)moved<CTRL, ROWS>((int)u, (int)n), hi = (unsigned)moved<CTRL, ROWS>((int)(u >> 32), (int)(n >> 32));
    return __longlong_as_double((long long)((u64)hi << 32 | lo));
}
// f over the lanes of each half of a wavefront, in its last lane
template <typename V, typename F> __device__ __forceinline__ V over_half(V v, V none, F f)
{
    v = f(v, moved<0x111, 0xF>(v, none));      // row_shr:1
    v = f(v, moved<0x112, 0xF>(v, none));
    v = f(v, moved<0x114, 0xF>(v, none));
    v = f(v, moved<0x118, 0xF>(v, none));
    return f(v, moved<0x142, 0xA>(v, none));   // row_bcast:15
}
// the last lane of this lane's half
__device__ __forceinline__ int of_half(int v, int lane) { return lane < 32 ? __builtin_amdgcn_readlane(v, 31) : __builtin_amdgcn_readlane(v, 63); }
__device__ __forceinline__ float of_half(float v, int lane) { return __int_as_float(of_half(__float_as_int(v), lane)); }
__device__ __forceinline__ double of_half(double v, int lane)
{
    const long long u = __double_as_longlong(v);
    return __longlong_as_double((long long)((u64)(unsigned)of_half((int)(u >> 32), lane) << 32 | (unsigned)of_half((int)u, lane)));
}
// f over all lanes
template <typename F> __device__ __forceinline__ int over_all(int v, int none, F f)
{
    v = over_half(v, none, f);
    return __builtin_amdgcn_readlane(f(v, moved<0x143, 0xC>(v, none)), 63);      // row_bcast:31
}
template <typename F> __device__ __forceinline__ float over_all(float v, float none, F f)
{
    v = over_half(v, none, f);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f(v, moved<0x143, 0xC>(v, none))), 63));
}
constexpr auto kMax = [](auto a, auto b) { return a > b ? a : b; };
constexpr auto kMin = [](auto a, auto b) { return a < b ? a : b; };
constexpr auto kSum = [](auto a, auto b) { return a + b; };

// the request of a row: the last b with cu[b] <= row (target rows) or cu[b] - b <= row (drafts' rows); by the lanes of a wavefront
__device__ __forceinline__ int request_of(const int32_t *cu, int B, int row, bool draft, int lane)
{
    int lo = 0, n = B;                         // b in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 63) / 64, b = lo + lane * step;
        const bool in = lane * step < n && cu[b] - (draft ? b : 0) <= row;
        const u64 mask = __ballot(in);
        const int last = mask ? 63 - __builtin_clzll(mask) : 0;
        n = min(step, n - last * step);
        lo += last * step;
    }
    return lo;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sd_stats_kernel(const sd_logits s, Stat *stat, Race *race)
{
    typedef Vec<T> E;
    constexpr int kC = kPer / E::kVec;
    __shared__ float top_sh[kWaves], sum_sh[kWaves];
    __shared__ int at_sh[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int B = (int)s.B, V = (int)s.V, rows = (int)s.rows;
    const int row = blockIdx.x, seg = blockIdx.y;
    if (seg == 0 && row < B && tid == 0) race[row] = Race{0, 0, 0};
    const bool draft = row >= rows;
    const T *l = draft ? static_cast<const T *>(s.q) + (int64_t)(row - rows) * s.q_stride : static_cast<const T *>(s.p) + (int64_t)row * s.p_stride;
    typename E::Raw raw[kC];
#pragma unroll
    for (int c = 0; c < kC; ++c) raw[c] = load(l, place<T, kSeg>(seg, c), V);
    const float tau = s.tau[request_of(s.cu, B, draft ? row - rows : row, draft, lane)];
    const bool hot = tau > 0.f;
    const Heat h = heat(hot ? tau : 1.f);
    float top = kNone;                         // (a maximum leaves NaN out)
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
        for (int e = 0; e < E::kVec; ++e) top = fmaxf(top, E::get(raw[c], e));
    top = over_all(top, kNone, kMax);
    if (lane == 0) top_sh[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, top_sh[w]);
    int at = 0x7fffffff;
    float sum = 0.f;
    if (hot) {
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int e = 0; e < E::kVec; ++e) sum += power(E::get(raw[c], e), top, h);
        if (sum != sum) {
            sum = 0.f;
#pragma unroll
            for (int c = 0; c < kC; ++c)
#pragma unroll
                for (int e = 0; e < E::kVec; ++e) sum += power_any(clean(E::get(raw[c], e)), clean(top), h);
        }
    } else {
        const float most = clean(top);         // (of +inf and the largest float the first one counts)
#pragma unroll
        for (int c = kC - 1; c >= 0; --c)
#pragma unroll
            for (int e = E::kVec - 1; e >= 0; --e)
                if (E::get(raw[c], e) >= most) at = place<T, kSeg>(seg, c) + e;
    }
    if (hot) sum = over_all(sum, 0.f, kSum); else at = over_all(at, 0x7fffffff, kMin);
    if (lane == 0) { at_sh[wave] = at; sum_sh[wave] = sum; }
    __syncthreads();
    if (tid == 0) {
        Stat r;
        r.top = clean(top);
        r.sum = (sum_sh[0] + sum_sh[1]) + (sum_sh[2] + sum_sh[3]);
        r.at = min(min(at_sh[0], at_sh[1]), min(at_sh[2], at_sh[3]));
        stat[(int64_t)row * gridDim.y + seg] = r;
    }
}

// A row's parts joined by the 32 lanes of half a wavefront, in a fixed order; each of them gets the result.
struct Row { float top, inv; int best; };      // inv: 1 / the sum of the weights, 0 without a finite logit
__device__ __forceinline__ Stat part(const Stat *stat, int segs, int lane)
{
    const int s = lane & 31;
    return s < segs ? stat[s] : Stat{kNone, 0.f, 0x7fffffff};
}
__device__ __forceinline__ Row join(const Stat &r, Heat h, int lane)
{
    const float top = of_half(over_half(r.top, kNone, kMax), lane);
    const int best = of_half(over_half(r.top == top ? r.at : 0x7fffffff, 0x7fffffff, kMin), lane);
    double sum = (double)r.sum * (double)power_any(r.top, top, h);
    sum = of_half(over_half(sum, 0.0, kSum), lane);
    Row w;
    w.top = top;
    w.best = top > kNone ? best : 0;
    w.inv = top > kNone ? (float)(1.0 / sum) : 0.f;
    return w;
}

// w - v i with the product rounded by itself, as w's was: equal rows leave nothing
__device__ __forceinline__ float less(float w, float v, float i)
{
#pragma clang fp contract(off)
    const float x = v * i;
    return w - x;
}

// a probability
__device__ __forceinline__ float weight(float l, const Row &r, Heat h) { return power_any(clean(l), r.top, h) * r.inv; }

// Scores are taken with the reciprocal instruction, which is off by a unit in the last place, less than a weight is; a division is a chain of about ten.
// larger scores win, of equal ones the lowest place
__device__ __forceinline__ u64 entry(float score, int x) { return ((u64)__float_as_uint(score) << 32) | (0xffffffffu - (unsigned)x); }
__device__ __forceinline__ u64 larger(u64 a, u64 b) { return a > b ? a : b; }

// the entry of a workgroup's best score, which is positive or 0 for none
__device__ __forceinline__ u64 first_of(float score, int x, u64 *sh)
{
    const float best = over_all(score, 0.f, kMax);
    const int at = over_all(score == best ? x : 0x7fffffff, 0x7fffffff, kMin);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = best > 0.f ? entry(best, at) : 0;
    __syncthreads();
    return larger(larger(sh[0], sh[1]), larger(sh[2], sh[3]));
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sd_draw_kernel(const sd_logits s, const Stat *stat, Race *race, int segs, int32_t *n_out, int32_t *next_out)
{
    typedef Vec<T> E;
    constexpr int kC = kRacePer / E::kVec;
    constexpr int kKeep = SD_MAX_K + 1;                     // rows whose parts are kept joined; further ones are joined again
    __shared__ Row row_sh[2][kKeep];
    __shared__ int n_sh, last_sh;
    __shared__ u64 best_sh[kWaves];
    const int tid = threadIdx.x, lane = tid & 63;
    const int V = (int)s.V, rows = (int)s.rows, drafts = rows - (int)s.B;
    const int b = blockIdx.x, seg = blockIdx.y;
    const int row0 = min(max(s.cu[b], 0), rows - 1), row1 = min(max(s.cu[b + 1], row0 + 1), rows);
    const int first = min(max(row0 - b, 0), drafts), k = min(row1 - row0 - 1, drafts - first);   // drafts first .. first + k - 1
    const float tau = s.tau[b];
    const bool hot = tau > 0.f;
    const Heat h = heat(hot ? tau : 1.f);
    const T *P = static_cast<const T *>(s.p), *Q = static_cast<const T *>(s.q);
    const float *noise = s.noise + (int64_t)b * s.noise_stride;
    typename Vec<float>::Raw e[kC * E::kVec / 4];
    if (hot) {                                              // (under way while the drafts are tested)
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int i = 0; i < E::kVec / 4; ++i) e[c * (E::kVec / 4) + i] = load(noise, place<T, kRace>(seg, c) + 4 * i, V);
    }
    if (tid == 0) n_sh = k;
    __syncthreads();
    // half a wavefront to a draft: its target row and, if there is one, its own
    for (int j0 = 0; j0 <= k; j0 += kThreads / 32) {
        const int j = j0 + tid / 32;
        if (j <= k) {
            int x = 0;
            float pl = 0.f, ql = 0.f, r = 0.f;
            if (j < k) {
                x = min(max(s.tok[first + j], 0), V - 1);
                if (hot) {
                    r = s.r[first + j];
                    pl = one(P + (int64_t)(row0 + j) * s.p_stride + x);
                    if (Q) ql = one(Q + (int64_t)(first + j) * s.q_stride + x);
                }
            }
            const Stat ps = part(stat + (int64_t)(row0 + j) * segs, segs, lane), qs = Q && j < k ? part(stat + (int64_t)(rows + first + j) * segs, segs, lane) : ps;
            const Row p = join(ps, h, lane);
            Row q{0.f, 0.f, 0};
            if (Q && j < k) q = join(qs, h, lane);
            if ((tid & 31) == 0) {
                if (j < kKeep) { row_sh[0][j] = p; row_sh[1][j] = q; }
                if (j < k && !(hot ? __fmul_rn(r, Q ? weight(ql, q, h) : 1.f) <= weight(pl, p, h) : x == p.best)) atomicMin(&n_sh, j);
            }
        }
        __syncthreads();
        if (n_sh < j0 + kThreads / 32) break;               // (the same for everyone: nobody writes before all have read)
        __syncthreads();
    }
    const int n = n_sh;
    const bool rejected = n < k;
    Row p, q{0.f, 0.f, 0};
    if (n < kKeep) { p = row_sh[0][n]; q = row_sh[1][n]; }
    else {
        p = join(part(stat + (int64_t)(row0 + n) * segs, segs, lane), h, lane);
        if (Q && rejected) q = join(part(stat + (int64_t)(rows + first + n) * segs, segs, lane), h, lane);
    }
    if (!hot || p.top == kNone) {
        if (seg == 0 && tid == 0) { n_out[b] = n; next_out[b] = p.top == kNone ? 0 : p.best; }
        return;
    }
    const T *prow = P + (int64_t)(row0 + n) * s.p_stride, *qrow = Q && rejected ? Q + (int64_t)(first + n) * s.q_stride : nullptr;
    typename E::Raw f[kC], g[kC];
#pragma unroll
    for (int c = 0; c < kC; ++c) f[c] = load(prow, place<T, kRace>(seg, c), V);
    if (qrow) {
#pragma unroll
        for (int c = 0; c < kC; ++c) g[c] = load(qrow, place<T, kRace>(seg, c), V);
    } else {
#pragma unroll
        for (int c = 0; c < kC; ++c) g[c] = E::none();
    }
    const int drafted = rejected && !Q ? min(max(s.tok[first + n], 0), V - 1) : -1;
    float won = 0.f;
    int at = 0;
    if (fmaxf(p.top, q.top) < kLargest) {
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int i = 0; i < E::kVec; ++i) {
                float w = power(E::get(f[c], i), p.top, h) * p.inv;
                // (the maximum takes what is no number for 0)
                if (qrow) w = less(w, fmaxf(power(E::get(g[c], i), q.top, h), 0.f), q.inv);
                else if (drafted == place<T, kRace>(seg, c) + i) w = 0.f;
                const float sc = w * __builtin_amdgcn_rcpf(e[(c * E::kVec + i) / 4][i % 4]);
                if (sc > won) { won = sc; at = c * E::kVec + i; }     // (places ascend within a thread: of equal scores the first stays)
            }
    } else {
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int i = 0; i < E::kVec; ++i) {
                float w = weight(E::get(f[c], i), p, h);
                if (qrow) w = less(w, power_any(clean(E::get(g[c], i)), q.top, h), q.inv);
                else if (drafted == place<T, kRace>(seg, c) + i) w = 0.f;
                const float sc = w * __builtin_amdgcn_rcpf(e[(c * E::kVec + i) / 4][i % 4]);
                if (sc > won) { won = sc; at = c * E::kVec + i; }
            }
    }
    u64 best = first_of(won, place<T, kRace>(seg, at / E::kVec) + at % E::kVec, best_sh);
    if (tid == 0) {
        bool last = true;
        if (gridDim.y > 1) {
            // Only atomics carry data between the workgroups, each done (its old value is back) before the next is issued: a fence,
            // which would write back and drop caches, is not needed for that.
            if (best) {
                u64 old = __hip_atomic_fetch_max(&race[b].best, best, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                asm volatile("s_waitcnt vmcnt(0)" : "+v"(old)::"memory");
            }
            last = __hip_atomic_fetch_add(&race[b].met, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.y - 1;
            if (last) best = __hip_atomic_fetch_max(&race[b].best, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        if (last && (best || !rejected)) { n_out[b] = n; next_out[b] = best ? (int)(0xffffffffu - (unsigned)best) : 0; }
        last_sh = last && !best && rejected;
    }
    __syncthreads();
    if (!last_sh) return;
    // The residual is zero everywhere: the last workgroup races the target's whole row.
    won = 0.f;
    int x_won = 0;
    for (int x = tid; x < V; x += kThreads) {
        const float sc = weight(one(prow + x), p, h) * __builtin_amdgcn_rcpf(noise[x]);
        if (sc > won) { won = sc; x_won = x; }
    }
    best = first_of(won, x_won, best_sh);
    if (tid == 0) { n_out[b] = n; next_out[b] = best ? (int)(0xffffffffu - (unsigned)best) : 0; }
}

bool misaligned(const void *p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

int64_t stat_rows(const sd_logits &s) { return s.rows + (s.q ? s.rows - s.B : 0); }

int check(const sd_logits &s)
{
    if (s.B <= 0 || s.V <= 0 || s.rows < s.B || s.p_stride < s.V || s.noise_stride < s.V) return SD_EINVAL;
    if (s.dtype != SD_F32 && s.dtype != SD_BF16 && s.dtype != SD_F16) return SD_EINVAL;
    if (s.q && s.rows > s.B && s.q_stride < s.V) return SD_EINVAL;
    if (s.V > SD_MAX_V || s.B > SD_MAX_REQUESTS || s.rows > (1 << 24)) return SD_EUNSUPPORTED;
    if (stat_rows(s) * kThreads > 0xffffffffll) return SD_EUNSUPPORTED;      // (threads of a launch)
    return SD_OK;
}
int segments(const sd_logits &s) { return (int)((s.V + kSeg - 1) / kSeg); }
size_t race_bytes(const sd_logits &s) { return (size_t)s.B * sizeof(Race); }

template <typename T> void launch(const sd_logits &s, Stat *stat, Race *race, int32_t *n, int32_t *next, hipStream_t st)
{
    const unsigned segs = (unsigned)segments(s);
    hipLaunchKernelGGL(sd_stats_kernel<T>, dim3((unsigned)stat_rows(s), segs), dim3(kThreads), 0, st, s, stat, race);
    hipLaunchKernelGGL(sd_draw_kernel<T>, dim3((unsigned)s.B, (unsigned)((s.V + kRace - 1) / kRace)), dim3(kThreads), 0, st, s, stat, race, (int)segs, n, next);
}

}  // namespace

extern "C" {

size_t sd_verify_logits_workspace_bytes(const sd_logits *a)
{
    if (!a || check(*a) != SD_OK) return 0;
    return race_bytes(*a) + (size_t)stat_rows(*a) * segments(*a) * sizeof(Stat);
}

int sd_verify_logits(const sd_logits *a, int32_t *n_dev, int32_t *next_dev, void *ws, size_t ws_bytes, void *hip_stream)
{
    if (!a) return SD_EINVAL;
    const sd_logits &s = *a;
    const int rc = check(s);
    if (rc != SD_OK) return rc;
    const unsigned es = s.dtype == SD_F32 ? 4 : 2;
    if (!s.p || !s.noise || !s.tau || !s.cu || !n_dev || !next_dev || !ws) return SD_EINVAL;
    if (s.rows > s.B && (!s.tok || !s.r)) return SD_EINVAL;
    if (misaligned(s.p, es) || misaligned(s.q, es) || misaligned(s.tok, 4) || misaligned(s.r, 4) || misaligned(s.noise, 4) || misaligned(s.tau, 4) ||
        misaligned(s.cu, 4) || misaligned(n_dev, 4) || misaligned(next_dev, 4) || misaligned(ws, 16))
        return SD_EINVAL;
    if (ws_bytes < sd_verify_logits_workspace_bytes(a)) return SD_ENOMEM;
    Race *race = static_cast<Race *>(ws);
    Stat *stat = reinterpret_cast<Stat *>(static_cast<char *>(ws) + race_bytes(s));
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (s.dtype == SD_F32) launch<float>(s, stat, race, n_dev, next_dev, st);
    else if (s.dtype == SD_BF16) launch<bf16>(s, stat, race, n_dev, next_dev, st);
    else launch<_Float16>(s, stat, race, n_dev, next_dev, st);
    return hipGetLastError() == hipSuccess ? SD_OK : SD_EHIP;
}

}  // extern "C"
