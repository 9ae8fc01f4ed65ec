// Verification of drafted tokens from logits (sd_verify_logits): two launches.
//
//   stats   every row of V logits in segments of kSeg, a workgroup each: largest logit, its first place, and
//           sum exp((l - segment's largest) / tau).  All segments are independent, so a batch of one request fills
//           V / kSeg workgroups a row and a large one the chip; each logit is read once, and stays in registers between
//           the maximum and the sum.
//   draw    per request and segment: the rows' partial sums are joined (again by every workgroup of the request: a few
//           hundred numbers from L2, in a fixed order), the drafts tested, and the segment of row n raced:
//           score(x) = weight(x) / noise(x).  Workgroups of a request meet in a 64-bit maximum of
//           (score's bits, lowest place), whose order does not matter; the last one writes n and next.
//
// Bound by the logits' way from HBM: 2 k + 1 rows a request in `stats`, two rows and the noise again in `draw`.
//
// exp((l - m) / tau) = 2^((l - m) log2e / tau): the factor is kept as a sum of two floats, since its own rounding would move all
// of a row's weights together, by |l - m| / tau 6e-8.
#include "../../include/specdec.h"

#include <hip/hip_runtime.h>

namespace {

typedef unsigned long long u64;
typedef unsigned int u4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kPer = 32;                       // logits of a thread
constexpr int kSeg = kThreads * kPer;          // of a workgroup
constexpr float kNone = -__builtin_inff();

struct Stat { float top, sum; int at; };       // of a row's segment; sum is of exp((l - top) / tau)
struct Race { u64 residual, target; unsigned met, pad; };   // of a request, cleared by `stats`

// ---- element types ----
template <typename T> struct Vec;              // kVec logits of 16 bytes
template <> struct Vec<float> {
    static constexpr int kVec = 4;
    static __device__ __forceinline__ void get(u4 v, float (&f)[4]) { for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(v[e]); }
    static __device__ __forceinline__ float one(const float *p) { return *p; }
};
struct bf16 { uint16_t u; };
template <> struct Vec<bf16> {
    static constexpr int kVec = 8;
    static __device__ __forceinline__ void get(u4 v, float (&f)[8])
    {
        for (int e = 0; e < 4; ++e) { f[2 * e] = __uint_as_float(v[e] << 16); f[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u); }
    }
    static __device__ __forceinline__ float one(const bf16 *p) { return __uint_as_float((unsigned)p->u << 16); }
};
template <> struct Vec<_Float16> {
    static constexpr int kVec = 8;
    static __device__ __forceinline__ void get(u4 v, float (&f)[8])
    {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        for (int e = 0; e < 4; ++e) { const h2 h = __builtin_bit_cast(h2, (unsigned)v[e]); f[2 * e] = (float)h[0]; f[2 * e + 1] = (float)h[1]; }
    }
    static __device__ __forceinline__ float one(const _Float16 *p) { return (float)*p; }
};

// NaN counts as -inf, +inf as the largest float
__device__ __forceinline__ float logit(float l) { return l == l ? fminf(l, 3.4028234663852886e38f) : kNone; }

// the logits of a thread's share of segment `seg`: places seg * kSeg + (c * kThreads + tid) * kVec + e
template <typename T, bool WIDE>
__device__ __forceinline__ void load_row(const T *row, int seg, int V, float (&f)[kPer])
{
    constexpr int kVec = Vec<T>::kVec;
    if (WIDE) {
        u4 v[kPer / kVec];
#pragma unroll
        for (int c = 0; c < kPer / kVec; ++c) {
            const int x = seg * kSeg + (c * kThreads + (int)threadIdx.x) * kVec;
            if (x < V) v[c] = *reinterpret_cast<const u4 *>(row + x);
        }
#pragma unroll
        for (int c = 0; c < kPer / kVec; ++c) {
            const int x = seg * kSeg + (c * kThreads + (int)threadIdx.x) * kVec;
            float g[kVec];
            Vec<T>::get(v[c], g);
#pragma unroll
            for (int e = 0; e < kVec; ++e) f[c * kVec + e] = x < V ? logit(g[e]) : kNone;
        }
    } else {
#pragma unroll
        for (int c = 0; c < kPer / kVec; ++c)
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const int x = seg * kSeg + (c * kVec + e) * kThreads + (int)threadIdx.x;
                f[c * kVec + e] = x < V ? logit(Vec<T>::one(row + x)) : kNone;
            }
    }
}
// the place of f[i] above
template <typename T, bool WIDE> __device__ __forceinline__ int place(int seg, int i)
{
    constexpr int kVec = Vec<T>::kVec;
    return WIDE ? seg * kSeg + ((i / kVec) * kThreads + (int)threadIdx.x) * kVec + i % kVec : seg * kSeg + i * kThreads + (int)threadIdx.x;
}

// ---- temperature: exp((l - top) / tau) ----
struct Heat { float hi, lo; };                 // log2(e) / tau as a sum
__device__ __forceinline__ Heat heat(float tau)
{
    const double c = fmin(1.4426950408889634 / (double)tau, 1e30);
    Heat h;
    h.hi = (float)c;
    h.lo = (float)(c - (double)h.hi);
    return h;
}
// (below 2^-125 of the largest: 0, as for l = -inf and where l - top is no number)
__device__ __forceinline__ float weight(float l, float top, Heat h)
{
    const float d = l - top;
    return d * h.hi >= -125.f ? __builtin_amdgcn_exp2f(__builtin_fmaf(d, h.hi, d * h.lo)) : 0.f;
}

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

template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads) sd_stats_kernel(const sd_logits s, Stat *stat, Race *race)
{
    __shared__ float top_sh[kWaves], sum_sh[kWaves];
    __shared__ int at_sh[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int B = (int)s.B, V = (int)s.V, rows = (int)s.rows;
    const int row = blockIdx.x, seg = blockIdx.y;
    if (seg == 0 && row < B && tid == 0) race[row] = Race{0, 0, 0, 0};
    const bool draft = row >= rows;
    const T *l = draft ? static_cast<const T *>(s.q) + (int64_t)(row - rows) * s.q_stride : static_cast<const T *>(s.p) + (int64_t)row * s.p_stride;
    float f[kPer];
    load_row<T, WIDE>(l, seg, V, f);
    const float tau = s.tau[request_of(s.cu, B, draft ? row - rows : row, draft, lane)];
    float top = kNone;
#pragma unroll
    for (int i = 0; i < kPer; ++i) top = fmaxf(top, f[i]);
#pragma unroll
    for (int sh = 32; sh >= 1; sh >>= 1) top = fmaxf(top, __shfl_xor(top, sh));
    if (lane == 0) top_sh[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, top_sh[w]);
    const bool hot = tau > 0.f;
    const Heat h = heat(hot ? tau : 1.f);
    int at = 0x7fffffff;
    float sum = 0.f;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i) {
        if (f[i] == top) at = min(at, place<T, WIDE>(seg, i));
        sum += weight(f[i], top, h);
    }
#pragma unroll
    for (int sh = 32; sh >= 1; sh >>= 1) { at = min(at, __shfl_xor(at, sh)); sum += __shfl_xor(sum, sh); }
    if (lane == 0) { at_sh[wave] = at; sum_sh[wave] = sum; }
    __syncthreads();
    if (tid == 0) {
        Stat r;
        r.top = top;
        r.sum = (sum_sh[0] + sum_sh[1]) + (sum_sh[2] + sum_sh[3]);
        r.at = min(min(at_sh[0], at_sh[1]), min(at_sh[2], at_sh[3]));
        stat[(int64_t)row * gridDim.y + seg] = r;
    }
}

// a row's parts joined by the lanes of a wavefront, in a fixed order; every lane gets the result
struct Row { float top; float inv; int best; };   // inv: 1 / sum exp((l - top) / tau), 0 without a finite logit
__device__ __forceinline__ Row join(const Stat *stat, int segs, Heat h, int lane)
{
    float top = kNone;
    int best = 0x7fffffff;
    for (int s = lane; s < segs; s += 64) top = fmaxf(top, stat[s].top);
#pragma unroll
    for (int sh = 32; sh >= 1; sh >>= 1) top = fmaxf(top, __shfl_xor(top, sh));
    double sum = 0.0;
    for (int s = lane; s < segs; s += 64) {
        const Stat r = stat[s];
        if (r.top == top) best = min(best, r.at);
        if (r.top > kNone) sum += (double)r.sum * (double)weight(r.top, top, h);
    }
#pragma unroll
    for (int sh = 32; sh >= 1; sh >>= 1) { best = min(best, __shfl_xor(best, sh)); sum += __shfl_xor(sum, sh); }
    Row r;
    r.top = top;
    r.best = best;
    r.inv = top > kNone ? (float)(1.0 / sum) : 0.f;
    return r;
}

// larger scores win, of equal ones the lowest place
__device__ __forceinline__ u64 entry(float score, int x) { return ((u64)__float_as_uint(score) << 32) | (0xffffffffu - (unsigned)x); }

template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads) sd_draw_kernel(const sd_logits s, const Stat *stat, Race *race, int segs, int32_t *n_out, int32_t *next_out)
{
    __shared__ int n_sh;
    __shared__ u64 best_sh[2][kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int V = (int)s.V, rows = (int)s.rows, drafts = rows - (int)s.B;
    const int b = blockIdx.x, seg = blockIdx.y;
    const int row0 = min(max(s.cu[b], 0), rows - 1), row1 = min(max(s.cu[b + 1], row0 + 1), rows);
    const int k = row1 - row0 - 1, first = min(max(row0 - b, 0), drafts);   // drafts first .. first + k - 1
    const float tau = s.tau[b];
    const bool hot = tau > 0.f;
    const Heat h = heat(hot ? tau : 1.f);
    const T *P = static_cast<const T *>(s.p), *Q = static_cast<const T *>(s.q);
    if (tid == 0) n_sh = k;
    __syncthreads();
    for (int j = wave; j < k && first + j < drafts; j += kWaves) {
        const int x = min(max(s.tok[first + j], 0), V - 1);
        const Row p = join(stat + (int64_t)(row0 + j) * segs, segs, h, lane);
        bool ok;
        if (hot) {
            const float px = weight(logit(Vec<T>::one(P + (int64_t)(row0 + j) * s.p_stride + x)), p.top, h) * p.inv;
            float qx = 1.f;
            if (Q) {
                const Row q = join(stat + (int64_t)(rows + first + j) * segs, segs, h, lane);
                qx = weight(logit(Vec<T>::one(Q + (int64_t)(first + j) * s.q_stride + x)), q.top, h) * q.inv;
            }
            ok = __fmul_rn(s.r[first + j], qx) <= px;
        } else {
            ok = x == p.best;
        }
        if (!ok) { if (lane == 0) atomicMin(&n_sh, j); break; }
    }
    __syncthreads();
    const int n = n_sh;
    const Row p = join(stat + (int64_t)(row0 + n) * segs, segs, h, lane);
    if (!hot || p.top == kNone) {
        if (seg == 0 && tid == 0) { n_out[b] = n; next_out[b] = p.top == kNone ? 0 : p.best; }
        return;
    }
    const bool rejected = n < k && first + n < drafts;
    float f[kPer], g[kPer], e[kPer];
    load_row<T, WIDE>(P + (int64_t)(row0 + n) * s.p_stride, seg, V, f);
    const float *noise = s.noise + (int64_t)b * s.noise_stride;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int x = place<T, WIDE>(seg, i);
        e[i] = x < V ? noise[x] : 1.f;
    }
    Row q{0.f, 0.f, 0};
    int drafted = -1;
    if (rejected) {
        if (Q) {
            q = join(stat + (int64_t)(rows + first + n) * segs, segs, h, lane);
            load_row<T, WIDE>(Q + (int64_t)(first + n) * s.q_stride, seg, V, g);
        } else {
            drafted = min(max(s.tok[first + n], 0), V - 1);
        }
    }
    // the races for the residual and for the target (which counts where the residual is zero everywhere)
    float won[2] = {0.f, 0.f};
    int at[2] = {0x7fffffff, 0x7fffffff};
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int x = place<T, WIDE>(seg, i);
        const float w = weight(f[i], p.top, h) * p.inv;
        float left = w;
        if (rejected) left = Q ? w - weight(g[i], q.top, h) * q.inv : x == drafted ? 0.f : w;
        // (places of a thread ascend, so of equal scores the first stays)
        if (left > 0.f) { const float sc = left / e[i]; if (sc > won[0]) { won[0] = sc; at[0] = x; } }
        if (rejected && w > 0.f) { const float sc = w / e[i]; if (sc > won[1]) { won[1] = sc; at[1] = x; } }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        u64 v = won[c] > 0.f ? entry(won[c], at[c]) : 0;
#pragma unroll
        for (int sh = 32; sh >= 1; sh >>= 1) { const u64 o = __shfl_xor(v, sh); v = o > v ? o : v; }
        if (lane == 0) best_sh[c][wave] = v;
    }
    __syncthreads();
    if (tid == 0) {
        u64 v[2] = {0, 0};
#pragma unroll
        for (int c = 0; c < 2; ++c)
            for (int w = 0; w < kWaves; ++w) v[c] = best_sh[c][w] > v[c] ? best_sh[c][w] : v[c];
        if (segs > 1) {
            // only atomics carry data between the workgroups, so their order is all that is needed
            if (v[0]) atomicMax(&race[b].residual, v[0]);
            if (v[1]) atomicMax(&race[b].target, v[1]);
            __threadfence();
            if (atomicAdd(&race[b].met, 1u) != (unsigned)segs - 1) return;
            __threadfence();
            v[0] = atomicMax(&race[b].residual, 0ull);
            v[1] = atomicMax(&race[b].target, 0ull);
        }
        const u64 best = v[0] ? v[0] : v[1];
        n_out[b] = n;
        next_out[b] = best ? (int)(0xffffffffu - (unsigned)best) : 0;
    }
}

bool misaligned(const void *p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

int check(const sd_logits &s)
{
    if (s.B <= 0 || s.V <= 0 || s.rows < s.B || s.p_stride < s.V || s.noise_stride < s.V) return SD_EINVAL;
    if (s.dtype != SD_F32 && s.dtype != SD_BF16 && s.dtype != SD_F16) return SD_EINVAL;
    if (s.q && s.rows > s.B && s.q_stride < s.V) return SD_EINVAL;
    if (s.V > SD_MAX_V || s.B > SD_MAX_REQUESTS || s.rows > (1 << 24)) return SD_EUNSUPPORTED;
    return SD_OK;
}
int segments(const sd_logits &s) { return (int)((s.V + kSeg - 1) / kSeg); }
int64_t stat_rows(const sd_logits &s) { return s.rows + (s.q ? s.rows - s.B : 0); }
size_t race_bytes(const sd_logits &s) { return (size_t)s.B * sizeof(Race); }

template <typename T, bool WIDE> void launch(const sd_logits &s, Stat *stat, Race *race, int32_t *n, int32_t *next, hipStream_t st)
{
    const unsigned segs = (unsigned)segments(s);
    hipLaunchKernelGGL((sd_stats_kernel<T, WIDE>), dim3((unsigned)stat_rows(s), segs), dim3(kThreads), 0, st, s, stat, race);
    hipLaunchKernelGGL((sd_draw_kernel<T, WIDE>), dim3((unsigned)s.B, segs), dim3(kThreads), 0, st, s, stat, race, (int)segs, n, next);
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
    // 16-byte loads need rows that start and end on 16 bytes
    const unsigned vec = 16 / es;
    const bool wide = s.V % vec == 0 && s.p_stride % vec == 0 && !misaligned(s.p, 16) && (!s.q || (s.q_stride % vec == 0 && !misaligned(s.q, 16)));
    if (s.dtype == SD_F32) { if (wide) launch<float, true>(s, stat, race, n_dev, next_dev, st); else launch<float, false>(s, stat, race, n_dev, next_dev, st); }
    else if (s.dtype == SD_BF16) { if (wide) launch<bf16, true>(s, stat, race, n_dev, next_dev, st); else launch<bf16, false>(s, stat, race, n_dev, next_dev, st); }
    else { if (wide) launch<_Float16, true>(s, stat, race, n_dev, next_dev, st); else launch<_Float16, false>(s, stat, race, n_dev, next_dev, st); }
    return hipGetLastError() == hipSuccess ? SD_OK : SD_EHIP;
}

}  // extern "C"
