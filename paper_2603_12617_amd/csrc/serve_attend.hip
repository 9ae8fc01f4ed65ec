// Attention of a chunk of new tokens over a paged cache (sd_attend).
//
// The rows of a request and key head are its (token, query head of the group) pairs, R = token * G + head, so the G
// heads that share a key head share its keys' way through LDS.  A workgroup works a tile of rows over a range of keys in one
// pass with a running maximum and sum per row.  Both products go through the 32x32x16 matrix instructions, transposed:
//
//   S^T (keys x rows)  = K Q^T     A: 32 keys from LDS, 16 bytes a lane;  B: 32 rows of q, in registers for the whole pass
//   O^T (D x rows)    += V^T P^T   A: V from LDS, transposed by the read (ds_read_tr);  B: the weights
//
// A lane then holds 16 scores of ONE row (column lane & 31; the other half of its keys is in lane ^ 32): the maximum and
// sum of a row are in-lane but for one exchange, the row's scale factors are a register of the lane, and the weights, rounded to
// the cache's type (the products take both sides in one type; keeping more of them would be a second set of products, and the error against 64 bits is 1.35
// times that of the rounded exact result as it is), are already where the second product wants them: register r of half h is key
// 8 (r >> 2) + 4 h + (r & 3) of 32, and since a sum over keys may take them in any order, the V operand is read in
// that order.  Weights are not moved between lanes or through LDS.
//
// Keys and values go from the pages to LDS without passing registers (global_load_lds), one tile or two ahead of the products,
// their 16-byte pieces permuted within a row (at the source, LDS order being fixed) so that the reads above find different banks.
//
// Two shapes of a workgroup:
//   four wavefronts of 32 rows each that load and use the same tiles of 64 keys, one tile ahead (LDS: 64 KB at D = 128, two workgroups to a compute unit;
//   wavefronts without a row only load).  Prompts' chunks, bound by the matrix units: 4 x 2048 tokens of 32 heads over 8192 keys of 8, D = 128: 945 us,
//   1.0 PFLOP/s of the 1.16 that a large matrix product reaches; the softmax's vector instructions beside the products keep these from
//   more.  And decoding with keys split to fill the chip, bound by the cache's way from HBM: 2 x 5 tokens over 100000 keys, D = 128, 151 us, 5.4 TB/s
//   of the 6.1 that a pure read reaches.
//   one tile of 32 rows, and two wavefronts with 32 keys of their own, two tiles ahead each, that never wait for each other until they are joined in LDS at the
//   end: decoding of whole requests, of which the long ones end alone on their compute units (64 x 5 tokens over 200 to 4096 keys, 115 us, 5.1 TB/s).
// Where tiles are few, the range of keys is split over workgroups, and a second kernel joins their parts.
#include "../../include/specdec.h"

#include <hip/hip_runtime.h>

#include <math.h>

#include <type_traits>

namespace {

typedef unsigned int u2 __attribute__((ext_vector_type(2)));
typedef unsigned int u4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

// ---- element types ----
template <typename T> __device__ __forceinline__ f16v mfma(u4 a, u4 b, f16v c);
template <> __device__ __forceinline__ f16v mfma<__bf16>(u4 a, u4 b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f16v mfma<_Float16>(u4 a, u4 b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
// Weights are powers of two times 2^kLift.  The largest is at most 2^8 (the maximum that they are relative to may lag by that); float16 holds up to
// 2^15.9 and nothing below 2^-25, so of a lift of 7 no weight is too large, and those between 2^-25 and 2^-32 of the largest still count: without it 131072
// keys of 2^-25.02 beside one of 1 were 0 in the values' sum but not in the weights', 0.4 % of the result.  bfloat16 has the range of float32.
template <typename T> constexpr float kLift = 0.f;
template <> constexpr float kLift<_Float16> = 7.f;
// two floats rounded to nearest even
template <typename T> __device__ __forceinline__ unsigned pack(float x, float y);
template <> __device__ __forceinline__ unsigned pack<__bf16>(float x, float y) { const f2 f = {x, y}; return __builtin_bit_cast(unsigned, __builtin_convertvector(f, b2)); }
template <> __device__ __forceinline__ unsigned pack<_Float16>(float x, float y) { const f2 f = {x, y}; return __builtin_bit_cast(unsigned, __builtin_convertvector(f, h2)); }

// the value of lane ^ 32 and this lane's, in some order
__device__ __forceinline__ f2 halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}

// the next `n` instructions of a kind (0x8 matrix products, 0x100 reads of LDS), as the compiler orders them
template <int MASK> __device__ __forceinline__ void order(int n)
{
    switch (n) {
        case 1: __builtin_amdgcn_sched_group_barrier(MASK, 1, 0); break;
        case 2: __builtin_amdgcn_sched_group_barrier(MASK, 2, 0); break;
        case 4: __builtin_amdgcn_sched_group_barrier(MASK, 4, 0); break;
        case 8: __builtin_amdgcn_sched_group_barrier(MASK, 8, 0); break;
        default: break;
    }
}
// f(0), f(1), .. f(N - 1), each with its number as a type
template <int N, int I = 0, typename F> __device__ __forceinline__ void unroll(F f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        unroll<N, I + 1>(f);
    }
}
// an address from lane I of each 16 lanes (kSides = 2: from lane 2 I for the first eight of them, lane 2 I + 1 for the others)
template <int I, int kSides> __device__ __forceinline__ int from_lane(int x)
{
    if constexpr (kSides == 1) return __builtin_amdgcn_mov_dpp(x, 0x150 + I, 0xF, 0xF, false);                       // row_newbcast
    else return __builtin_amdgcn_update_dpp(__builtin_amdgcn_mov_dpp(x, 0x150 + 2 * I, 0xF, 0xF, false), x, 0x150 + 2 * I + 1, 0xF, 0xC, false);
}
template <int I, int kSides> __device__ __forceinline__ const char *from_lane(const char *x)
{
    const uint64_t u = reinterpret_cast<uint64_t>(x);
    const uint64_t lo = (unsigned)from_lane<I, kSides>((int)(unsigned)u), hi = (unsigned)from_lane<I, kSides>((int)(unsigned)(u >> 32));
    return reinterpret_cast<const char *>(hi << 32 | lo);
}

struct Attend {
    sd_attention a;
    int G, page_shift;             // query heads of a key head; key / page = mulhi(2 key, page_mul) >> page_shift
    unsigned page_mul;
    float scale;                   // scale * log2(e): weights are powers of two
    int splits, min_steps;         // chunks: parts that a tile's keys are split into at most; steps of keys that a part has at least
    int row_tiles;                 // chunks: tiles of rows there may be
    bool grouped;                  // chunks: an eighth of the heads to each die
    int units, once;               // decoding: workgroups of a key head; so many of them find room at once (0: they are not split to fill it)
    bool level;                    // decoding: what is far longer than the others is split
    int pairs;                     // decoding: where all workgroups find room at once, so many come longest first, the others shortest first (0: as they come)
    float *part, *part_ml;         // [.][D], [.][2]: weighted values, (maximum, sum) of a row's part
    int64_t part_rows;             // rows of parts there are
    int4 *info;                    // [tokens * Hq]: how many parts a row has, where its first is, how far apart they are
};

__device__ __forceinline__ int page_of(const Attend &p, int key) { return (int)(__umulhi(2u * (unsigned)key, p.page_mul) >> p.page_shift); }

// 16 bytes a lane from `src` to LDS bytes to .. to + 1023 (lane by lane; lanes that are off leave theirs alone).  In assembly
// because the compiler, which cannot tell the buffers apart, would wait for the loads of the next tile before the reads of this one; it
// has no output registers, and whoever reads the bytes waits for vmcnt first.
__device__ __forceinline__ void load_to_lds(const char *src, unsigned to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(src) : "memory");
}
__device__ __forceinline__ unsigned lds_address(const void *p) { return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }

struct Rows { int first, count, m, kv, before; };   // a request's first token, its tokens, keys, and keys before its first token (may be negative)
__device__ __forceinline__ Rows rows_of(const sd_attention &a, int b)
{
    Rows r;
    const int T = (int)a.tokens;
    r.first = min(max(a.cu[b], 0), T);
    r.m = min(max(a.cu[b + 1] - r.first, 0), T - r.first);
    r.kv = (int)min((int64_t)max(a.kv[b], 0), a.width * a.cache.page);
    r.before = r.kv - r.m;
    r.count = r.m;
    return r;
}
// the keys that a token of a request sees
__device__ __forceinline__ int see_to(const Rows &r, int tok) { return min(max(r.before + tok + 1, 0), r.kv); }
__device__ __forceinline__ int see_from(const sd_attention &a, const Rows &r, int tok)
{
    return a.window > 0 ? (int)min((int64_t)r.kv, max((int64_t)0, (int64_t)r.before + tok + 1 - a.window)) : 0;
}

// sums over the lanes up to this one, as lane moves within the wavefront's registers
template <int CTRL, int ROWS> __device__ __forceinline__ int moved(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false); }
__device__ __forceinline__ int scan(int v)
{
    v += moved<0x111, 0xF>(v);      // row_shr:1
    v += moved<0x112, 0xF>(v);
    v += moved<0x114, 0xF>(v);
    v += moved<0x118, 0xF>(v);
    v += moved<0x142, 0xA>(v);      // row_bcast:15: rows 1, 3 += the end of the row before
    v += moved<0x143, 0xC>(v);      // row_bcast:31: rows 2, 3 += the end of row 1
    return v;
}
__device__ __forceinline__ int total(int v) { return __builtin_amdgcn_readlane(scan(v), 63); }
__device__ __forceinline__ int largest(int v)       // of numbers that are not negative
{
    v = max(v, moved<0x111, 0xF>(v));
    v = max(v, moved<0x112, 0xF>(v));
    v = max(v, moved<0x114, 0xF>(v));
    v = max(v, moved<0x118, 0xF>(v));
    v = max(v, moved<0x142, 0xA>(v));
    v = max(v, moved<0x143, 0xC>(v));
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ float total(float v)
{
    auto from = [](float x, auto step) { return __int_as_float(step(__float_as_int(x))); };
    v += from(v, [](int x) { return moved<0x111, 0xF>(x); });
    v += from(v, [](int x) { return moved<0x112, 0xF>(x); });
    v += from(v, [](int x) { return moved<0x114, 0xF>(x); });
    v += from(v, [](int x) { return moved<0x118, 0xF>(x); });
    v += from(v, [](int x) { return moved<0x142, 0xA>(x); });
    v += from(v, [](int x) { return moved<0x143, 0xC>(x); });
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Up to 64 requests, one to a lane, each with `count` workgroups of `length`: the counts of those with any, the longest first, and which request each is.
// (A request without workgroups may stand anywhere: the others close up before it.)
struct Order { int count, who; };
__device__ __forceinline__ Order longest_first(int B, int length, int count, int lane)
{
    const int key = count ? min(length, 1 << 24) * 64 + 63 - lane : 0;
    int rank = 0;
    for (int j = 0; j < B; ++j) rank += __builtin_amdgcn_readlane(key, j) > key;
    const unsigned long long there = __ballot(count > 0);
    if (!count) rank = __builtin_popcountll(there) + __builtin_popcountll(~there & ((1ull << lane) - 1));
    return Order{__builtin_amdgcn_ds_permute(4 * rank, count), __builtin_amdgcn_ds_permute(4 * rank, lane)};
}

// Tile x of all requests' tiles of rows: its request, and which of that request's it is; false past the last.  By the
// lanes of a wavefront: sums over a 64th of the requests each, then over those one by one.  Exact, so that the workgroups without a tile are the
// last ones: workgroups go to the parts of a die in turn, and were every other one without work, half of the chip would be.
struct Tile { int b, at; };
__device__ __forceinline__ bool tile_of(const sd_attention &a, int G, int tile, int x, int lane, Tile &out)
{
    const int B = (int)a.B;
    auto tiles = [&](int b) { return (int)(((unsigned)(rows_of(a, b).m * G) + tile - 1) / (unsigned)tile); };
    if (B <= 64) {
        // longest requests first, so that the last workgroups to start are short ones (24 x 1 to 301 tokens behind 0 to 3000, 20 heads of 80: 97 us, in order 125)
        const Rows r = lane < B ? rows_of(a, lane) : Rows{0, 0, 0, 0, 0};
        const int m = r.m, keys = m ? see_to(r, m - 1) - see_from(a, r, max(m - tile / G, 0)) : 0;
        const Order o = longest_first(B, max(keys, 0) >> 6, lane < B ? tiles(lane) : 0, lane);
        const int sum = scan(o.count);
        const unsigned long long past = __ballot(sum > x);
        if (past == 0) return false;
        const int at = __builtin_ctzll(past);
        out.b = __builtin_amdgcn_readlane(o.who, at);
        out.at = x - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(o.count, at));
        return true;
    }
    int lo = 0, n = B;
    for (;;) {
        const int chunk = (n + 63) / 64;
        int count = 0;
        for (int e = 0; e < chunk; ++e)
            if (lane * chunk + e < n) count += tiles(lo + lane * chunk + e);
        const int sum = scan(count);
        const unsigned long long past = __ballot(sum > x);
        if (past == 0) return false;
        const int at = __builtin_ctzll(past);
        x -= __builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(count, at);
        lo += at * chunk;
        if (chunk == 1) break;
        n = min(chunk, n - at * chunk);
    }
    out.b = lo;
    out.at = x;
    return true;
}

// The steps (of `keys` keys) of a tile of rows, and those of one of its splits.
struct Span { int first, count, per, used; };
__device__ __forceinline__ Span span_of(const sd_attention &a, const Rows &r, int tok0, int tok1, int keys, int splits, int min_steps)
{
    Span s;
    const int lo = see_from(a, r, tok0), hi = see_to(r, tok1);
    s.first = lo / keys;
    s.count = hi > lo ? (hi + keys - 1) / keys - s.first : 0;
    s.per = max((s.count + splits - 1) / splits, min_steps);
    s.used = (s.count + s.per - 1) / s.per;
    return s;
}

constexpr int kMaxParts = 256;     // of a row

// ---- decoding: what a workgroup does ----
// A request's tiles of rows, and the steps of keys that they see
struct Work { int tiles, first, steps; };
__device__ __forceinline__ Work work_of(const Attend &p, int b, int rows, int keys)
{
    const Rows r = rows_of(p.a, b);
    Work w;
    w.tiles = (int)((unsigned)(r.m * p.G) + rows - 1) / rows;
    w.first = see_from(p.a, r, 0) / keys;
    w.steps = r.m ? max((see_to(r, r.m - 1) + keys - 1) / keys - w.first, 0) : 0;
    return w;
}

// Workgroups of a key head: every tile of a request, times the parts of at most `per` steps that its keys are split into.  Workgroup x
// works part `split` of tile `tile` of request b; its parts of a tile are `tiles` places apart.
struct Unit { int b, tile, split, tiles, splits, per, place; Work w; };
__device__ __forceinline__ bool unit_of(const Attend &p, int x, int rows, int keys, int lane, Unit &u)
{
    const int B = (int)p.a.B;
    // A lane holds a request, or of more than 64 the sums over a 64th of them
    const int chunk = (B + 63) / 64, b0 = lane * chunk;
    Work w{0, 0, 0};
    int tiles = 0, longest = 0;
    float all = 0.f;                                         // steps of all workgroups (tiles' parts), for means
    for (int e = 0; e < chunk; ++e)
        if (b0 + e < B) {
            w = work_of(p, b0 + e, rows, keys);
            tiles += w.tiles;
            all += (float)w.tiles * (float)w.steps;
            if (w.tiles) longest = max(longest, w.steps);
        }
    longest = max(largest(longest), 1);
    int per = longest;                                       // nothing is split
    if (p.once || p.level) {
        const int n = total(tiles);
        if (n == 0) return false;                            // no request has a row
        all = total(all);
        const int least = min(max(p.min_steps, (longest + kMaxParts - 1) / kMaxParts), longest);   // (a row is joined from at most kMaxParts)
        if (n < p.once) {
            // Parts of one length, as many as find room at once: sum tiles ceil(steps / per) <= once holds for per >= all / (once - n), fails below all / once.
            int hi = __builtin_amdgcn_readfirstlane(min((int)(all / (float)(p.once - n)) + 1, longest));
            int lo = __builtin_amdgcn_readfirstlane(min((int)(all / (float)p.once), hi));
            if (B == 1) hi = (longest + p.once / n - 1) / (p.once / n);
            else if (chunk == 1)
                for (int i = 0; i < 5 && lo + 1 < hi; ++i) {
                    const int mid = (lo + hi) >> 1;
                    if (total(w.tiles * max((w.steps + mid - 1) / mid, 1)) <= p.once) hi = mid; else lo = mid;
                }
            per = max(hi, least);
        }
        // What is more than twice as long as the mean is split in any case.
        if (p.level && p.units > n)
            per = min(per, max(max((int)(all / (float)(p.units - n)) + 1, (int)(2.f * all / (float)n)), least));
        per = __builtin_amdgcn_readfirstlane(per);
    }
    auto splits_of = [&](const Work &v) { return max((v.steps + per - 1) / per, 1); };
    if (chunk == 1) {
        int mine = lane < B ? w.tiles * splits_of(w) : 0;
        if (total(mine) > p.units) {                         // (row offsets that overlap: there may be more tiles than workgroups, but no part without a place)
            per = longest;
            mine = w.tiles;
        }
        int count = mine, who = lane;
        if (p.pairs && B > 1) {                              // in the order of their lengths, longest first
            const Order o = longest_first(B, w.steps, mine, lane);
            count = o.count;
            who = o.who;
        }
        const int sum = scan(count), n = __builtin_amdgcn_readlane(sum, 63);
        if (x >= n) return false;
        if (n <= 2 * p.pairs && x >= p.pairs) x = n - 1 - (x - p.pairs);
        const int at = __builtin_ctzll(__ballot(sum > x));
        u.b = __builtin_amdgcn_readlane(who, at);
        u.place = x;
        x -= __builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(count, at);
        u.w = Work{__builtin_amdgcn_readlane(w.tiles, u.b), __builtin_amdgcn_readlane(w.first, u.b), __builtin_amdgcn_readlane(w.steps, u.b)};
    } else {
        u.place = x;
        int count = 0;
        for (int e = 0; e < chunk; ++e)
            if (b0 + e < B) { const Work v = work_of(p, b0 + e, rows, keys); count += v.tiles * splits_of(v); }
        if (total(count) > p.units) {
            per = longest;
            count = tiles;
        }
        int sum = scan(count);
        unsigned long long past = __ballot(sum > x);
        if (past == 0) return false;
        int at = __builtin_ctzll(past);
        x -= __builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(count, at);
        const int first = at * chunk;                        // (chunk <= 64: its requests one by one)
        w = lane < chunk && first + lane < B ? work_of(p, first + lane, rows, keys) : Work{0, 0, 0};
        count = w.tiles * splits_of(w);
        sum = scan(count);
        past = __ballot(sum > x);
        if (past == 0) return false;
        at = __builtin_ctzll(past);
        x -= __builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(count, at);
        u.b = first + at;
        u.w = Work{__builtin_amdgcn_readlane(w.tiles, at), __builtin_amdgcn_readlane(w.first, at), __builtin_amdgcn_readlane(w.steps, at)};
    }
    u.per = per;
    u.tiles = u.w.tiles;
    u.splits = splits_of(u.w);
    u.tile = x % u.tiles;
    u.split = x / u.tiles;
    return true;
}

constexpr int kIds = 256;          // page ids that a wavefront keeps

template <int DK> struct Shape {
    static constexpr int kPitch = DK <= 64 ? 128 : DK <= 128 ? 256 : 512;   // bytes of a row in LDS
    static constexpr int kPieces = kPitch / 16;
    static constexpr int kPerLoad = 64 / kPieces;                            // rows that one load of a wavefront brings
    // where piece c of a row lies: a bijection of the row's pieces.  K is read 16 bytes a lane, eight lanes (rows) in a row
    // of banks; V eight bytes a lane, four rows of 64 bytes together.
    static __device__ __forceinline__ int k_at(int row, int c) { return c ^ (row & 7); }
    static __device__ __forceinline__ int v_at(int row, int c) { return kPieces >= 16 ? c ^ (4 * (row & 3)) : c ^ (4 * ((row >> 1) & 1)); }
};

template <typename T, int DK, bool kFull, int kRows, int kKeys, int KT, bool kUnits>
__global__ void __launch_bounds__(64 * kRows * kKeys, DK > 192 || (kRows == 1 && DK > 128) ? 1 : 2) sd_attend_kernel(const Attend p)
{
    static_assert(kRows == 1 || kKeys == 1, "wavefronts differ in rows or in keys");
    static_assert(!kFull || 2 * DK == Shape<DK>::kPitch, "loads without a test take every piece of a row of LDS, so each has to be one of the head's");
    constexpr bool kOwn = kRows == 1;                        // a wavefront has keys of its own
    typedef Shape<DK> S;
    constexpr int kTile = KT * S::kPitch;                    // bytes of a tile of keys or values
    constexpr int kLoads = KT / S::kPerLoad / kRows;         // of a wavefront, per tile and side
    constexpr int kBlocks = KT / 32, kD = DK / 32, kQ = DK / 16;
    constexpr int kBM = 32 * kRows;
    constexpr int kSides = S::kPieces >= 16 ? 1 : 2;         // rows of a load within 16 lanes
    static_assert(kLoads * kSides <= 16, "16 lanes hold the keys of their loads");
    extern __shared__ char lds[];
    const sd_attention &a = p.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = kRows > 1 ? wave : 0, wk = kRows > 1 ? 0 : wave;
    const int half = lane >> 5, col = lane & 31;
    // The chip deals workgroups to its eight dies in turn, and so go the heads of a tile, but where neighbouring heads share lines of memory or a
    // request's tiles its keys (plan_of).  Chunks, grouped: an eighth of the key heads, neighbours, to each die; where the heads are no multiple of
    // eight, the borders move from tile to tile.  Decoding, grouped: all heads of a range of keys one after the other on one die.
    const unsigned heads = (unsigned)a.cache.heads, die = blockIdx.x % 8, turn = blockIdx.x / 8;
    unsigned item;
    int kh;
    if (!p.grouped) {
        item = blockIdx.x / heads;
        kh = blockIdx.x % heads;
    } else if (kUnits) {
        item = turn / heads * 8 + die;
        kh = turn % heads;
    } else {
        const unsigned each = (heads + 7) / 8, shift = 7 - (item = turn / each) % 8;     // (head h is on die (8 h + 7 - shift) / heads)
        kh = (die * heads + shift) / 8 + turn % each;
        if (kh >= (int)(((die + 1) * heads + shift) / 8)) return;
    }
    const int D = kFull ? DK : (int)a.cache.D, G = p.G, page = (int)a.cache.page;

    int b, row0, t0, t1, parts, part_row = 0, part_step = 0, split;      // tiles of keys t0, t0 + kKeys, .. < t1; where the parts of row 0 lie, by rows
    Rows rq;
    if (kUnits) {
        Unit u;
        if ((int)item >= p.units || !unit_of(p, item, kBM, KT * kKeys, lane, u)) return;
        b = u.b;
        rq = rows_of(a, b);
        row0 = kBM * u.tile;
        split = u.split;
        parts = u.splits;
        t0 = u.w.first + split * u.per;
        t1 = u.w.first + min((split + 1) * u.per, u.w.steps);
        part_step = u.tiles * (int)heads * kBM;
        part_row = (u.place * (int)heads + kh) * kBM - split * part_step;
    } else {
        split = item / (unsigned)p.row_tiles;
        Tile tile;
        if (split >= p.splits || !tile_of(a, G, kBM, item % (unsigned)p.row_tiles, lane, tile)) return;
        b = tile.b;
        rq = rows_of(a, b);
        row0 = kBM * ((rq.m * G - 1) / kBM - tile.at);       // (of a request's tiles the last, which sees most keys, first)
        t0 = t1 = parts = 0;
    }
    const int rows = rq.m * G, tok0 = row0 / G, tok1 = (min(row0 + kBM, rows) - 1) / G;
    const Span sp = span_of(a, rq, tok0, tok1, KT * kKeys, kUnits ? 1 : p.splits, p.min_steps);
    if (kUnits) {                                              // (a request's tiles see a little less than all of its keys)
        t0 = max(t0, sp.first) * kKeys + wk;
        t1 = min(t1, sp.first + sp.count) * kKeys;
    } else {
        if (split >= max(sp.used, 1)) return;
        parts = sp.used;
        t0 = (sp.first + split * sp.per) * kKeys;
        t1 = (sp.first + min((split + 1) * sp.per, sp.count)) * kKeys;
    }
    const int first_key = see_from(a, rq, tok0), last_key = max(see_to(rq, tok1) - 1, 0);

    // this lane's row
    const int R = row0 + wm * 32 + col;
    const bool there = R < rows;
    const int tok = min(R, rows - 1) / G, head = kh * G + min(R, rows - 1) % G;
    const int from = see_from(a, rq, tok), to = see_to(rq, tok);
    // the wavefront's: keys in [whole_from, whole_to) are seen by all of its rows, those outside [any_from, any_to) by none
    const int w0 = min(row0 + wm * 32, rows - 1) / G, w1 = min(row0 + wm * 32 + 31, rows - 1) / G;
    const int any_from = see_from(a, rq, w0), whole_to = see_to(rq, w0), whole_from = see_from(a, rq, w1);
    const int any_to = row0 + wm * 32 < rows ? see_to(rq, w1) : 0;

    char *const kbuf = lds + wk * 4 * kTile, *const vbuf = kbuf + 2 * kTile;
    if (!kFull) {                                            // pieces past D are never loaded
        for (int i = tid; i < kKeys * 4 * kTile / 16; i += 64 * kRows * kKeys) reinterpret_cast<u4 *>(lds)[i] = u4{0, 0, 0, 0};
        __syncthreads();
    }

    u4 q[kQ];
    {
        const T *src = static_cast<const T *>(a.q) + (int64_t)(rq.first + tok) * a.q_tok_stride + (int64_t)head * a.q_head_stride;
#pragma unroll
        for (int c = 0; c < kQ; ++c) {
            const int d = 16 * c + 8 * half;
            q[c] = d < D ? *reinterpret_cast<const u4 *>(src + d) : u4{0, 0, 0, 0};
        }
    }

    // ---- from the pages to LDS: load i of a tile brings rows (i * kRows + wm) * kPerLoad + lane / kPieces ----
    // Where a key lies is worked out once a tile by one of the 16 lanes that load from it (lane i of 16 for load i; for rows of eight pieces,
    // lanes 2 i and 2 i + 1), and handed to the others as the load is issued.
    const int lrow = wm * S::kPerLoad + lane / S::kPieces, lpiece = lane % S::kPieces;
    const int own_row = min((lane & 15) / kSides, kLoads - 1) * kRows * S::kPerLoad + wm * S::kPerLoad +
                        (kSides == 1 ? lane / S::kPieces : 2 * (lane >> 4) + (lane & 1));
    const char *const kbase = static_cast<const char *>(a.cache.k) + 2 * (int64_t)kh * a.cache.k_head_stride;
    const char *const vbase = static_cast<const char *>(a.cache.v) + 2 * (int64_t)kh * a.cache.v_head_stride;
    const int32_t *const table = a.table + (int64_t)b * a.table_stride;
    // (places that none of the tile's rows sees get a key that one does see, so that a zero weight never meets what a page happens to hold)
    auto key_in = [&](int key) { return min(max(key, first_key), last_key); };
    auto own_key = [&](int t) { return key_in(t * KT + own_row); };
    unsigned kto = __builtin_amdgcn_readfirstlane(lds_address(kbuf));
    asm("" : "+s"(kto));                                     // (not worked out again for each load)
    const unsigned vto = kto + 2 * kTile;
    auto issue = [&](int t, int buf, auto page_id) {
        const int key = own_key(t), place = page_of(p, key), at = key - place * page;
        const int64_t id = min(max(page_id(place), 0), (int)a.cache.pages - 1);
        const char *const ks = kbase + 2 * (id * a.cache.k_page_stride + at * a.cache.k_tok_stride);
        const char *const vs = vbase + 2 * (id * a.cache.v_page_stride + at * a.cache.v_tok_stride);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // what was read from the buffer is there
        unroll<kLoads>([&](auto n) {
            constexpr int i = decltype(n)::value;
            const int row = i * kRows * S::kPerLoad + lrow;
            const unsigned to = buf * kTile + (i * kRows + wm) * 1024;
            const int kp = S::k_at(row, lpiece), vp = S::v_at(row, lpiece);
            const char *const kx = from_lane<i, kSides>(ks) + 16 * kp, *const vx = from_lane<i, kSides>(vs) + 16 * vp;   // (with all lanes on)
            if (kFull || 8 * kp < D) load_to_lds(kx, kto + to);     // (every row has a piece below D, so every load is issued)
            if (kFull || 8 * vp < D) load_to_lds(vx, vto + to);
        });
    };

    f16v o[kD];
#pragma unroll
    for (int d = 0; d < kD; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
    float top = -INFINITY, sum = 0.f;                        // of the row: what weights are relative to (powers of two); sum: of this half's keys

    auto work = [&](int t, int buf) {
        const int key0 = t * KT;
        if (key0 >= any_to || key0 + KT <= any_from) return;
        const char *kt = kbuf + buf * kTile, *vt = vbuf + buf * kTile;
        // Scores.  Fragments of the keys are read kAhead before they are used: read as they are needed, each product would wait out LDS's latency.
        constexpr int kFrags = kQ * kBlocks, kAhead = kFrags < 8 ? kFrags : 8;
        auto k_frag = [&](int f) {
            const int row = 32 * (f % kBlocks) + col;
            return *reinterpret_cast<const u4 *>(kt + row * S::kPitch + 16 * S::k_at(row, 2 * (f / kBlocks) + half));
        };
        f16v s[kBlocks];
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[n][r] = 0.f;
        u4 kf[kAhead];
#pragma unroll
        for (int f = 0; f < kAhead; ++f) kf[f] = k_frag(f);
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
            s[f % kBlocks] = mfma<T>(kf[f % kAhead], q[f / kBlocks], s[f % kBlocks]);
            if (f + kAhead < kFrags) kf[f % kAhead] = k_frag(f + kAhead);
        }
        // Values, 16 keys (a part) at a time: this lane's are 16 part + 4 half + (0..3) and those + 8, at d = 32 dblock + col; a part ahead
        const int vrow = 4 * half + ((lane & 15) >> 2), vpiece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), voff = 8 * (lane & 1);
        auto v_frag = [&](int part, int d) {
            const int r0 = 16 * part + vrow, r1 = r0 + 8;
            const char *x0 = vt + r0 * S::kPitch + 16 * S::v_at(r0, 4 * d + vpiece) + voff;
            const char *x1 = vt + r1 * S::kPitch + 16 * S::v_at(r1, 4 * d + vpiece) + voff;
            const u2 v0 = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)x0));
            const u2 v1 = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)x1));
            return u4{v0[0], v0[1], v1[0], v1[1]};
        };
        u4 vf[2][kD];
#pragma unroll
        for (int d = 0; d < kD; ++d) vf[0][d] = v_frag(0, d);
        order<0x100>(kAhead);
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
            order<0x8>(1);
            order<0x100>(f + kAhead < kFrags ? 1 : f - (kFrags - kAhead) < 2 * kD ? 1 : 0);
        }
        if (key0 < whole_from || key0 + KT > whole_to) {
            const int base = key0 + 4 * half - from;
            const unsigned seen = (unsigned)(to - from);
#pragma unroll
            for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[n][r] = (unsigned)(base + 32 * n + 8 * (r >> 2) + (r & 3)) < seen ? s[n][r] : -INFINITY;
        }
        float most = s[0][0];
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, s[n][r]);
        const f2 both = halves(most);
        most = fmaxf(both[0], both[1]) * p.scale;
        // the weights are taken relative to a maximum that lags behind by at most a factor of 2^8 (row by row: what a row gets does not depend on its neighbours),
        // less the lift: `top` is that, so that all that is rescaled or joined has one exact reference
        const bool behind = most > top + (8.f + kLift<T>);
        if (__any(behind)) {
            const float now = behind ? most - kLift<T> : top, back = behind ? __builtin_amdgcn_exp2f(top - now) : 1.f;
            top = now;
            sum *= back;
#pragma unroll
            for (int d = 0; d < kD; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[d][r] *= back;
        }
        const float ref = top == -INFINITY ? 0.f : top;
        // weights of part i: registers 8 (i % 2) .. + 7 of block i / 2; those of the next part are made while the products of this one run
        auto weigh = [&](int part) {
            u4 w;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[part / 2][8 * (part % 2) + 2 * r], p.scale, -ref));
                const float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[part / 2][8 * (part % 2) + 2 * r + 1], p.scale, -ref));
                sum += w0 + w1;
                w[r] = pack<T>(w0, w1);
            }
            return w;
        };
        u4 w = weigh(0);
#pragma unroll
        for (int part = 0; part < 2 * kBlocks; ++part) {
            u4 next = w;
            if (part + 1 < 2 * kBlocks) {
#pragma unroll
                for (int d = 0; d < kD; ++d) vf[(part + 1) % 2][d] = v_frag(part + 1, d);
                next = weigh(part + 1);
            }
#pragma unroll
            for (int d = 0; d < kD; ++d) o[d] = mfma<T>(vf[part % 2][d], w, o[d]);
            w = next;
        }
    };

    if (kOwn) {
        // Two tiles on the way: a buffer is filled again as soon as it has been read.  The wavefront's page ids lie in LDS, kIds of them at a time: a
        // load to registers would be waited for together with the tiles behind it.
        int *const ids = reinterpret_cast<int *>(lds + kKeys * 4 * kTile) + wk * kIds;
        const int last_place = page_of(p, last_key);
        int ids_from = -kIds;
        auto fetch = [&](int t, int buf) {
            const int p0 = page_of(p, key_in(t * KT)), p1 = page_of(p, key_in(t * KT + KT - 1));
            if (p0 < ids_from || p1 >= ids_from + kIds) {
                ids_from = p0;
#pragma unroll
                for (int i = 0; i < kIds; i += 64) ids[i + lane] = table[min(p0 + i + lane, last_place)];
            }
            issue(t, buf, [&](int place) { return ids[place - ids_from]; });
        };
        if (t0 < t1) fetch(t0, 0);
        if (t0 + kKeys < t1) fetch(t0 + kKeys, 1);
        int buf = 0;
        for (int t = t0; t < t1; t += kKeys, buf ^= 1) {
            if (t + kKeys < t1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kLoads) : "memory");   // all but the loads of the next tile
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            work(t, buf);
            if (t + 2 * kKeys < t1) fetch(t + 2 * kKeys, buf);
        }
    } else {
        // One tile on the way, and the page ids of the one behind it
        int id = 0;
        auto fetch_id = [&](int t) { id = table[page_of(p, own_key(t))]; };
        auto id_of = [&](int) { return id; };
        if (t0 < t1) {
            fetch_id(t0);
            issue(t0, 0, id_of);
            if (t0 + 1 < t1) fetch_id(t0 + 1);
        }
        int buf = 0;
        for (int t = t0; t < t1; ++t, buf ^= 1) {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // tile t, and the pages of the next
            asm volatile("" : "+v"(id));                     // (it is not waited for again behind the loads below)
            __builtin_amdgcn_s_barrier();                    // everyone's part of tile t is there, and tile t - 1 has been read
            asm volatile("" ::: "memory");
            if (t + 1 < t1) {
                issue(t + 1, buf ^ 1, id_of);
                if (t + 2 < t1) fetch_id(t + 2);
            }
            work(t, buf);
        }
    }
    {
        const f2 both = halves(sum);
        sum = both[0] + both[1];
        if (sum != sum) top = INFINITY;                      // (the maximum left it out: no part without it may pass for the whole row)
    }

    const bool whole = parts <= 1;
    const int64_t orow = (int64_t)(rq.first + tok) * a.Hq + head;
    const int64_t first_part = kUnits ? part_row + wm * 32 + col : orow, part_stride = kUnits ? part_step : a.tokens * a.Hq, prow = first_part + split * part_stride;
    if (kKeys > 1) {
        // join the wavefronts: maximum, sum and values of each to LDS, then a share of D to each
        constexpr int kP = DK + 4;                           // floats of a row
        __syncthreads();
        float *ml = reinterpret_cast<float *>(lds), *os = ml + kKeys * 64;
        if (half == 0) { ml[wk * 64 + col] = top; ml[wk * 64 + 32 + col] = sum; }
#pragma unroll
        for (int d = 0; d < kD; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<float4 *>(os + (wk * 32 + col) * kP + 32 * d + 2 * r + 4 * half) = float4{o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]};
        __syncthreads();
        float now = -INFINITY, all = 0.f, part[kKeys];
#pragma unroll
        for (int k = 0; k < kKeys; ++k) now = fmaxf(now, ml[k * 64 + col]);
#pragma unroll
        for (int k = 0; k < kKeys; ++k) {
            part[k] = ml[k * 64 + col] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[k * 64 + col] - now);
            all += part[k] * ml[k * 64 + 32 + col];
        }
        top = now;
        sum = all;
        constexpr int kShare = DK / kKeys / 2;               // of D, per half of a wavefront
        const int d0 = (wk * 2 + half) * kShare;
        const float inv = whole ? (sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum) : 1.f;
        if (there) {
#pragma unroll
            for (int d = d0; d < d0 + kShare; d += 4) {
                if (d >= D) break;
                float4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < kKeys; ++k) {
                    const float4 e = *reinterpret_cast<const float4 *>(os + (k * 32 + col) * kP + d);
                    if (part[k] != 0.f) { v.x += part[k] * e.x; v.y += part[k] * e.y; v.z += part[k] * e.z; v.w += part[k] * e.w; }
                }
                if (whole)
                    *reinterpret_cast<u2 *>(static_cast<T *>(a.out) + (int64_t)(rq.first + tok) * a.out_tok_stride + (int64_t)head * a.out_head_stride + d) =
                        u2{pack<T>(v.x * inv, v.y * inv), pack<T>(v.z * inv, v.w * inv)};
                else
                    *reinterpret_cast<float4 *>(p.part + prow * D + d) = v;
            }
        }
    } else if (there) {
        const float inv = whole ? (sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum) : 1.f;
#pragma unroll
        for (int d = 0; d < kD; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int at = 32 * d + 2 * r + 4 * half;
                if (at >= D) break;
                if (whole)
                    *reinterpret_cast<u2 *>(static_cast<T *>(a.out) + (int64_t)(rq.first + tok) * a.out_tok_stride + (int64_t)head * a.out_head_stride + at) =
                        u2{pack<T>(o[d][r] * inv, o[d][r + 1] * inv), pack<T>(o[d][r + 2] * inv, o[d][r + 3] * inv)};
                else
                    *reinterpret_cast<float4 *>(p.part + prow * D + at) = float4{o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]};
            }
    }
    if (there && half == 0 && wk == 0) {
        if (p.info && split == 0) p.info[orow] = int4{parts, (int)first_part, (int)part_stride, 0};
        if (whole) {
            if (a.lse) a.lse[orow] = sum != 0.f ? (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f : -INFINITY;
        } else {
            float *ml = p.part_ml + 2 * prow;
            ml[0] = top; ml[1] = sum;
        }
    }
}

// The parts of rows whose keys were split: kLanes lanes a row (a workgroup where rows are few, a wavefront otherwise), D / 4 of them to a
// part.  How many there are and where was left by the workgroups of the first ones, so that nothing of the requests is looked up again; a row is
// two dependent trips to memory.
template <typename T, int kLanes> __global__ void __launch_bounds__(256) sd_join_kernel(const Attend p)
{
    constexpr int kRows = 256 / kLanes, kEach = kMaxParts / 64;
    __shared__ float w_sh[kRows][kMaxParts];
    __shared__ float4 v_sh[kRows][kLanes];
    const sd_attention &a = p.a;
    const int tid = threadIdx.x % kLanes, group = threadIdx.x / kLanes, lane = threadIdx.x & 63;
    const int64_t rows = a.tokens * a.Hq, orow = (int64_t)blockIdx.x * kRows + group;
    const int D = (int)a.cache.D;
    int4 info{0, 0, 0, 0};
    if (orow < rows) info = p.info[orow];
    const int64_t first = info.y, stride = info.z, token = orow / a.Hq;
    // Tokens of no request have no parts, only what the workspace held; row offsets that do not ascend may leave such tokens between requests, too.
    const bool of_one = orow < rows && token >= a.cu[0] && token < a.cu[a.B] && info.x > 1 && info.x <= kMaxParts && first >= 0 && stride >= 0 &&
                        first + (info.x - 1) * stride < p.part_rows;
    const int used = of_one ? info.x : 0;
    if (used <= 1 && kLanes > 64) return;                    // (all of a workgroup; otherwise it has a barrier to reach)
    // maximum and sum (every wavefront of the row by itself), and the parts' weights
    f2 mine[kEach];
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        mine[i] = f2{-INFINITY, 0.f};
        if (lane + 64 * i < used) mine[i] = reinterpret_cast<const f2 *>(p.part_ml)[first + (lane + 64 * i) * stride];
    }
    const int lanes = D / 4, parts = kLanes / lanes, s0 = tid / lanes, d = 4 * (tid % lanes);
    float4 e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (s0 < parts && s0 + i * parts < used) e[i] = *reinterpret_cast<const float4 *>(p.part + (first + (s0 + i * parts) * stride) * D + d);
#pragma unroll
    for (int i = 0; i < kEach; ++i) top = fmaxf(top, mine[i][0]);
#pragma unroll
    for (int sh = 32; sh >= 1; sh >>= 1) top = fmaxf(top, __shfl_xor(top, sh));
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const float w = mine[i][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mine[i][0] - top);
        if (w != 0.f) sum += w * mine[i][1];
        if (lane + 64 * i < used) w_sh[group][lane + 64 * i] = w;       // (the same from every wavefront of the row)
    }
#pragma unroll
    for (int sh = 32; sh >= 1; sh >>= 1) sum += __shfl_xor(sum, sh);
    __syncthreads();
    float4 v{0.f, 0.f, 0.f, 0.f};
    if (s0 < parts) {
        for (int s1 = s0; s1 < used; s1 += 8 * parts) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (s1 > s0 && s1 + i * parts < used) e[i] = *reinterpret_cast<const float4 *>(p.part + (first + (s1 + i * parts) * stride) * D + d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float w = s1 + i * parts < used ? w_sh[group][s1 + i * parts] : 0.f;
                if (w != 0.f) { v.x += w * e[i].x; v.y += w * e[i].y; v.z += w * e[i].z; v.w += w * e[i].w; }
            }
        }
    }
    v_sh[group][tid] = v;
    __syncthreads();
    if (used > 1 && tid < lanes) {
        for (int s = 1; s < parts; ++s) {
            const float4 o = v_sh[group][s * lanes + tid];
            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
        const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
        const int64_t t = orow / a.Hq, head = orow % a.Hq;
        *reinterpret_cast<u2 *>(static_cast<T *>(a.out) + t * a.out_tok_stride + head * a.out_head_stride + d) =
            u2{pack<T>(v.x * inv, v.y * inv), pack<T>(v.z * inv, v.w * inv)};
        if (tid == 0 && a.lse) a.lse[orow] = sum != 0.f ? (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f : -INFINITY;
    }
}

bool misaligned(const void *p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

int check(const sd_attention &a)
{
    const sd_cache &c = a.cache;
    if (a.B <= 0 || a.tokens < 0 || a.Hq <= 0 || a.width <= 0 || a.table_stride < a.width || a.window < 0) return SD_EINVAL;
    if (c.pages <= 0 || c.page <= 0 || c.heads <= 0 || c.D <= 0 || a.Hq % c.heads != 0) return SD_EINVAL;
    if (!(a.scale > 0.0) || !(a.scale <= 1e30)) return SD_EINVAL;
    if (c.dtype != SD_F32 && c.dtype != SD_BF16 && c.dtype != SD_F16) return SD_EINVAL;
    const int64_t strides[] = {c.k_page_stride, c.k_tok_stride, c.k_head_stride, c.v_page_stride, c.v_tok_stride, c.v_head_stride,
                               a.q_tok_stride, a.q_head_stride, a.out_tok_stride, a.out_head_stride};
    for (int64_t s : strides)
        if (s < 0 || s % 8 != 0) return SD_EINVAL;
    const int64_t most = 0x7fffffff;
    if (c.dtype == SD_F32 || c.D % 8 != 0 || c.D > SD_MAX_HEAD_DIM || a.B > SD_MAX_REQUESTS) return SD_EUNSUPPORTED;
    if (c.pages > most || c.page > most || c.pages * c.page > most || a.width > most || a.width * c.page > most - 4096 ||
        c.heads > most || a.tokens > most || a.Hq > most || a.tokens * a.Hq > most || a.Hq * a.B > most)
        return SD_EUNSUPPORTED;
    return SD_OK;
}

// ---- which kernel, and how many workgroups: by the shapes alone ----
struct Plan { int dk, rows, tiles, splits, min_steps, units, once, pairs; bool many, level, join, grouped; };
Plan plan_of(const sd_attention &a)
{
    Plan p;
    const int64_t heads = a.cache.heads, G = a.Hq / heads, D = a.cache.D, rows = a.tokens * G;
    // heads are padded to the next of these (8 x 512 tokens over 2048 keys: D = 80 in 96 119 us, in 128 134; 144 in 192 200, in 256 374)
    p.dk = D <= 64 ? 64 : D <= 96 ? 96 : D <= 128 ? 128 : D <= 192 ? 192 : 256;
    // Chunks: more than 32 rows a request and key head (in the mean), so that its keys would be read more than once by tiles of 32, and are shared
    // by 128 (64 requests of 40 rows over 2000 keys, D = 128: 99 us, in tiles of 32 162; of 32 rows 98 and 106; 8 of 36 over 8000: 53 and 89).
    const bool many = p.many = rows > 32 * a.B;
    const int64_t there = (rows / 128 > a.B ? rows / 128 : a.B) * heads;          // workgroups, nothing split
    // Keys are split where the requests' tiles do not fill the chip, which has room for 512 workgroups.  Chunks: below 256 (8192 keys: 1 x 128 tokens
    // 38 us, unsplit 152; 1 x 512 90 and 153; but 24 chunks of 40 tokens, 20 heads, 480 workgroups: 67 and 50).  Decoding: below 512, though equal lengths lose
    // by it (32 requests, 8 heads, 2000 keys each: 50 and 43 us; 200 to 4096: 49 and 76; with 5 tokens 66 and 89; 40 of these 94 and 104).
    // Decoding of whole requests takes wavefronts with keys of their own where the head fills its row in LDS (64 x 5 tokens, D = 128, 200 to
    // 4096 keys: 115 us, shared tiles 119; 2000 each: 100 and 98); else (2048 each; D = 80, 96, 144, 192) shared tiles: 64, 75, 110, 143 us to 71, 79, 157, 171.
    const bool fill = there < (many ? 256 : 512), own = !many && !fill && (D == 64 || D == 128);
    p.rows = own ? 32 : 128;
    const int64_t step = p.dk != 192 ? 64 : 32;                                         // keys
    int64_t longest = a.width * a.cache.page;
    if (a.window > 0 && a.window < longest && a.window + p.rows / G + 1 < longest) longest = a.window + p.rows / G + 1;
    // Short parts where workgroups are few and wait for nothing but their own keys (1 request, 1500 keys, parts of 64, 128, 256, 1024 keys at least: 11.4, 12.3,
    // 14.3, 26 us); where there are more, the room for workgroups ends the splitting first.
    p.min_steps = there >= 64 ? 4 : 1;
    const int64_t most = (longest + p.min_steps * step - 1) / (p.min_steps * step);     // parts of the longest context
    p.tiles = (int)(rows / p.rows + a.B);
    p.splits = 1;
    p.units = p.once = p.pairs = 0;
    p.level = p.grouped = false;
    if (many) {
        // a compute unit has room for two workgroups: where they do not fill the chip once, the keys are split
        int64_t splits = fill ? (512 + there - 1) / there : 1;
        splits = splits > most ? most : splits;
        p.splits = (int)(splits > 256 ? 256 : splits < 1 ? 1 : splits);
        p.join = p.splits > 1;
        // Neighbouring heads share lines of memory where a head's piece is no multiple of 128 bytes (20 heads, 24 chunks of 150 tokens over 1500 keys, D = 96:
        // 144 us in turn, 99 grouped); where it is, the places that 20 heads leave empty cost more than the keys shared by a request's tiles bring (25
        // chunks of 128, D = 64: 35 and 44).
        p.grouped = heads > 8 && (heads % 8 == 0 || (D % 64 != 0 && a.cache.k_head_stride < a.cache.k_tok_stride));
        return p;
    }
    // Decoding: parts of one length, as many as find room at once (1024 of them: 2 x 5 tokens over 100000 keys 160 us instead of 151); a context of 512 keys is as
    // fast whole as split and joined (300 keys: 10.0 and 12.6 us, 400 12.1 and 11.5, 1500 29 and 11.4).  Contexts far beyond the mean are split in
    // any case, if the tables are wide enough for such that a workgroup would be long at it: 8192 keys of D = 128 take about 170 us, and joining
    // costs 8 (64 x 5 tokens over 2000 keys 106 and 114 us; 63 requests of 500 keys and one of 60000: 96 us, 1120 unsplit).
    const int64_t room1 = (512 + heads - 1) / heads, once = room1 < (int64_t)p.tiles * most ? room1 : (int64_t)p.tiles * most;
    p.once = fill && longest > 512 ? (int)once : 0;
    // (heads whose pieces share lines of 128 bytes on one die: 64 x 5 tokens over 2048 keys, D = 80 and 96: 64 and 75 us, in turn 81 and 83; D = 128 and 192 103
    // and 147, in turn 99 and 144)
    p.grouped = D % 64 != 0 && a.cache.k_head_stride < a.cache.k_tok_stride;
    p.level = longest * D > 8192 * 128;
    const int64_t room = p.tiles + (a.B / 2 > 8 ? a.B / 2 : 8), units = p.level && room > p.once ? room : p.once > p.tiles ? p.once : p.tiles;
    if (units * heads * p.rows > 0x7fffffff) { p.once = 0; p.level = false; }            // (rows of parts are numbered in 32 bits)
    p.units = p.once || p.level ? (int)units : p.tiles;
    // A compute unit gets the i-th and the i + 256-th workgroup: a long request next to a short one (64 x 5 tokens over 200 to 4096 keys: 122 us; as they
    // come 135, longest first 136).
    p.pairs = there >= 256 ? (int)((256 + heads - 1) / heads) : 0;
    p.join = p.once || p.level;
    return p;
}
// workgroups of the first launch
int64_t groups(const sd_attention &a, const Plan &p)
{
    const int64_t heads = a.cache.heads, items = (int64_t)p.tiles * p.splits;
    return !p.many ? ((int64_t)p.units + 7) / 8 * 8 * heads : p.grouped ? items * ((heads + 7) / 8 * 8) : items * heads;
}
// lanes of a row of the second: few rows are as long as one's chain of parts (1 token over 8000 keys 16.8 us by workgroups, 23.5 by wavefronts; 2560 rows over 2000 keys 38 and 35)
int64_t join_lanes(const sd_attention &a) { return a.tokens * a.Hq <= 1024 ? 256 : 64; }
// whether a launch can have so many threads
bool fits(const sd_attention &a, const Plan &p)
{
    const int64_t most = 0xffffffffll;
    return groups(a, p) * (p.rows == 128 ? 256 : 128) <= most && (!p.join || (a.tokens * a.Hq + 3) * join_lanes(a) <= most);
}
int64_t part_rows(const sd_attention &a, const Plan &p) { return p.many ? (int64_t)p.splits * a.tokens * a.Hq : (int64_t)p.units * a.cache.heads * p.rows; }
// parts, (maximum, sum) of each, and where a row's parts are
size_t part_bytes(const sd_attention &a, const Plan &p) { return p.join ? (size_t)part_rows(a, p) * (a.cache.D + 2) * 4 + (size_t)a.tokens * a.Hq * sizeof(int4) : 0; }

template <typename T, int DK, bool kFull, int kRows, int kKeys, int KT, bool kUnits> hipError_t launch_shape(const Attend &p, dim3 grid, hipStream_t st)
{
    constexpr int tiles = kKeys * 4 * KT * Shape<DK>::kPitch, bytes = tiles + (kRows == 1 ? 4 * kIds * kKeys : 0);
    static_assert(kKeys == 1 || kKeys * (64 + 32 * (DK + 4)) * 4 <= tiles, "the join has room");
    const auto kernel = sd_attend_kernel<T, DK, kFull, kRows, kKeys, KT, kUnits>;
    if (bytes > 64 * 1024) {                                 // (each call: it is the current device's)
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, grid, dim3(64 * kRows * kKeys), bytes, st, p);
    return hipGetLastError();
}
template <typename T, int DK, bool kFull> hipError_t launch(const Attend &p, const Plan &plan, hipStream_t st)
{
    const dim3 grid((unsigned)groups(p.a, plan));
    // (shared tiles of 64 and 32 keys, 8 x 512 tokens over 2048 keys, D = 64: 88 and 98 us, 128: 140 and 150, 192, where 64 leave no room for a second workgroup: 236 and
    // 213, 256, where 32 do not either, the accumulators being so many: 306 and 370)
    constexpr int KT = DK != 192 ? 64 : 32;
    hipError_t e = hipErrorInvalidValue;
    if (plan.many) e = launch_shape<T, DK, kFull, 4, 1, KT, false>(p, grid, st);
    else if (plan.rows == 128) e = launch_shape<T, DK, kFull, 4, 1, KT, true>(p, grid, st);
    else if constexpr (kFull && DK <= 128) e = launch_shape<T, DK, kFull, 1, 2, 32, true>(p, grid, st);
    if (e == hipSuccess && plan.join) {
        const int64_t rows = p.a.tokens * p.a.Hq;
        if (join_lanes(p.a) == 256) hipLaunchKernelGGL((sd_join_kernel<T, 256>), dim3((unsigned)rows), dim3(256), 0, st, p);
        else hipLaunchKernelGGL((sd_join_kernel<T, 64>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, p);
        e = hipGetLastError();
    }
    return e;
}
template <typename T, int DK> hipError_t launch(const Attend &p, const Plan &plan, hipStream_t st)
{
    // (a head of 96 or 192 fills its row of products, but not the 128 or 256 elements from row to row in LDS)
    if constexpr (2 * DK == Shape<DK>::kPitch) {
        if (p.a.cache.D == DK) return launch<T, DK, true>(p, plan, st);
    }
    return launch<T, DK, false>(p, plan, st);
}
template <typename T> hipError_t launch(const Attend &p, const Plan &plan, hipStream_t st)
{
    switch (plan.dk) {
        case 64: return launch<T, 64>(p, plan, st);
        case 96: return launch<T, 96>(p, plan, st);
        case 128: return launch<T, 128>(p, plan, st);
        case 192: return launch<T, 192>(p, plan, st);
        default: return launch<T, 256>(p, plan, st);
    }
}

}  // namespace

extern "C" {

size_t sd_attend_workspace_bytes(const sd_attention *a)
{
    if (!a || check(*a) != SD_OK) return 0;
    const Plan plan = plan_of(*a);
    return fits(*a, plan) ? 16 + part_bytes(*a, plan) : 0;
}

int sd_attend(const sd_attention *args, void *ws, size_t ws_bytes, void *hip_stream)
{
    if (!args) return SD_EINVAL;
    const sd_attention &a = *args;
    const int rc = check(a);
    if (rc != SD_OK) return rc;
    const Plan plan = plan_of(a);
    if (!fits(a, plan)) return SD_EUNSUPPORTED;
    if (!a.cache.k || !a.cache.v || !a.cu || !a.kv || !a.table || !ws) return SD_EINVAL;
    if (a.tokens > 0 && (!a.q || !a.out)) return SD_EINVAL;
    if (misaligned(a.cache.k, 16) || misaligned(a.cache.v, 16) || misaligned(a.q, 16) || misaligned(a.out, 16) || misaligned(a.lse, 4) ||
        misaligned(a.cu, 4) || misaligned(a.kv, 4) || misaligned(a.table, 4) || misaligned(ws, 16))
        return SD_EINVAL;
    if (ws_bytes < 16 + part_bytes(a, plan)) return SD_ENOMEM;
    if (a.tokens == 0) return SD_OK;
    Attend p;
    p.a = a;
    p.G = (int)(a.Hq / a.cache.heads);
    p.scale = fmaxf((float)(a.scale * 1.4426950408889634), 1.2e-38f);    // (not 0: a masked score is -inf and has to stay that)
    // key / page for keys below 2^31: with s = ceil(log2(page)), floor(key m / 2^(31 + s)), m = floor(2^(31 + s) / page) + 1 <= 2^32 - 1
    int s = 0;
    while ((1ll << s) < a.cache.page) ++s;
    p.page_mul = (unsigned)((1ull << (31 + s)) / (unsigned long long)a.cache.page + 1);
    p.page_shift = s;
    p.splits = plan.splits;
    p.min_steps = plan.min_steps;
    p.row_tiles = plan.tiles;
    p.grouped = plan.grouped;
    p.units = plan.units;
    p.once = plan.once;
    p.level = plan.level;
    p.pairs = plan.pairs;
    const size_t parts = (size_t)part_rows(a, plan);
    p.part_rows = plan.join ? (int64_t)parts : 0;
    p.info = plan.join ? static_cast<int4 *>(ws) : nullptr;
    p.part = reinterpret_cast<float *>(static_cast<int4 *>(ws) + (size_t)a.tokens * a.Hq);
    p.part_ml = p.part + parts * a.cache.D;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return (a.cache.dtype == SD_BF16 ? launch<__bf16>(p, plan, st) : launch<_Float16>(p, plan, st)) == hipSuccess ? SD_OK : SD_EHIP;
}

}  // extern "C"
