// Attention over the 4-bit sequence cache.
#include <algorithm>
#include <array>
#include <type_traits>

#include "ice_cache.h"

namespace ice {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;      // of a workgroup
constexpr int kStep = 32;      // keys per step of a wave
constexpr int kQuantum = kWaves * kStep;
constexpr int kRows = 16;      // columns of a tile of query rows
constexpr int kRecord = 132;   // floats per row of a partial result: 128 sums, maximum, denominator
constexpr int kEntries = 1024; // requests of one launch at most
constexpr float kNoMax = -3.402823466e38f;  // maximum of a row that has seen no key: below every finite score
constexpr float kSlack = 8.f;  // a row's reference may lie this far (in powers of two) below its maximum before sums are rescaled

__device__ inline f32x4 mfma(const u32x4 &a, const u32x4 &b, const f32x4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <int SEL> __device__ inline uint32_t two(uint32_t codes, float scale) {  // values 2 SEL and 2 SEL + 1 of a dword of codes
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}
__device__ inline u32x4 eight(uint32_t codes, float scale) {
    return u32x4{two<0>(codes, scale), two<1>(codes, scale), two<2>(codes, scale), two<3>(codes, scale)};
}
__device__ inline uint32_t pack2(float a, float b) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
// Scale i of a dword of scale bytes.  The conversion takes the exponent field of its scale operand and nothing else of it.
__device__ inline float scale_of(uint32_t bytes, int i) { return __uint_as_float(i < 3 ? bytes << (23 - 8 * i) : bytes >> 1); }
__device__ inline float cut(float v, uint32_t mask) { return v - __uint_as_float(__float_as_uint(v) & mask); }

// A request's query rows and the keys they see; for listed tokens, those of one KV head.
template <bool LIST>
struct Unit {
    int row0, n_query, first;  // first query row, queries, the position behind the first one's own (listed: entries of the list)
    int tokens;              // the length, or what the table has room for if that is less: the queries' positions follow the length all the same
    // t: the request's length; x, y: its entry of query_start and the next one, or x the length of its list.
    __host__ __device__ Unit(const CacheAttend &a, int s, int t, int x, int y) { set(a, s, t, x, y); }
    // UNIFORM: the same on all lanes.  A request's words are asked for before one is looked at: left to the compiler, the length was asked for
    // once the request was known to have queries, a trip more (0.1 to 1 us a call).
    template <bool UNIFORM>
    __device__ Unit(const CacheAttend &a, int s, int h, std::integral_constant<bool, UNIFORM>) {
        int t = a.seq_len[s], x = LIST ? a.n_tok[s * a.c.H + h] : a.query_start[s], y = LIST ? 0 : a.query_start[s + 1];
        if constexpr (LIST) {
        } else if constexpr (UNIFORM) {
            t = __builtin_amdgcn_readfirstlane(t);
            x = __builtin_amdgcn_readfirstlane(x);
            y = __builtin_amdgcn_readfirstlane(y);
            asm volatile("" : "+s"(t), "+s"(x), "+s"(y));
        } else {
            asm volatile("" : "+v"(t), "+v"(x), "+v"(y));
        }
        set(a, s, t, x, y);
    }
    __host__ __device__ void set(const CacheAttend &a, int s, int t, int x, int y) {
        tokens = (int)min((long long)max(t, 0), (long long)a.max_blocks << (a.c.tile_shift + 4));
        if constexpr (LIST) {
            row0 = s;
            n_query = 1;
            first = min(max(x, 0), a.max_keys);
        } else {
            row0 = min(max(x, 0), a.T);
            n_query = min(max(y, row0), a.T) - row0;
            first = (int)((unsigned)max(t, 0) - (unsigned)n_query + 1u);  // (of a request without queries it may wrap)
        }
    }
    __host__ __device__ int queries(const CacheAttend &a) const { return min(n_query, a.max_query); }
    // Keys [low, high) that query t sees; sees_from and sees_to: the same for who keeps to keys that some query sees.
    __host__ __device__ int sees_to(int t) const { return LIST ? first : first + t; }
    __host__ __device__ int sees_from(const CacheAttend &a, int t) const { return !LIST && a.window > 0 ? max(first + t, 0) - a.window : 0; }
    __host__ __device__ int high(int t) const { return LIST ? first : min(max(sees_to(t), 0), tokens); }
    __host__ __device__ int low(const CacheAttend &a, int t) const { return !LIST && a.window > 0 ? min(max(sees_from(a, t), 0), tokens) : 0; }
};

// Quanta of `quantum` keys that the queries t0 .. t1 see, at least one: rows that see nothing want their outputs too.
template <typename U> __host__ __device__ inline int quanta_of(const CacheAttend &a, const U &u, int t0, int t1, int quantum) {
    return max((u.high(t1) + quantum - 1) / quantum - u.low(a, t0) / quantum, 1);
}
// The same of a request in the kernel for few queries, if it takes that many rows.
template <typename U> __host__ __device__ inline int few_quanta(const CacheAttend &a, const U &u, int most_rows, int quantum) {
    const int q = u.queries(a);
    return q > 0 && q * a.G <= most_rows ? quanta_of(a, u, 0, q - 1, quantum) : 0;
}

// Keys [from, to) of the part [now, stop) of the flat work's unit [u0, u1), the queries t0 .. t1.
struct PartKeys {
    int from, to;
    template <typename U>
    __host__ __device__ PartKeys(const CacheAttend &a, const U &u, int t0, int t1, int quantum, unsigned u0, unsigned u1, unsigned now, unsigned stop) {
        const int low = u.low(a, t0), high = u.high(t1), q0 = low / quantum;
        from = max(low, (q0 + (int)(now - u0)) * quantum);
        // (the last part takes its keys to the end, whatever the unit's nominal length)
        to = stop == u1 ? high : min(high, (q0 + (int)(stop - u0)) * quantum);
    }
};
// The partial result that a part of a unit that was cut leaves: two a workgroup, of a unit that began before it and of one that goes on behind it.
__host__ __device__ inline unsigned record_of(unsigned workgroup, bool began_before) { return 2 * workgroup + (began_before ? 0 : 1); }

// Writes four dims of a row from its sums relative to 2^top, and the logarithm of its denominator.
__device__ inline void put_row(const CacheAttend &a, size_t row, int d0, f32x4 sum, float top, float total) {
    const bool none = total == 0.f;  // no key at all: the largest of any weights is 2^-kSlack or more
    sum = none ? f32x4{0.f, 0.f, 0.f, 0.f} : sum * (1.f / total);
    if (a.out_bf16) *(uint2 *)((bf16_t *)a.out + row * kD + d0) = make_uint2(pack2(sum[0], sum[1]), pack2(sum[2], sum[3]));
    else *(f32x4 *)((float *)a.out + row * kD + d0) = sum;
    if (a.lse && d0 == 0) a.lse[row] = none ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
}

// ------------------------------------------------------------------------------------------------------------- few queries
// What a wave holds of 32 keys: two tiles of 16.  Key codes: lane (g, c) has dims [32 g, 32 g + 32) of the token that is
// row c of the product's left operand.  Value codes: lane (g, c) has dims [8 c, 8 c + 8) of tokens g, 4 + g, 8 + g, 12 + g.
struct Keys {
    u32x4 k[2], v[2];
    uint32_t ks[2], vs[2];
    uint32_t bad;  // tokens that do not exist, one bit each
};

// The part of the flat work that a workgroup does.  A CU issues its older waves' instructions first: of two or three workgroups on it the
// first one is done long before the last (16 requests of up to 32 K tokens: 108, 124 and 141 thousand cycles for equal pieces).  So
// where every CU has two or three, in the order of their indexes, the first kCus pieces are 3 / 16 longer than the average and the last ones as
// much shorter, if pieces are long enough for whole quanta to follow that.  Equal pieces and these: a chunk of 2048 queries on 32 K keys, two
// requests, 1750 and 1637 us; 24 mixed requests 273 and 259; 16 requests of up to 32 K tokens 71.0 and 68.5; drafts of 32 requests, 16 quanta a
// piece, 57.3 and 55.5; but one request of 131 K tokens, 11 quanta a piece, 36.3 and 39.0.  The line is drawn between these two; where it is best was not
// measured.
constexpr unsigned kCus = 256;
struct Pieces {
    unsigned groups, per, from1, from2, total;  // workgroups, those of a third (half, whole), where the pieces of the second and third begin
    // whole: pieces are units, which must not be cut (there is no room for records)
    __host__ __device__ Pieces(unsigned total_, unsigned most, bool whole) : total(total_) {
        groups = total < 1 ? 1 : total < most ? total : most;
        const bool uneven = !whole && (groups == 2 * kCus || groups == 3 * kCus) && total >= 12 * groups;
        per = uneven ? kCus : groups;
        from1 = from2 = total;
        if (uneven && groups == 2 * kCus) from1 = total / 32 * 19;
        if (uneven && groups == 3 * kCus) {
            from1 = total / 48 * 19;
            from2 = total / 48 * 35;
        }
    }
    __host__ __device__ unsigned begin(unsigned i) const {
        const unsigned t = i < per ? 0 : i < 2 * per || from2 == total ? 1 : 2, k = i - t * per;
        if (i == per && per == groups) return total;
        const unsigned from = t == 0 ? 0 : t == 1 ? from1 : from2, n = (t == 0 ? from1 : t == 1 ? from2 : total) - from;
        return from + k * (n / per) + (k < n % per ? k : n % per);
    }
    __host__ __device__ unsigned owner(unsigned x) const {
        const unsigned t = x < from1 ? 0 : x < from2 ? 1 : 2, from = t == 0 ? 0 : t == 1 ? from1 : from2;
        const unsigned n = (t == 0 ? from1 : t == 1 ? from2 : total) - from, base = n / per, longer = n % per * (base + 1);
        x -= from;
        return t * per + (x < longer ? x / (base + 1) : n % per + (x - longer) / base);
    }
};

// One step of a row's softmax: p, scores of eight keys, become weights relative to 2^m; the sums so far follow when m moves.
__device__ inline void softmax(float (&p)[8], float scale_log2, float &m, float &l, f32x4 (&acc)[8]) {
    float top = fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7]))) * scale_log2;
    if (__any(top > m + kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= alpha;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] *= alpha;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[e], scale_log2, -m));
        l += p[e];
    }
}
// The upper halves of eight floats: bf16, cut off.
__device__ inline u32x4 tops(const float (&p)[8]) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 8; e += 2) w[e >> 1] = __builtin_amdgcn_perm(__float_as_uint(p[e + 1]), __float_as_uint(p[e]), 0x07060302u);
    return w;
}
// Left operands of the value product for dims 8 c + 2 J and 8 c + 2 J + 1, from codes of four tokens at a time: pairs of dims of a
// token become pairs of tokens of a dim.
template <int J> __device__ inline void half_values(const u32x4 &codes, const float *scale, uint32_t *v0, uint32_t *v1) {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const uint32_t r0 = two<J>(codes[i], scale[i]), r1 = two<J>(codes[i + 1], scale[i + 1]);
        v0[i >> 1] = __builtin_amdgcn_perm(r1, r0, 0x05040100u);
        v1[i >> 1] = __builtin_amdgcn_perm(r1, r0, 0x07060302u);
    }
}
template <int J> __device__ inline void values(const Keys &y, const float (&scale)[8], u32x4 &v0, u32x4 &v1) {
    uint32_t a[4], b[4];
    half_values<J>(y.v[0], scale, a, b);
    half_values<J>(y.v[1], scale + 4, a + 2, b + 2);
    v0 = u32x4{a[0], a[1], a[2], a[3]};
    v1 = u32x4{b[0], b[1], b[2], b[3]};
}
// A value block that is held as NaN makes the outputs of the rows that see it NaN, and of no other row: its weight of 0 in the others
// would.  So where a step's keys are not seen by all rows, such blocks are taken out of the product (take_nan says whether there were any)
// and looked for again, key by key: nan[x] becomes NaN on the lanes whose dims and row x are hit.  Rare.
__device__ inline bool take_nan(Keys &y) {
    bool any = false;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (((y.vs[e >> 2] >> (8 * (e & 3))) & 0xFF) == 0xFF) {
            any = true;
            y.vs[e >> 2] &= ~(0xFFu << (8 * (e & 3)));
        }
    return __any(any);
}
template <int NT>
__device__ inline void find_nan(const CacheAttend &a, const int *table, int h, int key0, int from, int to, int g, const int (&low)[NT],
                                const int (&high)[NT], float (&nan)[NT]) {
    for (int key = max(key0, from); key < min(key0 + kStep, to); ++key) {
        const int id = table[key >> (a.c.tile_shift + 4)];
        if (id < 0 || id >= a.c.n_blocks) continue;
        const size_t tile = (((size_t)id * a.c.H + h) << a.c.tile_shift) + ((key >> 4) & ((1 << a.c.tile_shift) - 1));
        if (a.c.data[tile * kCacheTileBytes + kCacheVS + cache_scale_byte(key & 15, g)] != 255) continue;
#pragma unroll
        for (int x = 0; x < NT; ++x)
            if (key >= low[x] && key < high[x]) nan[x] = __builtin_nanf("");
    }
}

// Attention of few query rows (queries times heads of a group: at most 16 NT) of every request over its keys.
//
// S^T = K Q^T puts a row's scores on one lane (g, c): column c, tokens 4 i + g of each tile; these registers are the
// right operand of O^T = V^T P^T as they are (contraction slot 8 g + 4 tile + i), and a row's sums come out on the lanes that hold its
// softmax, so that neither the weights nor the rescaling cross lanes.  Codes become bf16 in registers, without rounding (three
// significant bits at most).
//
// A weight enters the second product as bf16 terms whose products add up in fp32, cut off and not rounded, so that three terms are the
// float32 weight and two are 16 bits of it.  Few rows leave columns free: with PACK = 3 (up to 5 rows) or 2 (up to 8) the terms of a row stand in
// columns c, c + R, c + 2 R, whose lanes all compute the row's scores, and one set of products carries them; further terms take a set of
// their own.  PACK, SETS = 3, 1; 2, 2; 1, 3: three terms, float32 outputs; 3, 1; 2, 1; 1, 2: bf16 outputs; 1, 1: bf16 outputs
// of more than 16 rows, weights rounded to bf16 (their errors of half a step average out over the keys).
//
// The work is flat: the requests' keys in units of 128, KV head behind KV head, cut into equal pieces, one per workgroup, wherever the
// cuts fall.  Lengths are device values and ragged; so no workgroup is idle while another has more to read.  Every workgroup finds its
// piece from the lengths.  The part of a (request, KV head) that does not span it leaves its sums in a record; the workgroup
// whose piece holds the end of one that was cut notes it for the merge.
//
// Bound by the vector unit (busy 61 %) and HBM together where there is much to read: one token of 16 requests of up to 32 K tokens, 8 KV heads,
// 68 us with the merge, 5.3 TB/s; about 220 vector instructions beside 16 products for 32 keys.  Else by its trips: one request of
// 4 K tokens 10 us.  Five drafted tokens of 32 requests, 40 rows, a window of 4096: 55 us, 23 of them products.  Lists of 1024 for 128 units 13.5.
template <int W, int PACK, int NT, int SETS, bool LIST>
__global__ __launch_bounds__(W * 64, NT > 1 || W > 4 ? 2 : 3) void cache_attend_kernel(CacheAttend a) {
    static_assert(PACK == 1 || NT == 1, "terms share the columns of one tile");
    constexpr int R = kRows / PACK;  // rows in a tile of columns
    constexpr int Q = W * kStep;     // keys of a step of all waves
    // More than one tile of columns leaves no registers for a step on its way: three steps of a wave are copied to LDS by direct loads
    // (where the waves' sums meet later), [two tiles' key codes in operand order][their value codes][their scales].
    constexpr int kDepth = 3, kStage = 4352;
    constexpr size_t kSums = sizeof(float) * W * kRows * kRecord, kStages = NT > 1 ? (size_t)W * kDepth * kStage : 0;
    __shared__ __attribute__((aligned(16))) char s_raw[kSums > kStages ? kSums : kStages];
    float(*s_acc)[kRows][kRecord] = reinterpret_cast<float(*)[kRows][kRecord]>(s_raw);
    __shared__ unsigned s_before[LIST ? 1 : kEntries + 1];  // quanta of Q keys before each request
    __shared__ unsigned s_wave[W];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
    const int term = PACK == 1 ? 0 : c / R, col_row = PACK == 1 ? c : c % R;

    unsigned total = 0;
    const bool even = LIST || a.per_unit > 0;  // units of equal nominal length: no need to look at the lengths
    if (even) {
        total = (unsigned)a.n_here * a.c.H * (unsigned)a.per_unit;
    } else {
        for (int e0 = 0; e0 < a.n_here; e0 += W * 64) {
            const int e = e0 + tid;
            unsigned n = 0;
            if (e < a.n_here) {
                const Unit<LIST> u(a, a.first + e, 0, std::false_type());
                n = (unsigned)few_quanta(a, u, NT * R, Q) * (unsigned)a.c.H;
            }
            const unsigned incl = (unsigned)wave_scan_add((int)n);
            if (lane == 63) s_wave[wave] = incl;
            __syncthreads();
            unsigned before = total;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                if (w < wave) before += s_wave[w];
                total += s_wave[w];
            }
            if (e < a.n_here) s_before[e] = before + incl - n;
            __syncthreads();
        }
        if (tid == 0) s_before[a.n_here] = total;
        __syncthreads();
    }
    const Pieces pieces(__builtin_amdgcn_readfirstlane(total), gridDim.x, a.whole);
    if (blockIdx.x >= pieces.groups || total == 0) {
        if (tid == 0 && a.notes) a.notes[blockIdx.x].first = -1;
        return;
    }
    const unsigned begin = pieces.begin(blockIdx.x), end = pieces.begin(blockIdx.x + 1);
    MergeNote note = {-1, 0, 0, 0, 0};
    int entry = 0;
    if (!even) {  // the last request that begins at or before the piece (of those, the one that is not empty)
        for (int width = 1 << (31 - __builtin_clz(a.n_here)); width; width >>= 1)
            if (entry + width < a.n_here && s_before[entry + width] <= begin) entry += width;
    }
    const int tiles_mask = (1 << a.c.tile_shift) - 1;
    const int k_row = 4 * (c & 3) + (c >> 2);  // token that is row c of the key operand: row 4 g + i is token 4 i + g
    const uint32_t k_at = 64 * k_row + 16 * g, ks_at = kCacheKS + cache_scale_byte(k_row, g);
    const uint32_t v_at = kCacheV + 64 * g + 4 * c, vs_at = kCacheVS + 16 * g + 4 * (c >> 2);

    for (unsigned now = begin; now < end;) {
        int s, h;
        unsigned u0, u1;
        if (even) {
            const unsigned u = now / (unsigned)a.per_unit;
            s = (int)(u / (unsigned)a.c.H);
            h = (int)(u % (unsigned)a.c.H);
            u0 = u * (unsigned)a.per_unit;
            u1 = u0 + (unsigned)a.per_unit;
        } else {
            while (s_before[entry + 1] <= now) ++entry;
            const unsigned first = s_before[entry], per = (s_before[entry + 1] - first) / (unsigned)a.c.H;
            s = entry;
            h = (int)((now - first) / per);
            u0 = first + (unsigned)h * per;
            u1 = u0 + per;
        }
        s = __builtin_amdgcn_readfirstlane(s) + a.first;
        h = __builtin_amdgcn_readfirstlane(h);
        const unsigned stop = min(u1, end);
        const Unit<LIST> unit(a, s, h, std::true_type());
        const int n_rows = unit.queries(a) * a.G, t_last = (n_rows - 1) / a.G;
        if (!LIST && (n_rows <= 0 || n_rows > NT * R)) {  // (equal units: nothing to do here, or the other kernel's)
            now = stop;
            continue;
        }
        // keys of this part that any row sees, that every row sees, that this lane's rows see
        const int q0 = unit.low(a, 0) / Q;
        const PartKeys keys(a, unit, 0, t_last, Q, u0, u1, now, stop);
        const int from = keys.from, to = keys.to;
        const int all_low = max(unit.sees_from(a, t_last), from), all_high = min(unit.sees_to(0), to);
        int low[NT], high[NT];
        u32x4 qv[NT][4];  // right operand of step j: dims 32 g + 8 j .. + 8 of the column's row
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            const int row = min(R * x + col_row, n_rows - 1), t = row / a.G;
            low[x] = max(unit.sees_from(a, t), from);
            high[x] = min(unit.sees_to(t), to);
            const bf16_t *p = a.q + (long long)(unit.row0 + t) * a.q_stride + (long long)(h * a.G + row % a.G) * kD + 32 * g;
#pragma unroll
            for (int j = 0; j < 4; ++j) qv[x][j] = *(const u32x4 *)(p + 8 * j);
        }
        const int step0 = (q0 + (int)(now - u0)) * W;  // the wave's steps: step0 + wave + W n
        const int n_mine = to > from ? max((to - kStep * (step0 + wave) + Q - 1) / Q, 0) : 0;
        const int *table = a.table + (size_t)s * a.max_blocks;
        const int *list = LIST ? a.pos + ((size_t)s * a.c.H + h) * a.max_keys : nullptr;

        // Up to 64 places on the lanes.  Dense: index of tile l & 1 of the wave's step n + l / 2, in units of tiles of the pool.  Listed:
        // index of key l & 31 of step n + l / 32, in units of rows of the pool.  -1: no such place.  A list's positions are
        // looked up two lots ahead, its blocks one lot, so that neither trip is waited for but at the start (16 requests x 8 heads x 1024 tokens:
        // 14.4 us, 17.6 without; a dense lot lasts 32 steps, and a register more costs as much as its wait).
        constexpr int kAhead = LIST ? 2 : 32;  // steps whose places lie on the lanes
        auto position = [&](int n) __attribute__((always_inline)) -> int {  // listed
            const long long e = (long long)(step0 + wave + W * (n + (lane >> 5))) * kStep + (lane & 31);
            const int p = e < to ? list[e] : -1;
            return p < unit.tokens ? p : -1;
        };
        auto block_of = [&](int p) __attribute__((always_inline)) -> int { return p >= 0 ? table[p >> (a.c.tile_shift + 4)] : -1; };
        auto row_of = [&](int p, int id) __attribute__((always_inline)) -> int {
            return (unsigned)id < (unsigned)a.c.n_blocks
                       ? (int)(((((unsigned)id * a.c.H + h) << a.c.tile_shift) + ((p >> 4) & tiles_mask)) * 16u + (p & 15)) : -1;
        };
        auto tile_of = [&](int n) __attribute__((always_inline)) -> int {  // dense
            const int tile = (step0 + wave + W * (n + (lane >> 1))) * 2 + (lane & 1);
            const int id = (long long)tile * 16 < to ? table[tile >> a.c.tile_shift] : -1;
            return (unsigned)id < (unsigned)a.c.n_blocks ? (int)((((unsigned)id * a.c.H + h) << a.c.tile_shift) + (tile & tiles_mask)) : -1;
        };
        struct Places {
            int held, next, id, pos;  // on the lanes now; the next lot (listed: its positions and blocks), positions of the one behind it
        } at = {-1, -1, -1, -1};
        auto begin_places = [&]() __attribute__((always_inline)) {
            if constexpr (LIST) {
                const int p = position(0);
                at.next = position(kAhead);
                at.held = row_of(p, block_of(p));
                at.id = block_of(at.next);
                at.pos = position(2 * kAhead);
            } else {
                at.held = tile_of(0);
            }
        };
        auto turn_places = [&](int n) __attribute__((always_inline)) {  // step n begins a lot
            if constexpr (LIST) {
                at.held = row_of(at.next, at.id);
                at.next = at.pos;
                at.id = block_of(at.next);
                at.pos = position(n + 2 * kAhead);
            } else {
                at.held = tile_of(n);
            }
        };
        // step n of this wave: key codes, value codes
        auto request_keys = [&](int held, int n, Keys &x) __attribute__((always_inline)) {
            x.bad = 0;
            if constexpr (LIST) x.bad = (uint32_t)(__ballot(held == -1) >> (32 * (n & 1)));
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if constexpr (LIST) {
                    const uint32_t row = (uint32_t)max(__shfl(held, 32 * (n & 1) + 16 * b + k_row), 0);
                    const uint8_t *t = a.c.data + (size_t)(row >> 4) * kCacheTileBytes;
                    x.k[b] = *(const u32x4 *)(t + 64 * (row & 15) + 16 * g);
                    x.ks[b] = t[kCacheKS + cache_scale_byte(row & 15, g)];
                } else {
                    const int id = __builtin_amdgcn_readlane(held, 2 * (n % kAhead) + b);
                    if (id < 0) x.bad |= 0xFFFFu << (16 * b);
                    const uint8_t *t = a.c.data + (size_t)max(id, 0) * kCacheTileBytes;
                    x.k[b] = __builtin_nontemporal_load((const u32x4 *)(t + k_at));
                    x.ks[b] = t[ks_at];
                }
            }
        };
        auto request_values = [&](int held, int n, Keys &x) __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if constexpr (LIST) {
                    uint32_t scales = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t row = (uint32_t)max(__shfl(held, 32 * (n & 1) + 16 * b + 4 * i + g), 0);
                        const uint8_t *t = a.c.data + (size_t)(row >> 4) * kCacheTileBytes;
                        x.v[b][i] = *(const uint32_t *)(t + kCacheV + 64 * (row & 15) + 4 * c);
                        scales |= (uint32_t)t[kCacheVS + cache_scale_byte(row & 15, c >> 2)] << (8 * i);
                    }
                    x.vs[b] = scales;
                } else {
                    const uint8_t *t = a.c.data + (size_t)max(__builtin_amdgcn_readlane(held, 2 * (n % kAhead) + b), 0) * kCacheTileBytes;
#pragma unroll
                    for (int i = 0; i < 4; ++i) x.v[b][i] = __builtin_nontemporal_load((const uint32_t *)(t + v_at + 256 * i));
                    x.vs[b] = *(const uint32_t *)(t + vs_at);
                }
            }
        };

        f32x4 acc[NT][8];  // acc[x][j][i]: dim 32 g + 8 i + j of column c of tile x
        float m[NT], l[NT];
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            m[x] = kNoMax;
            l[x] = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[x][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const uint32_t cut1 = PACK > 1 && term >= 1 ? 0xFFFF0000u : 0u, cut2 = PACK > 2 && term >= 2 ? 0xFFFF0000u : 0u;
        // Step n; take_values(): where the value codes are still to be fetched into y.
        auto attend = [&](int n, Keys &y, auto take_values) __attribute__((always_inline)) {
            const int key0 = (step0 + wave + W * n) * kStep;
            f32x4 d[NT][2];
#pragma unroll
            for (int x = 0; x < NT; ++x) d[x][0] = d[x][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const float sc = __uint_as_float(y.ks[b] << 23);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const u32x4 k = eight(y.k[b][j], sc);
#pragma unroll
                    for (int x = 0; x < NT; ++x) d[x][b] = mfma(k, qv[x][j], d[x][b]);
                }
            }
            const uint32_t bad = y.bad;
            take_values();
            if (key0 < all_low || key0 + kStep > all_high || bad != 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int in = 16 * (e >> 2) + 4 * (e & 3) + g, key = key0 + in;
                    const bool gone = (bad >> in) & 1;
#pragma unroll
                    for (int x = 0; x < NT; ++x)
                        if (gone || key < low[x] || key >= high[x]) d[x][e >> 2][e & 3] = -INFINITY;
                    // what no row sees may hold anything: its value scale must not turn a weight of 0 into NaN
                    if (gone || key < from || key >= to) y.vs[e >> 2] &= ~(0xFFu << (8 * (e & 3)));
                }
                if (!LIST && take_nan(y)) {
                    float nan[NT] = {};
                    find_nan<NT>(a, table, h, key0, from, to, g, low, high, nan);
#pragma unroll
                    for (int x = 0; x < NT; ++x)
#pragma unroll
                        for (int j = 0; j < 8; ++j) acc[x][j] += nan[x];
                }
            }
            u32x4 w[NT][SETS];  // the weights' terms
#pragma unroll
            for (int x = 0; x < NT; ++x) {
                float p[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) p[e] = d[x][e >> 2][e & 3];
                softmax(p, a.scale_log2, m[x], l[x], acc[x]);
                if constexpr (PACK == 2 && SETS == 2) {  // first and second term in the first set; the third one on the first's lanes
                    float third[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float second = cut(p[e], 0xFFFF0000u);
                        third[e] = term == 0 ? cut(second, 0xFFFF0000u) : 0.f;
                        p[e] = term == 0 ? p[e] : second;
                    }
                    w[x][0] = tops(p);
                    w[x][1] = tops(third);
                } else if constexpr (PACK == 1 && SETS == 1) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) w[x][0][e >> 1] = pack2(p[e], p[e + 1]);
                } else {
#pragma unroll
                    for (int t = 0; t < SETS; ++t) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            if (t > 0) p[e] = cut(p[e], 0xFFFF0000u);
                            if (PACK > 1) p[e] = cut(p[e], cut1);
                            if (PACK > 2) p[e] = cut(p[e], cut2);
                        }
                        w[x][t] = tops(p);
                    }
                }
            }
            float vsc[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) vsc[e] = scale_of(y.vs[e >> 2], e & 3);
            auto dims = [&](auto sel) __attribute__((always_inline)) {
                constexpr int j = decltype(sel)::value;
                u32x4 v0, v1;
                values<j>(y, vsc, v0, v1);
#pragma unroll
                for (int x = 0; x < NT; ++x)
#pragma unroll
                    for (int t = 0; t < SETS; ++t) {
                        acc[x][2 * j] = mfma(v0, w[x][t], acc[x][2 * j]);
                        acc[x][2 * j + 1] = mfma(v1, w[x][t], acc[x][2 * j + 1]);
                    }
            };
            dims(std::integral_constant<int, 0>());
            dims(std::integral_constant<int, 1>());
            dims(std::integral_constant<int, 2>());
            dims(std::integral_constant<int, 3>());
        };

        if (n_mine > 0) {
            begin_places();
            if constexpr (NT == 1) {  // two steps in registers: one worked on, one on its way
                Keys x, y;
                auto request = [&](int n, Keys &z) __attribute__((always_inline)) {
                    if (n >= n_mine) return;
                    if (n % kAhead == 0 && n) turn_places(n);
                    request_keys(at.held, n, z);
                    request_values(at.held, n, z);
                };
                request(0, x);
                for (int n = 0; n < n_mine; n += 2) {
                    request(n + 1, y);
                    attend(n, x, [] {});
                    if (n + 1 >= n_mine) break;
                    request(n + 2, x);
                    attend(n + 1, y, [] {});
                }
            } else {
                char *const stage = s_raw + wave * (kDepth * kStage);
                uint32_t missing = 0;  // tiles that do not exist, two bits a step, the latest request's lowest
                auto request = [&](int n) __attribute__((always_inline)) {
                    if (n % kAhead == 0 && n) turn_places(n);
                    const int id0 = __builtin_amdgcn_readlane(at.held, 2 * (n % kAhead)), id1 = __builtin_amdgcn_readlane(at.held, 2 * (n % kAhead) + 1);
                    missing = missing << 2 | (id0 < 0 ? 1u : 0u) | (id1 < 0 ? 2u : 0u);
                    const uint8_t *t0 = a.c.data + (size_t)max(id0, 0) * kCacheTileBytes, *t1 = a.c.data + (size_t)max(id1, 0) * kCacheTileBytes;
                    char *to_lds = stage + (n % kDepth) * kStage;
                    lds_dma_stream<16>((t0 + k_at), to_lds);
                    lds_dma_stream<16>((t1 + k_at), to_lds + 1024);
                    lds_dma_stream<16>((t0 + kCacheV + 16 * lane), to_lds + 2048);
                    lds_dma_stream<16>((t1 + kCacheV + 16 * lane), to_lds + 3 * 1024);
                    lds_dma_stream<4>(((lane < 32 ? t0 : t1) + kCacheKS + 4 * (lane & 31)), to_lds + 4096);
                };
                for (int n = 0; n < min(kDepth, n_mine); ++n) request(n);
                for (int n = 0; n < n_mine; ++n) {
                    const int later = min(kDepth - 1, n_mine - 1 - n);  // steps requested after this one, five loads each
                    if (later == 2) asm volatile("s_waitcnt vmcnt(10)" ::: "memory");
                    else if (later == 1) asm volatile("s_waitcnt vmcnt(5)" ::: "memory");
                    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    const char *from_lds = stage + (n % kDepth) * kStage;
                    const uint32_t gone = missing >> (2 * later);
                    Keys x;
                    x.bad = (gone & 1 ? 0xFFFFu : 0u) | (gone & 2 ? 0xFFFF0000u : 0u);
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        x.k[b] = *(const u32x4 *)(from_lds + 1024 * b + 16 * lane);
                        x.ks[b] = *(const uint8_t *)(from_lds + 4096 + 128 * b + (ks_at - kCacheKS));
                    }
                    attend(n, x, [&]() __attribute__((always_inline)) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) x.v[b][i] = *(const uint32_t *)(from_lds + 2048 + 1024 * b + (v_at - kCacheV) + 256 * i);
                            x.vs[b] = *(const uint32_t *)(from_lds + 4096 + 128 * b + (vs_at - kCacheKS));
                        }
                    });
                    if (n + kDepth < n_mine) {
                        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the stage has been read)
                        request(n + kDepth);
                    }
                }
                __syncthreads();  // (the sums go where the stages were)
            }
        } else if constexpr (NT > 1) {
            __syncthreads();
        }

        // the waves' sums, and the terms', meet in LDS; 32 threads to a row, four dims each
        const bool whole = now == u0 && stop == u1;
        float *record = a.part + (size_t)record_of(blockIdx.x, now > u0) * a.rows * kRecord;
        const int d0 = 4 * (tid & 31);
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            if (x > 0 && R * x >= n_rows) break;
            l[x] += __shfl_xor(l[x], 16);
            l[x] += __shfl_xor(l[x], 32);
            if (R * x + col_row < n_rows && term < PACK) {
                float *r = s_acc[wave][c];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    *(f32x4 *)(r + 32 * g + 8 * i) = f32x4{acc[x][0][i], acc[x][1][i], acc[x][2][i], acc[x][3][i]};
                    *(f32x4 *)(r + 32 * g + 8 * i + 4) = f32x4{acc[x][4][i], acc[x][5][i], acc[x][6][i], acc[x][7][i]};
                }
                if (g == 0) {
                    r[kD] = m[x];
                    r[kD + 1] = l[x];
                }
            }
            __syncthreads();
            // (with one tile the reads of a thread's rows stand side by side, rows behind the last one read what lies there and write nothing: 24
            // requests of mixed lengths 273 us, 281 row by row; with three tiles the registers for that are not there: drafts 64 us, 58)
            constexpr int kPasses = NT == 1 ? (R + 2 * W - 1) / (2 * W) : 1;
            for (int in0 = tid >> 5; in0 < (NT == 1 ? 2 * W : min(R, n_rows - R * x)); in0 += 2 * W * kPasses) {
                f32x4 sum[kPasses];
                float top[kPasses], all[kPasses];
#pragma unroll
                for (int pass = 0; pass < kPasses; ++pass) {
                    const int in = min(in0 + 2 * W * pass, R - 1);
                    float2 ml[W];
#pragma unroll
                    for (int w = 0; w < W; ++w) ml[w] = *(const float2 *)&s_acc[w][in][kD];
                    top[pass] = kNoMax;
#pragma unroll
                    for (int w = 0; w < W; ++w) top[pass] = fmaxf(top[pass], ml[w].x);
                    sum[pass] = f32x4{0.f, 0.f, 0.f, 0.f};
                    all[pass] = 0.f;
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        const float f = __builtin_amdgcn_exp2f(ml[w].x - top[pass]);
                        f32x4 v = *(const f32x4 *)(s_acc[w][in] + d0);
#pragma unroll
                        for (int t = 1; t < PACK; ++t) v += *(const f32x4 *)(s_acc[w][in + t * R] + d0);
                        sum[pass] += v * f;
                        all[pass] += ml[w].y * f;
                    }
                }
#pragma unroll
                for (int pass = 0; pass < kPasses; ++pass) {
                    const int in = in0 + 2 * W * pass, row = R * x + in;
                    if (in >= R || row >= n_rows) continue;
                    if (whole) {
                        put_row(a, (size_t)(unit.row0 + row / a.G) * a.c.H * a.G + h * a.G + row % a.G, d0, sum[pass], top[pass], all[pass]);
                    } else {
                        float *r = record + (size_t)row * kRecord;
                        *(f32x4 *)(r + d0) = sum[pass];
                        if (d0 == 0) {
                            r[kD] = top[pass];
                            r[kD + 1] = all[pass];
                        }
                    }
                }
            }
            __syncthreads();
        }
        if (now > u0 && stop == u1) note = {(int)pieces.owner(u0), h, unit.row0, 0, n_rows};
        now = stop;
    }
    if (tid == 0 && a.notes) a.notes[blockIdx.x] = note;
}

// ------------------------------------------------------------------------------------------------------------ many queries
// Attention of many query rows of a (request, KV head): 192 at a time, tiles of 16 dealt to the four waves, three each (two: 2091 us for
// the case below; four do not fit the registers of two workgroups on a CU).
//
// Bound by the matrix unit, so the codes are converted once per workgroup and not once per wave: of a round of 64 keys a wave converts 16, as
// the few-query kernel does in registers, and leaves the operands in LDS as they are (a KiB each, 16 bytes a lane), from where all waves take
// them.  Two buffers of 32 KiB: one barrier per round, and a wave may run a round ahead.  The next round's codes are on their way
// meanwhile.  Outputs in bf16: weights rounded to bf16, one set of products; float32: three terms, cut off (three sets).  Two chunks of
// 2048 queries on 32 K keys, 8 KV heads of 4 query heads, bf16: 1620 to 1730 us on several cards, 1.12 to 1.19 PFLOP/s; a library product of 8192^3 in a
// steady loop reaches 1.21 to 1.64 by the operands' layout (1.64 beside 1.18 here on one card).
//
// The work is flat as above.  A causal row tile sees the more keys the later it stands; so the tiles of a (request, KV head) are taken
// in pairs, the last and the first, the last but one and the second, which cost the same together, and a pair's place in the flat
// work is found by a division.
constexpr int kTiles = 3;                            // tiles of 16 rows per wave
constexpr int kChunkRows = kWaves * kTiles * kRows;  // rows of a workgroup
constexpr int kRound = kWaves * 16;                  // keys of a round
// What the compiler is asked for between the products (kinds of instructions, and how many).  A chunk of 2048 queries on 32 K keys, two
// requests: its own order 1852 us; operands two ahead 1826; weights beside products, 4 a product 1781, 3 1749, 2 1728, 1 1746.
constexpr int kVector = 0x002, kMatrix = 0x008, kLdsRead = 0x100;
constexpr int kAhead = 2, kWeightOps = 28, kBeside = 2;

struct Chunks {  // how a request's row tiles lie in the flat work of one KV head
    int n_rows, tiles;
    unsigned pair, single, per_head;  // quanta of a pair, of the middle tile of an odd number, of all
    template <typename U> __host__ __device__ static int quanta(const CacheAttend &a, const U &u, int n_rows, int tile) {
        return quanta_of(a, u, kChunkRows * tile / a.G, (min(kChunkRows * (tile + 1), n_rows) - 1) / a.G, kQuantum);
    }
    template <typename U> __host__ __device__ Chunks(const CacheAttend &a, const U &u) {
        n_rows = u.queries(a) * a.G;
        tiles = 0;
        pair = single = per_head = 0;
        if (n_rows <= kRows) return;  // (the few-query kernel's, which takes that many where there are requests with more than kFewRows)
        tiles = (n_rows + kChunkRows - 1) / kChunkRows;
        const int middle = quanta(a, u, n_rows, (tiles - 1) / 2);
        // An estimate for the pairs: with as many keys as queries the tiles' quanta are a line, or with a window concave, and twice the middle covers any
        // pair.  It is no bound: tiles of queries in front of the first key see nothing, and then a pair's first tile alone may need more.
        // So a pair's second tile gets what the first one leaves of it, and that is one quantum at least (see at()); what a unit needs beyond its nominal length its last
        // part takes along (PartKeys).
        if (tiles > 1) pair = (unsigned)max(2 * middle + 2, quanta(a, u, n_rows, tiles - 1) + 1);
        if (tiles & 1) single = (unsigned)middle;
        per_head = (unsigned)(tiles / 2) * pair + single;
    }
    // The row tile that the flat work's quantum `now` belongs to, and its place there; head0: where the KV head begins.
    struct Tile {
        int tile;
        unsigned u0, u1;
    };
    template <typename U> __host__ __device__ Tile at(const CacheAttend &a, const U &u, unsigned head0, unsigned now) const {
        const unsigned paired = head0 + (unsigned)(tiles / 2) * pair;
        if (now >= paired) return {tiles / 2, paired, paired + single};
        const int p = (int)((now - head0) / pair);
        const unsigned p0 = head0 + (unsigned)p * pair, split = p0 + (unsigned)min(quanta(a, u, n_rows, tiles - 1 - p), (int)pair - 1);
        return now >= split ? Tile{p, split, p0 + pair} : Tile{tiles - 1 - p, p0, split};
    }
};

template <int SETS>
__global__ __launch_bounds__(kWaves * 64, 2) void cache_chunk_kernel(CacheAttend a) {
    __shared__ u32x4 s_k[2][kWaves][4][64], s_v[2][kRound / kStep][8][64];
    __shared__ unsigned s_before[kEntries + 1], s_wave[kWaves];
    __shared__ uint32_t s_flags[2][kWaves];  // of a tile of keys: bit 0: in no block, bit 1: values held as NaN were taken out
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
    unsigned total = 0;
    for (int e0 = 0; e0 < a.n_here; e0 += kWaves * 64) {
        const int e = e0 + tid;
        const unsigned n = e < a.n_here ? Chunks(a, Unit<false>(a, a.first + e, 0, std::false_type())).per_head * (unsigned)a.c.H : 0u;
        const unsigned incl = (unsigned)wave_scan_add((int)n);
        if (lane == 63) s_wave[wave] = incl;
        __syncthreads();
        unsigned before = total;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) before += s_wave[w];
            total += s_wave[w];
        }
        if (e < a.n_here) s_before[e] = before + incl - n;
        __syncthreads();
    }
    if (tid == 0) s_before[a.n_here] = total;
    __syncthreads();
    const Pieces pieces(__builtin_amdgcn_readfirstlane(total), gridDim.x, false);
    if (blockIdx.x >= pieces.groups || total == 0) {
        if (tid == 0) a.notes[blockIdx.x].first = -1;
        return;
    }
    const unsigned begin = pieces.begin(blockIdx.x), end = pieces.begin(blockIdx.x + 1);
    MergeNote note = {-1, 0, 0, 0, 0};
    int entry = 0;
    for (int width = 1 << (31 - __builtin_clz(a.n_here)); width; width >>= 1)
        if (entry + width < a.n_here && s_before[entry + width] <= begin) entry += width;
    const int tiles_mask = (1 << a.c.tile_shift) - 1;
    const int k_row = 4 * (c & 3) + (c >> 2);
    const uint32_t k_at = 64 * k_row + 16 * g, ks_at = kCacheKS + cache_scale_byte(k_row, g);
    const uint32_t v_at = kCacheV + 64 * g + 4 * c, vs_at = kCacheVS + 16 * g + 4 * (c >> 2);

    for (unsigned now = begin; now < end;) {
        while (s_before[entry + 1] <= now) ++entry;
        const int s = __builtin_amdgcn_readfirstlane(entry) + a.first;
        const Unit<false> unit(a, s, 0, std::true_type());
        const Chunks ch(a, unit);
        const unsigned first = s_before[entry];
        const int h = __builtin_amdgcn_readfirstlane((int)((now - first) / ch.per_head));
        const Chunks::Tile place = ch.at(a, unit, first + (unsigned)h * ch.per_head, now);
        const int all_rows = ch.n_rows, tile = __builtin_amdgcn_readfirstlane(place.tile);
        const unsigned u0 = place.u0, u1 = place.u1, stop = min(u1, end);
        const int base = kChunkRows * tile, n_rows = min(all_rows - base, kChunkRows);
        const int t_first = base / a.G, t_last = (base + n_rows - 1) / a.G;
        const int q0 = unit.low(a, t_first) / kQuantum + (int)(now - u0);
        const PartKeys keys(a, unit, t_first, t_last, kQuantum, u0, u1, now, stop);
        const int from = keys.from, to = keys.to;
        const int all_low = max(unit.sees_from(a, t_last), from), all_high = min(unit.sees_to(t_first), to);
        const int key_at = q0 * kQuantum;  // of the first round
        const int rounds = to > from ? (to - key_at + kRound - 1) / kRound : 0;
        // this lane's rows: columns of tiles wave + 4 x
        int low[kTiles], high[kTiles], wave_low = 0, wave_high = to;
        u32x4 qv[kTiles][4];
#pragma unroll
        for (int x = 0; x < kTiles; ++x) {
            const int row = base + min(kRows * (kWaves * x + wave) + c, n_rows - 1), t = row / a.G;
            low[x] = max(unit.sees_from(a, t), from);
            high[x] = min(unit.sees_to(t), to);
            const bf16_t *p = a.q + (long long)(unit.row0 + t) * a.q_stride + (long long)(h * a.G + row % a.G) * kD + 32 * g;
#pragma unroll
            for (int j = 0; j < 4; ++j) qv[x][j] = *(const u32x4 *)(p + 8 * j);
        }
        {  // keys that all rows of this wave see
            const int r0 = min(kRows * wave, n_rows - 1), r1 = min(kRows * (kWaves * (kTiles - 1) + wave) + kRows - 1, n_rows - 1);
            wave_low = max(unit.sees_from(a, (base + r1) / a.G), from);
            wave_high = min(unit.sees_to((base + r0) / a.G), to);
        }
        const int *table = a.table + (size_t)s * a.max_blocks;
        auto places = [&](int n0) __attribute__((always_inline)) -> int {  // this wave's tile of round n0 + l
            const long long t = (long long)(key_at >> 4) + (long long)(n0 + lane) * kWaves + wave;
            if (t * 16 >= to) return -1;
            const int id = table[t >> a.c.tile_shift];
            if (id < 0 || id >= a.c.n_blocks) return -1;
            return (int)((((unsigned)id * a.c.H + h) << a.c.tile_shift) + ((int)t & tiles_mask));
        };
        u32x4 kc, vc;  // this wave's codes of the next round
        uint32_t ksc, vsc;
        bool gone;
        auto request = [&](int held, int n) __attribute__((always_inline)) {
            const int id = __builtin_amdgcn_readlane(held, n & 63);
            gone = id < 0;
            const uint8_t *t = a.c.data + (size_t)max(id, 0) * kCacheTileBytes;
            kc = *(const u32x4 *)(t + k_at);
#pragma unroll
            for (int i = 0; i < 4; ++i) vc[i] = *(const uint32_t *)(t + v_at + 256 * i);
            ksc = t[ks_at];
            vsc = *(const uint32_t *)(t + vs_at);
        };
        f32x4 acc[kTiles][8];
        float m[kTiles], l[kTiles];
#pragma unroll
        for (int x = 0; x < kTiles; ++x) {
            m[x] = kNoMax;
            l[x] = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[x][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const int n_tiles = (n_rows - kRows * wave + kRows * kWaves - 1) / (kRows * kWaves);  // of this wave (may be 0 or less)
        int held = rounds > 0 ? places(0) : -1;
        if (rounds > 0) request(held, 0);
        // the rounds of a wave with NX tiles of rows, without a branch on the tile between the products
        auto run = [&](auto count) __attribute__((always_inline)) {
            for (int n = 0; n < rounds; ++n) {
                const int buf = n & 1;
                {  // this wave's keys of the round become operands
                    const int key0 = key_at + n * kRound + 16 * wave;
                    bool nan = false;
                    if (key0 < all_low || key0 + 16 > all_high || gone) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = key0 + 4 * i + g;
                            const uint32_t byte = 0xFFu << (8 * i);
                            if (gone || key < from || key >= to) vsc &= ~byte;  // (what no row sees may hold anything)
                            if ((vsc & byte) == byte) {
                                nan = true;
                                vsc &= ~byte;
                            }
                        }
                        nan = __any(nan);
                    }
                    if (lane == 0) s_flags[buf][wave] = (gone ? 1u : 0u) | (nan ? 2u : 0u);
                    const float sc = __uint_as_float(ksc << 23);
#pragma unroll
                    for (int j = 0; j < 4; ++j) s_k[buf][wave][j][lane] = eight(kc[j], sc);
                    float vf[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) vf[i] = scale_of(vsc, i);
                    auto dims = [&](auto sel) __attribute__((always_inline)) {
                        constexpr int j = decltype(sel)::value;
                        uint32_t v0[2], v1[2];
                        half_values<j>(vc, vf, v0, v1);
                        uint2 *at = (uint2 *)&s_v[buf][wave >> 1][2 * j][lane] + (wave & 1);
                        at[0] = make_uint2(v0[0], v0[1]);
                        at[2 * 64] = make_uint2(v1[0], v1[1]);
                    };
                    dims(std::integral_constant<int, 0>());
                    dims(std::integral_constant<int, 1>());
                    dims(std::integral_constant<int, 2>());
                    dims(std::integral_constant<int, 3>());
                }
                if (n + 1 < rounds) {
                    if (((n + 1) & 63) == 0) held = places(n + 1);
                    request(held, n + 1);
                }
                lds_barrier();
                // scores of the round's 64 keys (those behind the last one are masked)
                constexpr int NX = decltype(count)::value, NB = kRound / 16;
                const int key0 = key_at + n * kRound;
                f32x4 d[NX][NB];
#pragma unroll
                for (int b = 0; b < NB; ++b) {
#pragma unroll
                    for (int x = 0; x < NX; ++x) d[x][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const u32x4 k = s_k[buf][b][j][lane];
#pragma unroll
                        for (int x = 0; x < NX; ++x) d[x][b] = mfma(k, qv[x][j], d[x][b]);
                    }
                }
                // (operands are read kAhead ahead of their products)
                __builtin_amdgcn_sched_group_barrier(kLdsRead, kAhead, 0);
#pragma unroll
                for (int i = 0; i < 4 * NB; ++i) {
                    __builtin_amdgcn_sched_group_barrier(kMatrix, NX, 0);
                    if (i + kAhead < 4 * NB) __builtin_amdgcn_sched_group_barrier(kLdsRead, 1, 0);
                }
                uint32_t flags = 0;
#pragma unroll
                for (int b = 0; b < NB; ++b) flags |= s_flags[buf][b] << (2 * b);
                flags = (uint32_t)__builtin_amdgcn_readfirstlane((int)flags);
                if (key0 < wave_low || key0 + kRound > wave_high || flags != 0) {
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = key0 + 16 * b + 4 * i + g;
                            const bool none = (flags >> (2 * b)) & 1;
#pragma unroll
                            for (int x = 0; x < NX; ++x)
                                if (none || key < low[x] || key >= high[x]) d[x][b][i] = -INFINITY;
                        }
                    if (flags & 0xAAu) {
                        float nan[kTiles] = {};
                        for (int step = 0; step < kRound / kStep; ++step)
                            find_nan<kTiles>(a, table, h, key0 + step * kStep, from, to, g, low, high, nan);
#pragma unroll
                        for (int x = 0; x < NX; ++x)
#pragma unroll
                            for (int j = 0; j < 8; ++j) acc[x][j] += nan[x];
                    }
                }
                float top[NX];
                bool rise = false;
#pragma unroll
                for (int x = 0; x < NX; ++x) {
                    float t = d[x][0][0];
#pragma unroll
                    for (int e = 1; e < 4 * NB; ++e) t = fmaxf(t, d[x][e >> 2][e & 3]);
                    top[x] = t * a.scale_log2;
                    rise |= top[x] > m[x] + kSlack;
                }
                if (__any(rise)) {
#pragma unroll
                    for (int x = 0; x < NX; ++x) {
                        float t = fmaxf(top[x], __shfl_xor(top[x], 16));
                        t = fmaxf(t, __shfl_xor(t, 32));
                        const float mn = t > m[x] + kSlack ? t : m[x], alpha = __builtin_amdgcn_exp2f(m[x] - mn);
                        m[x] = mn;
                        l[x] *= alpha;
#pragma unroll
                        for (int j = 0; j < 8; ++j) acc[x][j] *= alpha;
                    }
                }
                // weights and the value product, without a branch, so that the one's instructions fill the other's time
#pragma unroll
                for (int step = 0; step < kRound / kStep; ++step) {
                    u32x4 w[NX][SETS];
#pragma unroll
                    for (int x = 0; x < NX; ++x) {
                        float p[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(d[x][2 * step + (e >> 2)][e & 3], a.scale_log2, -m[x]));
                            l[x] += p[e];
                        }
                        if constexpr (SETS == 1) {
#pragma unroll
                            for (int e = 0; e < 8; e += 2) w[x][0][e >> 1] = pack2(p[e], p[e + 1]);
                        } else {
#pragma unroll
                            for (int t = 0; t < SETS; ++t) {
                                if (t > 0)
#pragma unroll
                                    for (int e = 0; e < 8; ++e) p[e] = cut(p[e], 0xFFFF0000u);
                                w[x][t] = tops(p);
                            }
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const u32x4 v = s_v[buf][step][j][lane];
#pragma unroll
                        for (int x = 0; x < NX; ++x)
#pragma unroll
                            for (int t = 0; t < SETS; ++t) acc[x][j] = mfma(v, w[x][t], acc[x][j]);
                    }
                }
                // the order of the products: the first step's weights (kWeightOps a tile); its products, beside each of which kBeside
                // instructions of the second step's weights go; the second step's products
                __builtin_amdgcn_sched_group_barrier(kVector, kWeightOps * NX, 1);
                __builtin_amdgcn_sched_group_barrier(kLdsRead, kAhead, 1);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
#pragma unroll
                    for (int x = 0; x < NX * SETS; ++x) {
                        __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 1);
                        __builtin_amdgcn_sched_group_barrier(kVector, kBeside, 1);
                    }
                    __builtin_amdgcn_sched_group_barrier(kLdsRead, 1, 1);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    __builtin_amdgcn_sched_group_barrier(kMatrix, NX * SETS, 1);
                    __builtin_amdgcn_sched_group_barrier(kLdsRead, 1, 1);
                }
            }
        };
        // (a wave without rows converts all the same; its one tile is not written)
        if (n_tiles > 1) run(std::integral_constant<int, kTiles>());
        else run(std::integral_constant<int, 1>());
        lds_barrier();  // (the last operands have been used: the next part writes others)
        const bool whole = now == u0 && stop == u1;
        float *record = a.part + (size_t)record_of(blockIdx.x, now > u0) * a.rows * kRecord;
#pragma unroll
        for (int x = 0; x < kTiles; ++x) {
            const int in = kRows * (kWaves * x + wave) + c, row = base + in;
            l[x] += __shfl_xor(l[x], 16);
            l[x] += __shfl_xor(l[x], 32);
            if (in >= n_rows) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int d0 = 32 * g + 8 * i + 4 * half;
                    const f32x4 sum = {acc[x][4 * half][i], acc[x][4 * half + 1][i], acc[x][4 * half + 2][i], acc[x][4 * half + 3][i]};
                    if (whole) put_row(a, (size_t)(unit.row0 + row / a.G) * a.c.H * a.G + h * a.G + row % a.G, d0, sum, m[x], l[x]);
                    else *(f32x4 *)(record + (size_t)in * kRecord + d0) = sum;
                }
            if (!whole && g == 0) {
                record[(size_t)in * kRecord + kD] = m[x];
                record[(size_t)in * kRecord + kD + 1] = l[x];
            }
        }
        if (now > u0 && stop == u1) note = {(int)pieces.owner(u0), h, unit.row0, base, all_rows};
        now = stop;
    }
    if (tid == 0) a.notes[blockIdx.x] = note;
}

// Joins the records of the unit whose end workgroup blockIdx.x noted, if it did: one of workgroup `first` (its last part), one each of
// those behind it up to this one (their first parts).  Groups of 32 threads take a row, four dims each; GROUPS of them share a row's records.
// Bound by two round trips to memory: the note, the records.
constexpr int kMergeThreads = 256;
template <int GROUPS>
__global__ __launch_bounds__(kMergeThreads) void cache_merge_kernel(CacheAttend a) {
    __shared__ float s_sum[kMergeThreads / 32][kRecord];
    const MergeNote note = a.notes[blockIdx.x];
    if (note.first < 0) return;
    const int all = threadIdx.x >> 5, group = all % GROUPS, d0 = 4 * (threadIdx.x & 31);
    const int in = (int)blockIdx.y * (kMergeThreads / 32 / GROUPS) + all / GROUPS;
    const int n = (int)blockIdx.x - note.first + 1, row = note.base + in;
    const bool mine = in < a.rows && row < note.rows;
    float top = kNoMax, total = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    auto join = [&](float m, float l, const f32x4 &v) {
        const float mn = fmaxf(top, m), f0 = __builtin_amdgcn_exp2f(top - mn), f1 = __builtin_amdgcn_exp2f(m - mn);
        sum = sum * f0 + v * f1;
        total = total * f0 + l * f1;
        top = mn;
    };
    if (mine) {
        constexpr int kAtOnce = 4;
        for (int k = group; k < n; k += GROUPS * kAtOnce) {
            float m[kAtOnce], l[kAtOnce];
            f32x4 v[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const int kk = min(k + GROUPS * j, n - 1);
                const float *x = a.part + ((size_t)record_of(note.first + kk, kk > 0) * a.rows + in) * kRecord;
                v[j] = *(const f32x4 *)(x + d0);
                m[j] = x[kD];
                l[j] = x[kD + 1];
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                if (k + GROUPS * j < n) join(m[j], l[j], v[j]);
        }
    }
    if constexpr (GROUPS > 1) {
        float *r = s_sum[all];
        *(f32x4 *)(r + d0) = sum;
        if (d0 == 0) {
            r[kD] = top;
            r[kD + 1] = total;
        }
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int w = 1; w < GROUPS; ++w) join(s_sum[all + w][kD], s_sum[all + w][kD + 1], *(const f32x4 *)(s_sum[all + w] + d0));
    }
    if (mine) put_row(a, (size_t)(note.row0 + row / a.G) * a.c.H * a.G + note.h * a.G + row % a.G, d0, sum, top, total);
}

}  // namespace

// Query rows of the launch for few: all of them up to kFewRows, else the requests' with at most 16, and a launch of the many-query
// kernel serves the others.  768 or (more than 16 rows) 512 workgroups of the first are resident at a time, 512 of the second; there are no
// more of them than quanta.
constexpr int kFewRows = 48;
static int few_rows(const CacheAttend &a) {
    const long long rows = (long long)a.max_query * a.G;
    return rows <= 5 ? 5 : rows <= 8 ? 8 : rows <= 16 || rows > kFewRows ? 16 : rows <= 32 ? 32 : 48;
}
// ... and those of a unit of the many-query kernel: a record has room for what a request can have (single tokens of 16 requests whose most queries are not
// known, 64 rows: 35 MB for 512 workgroups instead of 104).
static int chunk_rows(const CacheAttend &a) { return (int)std::min<long long>(kChunkRows, (long long)a.max_query * a.G); }
static size_t attend_bytes(int groups, int rows) { return (size_t)groups * (2 * rows * kRecord * 4 + sizeof(MergeNote)); }

// Units (request, KV head) that stay whole, one workgroup each, no merge behind it: short ones, where the merge costs more than the cut gains, longer
// ones too where they are many, and lists of as many units as there are CUs.  Cut and whole, us: dense, 8 units of 512 keys 9.4 and 7.9, of
// 1024 9.3 and 11.3; 128 units of up to 1024 keys 14.6 and 11.9, of up to 4096 22 and 32; 512 units of up to 2048 keys 30 and 27, of up to 4096 44
// and 43.  Lists, 8 units of 512 tokens 8.9 and 8.0, of 1024 9.5 and 11.0; 128 units of 1024 15.9 and 14.1, of 2048 22 and 26; 256 units of 2048
// 36.7 and 34.8, of 4096 62 and 60.
constexpr int kListWaves = 8;
static int whole_keys(long long units) { return units >= 512 ? 2048 : units >= 128 ? 1024 : 512; }

size_t plan_cache_attend(CacheAttend &a, bool listed) {
    const long long units = (long long)std::min(a.S, kEntries) * a.c.H;
    const int rows = few_rows(a);
    a.many = (long long)a.max_query * a.G > kFewRows;
    a.many_groups = 0;
    if (listed) {
        const int quantum = kListWaves * kStep;
        a.per_unit = (a.max_keys + quantum - 1) / quantum;
        a.whole = a.max_keys <= whole_keys(units) || units >= 256;
        a.few_groups = (int)(a.whole ? units : std::min<long long>(256, units * a.per_unit));
        return a.whole ? 0 : attend_bytes(a.few_groups, rows);
    }
    a.whole = a.max_keys <= whole_keys(units) && !a.many;
    a.per_unit = a.whole ? 1 : 0;
    if (a.whole) {
        a.few_groups = (int)units;
        return 0;
    }
    const long long quanta = ((long long)a.max_keys + kQuantum - 1) / kQuantum * units;
    a.few_groups = (int)std::min<long long>(rows > 16 ? 512 : 768, quanta);
    const long long tiles = ((long long)a.max_query * a.G + kChunkRows - 1) / kChunkRows;
    if (a.many) a.many_groups = (int)std::min<long long>(512, quanta * tiles);
    return std::max(attend_bytes(a.few_groups, rows), attend_bytes(a.many_groups, chunk_rows(a)));
}

// The launches of a call, workgroup by workgroup as the kernels take their pieces, from the lengths on the host.
template <bool LIST, typename F> static void cut_few(const CacheAttend &a, const int *start, const int *len, F put) {
    const int quantum = (LIST ? kListWaves : kWaves) * kStep, rows = few_rows(a);
    const bool even = LIST || a.per_unit > 0;
    const auto unit = [&](int s, int h) {
        return LIST ? Unit<LIST>(a, s, 1 << 30, len[s * a.c.H + h], 0) : Unit<LIST>(a, s, len[s], start[s], start[s + 1]);
    };
    unsigned before[kEntries + 1] = {0};  // quanta before each request
    for (int e = 0; e < a.n_here; ++e)
        before[e + 1] = before[e] + (unsigned)a.c.H * (unsigned)(even ? a.per_unit : few_quanta(a, unit(a.first + e, 0), rows, quantum));
    const unsigned total = before[a.n_here];
    const unsigned launched = a.whole ? a.n_here * a.c.H : a.few_groups;
    const Pieces pieces(total, launched, a.whole);
    if (total == 0) return;
    for (unsigned i = 0; i < pieces.groups && i < launched; ++i)
        for (unsigned now = pieces.begin(i), end = pieces.begin(i + 1), stop; now < end; now = stop) {
            const int entry = (int)(std::upper_bound(before, before + a.n_here + 1, now) - before) - 1;
            const unsigned per = (before[entry + 1] - before[entry]) / a.c.H, h = (now - before[entry]) / per;
            const unsigned u0 = before[entry] + h * per, u1 = u0 + per;
            stop = std::min(u1, end);
            const auto u = unit(a.first + entry, (int)h);
            const int n_rows = u.queries(a) * a.G;
            if (n_rows <= 0 || n_rows > rows) continue;
            const PartKeys keys(a, u, 0, (n_rows - 1) / a.G, quantum, u0, u1, now, stop);
            const bool cut = now > u0 || stop < u1;
            put({a.first, 0, (int)i, a.first + entry, (int)h, 0, n_rows, keys.from, keys.to, (int)u0, (int)u1, (int)now, (int)stop,
                 cut ? (int)record_of(i, now > u0) : -1, now > u0 && stop == u1 ? (int)pieces.owner(u0) : -1});
        }
}
template <typename F> static void cut_many(const CacheAttend &a, const int *start, const int *len, F put) {
    const auto unit = [&](int s) { return Unit<false>(a, s, len[s], start[s], start[s + 1]); };
    unsigned before[kEntries + 1] = {0};
    for (int e = 0; e < a.n_here; ++e) before[e + 1] = before[e] + (unsigned)a.c.H * Chunks(a, unit(a.first + e)).per_head;
    const Pieces pieces(before[a.n_here], a.many_groups, false);
    if (before[a.n_here] == 0) return;
    for (unsigned i = 0; i < pieces.groups && i < (unsigned)a.many_groups; ++i)
        for (unsigned now = pieces.begin(i), end = pieces.begin(i + 1), stop; now < end; now = stop) {
            const int entry = (int)(std::upper_bound(before, before + a.n_here + 1, now) - before) - 1;
            const auto u = unit(a.first + entry);
            const Chunks ch(a, u);
            const unsigned h = (now - before[entry]) / ch.per_head;
            const Chunks::Tile p = ch.at(a, u, before[entry] + h * ch.per_head, now);
            stop = std::min(p.u1, end);
            const int base = kChunkRows * p.tile, n_rows = std::min(ch.n_rows - base, kChunkRows);
            const PartKeys keys(a, u, base / a.G, (base + n_rows - 1) / a.G, kQuantum, p.u0, p.u1, now, stop);
            const bool cut = now > p.u0 || stop < p.u1;
            put({a.first, 1, (int)i, a.first + entry, (int)h, base, n_rows, keys.from, keys.to, (int)p.u0, (int)p.u1, (int)now, (int)stop,
                 cut ? (int)record_of(i, now > p.u0) : -1, now > p.u0 && stop == p.u1 ? (int)pieces.owner(p.u0) : -1});
        }
}
long long cut_cache_attend(CacheAttend a, bool listed, const int *start, const int *len, int *parts, long long most) {
    long long n = 0;
    const auto put = [&](const std::array<int, kCutInts> &part) {
        if (n < most) std::copy(part.begin(), part.end(), parts + n * kCutInts);
        ++n;
    };
    for (a.first = 0; a.first < a.S; a.first += kEntries) {
        a.n_here = std::min(a.S - a.first, kEntries);
        if (listed) cut_few<true>(a, start, len, put);
        else cut_few<false>(a, start, len, put);
        if (a.many) cut_many(a, start, len, put);
    }
    return n;
}

template <int W, bool LIST>
static void launch_few(const CacheAttend &a, hipStream_t stream) {
    const dim3 grid(a.whole ? a.n_here * a.c.H : a.few_groups), block(W * 64);
    if (a.rows == 5) cache_attend_kernel<W, 3, 1, 1, LIST><<<grid, block, 0, stream>>>(a);
    else if (a.rows == 8 && a.out_bf16) cache_attend_kernel<W, 2, 1, 1, LIST><<<grid, block, 0, stream>>>(a);
    else if (a.rows == 8) cache_attend_kernel<W, 2, 1, 2, LIST><<<grid, block, 0, stream>>>(a);
    else if (a.rows == 16 && a.out_bf16) cache_attend_kernel<W, 1, 1, 2, LIST><<<grid, block, 0, stream>>>(a);
    else if (a.rows == 16) cache_attend_kernel<W, 1, 1, 3, LIST><<<grid, block, 0, stream>>>(a);
    else if constexpr (!LIST) {
        if (a.rows == 32 && a.out_bf16) cache_attend_kernel<W, 1, 2, 1, LIST><<<grid, block, 0, stream>>>(a);
        else if (a.rows == 32) cache_attend_kernel<W, 1, 2, 3, LIST><<<grid, block, 0, stream>>>(a);
        else if (a.out_bf16) cache_attend_kernel<W, 1, 3, 1, LIST><<<grid, block, 0, stream>>>(a);
        else cache_attend_kernel<W, 1, 3, 3, LIST><<<grid, block, 0, stream>>>(a);
    }
    if (a.whole) return;
    // threads for four records of a unit at a time: one trip for most
    const int rows = std::min(a.rows, a.max_query * a.G), per_unit = a.few_groups / std::max(1, a.n_here * a.c.H) + 2;
    if (per_unit <= 4) cache_merge_kernel<1><<<dim3(a.few_groups, (rows + 7) / 8), kMergeThreads, 0, stream>>>(a);
    else if (per_unit <= 8) cache_merge_kernel<2><<<dim3(a.few_groups, (rows + 3) / 4), kMergeThreads, 0, stream>>>(a);
    else cache_merge_kernel<8><<<dim3(a.few_groups, rows), kMergeThreads, 0, stream>>>(a);
}

void launch_cache_attend(CacheAttend a, hipStream_t stream) {
    float *const part = a.part;
    for (a.first = 0; a.first < a.S; a.first += kEntries) {
        a.n_here = std::min(a.S - a.first, kEntries);
        a.rows = few_rows(a);
        a.notes = a.whole ? nullptr : (MergeNote *)part;
        a.part = a.whole ? nullptr : (float *)(a.notes + a.few_groups);
        if (a.pos) launch_few<kListWaves, true>(a, stream);
        else launch_few<kWaves, false>(a, stream);
        if (!a.many) continue;
        a.rows = chunk_rows(a);
        a.notes = (MergeNote *)part;
        a.part = (float *)(a.notes + a.many_groups);
        if (a.out_bf16) cache_chunk_kernel<1><<<a.many_groups, kWaves * 64, 0, stream>>>(a);
        else cache_chunk_kernel<3><<<a.many_groups, kWaves * 64, 0, stream>>>(a);
        cache_merge_kernel<1><<<dim3(a.many_groups, (a.rows + kMergeThreads / 32 - 1) / (kMergeThreads / 32)), kMergeThreads, 0, stream>>>(a);
    }
}

}  // namespace ice
