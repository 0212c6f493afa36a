// Attention over the 4-bit sequence cache.
#include <algorithm>

#include "ice_cache.h"

namespace ice {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8;      // of a workgroup
constexpr int kStep = 32;      // keys per step of a wave
constexpr int kRows = 16;      // query rows (token, head of the group) of a workgroup
constexpr int kRecord = 132;   // floats per row of a share's partial result: 128 sums, maximum, denominator
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

// Where a request's queries and keys lie.
struct Span {
    int row0, n_query, len;  // first query row, queries, cached tokens
    __device__ Span(const CacheAttend &a, int s) {
        row0 = min(max(a.query_start[s], 0), a.T);
        n_query = min(max(a.query_start[s + 1], row0), a.T) - row0;
        len = max(a.seq_len[s], 0);
        len = (int)min((long long)len, (long long)a.max_blocks << (a.c.tile_shift + 4));
    }
    // keys [low, high) that query t sees
    __device__ int high(int t) const { return max(len - n_query + t + 1, 0); }
    __device__ int low(const CacheAttend &a, int t) const { return a.window > 0 ? max(high(t) - a.window, 0) : 0; }
};

// What a wave holds of 32 keys: two tiles of 16.  Key codes: lane (g, c) has dims [32 g, 32 g + 32) of the token that is
// row c of the product's left operand.  Value codes: lane (g, c) has dims [8 c, 8 c + 8) of tokens g, 4 + g, 8 + g, 12 + g.
struct Keys {
    u32x4 k[2], v[2];
    uint32_t ks[2], vs[2];
};

// One workgroup: 16 query rows of one (request, KV head) against one share of its keys.
//
// S^T = K Q^T puts a row's scores on one lane (g, c): head row c, tokens 4 i + g of each tile; these registers are the
// right operand of O^T = V^T P^T as they are (contraction slot 8 g + 4 tile + i), and a row's sums come out on the lanes that hold its
// softmax, so that neither the weights nor the rescaling cross lanes.  Codes become bf16 in registers, without rounding (three
// significant bits at most).  The weights are split into TERMS bf16 terms whose products add up in fp32: three carry all of a float32
// weight (float32 outputs), two 16 bits of it.
template <int TERMS, bool LIST>
__global__ __launch_bounds__(kWaves * 64) void cache_attend_kernel(CacheAttend a) {
    __shared__ float s_acc[kWaves][kRows][kRecord];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
    unsigned at = blockIdx.x;
    const int share = (int)(at % (unsigned)a.n_chunks);
    at /= (unsigned)a.n_chunks;
    const int rt = (int)(at % (unsigned)a.row_tiles);
    at /= (unsigned)a.row_tiles;
    const int h = (int)(at % (unsigned)a.c.H), s = (int)(at / (unsigned)a.c.H);

    // rows of this workgroup and the keys they see
    int row0, n_rows, low, high, len;  // low, high: of this lane's row c
    int from, to;                      // keys that any row sees, inside this share
    int all_low, all_high;             // keys that every row sees
    if constexpr (LIST) {
        row0 = s;
        n_rows = a.G;
        len = min(max(a.seq_len[s], 0), (int)min((long long)a.max_blocks << (a.c.tile_shift + 4), 0x7FFFFFFFll));
        low = 0;
        high = min(max(a.n_tok[s * a.c.H + h], 0), a.max_keys);
        from = all_low = 0;
        to = all_high = high;
    } else {
        const Span span(a, s);
        const int total = min(span.n_query, a.max_query) * a.G;
        n_rows = min(total - kRows * rt, kRows);
        if (n_rows <= 0) return;
        row0 = span.row0;
        len = span.len;
        const int t_first = kRows * rt / a.G, t_last = (kRows * rt + n_rows - 1) / a.G, t = (kRows * rt + min(c, n_rows - 1)) / a.G;
        low = span.low(a, t);
        high = span.high(t);
        from = span.low(a, t_first);
        to = span.high(t_last);
        all_low = span.low(a, t_last);
        all_high = span.high(t_first);
    }
    const bool whole = a.n_chunks == 1;
    {
        const int begin = share * a.chunk;
        const bool last = share == a.n_chunks - 1;
        from = max(from, begin);
        if (!last) to = min(to, begin + a.chunk);
    }
    if (from >= to && !whole) return;  // (the merge knows which shares are empty)

    // query rows: right operand of step j holds dims 32 g + 8 j .. + 8 of row c
    u32x4 qv[4];
    {
        const int row = kRows * rt + min(c, n_rows - 1), t = row / a.G;
        const bf16_t *p = a.q + (long long)(row0 + t) * a.q_stride + (long long)(h * a.G + row % a.G) * kD + 32 * g;
#pragma unroll
        for (int j = 0; j < 4; ++j) qv[j] = *(const u32x4 *)(p + 8 * j);
    }
    const int tiles_mask = (1 << a.c.tile_shift) - 1;
    const int step0 = from / kStep, steps = (to + kStep - 1) / kStep;  // steps of 32 keys: [step0, steps)
    const int k_row = 4 * (c & 3) + (c >> 2);                          // token that is row c of the key operand: row 4 g + i is token 4 i + g
    const uint32_t k_at = 64 * k_row + 16 * g, ks_at = kCacheKS + cache_scale_byte(k_row, g);
    const uint32_t v_at = kCacheV + 64 * g + 4 * c, vs_at = kCacheVS + 16 * g + 4 * (c >> 2);
    const int *table = a.table + (size_t)s * a.max_blocks;
    const int *list = LIST ? a.pos + ((size_t)s * a.c.H + h) * a.max_keys : nullptr;

    // Up to 64 places on the lanes.  Dense: index of tile l & 1 of the wave's step n0 + l / 2, in units of tiles of the pool.  Listed:
    // index of key l & 31 of step n0 + l / 32, in units of rows of the pool.  -1: no such place.
    auto places = [&](int n0) -> int {
        if constexpr (LIST) {
            const long long e = (long long)(step0 + wave + kWaves * (n0 + (lane >> 5))) * kStep + (lane & 31);
            if (e >= to) return -1;
            const int p = list[e];
            if (p < 0 || p >= len) return -1;
            const int id = table[p >> (a.c.tile_shift + 4)];
            if (id < 0 || id >= a.c.n_blocks) return -1;
            return (int)(((((unsigned)id * a.c.H + h) << a.c.tile_shift) + ((p >> 4) & tiles_mask)) * 16u + (p & 15));
        } else {
            const int tile = (step0 + wave + kWaves * (n0 + (lane >> 1))) * 2 + (lane & 1);
            if (tile * 16 >= to) return -1;
            const int id = table[tile >> a.c.tile_shift];
            if (id < 0 || id >= a.c.n_blocks) return -1;
            return (int)((((unsigned)id * a.c.H + h) << a.c.tile_shift) + (tile & tiles_mask));
        }
    };
    constexpr int kAhead = LIST ? 2 : 32;  // steps whose places lie on the lanes
    // requests step n (of this wave); bad: tokens of the step that do not exist, one bit each
    auto request = [&](int held, int n, Keys &x, uint32_t &bad) {
        bad = 0;
        if constexpr (LIST) {
            bad = (uint32_t)(__ballot(held == -1) >> (32 * (n & 1)));
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint32_t kr = (uint32_t)max(__shfl(held, 32 * (n & 1) + 16 * b + k_row), 0);
                const uint8_t *kt = a.c.data + (size_t)(kr >> 4) * kCacheTileBytes;
                x.k[b] = *(const u32x4 *)(kt + 64 * (kr & 15) + 16 * g);
                x.ks[b] = kt[kCacheKS + cache_scale_byte(kr & 15, g)];
                uint32_t sc = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t vr = (uint32_t)max(__shfl(held, 32 * (n & 1) + 16 * b + 4 * i + g), 0);
                    const uint8_t *vt = a.c.data + (size_t)(vr >> 4) * kCacheTileBytes;
                    x.v[b][i] = *(const uint32_t *)(vt + kCacheV + 64 * (vr & 15) + 4 * c);
                    sc |= (uint32_t)vt[kCacheVS + cache_scale_byte(vr & 15, c >> 2)] << (8 * i);
                }
                x.vs[b] = sc;
            }
        } else {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int id = __builtin_amdgcn_readlane(held, 2 * (n % kAhead) + b);
                if (id < 0) bad |= 0xFFFFu << (16 * b);
                const uint8_t *t = a.c.data + (size_t)max(id, 0) * kCacheTileBytes;
                x.k[b] = __builtin_nontemporal_load((const u32x4 *)(t + k_at));
#pragma unroll
                for (int i = 0; i < 4; ++i) x.v[b][i] = __builtin_nontemporal_load((const uint32_t *)(t + v_at + 256 * i));
                x.ks[b] = t[ks_at];
                x.vs[b] = *(const uint32_t *)(t + vs_at);
            }
        }
    };

    f32x4 acc[8];  // acc[j][i]: dim 32 g + 8 i + j of row c
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kNoMax, l = 0.f;
    const int n_mine = steps - step0 - wave > 0 ? (steps - step0 - wave + kWaves - 1) / kWaves : 0;
    int held = n_mine > 0 ? places(0) : -1;
    Keys x, y;
    uint32_t bad_x = 0, bad_y = 0;
    if (n_mine > 0) request(held, 0, x, bad_x);
    for (int n = 0; n < n_mine; ++n) {
        if (n + 1 < n_mine) {
            if ((n + 1) % kAhead == 0) held = places(n + 1);
            request(held, n + 1, y, bad_y);
        }
        const int key0 = (step0 + wave + kWaves * n) * kStep;
        f32x4 d[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const float sc = __uint_as_float(x.ks[b] << 23);
            d[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4; ++j) d[b] = mfma(eight(x.k[b][j], sc), qv[j], d[b]);
        }
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = d[e >> 2][e & 3] * a.scale_log2;
        const bool edge = key0 < max(all_low, from) || key0 + kStep > min(all_high, to) || bad_x != 0;
        if (edge) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int in = 16 * (e >> 2) + 4 * (e & 3) + g, key = key0 + in;
                const bool gone = (bad_x >> in) & 1;
                if (gone || key < max(low, from) || key >= min(high, to)) p[e] = -INFINITY;
                // what no row sees may hold anything: its value scale must not turn a weight of 0 into NaN
                if (gone || key < from || key >= to) x.vs[e >> 2] &= ~(0xFFu << (8 * (e & 3)));
            }
        }
        float top = fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7])));
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
            p[e] = __builtin_amdgcn_exp2f(p[e] - m);
            l += p[e];
        }
        if (!LIST && edge) {
            // A value block that is held as NaN makes the outputs of the rows that see it NaN, and of no other row: its weight
            // of 0 in the others would.  Rare: found by a scan of the step's scales, taken out of the product.
            bool nan = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) nan |= ((x.vs[e >> 2] >> (8 * (e & 3))) & 0xFF) == 0xFF;
            if (__any(nan)) {
                for (int in = 0; in < kStep; ++in) {
                    const int key = key0 + in;
                    const int blk = table[key >> (a.c.tile_shift + 4)];
                    if (key >= min(high, to) || key < max(low, from) || blk < 0 || blk >= a.c.n_blocks) continue;
                    const uint8_t *t = a.c.data + (((((size_t)blk * a.c.H + h) << a.c.tile_shift) + ((key >> 4) & tiles_mask))) * kCacheTileBytes;
                    if (t[kCacheVS + cache_scale_byte(key & 15, g)] == 255)
#pragma unroll
                        for (int j = 0; j < 8; ++j) acc[j] += __builtin_nanf("");
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (((x.vs[e >> 2] >> (8 * (e & 3))) & 0xFF) == 0xFF) x.vs[e >> 2] &= ~(0xFFu << (8 * (e & 3)));
            }
        }
        // weights in terms
        u32x4 w[TERMS];
#pragma unroll
        for (int t = 0; t < TERMS; ++t)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const uint32_t two = pack2(p[e], p[e + 1]);
                w[t][e >> 1] = two;
                if (t + 1 < TERMS) {
                    p[e] -= bf16_lo(two);
                    p[e + 1] -= bf16_hi(two);
                }
            }
        // values: pairs of dims of a token, then pairs of tokens of a dim
        u32x4 va[8];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const int b = e >> 2, i = e & 3;
            const float s0 = __uint_as_float(((x.vs[b] >> (8 * i)) & 0xFF) << 23), s1 = __uint_as_float(((x.vs[b] >> (8 * i + 8)) & 0xFF) << 23);
            const u32x4 r0 = eight(x.v[b][i], s0), r1 = eight(x.v[b][i + 1], s1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                va[2 * j][e >> 1] = __builtin_amdgcn_perm(r1[j], r0[j], 0x05040100u);
                va[2 * j + 1][e >> 1] = __builtin_amdgcn_perm(r1[j], r0[j], 0x07060302u);
            }
        }
#pragma unroll
        for (int t = 0; t < TERMS; ++t)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] = mfma(va[j], w[t], acc[j]);
        x = y;
        bad_x = bad_y;
    }

    // the waves' sums meet in LDS
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (c < n_rows) {
        float *r = s_acc[wave][c];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            *(f32x4 *)(r + 32 * g + 8 * i) = f32x4{acc[0][i], acc[1][i], acc[2][i], acc[3][i]};
            *(f32x4 *)(r + 32 * g + 8 * i + 4) = f32x4{acc[4][i], acc[5][i], acc[6][i], acc[7][i]};
        }
        if (g == 0) {
            r[kD] = m;
            r[kD + 1] = l;
        }
    }
    __syncthreads();
    const int row = tid >> 5, d0 = 4 * (tid & 31);  // 32 threads to a row, four dims each
    if (row >= n_rows) return;
    float top = kNoMax;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_acc[w][row][kD]);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(s_acc[w][row][kD] - top);
        sum += *(const f32x4 *)(s_acc[w][row] + d0) * f;
        total += s_acc[w][row][kD + 1] * f;
    }
    if (!whole) {
        float *r = a.part + ((((size_t)(s * a.c.H + h) * a.row_tiles + rt) * a.n_chunks + share) * kRows + row) * kRecord;
        *(f32x4 *)(r + d0) = sum;
        if (d0 == 0) {
            r[kD] = top;
            r[kD + 1] = total;
        }
        return;
    }
    const int t_r = LIST ? 0 : (kRows * rt + row) / a.G;
    const int head = h * a.G + (kRows * rt + row) % a.G;
    const size_t o = ((size_t)(row0 + t_r) * a.c.H * a.G + head);
    const bool none = total == 0.f;  // no key at all: the largest of any weights is 1 or more
    sum = none ? f32x4{0.f, 0.f, 0.f, 0.f} : sum * (1.f / total);
    if (a.out_bf16) {
        uint2 w = {pack2(sum[0], sum[1]), pack2(sum[2], sum[3])};
        *(uint2 *)((bf16_t *)a.out + o * kD + d0) = w;
    } else {
        *(f32x4 *)((float *)a.out + o * kD + d0) = sum;
    }
    if (a.lse && d0 == 0) a.lse[o] = none ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
}

// Joins the shares of a call that was cut along the keys: 32 threads to a row.
template <bool LIST>
__global__ __launch_bounds__(256) void cache_merge_kernel(CacheAttend a) {
    const int row = threadIdx.x >> 5, d0 = 4 * (threadIdx.x & 31);
    unsigned at = blockIdx.x;
    const int half = (int)(at & 1);
    at >>= 1;
    const int rt = (int)(at % (unsigned)a.row_tiles);
    at /= (unsigned)a.row_tiles;
    const int h = (int)(at % (unsigned)a.c.H), s = (int)(at / (unsigned)a.c.H);
    const int r = 8 * half + row, in = kRows * rt + r;
    int row0, t, from, to;
    if constexpr (LIST) {
        if (r >= a.G) return;
        row0 = s;
        t = 0;
        from = 0;
        to = min(max(a.n_tok[s * a.c.H + h], 0), a.max_keys);
    } else {
        const Span span(a, s);
        const int total = min(span.n_query, a.max_query) * a.G, n_rows = min(total - kRows * rt, kRows);
        if (r >= n_rows) return;
        row0 = span.row0;
        t = in / a.G;
        from = span.low(a, kRows * rt / a.G);
        to = span.high((kRows * rt + n_rows - 1) / a.G);
    }
    const float *p = a.part + (((size_t)(s * a.c.H + h) * a.row_tiles + rt) * a.n_chunks * kRows + r) * kRecord;
    const int c0 = min(from / a.chunk, a.n_chunks - 1), c1 = from < to ? min((to + a.chunk - 1) / a.chunk, a.n_chunks) : 0;
    float top = kNoMax, total = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int c = c0; c < c1; ++c) {
        const float *x = p + (size_t)c * kRows * kRecord;
        const float m = x[kD], mn = fmaxf(top, m), f0 = __builtin_amdgcn_exp2f(top - mn), f1 = __builtin_amdgcn_exp2f(m - mn);
        sum = sum * f0 + *(const f32x4 *)(x + d0) * f1;
        total = total * f0 + x[kD + 1] * f1;
        top = mn;
    }
    const bool none = total == 0.f;
    const size_t o = (size_t)(row0 + t) * a.c.H * a.G + h * a.G + in % a.G;
    sum = none ? f32x4{0.f, 0.f, 0.f, 0.f} : sum * (1.f / total);
    if (a.out_bf16) {
        uint2 w = {pack2(sum[0], sum[1]), pack2(sum[2], sum[3])};
        *(uint2 *)((bf16_t *)a.out + o * kD + d0) = w;
    } else {
        *(f32x4 *)((float *)a.out + o * kD + d0) = sum;
    }
    if (a.lse && d0 == 0) a.lse[o] = none ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
}

}  // namespace

size_t plan_cache_attend(CacheAttend &a) {
    const int rows = a.max_query * a.G;
    a.row_tiles = (rows + kRows - 1) / kRows;
    const long long units = (long long)a.S * a.c.H * a.row_tiles;
    const int quantum = kWaves * kStep;  // keys of one step of all waves
    const long long most = std::max(1, (a.max_keys + quantum - 1) / quantum);
    const long long want = std::min(most, std::max(1ll, 1024 / units));
    a.chunk = (int)((most + want - 1) / want) * quantum;
    a.n_chunks = (int)((most * quantum + a.chunk - 1) / a.chunk);
    return a.n_chunks > 1 ? (size_t)units * a.n_chunks * kRows * kRecord * 4 : 0;
}

void launch_cache_attend(const CacheAttend &a, hipStream_t stream) {
    const unsigned units = (unsigned)a.S * a.c.H * a.row_tiles;
    if (a.pos) {
        cache_attend_kernel<3, true><<<units * a.n_chunks, kWaves * 64, 0, stream>>>(a);
        if (a.n_chunks > 1) cache_merge_kernel<true><<<units * 2, 256, 0, stream>>>(a);
    } else {
        if (a.out_bf16) cache_attend_kernel<2, false><<<units * a.n_chunks, kWaves * 64, 0, stream>>>(a);
        else cache_attend_kernel<3, false><<<units * a.n_chunks, kWaves * 64, 0, stream>>>(a);
        if (a.n_chunks > 1) cache_merge_kernel<false><<<units * 2, 256, 0, stream>>>(a);
    }
}

}  // namespace ice
