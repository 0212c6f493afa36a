// The 4-bit sequence cache: block tables and slots of a step, writing rows as codes and scales, reading them back.
#include "ice_cache.h"

namespace ice {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------------------------------------ block tables and slots
// One workgroup: requests are scanned 1024 at a time (sums of new tokens, blocks taken and blocks given back), blocks given
// back are pushed on the free stack, then those taken are popped.  Everything is read before anything is written that it
// may share memory with, so lengths and the stack's height may be updated in place.
constexpr int kPlanThreads = 1024;
constexpr unsigned kPlanMost = 0x7FFFFFFFu;  // sums stop here: they only have to be known exactly where the step is possible

enum { kPlanErrFree = 1, kPlanErrRow = 2, kPlanErrSlots = 4, kPlanErrLen = 8 };

struct PlanItem {
    unsigned fresh, take, back;  // new tokens, blocks taken, blocks given back
    int held, err;               // blocks before the step
};

__device__ inline PlanItem plan_item(const CachePlan &p, int i, int &after) {
    PlanItem x = {0, 0, 0, 0, 0};
    after = 0;
    if (i >= p.n_requests) return x;
    const long long cap = (long long)p.max_blocks << p.block_shift;
    const long long cached = p.cached_len[i], gain = p.new_len[i];
    if (cached < 0 || cached > cap) {
        x.err = kPlanErrLen;
        return x;
    }
    const long long len = max(cached + gain, 0ll);
    if (len > cap) x.err = kPlanErrRow;
    const long long up = (1ll << p.block_shift) - 1;
    x.held = (int)((cached + up) >> p.block_shift);
    const int need = (int)((len + up) >> p.block_shift);
    x.fresh = (unsigned)max(gain, 0ll);
    x.take = (unsigned)max(need - x.held, 0);
    x.back = (unsigned)max(x.held - need, 0);
    after = (int)len;
    return x;
}

__device__ inline unsigned sat_add(unsigned a, unsigned b) { return min(a + b, kPlanMost); }

// Exclusive sums of (fresh, take, back) over the workgroup's threads; totals in tot.
__device__ inline void plan_scan(PlanItem &x, unsigned (*sums)[3], unsigned (&tot)[3]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned v[3] = {x.fresh, x.take, x.back};
    const unsigned own[3] = {x.fresh, x.take, x.back};
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const unsigned o = (unsigned)__shfl_up((int)v[k], d);
            if (lane >= d) v[k] = sat_add(v[k], o);
        }
    __syncthreads();  // (the last scan's sums have been read)
    if (lane == 63)
        for (int k = 0; k < 3; ++k) sums[wave][k] = v[k];
    __syncthreads();
    unsigned before[3] = {0, 0, 0};
    for (int k = 0; k < 3; ++k) tot[k] = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w)
        for (int k = 0; k < 3; ++k) {
            if (w == wave) before[k] = tot[k];
            tot[k] = sat_add(tot[k], sums[w][k]);
        }
    // (own is at most the inclusive sum; where that stopped at the limit the step is refused and the sums are not used)
    x.fresh = sat_add(before[0], v[0] - min(v[0], own[0]));
    x.take = sat_add(before[1], v[1] - min(v[1], own[1]));
    x.back = sat_add(before[2], v[2] - min(v[2], own[2]));
}

// Slot of the step's token k, whose request is the last one with start <= k (requests without new tokens share a start).
template <typename Start>
__device__ inline int plan_slot(const CachePlan &p, int k, Start start) {
    if (k >= start(p.n_requests)) return -1;
    int lo = 0, hi = p.n_requests;  // start(lo) <= k < start(hi)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start(mid) <= k) lo = mid;
        else hi = mid;
    }
    const int at = p.seq_len[lo] - (start(lo + 1) - k);
    const int id = p.table[(size_t)lo * p.max_blocks + (at >> p.block_shift)];
    return (id << p.block_shift) + (at & ((1 << p.block_shift) - 1));
}

constexpr int kPlanSlotsHere = 4096;  // so many slots are filled by the planning workgroup itself, without a second launch

__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(CachePlan p) {
    __shared__ unsigned sums[kPlanThreads / 64][3];
    __shared__ int s_err;
    const int tid = threadIdx.x;
    if (tid == 0) s_err = 0;
    const int n_free = *p.n_free;
    const int rounds = (p.n_requests + kPlanThreads - 1) / kPlanThreads;
    unsigned total[3] = {0, 0, 0}, tot[3];
    int err = 0, after;
    __syncthreads();
    for (int r = 0; r < rounds; ++r) {
        PlanItem x = plan_item(p, r * kPlanThreads + tid, after);
        err |= x.err;
        plan_scan(x, sums, tot);
        for (int k = 0; k < 3; ++k) total[k] = sat_add(total[k], tot[k]);
    }
    if (err) atomicOr(&s_err, err);
    __syncthreads();
    err = s_err;
    if (n_free < 0 || n_free > p.n_blocks || total[2] > (unsigned)p.n_blocks || n_free + (int)total[2] > p.n_blocks) err |= kPlanErrLen;
    else if (total[1] > (unsigned)n_free + total[2]) err |= kPlanErrFree;
    if (total[0] > (unsigned)p.n_slots) err |= kPlanErrSlots;
    // a group of threads per request copies its blocks: all of them where there are few requests, a wave where there are many
    const int group = p.n_requests >= 16 ? 64 : p.n_requests >= 4 ? 256 : kPlanThreads;
    const int groups = kPlanThreads / group, mine = tid / group, at = tid % group;
    __shared__ int s_base[kPlanThreads], s_from[kPlanThreads], s_n[kPlanThreads];
    if (!err) {
        const int height = n_free + (int)total[2];
        unsigned done = 0;
        for (int r = 0; total[2] && r < rounds; ++r) {  // pushes
            PlanItem x = plan_item(p, r * kPlanThreads + tid, after);
            const unsigned back = x.back;
            plan_scan(x, sums, tot);
            s_base[tid] = n_free + (int)(done + x.back);
            s_from[tid] = x.held - (int)back;
            s_n[tid] = (int)back;
            __syncthreads();
            for (int i = mine; i < kPlanThreads; i += groups)
                for (int b = at; b < s_n[i]; b += group)
                    p.free_ids[s_base[i] + b] = p.table[(size_t)(r * kPlanThreads + i) * p.max_blocks + s_from[i] + b];
            done += tot[2];
        }
        __threadfence_block();
        __syncthreads();
        unsigned taken = 0, fresh = 0;
        for (int r = 0; r < rounds; ++r) {  // pops, lengths, starts
            const int i0 = r * kPlanThreads + tid;
            PlanItem x = plan_item(p, i0, after);
            const unsigned take = x.take;
            plan_scan(x, sums, tot);
            if (i0 < p.n_requests) {
                p.seq_len[i0] = after;
                p.query_start[i0] = (int)(fresh + x.fresh);
            }
            s_base[tid] = height - 1 - (int)(taken + x.take);
            s_from[tid] = x.held;
            s_n[tid] = (int)take;
            __syncthreads();
            for (int i = mine; i < kPlanThreads; i += groups)
                for (int b = at; b < s_n[i]; b += group)
                    p.table[(size_t)(r * kPlanThreads + i) * p.max_blocks + s_from[i] + b] = p.free_ids[s_base[i] - b];
            taken += tot[1];
            fresh += tot[0];
        }
    } else {
        for (int i = tid; i < p.n_requests; i += kPlanThreads) {
            p.seq_len[i] = p.cached_len[i];
            p.query_start[i] = 0;
        }
        total[0] = total[1] = total[2] = 0;
    }
    if (tid == 0) {
        p.query_start[p.n_requests] = (int)total[0];
        *p.n_free_left = n_free + (int)total[2] - (int)total[1];
        p.info[0] = (int)total[0];
        p.info[1] = (int)total[1];
        p.info[2] = (int)total[2];
        p.info[3] = err;
    }
    if (p.n_slots <= kPlanSlotsHere) {
        __threadfence_block();
        __syncthreads();
        for (int k = tid; k < p.n_slots; k += kPlanThreads) p.slots[k] = plan_slot(p, k, [&](int i) { return p.query_start[i]; });
    }
}

constexpr int kPlanStarts = 4096;  // starts that fit the workgroup's copy

__global__ __launch_bounds__(256) void cache_slots_kernel(CachePlan p) {
    __shared__ int starts[kPlanStarts + 1];
    const bool here = p.n_requests <= kPlanStarts;
    if (here)
        for (int i = threadIdx.x; i <= p.n_requests; i += 256) starts[i] = p.query_start[i];
    __syncthreads();
    const long long k0 = (long long)blockIdx.x * 1024 + threadIdx.x;
    for (int j = 0; j < 4; ++j) {
        const long long k = k0 + 256 * j;
        if (k >= p.n_slots) return;
        p.slots[k] = here ? plan_slot(p, (int)k, [&](int i) { return starts[i]; }) : plan_slot(p, (int)k, [&](int i) { return p.query_start[i]; });
    }
}

// ----------------------------------------------------------------------------------------------------------------- write
// A wave takes 16 tokens of one KV head, keys or values: four rows per load, 16 lanes of 8 values to a row, four lanes to a block
// of 32.  Bound by the read of the rows: 256 bytes in, 68 out.
__global__ __launch_bounds__(256) void cache_write_kernel(CacheDims c, const bf16_t *k, const bf16_t *v, long long k_stride,
                                                          long long v_stride, const int *slots, int n_tokens) {
    const int lane = threadIdx.x & 63, i = lane & 15, r = lane >> 4;
    const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);  // (16 tokens, KV head, side)
    const int side = (int)(unit & 1);
    const long long rest = unit >> 1;
    const int h = (int)(rest % c.H);
    const long long t0 = rest / c.H * 16;
    if (t0 >= n_tokens) return;
    const bf16_t *x = side ? v : k;
    const long long stride = side ? v_stride : k_stride;
    uint4 w[4];
    int slot[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const long long t = t0 + 4 * j + r;
        slot[j] = t < n_tokens ? slots[t] : -1;
        w[j] = make_uint4(0, 0, 0, 0);
        if (t < n_tokens) w[j] = *(const uint4 *)(x + t * stride + h * kD + 8 * i);
    }
    const int tokens_shift = c.tile_shift + 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t d[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
        // largest magnitude of the block: bf16 magnitudes order as their bits
        u16x2 m = __builtin_bit_cast(u16x2, d[0] & 0x7FFF7FFFu);
        for (int e = 1; e < 4; ++e) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, d[e] & 0x7FFF7FFFu));
        uint32_t top = max((uint32_t)m[0], (uint32_t)m[1]);
        top = max(top, dpp_u32<0xB1>(top));
        top = max(top, dpp_u32<0x4E>(top));
        const int exponent = (int)(top >> 7);
        const bool lost = exponent == 255;
        const int scale = lost ? 255 : min(max(exponent - 2 + ((top & 127) > 96 ? 1 : 0), 27), 252);
        const float sf = __uint_as_float((uint32_t)scale << 23);
        uint32_t code = 0;
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2, d[0]), sf, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2, d[1]), sf, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2, d[2]), sf, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2, d[3]), sf, 3);
        if (lost) code = 0;
        const int block = slot[j] >> tokens_shift;
        if (slot[j] < 0 || block >= c.n_blocks) continue;
        const int place = slot[j] & ((16 << c.tile_shift) - 1), t = place & 15;
        uint8_t *tile = c.data + ((((size_t)block * c.H + h) << c.tile_shift) + (place >> 4)) * kCacheTileBytes;
        *(uint32_t *)(tile + kCacheV * side + 64 * t + 4 * i) = code;
        if ((i & 3) == 0) tile[kCacheKS + 64 * side + cache_scale_byte(t, i >> 2)] = (uint8_t)scale;
    }
}

// ------------------------------------------------------------------------------------------------------------------ read
// A wave takes 16 consecutive positions of one (request, KV head), keys or values; 16 lanes to a row.  Bound by the writes.
__global__ __launch_bounds__(256) void cache_read_kernel(CacheDims c, int n_requests, const int *seq_len, const int *table, int max_blocks,
                                                         const int *first, int n_rows, bf16_t *k, bf16_t *v) {
    const int lane = threadIdx.x & 63, i = lane & 15, r = lane >> 4;
    const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int side = (int)(unit & 1);
    const int groups = (n_rows + 15) / 16;
    const long long rest = unit >> 1;
    const long long u = rest / groups;
    if (u >= (long long)n_requests * c.H) return;
    const int s = (int)(u / c.H), h = (int)(u % c.H), row0 = (int)(rest % groups) * 16;
    const long long from = first ? first[s] : 0;
    const long long len = min((long long)seq_len[s], (long long)max_blocks << (c.tile_shift + 4));
    bf16_t *out = (side ? v : k) + u * n_rows * kD;
    uint32_t code[4], scale[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = row0 + 4 * j + r;
        const long long p = from + row;
        code[j] = 0;
        scale[j] = 1;
        if (row < n_rows && p >= 0 && p < len) {
            const int id = table[(size_t)s * max_blocks + (p >> (c.tile_shift + 4))];
            if (id >= 0 && id < c.n_blocks) {
                const int place = (int)p & ((16 << c.tile_shift) - 1), t = place & 15;
                const uint8_t *tile = c.data + ((((size_t)id * c.H + h) << c.tile_shift) + (place >> 4)) * kCacheTileBytes;
                code[j] = *(const uint32_t *)(tile + kCacheV * side + 64 * t + 4 * i);
                scale[j] = tile[kCacheKS + 64 * side + cache_scale_byte(t, i >> 2)];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = row0 + 4 * j + r;
        if (row >= n_rows) continue;
        const float sf = __uint_as_float(scale[j] << 23);
        uint4 w;
        w.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[j], sf, 0));
        w.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[j], sf, 1));
        w.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[j], sf, 2));
        w.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[j], sf, 3));
        if (scale[j] == 255) w = make_uint4(0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u);
        *(uint4 *)(out + (size_t)row * kD + 8 * i) = w;
    }
}

}  // namespace

void launch_cache_plan(const CachePlan &p, hipStream_t stream) {
    cache_plan_kernel<<<1, kPlanThreads, 0, stream>>>(p);
    if (p.n_slots > kPlanSlotsHere) cache_slots_kernel<<<(p.n_slots + 1023) / 1024, 256, 0, stream>>>(p);
}

void launch_cache_write(const CacheDims &c, const bf16_t *k, const bf16_t *v, long long k_stride, long long v_stride, const int *slots,
                        int n_tokens, hipStream_t stream) {
    const long long units = ((long long)n_tokens + 15) / 16 * c.H * 2;
    cache_write_kernel<<<(unsigned)((units + 3) / 4), 256, 0, stream>>>(c, k, v, k_stride, v_stride, slots, n_tokens);
}

void launch_cache_read(const CacheDims &c, int n_requests, const int *seq_len, const int *table, int max_blocks, const int *first,
                       int n_rows, bf16_t *k, bf16_t *v, hipStream_t stream) {
    const long long units = ((long long)n_rows + 15) / 16 * n_requests * c.H * 2;
    cache_read_kernel<<<(unsigned)((units + 3) / 4), 256, 0, stream>>>(c, n_requests, seq_len, table, max_blocks, first, n_rows, k, v);
}

}  // namespace ice
