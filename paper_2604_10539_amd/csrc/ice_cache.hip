// The 4-bit sequence cache: block tables and slots of a step, writing rows as codes and scales, reading them back.
#include <algorithm>

#include "ice_cache.h"

namespace ice {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------------------------------------ block tables and slots
// Every workgroup scans all requests (sums of new tokens, blocks taken, blocks given back, kept in LDS) and does its share of the
// rest: a slot, a block taken and a block given back each find their request by bisection and read one id.  A taken block that the
// same call gives back is read from the row it comes from, not from the stack, so nothing waits for anything and the workgroups are
// independent.  Lengths and the stack's height that are updated in place are written last: by the workgroup itself where there is one,
// else by a second launch.  Bound by latency: a trip for the lengths, the scan, the lengths again (a cache's trip), a trip for the ids.
constexpr int kPlanThreads = 1024;           // at most
constexpr int kPlanItems = 4096;             // requests whose lengths fit LDS beside the sums
constexpr unsigned kPlanMost = 0x7FFFFFFFu;  // sums stop here: they only have to be known exactly where the step is possible

enum { kPlanErrFree = 1, kPlanErrRow = 2, kPlanErrSlots = 4, kPlanErrLen = 8 };

struct PlanItem {
    unsigned fresh, take, back;  // new tokens, blocks taken, blocks given back
    int held, need, after, err;  // blocks before the step and after it, length after it
    __device__ PlanItem(const CachePlan &p, int i) : fresh(0), take(0), back(0), held(0), need(0), after(0), err(0) {
        const long long cap = (long long)p.max_blocks << p.block_shift;
        const long long cached = p.cached_len[i], gain = p.new_len[i];
        if (cached < 0 || cached > cap) {
            err = kPlanErrLen;
            return;
        }
        const long long len = max(cached + gain, 0ll), up = (1ll << p.block_shift) - 1;
        if (len > cap) err = kPlanErrRow;
        held = (int)((cached + up) >> p.block_shift);
        need = (int)((len + up) >> p.block_shift);
        fresh = (unsigned)max(gain, 0ll);
        take = (unsigned)max(need - held, 0);
        back = (unsigned)max(held - need, 0);
        after = (int)min(len, (long long)kPlanMost);
    }
};

__device__ inline unsigned sat_add(unsigned a, unsigned b) { return min(a + b, kPlanMost); }

// Index of the last entry of sums[0 .. n] that is at most k < sums[n]: entries that add nothing share a sum with the next.
__device__ inline int plan_owner(const unsigned *sums, int n, unsigned k) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] <= k) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(CachePlan p) {
    extern __shared__ unsigned plan_lds[];
    const int n = p.n_requests, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, threads = blockDim.x, waves = threads >> 6;
    const bool kept = n <= kPlanItems;  // blocks before the step, and lengths after it, stay in LDS
    unsigned *sums[3] = {plan_lds, plan_lds + (n + 1), plan_lds + 2 * (n + 1)};  // before each request: fresh, take, back
    int *s_held = (int *)plan_lds + 3 * (n + 1), *s_after = s_held + n;
    __shared__ unsigned s_wave[kPlanThreads / 64][3];
    __shared__ int s_err;
    if (tid == 0) s_err = 0;
    const int n_free = *p.n_free;
    const int each = (n + threads - 1) / threads, i0 = min(tid * each, n), i1 = min(i0 + each, n);
    unsigned own[3] = {0, 0, 0};
    int err = 0;
    for (int i = i0; i < i1; ++i) {
        const PlanItem x(p, i);
        own[0] = sat_add(own[0], x.fresh);
        own[1] = sat_add(own[1], x.take);
        own[2] = sat_add(own[2], x.back);
        err |= x.err;
        if (kept) {
            s_held[i] = x.held;
            s_after[i] = x.after;
        }
    }
    unsigned v[3] = {own[0], own[1], own[2]}, total[3] = {0, 0, 0};
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const unsigned o = (unsigned)__shfl_up((int)v[k], d);
            if (lane >= d) v[k] = sat_add(v[k], o);
        }
    if (lane == 63)
        for (int k = 0; k < 3; ++k) s_wave[wave][k] = v[k];
    __syncthreads();
    if (err) atomicOr(&s_err, err);
    unsigned at[3];
    for (int k = 0; k < 3; ++k) {
        at[k] = v[k] - min(v[k], own[k]);  // (where a sum stopped at the limit the step is refused and no sum is used)
        for (int w = 0; w < waves; ++w) {
            if (w == wave) at[k] = sat_add(at[k], total[k]);
            total[k] = sat_add(total[k], s_wave[w][k]);
        }
    }
    for (int i = i0; i < i1; ++i) {
        const PlanItem x(p, i);
        const unsigned more[3] = {x.fresh, x.take, x.back};
        for (int k = 0; k < 3; ++k) {
            sums[k][i] = at[k];
            at[k] = sat_add(at[k], more[k]);
        }
    }
    if (tid < 3) sums[tid][n] = total[tid];
    __syncthreads();
    err = s_err;
    const unsigned fresh = total[0], taken = total[1], back = total[2];
    if (n_free < 0 || n_free > p.n_blocks || back > (unsigned)p.n_blocks || n_free + (int)back > p.n_blocks) err |= kPlanErrLen;
    else if (taken > (unsigned)n_free + back) err |= kPlanErrFree;
    if (fresh > (unsigned)p.n_slots) err |= kPlanErrSlots;

    auto held_of = [&](int s) { return kept ? s_held[s] : PlanItem(p, s).held; };
    auto after_of = [&](int s) { return kept ? s_after[s] : PlanItem(p, s).after; };
    auto given_back = [&](unsigned k) {  // id of the k-th block given back
        const int s = plan_owner(sums[2], n, k);
        const int need = (int)(((long long)after_of(s) + (1ll << p.block_shift) - 1) >> p.block_shift);
        return p.table[(size_t)s * p.max_blocks + need + (k - sums[2][s])];
    };
    auto popped = [&](unsigned k) {  // id of the k-th block taken
        const unsigned place = (unsigned)n_free + back - 1 - k;
        return place < (unsigned)n_free ? p.free_ids[place] : given_back(place - (unsigned)n_free);
    };
    const unsigned items = (unsigned)p.n_slots + (err ? 0u : taken + back);
    for (unsigned k = blockIdx.x * threads + tid; k < items; k += gridDim.x * threads) {
        if (k < (unsigned)p.n_slots) {
            int slot = -1;
            if (!err && k < fresh) {
                const int s = plan_owner(sums[0], n, k);
                const int pos = after_of(s) - (int)(sums[0][s + 1] - k), j = pos >> p.block_shift, held = held_of(s);
                const int id = j < held ? p.table[(size_t)s * p.max_blocks + j] : popped(sums[1][s] + (unsigned)(j - held));
                if (id >= 0 && id < p.n_blocks) slot = (id << p.block_shift) + (pos & ((1 << p.block_shift) - 1));
            }
            p.slots[k] = slot;
        } else if (k - p.n_slots < taken) {
            const unsigned t = k - p.n_slots;
            const int s = plan_owner(sums[1], n, t);
            p.table[(size_t)s * p.max_blocks + held_of(s) + (t - sums[1][s])] = popped(t);
        } else {
            const unsigned g = k - p.n_slots - taken;
            p.free_ids[(unsigned)n_free + g] = given_back(g);
        }
    }
    if (blockIdx.x == 0) {
        for (int i = tid; i <= n; i += threads) p.query_start[i] = err ? 0 : (int)sums[0][i];
        if (tid == 0) {
            p.info[0] = err ? 0 : (int)fresh;
            p.info[1] = err ? 0 : (int)taken;
            p.info[2] = err ? 0 : (int)back;
            p.info[3] = err;
        }
        if (!p.end_later) {
            __syncthreads();  // (the lengths have been read)
            for (int i = tid; i < n; i += threads) p.seq_len[i] = err ? p.cached_len[i] : after_of(i);
            if (tid == 0) *p.n_free_left = err ? n_free : n_free + (int)back - (int)taken;
        }
    }
}

__global__ __launch_bounds__(256) void cache_plan_end_kernel(CachePlan p) {
    const int i = blockIdx.x * 256 + threadIdx.x, err = p.info[3];
    if (i < p.n_requests) p.seq_len[i] = err ? p.cached_len[i] : PlanItem(p, i).after;
    if (i == 0) *p.n_free_left = *p.n_free + p.info[2] - p.info[1];
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

// A workgroup's threads for the scan of the lengths (256 requests: 256 threads 5.8 us, 1024 7.3; 512 requests: 512 threads 6.2 us, 1024 8.0; 1000: 6.9
// and 8.6, 256 threads 8 to 10; 2000: 512 threads 8.5 to 10.5, 1024 9.7).  As many workgroups as CUs at most for what the step can
// bring; one where few slots are filled and a second launch would have to write the lengths (one and many, us: 16 requests x 1 token
// 4.4 and 5.8, 512 x 1 5.5 and 7.0, 64 x 16 5.9 and 6.0, 1000 x 1 8.6 and 7.8).
constexpr int kPlanAlone = 512;
void launch_cache_plan(CachePlan p, hipStream_t stream) {
    const long long most = p.n_slots + std::min<long long>((long long)p.n_requests * p.max_blocks, p.n_blocks);
    const bool in_place = p.seq_len == p.cached_len || p.n_free_left == p.n_free;
    const int threads = p.n_requests <= 256 ? 256 : p.n_requests <= 1024 ? 512 : kPlanThreads;
    const int groups = in_place && p.n_slots <= kPlanAlone ? 1 : (int)std::min<long long>(256, (most + threads - 1) / threads);
    const size_t lds = (3 * (p.n_requests + 1) + (p.n_requests <= kPlanItems ? 2 * p.n_requests : 0)) * sizeof(unsigned);
    if (lds > 65536 - 1024) allow_dynamic_lds((const void *)cache_plan_kernel, lds);
    p.end_later = groups > 1 && in_place;
    cache_plan_kernel<<<groups, threads, lds, stream>>>(p);
    if (p.end_later) cache_plan_end_kernel<<<(p.n_requests + 255) / 256, 256, 0, stream>>>(p);
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
