// What requests of the 4-bit sequence cache share: the step's queries sorted by source, attention to all tokens of a source, and attention of
// requests behind one.
#include <algorithm>

#include "ice_cache_attend.h"

namespace ice {

namespace {

// ------------------------------------------------------------------------------------------------------------ sorted queries
// Where a request's queries stand in the list is the number of those with a lower source, or the same one and a lower request.  A wave counts
// them for a request, and for a row of the table those with a lower source, over all requests in LDS; so no workgroup waits for another and the order is
// always the same.
constexpr int kSourceThreads = 1024, kSourceShare = 64;  // requests of a workgroup at most
__global__ __launch_bounds__(kSourceThreads) void plan_sources_kernel(CacheSources p, int share, int row_share) {
    extern __shared__ int sources_lds[];
    const int n = p.n_requests, rows = p.n_rows, T = p.n_tokens, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int *s_to = sources_lds, *s_many = sources_lds + n, *s_place = sources_lds + 2 * n;
    __shared__ unsigned s_at[kSourceShare], s_total;
    int *start = p.plan, *lowest = p.plan + rows + 2, *token = p.plan + 2 * rows + 2, *place = token + T;
    if (tid == 0) s_total = 0;
    __syncthreads();
    unsigned total = 0;
    for (int s = tid; s < n; s += kSourceThreads) {
        const int from = min(max(p.query_start[s], 0), T), many = min(max(p.query_start[s + 1], from), T) - from, to = p.source[s];
        s_to[s] = (unsigned)to >= (unsigned)rows || (p.seq_len && to == s) ? rows : to;
        s_many[s] = many;
        s_place[s] = p.seq_len ? (int)((unsigned)max(p.seq_len[s], 0) - (unsigned)many) : 0;
        total += (unsigned)many;
    }
    if (total) atomicAdd(&s_total, total);
    __syncthreads();
    const int r0 = min((int)blockIdx.x * share, n), r1 = min(r0 + share, n);
    const int g0 = min((int)blockIdx.x * row_share, rows + 2), g1 = min(g0 + row_share, rows + 2);
    for (int item = wave; item < r1 - r0 + g1 - g0; item += kSourceThreads / 64) {
        const bool request = item < r1 - r0;
        const int s = r0 + item, g = request ? s_to[s] : g0 + item - (r1 - r0), before = request ? s : 0;
        unsigned sum = 0;
        int least = 0x7FFFFFFF;
        for (int e = lane; e < n; e += 64) {
            const int to = s_to[e], many = s_many[e];
            if (to < g || (to == g && e < before)) sum += (unsigned)many;
            if (to == g && many > 0) least = min(least, s_place[e]);
        }
        sum = (unsigned)wave_scan_add((int)sum);
        if (request) {
            if (lane == 63) s_at[item] = sum;
            continue;
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) least = min(least, __shfl_xor(least, d));
        if (lane == 63) {
            start[g] = (int)min(sum, (unsigned)T);
            if (g < rows) lowest[g] = least;
        }
    }
    __syncthreads();
    for (int s = r0; s < r1; ++s) {
        const int from = min(max(p.query_start[s], 0), T), many = s_many[s];
        for (int j = tid; j < many; j += kSourceThreads) {
            const unsigned at = s_at[s - r0] + (unsigned)j;
            if (at >= (unsigned)T) break;
            token[at] = from + j;
            place[at] = p.seq_len ? (int)((unsigned)s_place[s] + (unsigned)j) : 0;
        }
    }
    for (long long e = (long long)min(s_total, (unsigned)T) + (long long)blockIdx.x * kSourceThreads + tid; e < T; e += (long long)gridDim.x * kSourceThreads)
        token[e] = place[e] = -1;
}

}  // namespace

void launch_plan_sources(const CacheSources &p, hipStream_t stream) {
    const int items = p.n_requests + p.n_rows + 2;
    const int groups = std::min(256, (items + 15) / 16);
    const size_t lds = 3 * (size_t)p.n_requests * sizeof(int);
    if (lds > 65536 - 1024) allow_dynamic_lds((const void *)plan_sources_kernel, lds);
    plan_sources_kernel<<<groups, kSourceThreads, lds, stream>>>(p, (p.n_requests + groups - 1) / groups, (p.n_rows + 2 + groups - 1) / groups);
}

// ------------------------------------------------------------------------------------------------------------------ attention
static size_t note_bytes(const CacheAttend &a) { return 2 * (size_t)a.T * a.c.H * sizeof(TokenNote); }
static size_t state_bytes(const CacheAttend &a) { return 2 * (size_t)a.T * a.c.H * a.G * kRecord * sizeof(float); }

size_t plan_cache_shared(CacheAttend &a, int max_source) {
    const long long most = std::max(a.max_query, a.max_shared), tile = kChunkRows / a.G;
    a.many = most * a.G > kFewRows;
    CacheAttend rows = a;
    rows.max_query = (int)most;
    a.rows = a.many ? (int)std::min<long long>(tile, most) * a.G : few_rows(rows);
    const auto quanta = [&](int keys, long long queries) { return ((long long)keys + kQuantum - 1) / kQuantum * (a.many ? (queries + tile - 1) / tile : 1); };
    const double all = (double)a.c.H * ((double)a.S * quanta(a.max_keys, a.max_query) + quanta(max_source, a.max_shared));
    a.groups = (int)std::min<double>(a.rows > kRows ? 512 : 768, all);
    return note_bytes(a) + state_bytes(a) + (size_t)a.groups * 2 * a.rows * kRecord * sizeof(float);
}

long long cut_cache_cross(CacheAttend a, const int *start, const int *len, int *parts, long long most) { return cut_attend<kCross>(a, start, len, parts, most); }
long long cut_cache_shared(const CacheAttend &a, int *parts, long long most) { return cut_attend<kBoth>(a, nullptr, nullptr, parts, most); }

void launch_cache_cross(const CacheAttend &a, hipStream_t stream) { launch_attend<kCross>(a, stream); }

constexpr long long kJoinRows = 4096;  // rows whose sums are joined by many threads each: few rows have many records
static void launch_both(const CacheAttend &a, hipStream_t stream) {
    if (!a.many) launch_few<kWaves, kBoth>(a, stream);
    else launch_chunks<kBoth>(a, a.groups, stream);
    const unsigned units = (unsigned)a.T * (unsigned)a.c.H;
    if ((long long)units * a.G <= kJoinRows) cache_join_kernel<8><<<dim3(units, a.G), kMergeThreads, 0, stream>>>(a);
    else cache_join_kernel<2><<<dim3(units, (a.G + 3) / 4), kMergeThreads, 0, stream>>>(a);
}

void launch_cache_shared(CacheAttend a, void *workspace, hipStream_t stream) {
    a.token_notes = static_cast<TokenNote *>(workspace);
    a.state = reinterpret_cast<float *>(static_cast<char *>(workspace) + note_bytes(a));
    a.part = a.state + state_bytes(a) / sizeof(float);
    launch_both(a, stream);
}

}  // namespace ice
