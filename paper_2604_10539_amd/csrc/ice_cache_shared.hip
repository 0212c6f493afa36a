// What requests of the 4-bit sequence cache share: the step's queries sorted by source, attention to all tokens of a source, and attention of
// requests behind one.
#include <algorithm>

#include "ice_cache_attend.h"

namespace ice {

namespace {

// ------------------------------------------------------------------------------------------------------------ sorted queries
// Every workgroup counts all requests' queries by row of the table in LDS (whole numbers: the order of the additions does not matter), those of the requests
// before its own share apart, and sums them up; so it knows where the queries of its requests stand, no workgroup waits for another, and the order is always the
// same.  Bound by latency: a trip for the requests' words, the counts (a lane at a time where requests share a row), the sums, the stores.
// 34 rows 4.4 us, 2000 requests with 217 K queries 7.1, 8000 requests of 40 sources 14 (a wave that counted the requests in front of each: 13.2 and 84).
constexpr int kSourceThreads = 1024, kSourceShare = 64;  // of a workgroup, and requests of one, at most
__global__ __launch_bounds__(kSourceThreads) void plan_sources_kernel(CacheSources p, int share, int row_share) {
    extern __shared__ unsigned sources_lds[];
    const int n = p.n_requests, rows = p.n_rows, T = p.n_tokens, threads = blockDim.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = threads >> 6;
    unsigned *before = sources_lds, *begin = before + rows + 1;  // queries of the requests before this share; all others, later where a row's queries begin
    int *least = (int *)(begin + rows + 1);
    __shared__ unsigned s_wave[kSourceThreads / 64], s_total, s_at[kSourceShare];
    __shared__ int s_from[kSourceShare], s_to[kSourceShare], s_many[kSourceShare], s_place[kSourceShare];
    const int r0 = min((int)blockIdx.x * share, n), r1 = min(r0 + share, n);
    int *start = p.plan, *lowest = p.plan + rows + 2, *token = p.plan + 2 * rows + 2, *place = token + T;
    for (int g = tid; g <= rows; g += threads) {
        before[g] = begin[g] = 0;
        if (g < rows) least[g] = 0x7FFFFFFF;
    }
    constexpr int kTogether = 4;  // requests whose words a thread asks for side by side
    for (int s0 = tid; s0 - tid < n; s0 += kTogether * threads) {
        int x[kTogether], y[kTogether], named[kTogether], len[kTogether];
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
            const int s = min(s0 + k * threads, n - 1);
            x[k] = p.query_start[s];
            y[k] = p.query_start[s + 1];
            named[k] = p.source[s];
            len[k] = p.seq_len ? p.seq_len[s] : 0;
        }
        if (s0 == tid) __syncthreads();  // (the counts are 0)
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
            const int s = s0 + k * threads;
            if (s >= n) break;
            const int from = min(max(x[k], 0), T), many = min(max(y[k], from), T) - from;
            const int to = (unsigned)named[k] >= (unsigned)rows || (p.seq_len && named[k] == s) ? rows : named[k];
            const int at = p.seq_len ? (int)((unsigned)max(len[k], 0) - (unsigned)many) : 0;
            if (many > 0) {
                atomicAdd((s < r0 ? before : begin) + to, (unsigned)many);
                if (to < rows) atomicMin(least + to, at);
            }
            if (s >= r0 && s < r1) {
                s_from[s - r0] = from;
                s_to[s - r0] = to;
                s_many[s - r0] = many;
                s_place[s - r0] = at;
            }
        }
    }
    __syncthreads();
    const int each = (rows + threads) / threads, g0 = min(tid * each, rows + 1), g1 = min(g0 + each, rows + 1);
    unsigned own = 0;
    for (int g = g0; g < g1; ++g) own += before[g] + begin[g];
    const unsigned incl = (unsigned)wave_scan_add((int)own);
    if (lane == 63) s_wave[wave] = incl;
    __syncthreads();
    unsigned at = incl - own;
    for (int w = 0; w < wave; ++w) at += s_wave[w];
    for (int g = g0; g < g1; ++g) {
        const unsigned here = before[g] + begin[g];
        begin[g] = at;
        at += here;
    }
    if (tid == threads - 1) s_total = at;
    __syncthreads();
    for (int s = r0 + wave; s < r1; s += waves) {  // (a share is no longer than a wave)
        const int to = s_to[s - r0];
        const bool same = lane < s - r0 && s_to[lane] == to;
        const unsigned sum = (unsigned)wave_scan_add(same ? s_many[lane] : 0);
        if (lane == 63) s_at[s - r0] = begin[to] + before[to] + sum;
    }
    for (int g = min((int)blockIdx.x * row_share, rows + 2) + tid; g < min(((int)blockIdx.x + 1) * row_share, rows + 2); g += threads) {
        start[g] = (int)min(g <= rows ? begin[g] : s_total, (unsigned)T);
        if (g < rows) lowest[g] = least[g];
    }
    __syncthreads();
    // a wave to a request, but all of them to one of many queries
    auto put = [&](int s, int from, int step) {
        for (int j = from; j < s_many[s]; j += step) {
            const unsigned e = s_at[s] + (unsigned)j;
            if (e >= (unsigned)T) break;
            token[e] = s_from[s] + j;
            place[e] = p.seq_len ? (int)((unsigned)s_place[s] + (unsigned)j) : 0;
        }
    };
    for (int s = wave; s < r1 - r0; s += waves)
        if (s_many[s] <= kSourceThreads) put(s, lane, 64);
    for (int s = 0; s < r1 - r0; ++s)
        if (s_many[s] > kSourceThreads) put(s, tid, threads);
    for (long long e = (long long)min(s_total, (unsigned)T) + (long long)blockIdx.x * threads + tid; e < T; e += (long long)gridDim.x * threads)
        token[e] = place[e] = -1;
}

}  // namespace

void launch_plan_sources(const CacheSources &p, hipStream_t stream) {
    const int threads = p.n_requests <= 256 ? 256 : kSourceThreads;
    const int groups = std::min(256, (std::max(p.n_requests, p.n_rows + 2) + threads / 64 - 1) / (threads / 64));
    const size_t lds = (3 * (size_t)p.n_rows + 2) * sizeof(int);
    if (lds > 65536 - 4096) allow_dynamic_lds((const void *)plan_sources_kernel, lds);
    plan_sources_kernel<<<groups, threads, lds, stream>>>(p, (p.n_requests + groups - 1) / groups, (p.n_rows + 2 + groups - 1) / groups);
}

// ------------------------------------------------------------------------------------------------------------------ attention
static size_t note_bytes(const CacheAttend &a) { return 2 * (size_t)a.T * a.c.H * sizeof(TokenNote); }
static size_t state_bytes(const CacheAttend &a) { return 2 * (size_t)a.T * a.c.H * a.G * kRecord * sizeof(float); }

// Rows from which a call that is not small goes to the kernel for many queries: it does the few rows of a request's own as they are, the one for few
// queries with as many tiles as the sources' take.  Four drafted tokens of 24 requests, six sources of 8 K, 32 rows, float32: 65 us there and 40 here; eight requests
// behind 32 K, 32 rows, bf16, 35.4 and 28.8; twelve, 48 rows, 42.7 and 31.9.  But eight requests behind 2 K, 64 quanta: 15.0 and 18.5; behind 4 K, 768 of them, the two are even,
// 17.7 and 18.0.
static bool for_many(long long rows, double quanta) { return rows > kFewRows || (rows > kRows && quanta > 512); }

// (How many sources a step has is not known here: quanta are those of the requests and of one source.  Of several a piece is longer than it need be: one token each of
// eight requests, 1 KV head of 8, behind four sources of 8 K 20.3 us, behind one 18.9; 2 KV heads, behind eight of 4 K 18.2, behind one 18.9.)
size_t plan_cache_shared(CacheAttend &a, int max_source) {
    const long long most = std::max(a.max_query, a.max_shared), tile = kChunkRows / a.G;
    const auto quanta = [&](int keys, long long queries) { return ((long long)keys + kQuantum - 1) / kQuantum * (a.many ? (queries + tile - 1) / tile : 1); };
    const auto all = [&]() { return (double)a.c.H * ((double)a.S * quanta(a.max_keys, a.max_query) + quanta(max_source, a.max_shared)); };
    a.many = false;  // (quanta without their row tiles)
    a.many = for_many(most * a.G, all());
    CacheAttend rows = a;
    rows.max_query = (int)most;
    a.rows = a.many ? (int)std::min<long long>(tile, most) * a.G : few_rows(rows);
    // (the flat work of the kernel for many queries counts what a unit costs beside its keys, so pieces may be shorter than a quantum of keys.  Six requests of 16
    // heads a group behind 1900 tokens: 17.6 us, 21.6 with as many pieces as quanta of keys.)
    a.groups = (int)std::min<double>(a.rows > kRows ? 512 : 768, a.many ? 2 * all() : all());
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
