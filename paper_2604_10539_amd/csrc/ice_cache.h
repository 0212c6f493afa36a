// Internal declarations of the 4-bit sequence cache: its layout and the launches of its kernels.
#pragma once
#include "ice_internal.h"

namespace ice {

// One tile holds 16 consecutive tokens of one KV head: key codes [16][64 bytes], value codes [16][64], key scales [64], value
// scales [64] (17 cache lines).  A row's codes lie together, so that a listed token costs one 64-byte piece, and a tile's
// rows follow each other, so that a wave's load of 16 bytes a lane covers a whole KiB.  The scale of token t's block j of 32
// dimensions is byte 16 (t mod 4) + 4 j + t / 4: a lane of the value product works on tokens g, 4 + g, 8 + g, 12 + g and finds their
// four scales in one dword.
constexpr int kCacheTile = 16;
constexpr int kCacheTileBytes = 2176;
constexpr int kCacheV = 1024, kCacheKS = 2048, kCacheVS = 2112;
__host__ __device__ inline int cache_scale_byte(int t, int j) { return 16 * (t & 3) + 4 * j + (t >> 2); }

struct CacheDims {
    uint8_t *data;
    int n_blocks, H, tile_shift;  // tiles per block = 1 << tile_shift
};

struct CachePlan {
    int n_requests, block_shift, max_blocks, n_blocks;
    const int *new_len, *cached_len;
    int *seq_len, *table, *free_ids;
    const int *n_free;
    int *n_free_left, *query_start, *slots;
    int n_slots;
    int *info;
    bool end_later;  // lengths and the stack's height are written by a second launch
};
constexpr int kPlanRequests = 8192;  // of one plan at most: three sums each in LDS
void launch_cache_plan(CachePlan p, hipStream_t stream);

void launch_cache_write(const CacheDims &c, const bf16_t *k, const bf16_t *v, long long k_stride, long long v_stride, const int *slots,
                        int n_tokens, hipStream_t stream);
void launch_cache_read(const CacheDims &c, int n_requests, const int *seq_len, const int *table, int max_blocks, const int *first,
                       int n_rows, bf16_t *k, bf16_t *v, hipStream_t stream);

// A (request, KV head) that was cut between workgroups: the first one of them, the KV head, the request's first query row, the first of the
// unit's rows and the number of the request's rows (query, head of the group).  
struct alignas(16) MergeNote {
    int first, h, row0, base, rows;
};

struct CacheAttend {
    CacheDims c;
    const bf16_t *q;
    long long q_stride;  // elements between the query rows of two tokens
    const int *query_start, *seq_len, *table;
    const int *pos, *n_tok;  // listed tokens (then one query per request), or null
    void *out;
    float *lse, *part;
    MergeNote *notes;
    int S, T, G, max_query, max_blocks, max_keys, window;
    int rows;                     // query rows (query, head of the group) that a record has room for
    int few_groups, many_groups;  // workgroups of the kernel for few queries a request, of the one for many
    bool many;                    // some request may have more query rows than the first one takes
    int per_unit;       // > 0: nominal pieces of every (request, KV head); 0: by the lengths
    bool whole;         // one workgroup each
    int first, n_here;  // the launch's requests
    float scale_log2;
    bool out_bf16;
};
// How a call is cut, from the sizes: fills few_groups, many_groups, many, per_unit and whole; returns the bytes of workspace.
size_t plan_cache_attend(CacheAttend &a, bool listed);
void launch_cache_attend(CacheAttend a, hipStream_t stream);
// The parts that the workgroups of a planned call take, from lengths on the host (query_start and seq_len, or n_tok): their number, the first `most` of
// them in parts, kCutInts words each (see ice_debug_cache_cut).
constexpr int kCutInts = 15;
long long cut_cache_attend(CacheAttend a, bool listed, const int *query_start, const int *len, int *parts, long long most);

}  // namespace ice
