// Attention over the 4-bit sequence cache: how a call is cut, and the causal and the listed form.
#include "ice_cache_attend.h"

namespace ice {

// Units (request, KV head) that stay whole, one workgroup each, no merge behind it: short ones, where the merge costs more than the cut gains, longer
// ones too where they are many, and lists of as many units as there are CUs.  Cut and whole, us: dense, 8 units of 512 keys 9.4 and 7.9, of
// 1024 9.3 and 11.3; 128 units of up to 1024 keys 14.6 and 11.9, of up to 4096 22 and 32; 512 units of up to 2048 keys 30 and 27, of up to 4096 44
// and 43.  Lists, 8 units of 512 tokens 8.9 and 8.0, of 1024 9.5 and 11.0; 128 units of 1024 15.9 and 14.1, of 2048 22 and 26; 256 units of 2048
// 36.7 and 34.8, of 4096 62 and 60.
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

long long cut_cache_attend(CacheAttend a, bool listed, const int *start, const int *len, int *parts, long long most) {
    return listed ? cut_attend<kListed>(a, start, len, parts, most) : cut_attend<kCausal>(a, start, len, parts, most);
}

void launch_cache_attend(CacheAttend a, hipStream_t stream) {
    if (a.pos) launch_attend<kListed>(a, stream);
    else launch_attend<kCausal>(a, stream);
}

}  // namespace ice
