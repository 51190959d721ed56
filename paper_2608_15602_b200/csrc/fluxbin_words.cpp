// fluxbin_call_words: the attention-side calls with their arguments as an array of 64-bit words.
#include "../../include/fluxbin.h"

#include <cstring>

namespace {

template <typename T> T *ptr(int64_t w) { return reinterpret_cast<T *>(static_cast<intptr_t>(w)); }
int32_t i32(int64_t w) { return static_cast<int32_t>(w); }
float f32(int64_t w)
{
    double x;
    std::memcpy(&x, &w, sizeof(x));
    return static_cast<float>(x);
}

} // namespace

extern "C" fluxbin_status_t fluxbin_call_words(int32_t which, const int64_t *w)
{
    if (!w) return FLUXBIN_ERR_NULL;
    using cache_t = const fluxbin_kv_cache_t;
    using rotary_t = const fluxbin_rotary_t;
    using ints = const int32_t;
    switch (which) {
    case FLUXBIN_CALL_ROTARY:
        return fluxbin_rotary(ptr<rotary_t>(w[0]), i32(w[1]), i32(w[2]), i32(w[3]), ptr<ints>(w[4]), ptr<const void>(w[5]), i32(w[6]), w[7], w[8],
                              ptr<void>(w[9]), w[10], w[11], ptr<const void>(w[12]), i32(w[13]), w[14], w[15], ptr<void>(w[16]), w[17], w[18],
                              ptr<void>(w[19]));
    case FLUXBIN_CALL_KV_APPEND:
        return fluxbin_kv_append(ptr<cache_t>(w[0]), i32(w[1]), i32(w[2]), ptr<ints>(w[3]), ptr<const void>(w[4]), w[5], w[6], ptr<const void>(w[7]),
                                 w[8], w[9], ptr<rotary_t>(w[10]), ptr<ints>(w[11]), ptr<const void>(w[12]), i32(w[13]), w[14], w[15],
                                 ptr<void>(w[16]), w[17], w[18], ptr<void>(w[19]));
    case FLUXBIN_CALL_KV_READ:
        return fluxbin_kv_read(ptr<cache_t>(w[0]), i32(w[1]), i32(w[2]), ptr<ints>(w[3]), ptr<void>(w[4]), ptr<void>(w[5]), ptr<void>(w[6]));
    case FLUXBIN_CALL_KV_ATTEND:
        return fluxbin_kv_attend(ptr<cache_t>(w[0]), i32(w[1]), i32(w[2]), i32(w[3]), ptr<const void>(w[4]), i32(w[5]), w[6], w[7], ptr<ints>(w[8]),
                                 ptr<ints>(w[9]), ptr<ints>(w[10]), w[11], i32(w[12]), f32(w[13]), ptr<void>(w[14]), w[15], w[16],
                                 ptr<float>(w[17]), ptr<void>(w[18]), static_cast<size_t>(w[19]), ptr<void>(w[20]));
    case FLUXBIN_CALL_NORM_ROTARY:
        return fluxbin_norm_rotary(ptr<rotary_t>(w[0]), f32(w[1]), i32(w[2]), i32(w[3]), i32(w[4]), ptr<ints>(w[5]), ptr<const void>(w[6]), i32(w[7]), w[8],
                                   w[9], ptr<const void>(w[10]), ptr<void>(w[11]), w[12], w[13], ptr<const void>(w[14]), i32(w[15]), w[16], w[17],
                                   ptr<const void>(w[18]), ptr<void>(w[19]), w[20], w[21], ptr<void>(w[22]));
    case FLUXBIN_CALL_NORM_ROTARY_BACKWARD:
        return fluxbin_norm_rotary_backward(ptr<rotary_t>(w[0]), f32(w[1]), i32(w[2]), i32(w[3]), i32(w[4]), ptr<ints>(w[5]), ptr<const void>(w[6]), i32(w[7]),
                                            w[8], w[9], ptr<const void>(w[10]), ptr<const void>(w[11]), w[12], w[13], ptr<void>(w[14]), w[15], w[16],
                                            ptr<void>(w[17]), ptr<const void>(w[18]), i32(w[19]), w[20], w[21], ptr<const void>(w[22]), ptr<const void>(w[23]),
                                            w[24], w[25], ptr<void>(w[26]), w[27], w[28], ptr<void>(w[29]), ptr<void>(w[30]), static_cast<size_t>(w[31]),
                                            ptr<void>(w[32]));
    case FLUXBIN_CALL_DRAFT_TREE:
        return fluxbin_draft_tree(i32(w[0]), i32(w[1]), i32(w[2]), ptr<ints>(w[3]), ptr<ints>(w[4]), ptr<ints>(w[5]), ptr<int32_t>(w[6]), ptr<int32_t>(w[7]),
                                  ptr<void>(w[8]));
    case FLUXBIN_CALL_DRAFT_ACCEPT:
        return fluxbin_draft_accept(i32(w[0]), i32(w[1]), i32(w[2]), ptr<ints>(w[3]), ptr<ints>(w[4]), ptr<ints>(w[5]), ptr<ints>(w[6]), ptr<int32_t>(w[7]),
                                    ptr<int32_t>(w[8]), ptr<int32_t>(w[9]), ptr<int32_t>(w[10]), ptr<void>(w[11]));
    case FLUXBIN_CALL_KV_ATTEND_TREE:
        return fluxbin_kv_attend_tree(ptr<cache_t>(w[0]), i32(w[1]), i32(w[2]), i32(w[3]), ptr<const void>(w[4]), i32(w[5]), w[6], w[7], ptr<ints>(w[8]),
                                      ptr<ints>(w[9]), ptr<ints>(w[10]), w[11], i32(w[12]), ptr<ints>(w[13]), w[14], i32(w[15]), f32(w[16]), ptr<void>(w[17]),
                                      w[18], w[19], ptr<float>(w[20]), ptr<void>(w[21]), static_cast<size_t>(w[22]), ptr<void>(w[23]));
    case FLUXBIN_CALL_KV_KEEP:
        return fluxbin_kv_keep(ptr<cache_t>(w[0]), i32(w[1]), i32(w[2]), ptr<ints>(w[3]), ptr<ints>(w[4]), ptr<ints>(w[5]), ptr<void>(w[6]));
    case FLUXBIN_CALL_KV_ADVANCE:
        return fluxbin_kv_advance(i32(w[0]), i32(w[1]), i32(w[2]), ptr<ints>(w[3]), ptr<ints>(w[4]), ptr<int32_t>(w[5]), w[6], i32(w[7]),
                                  ptr<int32_t>(w[8]), i32(w[9]), ptr<ints>(w[10]), ptr<int32_t>(w[11]), ptr<int32_t>(w[12]), ptr<int32_t>(w[13]),
                                  ptr<int32_t>(w[14]), ptr<int32_t>(w[15]), ptr<int32_t>(w[16]), ptr<int32_t>(w[17]), ptr<void>(w[18]));
    }
    return FLUXBIN_ERR_UNSUPPORTED;
}
