// fluxbin_call_words: the attention-side calls with their arguments as an array of 64-bit words.
#include "../../include/fluxbin.h"

#include <cstring>

namespace {

template <typename T> T *ptr(int64_t w) { return reinterpret_cast<T *>(static_cast<intptr_t>(w)); }
int32_t i32(int64_t w) { return static_cast<int32_t>(w); }

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
    case FLUXBIN_CALL_KV_ATTEND: {
        double scale;
        std::memcpy(&scale, &w[13], sizeof(scale));
        return fluxbin_kv_attend(ptr<cache_t>(w[0]), i32(w[1]), i32(w[2]), i32(w[3]), ptr<const void>(w[4]), i32(w[5]), w[6], w[7], ptr<ints>(w[8]),
                                 ptr<ints>(w[9]), ptr<ints>(w[10]), w[11], i32(w[12]), static_cast<float>(scale), ptr<void>(w[14]), w[15], w[16],
                                 ptr<float>(w[17]), ptr<void>(w[18]), static_cast<size_t>(w[19]), ptr<void>(w[20]));
    }
    case FLUXBIN_CALL_KV_ADVANCE:
        return fluxbin_kv_advance(i32(w[0]), i32(w[1]), i32(w[2]), ptr<ints>(w[3]), ptr<ints>(w[4]), ptr<int32_t>(w[5]), w[6], i32(w[7]),
                                  ptr<int32_t>(w[8]), i32(w[9]), ptr<ints>(w[10]), ptr<int32_t>(w[11]), ptr<int32_t>(w[12]), ptr<int32_t>(w[13]),
                                  ptr<int32_t>(w[14]), ptr<int32_t>(w[15]), ptr<int32_t>(w[16]), ptr<int32_t>(w[17]), ptr<void>(w[18]));
    }
    return FLUXBIN_ERR_UNSUPPORTED;
}
