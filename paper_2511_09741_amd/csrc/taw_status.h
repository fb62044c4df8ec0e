// Status and argument checks shared by the C-ABI front ends.  fail() records the message that taw_last_error() returns on the calling
// thread and returns its code.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/model/taw_model.h"

namespace taw {

int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int hip_fail(int hip_code, const char* what);

// taw_optimizer_step, with a clip state (device) or without (nullptr)
int optimizer_step(const taw_adamw_desc* opt, const taw_clip_state* clip, void* W_chunk, int32_t chunk_dtype, float* master, float* m, float* v, float* G_shard,
                   size_t n_elems, hipStream_t stream);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace taw

#define TAW_REQUIRE_PTR(p) do { if (!(p)) return fail(TAW_ERR_NULL, "%s is NULL", #p); } while (0)
#define TAW_REQUIRE_ALIGNED(p) do { if (!aligned16(p)) return fail(TAW_ERR_ALIGN, "%s is not 16-byte aligned", #p); } while (0)
#define TAW_LAUNCH(call, what) do { int e_ = (call); if (e_) return hip_fail(e_, what); } while (0)
