// Host-side argument checks shared by the ABI's translation units (defined in abi.cu).
#pragma once

#include "internal.cuh"

namespace conduit {
namespace abi {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Records the text of conduit_last_error_string and returns the code.
conduit_status fail(conduit_status code, const char* fmt, ...);
conduit_status cuda_fail(cudaError_t err, const char* what);
conduit_status check_batch(const conduit_batch* b);
conduit_status check_kv(const conduit_kv* kv, const conduit_batch* b);
conduit_status check_workspace(void* ws, size_t have, size_t need);
KvDev make_kv(const conduit_kv* kv, const conduit_batch* b);
BatchDev make_batch(const conduit_batch* b);

}  // namespace abi
}  // namespace conduit
