// What the host layer of the GEMM calls (sfcgemm_api.cpp) shares with the other entry
// points: error text, the lock, curve tables and the per-stream workspace.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <mutex>

namespace sfc {

// Sets sfc_last_error()'s text and returns `code`.
int host_error(int code, const char* what);
int host_hip_error(hipError_t e, const char* where);

// Held from the first of the calls below to the launch that uses what they gave.
std::mutex& host_mutex();
int host_num_cus(int* num_cus);
int host_table(int gm, int gn, hipStream_t stream, const int32_t** table);
int host_workspace(hipStream_t stream, size_t bytes, void** ws);

}  // namespace sfc
