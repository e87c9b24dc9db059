// Rows in 8 bits as the integer products read them, weights and inputs alike: pieces of 16 rows by 64 inputs (1 KB), byte
// [g][r][j] of a piece being row r, input 16 g + j.  What lane 16 g + r of a wavefront hands the 16x16x64 matrix
// instruction is 16 bytes in order, and a wavefront's load is 1 KB in order, from memory and from LDS alike.
#pragma once

#include "serving.h"

constexpr int kRows = 16, kDepth = 64, kPiece = kRows * kDepth;  // a piece
constexpr int64_t kMostDepth = 131072;                            // 127 * 127 * d_in < 2^31
// Rows that one launch takes, up to 1024 lanes each: of 2^32 lanes or more HIP launches what 32 bits hold of the number, as a rule
// without an error.
constexpr int64_t kRowsOfLaunch = 1 << 21;

// The host's checks of cmpq_rms_norm and cmpq_int8_product_job (but for its workspace), for calls that make several of these.
int cmpq_check_rms_norm(const cmpq_norm_job *job);
int cmpq_check_int8_product(const cmpq_int8_job *job);
size_t cmpq_ws_int8_product(int64_t d_in, int64_t m);

__host__ __device__ inline int64_t pieces_deep(int64_t d) { return (d + 127) / 128 * 2; }

// Workgroups in the order in which they are handed to the eight dies, so that each die gets a run of them.
__device__ __forceinline__ int64_t die_order(int64_t x, int64_t n) {
    const int64_t each = n / 8, more = n % 8, die = x % 8;
    return die * each + min(die, more) + x / 8;
}
