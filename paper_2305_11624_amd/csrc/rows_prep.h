// What the products of mm_tile.h want done to their operands first: launchers of rows_prep.hip.
#pragma once
#include "f8_code.h"

namespace convbn {

// Rows of whole 16-byte pieces with zeros past the last number, for operands that are not read where they are; fp32 numbers in three planes
struct RowsCopy { i64 rows, ld; int width; const void* x; bf16_t* out; };   // (out null: none)
hipError_t launch_rows_copies(int dtype, const RowsCopy& a, const RowsCopy& b, hipStream_t st);

// Column sums: slices of the rows add up theirs, 16 rows at a time, and a later launch joins the slices in order
constexpr int SUM_ROWS = 16;
int row_slices(i64 M, int N);
hipError_t launch_sums(const float* part, int slices, int N, float* out, hipStream_t st);
// dz [M][N] (ldz apart), a copy of it as above, its column sums (part: [row_slices(M, N)][N], where there are several); either output null = not wanted
hipError_t launch_rows_sums(int dtype, i64 M, int N, i64 ldz, const void* dz, bf16_t* copy, float* part, float* out, hipStream_t st);

// What codes stand for, as bf16 rows of K rounded up to 8 with zeros past K
struct F8Widen { i64 rows; int K; const uint8_t* q; const uint8_t* s; bf16_t* out; };   // (out null: none)
hipError_t launch_f8_widen(const F8Widen& a, const F8Widen& b, hipStream_t st);

}  // namespace convbn
