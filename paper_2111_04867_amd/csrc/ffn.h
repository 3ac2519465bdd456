// Launch interface between the C ABI layer and the kernels of the experts'
// feed-forward, of its few-token form and of dropout.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "taccl.h"

namespace taccl {

constexpr int kFfnMaxSources = 1024;
constexpr int kFfnMaxCols = 65536;
constexpr int kFfnTokens = 64;
constexpr int kDropoutMaxCols = 1 << 20;

// Parts of the workspace of taccl_ffn and taccl_ffn_backward, in bytes from its
// start. Rows there are compact: those of expert e follow each other from
// e * sources * capacity on.
struct FfnSpace {
  int64_t rows;       // int32 [E]: rows of each expert
  int64_t num_tiles;  // int32 [4]
  int64_t tiles[4];   // FfnTile[]: tiles of 32, 64, 128 and 256 rows
  int64_t map;        // int32 [E][sources * capacity]: row numbers in the buffer (sources > 1)
  int64_t act;        // T [E][sources * capacity][hidden]
  int64_t dpre;       // T [E][sources * capacity][2 hidden] (backward)
  int64_t done;       // int32 [4][kSplitTiles]: parts of a product's tiles that are there
  int64_t partial;    // float: their sums
  int64_t least;      // bytes that a call needs
  int64_t bytes;      // and that it uses
};
constexpr int kSplitTiles = 1024;
FfnSpace ffn_space(int64_t sources, int64_t experts, int64_t capacity, int64_t hidden, int dtype,
                   bool backward);

// Arguments are the C ABI's, checked.
hipError_t launch_ffn(const taccl_ffn_t &a, int cus, hipStream_t stream);
hipError_t launch_ffn_backward(const taccl_ffn_backward_t &a, int cus, hipStream_t stream);
int64_t ffn_tokens_space(int64_t tokens, int64_t k, int64_t cols, int64_t hidden);
hipError_t launch_ffn_tokens(const taccl_ffn_tokens_t &a, int cus, hipStream_t stream);
hipError_t launch_dropout(const taccl_dropout_t &a, hipStream_t stream);

}  // namespace taccl
