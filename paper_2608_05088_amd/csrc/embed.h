// Arguments and launchers of the token table's kernels (embed.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace malt {

constexpr int SORT_THREADS = 256, SORT_TILE = 2048;   // keys a block of the sort takes
constexpr int SORT_ONE = 8192;                        // tokens one workgroup sorts by itself
constexpr int FEW = 256;                              // tokens that need no workspace
constexpr int64_t LOOK_MOST = 1 << 19;                // looks of rows at tokens in one launch
constexpr int FIRST_MOST = 4096;                      // tokens (times strips) that need no sort

struct EmbedLookupArgs {
  const void* ids;
  const void* table;
  void* out;
  int64_t tokens, vocab, table_ld, out_ld;
  int32_t width;
  bool wide_ids;
  float scale;
  int32_t lanes_log2;   // set by the launcher
};

struct EmbedGradArgs {
  const void* ids;
  const void* grad;
  void* dtable;
  int64_t tokens, vocab, grad_ld, dtable_ld;
  int32_t width;
  bool wide_ids, accumulate;
  float scale;
  // set by the launcher
  const uint32_t* keys;    // sorted keys and the tokens they belong to
  const uint32_t* order;
  uint32_t* table;         // [digit][block] counts of the sort
  uint32_t* seg;           // [vocab][2]: first and one past the last sorted token
  float* part;             // [chunk][2][part_ld]
  float* groups;           // [chunk / GROUP][part_ld], or null
  int64_t part_ld;
  int64_t chunks;          // of the sorted tokens, `chunk` of them each
  int32_t chunk;
};

struct EmbedGradLayout {
  size_t keys[2], index[2], table, seg, part, groups, bytes;
  int64_t blocks, part_ld;
  int32_t chunk;
};

EmbedGradLayout embed_grad_layout(int64_t tokens, int64_t vocab, int64_t width);
hipError_t launch_embed_lookup(EmbedLookupArgs a, bool table_f32, bool out_f32, hipStream_t s);
hipError_t launch_embed_grad(const EmbedGradArgs& a, const EmbedGradLayout& L, char* ws, bool grad_f32, bool out_f32,
                             hipStream_t s);

}  // namespace malt
