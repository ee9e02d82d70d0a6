// Host-side declarations of the two ends of a language model: mhcl_ends.hip (embedding, norm), mhcl_head.hip
// (cross entropy), mhcl_ends_api.hip (their C ABI).
#pragma once
#include "../csrc/mhcl_internal.h"

namespace mhcl {

inline size_t dtype_bytes(int dtype) { return dtype == MHCL_BF16 ? 2 : 4; }

hipError_t launch_embed(const mhcl_ends_desc &d, const void *table, const void *ids, void *x, hipStream_t s);

// Backward of the embedding: the tokens in the order of their ids (equal ids in the order of the tokens), the sums of
// every `chunk` of them, and the rows that lie in several chunks joined from those.
struct EmbedBwdWs {
  int32_t chunk;         // tokens
  int64_t chunks;
  int32_t *key, *pos;    // [T] sorted ids and the tokens they belong to
  int32_t *key2, *pos2;  // [T] the same on the way there
  int32_t *counts;       // [64][512] digits of the blocks of a pass
  int32_t *shared_rows;  // [1 + chunks] number and list of the chunks in which a row begins that goes on in others
  float *part;           // [chunks][2][C] sums of a chunk's first and last row where others share it
  size_t bytes;
  EmbedBwdWs(const mhcl_ends_desc &d, void *ws) {
    WsCursor c(ws);
    chunk = embed_chunk(d);
    chunks = (d.T + chunk - 1) / chunk;
    key = c.take<int32_t>(d.T);
    pos = c.take<int32_t>(d.T);
    key2 = c.take<int32_t>(d.T);
    pos2 = c.take<int32_t>(d.T);
    counts = c.take<int32_t>(64 * 512);
    shared_rows = c.take<int32_t>(1 + static_cast<size_t>(chunks));
    part = c.take<float>(static_cast<size_t>(chunks) * 2 * d.C);
    bytes = c.off;
  }

 private:
  static int32_t embed_chunk(const mhcl_ends_desc &d);
};
hipError_t launch_embed_bwd(const mhcl_ends_desc &d, const void *ids, const void *g_x, void *g_table, bool accumulate,
                            const EmbedBwdWs &w, hipStream_t s);

hipError_t launch_streams_norm(const mhcl_ends_desc &d, const void *x, const float *gain, void *h, hipStream_t s);
constexpr int kNormBwdBlocks = 512;   // each leaves a row of g_gain's sums
inline size_t norm_bwd_ws_bytes(const mhcl_ends_desc &d) {
  return align_up(static_cast<size_t>(kNormBwdBlocks) * d.C * sizeof(float));
}
hipError_t launch_streams_norm_bwd(const mhcl_ends_desc &d, const void *x, const float *gain, const void *g_h, void *g_x,
                                   float *g_gain, float *part, hipStream_t s);
// zeros in `bytes` bytes (a multiple of 4), by a kernel
hipError_t launch_zero(void *p, size_t bytes, hipStream_t s);

}  // namespace mhcl
