// Records of the gradient norm and clipping kernels (gact_norm.hip), filled by their entry points.
#ifndef GACT_NORM_H
#define GACT_NORM_H

#include <stddef.h>
#include <stdint.h>

#include "gact_device.h"

namespace gact {

constexpr int kNormWaves = 8, kNormThreads = 64 * kNormWaves;
constexpr int kNormPieces = 2;                    // of 16 bytes, per thread and chunk
constexpr int64_t norm_chunk_elems(int dtype) { return kNormThreads * kNormPieces * (dtype == GACT_DT_F32 ? 4 : 8); }
// Blocks of a launch, each of which takes a run of neighbouring chunks and leaves one result.
constexpr uint32_t kNormBlocks = 1024;
static_assert(kNormBlocks <= 2 * kNormThreads, "two results a thread when a block adds them up");

struct NormBuffer {
    const void* in;
    void*       out;                              // null: norm only
    int64_t     n;
};
// A table small enough to travel in the kernel arguments: the buffers of one type behind those of the other
// (f32 of them are fp32), then the first chunk of each.
constexpr int kInlineNorm = 136;
struct NormTable {
    NormBuffer t[kInlineNorm];
    uint32_t   first[kInlineNorm + 1];
};
struct NormArgs {
    const NormBuffer* table;                      // device memory; null: the inline table
    const uint32_t*   first;
    uint32_t K, f32, chunks, blocks;
    double*  partial;                             // one a block
    double*  norm;
    double   max_norm;
};
static_assert(sizeof(NormTable) + sizeof(NormArgs) <= kKernelArguments, "a list's table and what precedes it");

// A piece of a table on its way to the workspace in the arguments of a kernel.
constexpr int kTablePiece = 3968;
struct TablePiece {
    uint32_t w[kTablePiece / 4];
};

}  // namespace gact

extern "C" int gact_launch_grad_norm(const gact::NormTable* t, const gact::NormArgs* a, int kind, int finish, void* stream);
extern "C" int gact_launch_grad_clip(const gact::NormTable* t, const gact::NormArgs* a, int kind, int given, void* stream);
extern "C" int gact_launch_table_piece(void* dst, const gact::TablePiece* piece, unsigned words, void* stream);

#endif
