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
// Blocks of a norm's launch, each of which takes a run of neighbouring chunks and leaves one result: as many as the compute units
// hold at a time (three of eight wavefronts, by their registers), twice as many from kClipOnceBytes on.  Clipping and the norm alone
// have the same number for a list, so that both add in one order.  Us, norm + scaling behind it, or norm alone, 768 blocks | 1024 |
// 1536: 50 MB fp32 9.3 + 15.4 | 11.8 + 15.4, 202 MB 34.5 + 58.5 | 35.8 + 59.4; 102 MB that need no scaling 17.5 + 4.4 | 17.9 + 5.8 |
// 17.5 + 7.5; 201 MB bf16 31.4 | 33.0 | 31.5, 608 MB 97 | 96 | 92.  Between, whole calls, 768 | 1536: clipping 270 MB 125 | 128,
// 403 MB 187 | 200; norm alone 270 MB 42.5 | 43.6, 403 MB 62.4 | 64.4, bf16 43.5 | 43.9, 65.1 | 64.8.
constexpr uint32_t kNormFit = 768, kNormBlocks = 1536;
// Lists of this many bytes and more do not stay in the 256 MB cache from one launch to the next: a norm alone reads them as data
// that nobody wants again, and clipping, which reads them twice, from the larger bound on.  Clipping has then kClipBlocks (each
// adds up the norm's results first), as it has by a given norm.  Us, ordinary | as said, measured with 1024 blocks: norm alone 201 MB
// bf16 32.0 | 33.4, 608 MB 108 | 95; clipping fp32, norm + scaling, 50 MB 27 | 31, 101 MB 49 | 57, 202 MB 95 | 102, 403 MB
// 193 | 199, 503 MB 244 | 241, 604 MB 301 | 294, 1.2 GB 632 | 610.
constexpr uint64_t kNormOnceBytes = 256ull << 20, kClipOnceBytes = 440ull << 20;
constexpr uint32_t kClipBlocks = 8192;

// A buffer from the first cache line of the input on, so that a wavefront's loads are whole lines: 608 MB at odd addresses 124 us
// from the first element on, 99 from the first 16 bytes, 95 from the first line (1024 blocks).
constexpr uintptr_t kNormLine = 128;
struct NormBuffer {
    const void* in;
    void*       out;                              // null: norm only
    int64_t     n : 56;                           // from there on
    int64_t     head : 8;                         // elements in front, up to 63
};
static_assert(sizeof(NormBuffer) == 24, "three words of a table");
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
    uint32_t K, f32, chunks, blocks, clip_blocks;
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

extern "C" int gact_launch_grad_norm(const gact::NormTable* t, const gact::NormArgs* a, int kind, int once, int finish, void* stream);
extern "C" int gact_launch_grad_clip(const gact::NormTable* t, const gact::NormArgs* a, int kind, int given, void* stream);
extern "C" int gact_launch_table_piece(void* dst, const gact::TablePiece* piece, unsigned words, void* stream);

#endif
