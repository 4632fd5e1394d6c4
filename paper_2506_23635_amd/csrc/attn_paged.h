// attn_paged.h -- what the paged cache's kernels (attn_paged.hip), its C-ABI
// (attn_paged_capi.cpp) and the attention block (attn_capi.cpp) share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/attn.h"

namespace paged {

constexpr int kXcds = 8;
constexpr int kFewRows = 16;       // query rows of one key/value head that few() takes at once
constexpr int kFewRuns = 512;      // workgroups that divided positions of few() go to: two per CU
constexpr int kTile = 32;          // positions of a step of one wave of few()
constexpr int kStep = 64;          // positions of a workgroup's step of tile()
constexpr int kPartPad = 4;        // maximum, weight and padding behind the hd sums of a partial row

// A token: its position and its page (the slot is position % page_size), or -1.
struct Token {
    int32_t pos, page;
};

// One page that gets new tokens: slots slot0 .. slot0 + n - 1 hold tokens
// tok0 .. of the batch.
struct PageWork {
    int32_t page, slot0, n, tok0;
};

// One workgroup's share of the attention: query rows row0 .. row0 + rows - 1
// of a sequence and key/value head (row = token * group + head in group) over
// positions begin .. end - 1.
struct Item {
    int32_t tok0;      // the sequence's first token in the batch
    int32_t row0, rows;
    int32_t kvh;
    int32_t pos0;      // position of the sequence's first new token
    int32_t n_pos;     // positions of the sequence, its new tokens included
    int32_t begin, end;
    int32_t table;     // its pages, from here in the table
    int32_t slot;      // where the unnormalised sums go, or -1: all of the positions, result to out
    int32_t holes;     // whether some of its table entries are -1
    int32_t next;      // of few()'s: the workgroup's next share in the list, or -1
};

// Rows whose positions several items share: their partial sums are slots
// slot0 .. slot0 + n - 1.
struct Merge {
    int32_t tok0, row0, rows, kvh;
    int32_t slot0, n;
    int32_t pad[2];
};

// Counts that the kernels read on the device, so that a captured launch
// follows a batch set after the capture.  A launch's q, qkv and out have as many
// rows as the batch that it was made for has tokens (Args::T): on a batch of
// another T the kernels do nothing.
struct Header {
    int32_t T, n_pages, n_few, n_tile[2];
    int32_t n_merge[2];        // few()'s entries, tile()'s
    int32_t pad;
};

// Device pointers and sizes of a context's batch.
struct Args {
    const Header* hdr;
    const double* freq;        // [hd/2] theta^(-2i/hd)
    const Token* tok;          // [T]
    const PageWork* pages;     // [n_pages]
    const Item* few;
    const Item* tile[2];       // row blocks of 128, of 64
    const Merge* merge[2];     // few()'s entries, tile()'s
    const int32_t* table;
    float* few_part;           // [slot][16][hd + kPartPad]
    float* tile_part;          // [slot][128][hd + kPartPad]
    uint8_t *k, *v;            // the layer's pages [page][kv head][slot][hd]
    float *k_scale, *v_scale;  // the layer's scales [page][kv head] (e4m3)
    int T;                     // the tokens of the batch that the launch is made for
    int H, G, hd, shift;       // page_size = 1 << shift
    int e4m3;
};

// Where append reads q | k | v: rows of fp32 or bf16, ld elements apart, or
// (packed) the projection's fp32 sums in packed row order, to be added over
// n_split ranges `stride` elements apart.
struct Source {
    const void* x;
    int64_t ld, stride;
    int n_split, bf16, packed;
};

// A batch's arrays lie one after another in pinned host memory, each from a
// multiple of 16 bytes on, and go to places of their own in the workspace.
struct Segment {
    uint64_t dst, src;
};
constexpr int kSegments = 10;
struct Unpack {
    const uint8_t* src;
    uint8_t* dst;
    uint64_t bytes;            // of all, a multiple of 16
    Segment seg[kSegments];
};

}  // namespace paged

extern "C" {
hipError_t attn_paged_launch_unpack(const paged::Unpack* u, hipStream_t s);
hipError_t attn_paged_launch_append(const paged::Args* a, const paged::Source* x, uint16_t* q, int T,
                                    int n_pages, hipStream_t s);
// n: workgroups for few()'s shares, for tile()'s blocks of 128 rows and of 64
hipError_t attn_paged_launch_attend(const paged::Args* a, const uint16_t* q, uint16_t* out, const int* n, hipStream_t s);
// n, slots: few()'s and tile()'s entries at once, and the most slots of one
hipError_t attn_paged_launch_merge(const paged::Args* a, uint16_t* out, const int* n, const int* slots, int few_rows,
                                   hipStream_t s);

// The batch of a paged context as the attention block needs it.
int32_t attn_paged_tokens(const attn_paged_ctx* ctx);
const attn_paged_config* attn_paged_cfg(const attn_paged_ctx* ctx);
int attn_paged_can_append(const attn_paged_ctx* ctx);   // a batch is set, and all its tokens have pages
hipError_t attn_paged_run_append(attn_paged_ctx* ctx, int32_t layer, const paged::Source* x, uint16_t* q,
                                 hipStream_t s);
hipError_t attn_paged_run_attend(attn_paged_ctx* ctx, int32_t layer, const uint16_t* q, uint16_t* out,
                                 hipStream_t s);
}
