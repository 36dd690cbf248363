// Device-side data model of the paged cache, shared by its kernels.
//
// One layer of the cache is n_pages pages of page_size tokens (a power of two, 16 to 256).
//   bf16, fp32   [page][2 (K, V)][kv_heads][page_size][head_dim], plain rows
//   4 bits       [page][kv_heads][page_size / 16 blocks]; a block holds 16 tokens of one head:
//     K codes   32-bit words [token][t 0..3][group j]: channels 32 j + 8 t + 0..7, low nibble first
//     V codes   32-bit words [token pair][g 0..7][group j]: low half = the even token's channels
//               32 j + 4 g + 0..3, high half = the odd token's
//     K scale   bf16 [token pair][group][token of the pair]
//     K lowest  bf16 [token][group]
//     V scale   as K scale
//     V lowest  as K scale
// A group is 32 channels of one token; value = lowest + scale * code.  lowest = bf16(min),
// scale = bf16((max - min) / 15), code = min(15, max(0, rint((x - lowest) / scale))) and 0 where
// scale is 0.  A group that holds a NaN or an infinity is stored as scale = NaN, lowest = 0.
//
// The order of the 4-bit words is the order in which the lanes of a warp need them as operands of
// m16n8k16 matrix instructions: one 16-byte shared-memory load per lane and token (K) or token
// pair (V), neighbouring lanes reading neighbouring 16 bytes, and a mask turns 32 bits into the
// register pair of an operand (see mkv_paged_mma.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/mkv.h"

namespace mkv {

constexpr int kPagedBlock = 16;     // tokens of a 4-bit block; also the granule of the attention kernels
constexpr int kPagedMaxGroup = 32;  // q_heads / kv_heads
constexpr int kPagedDecodeCtas = 512;   // most CTAs of a launch of the kernel for few rows
constexpr int kPagedJoinBytes = 65536;  // of the workspace, in front of the parts
constexpr int kPagedTileCtas = 160;    // most CTAs of a launch of the kernel for many rows
constexpr float kPagedNegInf = -INFINITY;

struct PagedDev {
    uint8_t* pages;      // of the call's layer
    size_t page_bytes;   // one page of one layer
    size_t head_bytes;   // bytes from one KV head to the next (bf16, fp32: within K or V)
    size_t kv_bytes;     // bf16, fp32: from a page's K to its V
    int32_t* status;
    int n_pages, page_shift, q_heads, kv_heads, group, kv_dtype, io_f32, out_f32;
};

// The new tokens of a batch: sequence b owns tokens [starts[b], starts[b + 1]) of the token
// buffers (starts == nullptr: token b), the last of which has position lens[b] - 1 in the cache.
struct PagedBatch {
    const int32_t* starts;
    const int32_t* lens;
    const int32_t* table;
    int n_tokens, batch, table_stride;
};

struct PagedAppendArgs {
    PagedDev c;
    PagedBatch b;
    const void *q, *k, *v;
    void* q_out;
    long long q_stride, k_stride, v_stride;   // elements from one token to the next
    const int32_t* positions;                 // or nullptr: the position in the cache
    const float* inv_freq;
    int rot_dim, interleaved;
};

struct PagedReadArgs {
    PagedDev c;
    PagedBatch b;
    const int32_t* first;   // or nullptr: 0
    void *K, *V;
    int rows;
};

struct PagedAttendArgs {
    PagedDev c;
    PagedBatch b;
    const void* q;
    long long q_stride;
    void* out;
    float* lse;             // or nullptr
    int max_new, window;
    float scale_log2;
    uint8_t* scratch;       // of the workspace
};

__host__ __device__ inline size_t paged_block_bytes(int head_dim) { return 16 * (size_t)head_dim + 128 * (size_t)(head_dim / 32); }

__device__ inline void paged_fail(const PagedDev& c, int code) { atomicCAS(c.status, 0, code); }

struct PagedSpan { int tok0, n, len; };   // first new token, number of new tokens, tokens in the cache

// Sequence b of the batch, brought into bounds whatever the arrays hold.
__device__ inline PagedSpan paged_span(const PagedDev& c, const PagedBatch& b, int s) {
    PagedSpan r;
    r.tok0 = b.starts ? b.starts[s] : s;
    const int end = b.starts ? b.starts[s + 1] : s + 1;
    r.len = max(b.lens[s], 0);
    if (r.tok0 < 0 || end < r.tok0 || end > b.n_tokens) {
        paged_fail(c, MKV_ERR_INVALID_ARG);
        r.tok0 = 0; r.n = 0;
    } else {
        r.n = end - r.tok0;
    }
    if (r.len > ((long long)b.table_stride << c.page_shift)) {
        paged_fail(c, MKV_ERR_CAPACITY);
        r.len = b.table_stride << c.page_shift;
    }
    return r;
}

// The page that holds position `pos` of sequence s (pos within the table); a number outside the
// pool is reported and replaced by page 0, so that no access leaves the pool.
__device__ inline int paged_page(const PagedDev& c, const PagedBatch& b, int s, int pos) {
    const int page = b.table[(size_t)s * b.table_stride + (pos >> c.page_shift)];
    if ((unsigned)page < (unsigned)c.n_pages) return page;
    paged_fail(c, MKV_ERR_INVALID_ARG);
    return 0;
}

__device__ inline float paged_bf16(uint32_t bits16) { return __uint_as_float(bits16 << 16); }

cudaError_t launch_paged_append(const PagedAppendArgs& a, int head_dim, cudaStream_t st);
cudaError_t launch_paged_read(const PagedReadArgs& a, int head_dim, cudaStream_t st);
size_t paged_decode_scratch();   // workspace of launch_paged_decode
bool make_paged_map(void* map, const void* pages, long long rows, int head_dim, int box_rows);   // bf16 pages as one list of rows
cudaError_t launch_paged_decode(const PagedAttendArgs& a, int head_dim, const void* map, long long layer_rows, int sm_count,
                                int device, cudaStream_t st);

size_t paged_tile_scratch();
cudaError_t launch_paged_tile(const PagedAttendArgs& a, int head_dim, const void* map, long long layer_rows, int sm_count,
                              int device, cudaStream_t st);

}  // namespace mkv
