// Internal interface of the paged key-value cache: what kv_api.cu hands to the kernel
// translation units, and what api.cu lends it.  Not part of the public ABI.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <cstdint>

namespace w4a16 {

// api.cu: the current device's state, and the encoder of tensor maps (128-byte swizzle).
struct LibraryState {
    int sm_count;
    int* status;  // device status word
};
int library_state(LibraryState* out);
int encode_5d(CUtensorMap* map, CUtensorMapDataType dtype, const void* base, const uint64_t dims[5],
              const uint64_t strides[4], const uint32_t box[5]);

constexpr int kKvHeadDim = 128;
constexpr int kKvMaxSlots = 1 << 16;
constexpr int kKvMaxPages = 1 << 24;

// A cache as the kernels see it.
struct KvView {
    uint8_t* pages;      // bf16 or e4m3 [layers, 2, num_pages, kv_heads, T, 128]
    uint8_t* exponents;  // e4m3: [layers, num_pages, kv_heads, T, 2]
    int32_t* table;      // [num_slots, max_pages]
    int32_t* seq_len;    // [num_slots]
    int32_t* refs;       // [num_pages]
    int32_t* scratch;    // KvScratch
    int32_t* refused;    // [num_slots], in the scratch buffer: kKvRefused where the last growth failed
    int* status;
    int layers, num_pages, kv_heads, page_shift /* log2 T */, num_slots, max_pages;
    int row_bytes;       // of a token's key: 256 or 128
};

// The scratch buffer: a header, kKvScratchLists lists of max(num_pages, num_slots) entries, and a
// mark for each slot.
constexpr int kKvScratchLists = 5;
// A slot's mark: its last kv_extend was refused, so the tokens that a prompt's write or a step would
// store were not added and their places are those of its last tokens (which others may share).
constexpr int32_t kKvRefused = 0x4B565245;
struct KvScratch {
    int32_t copies;  // entries of src / dst / tokens
    int32_t moved;   // compaction: pages from this index on have moved (a list says where), else -1
    int32_t refused; // slots with a mark: where there are none no mark is read
    int32_t pad[13];
};
constexpr int kKvScratchHeader = sizeof(KvScratch) / sizeof(int32_t);
inline __host__ __device__ int kv_scratch_list(int num_pages, int num_slots) {
    return num_pages > num_slots ? num_pages : num_slots;
}

cudaError_t launch_kv_extend(const KvView& kv, const int32_t* slots, const int32_t* add, int n,
                             int sm_count, cudaStream_t stream);
cudaError_t launch_kv_fork(const KvView& kv, const int32_t* parents, const int32_t* children, int n,
                           cudaStream_t stream);
cudaError_t launch_kv_trim(const KvView& kv, const int32_t* slots, const int32_t* keep, int n,
                           cudaStream_t stream);
cudaError_t launch_kv_compact(const KvView& kv, int sm_count, cudaStream_t stream);

struct KvWriteParams {
    const uint16_t* qkv;  // [M, (H + 2 kv_heads) * 128]
    const int32_t* seq_start;
    const int32_t* slots;
    int layer, nseq, M, H;
};
cudaError_t launch_kv_write(const KvView& kv, const KvWriteParams& p, int sm_count, cudaStream_t stream);

struct DecodeParams {
    const uint16_t* qkv;  // [n, (H + 2 kv_heads) * 128]
    const int32_t* slots;
    uint16_t* out;        // [n, H * 128]
    void* workspace;
    int layer, n, H, window;
    float scale;          // 1 / sqrt(128)
    uint64_t wait_ns;
};
int64_t decode_workspace_bytes(int H, int kv_heads, int sm_count);
// Tensor maps of a layer's keys and values: of a page's groups of 16 tokens, or as many as a tile
// has, and of one group.
struct CacheMaps {
    CUtensorMap box, group;
    int groups;  // of `box`: a power of two
};
int encode_cache(CacheMaps* maps, const KvView& kv, int layer);
cudaError_t launch_attention_decode(const CacheMaps& maps, const KvView& kv, const DecodeParams& p,
                                    int sm_count, cudaStream_t stream);

uint64_t wait_limit_ns();  // internal.h

// A launch that may begin while the kernel before it in the stream ends; the kernel calls
// grid_wait (ptx.cuh) before it touches global memory.
template <typename... P, typename... A>
cudaError_t launch_overlapped(void (*kernel)(P...), dim3 grid, int block, int smem, cudaStream_t stream,
                              const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace w4a16
