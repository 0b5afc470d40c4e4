// Internal launch interface of the sampling calls between the C ABI (gen_api.cu) and the kernel files.
#pragma once
#include <cuda_runtime.h>

#include <atomic>
#include <cstddef>
#include <cstdint>

#include "../../include/harts_gen.h"

namespace harts {

struct GenLaArgs {
    int32_t n_seq;
    const int32_t *seq_begin, *seq_len, *in_state, *out_state;
    int32_t max_len;
    int64_t n_rows;
    const void *q, *k, *v;
    int64_t ld_q, ld_k, ld_v;
    const float* g;
    void* o;
    float* states;
    int32_t n_states, H, d, dtype;
    void* workspace;
    int32_t* dev_status;
    cudaStream_t stream;
};

int32_t gen_la_walk(const GenLaArgs& a);          // gen_la_walk.cu: token by token, state in registers

// Chunked form (bf16, d = 128): a sequence is one item, or several segments of whole chunks that one item each walks.
struct GenItems {
    const int32_t* count;     // device: items there are
    int32_t* ticket;          // device: 0; how many CTAs have drawn
    const int4* items;        // device: first row, rows, start state (>= 0: in the pool, -1: zero, -2 - i: starts[i]), last state's place or -1
    float* starts;            // [item, H, 128, 128] start states of segments
};
int32_t gen_la_chunks(const GenLaArgs& a);        // gen_la_chunk.cu
bool gen_la_chunked(const GenLaArgs& a);
size_t gen_la_chunk_bytes(const GenLaArgs& a);    // workspace of gen_la_chunks
int32_t pipe_gen(const GenLaArgs& a, const GenItems& items, int64_t max_items);      // la_pipe_fwd.cu

struct GenCache {
    void *k, *v;
    uint8_t *k_exp, *v_exp;
    int32_t n_pages, page, Hkv, type;
};
struct GenRows {              // rows of the cache and of k, v
    int64_t n;
    const int32_t* slot;
    void *k, *v;
    int64_t ld_k, ld_v;
    int32_t* dev_status;
    cudaStream_t stream;
};
int32_t gen_cache_write(const GenCache& c, const GenRows& r);      // gen_cache.cu
int32_t gen_cache_read(const GenCache& c, const GenRows& r);

// Index of harts_gen_attn_index: header words, then the arrays (gen_attn_host.cc writes it, gen_attn.cu reads it).
namespace gen_attn {
enum Header { N_Q, HQ, HKV, PAGE, N_NARROW, N_WIDE, N_PARTS, MERGED, MAX_PAGE, WORDS, NARROW, WIDE, ENTRY, PAGES, PART_PTR, PART, NARROW_MAX, N_LISTS, LIST_PTR };
constexpr int NARROW_ROWS = 16, WIDE_ROWS = 128;
struct Unit {                 // rows that read the same tokens of a node: rows flat0 .. flat0 + n - 1 of (entry, head of the group)
    int32_t entry, flat0, n, k0, k1, page0, part0, pad;
};
struct Entry {                // a query that sees tokens of a node
    int32_t row;
    int32_t limit;            // how many it sees; -1: q_pos + 1
    int32_t least;            // limit -1: what q_pos + 1 is at least
    int32_t most;             // and at most; negative: minus that, and this is the query's only part
};
}  // namespace gen_attn
int32_t gen_attn_launch(const int32_t* hi, const int32_t* di, const void* q, int64_t ld_q, const GenCache& c, const int32_t* q_pos, void* o,
                 float* lse, float scale, void* workspace, int32_t* dev_status, cudaStream_t stream);

// The kernel's dynamic shared memory, once for each device of the process (a call to the driver otherwise, for every launch).
template <class Kernel>
inline bool gen_shared_memory(Kernel* kernel, int bytes, std::atomic<uint64_t>& done) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (bit && (done.load(std::memory_order_relaxed) & bit)) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    done.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

#ifdef __CUDACC__
// a sequence's entries, checked: false where one is out of range (one thread of the caller reports it)
struct GenSeq {
    int begin, len, in, out;
};
__device__ __forceinline__ bool gen_seq(const GenLaArgs& a, int i, GenSeq& s) {
    s.begin = a.seq_begin[i];
    s.len = a.seq_len[i];
    s.in = a.in_state[i];
    s.out = a.out_state[i];
    return s.begin >= 0 && s.len >= 0 && s.len <= a.max_len && (int64_t)s.begin + s.len <= a.n_rows && s.in >= -1 && s.in < a.n_states &&
           s.out >= -1 && s.out < a.n_states;
}
// 2^(exp - 127) of a cache row; 255: NaN
__device__ __forceinline__ float gen_power(int exp) {
    return __uint_as_float((uint32_t)exp << 23 | (exp == 0 || exp == 255 ? 0x400000u : 0u));
}
__device__ __forceinline__ void gen_report(int32_t* status, int position) {
    if (status && atomicCAS(status, 0, HARTS_EINVAL) == 0) status[1] = position;
}
#endif

}  // namespace harts
