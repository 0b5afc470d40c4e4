// C entry points of sampling on rollout trees: argument checks and the choice of the kernel.
#include "gen.h"

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// a tensor of n_rows rows with ld elements between them, heads contiguous
bool rows_ok(const void* p, int64_t ld, int64_t width, int64_t elem) { return p && aligned16(p) && ld >= width && ld * elem % 16 == 0; }

harts::GenLaArgs la_sizes(int32_t n_seq, int32_t max_len, int64_t n_rows, int32_t H, int32_t d, int32_t dtype) {
    harts::GenLaArgs a{};
    a.n_seq = n_seq;
    a.max_len = max_len;
    a.n_rows = n_rows;
    a.H = H;
    a.d = d;
    a.dtype = dtype;
    return a;
}
int32_t la_check(int32_t n_seq, int32_t max_len, int64_t n_rows, int32_t H, int32_t dk, int32_t dv, int32_t dtype) {
    if (n_seq < 0 || max_len < 0 || n_rows < 0 || n_rows > INT32_MAX || H < 1 || H > 65535 || n_seq > 65535) return HARTS_EINVAL;
    if ((dtype != HARTS_FP32 && dtype != HARTS_BF16) || dk != dv || (dk != 64 && dk != 128)) return HARTS_EUNSUPPORTED;
    return HARTS_OK;
}

}  // namespace

extern "C" {

int32_t harts_gen_la_workspace_bytes(int32_t n_seq, int32_t max_len, int64_t n_rows, int32_t H, int32_t dk, int32_t dv, int32_t dtype,
                                     size_t* bytes) {
    if (!bytes) return HARTS_EINVAL;
    *bytes = 0;
    const int32_t rc = la_check(n_seq, max_len, n_rows, H, dk, dv, dtype);
    if (rc != HARTS_OK) return rc;
    const harts::GenLaArgs a = la_sizes(n_seq, max_len, n_rows, H, dk, dtype);
    if (n_seq > 0 && harts::gen_la_chunked(a)) *bytes = harts::gen_la_chunk_bytes(a);
    return HARTS_OK;
}

int32_t harts_gen_la(int32_t n_seq, const int32_t* seq_begin, const int32_t* seq_len, const int32_t* in_state,
                     const int32_t* out_state, int32_t max_len, int64_t n_rows, const void* q, int64_t ld_q, const void* k,
                     int64_t ld_k, const void* v, int64_t ld_v, const float* g, void* o, float* states, int32_t n_states, int32_t H,
                     int32_t dk, int32_t dv, int32_t dtype, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                     void* stream) {
    int32_t rc = la_check(n_seq, max_len, n_rows, H, dk, dv, dtype);
    if (rc != HARTS_OK) return rc;
    if (n_states < 0) return HARTS_EINVAL;
    if (n_seq == 0) return HARTS_OK;
    if (!seq_begin || !seq_len || !in_state || !out_state) return HARTS_EINVAL;
    if (n_states > 0 && (!states || !aligned16(states))) return HARTS_EINVAL;
    harts::GenLaArgs a = la_sizes(n_seq, max_len, n_rows, H, dk, dtype);
    const int64_t width = (int64_t)H * dk, elem = dtype == HARTS_FP32 ? 4 : 2;
    if (n_rows > 0 && max_len > 0) {
        if (!rows_ok(k, ld_k, width, elem) || !rows_ok(v, ld_v, width, elem) || !g) return HARTS_EINVAL;
        if (o && (!aligned16(o) || !rows_ok(q, ld_q, width, elem))) return HARTS_EINVAL;
    }
    a.seq_begin = seq_begin;
    a.seq_len = seq_len;
    a.in_state = in_state;
    a.out_state = out_state;
    a.q = q;
    a.k = k;
    a.v = v;
    a.ld_q = ld_q;
    a.ld_k = ld_k;
    a.ld_v = ld_v;
    a.g = g;
    a.o = o;
    a.states = states;
    a.n_states = n_states;
    a.workspace = workspace;
    a.dev_status = dev_status;
    a.stream = static_cast<cudaStream_t>(stream);
    if (n_rows == 0 || !harts::gen_la_chunked(a)) return harts::gen_la_walk(a);
    if (!workspace || !aligned16(workspace) || workspace_bytes < harts::gen_la_chunk_bytes(a)) return HARTS_EINVAL;
    return harts::gen_la_chunks(a);
}

}  // extern "C"
