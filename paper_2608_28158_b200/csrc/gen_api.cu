// C entry points of sampling on rollout trees: argument checks and the choice of the kernel.
#include <cfloat>

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

// ---- cache ---------------------------------------------------------------------------------------------------------------------
static int32_t cache_check(int64_t n, int32_t n_pages, int32_t page, int32_t Hkv, int32_t d, int32_t type) {
    if (type != HARTS_BF16 && type != HARTS_E4M3) return HARTS_EUNSUPPORTED;
    if (d != 128) return HARTS_EUNSUPPORTED;
    if (n < 0 || n > INT32_MAX || n_pages < 0 || Hkv < 1 || Hkv > 65535 || (page != 16 && page != 32 && page != 64 && page != 128)) return HARTS_EINVAL;
    if ((int64_t)n_pages * page > INT32_MAX || (int64_t)n_pages * Hkv > INT32_MAX) return HARTS_EINVAL;
    return HARTS_OK;
}
static bool cache_ok(const harts::GenCache& c) {
    if (c.n_pages == 0) return true;
    if (!c.k || !c.v || !aligned16(c.k) || !aligned16(c.v)) return false;
    return c.type == HARTS_BF16 || (c.k_exp && c.v_exp && aligned16(c.k_exp) && aligned16(c.v_exp));
}

int32_t harts_gen_cache_write(int64_t n, const int32_t* slot, const void* k, int64_t ld_k, const void* v, int64_t ld_v, void* k_cache,
                              void* v_cache, uint8_t* k_exp, uint8_t* v_exp, int32_t n_pages, int32_t page, int32_t Hkv, int32_t d,
                              int32_t cache_type, int32_t* dev_status, void* stream) {
    const int32_t rc = cache_check(n, n_pages, page, Hkv, d, cache_type);
    if (rc != HARTS_OK) return rc;
    const harts::GenCache c{k_cache, v_cache, k_exp, v_exp, n_pages, page, Hkv, cache_type};
    if (n == 0) return HARTS_OK;
    if (!slot || !cache_ok(c) || !rows_ok(k, ld_k, (int64_t)Hkv * d, 2) || !rows_ok(v, ld_v, (int64_t)Hkv * d, 2)) return HARTS_EINVAL;
    return harts::gen_cache_write(c, {n, slot, const_cast<void*>(k), const_cast<void*>(v), ld_k, ld_v, dev_status, static_cast<cudaStream_t>(stream)});
}

int32_t harts_gen_cache_read(int64_t n, const int32_t* slot, const void* k_cache, const void* v_cache, const uint8_t* k_exp,
                             const uint8_t* v_exp, void* k, void* v, int32_t n_pages, int32_t page, int32_t Hkv, int32_t d,
                             int32_t cache_type, int32_t* dev_status, void* stream) {
    const int32_t rc = cache_check(n, n_pages, page, Hkv, d, cache_type);
    if (rc != HARTS_OK) return rc;
    const harts::GenCache c{const_cast<void*>(k_cache), const_cast<void*>(v_cache), const_cast<uint8_t*>(k_exp), const_cast<uint8_t*>(v_exp),
                            n_pages, page, Hkv, cache_type};
    if (n == 0 || (!k && !v)) return HARTS_OK;
    if (!slot || !cache_ok(c) || !aligned16(k) || !aligned16(v)) return HARTS_EINVAL;
    return harts::gen_cache_read(c, {n, slot, k, v, 0, 0, dev_status, static_cast<cudaStream_t>(stream)});
}

// ---- attention -------------------------------------------------------------------------------------------------------------------
static bool index_ok(const int32_t* hi) {
    using namespace harts::gen_attn;
    return hi && hi[N_Q] >= 0 && hi[HKV] >= 1 && hi[HQ] >= hi[HKV] && hi[WORDS] >= HARTS_GEN_ATTN_HEADER_WORDS && hi[N_PARTS] >= 0;
}

int32_t harts_gen_attn_workspace_bytes(const int32_t* host_index, size_t* bytes) {
    using namespace harts::gen_attn;
    if (!bytes || !index_ok(host_index)) return HARTS_EINVAL;
    *bytes = host_index[MERGED] ? (size_t)host_index[N_PARTS] * host_index[HKV] * (128 + 1) * sizeof(float) : 0;
    return HARTS_OK;
}

int32_t harts_gen_attn(const int32_t* host_index, const int32_t* dev_index, const void* q, int64_t ld_q, const void* k_cache,
                       const void* v_cache, const uint8_t* k_exp, const uint8_t* v_exp, int32_t n_pages, int32_t cache_type,
                       const int32_t* q_pos, void* o, float* lse, float scale, void* workspace, size_t workspace_bytes,
                       int32_t* dev_status, void* stream) {
    using namespace harts::gen_attn;
    size_t need = 0;
    constexpr float MOST_SCALE = (float)(FLT_MAX * 0.6931471805599453);            // exponents are base 2: scale / ln 2 has to be a number too
    if (harts_gen_attn_workspace_bytes(host_index, &need) != HARTS_OK || !dev_index || !aligned16(dev_index) || !(scale > 0.f && scale <= MOST_SCALE)) return HARTS_EINVAL;
    const int32_t rc = cache_check(host_index[N_Q], n_pages, host_index[PAGE], host_index[HKV], 128, cache_type);
    if (rc != HARTS_OK) return rc;
    if (host_index[N_Q] == 0) return HARTS_OK;
    const harts::GenCache c{const_cast<void*>(k_cache), const_cast<void*>(v_cache), const_cast<uint8_t*>(k_exp), const_cast<uint8_t*>(v_exp),
                            n_pages, host_index[PAGE], host_index[HKV], cache_type};
    if (host_index[MAX_PAGE] >= n_pages || !cache_ok(c) || !q_pos || !o || !lse || !aligned16(o) || !rows_ok(q, ld_q, (int64_t)host_index[HQ] * 128, 2))
        return HARTS_EINVAL;
    if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return HARTS_EINVAL;
    return harts::gen_attn_launch(host_index, dev_index, q, ld_q, c, q_pos, o, lse, scale, workspace, dev_status, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
