// C ABI of the calls on a cache of many sequences (pages, 4-bit keys and values): argument checking and launches.
#include <cstring>
#include <initializer_list>

#include "internal.h"

namespace pevlm {

// Rows of one call: its blocks (64 rows of a head at most, see packed_kernel.cu) have to be counted in 31 bits.
static bool countable_rows(const pevlm_shape_t* s, int64_t n_rows) {
    return n_rows <= 1ll << 30 && (n_rows + 255) / 64 * 2 * s->num_kv_heads < 1ll << 31;
}

static int check_pages(const pevlm_pages_t* g) {
    if (!g || g->num_pages < 1 || g->num_seqs < 1 || g->max_pages < 1) return PEVLM_EINVAL;
    if (g->page_len != 16 && g->page_len != 32 && g->page_len != 64 && g->page_len != 128) return PEVLM_EUNSUPPORTED;
    if (static_cast<int64_t>(g->num_pages) * g->page_len >= 1ll << 31) return PEVLM_EINVAL;
    if (static_cast<int64_t>(g->max_pages) * g->page_len > 1ll << 30 || g->num_seqs > 1 << 20) return PEVLM_EINVAL;
    return PEVLM_OK;
}

static int page_shift(const pevlm_pages_t* g) { return __builtin_ctz(static_cast<unsigned>(g->page_len)); }

// So many int32, and whether two such arrays share memory.
struct Ints {
    const int32_t* at;
    int64_t n;
};
static bool overlap(const Ints& a, const Ints& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    return a.n > 0 && b.n > 0 && x < y + 4 * static_cast<uintptr_t>(b.n) && y < x + 4 * static_cast<uintptr_t>(a.n);
}

// Whether an output of a call on pages shares memory with one of its inputs or with another output.  (Every CTA reads all inputs while others write.)
static bool outputs_shared(std::initializer_list<Ints> outputs, std::initializer_list<Ints> inputs) {
    for (const Ints* out = outputs.begin(); out != outputs.end(); ++out) {
        for (const Ints& in : inputs)
            if (overlap(*out, in)) return true;
        for (const Ints* other = out + 1; other != outputs.end(); ++other)
            if (overlap(*out, *other)) return true;
    }
    return false;
}

// What the packed calls ask of a shape.
static int check_packed(const pevlm_shape_t* s, const pevlm_pages_t* g) {
    int rc = check_shape(s);
    if (rc == PEVLM_OK) rc = check_pages(g);
    if (rc != PEVLM_OK) return rc;
    // (the kernels count the cache in 2^32 units of 128 bytes)
    if (static_cast<double>(g->num_pages) * s->num_kv_heads * (g->page_len / 16) * 18 * s->head_dim >= 128.0 * 4294967295.0) return PEVLM_EUNSUPPORTED;
    return s->batch == 1 ? PEVLM_OK : PEVLM_EUNSUPPORTED;
}

}  // namespace pevlm

using namespace pevlm;

extern "C" {

int pevlm_pages_release(const pevlm_pages_t* g, const int32_t* finished, const int32_t* lens, const int32_t* page_table,
                        int32_t* free_list, const int32_t* free_count, int32_t* lens_out, int32_t* free_count_out, void* stream) {
    int rc = check_pages(g);
    if (rc != PEVLM_OK) return rc;
    if (!finished || !lens || !page_table || !free_list || !free_count || !lens_out || !free_count_out) return PEVLM_EINVAL;
    if (!aligned_to(finished, 4) || !aligned_to(lens, 4) || !aligned_to(page_table, 4) || !aligned_to(free_list, 4) ||
        !aligned_to(free_count, 4) || !aligned_to(lens_out, 4) || !aligned_to(free_count_out, 4))
        return PEVLM_EALIGN;
    const int64_t n = g->num_seqs;
    if (outputs_shared({{free_list, g->num_pages}, {lens_out, n}, {free_count_out, 1}}, {{finished, n}, {lens, n}, {page_table, n * g->max_pages}, {free_count, 1}})) return PEVLM_EINVAL;
    rc = check_device();
    if (rc != PEVLM_OK) return rc;
    ReleaseParams p{finished, lens, page_table, free_count, free_list, lens_out, free_count_out, g->num_pages, g->num_seqs, g->max_pages, page_shift(g)};
    const cudaError_t e = launch_release(p, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? PEVLM_OK : cuda_fail(e, "release launch");
}

int pevlm_pages_assign(const pevlm_pages_t* g, const int32_t* lens, const int32_t* new_lens, int32_t* page_table,
                       const int32_t* free_list, const int32_t* free_count, int32_t* lens_out, int32_t* free_count_out,
                       int32_t* row_start, int32_t* slots, int32_t* positions, int64_t max_rows, void* stream) {
    return pevlm_pages_assign_rows(g, lens, new_lens, page_table, free_list, free_count, lens_out, free_count_out, row_start, slots, positions, max_rows, max_rows, nullptr, stream);
}

int pevlm_pages_assign_rows(const pevlm_pages_t* g, const int32_t* lens, const int32_t* new_lens, int32_t* page_table,
                            const int32_t* free_list, const int32_t* free_count, int32_t* lens_out, int32_t* free_count_out,
                            int32_t* row_start, int32_t* slots, int32_t* positions, int64_t max_rows, int64_t n_rows, int32_t* key_lens,
                            void* stream) {
    int rc = check_pages(g);
    if (rc != PEVLM_OK) return rc;
    if (max_rows < 0 || max_rows > 1ll << 30 || n_rows < 0 || n_rows > max_rows) return PEVLM_EINVAL;
    if (!lens || !new_lens || !page_table || !free_list || !free_count || !lens_out || !free_count_out || !row_start) return PEVLM_EINVAL;
    if (max_rows > 0 && (!slots || !positions)) return PEVLM_EINVAL;
    if (!aligned_to(lens, 4) || !aligned_to(new_lens, 4) || !aligned_to(page_table, 4) || !aligned_to(free_list, 4) ||
        !aligned_to(free_count, 4) || !aligned_to(lens_out, 4) || !aligned_to(free_count_out, 4) || !aligned_to(row_start, 4) ||
        !aligned_to(slots, 16) || !aligned_to(positions, 16) || !aligned_to(key_lens, 4))
        return PEVLM_EALIGN;
    const int64_t n = g->num_seqs;
    if (outputs_shared({{page_table, n * g->max_pages}, {lens_out, n}, {free_count_out, 1}, {row_start, n + 1}, {slots, max_rows}, {positions, max_rows}, {key_lens, key_lens ? n : 0}},
                       {{lens, n}, {new_lens, n}, {free_list, g->num_pages}, {free_count, 1}}))
        return PEVLM_EINVAL;
    rc = check_device();
    if (rc != PEVLM_OK) return rc;
    AssignParams p{lens, new_lens, free_list, free_count, page_table, lens_out, free_count_out, row_start, slots, positions, key_lens,
                   max_rows, n_rows, 0, g->num_pages, g->num_seqs, g->max_pages, page_shift(g)};
    const cudaError_t e = launch_assign(p, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? PEVLM_OK : cuda_fail(e, "assign launch");
}

size_t pevlm_packed_cache_bytes(const pevlm_shape_t* s, const pevlm_pages_t* g) {
    if (check_packed(s, g) != PEVLM_OK) return 0;
    return static_cast<size_t>(g->num_pages) * s->num_kv_heads * (g->page_len / 16) * 18 * s->head_dim;
}

int pevlm_packed_store(const pevlm_shape_t* s, const pevlm_pages_t* g, const void* k, const void* v, int64_t k_stride,
                       int64_t v_stride, const int32_t* slots, int64_t n_rows, void* cache, void* stream) {
    int rc = check_packed(s, g);
    if (rc != PEVLM_OK) return rc;
    if (n_rows < 0 || !countable_rows(s, n_rows)) return PEVLM_EINVAL;
    if (!cache || (n_rows > 0 && (!k || !v || !slots))) return PEVLM_EINVAL;
    const int64_t row = static_cast<int64_t>(s->num_kv_heads) * s->head_dim;
    if (k_stride == 0) k_stride = row;
    if (v_stride == 0) v_stride = row;
    if (n_rows > 1 && (k_stride < row || v_stride < row || k_stride > 1ll << 32 || v_stride > 1ll << 32)) return PEVLM_EINVAL;
    if (!aligned_to(k, 16) || !aligned_to(v, 16) || !aligned_to(cache, 16) || !aligned_to(slots, 4) || k_stride % 8 || v_stride % 8) return PEVLM_EALIGN;
    if (n_rows == 0) return PEVLM_OK;
    rc = check_device();
    if (rc != PEVLM_OK) return rc;
    PackedRows p;
    memset(&p, 0, sizeof(p));
    p.k = static_cast<const __nv_bfloat16*>(k);
    p.v = static_cast<const __nv_bfloat16*>(v);
    p.k_stride = k_stride; p.v_stride = v_stride;
    p.cache = static_cast<uint8_t*>(cache);
    p.slots = slots;
    p.n_rows = n_rows;
    p.Hkv = s->num_kv_heads; p.n_slots = g->num_pages * g->page_len; p.page_shift = page_shift(g);
    const cudaError_t e = launch_packed_store(p, s->head_dim, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? PEVLM_OK : cuda_fail(e, "packed store launch");
}

int pevlm_packed_load(const pevlm_shape_t* s, const pevlm_pages_t* g, const void* cache, const int32_t* slots, int64_t n_rows,
                      void* k_out, void* v_out, void* stream) {
    int rc = check_packed(s, g);
    if (rc != PEVLM_OK) return rc;
    if (n_rows < 0 || !countable_rows(s, n_rows)) return PEVLM_EINVAL;
    if (!cache || (n_rows > 0 && (!k_out || !v_out || !slots))) return PEVLM_EINVAL;
    if (!aligned_to(k_out, 32) || !aligned_to(v_out, 32) || !aligned_to(cache, 16) || !aligned_to(slots, 4)) return PEVLM_EALIGN;
    if (n_rows == 0) return PEVLM_OK;
    rc = check_device();
    if (rc != PEVLM_OK) return rc;
    PackedRows p;
    memset(&p, 0, sizeof(p));
    p.cache = static_cast<uint8_t*>(const_cast<void*>(cache));
    p.slots = slots;
    p.n_rows = n_rows;
    p.k_out = static_cast<__nv_bfloat16*>(k_out);
    p.v_out = static_cast<__nv_bfloat16*>(v_out);
    p.Hkv = s->num_kv_heads; p.n_slots = g->num_pages * g->page_len; p.page_shift = page_shift(g);
    const cudaError_t e = launch_packed_load(p, s->head_dim, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? PEVLM_OK : cuda_fail(e, "packed load launch");
}

// n_rows rows of a call, at most max_rows of one sequence.
static int check_rows(const pevlm_shape_t* s, int64_t n_rows, int64_t max_rows) {
    if (n_rows < 0 || max_rows < 0 || max_rows > n_rows) return PEVLM_EINVAL;
    return n_rows * (s->num_q_heads / s->num_kv_heads) <= 1ll << 30 ? PEVLM_OK : PEVLM_EINVAL;
}

size_t pevlm_packed_workspace_bytes(const pevlm_shape_t* s, const pevlm_pages_t* g, int64_t n_rows, int64_t max_rows) {
    if (check_packed(s, g) != PEVLM_OK || check_rows(s, n_rows, max_rows) != PEVLM_OK) return 0;
    return kStatusBytes + packed_attn_workspace_bytes(s->head_dim, max_rows * (s->num_q_heads / s->num_kv_heads));
}

int pevlm_packed_attn(const pevlm_shape_t* s, const pevlm_pages_t* g, int32_t window, const void* q, int64_t q_stride, const void* cache,
                      const int32_t* page_table, const int32_t* lens, const int32_t* row_start, int64_t n_rows, int64_t max_rows, void* o,
                      float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_packed(s, g);
    if (rc == PEVLM_OK) rc = check_rows(s, n_rows, max_rows);
    if (rc != PEVLM_OK) return rc;
    if (window < 0) return PEVLM_EINVAL;
    if (!cache || !page_table || !lens || !row_start || (n_rows > 0 && (!q || !o))) return PEVLM_EINVAL;
    const int64_t row = static_cast<int64_t>(s->num_q_heads) * s->head_dim;
    if (q_stride == 0) q_stride = row;
    if (n_rows > 1 && (q_stride < row || q_stride > 1ll << 32)) return PEVLM_EINVAL;
    if (!aligned_to(q, 16) || !aligned_to(cache, 16) || !aligned_to(page_table, 4) || !aligned_to(lens, 4) || !aligned_to(row_start, 4) ||
        !aligned_to(o, 32) || !aligned_to(lse, 16) || q_stride % 8)
        return PEVLM_EALIGN;
    if (!workspace || workspace_bytes < pevlm_packed_workspace_bytes(s, g, n_rows, max_rows)) return PEVLM_EWORKSPACE;
    if (!aligned_to(workspace, 256)) return PEVLM_EALIGN;
    if (n_rows == 0) return PEVLM_OK;
    rc = check_device();
    if (rc != PEVLM_OK) return rc;
    PackedAttnParams p;
    memset(&p, 0, sizeof(p));
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.cache = static_cast<const uint8_t*>(cache);
    p.page_table = page_table; p.lens = lens; p.row_start = row_start;
    p.o = static_cast<__nv_bfloat16*>(o);
    p.lse = lse;
    p.hdr = static_cast<WorkspaceHeader*>(workspace);
    p.joins = reinterpret_cast<PackedJoin*>(static_cast<uint8_t*>(workspace) + kStatusBytes);
    p.part = reinterpret_cast<float*>(p.joins + kNumSms);
    p.q_stride = q_stride;
    p.n_rows = static_cast<int32_t>(n_rows);
    p.num_seqs = g->num_seqs; p.num_pages = g->num_pages; p.max_pages = g->max_pages; p.page_shift = page_shift(g);
    p.Hq = s->num_q_heads; p.Hkv = s->num_kv_heads; p.G = p.Hq / p.Hkv;
    p.window = window < 1 << 30 ? window : 1 << 30;  // no sequence is longer
    p.sink = s->sink_len;
    p.div_g = make_divisor(p.G);
    p.scale_log2 = resolve_scale(s) * 1.4426950408889634f;
    const cudaError_t e = launch_packed_attn(p, s->head_dim, max_rows, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? PEVLM_OK : cuda_fail(e, "packed attention launch");
}

}  // extern "C"
