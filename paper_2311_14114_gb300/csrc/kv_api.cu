// C-ABI entry points of the key / value cache: argument validation on the
// host, geometry, and the kernels' launches.
#include <cmath>
#include <cstring>

#include "kv_internal.h"

namespace soniq {

namespace {

soniq_status make_side(const soniq_kv_rows* r, KvSide* s) {
    if (r == nullptr || r->D < 1 || (r->n_groups != 1 && r->n_groups != 2)) return SONIQ_ERR_INVALID_ARG;
    if (r->count[0] < 1 || r->count[1] < 0 || (int64_t)r->count[0] + r->count[1] != r->D) return SONIQ_ERR_INVALID_ARG;
    if ((r->n_groups == 2) != (r->count[1] > 0)) return SONIQ_ERR_INVALID_ARG;
    if (r->D > kKvMaxCodes) return SONIQ_ERR_UNSUPPORTED;
    int off = 0, codes = 0;
    for (int g = 0; g < 2; ++g) {
        const bool used = g < r->n_groups;
        const int n = used ? r->bits[g] : 8;
        if (n < 1 || n > 8) return SONIQ_ERR_INVALID_ARG;
        if (n != 2 && n != 4 && n != 8) return SONIQ_ERR_UNSUPPORTED;
        s->count[g] = used ? r->count[g] : 0;
        s->nb[g] = (s->count[g] + 31) / 32;
        s->bits[g] = n;
        s->off[g] = off;
        off += s->nb[g] * 4 * n;
        codes += 32 * s->nb[g];
    }
    if (codes > kKvMaxCodes) return SONIQ_ERR_UNSUPPORTED;
    s->D = r->D;
    s->ng = r->n_groups;
    s->row_bytes = (off + 15) / 16 * 16;
    s->perm = r->perm;
    return SONIQ_OK;
}

bool is_permutation(const int32_t* p, int heads, int D) {
    for (int h = 0; h < heads; ++h) {
        bool seen[kKvMaxCodes] = {};
        for (int i = 0; i < D; ++i) {
            const int32_t c = p[(int64_t)h * D + i];
            if (c < 0 || c >= D || seen[c]) return false;
            seen[c] = true;
        }
    }
    return true;
}

bool aligned_to(const void* p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }

soniq_status check_cache(const soniq_kv_cache* c, KvGeom* geo) {
    const soniq_status st = make_kv_geom(c, geo);
    if (st != SONIQ_OK) return st;
    for (const KvSide& s : geo->s) {
        if (s.codes == nullptr || s.scales == nullptr || s.perm == nullptr) return SONIQ_ERR_INVALID_ARG;
        if (!aligned_to(s.codes, 16) || !aligned_to(s.scales, 16) || !aligned_to(s.perm, 4)) return SONIQ_ERR_ALIGNMENT;
    }
    return SONIQ_OK;
}

soniq_status launched(cudaError_t e) {
    return e == cudaSuccess ? SONIQ_OK : (e == cudaErrorNotSupported ? SONIQ_ERR_UNSUPPORTED : SONIQ_ERR_CUDA);
}

// Sizes whose products with heads and pages stay far inside 63 bits.
constexpr int64_t kMaxTokens = (int64_t)1 << 40;
constexpr int32_t kMaxHeads = 4096;

}  // namespace

soniq_status make_kv_geom(const soniq_kv_cache* c, KvGeom* geo) {
    if (c == nullptr || c->heads < 1 || c->n_pages < 1) return SONIQ_ERR_INVALID_ARG;
    if (c->dtype != SONIQ_OUT_F16 && c->dtype != SONIQ_OUT_BF16) return SONIQ_ERR_INVALID_ARG;
    if (c->page_size < 1 || (c->page_size & (c->page_size - 1)) != 0) return SONIQ_ERR_INVALID_ARG;
    if (c->page_size < 16 || c->page_size > 256) return SONIQ_ERR_UNSUPPORTED;
    if (c->heads > kMaxHeads || c->n_pages > 2147483647) return SONIQ_ERR_UNSUPPORTED;
    soniq_status st = make_side(&c->k, &geo->s[0]);
    if (st == SONIQ_OK) st = make_side(&c->v, &geo->s[1]);
    if (st != SONIQ_OK) return st;
    geo->s[0].codes = c->k_codes;
    geo->s[0].scales = static_cast<uint16_t*>(c->k_scales);
    geo->s[1].codes = c->v_codes;
    geo->s[1].scales = static_cast<uint16_t*>(c->v_scales);
    geo->heads = c->heads;
    geo->page = c->page_size;
    geo->page_shift = 0;
    while ((1 << geo->page_shift) < geo->page) ++geo->page_shift;
    geo->bf16 = c->dtype == SONIQ_OUT_BF16;
    geo->n_pages = c->n_pages;
    return SONIQ_OK;
}

}  // namespace soniq

using namespace soniq;

extern "C" {

int64_t soniq_kv_row_bytes(const soniq_kv_rows* rows) {
    KvSide s;
    return make_side(rows, &s) == SONIQ_OK ? s.row_bytes : -1;
}

soniq_status soniq_kv_validate(const soniq_kv_cache* cache, const int32_t* k_perm, const int32_t* v_perm) {
    KvGeom geo;
    const soniq_status st = make_kv_geom(cache, &geo);
    if (st != SONIQ_OK) return st;
    if (k_perm != nullptr && !is_permutation(k_perm, geo.heads, geo.s[0].D)) return SONIQ_ERR_INVALID_ARG;
    if (v_perm != nullptr && !is_permutation(v_perm, geo.heads, geo.s[1].D)) return SONIQ_ERR_INVALID_ARG;
    return SONIQ_OK;
}

soniq_status soniq_kv_write(const soniq_kv_cache* cache, const void* K, int64_t k_token_stride, int64_t k_head_stride,
                            const void* V, int64_t v_token_stride, int64_t v_head_stride, const int64_t* slots,
                            int64_t n, soniq_stream_t stream) {
    KvGeom geo;
    const soniq_status st = check_cache(cache, &geo);
    if (st != SONIQ_OK) return st;
    if (n < 0) return SONIQ_ERR_INVALID_ARG;
    if (n > kMaxTokens) return SONIQ_ERR_UNSUPPORTED;
    if (n == 0) return SONIQ_OK;
    if (K == nullptr || V == nullptr || slots == nullptr) return SONIQ_ERR_INVALID_ARG;
    if (!aligned_to(K, 2) || !aligned_to(V, 2) || !aligned_to(slots, 8)) return SONIQ_ERR_ALIGNMENT;
    unsigned* err = device_error_word();
    if (err == nullptr) return SONIQ_ERR_CUDA;
    const KvRowsArg k{static_cast<const uint16_t*>(K), k_token_stride, k_head_stride};
    const KvRowsArg v{static_cast<const uint16_t*>(V), v_token_stride, v_head_stride};
    return launched(launch_kv_write(geo, k, v, slots, n, err, reinterpret_cast<cudaStream_t>(stream)));
}

soniq_status soniq_kv_read(const soniq_kv_cache* cache, const int64_t* slots, int64_t n, void* K, void* V,
                           soniq_stream_t stream) {
    KvGeom geo;
    const soniq_status st = check_cache(cache, &geo);
    if (st != SONIQ_OK) return st;
    if (n < 0) return SONIQ_ERR_INVALID_ARG;
    if (n > kMaxTokens) return SONIQ_ERR_UNSUPPORTED;
    if (n == 0 || (K == nullptr && V == nullptr)) return SONIQ_OK;
    if (slots == nullptr) return SONIQ_ERR_INVALID_ARG;
    if (!aligned_to(K, 2) || !aligned_to(V, 2) || !aligned_to(slots, 8)) return SONIQ_ERR_ALIGNMENT;
    unsigned* err = device_error_word();
    if (err == nullptr) return SONIQ_ERR_CUDA;
    return launched(launch_kv_read(geo, slots, n, static_cast<uint16_t*>(K), static_cast<uint16_t*>(V), err,
                                   reinterpret_cast<cudaStream_t>(stream)));
}

int64_t soniq_kv_attend_scratch_bytes(const soniq_kv_cache* cache, int32_t B, int32_t T, int32_t q_heads) {
    KvGeom geo;
    if (make_kv_geom(cache, &geo) != SONIQ_OK || B < 0 || T < 0 || q_heads < 1 || q_heads % geo.heads != 0) return -1;
    return kv_attend_scratch(geo, B, T, q_heads / geo.heads);
}

soniq_status soniq_kv_attend(const soniq_kv_cache* cache, const void* Q, int64_t q_seq_stride, int64_t q_token_stride,
                             int64_t q_head_stride, const int32_t* page_table, int64_t table_stride, int32_t max_pages,
                             const int32_t* lengths, const uint8_t* mask, int64_t mask_stride, int32_t B, int32_t T,
                             int32_t q_heads, float scale, void* out, void* scratch, size_t scratch_bytes,
                             soniq_stream_t stream) {
    KvGeom geo;
    const soniq_status st = check_cache(cache, &geo);
    if (st != SONIQ_OK) return st;
    if (B < 0 || T < 0 || max_pages < 0 || q_heads < 1 || q_heads % geo.heads != 0 || !std::isfinite(scale))
        return SONIQ_ERR_INVALID_ARG;
    // rows and positions are indexed in 32 bits
    if ((int64_t)T * q_heads > (1 << 28) || (int64_t)max_pages * geo.page > (1 << 30)) return SONIQ_ERR_UNSUPPORTED;
    if (B == 0 || T == 0) return SONIQ_OK;
    if (Q == nullptr || lengths == nullptr || out == nullptr || (page_table == nullptr && max_pages > 0))
        return SONIQ_ERR_INVALID_ARG;
    if (!aligned_to(Q, 2) || !aligned_to(out, 2) || !aligned_to(page_table, 4) || !aligned_to(lengths, 4))
        return SONIQ_ERR_ALIGNMENT;
    const int64_t need = kv_attend_scratch(geo, B, T, q_heads / geo.heads);
    if (need > 0) {
        if (scratch == nullptr || (int64_t)scratch_bytes < need) return SONIQ_ERR_INVALID_ARG;
        if (!aligned_to(scratch, 16)) return SONIQ_ERR_ALIGNMENT;
    }
    unsigned* err = device_error_word();
    if (err == nullptr) return SONIQ_ERR_CUDA;
    KvAttendArgs a{static_cast<const uint16_t*>(Q), q_seq_stride, q_token_stride, q_head_stride, page_table,
                   table_stride, max_pages, lengths, mask, mask_stride, B, T, q_heads / geo.heads, scale,
                   static_cast<uint16_t*>(out), scratch, err, 0};
    return launched(launch_kv_attend(geo, a, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
