// A paged cache of keys and values and what works on it: appending (norm, rotation, page bounds), attention of chunks and single
// tokens over all of a sequence or over listed pages, and the selection of those pages by a score on their bounds.
// include/ada.h says what each call computes.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <limits.h>
#include <math.h>
#include <mutex>

#include "../../include/ada.h"
#include "ada_hooks.hpp"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int MAX_TOKENS = 1 << 26;                        // positions of a sequence
constexpr long long MAX_SLOT_STRIDE = 1 << 25;             // 16 rows within 32-bit byte offsets
constexpr int NOWHERE = 1 << 30;                           // a position that no row sees

// What every kernel here is told about the cache and the new tokens.
struct PagedArgs {
    void *K, *V, *bounds;
    long long page_stride, head_stride, slot_stride;
    int pages, lg, H, H_kv, G;                             // page = 2^lg tokens, G = H / H_kv
    const int32_t* table;
    long long table_stride;
    int max_pages;
    const int32_t *start, *past;
    int B, rows, longest;
    int32_t* status;
    int causal;
};

struct Seq { int row0, n, past, len; };                    // len = past + n; n = 0 also for a sequence that is refused

__device__ inline void raise(const PagedArgs& p, int code) { atomicMax(p.status, code); }

__device__ inline Seq paged_seq(const PagedArgs& p, int b) {
    const int s0 = p.start[b], s1 = p.start[b + 1], past = p.past[b];
    const bool ok = s0 >= 0 && s1 >= s0 && s1 <= p.rows && s1 - s0 <= p.longest && past >= 0 &&
                    (long long)past + (s1 - s0) <= ((long long)p.max_pages << p.lg);
    if (!ok) {
        raise(p, ADA_ERR_SHAPE);
        return {0, 0, 0, 0};
    }
    return {s0, s1 - s0, past, past + s1 - s0};
}

// The sequence that `row` (the same in all lanes) belongs to: as many as end at or in front of it.  B where it is behind the last.
__device__ inline int paged_find(const PagedArgs& p, int row) {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int m = __popcll(__builtin_amdgcn_ballot_w64(b0 + lane < p.B && p.start[min(b0 + lane, p.B - 1) + 1] <= row));
        n += m;
        if (m < 64) break;
    }
    return n;
}

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ inline uint32_t bf16_pair(float a, float b) {   // round to nearest even
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// maximum over the four lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ inline float max_over_groups(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float sum_over_groups(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Workgroups go to the eight XCDs in turn by their number; this gives every XCD a contiguous eighth of the work, so that what
// neighbouring pieces share (a head's keys, a token's pages) is fetched into one L2.
__device__ inline int by_xcd(int id, int n) { return n % 8 ? id : (id % 8) * (n / 8) + id / 8; }

#include "ada_paged_append.hpp"
#include "ada_paged_attn.hpp"
#include "ada_paged_select.hpp"

// ------------------------------------------------------------------------------------------------
// host side

int elem_size(int dtype) { return dtype == ADA_BF16 ? 2 : 4; }

// Everything the host can see of cache and chunk; fills `a`.
int paged_args(const ada_paged_cache* c, const ada_paged_chunk* k, int H, int32_t* status, unsigned flags, PagedArgs& a) {
    if (!c || !k || !c->K || !c->V || !k->table || !k->start || !k->past || !status) return ADA_ERR_NULL;
    if (c->dtype != ADA_F32 && c->dtype != ADA_BF16) return ADA_ERR_DTYPE;
    const int esz = elem_size(c->dtype);
    const bool dh_ok = c->d_h == 64 || c->d_h == 128 || (c->d_h == 256 && c->dtype == ADA_BF16);
    if (!dh_ok || c->pages < 1 || c->H_kv < 1 || H < 1 || H > 65535 || H % c->H_kv != 0) return ADA_ERR_SHAPE;
    if (c->page < 16 || c->page > 256 || (c->page & (c->page - 1)) != 0) return ADA_ERR_SHAPE;
    if (c->slot_stride < c->d_h || c->head_stride < c->d_h || c->page_stride < c->d_h) return ADA_ERR_SHAPE;
    if (c->slot_stride * esz % 16 || c->head_stride * esz % 16 || c->page_stride * esz % 16) return ADA_ERR_SHAPE;
    if (c->slot_stride > MAX_SLOT_STRIDE) return ADA_ERR_SHAPE;
    if ((uintptr_t)c->K % 16 || (uintptr_t)c->V % 16 || (uintptr_t)c->bounds % 16) return ADA_ERR_SHAPE;
    if (k->B < 1 || k->B > ADA_MAX_BATCH || k->rows < 0 || k->rows > ADA_MAX_T || k->longest < 0 || k->longest > k->rows) return ADA_ERR_SHAPE;
    if (k->rows > 0 && k->longest < 1) return ADA_ERR_SHAPE;
    if (k->max_pages < 1 || (long long)k->max_pages * c->page > MAX_TOKENS || (k->B > 1 && k->table_stride < k->max_pages)) return ADA_ERR_SHAPE;
    if ((long long)k->rows * (H / c->H_kv) > 1 << 30) return ADA_ERR_SHAPE;
    int lg = 4;
    while ((1 << lg) < c->page) ++lg;
    a = {c->K, c->V, c->bounds, c->page_stride, c->head_stride, c->slot_stride, c->pages, lg, H, c->H_kv, H / c->H_kv,
         k->table, k->table_stride, k->max_pages, k->start, k->past, k->B, k->rows, k->longest, status,
         (flags & ADA_FLAG_ATTN_CAUSAL) ? 1 : 0};
    return ADA_OK;
}

// Rows of `heads` heads that 16-byte loads and stores can take.
bool rows_ok(const void* X, int64_t ld, int64_t width, int esz) { return (uintptr_t)X % 16 == 0 && ld >= width && ld * esz % 16 == 0; }

// f(In{}, std::integral_constant<int, d_h>{}) for the cache's types
template <typename F>
int paged_dispatch(int dtype, int d_h, F&& f) {
    hipError_t e;
    if (dtype == ADA_BF16)
        e = d_h == 64 ? f(uint16_t(), Const<64>()) : d_h == 128 ? f(uint16_t(), Const<128>()) : f(uint16_t(), Const<256>());
    else
        e = d_h == 64 ? f(float(), Const<64>()) : f(float(), Const<128>());
    return e == hipSuccess ? ADA_OK : ADA_ERR_DEVICE;
}

int attend(const ada_paged_cache* cache, const ada_paged_chunk* chunk, const void* Q, int H, int64_t ldq, const int32_t* pages,
           const int32_t* counts, int budget, void* out, int64_t ld_out, int32_t* status, void* ws, size_t ws_bytes, void* stream,
           unsigned flags) {
    AttendArgs a;
    if (int e = paged_args(cache, chunk, H, status, flags, a.p)) return e;
    if (!Q || !out || !ws) return ADA_ERR_NULL;
    const int esz = elem_size(cache->dtype);
    const int64_t width = (int64_t)H * cache->d_h;
    if (!rows_ok(Q, ldq, width, esz) || !rows_ok(out, ld_out, width, esz)) return ADA_ERR_SHAPE;
    if (ws_bytes < ada_paged_workspace_bytes(cache, chunk, H) || (uintptr_t)ws % 256) return ADA_ERR_WORKSPACE;
    if (chunk->rows == 0) return ADA_OK;
    a.Q = Q; a.ldq = ldq; a.out = out; a.ld_out = ld_out;
    a.sc2 = (float)(1.4426950408889634 / sqrt((double)cache->d_h));
    a.list = pages; a.count = counts; a.budget = budget;
    return paged_dispatch(cache->dtype, cache->d_h, [&](auto in, auto dh) {
        return launch_attend<decltype(in), decltype(dh)::value>(a, ws, (hipStream_t)stream);
    });
}

}  // namespace

extern "C" {

size_t ada_paged_workspace_bytes(const ada_paged_cache* cache, const ada_paged_chunk* chunk, int H) {
    PagedArgs a;
    int32_t unused = 0;
    if (paged_args(cache, chunk, H, &unused, 0, a) != ADA_OK) return 0;
    const size_t attention = attend_ws(a, cache->d_h, cache->dtype).bytes;
    const size_t selection = a.bounds && a.max_pages <= ADA_SELECT_MAX_PAGES ? ADA_PAGED_ZERO_BYTES + select_ws(a).bytes : 0;
    return attention > selection ? attention : selection;
}

int ada_cache_append(const ada_paged_cache* cache, const ada_paged_chunk* chunk, const void* Q, int64_t ldq, const void* K,
                     int64_t ldk, const void* V, int64_t ldv, int H, const void* q_norm, const void* k_norm, float eps,
                     const float* rope, int rot, int rope_len, void* q_out, int64_t ldq_out, int32_t* status, void* stream,
                     unsigned flags) {
    AppendArgs a;
    if (int e = paged_args(cache, chunk, H, status, flags, a.p)) return e;
    if (!K || !V || (Q == nullptr) != (q_out == nullptr)) return ADA_ERR_NULL;
    const int esz = elem_size(cache->dtype), d_h = cache->d_h;
    const int64_t width = (int64_t)H * d_h, width_kv = (int64_t)cache->H_kv * d_h;
    if (!rows_ok(K, ldk, width_kv, esz) || !rows_ok(V, ldv, width_kv, esz)) return ADA_ERR_SHAPE;
    if (Q && (!rows_ok(Q, ldq, width, esz) || !rows_ok(q_out, ldq_out, width, esz))) return ADA_ERR_SHAPE;
    if ((uintptr_t)q_norm % 16 || (uintptr_t)k_norm % 16 || (uintptr_t)rope % 16) return ADA_ERR_SHAPE;
    if (rope && (rot < 16 || rot > d_h || rot % 16 || rope_len < 1)) return ADA_ERR_SHAPE;
    if ((q_norm || k_norm) && !(eps >= 0.f && eps < INFINITY)) return ADA_ERR_SHAPE;
    if (chunk->rows == 0) return ADA_OK;
    a.Q = Q; a.ldq = ldq; a.Kn = K; a.ldk = ldk; a.Vn = V; a.ldv = ldv;
    a.q_norm = q_norm; a.k_norm = k_norm; a.eps = eps; a.rope = rope; a.rot = rope ? rot : 0; a.rope_len = rope_len;
    a.q_out = q_out; a.ldq_out = ldq_out; a.pairs = (flags & ADA_FLAG_ROPE_PAIRS) ? 1 : 0;
    return paged_dispatch(cache->dtype, d_h, [&](auto in, auto dh) {
        return launch_append<decltype(in), decltype(dh)::value>(a, (hipStream_t)stream);
    });
}

int ada_attention_paged(const ada_paged_cache* cache, const ada_paged_chunk* chunk, const void* Q, int H, int64_t ldq, void* out,
                        int64_t ld_out, int32_t* status, void* ws, size_t ws_bytes, void* stream, unsigned flags) {
    return attend(cache, chunk, Q, H, ldq, nullptr, nullptr, 0, out, ld_out, status, ws, ws_bytes, stream, flags);
}

int ada_attention_pages(const ada_paged_cache* cache, const ada_paged_chunk* chunk, const void* Q, int H, int64_t ldq,
                        const int32_t* pages, const int32_t* counts, int budget, void* out, int64_t ld_out, int32_t* status,
                        void* ws, size_t ws_bytes, void* stream, unsigned flags) {
    if (!pages || !counts) return ADA_ERR_NULL;
    if (budget < 1 || budget > MAX_TOKENS / 256) return ADA_ERR_SHAPE;
    return attend(cache, chunk, Q, H, ldq, pages, counts, budget, out, ld_out, status, ws, ws_bytes, stream, flags);
}

int ada_select_pages(const ada_paged_cache* cache, const ada_paged_chunk* chunk, const void* Q, int H, int64_t ldq, int budget,
                     int first, int last, int32_t* pages, int32_t* counts, int32_t* status, void* ws, size_t ws_bytes, void* stream,
                     unsigned flags) {
    SelectArgs a;
    if (int e = paged_args(cache, chunk, H, status, flags, a.p)) return e;
    if (!cache->bounds || !Q || !pages || !counts || !ws) return ADA_ERR_NULL;
    if (!rows_ok(Q, ldq, (int64_t)H * cache->d_h, elem_size(cache->dtype))) return ADA_ERR_SHAPE;
    if (budget < 1 || budget > MAX_TOKENS / 256 || first < 0 || last < 0 || first > budget || last > budget - first) return ADA_ERR_SHAPE;
    if (chunk->max_pages > ADA_SELECT_MAX_PAGES) return ADA_ERR_SHAPE;
    if (ws_bytes < ADA_PAGED_ZERO_BYTES + select_ws(a.p).bytes || (uintptr_t)ws % 256) return ADA_ERR_WORKSPACE;
    if (chunk->rows == 0) return ADA_OK;
    a.Q = Q; a.ldq = ldq; a.budget = budget; a.first = first; a.last = last; a.list = pages; a.count = counts;
    return paged_dispatch(cache->dtype, cache->d_h, [&](auto in, auto dh) {
        return launch_select<decltype(in), decltype(dh)::value>(a, ws, (hipStream_t)stream);
    });
}

}  // extern "C"
