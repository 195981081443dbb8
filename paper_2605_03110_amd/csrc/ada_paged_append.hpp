// Appending: every head of every new row is one unit, held by d_h / 16 lanes that have two pieces of eight columns each.  Which
// two goes by the rotation, so that a lane has both members of its pairs: with pairs (i, i + rot / 2) the pieces j and j + rot / 16, then,
// for the columns behind rot, neighbours; with pairs (2 i, 2 i + 1) neighbours everywhere.  No lane needs another's columns, and a norm is one
// sum over d_h / 16 lanes.  Read once, written once; everything between is fp32 and rounded once.
#pragma once

struct AppendArgs {
    PagedArgs p;
    const void *Q, *Kn, *Vn;
    long long ldq, ldk, ldv;
    const void *q_norm, *k_norm;
    float eps;
    const float* rope;
    int rot, rope_len, pairs;
    void* q_out;
    long long ldq_out;
};

template <typename In> struct Eight;                       // eight neighbouring columns
template <> struct Eight<uint16_t> {
    u32x4 w;
    __device__ static Eight load(const uint16_t* at) { return {*reinterpret_cast<const u32x4*>(at)}; }
    __device__ void store(uint16_t* at) const { *reinterpret_cast<u32x4*>(at) = w; }
    __device__ void widen(float (&f)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(w[i]); f[2 * i + 1] = bf16_hi(w[i]); }
    }
    __device__ static Eight round(const float (&f)[8]) {
        Eight e;
#pragma unroll
        for (int i = 0; i < 4; ++i) e.w[i] = bf16_pair(f[2 * i], f[2 * i + 1]);
        return e;
    }
};
template <> struct Eight<float> {
    f32x4 a, b;
    __device__ static Eight load(const float* at) { return {reinterpret_cast<const f32x4*>(at)[0], reinterpret_cast<const f32x4*>(at)[1]}; }
    __device__ void store(float* at) const { reinterpret_cast<f32x4*>(at)[0] = a; reinterpret_cast<f32x4*>(at)[1] = b; }
    __device__ void widen(float (&f)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[i] = a[i]; f[4 + i] = b[i]; }
    }
    __device__ static Eight round(const float (&f)[8]) { return {{f[0], f[1], f[2], f[3]}, {f[4], f[5], f[6], f[7]}}; }
};

// The lane's two pieces of a row: lane j of d_h / 16 has columns 8 c0 .. and 8 c1 ..
struct Pieces {
    int c0, c1;
    bool turns;
    __device__ Pieces(const AppendArgs& a, int j) {
        const int turned = a.rot / 16;                     // lanes whose pieces turn
        turns = j < turned;
        c0 = !a.pairs && turns ? j : 2 * j;
        c1 = !a.pairs && turns ? j + turned : 2 * j + 1;
    }
};

// Norm (w: weights or NULL) and rotation at `pos` of the lane's pieces of a head.
template <typename In, int DH>
__device__ inline void turn_row(const AppendArgs& a, const Pieces& c, int j, const In* w, int pos, float (&f0)[8], float (&f1)[8]) {
    f32x4 t[4];
    if (c.turns) {
        const f32x4* cs = reinterpret_cast<const f32x4*>(a.rope + (long long)pos * a.rot) + (a.pairs ? 4 * j : 4 * c.c0);
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = cs[e];
    }
    if (w) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += f0[e] * f0[e] + f1[e] * f1[e];
#pragma unroll
        for (int o = 1; o < DH / 16; o <<= 1) sum += __shfl_xor(sum, o, 64);
        const float scale = 1.f / sqrtf(sum * (1.f / DH) + a.eps);
        float w0[8], w1[8];
        Eight<In>::load(w + 8 * c.c0).widen(w0);
        Eight<In>::load(w + 8 * c.c1).widen(w1);
#pragma unroll
        for (int e = 0; e < 8; ++e) { f0[e] = f0[e] * scale * w0[e]; f1[e] = f1[e] * scale * w1[e]; }
    }
    if (!c.turns) return;
    auto turn = [](float& x, float& y, const f32x4& cs, int at) {
        const float u = x, v = y;
        x = u * cs[at] - v * cs[at + 1];
        y = u * cs[at + 1] + v * cs[at];
    };
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (!a.pairs) turn(f0[e], f1[e], t[e >> 1], 2 * (e & 1));
        else if (e < 4) turn(f0[2 * e], f0[2 * e + 1], t[e >> 1], 2 * (e & 1));           // lane j: pairs 8 j .. 8 j + 7, four in each piece
        else turn(f1[2 * e - 8], f1[2 * e - 7], t[e >> 1], 2 * (e & 1));
    }
}

// Bounds of one piece: widened by lo and hi, or started by them.
template <typename In>
__device__ inline void widen_bounds(In* low, In* high, float (&lo)[8], float (&hi)[8], bool fresh) {
    if (!fresh) {
        float l[8], h[8];
        Eight<In>::load(low).widen(l);
        Eight<In>::load(high).widen(h);
#pragma unroll
        for (int e = 0; e < 8; ++e) { lo[e] = fminf(lo[e], l[e]); hi[e] = fmaxf(hi[e], h[e]); }
    }
    Eight<In>::round(lo).store(low);                       // (values of the type itself: exact)
    Eight<In>::round(hi).store(high);
}

// Keys of chunks where bounds are kept: a workgroup takes 16 rows of a head of the cache and, for each of them that is the first new one in its page, appends
// that page's new keys and bounds them as they pass.
template <typename In, int DH>
__device__ inline void append_pages(const AppendArgs& a, int group) {
    constexpr int LPR = DH / 16, RPI = 256 / LPR;          // lanes per key, keys at a time
    __shared__ float red[4][LPR][2][17];                   // per wave and lane: 16 smallest, 16 largest (and a place against bank conflicts)
    const PagedArgs& p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = group % p.H_kv, block = group / p.H_kv, j = tid % LPR;
    const int row = min(block * 16 + (lane & 15), p.rows - 1);
    int b = paged_find(p, __builtin_amdgcn_readfirstlane(row));
    while (b < p.B && p.start[b + 1] <= row) ++b;
    int pos = 0, count = 0, page = -1;
    if (lane < 16 && block * 16 + lane < p.rows && b < p.B) {
        const Seq s = paged_seq(p, b);
        const int i = row - s.row0;
        if (i >= 0 && i < s.n) {
            pos = s.past + i;
            const int slot = pos & ((1 << p.lg) - 1);
            if (i == 0 || slot == 0) {
                count = min((1 << p.lg) - slot, s.n - i);
                page = p.table[b * p.table_stride + (pos >> p.lg)];
                if (page < 0 || page >= p.pages) {
                    raise(p, ADA_ERR_INDEX);
                    count = 0;
                } else if (a.rot && pos + count > a.rope_len) {                // keys behind the table's end are not appended
                    raise(p, ADA_ERR_INDEX);
                    count = a.rope_len - pos;
                }
            }
        }
    }
    const Pieces c(a, j);
    const In* w = reinterpret_cast<const In*>(a.k_norm);
    for (unsigned long long left = __builtin_amdgcn_ballot_w64(count > 0); left; left &= left - 1) {     // (the same in all waves)
        const int from = __ffsll(left) - 1, first = __shfl(pos, from, 64), slot = first & ((1 << p.lg) - 1), n = __shfl(count, from, 64);
        const long long pg = __shfl(page, from, 64), r0 = block * 16 + from;
        const In* keys = reinterpret_cast<const In*>(a.Kn) + r0 * a.ldk + h * DH;
        In* to = reinterpret_cast<In*>(p.K) + pg * p.page_stride + h * p.head_stride + slot * p.slot_stride;
        float lo[2][8], hi[2][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { lo[0][e] = lo[1][e] = INFINITY; hi[0][e] = hi[1][e] = -INFINITY; }
        for (int i = tid / LPR; i < n; i += RPI) {
            const In* x = keys + i * a.ldk;
            float f0[8], f1[8];
            Eight<In>::load(x + 8 * c.c0).widen(f0);
            Eight<In>::load(x + 8 * c.c1).widen(f1);
            turn_row<In, DH>(a, c, j, w, first + i, f0, f1);
            const Eight<In> y0 = Eight<In>::round(f0), y1 = Eight<In>::round(f1);
            y0.store(to + i * p.slot_stride + 8 * c.c0);
            y1.store(to + i * p.slot_stride + 8 * c.c1);
            y0.widen(f0);
            y1.widen(f1);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                lo[0][e] = fminf(lo[0][e], f0[e]); hi[0][e] = fmaxf(hi[0][e], f0[e]);
                lo[1][e] = fminf(lo[1][e], f1[e]); hi[1][e] = fmaxf(hi[1][e], f1[e]);
            }
        }
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                lo[e >> 3][e & 7] = fminf(lo[e >> 3][e & 7], __shfl_xor(lo[e >> 3][e & 7], o, 64));
                hi[e >> 3][e & 7] = fmaxf(hi[e >> 3][e & 7], __shfl_xor(hi[e >> 3][e & 7], o, 64));
            }
        __syncthreads();                                   // (the page before is done with)
        if (lane < LPR)
#pragma unroll
            for (int e = 0; e < 16; ++e) { red[wave][lane][0][e] = lo[e >> 3][e & 7]; red[wave][lane][1][e] = hi[e >> 3][e & 7]; }
        __syncthreads();
        if (tid < LPR) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
#pragma unroll
                for (int v = 1; v < 4; ++v) {
                    lo[e >> 3][e & 7] = fminf(lo[e >> 3][e & 7], red[v][lane][0][e]);
                    hi[e >> 3][e & 7] = fmaxf(hi[e >> 3][e & 7], red[v][lane][1][e]);
                }
            In* low = reinterpret_cast<In*>(p.bounds) + (pg * p.H_kv + h) * 2 * DH;
            widen_bounds<In>(low + 8 * c.c0, low + DH + 8 * c.c0, lo[0], hi[0], slot == 0);
            widen_bounds<In>(low + 8 * c.c1, low + DH + 8 * c.c1, lo[1], hi[1], slot == 0);
        }
    }
}

// Rows' heads.  PAGES: without the keys, behind page_groups workgroups that append_pages.  BOUNDS: no page has two new keys, and whoever has one bounds it.
template <typename In, int DH, bool PAGES, bool BOUNDS>
__global__ __launch_bounds__(256) void k_cache_append(AppendArgs a, int page_groups) {
    const PagedArgs& p = a.p;
    constexpr int LPR = DH / 16, UNITS = 256 / LPR;
    if (PAGES && (int)blockIdx.x < page_groups) {
        append_pages<In, DH>(a, blockIdx.x);
        return;
    }
    const int heads_q = a.Q ? p.H : 0, heads_k = PAGES ? 0 : p.H_kv, heads = heads_q + heads_k + p.H_kv;
    const long long unit = (long long)(blockIdx.x - page_groups) * UNITS + threadIdx.x / LPR;
    const int j = threadIdx.x % LPR;
    const int row = (int)min(unit / heads, (long long)p.rows - 1);
    int b = paged_find(p, __builtin_amdgcn_readfirstlane(row));      // of the wave's first row; the others are at it or just behind
    while (b < p.B && p.start[b + 1] <= row) ++b;
    if (unit >= (long long)p.rows * heads || b >= p.B) return;
    const Seq s = paged_seq(p, b);
    const int i = row - s.row0;
    if (i < 0 || i >= s.n) return;
    const int pos = s.past + i, head = (int)(unit % heads), slot = pos & ((1 << p.lg) - 1);
    const bool is_q = head < heads_q, is_v = head >= heads_q + heads_k;
    const int h = is_q ? head : is_v ? head - heads_q - heads_k : head - heads_q;
    int page = 0;
    if (!is_q) page = p.table[b * p.table_stride + (pos >> p.lg)];
    if (page < 0 || page >= p.pages || (a.rot && pos >= a.rope_len)) {
        raise(p, ADA_ERR_INDEX);
        return;
    }
    const In* from = is_q ? reinterpret_cast<const In*>(a.Q) + row * a.ldq + h * DH
                   : is_v ? reinterpret_cast<const In*>(a.Vn) + row * a.ldv + h * DH : reinterpret_cast<const In*>(a.Kn) + row * a.ldk + h * DH;
    In* to = is_q ? reinterpret_cast<In*>(a.q_out) + row * a.ldq_out + h * DH
                  : reinterpret_cast<In*>(is_v ? p.V : p.K) + page * p.page_stride + h * p.head_stride + slot * p.slot_stride;
    const Pieces c(a, j);
    const Eight<In> x0 = Eight<In>::load(from + 8 * c.c0), x1 = Eight<In>::load(from + 8 * c.c1);
    if (is_v) {
        x0.store(to + 8 * c.c0);
        x1.store(to + 8 * c.c1);
        return;
    }
    float f0[8], f1[8];
    x0.widen(f0);
    x1.widen(f1);
    turn_row<In, DH>(a, c, j, reinterpret_cast<const In*>(is_q ? a.q_norm : a.k_norm), pos, f0, f1);
    const Eight<In> y0 = Eight<In>::round(f0), y1 = Eight<In>::round(f1);
    y0.store(to + 8 * c.c0);
    y1.store(to + 8 * c.c1);
    if (BOUNDS && !is_q && p.bounds) {
        In* low = reinterpret_cast<In*>(p.bounds) + ((long long)page * p.H_kv + h) * 2 * DH;
        y0.widen(f0);
        y1.widen(f1);
        float g0[8], g1[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { g0[e] = f0[e]; g1[e] = f1[e]; }
        widen_bounds<In>(low + 8 * c.c0, low + DH + 8 * c.c0, f0, g0, slot == 0);
        widen_bounds<In>(low + 8 * c.c1, low + DH + 8 * c.c1, f1, g1, slot == 0);
    }
}

// Bounds behind an append of longer chunks: a wave takes 16 rows of a head of the cache and, for each that is the first new one in its
// page, reads that page's new keys.
template <typename In, int DH>
__global__ __launch_bounds__(256) void k_cache_bounds(PagedArgs p, int positions) {
    constexpr int LPR = DH / 8, RPI = 64 / LPR;            // lanes per key, keys at a time
    const int lane = threadIdx.x & 63, block = blockIdx.x * 4 + (threadIdx.x >> 6), h = blockIdx.y;
    const int row = min(block * 16 + (lane & 15), p.rows - 1);
    int b = paged_find(p, __builtin_amdgcn_readfirstlane(row));
    while (b < p.B && p.start[b + 1] <= row) ++b;
    int pos = 0, count = 0, page = -1;
    if (lane < 16 && block * 16 + lane < p.rows && b < p.B) {
        const Seq s = paged_seq(p, b);
        const int i = row - s.row0;
        if (i >= 0 && i < s.n) {
            pos = s.past + i;
            const int slot = pos & ((1 << p.lg) - 1);
            if (i == 0 || slot == 0) {
                count = min(min((1 << p.lg) - slot, s.n - i), positions - pos);            // (those that were appended)
                page = p.table[b * p.table_stride + (pos >> p.lg)];
                if (page < 0 || page >= p.pages) count = 0;                  // (reported by the append)
            }
        }
    }
    for (unsigned long long left = __builtin_amdgcn_ballot_w64(count > 0); left; left &= left - 1) {
        const int from = __ffsll(left) - 1;
        const int slot = __shfl(pos, from, 64) & ((1 << p.lg) - 1), n = __shfl(count, from, 64);
        const long long pg = __shfl(page, from, 64);
        const In* keys = reinterpret_cast<const In*>(p.K) + pg * p.page_stride + h * p.head_stride + slot * p.slot_stride + (lane % LPR) * 8;
        float lo[8], hi[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
        for (int k = 0; k < n; k += 8 * RPI) {             // eight reads under way (behind the last key: that one again)
            Eight<In> x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = Eight<In>::load(keys + (long long)min(k + i * RPI + lane / LPR, n - 1) * p.slot_stride);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float f[8];
                x[i].widen(f);
#pragma unroll
                for (int e = 0; e < 8; ++e) { lo[e] = fminf(lo[e], f[e]); hi[e] = fmaxf(hi[e], f[e]); }
            }
        }
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1)
#pragma unroll
            for (int e = 0; e < 8; ++e) { lo[e] = fminf(lo[e], __shfl_xor(lo[e], o, 64)); hi[e] = fmaxf(hi[e], __shfl_xor(hi[e], o, 64)); }
        if (lane < LPR) {
            In* low = reinterpret_cast<In*>(p.bounds) + (pg * p.H_kv + h) * 2 * DH + lane * 8;
            if (slot > 0) {
                float l[8], u[8];
                Eight<In>::load(low).widen(l);
                Eight<In>::load(low + DH).widen(u);
#pragma unroll
                for (int e = 0; e < 8; ++e) { lo[e] = fminf(lo[e], l[e]); hi[e] = fmaxf(hi[e], u[e]); }
            }
            Eight<In>::round(lo).store(low);
            Eight<In>::round(hi).store(low + DH);
        }
    }
}

// Where no sequence has more than one new token no page has two, and whoever has the key bounds it.  Else, while there is little to do, a page's new keys go to one
// workgroup of the same launch; where bandwidth counts, bounds are read back from the cache in a second one.  us, one and two launches: 512 tokens, 12 x 64 in fp32, 9.0
// and 14.9; four prompts of 2048 tokens, 16 x 256, 152 and 93 (131 registers instead of 59 for everybody).
template <typename In, int DH>
hipError_t launch_append(const AppendArgs& a, hipStream_t st) {
    const PagedArgs& p = a.p;
    constexpr int per = 256 / (DH / 16);
    const bool single = p.longest == 1 || !p.bounds;
    const long long heads = (a.Q ? p.H : 0) + 2 * (long long)p.H_kv, pages = (p.rows + 15) / 16 * (long long)p.H_kv;
    const long long groups = (p.rows * heads + per - 1) / per, beside = (p.rows * (heads - p.H_kv) + per - 1) / per;
    if (groups > INT_MAX) return hipErrorInvalidValue;
    if (!single && pages + beside <= 8 * ada_hook_cus()) {
        ProfHook ps(ADA_K_ATTN, st);
        hipLaunchKernelGGL((k_cache_append<In, DH, true, false>), dim3((unsigned)(pages + beside)), dim3(256), 0, st, a, (int)pages);
        return hipGetLastError();
    }
    {
        ProfHook ps(ADA_K_ATTN, st);
        if (single) hipLaunchKernelGGL((k_cache_append<In, DH, false, true>), dim3((unsigned)groups), dim3(256), 0, st, a, 0);
        else hipLaunchKernelGGL((k_cache_append<In, DH, false, false>), dim3((unsigned)groups), dim3(256), 0, st, a, 0);
    }
    if (hipError_t e = hipGetLastError()) return e;
    if (single) return hipSuccess;
    ProfHook ps(ADA_K_ATTN, st);
    hipLaunchKernelGGL((k_cache_bounds<In, DH>), dim3((p.rows + 63) / 64, p.H_kv), dim3(256), 0, st, p, a.rot ? a.rope_len : MAX_TOKENS);
    return hipGetLastError();
}
