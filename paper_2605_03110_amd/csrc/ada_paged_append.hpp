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

// Bounds of one piece: widened by k, or started by it.
template <typename In>
__device__ inline void widen_bounds(In* low, In* high, const Eight<In>& k, bool fresh) {
    Eight<In> lo = k, hi = k;
    if (!fresh) {
        float f[8], l[8], h[8];
        k.widen(f);
        Eight<In>::load(low).widen(l);
        Eight<In>::load(high).widen(h);
#pragma unroll
        for (int i = 0; i < 8; ++i) { l[i] = fminf(l[i], f[i]); h[i] = fmaxf(h[i], f[i]); }
        lo = Eight<In>::round(l);                          // (values of the type itself: exact)
        hi = Eight<In>::round(h);
    }
    lo.store(low);
    hi.store(high);
}

// BOUNDS: a page gets at most one new token (no sequence has more), so its bounds are widened here.
template <typename In, int DH, bool BOUNDS>
__global__ __launch_bounds__(256) void k_cache_append(AppendArgs a) {
    const PagedArgs& p = a.p;
    constexpr int LPR = DH / 16, UNITS = 256 / LPR;
    const int heads_q = a.Q ? p.H : 0, heads = heads_q + 2 * p.H_kv;
    const long long unit = (long long)blockIdx.x * UNITS + threadIdx.x / LPR;
    const int j = threadIdx.x % LPR;
    const int row = (int)min(unit / heads, (long long)p.rows - 1);
    int b = paged_find(p, __builtin_amdgcn_readfirstlane(row));      // of the wave's first row; the others are at it or just behind
    while (b < p.B && p.start[b + 1] <= row) ++b;
    if (unit >= (long long)p.rows * heads || b >= p.B) return;
    const Seq s = paged_seq(p, b);
    const int i = row - s.row0;
    if (i < 0 || i >= s.n) return;
    const int pos = s.past + i, head = (int)(unit % heads);
    const bool is_q = head < heads_q, is_v = head >= heads_q + p.H_kv;
    const int h = is_q ? head : is_v ? head - heads_q - p.H_kv : head - heads_q;
    In *to, *low = nullptr, *high = nullptr;
    const int slot = pos & ((1 << p.lg) - 1);
    if (is_q) {
        to = reinterpret_cast<In*>(a.q_out) + row * a.ldq_out + h * DH;
    } else {
        const int page = p.table[b * p.table_stride + (pos >> p.lg)];
        if (page < 0 || page >= p.pages) {
            raise(p, ADA_ERR_INDEX);
            return;
        }
        to = reinterpret_cast<In*>(is_v ? p.V : p.K) + page * p.page_stride + h * p.head_stride + slot * p.slot_stride;
        if (BOUNDS && !is_v && p.bounds) {
            low = reinterpret_cast<In*>(p.bounds) + ((long long)page * p.H_kv + h) * 2 * DH;
            high = low + DH;
        }
    }
    const In* from = is_q ? reinterpret_cast<const In*>(a.Q) + row * a.ldq + h * DH
                   : is_v ? reinterpret_cast<const In*>(a.Vn) + row * a.ldv + h * DH : reinterpret_cast<const In*>(a.Kn) + row * a.ldk + h * DH;
    const int turned = a.rot / 16;                         // lanes whose pieces turn
    const bool turns = j < turned && !is_v;
    if (a.rot && pos >= a.rope_len) {
        raise(p, ADA_ERR_INDEX);
        return;
    }
    int c0 = 2 * j, c1 = 2 * j + 1;
    if (!a.pairs && j < turned) { c0 = j; c1 = j + turned; }
    const Eight<In> x0 = Eight<In>::load(from + 8 * c0), x1 = Eight<In>::load(from + 8 * c1);
    if (is_v) {
        x0.store(to + 8 * c0);
        x1.store(to + 8 * c1);
        return;
    }
    float f0[8], f1[8];
    x0.widen(f0);
    x1.widen(f1);
    const In* w = reinterpret_cast<const In*>(is_q ? a.q_norm : a.k_norm);
    if (w) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += f0[e] * f0[e] + f1[e] * f1[e];
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) sum += __shfl_xor(sum, o, 64);
        const float scale = 1.f / sqrtf(sum * (1.f / DH) + a.eps);
        float w0[8], w1[8];
        Eight<In>::load(w + 8 * c0).widen(w0);
        Eight<In>::load(w + 8 * c1).widen(w1);
#pragma unroll
        for (int e = 0; e < 8; ++e) { f0[e] = f0[e] * scale * w0[e]; f1[e] = f1[e] * scale * w1[e]; }
    }
    if (turns) {
        const f32x4* cs = reinterpret_cast<const f32x4*>(a.rope + (long long)pos * a.rot) + (a.pairs ? 4 * j : 4 * c0);
        f32x4 t[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = cs[e];
        if (a.pairs) {                                     // lane j: pairs 8 j .. 8 j + 7, four in each piece
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float c0_ = t[e >> 1][2 * (e & 1)], s0_ = t[e >> 1][2 * (e & 1) + 1];
                const float c1_ = t[2 + (e >> 1)][2 * (e & 1)], s1_ = t[2 + (e >> 1)][2 * (e & 1) + 1];
                const float u = f0[2 * e], v = f0[2 * e + 1], x = f1[2 * e], y = f1[2 * e + 1];
                f0[2 * e] = u * c0_ - v * s0_;
                f0[2 * e + 1] = u * s0_ + v * c0_;
                f1[2 * e] = x * c1_ - y * s1_;
                f1[2 * e + 1] = x * s1_ + y * c1_;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float c = t[e >> 1][2 * (e & 1)], sn = t[e >> 1][2 * (e & 1) + 1], u = f0[e], v = f1[e];
                f0[e] = u * c - v * sn;
                f1[e] = u * sn + v * c;
            }
        }
    }
    const Eight<In> y0 = Eight<In>::round(f0), y1 = Eight<In>::round(f1);
    y0.store(to + 8 * c0);
    y1.store(to + 8 * c1);
    if (BOUNDS && low) {
        widen_bounds(low + 8 * c0, high + 8 * c0, y0, slot == 0);
        widen_bounds(low + 8 * c1, high + 8 * c1, y1, slot == 0);
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

template <typename In, int DH>
hipError_t launch_append(const AppendArgs& a, hipStream_t st) {
    const PagedArgs& p = a.p;
    const long long units = (long long)p.rows * ((a.Q ? p.H : 0) + 2 * p.H_kv), groups = (units + 256 / (DH / 16) - 1) / (256 / (DH / 16));
    if (groups > INT_MAX) return hipErrorInvalidValue;
    const bool in_one = p.longest == 1;
    {
        ProfHook ps(ADA_K_ATTN, st);
        if (in_one) hipLaunchKernelGGL((k_cache_append<In, DH, true>), dim3((unsigned)groups), dim3(256), 0, st, a);
        else hipLaunchKernelGGL((k_cache_append<In, DH, false>), dim3((unsigned)groups), dim3(256), 0, st, a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || in_one || !p.bounds) return e;
    ProfHook ps(ADA_K_ATTN, st);
    hipLaunchKernelGGL((k_cache_bounds<In, DH>), dim3((p.rows + 63) / 64, p.H_kv), dim3(256), 0, st, p, a.rot ? a.rope_len : MAX_TOKENS);
    return hipGetLastError();
}
