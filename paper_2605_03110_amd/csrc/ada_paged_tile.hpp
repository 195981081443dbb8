// Attention of chunks over a paged cache in bf16: matrix instructions bound it.
//
// A tile is TILE = 128 query rows (tokens x heads of a group, as in ada_paged_attn.hpp) that read one head of the cache; keys come in
// units of 64.  Each of the four waves has 32 rows: S^T = K Q^T with the queries in registers (lane = query), weights in the registers that the second product's
// operand wants them in, O^T += V^T P^T.  Keys and values go from memory to LDS directly, one unit ahead; values are read from there
// transposed.  The units of all tiles stand in one line and are cut into as many pieces as workgroups run at once, see ada_paged_attn.hpp.
// LDS rows are permuted in pieces of 16 bytes on the way in (the source address is, the destination is the lane's): keys by their row number, so that
// eight rows at one column fall on different banks; values by 64 bytes, so that four rows of 64 bytes do.
#pragma once

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4* LdsAt;

template <int DH> struct TileGeom {
    static constexpr int WAVES = 4, ROWS = 32 * WAVES, KEYS = 64, KS = DH / 16, NB = DH / 32, PPR = DH / 8;
    static constexpr int STAGE = KEYS * DH * 2, LDS = 4 * STAGE;               // keys and values, twice
    static constexpr int PER_CU = DH > 128 ? 1 : 2;
    __device__ static int key_slot(int row, int piece) { return piece ^ (row & (PPR >= 16 ? 15 : 7)); }
    __device__ static int value_slot(int row, int piece) { return piece ^ (PPR >= 16 ? (row & 3) << 2 : ((row >> 1) & 1) << 2); }
};

__device__ inline f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ inline float max_over_halves(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ inline float sum_over_halves(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// Row r of a tile: see tile_row.
template <int ROWS>
__device__ inline bool chunk_row(const AttendArgs& a, const Tile& t, int r, int& row, int& head, int& token) {
    const int flat = t.j * ROWS + r;
    token = flat / a.p.G;
    head = flat - token * a.p.G;
    row = t.s.row0 + token;
    return token < t.s.n;
}

// A wave's 32 rows to the output: lane has columns 32 i + 8 w + 4 half .. of row l32.
template <int DH>
__device__ inline void store_rows(const AttendArgs& a, const Tile& t, int row, int head, int half, const f32x16 (&o)[DH / 32], float f) {
    uint16_t* to = reinterpret_cast<uint16_t*>(a.out) + row * a.ld_out + (long long)(t.kvh * a.p.G + head) * DH + 4 * half;
#pragma unroll
    for (int i = 0; i < DH / 32; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w)
            *reinterpret_cast<u32x2*>(to + 32 * i + 8 * w) = u32x2{bf16_pair(o[i][4 * w] * f, o[i][4 * w + 1] * f), bf16_pair(o[i][4 * w + 2] * f, o[i][4 * w + 3] * f)};
}

template <int DH>
__global__ __launch_bounds__(256, TileGeom<DH>::PER_CU) void k_paged_tile(AttendArgs a) {
    using G = TileGeom<DH>;
    constexpr int KS = G::KS, NB = G::NB, PPR = G::PPR;
    extern __shared__ __align__(16) char lds[];
    char* kbuf = lds;
    char* vbuf = lds + 2 * G::STAGE;
    const PagedArgs& p = a.p;
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int me = by_xcd(blockIdx.x, gridDim.x);
    const long long total = line_length<false>(a), x0 = me * total / gridDim.x, x1 = (me + 1) * total / gridDim.x;
    // where this lane's columns of a value row start in LDS for the transposed reads: rows 4 half + (lane & 15) / 4 + 8 n, columns 16 ((lane >> 4) & 1) + 4 (lane & 3)
    const int vrow = 4 * half + ((lane & 15) >> 2);
    const int vpiece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);

    for (long long x = x0; x < x1;) {
        const Tile t = same_in_all(find_tile<false>(a, x));
        const int k0 = (int)(x - t.at), k1 = (int)(min(x1, t.at + t.units) - t.at);
        x = t.at + k1;
        int row, head, token;
        const bool mine = chunk_row<G::ROWS>(a, t, wave * 32 + l32, row, head, token);
        if (!mine) {                                       // (the sequence's last row again, never stored)
            token = t.s.n - 1;
            head = p.G - 1;
            row = t.s.row0 + token;
        }
        const uint16_t* q = reinterpret_cast<const uint16_t*>(a.Q) + row * a.ldq + (long long)(t.kvh * p.G + head) * DH + half * 8;
        u32x4 qf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const u32x4*>(q + ks * 16);
        const int limit = p.causal ? t.s.past + token + 1 : t.s.len;                  // keys below it are seen
        const int all_see = __builtin_amdgcn_readfirstlane(limit);                    // by all rows of the wave (its first row is the earliest)
        const int last16 = (t.s.len - 1) & ~15;
        const int32_t* table = p.table + t.b * p.table_stride;
        // lanes 0 .. 3: the pages of a unit's 16-key groups (behind the end: the last group again, whose keys nobody sees there)
        auto pages_of = [&](int u) { return table[min(u * G::KEYS + (lane & 3) * 16, last16) >> p.lg]; };
        auto bad_of = [&](int pg) { return (int)(__builtin_amdgcn_ballot_w64(pg < 0 || pg >= p.pages) & 15); };
        auto issue = [&](int u, int stage, int pg) {       // the wave's 16 keys and values of unit u
            const int page = __builtin_amdgcn_readlane(pg, wave), pos = min(u * G::KEYS + wave * 16, last16);
            const bool ok = page >= 0 && page < p.pages;
            // where there is no page a row of queries stands in: finite numbers, weight 0
            const long long at = page * p.page_stride + (pos & ((1 << p.lg) - 1)) * p.slot_stride + t.kvh * p.head_stride;
            const uint16_t* stand_in = reinterpret_cast<const uint16_t*>(a.Q) + t.s.row0 * a.ldq;
            const uint16_t* ks = ok ? reinterpret_cast<const uint16_t*>(p.K) + at : stand_in;
            const uint16_t* vs = ok ? reinterpret_cast<const uint16_t*>(p.V) + at : stand_in;
            const long long stride = ok ? p.slot_stride : 0;
            if (!ok && lane == 0) raise(p, ADA_ERR_INDEX);
#pragma unroll
            for (int c = 0; c < DH / 32; ++c) {
                const int r = c * (512 / DH) + lane / PPR, in = min(r, t.s.len - 1 - pos);
                __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)(ks + in * stride + G::key_slot(wave * 16 + r, lane % PPR) * 8),
                                                 (void __attribute__((address_space(3)))*)(kbuf + stage * G::STAGE + wave * 32 * DH + c * 1024), 16, 0, 0);
            }
#pragma unroll
            for (int c = 0; c < DH / 32; ++c) {
                const int r = c * (512 / DH) + lane / PPR, in = min(r, t.s.len - 1 - pos);
                __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)(vs + in * stride + G::value_slot(wave * 16 + r, lane % PPR) * 8),
                                                 (void __attribute__((address_space(3)))*)(vbuf + stage * G::STAGE + wave * 32 * DH + c * 1024), 16, 0, 0);
            }
        };
        f32x16 acc_o[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc_o[i][e] = 0.f;
        float m_run = -INFINITY, l_run = 0.f;              // of query l32; the sum over this half's keys
        int pg = pages_of(k0);
        __syncthreads();                                   // the tile before is done with LDS
        issue(k0, 0, pg);
        int bad = bad_of(pg);
        pg = pages_of(k0 + 1);
        for (int u = k0; u < k1; ++u) {
            const int stage = (u - k0) & 1;
            __builtin_amdgcn_s_waitcnt(0x0F70);            // vmcnt(0): this wave's part of the unit has landed
            __builtin_amdgcn_s_barrier();
            const int bad_now = bad;
            if (u + 1 < k1) {
                issue(u + 1, stage ^ 1, pg);
                bad = bad_of(pg);
                pg = pages_of(u + 2);
            }
            // ---- S^T: 64 keys x this wave's 32 queries
            const char* kc = kbuf + stage * G::STAGE;
            f32x16 s[2];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[b][e] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const u32x4 kf = *reinterpret_cast<const u32x4*>(kc + (b * 32 + l32) * DH * 2 + G::key_slot(l32, 2 * ks + half) * 16);
                    s[b] = mfma32(kf, qf[ks], s[b]);
                }
            // ---- weights in base 2 against a reference that moves when it is passed by more than 10
            const int key0 = u * G::KEYS;
            if (key0 + G::KEYS > all_see || bad_now) {     // (the same for the wave)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int k = b * 32 + (e & 3) + 8 * (e >> 2) + 4 * half;
                        if (key0 + k >= limit || (bad_now >> (2 * b + (e >> 3))) & 1) s[b][e] = -INFINITY;
                    }
            }
            float mx = -INFINITY;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[b][e]);
            mx = max_over_halves(mx) * a.sc2;
            const bool grow = mx > m_run + 10.f;
            if (__builtin_amdgcn_ballot_w64(grow) != 0ull) {
                const float f = grow ? __builtin_amdgcn_exp2f(m_run - mx) : 1.f;
                m_run = grow ? mx : m_run;
                l_run *= f;
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc_o[i][e] *= f;
            }
            const float m_use = m_run == -INFINITY ? 0.f : m_run;
            u32x4 pf[4];                                   // weights, one bf16 number each (half a step: 2^-9), by 16 keys
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float w0 = __builtin_amdgcn_exp2f(s[b][e] * a.sc2 - m_use), w1 = __builtin_amdgcn_exp2f(s[b][e + 1] * a.sc2 - m_use);
                    l_run += w0 + w1;
                    pf[2 * b + (e >> 3)][(e & 7) >> 1] = bf16_pair(w0, w1);
                }
            // ---- O^T += V^T P^T
            const char* vc = vbuf + stage * G::STAGE + 8 * (lane & 1);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    const int r0 = 16 * j + vrow, r1 = r0 + 8;
                    const u32x2 v0 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsAt)(vc + r0 * DH * 2 + G::value_slot(r0, 4 * i + vpiece) * 16)));
                    const u32x2 v1 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsAt)(vc + r1 * DH * 2 + G::value_slot(r1, 4 * i + vpiece) * 16)));
                    acc_o[i] = mfma32(u32x4{v0[0], v0[1], v1[0], v1[1]}, pf[j], acc_o[i]);
                }
        }
        const float l = sum_over_halves(l_run);
        if (k0 == 0 && k1 == t.units) {
            if (mine) store_rows<DH>(a, t, row, head, half, acc_o, l > 0.f ? 1.f / l : 0.f);
        } else {
            const long long slot = 2LL * me + (k0 == 0 ? 1 : 0);
            float* po = a.part_o + (slot * G::WAVES + wave) * (32 * DH) + lane;
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) po[(i * 16 + e) * 64] = acc_o[i][e];
            if (half == 0) *reinterpret_cast<f32x2*>(a.part_ml + ((slot * G::WAVES + wave) * 32 + l32) * 2) = f32x2{m_run, l};
        }
    }
}

// Puts a cut tile together, see k_paged_join.
template <int DH>
__global__ __launch_bounds__(256) void k_paged_tile_join(AttendArgs a) {
    using G = TileGeom<DH>;
    constexpr int NB = G::NB;
    const int W = gridDim.x, me = blockIdx.x, lane = threadIdx.x & 63, l32 = lane & 31, wave = threadIdx.x >> 6;
    const long long total = line_length<false>(a), x0 = me * total / W, x1 = (me + 1) * total / W;
    if (x0 >= x1 || x1 >= total) return;
    const Tile t = find_tile<false>(a, x1 - 1);
    const long long end = t.at + t.units;
    if (end == x1 || t.at < x0) return;
    int last = me;
    while ((last + 1) * total / W < end) ++last;
    int row, head, token;
    const bool mine = chunk_row<G::ROWS>(a, t, wave * 32 + l32, row, head, token);
    float m = -INFINITY, l = 0.f;
    f32x16 o[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    for (int w = me; w <= last; ++w) {
        if (w > me && w * total / W == (w + 1) * total / W) continue;
        const long long slot = 2LL * w + (w == me ? 1 : 0);
        const f32x2 ml = *reinterpret_cast<const f32x2*>(a.part_ml + ((slot * G::WAVES + wave) * 32 + l32) * 2);
        const float mn = fmaxf(m, ml[0]);
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn), fw = ml[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[0] - mn);
        m = mn;
        l = l * f + ml[1] * fw;
        const float* po = a.part_o + (slot * G::WAVES + wave) * (32 * DH) + lane;
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[i][e] = o[i][e] * f + po[(i * 16 + e) * 64] * fw;
    }
    if (mine) store_rows<DH>(a, t, row, head, lane >> 5, o, l > 0.f ? 1.f / l : 0.f);
}
