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
    static constexpr int KB = KEYS / 32, GROUPS = KEYS / 16, SPAN = 64 / GROUPS;        // blocks of 32 keys and groups of 16 in a unit; units whose groups' pages a wave holds
    static constexpr int STAGE = KEYS * DH * 2, LDS = 4 * STAGE + 16;          // keys and values, twice; comes_last's word
    static constexpr int PER_CU = DH > 128 ? 1 : 2;        // workgroups of a CU at once
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

// 16 bytes per lane from `base` (the same in all lanes) + `off` bytes to `to` (the same) + 16 lane.  Written out because the compiler, which sees the
// builtin write LDS, would wait for these loads in front of every transposed read of the other stage; a load without a destination register is waited for by the
// loop's own barrier.
__device__ inline void load_to_lds(const void* base, uint32_t off, char* to) {
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)to;
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(at)), "v"(off), "s"(base) : "m0", "memory");
}

template <int DH>
__global__ __launch_bounds__(256, TileGeom<DH>::PER_CU) void k_paged_tile(AttendArgs a) {
    using G = TileGeom<DH>;
    constexpr int KS = G::KS, NB = G::NB, PPR = G::PPR, KB = G::KB, MINE = G::KEYS / G::WAVES, PIECES = MINE * DH * 2 / 1024;      // a wave loads MINE rows, 1 KB at a time
    extern __shared__ __align__(16) char lds[];
    char* kbuf = lds;
    char* vbuf = lds + 2 * G::STAGE;
    const PagedArgs& p = a.p;
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool young = blockIdx.x >= gridDim.x / 2;
    const Line<CHUNKS> line(a);
    if (line.total == 0) return;
    const Piece piece(line.total, least_of((float)line.per_head / *a.tiles), G::PER_CU, DH == 128 ? 2 : 1);
    // where this lane's columns of a value row start in LDS for the transposed reads: rows 4 half + (lane & 15) / 4 + 8 n, columns 16 ((lane >> 4) & 1) + 4 (lane & 3)
    const int vrow = 4 * half + ((lane & 15) >> 2);
    const int vpiece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    const int row16 = (wave * MINE) & 15;                  // the wave's first row in its group of 16
    uint32_t koff[PIECES], voff[PIECES];                   // where this lane reads in a whole group
#pragma unroll
    for (int c = 0; c < PIECES; ++c) {
        const int r = row16 + c * (512 / DH) + lane / PPR;
        koff[c] = (uint32_t)(r * p.slot_stride + G::key_slot(r, lane % PPR) * 8) * 2;
        voff[c] = (uint32_t)(r * p.slot_stride + G::value_slot(r, lane % PPR) * 8) * 2;
    }

    for (long long x = piece.x0; x < piece.x1;) {
        const Tile t = line.find(x);
        const Part part(piece, t, x);
        const int k0 = part.k0, k1 = part.k1;
        x = t.at + BEGIN + t.units;
        if (k0 >= k1) continue;
        int row, head, token;
        if (!tile_row<CHUNKS, G::ROWS>(a, t, wave * 32 + l32, row, head, token)) {   // (the sequence's last row again, never stored)
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
        const long long head_at = t.kvh * p.head_stride;
        // pages of SPAN units, a lane per group of 16 keys (behind the end: the last group again, whose keys nobody sees there); the even spans and the odd ones
        auto pages_of = [&](int span) { return table[min((span * 64 + lane) * 16, last16) >> p.lg]; };
        int even = pages_of(k0 / G::SPAN + ((k0 / G::SPAN) & 1)), odd = pages_of(k0 / G::SPAN | 1);
        auto pages_at = [&](int u) { return (u / G::SPAN) & 1 ? odd : even; };
        auto bad_of = [&](int u) {
            const int pg = pages_at(u);
            return (int)(__builtin_amdgcn_ballot_w64(pg < 0 || pg >= p.pages) >> (u % G::SPAN * G::GROUPS)) & ((1 << G::GROUPS) - 1);
        };
        // the wave's rows of unit u's keys or values
        auto issue = [&](const void* from, const uint32_t (&off)[PIECES], bool values, int u) {
            const int group = wave * MINE / 16, page = __builtin_amdgcn_readlane(pages_at(u), u % G::SPAN * G::GROUPS + group);
            const int pos = min(u * G::KEYS + group * 16, last16);
            const bool ok = page >= 0 && page < p.pages;
            char* to = (values ? vbuf : kbuf) + (u & 1) * G::STAGE + wave * MINE * DH * 2;
            const uint16_t* src = reinterpret_cast<const uint16_t*>(from) + page * p.page_stride + (pos & ((1 << p.lg) - 1)) * p.slot_stride + head_at;
            if (ok && pos + 16 <= t.s.len) {
#pragma unroll
                for (int c = 0; c < PIECES; ++c) load_to_lds(src, off[c], to + c * 1024);
                return;
            }
            // rows behind the end are not read: the last one stands in; where there is no page, a row of queries: finite numbers, weight 0
            if (!ok) {
                src = reinterpret_cast<const uint16_t*>(a.Q) + t.s.row0 * a.ldq;
                if (lane == 0) raise(p, ADA_ERR_INDEX);
            }
#pragma unroll
            for (int c = 0; c < PIECES; ++c) {
                const int r = row16 + c * (512 / DH) + lane / PPR, in = ok ? min(r, t.s.len - 1 - pos) : 0;
                load_to_lds(src, (uint32_t)(in * p.slot_stride + (values ? G::value_slot(r, lane % PPR) : G::key_slot(r, lane % PPR)) * 8) * 2, to + c * 1024);
            }
        };
        auto landed = [] {                                 // this wave's loads have landed and its reads have returned, and so have everybody's
            __builtin_amdgcn_s_waitcnt(0x0070);
            asm volatile("s_barrier" ::: "memory");
        };
        u32x4 kf[3][KB];                                   // keys, read two steps ahead of their products
        auto read_k = [&](const char* kc, int ks) {
#pragma unroll
            for (int b = 0; b < KB; ++b)
                kf[ks % 3][b] = *reinterpret_cast<const u32x4*>(kc + (b * 32 + l32) * DH * 2 + G::key_slot(l32, 2 * ks + half) * 16);
        };
        // S^T of unit u, `beside` what goes between its products
        auto scores = [&](int u, f32x16 (&s)[KB], auto beside) {
            const char* kc = kbuf + (u & 1) * G::STAGE;
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[b][e] = 0.f;
            read_k(kc, 0);
            read_k(kc, 1);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                if (ks + 2 < KS) read_k(kc, ks + 2);
#pragma unroll
                for (int b = 0; b < KB; ++b) s[b] = mfma32(kf[ks % 3][b], qf[ks], s[b]);
                beside(ks);
            }
        };
        f32x16 acc_o[NB], s[KB], s2[KB];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc_o[i][e] = 0.f;
        float m_run = -INFINITY, l_run = 0.f;              // of query l32; the sum over this half's keys
        __syncthreads();                                   // the tile before is done with LDS
        issue(p.K, koff, false, k0);
        issue(p.V, voff, true, k0);
        landed();
        if (k0 + 1 < k1) issue(p.K, koff, false, k0 + 1);
        scores(k0, s, [](int) {});
        // one unit: s are its scores, s2 becomes the next one's
        auto step = [&](int u, f32x16 (&s)[KB], f32x16 (&s2)[KB]) {
            // Of two workgroups on a CU the older one is served first and ends a sixth earlier; the younger one goes first in every other unit
            // (8192 tokens: 600 and 715 us -> alike, 644 -> 628 us a call)
            if (G::PER_CU > 1 && young) {
                if (u & 1) __builtin_amdgcn_s_setprio(0); else __builtin_amdgcn_s_setprio(1);
            }
            landed();                                      // keys of u + 1, values of u
            if (u + 2 < k1) issue(p.K, koff, false, u + 2);
            if (u + 1 < k1) issue(p.V, voff, true, u + 1);
            const int bad = bad_of(u);
            if (u % G::SPAN == 6) {                        // (nobody asks for the span before this one any more)
                const int next = pages_of(u / G::SPAN + 1);
                if ((u / G::SPAN) & 1) even = next; else odd = next;
            }
            // ---- weights in base 2 against a reference that moves when it is passed by more than 10
            const int key0 = u * G::KEYS;
            if (key0 + G::KEYS > all_see || bad) {         // (the same for the wave)
#pragma unroll
                for (int b = 0; b < KB; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int k = b * 32 + (e & 3) + 8 * (e >> 2) + 4 * half;
                        if (key0 + k >= limit || (bad >> (2 * b + (e >> 3))) & 1) s[b][e] = -INFINITY;
                    }
            }
            float mx = -INFINITY;
#pragma unroll
            for (int b = 0; b < KB; ++b)
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
            u32x4 pf[2 * KB];                              // weights, one bf16 number each, by 16 keys
            auto weights = [&](int w) {                    // the w-th pair
                const int b = w >> 3, e = 2 * (w & 7);
                const float w0 = __builtin_amdgcn_exp2f(s[b][e] * a.sc2 - m_use), w1 = __builtin_amdgcn_exp2f(s[b][e + 1] * a.sc2 - m_use);
                l_run += w0 + w1;
                pf[2 * b + (e >> 3)][(e & 7) >> 1] = bf16_pair(w0, w1);
            };
            scores(u + 1, s2, [&](int ks) {                // (behind the last unit: of what lies in LDS, for nobody)
#pragma unroll
                for (int w = ks * 8 * KB / KS; w < (ks + 1) * 8 * KB / KS; ++w) weights(w);
            });
            // ---- O^T += V^T P^T
            const char* vc = vbuf + (u & 1) * G::STAGE + 8 * (lane & 1);
            constexpr int NV = 2 * KB * NB, VA = 3;        // products; how many of their operands are read ahead
            u32x2 vf[VA + 1][2];
            auto read_v = [&](int n) {
                const int r0 = 16 * (n / NB) + vrow, r1 = r0 + 8, piece = 4 * (n % NB) + vpiece;
                vf[n % (VA + 1)][0] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsAt)(vc + r0 * DH * 2 + G::value_slot(r0, piece) * 16)));
                vf[n % (VA + 1)][1] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsAt)(vc + r1 * DH * 2 + G::value_slot(r1, piece) * 16)));
            };
#pragma unroll
            for (int n = 0; n < VA; ++n) read_v(n);
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                if (n + VA < NV) read_v(n + VA);
                const u32x2 v0 = vf[n % (VA + 1)][0], v1 = vf[n % (VA + 1)][1];
                acc_o[n % NB] = mfma32(u32x4{v0[0], v0[1], v1[0], v1[1]}, pf[n / NB], acc_o[n % NB]);
            }
            __builtin_amdgcn_sched_group_barrier(0x100, 2 * VA, 1);
#pragma unroll
            for (int n = 0; n < NV - VA; ++n) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, VA, 1);
        };
        for (int u = k0; u < k1; u += 2) {
            step(u, s, s2);
            if (u + 1 == k1) break;
            step(u + 1, s2, s);
        }
        float l = sum_over_halves(l_run);
        int again = wave * 32 + l32;
        asm volatile("" : "+v"(again));                    // (found anew: kept over the loop it would cost registers)
        const bool mine = tile_row<CHUNKS, G::ROWS>(a, t, again, row, head, token);
        if (part.whole(t)) {
            if (mine) store_rows<DH>(a, t, row, head, half, acc_o, l > 0.f ? 1.f / l : 0.f);
            continue;
        }
        const long long slot = part.slot(piece);
        float* po = a.part_o + (slot * G::WAVES + wave) * (32 * DH) + 2 * lane;
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 2) put(po + (i * 16 + e) * 64, acc_o[i][e], acc_o[i][e + 1]);
        if (half == 0) put(a.part_ml + ((slot * G::WAVES + wave) * 32 + l32) * 2, m_run, l);
        int first, last;
        if (!comes_last(a, piece, t, first, last, reinterpret_cast<int*>(lds + 4 * G::STAGE))) continue;
        // Four parts at a time: every part is a trip to memory, and whoever joins is the last to end (512 tokens behind 16000, heads of 256, four or
        // five parts a tile: 266 us a call with one part at a time, 229 so).  C blocks of 32 columns at a time, as many as registers hold.
        constexpr int C = DH == 128 ? 1 : 2;
        auto part_at = [&](int w) { return (2LL * w + (w == first ? 1 : 0)) * G::WAVES + wave; };
        float m = -INFINITY;
        for (int w0 = first; w0 <= last; w0 += 4) {
            float mw[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) mw[q] = get(a.part_ml + (part_at(min(w0 + q, last)) * 32 + l32) * 2)[0];
#pragma unroll
            for (int q = 0; q < 4; ++q) m = fmaxf(m, mw[q]);
        }
        uint16_t* to = reinterpret_cast<uint16_t*>(a.out) + row * a.ld_out + (long long)(t.kvh * p.G + head) * DH + 4 * half;
#pragma unroll 1
        for (int i = 0; i < NB; i += C) {
            float o[C][16];
#pragma unroll
            for (int e = 0; e < 16 * C; ++e) o[e >> 4][e & 15] = 0.f;
            l = 0.f;
            for (int w0 = first; w0 <= last; w0 += 4) {
                f32x2 ml[4], v[4][C][8];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const long long s2 = part_at(min(w0 + q, last));
                    ml[q] = get(a.part_ml + (s2 * 32 + l32) * 2);
                    const float* from = a.part_o + s2 * (32 * DH) + 2 * lane + i * 16 * 64;
#pragma unroll
                    for (int e = 0; e < 8 * C; ++e) v[q][e >> 3][e & 7] = get(from + e * 128);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (w0 + q > last) break;
                    const float f = ml[q][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[q][0] - m);
                    l += ml[q][1] * f;
#pragma unroll
                    for (int e = 0; e < 8 * C; ++e) {
                        o[e >> 3][2 * (e & 7)] += v[q][e >> 3][e & 7][0] * f;
                        o[e >> 3][2 * (e & 7) + 1] += v[q][e >> 3][e & 7][1] * f;
                    }
                }
            }
            const float f = l > 0.f ? 1.f / l : 0.f;
            if (mine)
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int w = 0; w < 4; ++w)
                        *reinterpret_cast<u32x2*>(to + 32 * (i + c) + 8 * w) =
                            u32x2{bf16_pair(o[c][4 * w] * f, o[c][4 * w + 1] * f), bf16_pair(o[c][4 * w + 2] * f, o[c][4 * w + 3] * f)};
        }
    }
}
