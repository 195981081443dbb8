// Which pages a token attends to.  score(page) = max over the group's heads of sum_i max(q_i lo_i, q_i hi_i): as q+ = max(q, 0) and q- =
// min(q, 0), the sum is the product of [q+, q-] with [hi, lo], a matrix product of pages by query heads over 2 d_h columns.
//
// The lists are whole numbers and have to be the ones that exact arithmetic gives, while the matrix product adds in fp32.  So the fp32
// scores only narrow it down: with tau the k-th largest of them and E a bound of their error, a page above tau + 2 E is among the k
// largest and one below tau - 2 E is not; for those between, where they are more than the places left, the sum is taken again in fp64.
//   E = (2 d_h + 16) 2^-24 max_h |q_h|_1 max |bound|: at most 2 d_h roundings, each of no more than the sum of the products' magnitudes (and 16 to
//   spare for the bound's own arithmetic).
// Two launches: scores, a wave per 16 pages and some rows, to the workspace as integers in the numbers' order; then a wave per row and head of the cache
// that chooses.  (In one launch, scores in LDS: a workgroup per row took 33 us for 16 tokens at 20 to 32 thousand keys, most CUs without work, and 83 for
// 2048 tokens at 8 thousand.)
#pragma once

struct SelectArgs {
    PagedArgs p;
    const void* Q;
    long long ldq;
    int budget, first, last;
    int32_t *list, *count;
    int row0, rows;                                        // the rows of this pair of launches
    int lg_heads;                                          // columns of a product: 2^lg_heads heads (a group of up to 16, or a part of it) x tokens
    int slots;                                             // pages per row and head in the workspace: whole sixteens
    uint32_t* key;                                         // [rows][H_kv][slots], 0: no such page
    float* most;                                           // [rows][H_kv][slots / 16] largest |bound| of sixteen pages
};

__device__ inline uint32_t ordered(float f) {              // as unsigned integers in the order of the numbers; never 0
    const uint32_t u = __float_as_uint(f);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ inline float unordered(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }
__device__ inline unsigned long long ordered(double f) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(f);
    return u ^ ((u >> 63) ? ~0ull : 1ull << 63);
}

// maximum over lanes 2^lg at a time (neighbours), in all of them
__device__ __forceinline__ float max_over_neighbours(float v, int lg) {
    auto with = [&](auto ctrl) { return fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), decltype(ctrl)::value, 15, 15, false))); };
    if (lg > 0) v = with(Const<0xB1>());                   // lane ^ 1
    if (lg > 1) v = with(Const<0x4E>());                   // lane ^ 2
    if (lg > 2) v = with(Const<0x141>());                  // the other half of eight, mirrored
    if (lg > 3) v = with(Const<0x140>());                  // the other half of sixteen, mirrored
    return v;
}
// maximum over the wave
__device__ __forceinline__ uint32_t max_of_wave(uint32_t v) {
    auto with = [&](auto ctrl) { return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, 15, 15, false)); };
    v = with(Const<0xB1>());
    v = with(Const<0x4E>());
    v = with(Const<0x141>());
    v = with(Const<0x140>());
    auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max((uint32_t)a[0], (uint32_t)a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (uint32_t)__builtin_amdgcn_readfirstlane(max((uint32_t)b[0], (uint32_t)b[1]));
}

// n keys, a lane's every 64th; the first 64 HELD are held in registers, more are asked for again each time (0: no key).
template <typename Key, int HELD_, typename Get> struct Keys {
    static constexpr int HELD = HELD_;
    const Get& get;
    int n;
    Key held[HELD];
    __device__ __forceinline__ Keys(int count, const Get& g, const Key (&first)[HELD]) : get(g), n(count) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) held[i] = first[i];
    }
    __device__ __forceinline__ void block(int i0, Key (&k)[HELD]) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int at = i0 + i * 64 + lane;
            k[i] = i0 + i * 64 < n && at < n ? get(at) : 0;
        }
    }
    template <typename F> __device__ __forceinline__ void each(F&& f) const {  // f(first key's number, block of keys)
        f(0, held);
        for (int i0 = 64 * HELD; i0 < n; i0 += 64 * HELD) {
            Key k[HELD];
            block(i0, k);
            f(i0, k);
        }
    }
    __device__ __forceinline__ int count(Key from) const { // keys >= from (> 0)
        int c = 0;
        each([&](int i0, const Key (&k)[HELD]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) if (i0 + i * 64 < n) c += __popcll(__builtin_amdgcn_ballot_w64(k[i] >= from));
        });
        return c;
    }
    // The k-th largest key (0 < k <= keys)
    __device__ __forceinline__ Key kth(int k) const {
        Key t = 0;
        int bit = (int)sizeof(Key) * 8 - 1;
        if constexpr (sizeof(Key) == 4) {                  // what the keys have in common in front is known already
            Key most = 0, least = ~(Key)0;
            each([&](int, const Key (&key)[HELD]) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < HELD; ++i) {
                    most = max(most, key[i]);
                    least = min(least, key[i] ? key[i] : ~(Key)0);
                }
            });
            most = max_of_wave(most);
            least = ~max_of_wave(~least);
            if (most == least) return most;
            bit = 31 - __clz(most ^ least);
            t = bit == 31 ? 0 : most >> (bit + 1) << (bit + 1);
        }
        for (; bit >= 0; --bit) {
            const Key with = t | ((Key)1 << bit);
            const int c = count(with);
            if (c >= k) t = with;
            if (c == k) break;                             // (the k largest are those >= t: the smallest of them is meant)
        }
        Key least = ~(Key)0;
        each([&](int, const Key (&key)[HELD]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) if (key[i] != 0 && key[i] >= t && key[i] < least) least = key[i];
        });
        if constexpr (sizeof(Key) == 4) return ~max_of_wave(~least);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const Key other = __shfl_xor(least, o, 64);
            if (other < least) least = other;
        }
        return least;
    }
};

// the negative entries and the others, 0 elsewhere
template <typename In> __device__ inline void split(u32x4 w, u32x4& negative, u32x4& others);
template <> __device__ inline void split<uint16_t>(u32x4 w, u32x4& negative, u32x4& others) {
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const u32x4 m = __builtin_bit_cast(u32x4, __builtin_bit_cast(s16x8, w) >> 15);
    negative = w & m;
    others = w & ~m;
}
template <> __device__ inline void split<float>(u32x4 w, u32x4& negative, u32x4& others) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t m = (uint32_t)((int)w[i] >> 31);
        negative[i] = w[i] & m;
        others[i] = w[i] & ~m;
    }
}
template <typename In> __device__ inline float largest(u32x4 w);               // magnitude
template <> __device__ inline float largest<uint16_t>(u32x4 w) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(m, fmaxf(fabsf(bf16_lo(w[i])), fabsf(bf16_hi(w[i]))));
    return m;
}
template <> __device__ inline float largest<float>(u32x4 w) {
    return fmaxf(fmaxf(fabsf(__uint_as_float(w[0])), fabsf(__uint_as_float(w[1]))), fmaxf(fabsf(__uint_as_float(w[2])), fabsf(__uint_as_float(w[3]))));
}
template <typename In> __device__ inline float abs_sum(u32x4 w);
template <> __device__ inline float abs_sum<uint16_t>(u32x4 w) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) m += fabsf(bf16_lo(w[i])) + fabsf(bf16_hi(w[i]));
    return m;
}
template <> __device__ inline float abs_sum<float>(u32x4 w) {
    return fabsf(__uint_as_float(w[0])) + fabsf(__uint_as_float(w[1])) + fabsf(__uint_as_float(w[2])) + fabsf(__uint_as_float(w[3]));
}
template <typename In> __device__ inline double as_double(In v);
template <> __device__ inline double as_double<uint16_t>(uint16_t v) { return (double)__uint_as_float((uint32_t)v << 16); }
template <> __device__ inline double as_double<float>(float v) { return (double)v; }

// Scores: a wave takes 16 SETS pages, `per_group` rows and a head of the cache.  SETS: 2 where rows share pages, as every wave reads the queries again.
template <typename In, int DH, int SETS>
__global__ __launch_bounds__(256) void k_select_scores(SelectArgs a, int per_group) {
    constexpr int EPP = 16 / (int)sizeof(In), KF = DH / (4 * EPP);
    const PagedArgs& p = a.p;
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, kvh = blockIdx.z;
    const int j0 = (blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * 16 * SETS;
    const int per = 1 << a.lg_heads, tokens = 16 >> a.lg_heads;                // columns: a token's heads side by side
    const int end = min((int)(blockIdx.x + 1) * per_group, a.rows) + a.row0;
    for (int row = blockIdx.x * per_group + a.row0; row < end;) {
        const int b = paged_find(p, row);
        if (b >= p.B) return;                                                  // rows behind the last sequence
        const Seq s = paged_seq(p, b);
        if (row < s.row0 || row >= s.row0 + s.n) { ++row; continue; }
        const int stop = min(end, s.row0 + s.n);                               // this sequence's rows
        const int n_pages = (((p.causal ? s.past + stop - s.row0 : s.len) - 1) >> p.lg) + 1;  // that the last of them sees
        if (j0 >= n_pages) { row = stop; continue; }
        const int tok = l16 >> a.lg_heads, sub = l16 & (per - 1);
        auto query = [&](int r, int h0) {
            return reinterpret_cast<const In*>(a.Q) + min(r + tok, stop - 1) * a.ldq + (long long)(kvh * p.G + h0 + min(sub, min(p.G - h0, 16) - 1)) * DH + g * EPP;
        };
        u32x4 qf[KF];
        auto fetch = [&](const In* q) {
#pragma unroll
            for (int c = 0; c < KF; ++c) qf[c] = *reinterpret_cast<const u32x4*>(q + c * 4 * EPP);
        };
        fetch(query(row, 0));
        u32x4 kf[SETS][2][KF];
        bool there[SETS];
        unsigned long long known[SETS];                    // bit l16: page j0 + 16 set + l16
        float most[SETS];
        const In* low[SETS];
#pragma unroll
        for (int i = 0; i < SETS; ++i) {
            const int page = p.table[b * p.table_stride + min(j0 + i * 16 + l16, n_pages - 1)];
            there[i] = page >= 0 && page < p.pages;
            low[i] = reinterpret_cast<const In*>(p.bounds) + ((long long)(there[i] ? page : 0) * p.H_kv + kvh) * 2 * DH;
        }
#pragma unroll
        for (int i = 0; i < SETS; ++i)
#pragma unroll
            for (int side = 0; side < 2; ++side)
#pragma unroll
                for (int c = 0; c < KF; ++c) kf[i][side][c] = *reinterpret_cast<const u32x4*>(low[i] + side * DH + (c * 4 + g) * EPP);
#pragma unroll
        for (int i = 0; i < SETS; ++i) {
            if (!there[i]) raise(p, ADA_ERR_INDEX);
            most[i] = 0.f;
#pragma unroll
            for (int side = 0; side < 2; ++side)
#pragma unroll
                for (int c = 0; c < KF; ++c) most[i] = fmaxf(most[i], largest<In>(kf[i][side][c]));
            most[i] = __uint_as_float(max_of_wave(__float_as_uint(there[i] ? most[i] : 0.f)));                // (not negative: in the order of their bits)
            known[i] = __builtin_amdgcn_ballot_w64(there[i]);
        }
        for (; row < stop; row += tokens) {
            f32x4 best[SETS];
#pragma unroll
            for (int i = 0; i < SETS; ++i) best[i] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            for (int h0 = 0; h0 < p.G; h0 += 16) {                             // (groups of more than 16 heads in turns)
                f32x4 part[SETS][2];
#pragma unroll
                for (int i = 0; i < SETS; ++i) part[i][0] = part[i][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < KF; ++c) {
                    u32x4 qs[2];
                    split<In>(qf[c], qs[0], qs[1]);
#pragma unroll
                    for (int side = 0; side < 2; ++side)
#pragma unroll
                        for (int i = 0; i < SETS; ++i) {
                            if constexpr (sizeof(In) == 2) part[i][side] = mfma16(kf[i][side][c], qs[side], part[i][side]);
                            else
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    part[i][side] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[i][side][c][e]), __uint_as_float(qs[side][e]), part[i][side], 0, 0, 0);
                        }
                }
                const bool more = h0 + 16 < p.G;
                if (more || row + tokens < stop) fetch(query(more ? row : row + tokens, more ? h0 + 16 : 0));
#pragma unroll
                for (int i = 0; i < SETS; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) best[i][e] = fmaxf(best[i][e], part[i][0][e] + part[i][1][e]);
            }
#pragma unroll
            for (int i = 0; i < SETS; ++i) {
                u32x4 key;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = max_over_neighbours(best[i][e], a.lg_heads);
                    key[e] = (known[i] >> (4 * g + e)) & 1 ? ordered(v) : 0u;
                }
                if (sub == 0 && row + tok < stop && j0 + i * 16 < a.slots) {
                    const long long at = ((long long)(row + tok - a.row0) * p.H_kv + kvh) * a.slots + j0 + i * 16;
                    *reinterpret_cast<u32x4*>(a.key + at + 4 * g) = key;
                    if (g == 0) a.most[at >> 4] = most[i];
                }
            }
        }
        row = stop;
    }
}

// Scores of four pages in fp64, in all lanes: 16 lanes share a head, four heads at a time.
template <typename In, int DH>
__device__ __forceinline__ void exact_scores(int G, const In* q_row, const In* const (&low)[4], double (&best)[4]) {
    constexpr int C = DH / 16, W = C * (int)sizeof(In) / 4;                    // columns and 32-bit words of a lane
    const int lane = threadIdx.x & 63, c0 = (lane & 15) * C;
    uint32_t lo[4][W], hi[4][W];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __builtin_memcpy(lo[i], __builtin_assume_aligned(low[i] + c0, 8), sizeof(lo[i]));
        __builtin_memcpy(hi[i], __builtin_assume_aligned(low[i] + DH + c0, 8), sizeof(hi[i]));
        best[i] = -INFINITY;
    }
    auto value = [](const uint32_t (&w)[W], int c) {
        if constexpr (sizeof(In) == 4) return (double)__uint_as_float(w[c]);
        else return (double)(c & 1 ? bf16_hi(w[c >> 1]) : bf16_lo(w[c >> 1]));
    };
    for (int h0 = 0; h0 < G; h0 += 4) {
        uint32_t q[W];
        __builtin_memcpy(q, __builtin_assume_aligned(q_row + (long long)min(h0 + (lane >> 4), G - 1) * DH + c0, 8), sizeof(q));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            double sum = 0.0;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const double x = value(q, c);
                sum += x * (x < 0.0 ? value(lo[i], c) : value(hi[i], c));
            }
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) sum += __shfl_xor(sum, o, 64);
            best[i] = sum > best[i] ? sum : best[i];
        }
    }
#pragma unroll
    for (int o = 16; o < 64; o <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double other = __shfl_xor(best[i], o, 64);
            best[i] = other > best[i] ? other : best[i];
        }
}

// HELD: 2 where a sequence has up to 128 pages (2048 rows of 8 heads at 8 thousand keys: 35.8 -> 25.3 us), else 8.
template <typename In, int DH, int HELD>
__global__ __launch_bounds__(256, HELD == 2 && DH * sizeof(In) <= 256 ? 4 : 2) void k_select_choose(SelectArgs a) {
    constexpr int EPP = 16 / (int)sizeof(In), LPR = DH / EPP;                  // LPR: lanes that read a head
    const PagedArgs& p = a.p;
    const int lane = threadIdx.x & 63;
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (unit >= a.rows * p.H_kv) return;
    const int row = a.row0 + unit / p.H_kv, kvh = unit % p.H_kv;
    // asked for before it is known which of it is the row's: the keys that are held, the bounds' sizes, four heads or more of queries
    const uint32_t* key = a.key + (long long)unit * a.slots;
    uint32_t raw[HELD];
#pragma unroll
    for (int w = 0; w < HELD; ++w) raw[w] = w * 64 + lane < a.slots ? key[w * 64 + lane] : 0u;
    const float most0 = lane < a.slots >> 4 ? a.most[(long long)unit * (a.slots >> 4) + lane] : 0.f;
    const In* q_row = reinterpret_cast<const In*>(a.Q) + row * a.ldq + (long long)kvh * p.G * DH;
    auto size_of = [&](int h0) {                           // |q_h|_1 of heads h0 + lane / LPR
        float sum = abs_sum<In>(*reinterpret_cast<const u32x4*>(q_row + (long long)min(h0 + lane / LPR, p.G - 1) * DH + (lane % LPR) * EPP));
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) sum += __shfl_xor(sum, o, 64);
        return sum;
    };
    float q1 = size_of(0);
    const int b = paged_find(p, row);
    if (b >= p.B) return;
    const Seq s = paged_seq(p, b);
    if (row < s.row0 || row >= s.row0 + s.n) return;
    const int have = __builtin_amdgcn_readfirstlane(((p.causal ? s.past + row - s.row0 : s.len - 1) >> p.lg) + 1);
    const int lo = min(a.first, have), hi = max(lo, have - a.last), free = a.budget - lo - (have - hi);      // candidates lo .. hi - 1
    const int32_t* table = p.table + b * p.table_stride;
    const auto get = [&](int i) { return i >= lo && i < hi ? key[i] : 0u; };
    uint32_t first[HELD];
#pragma unroll
    for (int w = 0; w < HELD; ++w) {
        if (w * 64 + lane >= have) raw[w] = 0u;            // (what nobody has written)
        first[w] = w * 64 + lane >= lo && w * 64 + lane < hi ? raw[w] : 0u;
    }
    const Keys<uint32_t, HELD, decltype(get)> candidates(have, get, first);
    // chosen: pages that have to be; keys >= all_from; of the others from between_from on ("open") those whose exact score is above exact_from, and the
    // first `ties` equal to it
    uint32_t all_from = 1, between_from = 1;
    bool many = false;
    unsigned long long chosen = 0;                         // of up to 64 open ones, by their order
    int need = 0, open = 0;
    if (candidates.count(1) > free) {
        all_from = between_from = 0xFFFFFFFFu;             // (no key is that large)
        if (free > 0) {
            // what the scores are exact to
            for (int h0 = 64 / LPR; h0 < p.G; h0 += 64 / LPR) q1 = fmaxf(q1, size_of(h0));
            const int sixteens = (have + 15) >> 4;
            float most = lane < sixteens ? most0 : 0.f;
            for (int i = 64 + lane; i < sixteens; i += 64) most = fmaxf(most, a.most[(long long)unit * (a.slots >> 4) + i]);
            q1 = __uint_as_float(max_of_wave(__float_as_uint(q1)));            // (not negative: in the order of their bits)
            most = __uint_as_float(max_of_wave(__float_as_uint(most)));
            const float tau = unordered(candidates.kth(free)), err = (2 * DH + 16) * 5.9604645e-8f * q1 * most * 2.02f;
            between_from = max(ordered(tau - err), 1u);
            all_from = ordered(tau + err) + 1;
            const int sure = candidates.count(all_from);
            open = candidates.count(between_from) - sure;
            need = free - sure;
            if (open == need) all_from = between_from;
            else many = open > 64;
        }
    }
    auto is_open = [&](uint32_t k) { return k >= between_from && k < all_from; };
    int n = 0, seen = 0;
    int32_t* to = a.list + ((long long)row * p.H_kv + kvh) * a.budget;
    const unsigned long long below = (1ull << lane) - 1;
    auto put_out = [&](bool in, int page) __attribute__((always_inline)) {
        const unsigned long long ins = __builtin_amdgcn_ballot_w64(in);
        const int place = n + __popcll(ins & below);
        if (in && place < a.budget) to[place] = page;      // (scores that are not numbers can let too many in)
        n = min(n + __popcll(ins), a.budget);
    };
    auto forced = [&](int i0, int w, uint32_t k) {         // of the pages that have to be, those that are there
        const int i = i0 + w * 64 + lane;
        if (k != 0u || i >= have || (i >= lo && i < hi)) return false;
        return (i < 64 * HELD ? raw[w] : key[i]) != 0u;
    };
    if (!many) {
        if (between_from < all_from && open != need) {     // up to 64 open pages, four at a time
            unsigned long long mine = 0;                   // lane i: the exact score of the i-th
            int held = 0, at = 0, pages[4] = {0, 0, 0, 0};
            auto take = [&]() {
                const In* low[4];
                double e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) low[i] = reinterpret_cast<const In*>(p.bounds) + ((long long)table[pages[i < held ? i : 0]] * p.H_kv + kvh) * 2 * DH;
                exact_scores<In, DH>(p.G, q_row, low, e);
#pragma unroll
                for (int i = 0; i < 4; ++i) if (i < held && lane == at + i) mine = ordered(e[i]);
                at += held;
                held = 0;
            };
            candidates.each([&](int i0, const uint32_t (&k)[HELD]) __attribute__((always_inline)) {
#pragma unroll
                for (int w = 0; w < HELD; ++w)
                    for (unsigned long long left = i0 + w * 64 < have ? __builtin_amdgcn_ballot_w64(is_open(k[w])) : 0ull; left; left &= left - 1) {
                        const int page = i0 + w * 64 + __ffsll(left) - 1;
                        if (held == 0) pages[0] = page; else if (held == 1) pages[1] = page; else if (held == 2) pages[2] = page; else pages[3] = page;
                        if (++held == 4) take();
                    }
            });
            if (held) take();
            for (int i = 0; i < need; ++i) {               // one place after the other: the largest left, the first of equal ones
                unsigned long long top = (chosen >> lane) & 1 ? 0ull : mine;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const unsigned long long other = __shfl_xor(top, o, 64);
                    top = other > top ? other : top;
                }
                const unsigned long long same = __builtin_amdgcn_ballot_w64(mine == top && !((chosen >> lane) & 1));
                chosen |= same & (~same + 1);
            }
        }
        candidates.each([&](int i0, const uint32_t (&k)[HELD]) __attribute__((always_inline)) {
#pragma unroll
            for (int w = 0; w < HELD; ++w) {
                if (i0 + w * 64 >= have) continue;
                const bool o = is_open(k[w]);
                const unsigned long long os = __builtin_amdgcn_ballot_w64(o);
                put_out((k[w] != 0u && k[w] >= all_from) || (o && (chosen >> ((seen + __popcll(os & below)) & 63)) & 1) || forced(i0, w, k[w]), i0 + w * 64 + lane);
                seen += __popcll(os);
            }
        });
    } else {
        // more than 64 within the error of each other (alike pages, queries of zeros): every lane takes the sums of its own pages
        const auto open_key = [&](int i) {
            if (!is_open(get(i))) return 0ull;
            const In* low = reinterpret_cast<const In*>(p.bounds) + ((long long)table[i] * p.H_kv + kvh) * 2 * DH;
            double best = -INFINITY;
            for (int h = 0; h < p.G; ++h) {
                double sum = 0.0;
                for (int c = 0; c < DH; ++c) {
                    const double x = as_double<In>(q_row[(long long)h * DH + c]);
                    sum += x * (x < 0.0 ? as_double<In>(low[c]) : as_double<In>(low[DH + c]));
                }
                best = sum > best ? sum : best;
            }
            return ordered(best);
        };
        unsigned long long first_exact[HELD];
        for (int w = 0; w < HELD; ++w) first_exact[w] = 0;
        Keys<unsigned long long, HELD, decltype(open_key)> opens(have, open_key, first_exact);
        opens.block(0, opens.held);
        const unsigned long long exact_from = opens.kth(need);
        const int ties = need - opens.count(exact_from + 1);
        opens.each([&](int i0, const unsigned long long (&e)[HELD]) __attribute__((always_inline)) {
            uint32_t k[HELD];
            candidates.block(i0, k);
#pragma unroll
            for (int w = 0; w < HELD; ++w) {
                if (i0 + w * 64 >= have) continue;
                const unsigned long long ts = __builtin_amdgcn_ballot_w64(e[w] == exact_from);
                put_out(k[w] >= all_from || e[w] > exact_from || (e[w] == exact_from && seen + __popcll(ts & below) < ties) || forced(i0, w, k[w]), i0 + w * 64 + lane);
                seen += __popcll(ts);
            }
        });
    }
    for (int i = n + lane; i < a.budget; i += 64) to[i] = -1;
    if (lane == 0) a.count[(long long)row * p.H_kv + kvh] = n;
}

// ------------------------------------------------------------------------------------------------ host
struct SelectWs { int slots, rows; size_t most, bytes; };  // rows of one pair of launches

inline SelectWs select_ws(const PagedArgs& p) {
    SelectWs w;
    w.slots = (p.max_pages + 15) / 16 * 16;
    const size_t row = (size_t)p.H_kv * w.slots * 4, most = 64u << 20;        // 64 MB of keys at a time, or a row's
    w.rows = p.rows;
    if (row * p.rows > most) w.rows = row < most ? (int)(most / row) : 1;
    w.most = (row * w.rows + 255) / 256 * 256;
    w.bytes = w.most + (w.most / 16 + 255) / 256 * 256;
    return w;
}

template <typename In, int DH>
hipError_t launch_select(SelectArgs a, void* ws, hipStream_t st) {
    const PagedArgs& p = a.p;
    const SelectWs w = select_ws(p);
    a.lg_heads = 0;
    while ((1 << a.lg_heads) < (p.G < 16 ? p.G : 16)) ++a.lg_heads;
    a.slots = w.slots;
    char* at = reinterpret_cast<char*>(ws) + ADA_PAGED_ZERO_BYTES;
    a.key = reinterpret_cast<uint32_t*>(at);
    a.most = reinterpret_cast<float*>(at + w.most);
    const int per_group = p.longest == 1 ? 1 : 32, pages = p.longest == 1 ? 64 : 128;  // of a workgroup
    for (a.row0 = 0; a.row0 < p.rows; a.row0 += a.rows) {
        a.rows = p.rows - a.row0 < w.rows ? p.rows - a.row0 : w.rows;
        {
            ProfHook ps(ADA_K_ATTN, st);
            const dim3 grid((a.rows + per_group - 1) / per_group, (w.slots + pages - 1) / pages, p.H_kv);
            if (p.longest == 1) hipLaunchKernelGGL((k_select_scores<In, DH, 1>), grid, dim3(256), 0, st, a, per_group);
            else hipLaunchKernelGGL((k_select_scores<In, DH, 2>), grid, dim3(256), 0, st, a, per_group);
        }
        if (hipError_t e = hipGetLastError()) return e;
        ProfHook ps(ADA_K_ATTN, st);
        const dim3 grid((unsigned)(((long long)a.rows * p.H_kv + 3) / 4));
        if (w.slots <= 128) hipLaunchKernelGGL((k_select_choose<In, DH, 2>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((k_select_choose<In, DH, 8>), grid, dim3(256), 0, st, a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}
