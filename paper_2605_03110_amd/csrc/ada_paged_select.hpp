// Which pages a token attends to.  score(page) = max over the group's heads of sum_i max(q_i lo_i, q_i hi_i): as q+ = max(q, 0) and q- =
// min(q, 0), the sum is the product of [q+, q-] with [hi, lo], a matrix product of pages by query heads over 2 d_h columns.
//
// The lists are whole numbers and have to be the ones that exact arithmetic gives, while the matrix product adds in fp32.  So the fp32
// scores only narrow it down: with tau the k-th largest of them and E a bound of their error, a page above tau + 2 E is among the k
// largest and one below tau - 2 E is not; for those between, where they are more than the places left, the sum is taken again in fp64.
//   E = (2 d_h + 16) 2^-24 max_h |q_h|_1 max |bound|: at most 2 d_h roundings, each of no more than the sum of the products' magnitudes (and 16 to
//   spare for the bound's own arithmetic).
// Two launches: scores, a wave per 16 pages and some rows, to the workspace as integers in the numbers' order; then a wave per row and head of the cache
// that chooses.  (In one launch, scores in LDS: a workgroup per row was 33 us for 16 tokens at 20 to 32 thousand keys, most CUs without work, and 83 for
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

// n keys, a lane's every 64th; up to 512 are held in registers, more are asked for again each time (0: no key).
template <typename Key, typename Get> struct Keys {
    static constexpr int HELD = 8;
    const Get& get;
    int n;
    Key held[HELD];
    __device__ __forceinline__ Keys(int count, const Get& g) : get(g), n(count) { block(0, held); }
    __device__ __forceinline__ void block(int i0, Key (&k)[HELD]) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int at = i0 + i * 64 + lane;
            k[i] = i0 + i * 64 < n && at < n ? get(at) : 0;
        }
    }
    template <typename F> __device__ __forceinline__ void each(F&& f) const {                  // f(first key's number, block of keys)
        f(0, held);
        for (int i0 = 64 * HELD; i0 < n; i0 += 64 * HELD) {
            Key k[HELD];
            block(i0, k);
            f(i0, k);
        }
    }
    __device__ __forceinline__ int count(Key from) const {                 // keys >= from (> 0)
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
        for (int bit = (int)sizeof(Key) * 8 - 1; bit >= 0; --bit) {
            const Key with = t | ((Key)1 << bit);
            const int c = count(with);
            if (c >= k) t = with;
            if (c == k) break;                             // (the k largest are those >= t: the smallest of them is meant)
        }
        Key least = ~(Key)0;
        each([&](int, const Key (&key)[HELD]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) if (key[i] >= t && key[i] < least) least = key[i];
        });
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const Key other = __shfl_xor(least, o, 64);
            if (other < least) least = other;
        }
        return least;
    }
};
template <typename Key, typename Get> __device__ inline Keys<Key, Get> keys_of(int n, const Get& get) { return Keys<Key, Get>(n, get); }

template <typename In> __device__ inline u32x4 part(u32x4 w, bool negative);   // the negative entries, or the others; 0 elsewhere
template <> __device__ inline u32x4 part<uint16_t>(u32x4 w, bool negative) {
    const u32x4 m = ((w >> 15) & 0x00010001u) * 0xFFFFu;
    return negative ? w & m : w & ~m;
}
template <> __device__ inline u32x4 part<float>(u32x4 w, bool negative) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = ((w[i] >> 31) != 0) == negative ? w[i] : 0u;
    return r;
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

// Scores: a workgroup takes 64 pages (a wave 16), `per_group` rows and a head of the cache.
template <typename In, int DH>
__global__ __launch_bounds__(256) void k_select_scores(SelectArgs a, int per_group) {
    constexpr int EPP = 16 / (int)sizeof(In), KF = DH / (4 * EPP);
    const PagedArgs& p = a.p;
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, kvh = blockIdx.z;
    const int j0 = blockIdx.x * 64 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 16;
    const int per = 1 << a.lg_heads, tokens = 16 >> a.lg_heads;                // columns: a token's heads side by side
    const int end = min((int)(blockIdx.y + 1) * per_group, a.rows) + a.row0;
    for (int row = blockIdx.y * per_group + a.row0; row < end;) {
        const int b = paged_find(p, row);
        if (b >= p.B) return;                                                  // rows behind the last sequence
        const Seq s = paged_seq(p, b);
        if (row < s.row0 || row >= s.row0 + s.n) { ++row; continue; }
        const int stop = min(end, s.row0 + s.n);                               // this sequence's rows
        const int n_pages = (((p.causal ? s.past + stop - s.row0 : s.len) - 1) >> p.lg) + 1;  // that the last of them sees
        if (j0 >= n_pages) { row = stop; continue; }
        const int page = p.table[b * p.table_stride + min(j0 + l16, n_pages - 1)];
        const bool there = page >= 0 && page < p.pages;
        if (!there) raise(p, ADA_ERR_INDEX);
        const In* low = reinterpret_cast<const In*>(p.bounds) + ((long long)(there ? page : 0) * p.H_kv + kvh) * 2 * DH;
        u32x4 kf[2][KF];
#pragma unroll
        for (int side = 0; side < 2; ++side)
#pragma unroll
            for (int c = 0; c < KF; ++c) kf[side][c] = *reinterpret_cast<const u32x4*>(low + side * DH + (c * 4 + g) * EPP);
        float most = 0.f;
#pragma unroll
        for (int side = 0; side < 2; ++side)
#pragma unroll
            for (int c = 0; c < KF; ++c) most = fmaxf(most, largest<In>(kf[side][c]));
        most = there ? most : 0.f;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
        const unsigned long long known = __builtin_amdgcn_ballot_w64(there);  // bit l16: page j0 + l16
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
        for (; row < stop; row += tokens) {
            float best[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            for (int h0 = 0; h0 < p.G; h0 += 16) {                             // (groups of more than 16 heads in turns)
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int side = 0; side < 2; ++side)
#pragma unroll
                    for (int c = 0; c < KF; ++c) {
                        const u32x4 qs = part<In>(qf[c], side == 0);
                        if constexpr (sizeof(In) == 2) acc = mfma16(kf[side][c], qs, acc);
                        else
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[side][c][e]), __uint_as_float(qs[e]), acc, 0, 0, 0);
                    }
                const bool more = h0 + 16 < p.G;
                if (more || row + tokens < stop) fetch(query(more ? row : row + tokens, more ? h0 + 16 : 0));
#pragma unroll
                for (int e = 0; e < 4; ++e) best[e] = fmaxf(best[e], acc[e]);
            }
            u32x4 key;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float v = best[e];
                for (int o = 1; o < per; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
                key[e] = (known >> (4 * g + e)) & 1 ? ordered(v) : 0u;
            }
            if (sub == 0 && row + tok < stop) {
                const long long at = ((long long)(row + tok - a.row0) * p.H_kv + kvh) * a.slots + j0;
                *reinterpret_cast<u32x4*>(a.key + at + 4 * g) = key;
                if (g == 0) a.most[at >> 4] = most;
            }
        }
        row = stop;
    }
}

// One page's score in fp64, in all lanes: 16 lanes share a head, four heads at a time.
template <typename In, int DH>
__device__ inline double exact_score(int G, const In* q_row, const In* low) {
    constexpr int C = DH / 16, W = C * (int)sizeof(In) / 4;                    // columns and 32-bit words of a lane
    const int lane = threadIdx.x & 63, c0 = (lane & 15) * C;
    uint32_t lo[W], hi[W];
    __builtin_memcpy(lo, __builtin_assume_aligned(low + c0, 8), sizeof(lo));
    __builtin_memcpy(hi, __builtin_assume_aligned(low + DH + c0, 8), sizeof(hi));
    auto value = [](const uint32_t (&w)[W], int c) {
        if constexpr (sizeof(In) == 4) return (double)__uint_as_float(w[c]);
        else return (double)(c & 1 ? bf16_hi(w[c >> 1]) : bf16_lo(w[c >> 1]));
    };
    double best = -INFINITY;
    for (int h0 = 0; h0 < G; h0 += 4) {
        uint32_t q[W];
        __builtin_memcpy(q, __builtin_assume_aligned(q_row + (long long)min(h0 + (lane >> 4), G - 1) * DH + c0, 8), sizeof(q));
        double sum = 0.0;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const double x = value(q, c);
            sum += x * (x < 0.0 ? value(lo, c) : value(hi, c));
        }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) sum += __shfl_xor(sum, o, 64);
        best = sum > best ? sum : best;
    }
#pragma unroll
    for (int o = 16; o < 64; o <<= 1) {
        const double other = __shfl_xor(best, o, 64);
        best = other > best ? other : best;
    }
    return best;
}

template <typename In, int DH>
__global__ __launch_bounds__(256) void k_select_choose(SelectArgs a) {
    constexpr int EPP = 16 / (int)sizeof(In), LPR = DH / EPP;                  // lanes that read a head
    const PagedArgs& p = a.p;
    const int lane = threadIdx.x & 63;
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (unit >= a.rows * p.H_kv) return;
    const int row = a.row0 + unit / p.H_kv, kvh = unit % p.H_kv, b = paged_find(p, row);
    if (b >= p.B) return;
    const Seq s = paged_seq(p, b);
    if (row < s.row0 || row >= s.row0 + s.n) return;
    const int have = ((p.causal ? s.past + row - s.row0 : s.len - 1) >> p.lg) + 1;
    const int lo = min(a.first, have), hi = max(lo, have - a.last), free = a.budget - lo - (have - hi);      // candidates lo .. hi - 1
    const uint32_t* key = a.key + (long long)unit * a.slots;
    const int32_t* table = p.table + b * p.table_stride;
    const In* q_row = reinterpret_cast<const In*>(a.Q) + row * a.ldq + (long long)kvh * p.G * DH;
    int32_t* to = a.list + ((long long)row * p.H_kv + kvh) * a.budget;
    int n = 0;
    const unsigned long long below = (1ull << lane) - 1;
    auto put_out = [&](bool in, int page) __attribute__((always_inline)) {
        const unsigned long long ins = __builtin_amdgcn_ballot_w64(in);
        const int place = n + __popcll(ins & below);
        if (in && place < a.budget) to[place] = page;      // (scores that are not numbers can let too many in)
        n = min(n + __popcll(ins), a.budget);
    };
    auto forced = [&](int from, int end) {
        for (int i0 = from; i0 < end; i0 += 64) put_out(i0 + lane < end && key[min(i0 + lane, end - 1)] != 0u, i0 + lane);
    };
    forced(0, lo);
    const auto get = [&](int i) { return key[lo + i]; };
    const auto candidates = keys_of<uint32_t>(hi - lo, get);
    // chosen: keys >= all_from; of the others from between_from on ("open") those whose exact score is above exact_from, and the first `ties` equal to it
    uint32_t all_from = 1, between_from = 1;
    if (candidates.count(1) <= free) {
        candidates.each([&](int i0, const uint32_t (&k)[8]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) if (i0 + i * 64 < hi - lo) put_out(k[i] != 0u, lo + i0 + i * 64 + lane);
        });
    } else if (free > 0) {
        // what the scores are exact to
        float q1 = 0.f, most = 0.f;
        for (int h0 = 0; h0 < p.G; h0 += 64 / LPR) {
            float sum = abs_sum<In>(*reinterpret_cast<const u32x4*>(q_row + (long long)min(h0 + lane / LPR, p.G - 1) * DH + (lane % LPR) * EPP));
#pragma unroll
            for (int o = 1; o < LPR; o <<= 1) sum += __shfl_xor(sum, o, 64);
            q1 = fmaxf(q1, sum);
        }
        const float* m = a.most + (long long)unit * (a.slots >> 4);
        for (int i = lane; i < (have + 15) >> 4; i += 64) most = fmaxf(most, m[i]);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            q1 = fmaxf(q1, __shfl_xor(q1, o, 64));
            most = fmaxf(most, __shfl_xor(most, o, 64));
        }
        const float tau = unordered(candidates.kth(free)), err = (2 * DH + 16) * 5.9604645e-8f * q1 * most * 2.02f;
        between_from = max(ordered(tau - err), 1u);
        const uint32_t above = ordered(tau + err);
        all_from = above + 1;
        const int sure = candidates.count(all_from), open = candidates.count(between_from) - sure, need = free - sure;
        auto is_open = [&](uint32_t k) { return k >= between_from && k <= above; };
        if (open == need) all_from = between_from;
        if (open == need || open <= 64) {
            unsigned long long chosen = 0;                 // of the open pages, by their order
            if (open != need) {
                unsigned long long mine = 0;               // lane i: the exact score of the i-th
                int i = 0;
                candidates.each([&](int i0, const uint32_t (&k)[8]) __attribute__((always_inline)) {
#pragma unroll
                    for (int w = 0; w < 8; ++w)
                        for (unsigned long long left = i0 + w * 64 < hi - lo ? __builtin_amdgcn_ballot_w64(is_open(k[w])) : 0ull; left; left &= left - 1, ++i) {
                            const int page = lo + i0 + w * 64 + __ffsll(left) - 1;
                            const double e = exact_score<In, DH>(p.G, q_row, reinterpret_cast<const In*>(p.bounds) + ((long long)table[page] * p.H_kv + kvh) * 2 * DH);
                            if (lane == i) mine = ordered(e);
                        }
                });
                int taken = 0;                             // one place after the other: the largest left, the first of equal ones
                for (; taken < need; ++taken) {
                    unsigned long long top = (chosen >> lane) & 1 ? 0ull : mine;
#pragma unroll
                    for (int o = 1; o < 64; o <<= 1) {
                        const unsigned long long other = __shfl_xor(top, o, 64);
                        top = other > top ? other : top;
                    }
                    const unsigned long long at = __builtin_amdgcn_ballot_w64(mine == top && !((chosen >> lane) & 1));
                    chosen |= at & (~at + 1);
                }
            }
            int seen = 0;
            candidates.each([&](int i0, const uint32_t (&k)[8]) __attribute__((always_inline)) {
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    if (i0 + w * 64 >= hi - lo) continue;
                    const bool o = is_open(k[w]) && k[w] < all_from;
                    const unsigned long long os = __builtin_amdgcn_ballot_w64(o);
                    put_out((k[w] != 0u && k[w] >= all_from) || (o && (chosen >> ((seen + __popcll(os & below)) & 63)) & 1), lo + i0 + w * 64 + lane);
                    seen += __popcll(os);
                }
            });
        } else {
            // more than 64 within the error of each other (alike pages, queries of zeros): every lane takes the sums of its own pages
            const auto open_key = [&](int i) {
                if (!is_open(key[lo + i])) return 0ull;
                const In* low = reinterpret_cast<const In*>(p.bounds) + ((long long)table[lo + i] * p.H_kv + kvh) * 2 * DH;
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
            const auto opens = keys_of<unsigned long long>(hi - lo, open_key);
            const unsigned long long exact_from = opens.kth(need);
            const int ties = need - opens.count(exact_from + 1);
            int tied = 0;
            opens.each([&](int i0, const unsigned long long (&e)[8]) __attribute__((always_inline)) {
                uint32_t k[8];
                candidates.block(i0, k);
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    if (i0 + w * 64 >= hi - lo) continue;
                    const unsigned long long ts = __builtin_amdgcn_ballot_w64(e[w] == exact_from);
                    put_out(k[w] >= all_from || e[w] > exact_from || (e[w] == exact_from && tied + __popcll(ts & below) < ties), lo + i0 + w * 64 + lane);
                    tied += __popcll(ts);
                }
            });
        }
    }
    forced(hi, have);
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
    const int per_group = p.longest == 1 ? 1 : 64;         // rows that share a wave's pages
    for (a.row0 = 0; a.row0 < p.rows; a.row0 += a.rows) {
        a.rows = p.rows - a.row0 < w.rows ? p.rows - a.row0 : w.rows;
        {
            ProfHook ps(ADA_K_ATTN, st);
            hipLaunchKernelGGL((k_select_scores<In, DH>), dim3((w.slots + 63) / 64, (a.rows + per_group - 1) / per_group, p.H_kv), dim3(256), 0, st, a, per_group);
        }
        if (hipError_t e = hipGetLastError()) return e;
        ProfHook ps(ADA_K_ATTN, st);
        hipLaunchKernelGGL((k_select_choose<In, DH>), dim3((unsigned)(((long long)a.rows * p.H_kv + 3) / 4)), dim3(256), 0, st, a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}
