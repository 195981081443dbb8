// Which pages a token attends to.  score(page) = max over the group's heads of sum_i max(q_i lo_i, q_i hi_i): as q+ = max(q, 0) and q- =
// min(q, 0), the sum is the product of [q+, q-] with [hi, lo], a matrix product of pages by query heads over 2 d_h columns.
//
// The lists are whole numbers and have to be the ones that exact arithmetic gives, while the matrix product adds in fp32.  So the fp32
// scores only narrow it down: with tau the k-th largest of them and E a bound of their error, a page above tau + 2 E is among the k
// largest and one below tau - 2 E is not; for those between, where they are more than the places left, the sum is taken again in fp64.
//   E = (2 d_h + 16) 2^-24 max_h |q_h|_1 max |bound|: at most 2 d_h roundings, each of no more than the sum of the products' magnitudes (and 16 to
//   spare for the bound's own arithmetic).
// A workgroup takes `tokens` rows and one head of the cache; each of its waves scores 16 pages at a time, then a wave chooses for a token.
#pragma once

struct SelectArgs {
    PagedArgs p;
    const void* Q;
    long long ldq;
    int budget, first, last;
    int32_t *list, *count;
    int lg_heads, tokens, slots;                           // columns of a product: 2^lg_heads heads (a group of up to 16, or a part of it) x tokens; pages that LDS has room for
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

// The largest t with at least k of the n keys >= t (0 < k <= keys that are not 0): the k-th largest key, or, where that leaves exactly
// k of them, something between it and the next one.
template <typename Key, typename Get>
__device__ inline Key kth_largest(int n, int k, Get&& get) {
    const int lane = threadIdx.x & 63;
    Key t = 0;
    for (int bit = (int)sizeof(Key) * 8 - 1; bit >= 0; --bit) {
        const Key with = t | ((Key)1 << bit);
        int c = 0;
        for (int i0 = 0; i0 < n; i0 += 64) c += __popcll(__builtin_amdgcn_ballot_w64(i0 + lane < n && get(min(i0 + lane, n - 1)) >= with));
        if (c >= k) t = with;
        if (c == k) break;
    }
    return t;
}

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

__host__ __device__ inline size_t select_lds(int tokens, int slots) { return (size_t)tokens * slots * 12 + 16 * 4 + 64 * 4; }

template <typename In, int DH>
__global__ __launch_bounds__(512) void k_select_pages(SelectArgs a) {
    constexpr int EPP = 16 / (int)sizeof(In), KF = DH / (4 * EPP);
    extern __shared__ __align__(16) char lds[];
    const PagedArgs& p = a.p;
    double* exact_of = reinterpret_cast<double*>(lds);                         // [tokens][slots]
    uint32_t* key_of = reinterpret_cast<uint32_t*>(exact_of + a.tokens * a.slots);   // [tokens][slots]; 0: no such page
    float* qsum = reinterpret_cast<float*>(key_of + a.tokens * a.slots);       // [16] max_h |q_h|_1 of a token
    float* most = qsum + 16;                                                   // [waves] max |bound|
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4, waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kvh = blockIdx.y, end_row = min((int)(blockIdx.x + 1) * a.tokens, p.rows);
    const int per = 1 << a.lg_heads;
    for (int row0 = blockIdx.x * a.tokens; row0 < end_row;) {
        const int b = paged_find(p, row0);
        if (b >= p.B) return;                                                  // rows behind the last sequence
        const Seq s = paged_seq(p, b);
        const int stop = min(end_row, max(s.row0 + s.n, row0 + 1));            // this sequence's rows of the workgroup
        if (row0 < s.row0 || row0 >= s.row0 + s.n) { row0 = row0 + 1; continue; }
        const int n_tok = stop - row0, first_pos = s.past + row0 - s.row0;
        const int n_pages = (((p.causal ? first_pos + n_tok : s.len) - 1) >> p.lg) + 1;        // that the last of them sees
        const int32_t* table = p.table + b * p.table_stride;
        // ---- scores, 16 pages x 16 (token, head) at a time
        float largest_bound = 0.f;
        for (int h0 = 0; h0 < p.G; h0 += 16) {                                 // (groups of more than 16 heads in turns)
            const int tok = min(l16 >> a.lg_heads, n_tok - 1), head = h0 + min(l16 & (per - 1), min(p.G - h0, 16) - 1);
            const In* q = reinterpret_cast<const In*>(a.Q) + (row0 + tok) * a.ldq + (long long)(kvh * p.G + head) * DH;
            u32x4 qf[KF];
            float q1 = 0.f;
#pragma unroll
            for (int c = 0; c < KF; ++c) {
                qf[c] = *reinterpret_cast<const u32x4*>(q + (c * 4 + g) * EPP);
                q1 += abs_sum<In>(qf[c]);
            }
            q1 = sum_over_groups(q1);
            for (int o = 1; o < per; o <<= 1) q1 = fmaxf(q1, __shfl_xor(q1, o, 64));
            if (wave == 0 && g == 0 && (l16 & (per - 1)) == 0 && (l16 >> a.lg_heads) < n_tok)
                qsum[l16 >> a.lg_heads] = h0 ? fmaxf(qsum[l16 >> a.lg_heads], q1) : q1;
            for (int j0 = wave * 16; j0 < n_pages; j0 += waves * 16) {
                const int j = min(j0 + l16, n_pages - 1), page = table[j];
                const bool there = page >= 0 && page < p.pages;
                if (!there) raise(p, ADA_ERR_INDEX);
                const In* low = reinterpret_cast<const In*>(p.bounds) + ((long long)(there ? page : 0) * p.H_kv + kvh) * 2 * DH;
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
                float m = 0.f;
#pragma unroll
                for (int side = 0; side < 2; ++side) {
                    u32x4 kf[KF];
#pragma unroll
                    for (int c = 0; c < KF; ++c) kf[c] = *reinterpret_cast<const u32x4*>(low + side * DH + (c * 4 + g) * EPP);
#pragma unroll
                    for (int c = 0; c < KF; ++c) {
                        m = fmaxf(m, largest<In>(kf[c]));
                        const u32x4 qs = part<In>(qf[c], side == 0);
                        if constexpr (sizeof(In) == 2) acc = mfma16(kf[c], qs, acc);
                        else
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[c][e]), __uint_as_float(qs[e]), acc, 0, 0, 0);
                    }
                }
                if (there) largest_bound = fmaxf(largest_bound, m);
                const unsigned long long known = __builtin_amdgcn_ballot_w64(there);          // bit l16: page j0 + l16
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v = acc[e];
                    for (int o = 1; o < per; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
                    const int at = 4 * g + e, t = l16 >> a.lg_heads;
                    if ((l16 & (per - 1)) == 0 && t < n_tok && j0 + at < n_pages) {
                        uint32_t* to = key_of + t * a.slots + j0 + at;
                        const uint32_t k = (known >> at) & 1 ? ordered(v) : 0u;
                        *to = h0 ? max(*to, k) : k;
                    }
                }
            }
        }
        for (int o = 1; o < 64; o <<= 1) largest_bound = fmaxf(largest_bound, __shfl_xor(largest_bound, o, 64));
        if (lane == 0) most[wave] = largest_bound;
        __syncthreads();
        // ---- choice, a wave per token
        for (int t = wave; t < n_tok; t += waves) {
            const int row = row0 + t, have = ((p.causal ? first_pos + t : s.len - 1) >> p.lg) + 1;
            const uint32_t* key = key_of + t * a.slots;
            double* exact = exact_of + t * a.slots;
            const int lo = min(a.first, have), hi = max(lo, have - a.last), free = a.budget - lo - (have - hi);      // candidates lo .. hi - 1
            uint32_t all_from = 1, between_from = 1;       // chosen: keys >= all_from; and of those >= between_from the exact ones below
            unsigned long long exact_from = 0;
            int ties = 0;                                  // of those equal to exact_from, the first so many
            int there = 0;
            for (int i0 = lo; i0 < hi; i0 += 64) there += __popcll(__builtin_amdgcn_ballot_w64(i0 + lane < hi && key[min(i0 + lane, hi - 1)] != 0u));
            if (there > free) {
                if (free <= 0) all_from = between_from = 0xFFFFFFFFu;          // (no key is that large)
                else {
                    const uint32_t from = kth_largest<uint32_t>(hi - lo, free, [&](int i) { return key[lo + i]; });
                    uint32_t least = 0xFFFFFFFFu;          // the k-th largest key itself
                    for (int i = lo + lane; i < hi; i += 64) if (key[i] >= from) least = min(least, key[i]);
                    for (int o = 1; o < 64; o <<= 1) least = min(least, (uint32_t)__shfl_xor((int)least, o, 64));
                    float bound = 0.f;
                    for (int w = 0; w < waves; ++w) bound = fmaxf(bound, most[w]);
                    const float tau = unordered(least), err = (2 * DH + 16) * 5.9604645e-8f * qsum[t] * bound * 2.02f;
                    between_from = max(ordered(tau - err), 1u);
                    const uint32_t above = ordered(tau + err);
                    int sure = 0, open = 0;
                    for (int i0 = lo; i0 < hi; i0 += 64) {
                        const uint32_t k = i0 + lane < hi ? key[min(i0 + lane, hi - 1)] : 0u;
                        sure += __popcll(__builtin_amdgcn_ballot_w64(k > above));
                        open += __popcll(__builtin_amdgcn_ballot_w64(k >= between_from && k <= above));
                    }
                    all_from = above + 1;
                    const int need = free - sure;
                    if (open == need) all_from = between_from;
                    else {
                        for (int i0 = lo; i0 < hi; i0 += 64) {
                            const uint32_t k = i0 + lane < hi ? key[min(i0 + lane, hi - 1)] : 0u;
                            for (unsigned long long left = __builtin_amdgcn_ballot_w64(k >= between_from && k <= above); left; left &= left - 1) {
                                const int i = i0 + __ffsll(left) - 1;
                                const In* low = reinterpret_cast<const In*>(p.bounds) + ((long long)table[i] * p.H_kv + kvh) * 2 * DH;
                                double best = -INFINITY;
                                for (int h = 0; h < p.G; ++h) {
                                    const In* q = reinterpret_cast<const In*>(a.Q) + row * a.ldq + (long long)(kvh * p.G + h) * DH;
                                    double sum = 0.0;
#pragma unroll
                                    for (int c = 0; c < DH / 64; ++c) {
                                        const double x = as_double<In>(q[c * 64 + lane]);
                                        sum += x * (x < 0.0 ? as_double<In>(low[c * 64 + lane]) : as_double<In>(low[DH + c * 64 + lane]));
                                    }
                                    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
                                    best = sum > best ? sum : best;
                                }
                                if (lane == 0) exact[i] = best;
                            }
                        }
                        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                        auto open_key = [&](int i) { return key[lo + i] >= between_from && key[lo + i] <= above ? ordered(exact[lo + i]) : 0ull; };
                        const unsigned long long efrom = kth_largest<unsigned long long>(hi - lo, need, open_key);
                        unsigned long long eleast = ~0ull;
                        for (int i = lane; i < hi - lo; i += 64) {
                            const unsigned long long k = open_key(i);
                            if (k != 0ull && k >= efrom && k < eleast) eleast = k;
                        }
                        for (int o = 1; o < 64; o <<= 1) {
                            const unsigned long long k = __shfl_xor(eleast, o, 64);
                            if (k < eleast) eleast = k;
                        }
                        int over = 0;
                        for (int i0 = 0; i0 < hi - lo; i0 += 64) over += __popcll(__builtin_amdgcn_ballot_w64(i0 + lane < hi - lo && open_key(min(i0 + lane, hi - lo - 1)) > eleast));
                        exact_from = eleast;
                        ties = need - over;
                    }
                }
            }
            // ---- the list
            int32_t* to = a.list + ((long long)row * p.H_kv + kvh) * a.budget;
            const unsigned long long below = (1ull << lane) - 1;
            int n = 0, tied = 0;
            for (int i0 = 0; i0 < have; i0 += 64) {
                const int i = i0 + lane, ic = min(i, have - 1);
                const uint32_t k = key[ic];
                const bool forced = ic < lo || ic >= hi;
                bool in = i < have && k != 0u && (forced || k >= all_from), tie = false;
                if (exact_from != 0ull && i < have && !forced && k < all_from && k >= between_from) {
                    const unsigned long long e = ordered(exact[ic]);
                    in = e > exact_from;
                    tie = e == exact_from;
                }
                const unsigned long long ts = __builtin_amdgcn_ballot_w64(tie);
                if (tie && tied + __popcll(ts & below) < ties) in = true;
                tied += __popcll(ts);
                const unsigned long long ins = __builtin_amdgcn_ballot_w64(in);
                const int place = n + __popcll(ins & below);
                if (in && place < a.budget) to[place] = i;                     // (scores that are not numbers can let too many in)
                n = min(n + __popcll(ins), a.budget);
            }
            for (int i = n + lane; i < a.budget; i += 64) to[i] = -1;
            if (lane == 0) a.count[(long long)row * p.H_kv + kvh] = n;
        }
        __syncthreads();
        row0 = stop;
    }
}

template <typename In, int DH>
hipError_t launch_select(SelectArgs a, hipStream_t st) {
    const PagedArgs& p = a.p;
    a.lg_heads = 0;
    while ((1 << a.lg_heads) < (p.G < 16 ? p.G : 16)) ++a.lg_heads;
    a.slots = (p.max_pages + 1) / 2 * 2;
    // as many tokens as a product has columns for; fewer where their scores would leave room for one workgroup of a CU only
    a.tokens = p.longest == 1 ? 1 : 16 >> a.lg_heads;
    while (a.tokens > 1 && select_lds(a.tokens, a.slots) > 65536) a.tokens >>= 1;
    static std::once_flag once;
    static hipError_t attr_err = hipSuccess;
    std::call_once(once, [] {
        attr_err = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_select_pages<In, DH>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)select_lds(1, ADA_SELECT_MAX_PAGES));
    });
    if (attr_err != hipSuccess) return attr_err;
    ProfHook ps(ADA_K_ATTN, st);
    hipLaunchKernelGGL((k_select_pages<In, DH>), dim3((p.rows + a.tokens - 1) / a.tokens, p.H_kv), dim3(p.longest == 1 ? 512 : 256),
                       select_lds(a.tokens, a.slots), st, a);
    return hipGetLastError();
}
