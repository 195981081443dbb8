// Attention of new tokens over a paged cache, and over listed pages of it.
//
// A head of the cache and up to 16 of the query rows that read it (tokens x heads of the group, flat row = token * G + head) make a tile.  Its
// keys come in units of 128; the tiles stand in one line, each as long as its units and what beginning it costs, and the line is cut into as many equal
// pieces as there are workgroups, so that one long sequence and many short ones fill the chip alike.  A piece that holds a whole tile writes the
// output; a tile that is cut leaves rows, maxima and sums per piece, and whoever of its pieces comes last puts them together in the order of
// the keys (the same result on every run).
//
// Inside a unit each of the four waves takes 32 keys: S^T = K Q^T with keys straight from memory in registers (a lane's 16 bytes of one key are the operand
// as it is), softmax over keys = registers and two lane swaps, O^T += V^T P^T with the weights as they come out of the first product.  In bf16 the values
// pass through LDS and are read transposed; weights enter as pairs hi + lo of bf16 (2^-17 relative), which costs nothing where memory bounds.  In fp32
// the matrix instruction takes one number per lane and the column order of O is free, so that a lane's 16 bytes of a value row serve without LDS.
#pragma once

struct AttendArgs {
    PagedArgs p;
    const void* Q;
    long long ldq;
    void* out;
    long long ld_out;
    float sc2;                                             // log2(e) / sqrt(d_h)
    const int32_t *list, *count;                           // listed pages, or NULL
    int budget;
    const long long* prefix;                               // [tiles + 1] line in front of a tile of one head (k_paged_plan)
    const int2* tile;                                      // [tiles] its sequence and number in it
    const int* tiles;
    int* arrived;                                          // [pieces] parts of the tile that begins in a piece and is cut; zero between calls
    float *part_o, *part_ml;                               // per piece two cut tiles: rows, and [rows][2] maxima and sums
};

constexpr int TILE_ROWS = 16, UNIT = 128, WAVE_KEYS = 32;
constexpr int BEGIN = 2;                                   // what beginning a tile costs, in units (its place, queries, first keys, outputs)

// ------------------------------------------------------------------------------------------------ who does what
// How tiles stand in the line of one head of the cache.
enum { CHUNKS,                                             // sequences of many tiles: as k_paged_plan has put down
       TOKENS,                                             // a tile per sequence: every wave sums up the lengths itself
       LISTED };                                           // listed pages: tiles of one row, all alike

// One workgroup.  `room`: tiles that prefix and tile hold; more can only be where sequences overlap (a start that descends): they are left out.
__global__ __launch_bounds__(1024) void k_paged_plan(PagedArgs p, int tile_rows, int unit, int room, long long* prefix, int2* tile, int* tiles) {
    __shared__ int base[ADA_MAX_BATCH + 1];
    __shared__ long long sums[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // inclusive sum over the workgroup's values
    auto scan = [&](long long v) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const long long u = __shfl_up(v, o, 64);
            if (lane >= o) v += u;
        }
        __syncthreads();
        if (lane == 63) sums[wave] = v;
        __syncthreads();
        for (int w = 0; w < wave; ++w) v += sums[w];
        return v;
    };
    int carry = 0;
    for (int b0 = 0; b0 < p.B; b0 += 1024) {
        const int b = b0 + tid;
        const long long mine = b < p.B ? ((long long)paged_seq(p, b).n * p.G + tile_rows - 1) / tile_rows : 0;
        const long long upto = carry + scan(mine);
        if (upto > room) raise(p, ADA_ERR_SHAPE);
        if (b < p.B) base[b + 1] = (int)min(upto, (long long)room);
        __syncthreads();
        carry = base[min(b0 + 1024, p.B)];
    }
    if (tid == 0) base[0] = 0;
    __syncthreads();
    const int n_tiles = base[p.B];
    long long front = 0;
    for (int t0 = 0; t0 < n_tiles; t0 += 1024) {
        const int t = t0 + tid;
        long long mine = 0;
        if (t < n_tiles) {
            int lo = 0, hi = p.B;                          // the last b with base[b] <= t
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (base[mid] <= t) lo = mid; else hi = mid;
            }
            const int j = t - base[lo];
            const Seq s = paged_seq(p, lo);
            const int last = (int)min((long long)s.n - 1, ((long long)(j + 1) * tile_rows - 1) / p.G);
            mine = ((p.causal ? s.past + last + 1 : s.len) + unit - 1) / unit + BEGIN;
            tile[t] = {lo, j};
        }
        const long long upto = front + scan(mine);
        if (t < n_tiles) prefix[t + 1] = upto;
        __syncthreads();
        if (tid == 1023) sums[0] = upto;
        __syncthreads();
        front = sums[0];
        __syncthreads();
    }
    if (tid == 0) { prefix[0] = 0; *tiles = n_tiles; }
}

// The same for up to 64 sequences and as many tiles as make 16 rounds of one wave: no barriers (six sequences, fp32, 12 x 64: 20.7 -> 19.4 us a call).
__global__ __launch_bounds__(64) void k_paged_plan_few(PagedArgs p, int tile_rows, int unit, int room, long long* prefix, int2* tile, int* tiles) {
    const int lane = threadIdx.x;
    Seq mine = {0, 0, 0, 0};
    if (lane < p.B) mine = paged_seq(p, lane);
    long long upto = ((long long)mine.n * p.G + tile_rows - 1) / tile_rows;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long long u = __shfl_up(upto, o, 64);
        if (lane >= o) upto += u;
    }
    if (upto > room) raise(p, ADA_ERR_SHAPE);
    const int ends = (int)min(upto, (long long)room), n_tiles = __shfl(ends, 63, 64);     // tiles up to and with sequence `lane`
    long long front = 0;
    for (int t0 = 0; t0 < n_tiles; t0 += 64) {
        const int t = t0 + lane;
        int b = 0;                                         // the first whose tiles end behind t
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) b += __shfl(ends, b + o - 1, 64) <= t ? o : 0;
        const int before = __shfl(ends, max(b - 1, 0), 64), j = t - (b > 0 ? before : 0);
        const int n = __shfl(mine.n, b, 64), past = __shfl(mine.past, b, 64);
        const int last = (int)min((long long)n - 1, ((long long)(j + 1) * tile_rows - 1) / p.G);
        long long sum = t < n_tiles ? ((p.causal ? past + last + 1 : past + n) + unit - 1) / unit + BEGIN : 0;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const long long u = __shfl_up(sum, o, 64);
            if (lane >= o) sum += u;
        }
        if (t < n_tiles) {
            tile[t] = {b, j};
            prefix[t + 1] = front + sum;
        }
        front += __shfl(sum, 63, 64);
    }
    if (lane == 0) { prefix[0] = 0; *tiles = n_tiles; }
}

// A tile of one head, and where it stands in the line.
struct Tile {
    long long at;
    int units, kvh;
    Seq s;
    int b, j;                                              // rows j * (rows of a tile) .. of the sequence's n G, or (LISTED) of the token's G
    int row;                                               // LISTED: the token's row
    bool any;                                              // somebody's (LISTED: the row may be nobody's)
};

template <int MODE> struct Line {
    const AttendArgs& a;
    long long per_head, total;
    int units;                                             // LISTED: of every tile
    long long upto;                                        // TOKENS: the line up to and with sequence `lane` of the first 64
    __device__ explicit Line(const AttendArgs& args) : a(args), units(0), upto(0) {
        const PagedArgs& p = a.p;
        if (MODE == LISTED) {
            units = (int)((((long long)a.budget << p.lg) + UNIT - 1) / UNIT);
            per_head = (long long)p.rows * ((p.G + TILE_ROWS - 1) / TILE_ROWS) * (units + BEGIN);
        } else if (MODE == TOKENS) {
            upto = sums(0);
            per_head = scalar(__shfl(upto, 63, 64));
            for (int b0 = 64; b0 < p.B; b0 += 64) per_head += scalar(__shfl(sums(b0), 63, 64));
        } else {
            per_head = a.prefix[*a.tiles];
        }
        per_head = scalar(per_head);
        total = per_head * p.H_kv;
    }
    __device__ static int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }
    __device__ static long long scalar(long long v) {
        return (long long)(((unsigned long long)(uint32_t)scalar((int)(v >> 32)) << 32) | (uint32_t)scalar((int)v));
    }
    // inclusive sums of the lengths of sequences b0 .. b0 + 63
    __device__ long long sums(int b0) const {
        const int lane = threadIdx.x & 63;
        long long v = 0;
        if (b0 + lane < a.p.B) {
            const Seq s = paged_seq(a.p, b0 + lane);
            if (s.n > 0) v = (s.len + UNIT - 1) / UNIT + BEGIN;
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const long long u = __shfl_up(v, o, 64);
            if (lane >= o) v += u;
        }
        return v;
    }
    // The tile at x, all of it in scalar registers.
    __device__ Tile find(long long x) const {
        const PagedArgs& p = a.p;
        const int lane = threadIdx.x & 63;
        Tile t;
        t.s = {0, 0, 0, 0};
        t.row = 0;
        t.j = 0;
        t.any = true;
        t.kvh = scalar((int)(x / per_head));
        const long long y = x - t.kvh * per_head;
        if (MODE == LISTED) {
            const int per_row = (p.G + TILE_ROWS - 1) / TILE_ROWS;
            const long long i = y / (units + BEGIN);
            t.units = units;
            t.at = scalar(t.kvh * per_head + i * (units + BEGIN));
            t.row = scalar((int)(i / per_row));
            t.j = scalar((int)(i % per_row));
            t.b = scalar(paged_find(p, t.row));
            t.any = t.b < p.B;
            if (!t.any) return t;
        } else if (MODE == TOKENS) {
            long long front = 0, v = upto;
            int b0 = 0;
            for (;;) {
                const long long all = __shfl(v, 63, 64);
                if (y < front + all || b0 + 64 >= p.B) break;
                front += all;
                b0 += 64;
                v = sums(b0);
            }
            const int in = __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(front + v > y)) - 1;
            t.b = scalar(b0 + in);
            t.at = scalar(t.kvh * per_head + front + (in > 0 ? __shfl(v, in - 1, 64) : 0));
        } else {
            int lo = 0, hi = *a.tiles;                     // prefix[lo] <= y < prefix[hi]
            while (hi - lo > 1) {
                const int step = (hi - lo + 63) / 64, at = lo + lane * step;
                const int k = __popcll(__builtin_amdgcn_ballot_w64(at < hi && a.prefix[min(at, hi - 1)] <= y)) - 1;
                lo += k * step;
                hi = min(hi, lo + step);
            }
            lo = scalar(lo);
            t.at = scalar(t.kvh * per_head + a.prefix[lo]);
            t.units = scalar((int)(a.prefix[lo + 1] - a.prefix[lo])) - BEGIN;
            t.b = scalar(a.tile[lo].x);
            t.j = scalar(a.tile[lo].y);
        }
        const Seq s = paged_seq(p, t.b);
        t.s = {scalar(s.row0), scalar(s.n), scalar(s.past), scalar(s.len)};
        if (MODE == TOKENS) t.units = (t.s.len + UNIT - 1) / UNIT;
        if (MODE == LISTED) t.any = t.row >= t.s.row0 && t.row < t.s.row0 + t.s.n;
        return t;
    }
};

// The shortest piece worth having, for tiles of so many units: the workgroups of a tile do units / parts of its work beside each other, the one that joins takes
// the parts one after the other, and a part costs it about what a unit does (16-row tiles: a quarter): least where parts = sqrt(units).  us a call with
// a piece for every workgroup and so: one token at 8000 keys, 32 x 128 over 8, 23.6 and 16.5; with 16 x 256 over 8 58.6 and 31.8; 64 rows of two heads at 8000 keys in
// 128-row tiles 92 and 41.
__device__ inline long long least_of(float units) { return max((long long)__builtin_sqrtf(units), 1LL); }

// The workgroup's piece of the line: x0 .. x1 - 1 of `pieces`.  Where not every workgroup could have `many` of the shortest, one per CU gets a piece: two of
// them on a CU run at half the rate each, and the parts would be twice as many.  16-row tiles, 4 (fp32 2): 16 sequences with 32 listed pages 32.1 -> 28.5 us a call, 4 tokens at
// 8000 keys 32.2 -> 28.5.  128-row tiles: 1, and 2 with heads of 128: 512 rows at 8000 keys 71 -> 50, eight times 128 rows 82 -> 71.
struct Piece {
    long long total, x0, x1;
    int me, pieces;
    __device__ Piece(long long length, long long least, int per_cu, int many) : total(length) {
        long long most = total / least;
        if (most < (long long)many * gridDim.x) most = min(most, (long long)gridDim.x / per_cu);
        pieces = (int)max(min((long long)gridDim.x, most), 1LL);               // (none is empty)
        me = (int)blockIdx.x < pieces ? by_xcd(blockIdx.x, pieces) : (int)blockIdx.x;
        x0 = me < pieces ? from(me) : 0;
        x1 = me < pieces ? from(me + 1) : 0;
    }
    __device__ long long from(int w) const { return w * total / pieces; }
    __device__ int of(long long x) const { return (int)(((x + 1) * pieces - 1) / total); }
};

// A tile's units in a piece: k0 .. k1 - 1.
struct Part {
    int k0, k1;
    __device__ Part(const Piece& c, const Tile& t, long long x) {
        k0 = (int)max(x - t.at - BEGIN, 0LL);
        k1 = (int)min(max(c.x1 - t.at - BEGIN, 0LL), (long long)t.units);
    }
    __device__ bool whole(const Tile& t) const { return k0 == 0 && k1 == t.units; }
    __device__ long long slot(const Piece& c) const { return 2LL * c.me + (k0 == 0 ? 1 : 0); }
};

// Parts of cut tiles pass between XCDs, each of which has an L2 of its own: stored through it, read past it.  (Fences instead, which write back and drop
// whole L2s: 64 single tokens at 100 to 8191 keys took 382 us.)
__device__ inline void put(float* at, float x, float y) {
    const f32x2 v = {x, y};
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(at), __builtin_bit_cast(unsigned long long, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline f32x2 get(const float* at) {
    return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<const unsigned long long*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// Behind the stores of a cut tile's part: true in the workgroup that comes last, with the pieces first .. last that have one.  flag: a word in LDS.
__device__ inline bool comes_last(const AttendArgs& a, const Piece& c, const Tile& t, int& first, int& last, int* flag) {
    first = c.of(t.at + BEGIN);
    last = c.of(t.at + BEGIN + t.units - 1);
    __builtin_amdgcn_s_waitcnt(0x0F70);                    // vmcnt(0): this wave's stores have arrived
    __syncthreads();
    if (threadIdx.x == 0) {
        const bool all = __hip_atomic_fetch_add(a.arrived + first, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == last - first;
        if (all) __hip_atomic_store(a.arrived + first, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // as it was found
        *flag = all;
    }
    __syncthreads();
    return *flag != 0;
}

// Row r of a tile of ROWS: its row of Q and head of the group; false where the tile has no such row.
template <int MODE, int ROWS>
__device__ inline bool tile_row(const AttendArgs& a, const Tile& t, int r, int& row, int& head, int& token) {
    if (MODE == LISTED) {
        head = t.j * ROWS + r;
        row = t.row;
        token = t.row - t.s.row0;
        return head < a.p.G;
    }
    const int flat = t.j * ROWS + r;
    token = flat / a.p.G;
    head = flat - token * a.p.G;
    row = t.s.row0 + token;
    return token < t.s.n;
}

// ------------------------------------------------------------------------------------------------ products
template <typename In, int DH> struct Rows {               // bf16
    static constexpr int EPP = 8, KF = DH / 32, VF = DH / 16, NB = DH / 16;
    static constexpr int PITCH = DH * 2 + 32;              // 16 rows read 32 bytes each without meeting on a bank
    static constexpr int V_LDS = WAVE_KEYS * PITCH;
};
template <int DH> struct Rows<float, DH> {
    static constexpr int EPP = 4, KF = DH / 16, VF = DH / 8, NB = DH / 16;
    static constexpr int V_LDS = 0;
};

__device__ inline f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <typename In, int DH> constexpr int rows_lds() {
    constexpr int out = 4 * TILE_ROWS * (DH + 4) * 4, v = 4 * Rows<In, DH>::V_LDS;
    return (out > v ? out : v) + 2 * 4 * TILE_ROWS * 4 + 16;
}

// A row of the output, or of a cut tile, from the thread that has DH / 16 columns of it.
template <typename In, int DH>
__device__ inline void store_out(In* to, const float (&o)[DH / 16], float f) {
    if constexpr (sizeof(In) == 4) {
#pragma unroll
        for (int c = 0; c < DH / 16; c += 4) *reinterpret_cast<f32x4*>(to + c) = f32x4{o[c] * f, o[c + 1] * f, o[c + 2] * f, o[c + 3] * f};
    } else {
        uint32_t w[DH / 32];
#pragma unroll
        for (int c = 0; c < DH / 32; ++c) w[c] = bf16_pair(o[2 * c] * f, o[2 * c + 1] * f);
        if constexpr (DH == 64) *reinterpret_cast<u32x2*>(to) = u32x2{w[0], w[1]};
        else
#pragma unroll
            for (int c = 0; c < DH / 32; c += 4) *reinterpret_cast<u32x4*>(to + 2 * c) = u32x4{w[c], w[c + 1], w[c + 2], w[c + 3]};
    }
}

template <typename In, int DH, int MODE>
__global__ __launch_bounds__(256, DH * sizeof(In) > 256 ? 1 : 2) void k_paged_rows(AttendArgs a) {
    using R = Rows<In, DH>;
    constexpr int KF = R::KF, VF = R::VF, NB = R::NB;
    extern __shared__ __align__(16) char lds[];
    const PagedArgs& p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    float* obuf = reinterpret_cast<float*>(lds);           // [4][16][DH + 4], over the values' place
    float* mbuf = reinterpret_cast<float*>(lds + rows_lds<In, DH>() - 2 * 4 * TILE_ROWS * 4 - 16);
    float* lbuf = mbuf + 4 * TILE_ROWS;
    int* flag = reinterpret_cast<int*>(lbuf + 4 * TILE_ROWS);
    const Line<MODE> line(a);
    if (line.total == 0) return;
    const Piece piece(line.total, least_of(0.25f * (float)line.per_head / (MODE == CHUNKS ? *a.tiles : MODE == TOKENS ? p.B : p.rows)), 2, sizeof(In) == 2 ? 4 : 2);

    for (long long x = piece.x0; x < piece.x1;) {
        const Tile t = line.find(x);
        const Part part(piece, t, x);
        const int k0 = part.k0, k1 = part.k1;
        x = t.at + BEGIN + t.units;
        if (!t.any || k0 >= k1) continue;
        // ---- queries: the operand of lane (column l16 = row of the tile)
        int row, head, token;
        const bool mine = tile_row<MODE, TILE_ROWS>(a, t, l16, row, head, token);
        if (!mine) {                                       // (products with row 0, never stored)
            int h0, t0;
            tile_row<MODE, TILE_ROWS>(a, t, 0, row, h0, t0);
            head = h0; token = t0;
        }
        const In* q = reinterpret_cast<const In*>(a.Q) + row * a.ldq + (long long)(t.kvh * p.G + head) * DH;
        u32x4 qf[KF];
#pragma unroll
        for (int c = 0; c < KF; ++c) qf[c] = *reinterpret_cast<const u32x4*>(q + (c * 4 + g) * R::EPP);
        const int limit = p.causal ? t.s.past + token + 1 : t.s.len;                  // keys below it are seen
        const long long lrow = MODE == LISTED ? (long long)t.row * p.H_kv + t.kvh : 0;
        const int32_t* list = MODE == LISTED ? a.list + lrow * a.budget : nullptr;
        const int n_list = MODE == LISTED ? min(max(a.count[lrow], 0), a.budget) : 0;
        const int n_pages = MODE == LISTED ? n_list : ((t.s.len - 1) >> p.lg) + 1;

        // Pages, 64 at a time, a lane each: number in the sequence (listed ones are in any place) and in the pool, -1 where there is none.  The even sixty-fours and
        // the odd ones; the next come in while this one's keys are taken, so that no unit waits for a number.
        struct Window { int named, page; };
        auto window = [&](int w) {
            const int i = w * 64 + lane;
            Window r = {i, -1};
            bool ok = i < n_pages;
            if (MODE == LISTED && ok) {
                const int before = i > 0 ? list[i - 1] : -1;
                r.named = list[i];
                ok = r.named > before && r.named <= (t.s.len - 1) >> p.lg;
                if (!ok) raise(p, ADA_ERR_INDEX);
            }
            if (ok) {
                r.page = p.table[t.b * p.table_stride + r.named];
                if (r.page < 0 || r.page >= p.pages) {
                    raise(p, ADA_ERR_INDEX);
                    r.page = -1;
                }
            }
            return r;
        };
        const int lg_span = p.lg - 1;                      // units of a window
        Window even, odd;
        {
            const int w = k0 >> lg_span;
            const Window w0 = window(w), w1 = window(w + 1);
            even = w & 1 ? w1 : w0;
            odd = w & 1 ? w0 : w1;
        }
        // the wave's two groups of 16 keys: first position (NOWHERE: nothing to see), the last row that is there, where they lie
        u32x4 kf[2][KF], vf[VF];
        int pos[2], rows[2];
        const char *kat[2], *vat[2];
        const uint32_t step = (uint32_t)p.slot_stride * (uint32_t)sizeof(In);          // bytes from key to key: 15 of them fit into 32 bits
        auto where = [&](int u) {                          // false: none of the wave's 32 keys of unit u is there
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int v = u * UNIT + wave * WAVE_KEYS + 16 * i, n = v >> p.lg, in = v & ((1 << p.lg) - 1);
                const bool second = (n >> 6) & 1;
                const int page = __builtin_amdgcn_readlane(second ? odd.page : even.page, n & 63);
                const int named = MODE == LISTED ? __builtin_amdgcn_readlane(second ? odd.named : even.named, n & 63) : n;
                pos[i] = n < n_pages && page >= 0 ? (named << p.lg) + in : NOWHERE;
                if (pos[i] >= t.s.len) pos[i] = NOWHERE;
                rows[i] = t.s.len - 1 - pos[i];
                const long long at = (page * p.page_stride + in * p.slot_stride + t.kvh * p.head_stride) * (long long)sizeof(In);
                kat[i] = reinterpret_cast<const char*>(p.K) + at;
                vat[i] = reinterpret_cast<const char*>(p.V) + at;
            }
            if (pos[0] == NOWHERE && pos[1] == NOWHERE) return false;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (pos[i] == NOWHERE) { rows[i] = rows[1 - i]; kat[i] = kat[1 - i]; vat[i] = vat[1 - i]; }     // (read, and seen by nobody)
            return true;
        };
        // rows behind the sequence's end are not read: the last one stands in (its weight is 0)
        const uint32_t koff = l16 * step + g * 16;
        auto fetch_k = [&]() {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t off = rows[i] >= 15 ? koff : min(l16, rows[i]) * step + g * 16;
#pragma unroll
                for (int c = 0; c < KF; ++c) kf[i][c] = *reinterpret_cast<const u32x4*>(kat[i] + off + c * 64);
            }
        };
        auto fetch_v = [&]() {
            if constexpr (sizeof(In) == 2) {               // rows by pieces, as LDS takes them
                constexpr int PPR = DH / 8, RPI = 64 / PPR;
#pragma unroll
                for (int u = 0; u < VF; ++u) {
                    const int i = u * RPI / 16, r = u * RPI % 16;
                    const uint32_t off = (rows[i] >= 15 ? (lane / PPR) * step + r * step : min(r + lane / PPR, rows[i]) * step) + (lane % PPR) * 16;
                    vf[u] = *reinterpret_cast<const u32x4*>(vat[i] + off);
                }
            } else {                                       // columns l16 DH / 16 .. of keys 4 g + e
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t off = (rows[i] >= 15 ? 4 * g * step + e * step : min(4 * g + e, rows[i]) * step) + l16 * (DH / 4);
#pragma unroll
                        for (int c = 0; c < DH / 64; ++c) vf[(i * 4 + e) * (DH / 64) + c] = *reinterpret_cast<const u32x4*>(vat[i] + off + 16 * c);
                    }
            }
        };

        float m_run = -INFINITY, l_run = 0.f;              // of query l16; the sum over this lane's keys only
        f32x4 acc[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        bool have = where(k0);
        if (have) { fetch_k(); fetch_v(); }
        for (int u = k0; u < k1; ++u) {
            if ((u & ((1 << lg_span) - 1)) == 0 && u > k0 && u + (1 << lg_span) < k1) {      // (the window before this one is done with)
                const Window next = window((u >> lg_span) + 1);
                if ((u >> lg_span) & 1) even = next; else odd = next;
            }
            if (!have) {
                if (u + 1 < k1 && (have = where(u + 1))) { fetch_k(); fetch_v(); }
                continue;
            }
            f32x4 s[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < KF; ++c) {
                    if constexpr (sizeof(In) == 2) s[i] = mfma16(kf[i][c], qf[c], s[i]);
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[i][c][e]), __uint_as_float(qf[c][e]), s[i], 0, 0, 0);
                }
            }
            const int p0 = pos[0], p1 = pos[1];
            char* vbuf = lds + wave * R::V_LDS;
            if constexpr (sizeof(In) == 2) {
                constexpr int PPR = DH / 8;
#pragma unroll
                for (int w = 0; w < VF; ++w) {
                    const int i = w * 64 + lane;
                    *reinterpret_cast<u32x4*>(vbuf + (i / PPR) * R::PITCH + (i % PPR) * 16) = vf[w];
                }
            }
            have = u + 1 < k1 && where(u + 1);
            if (have) {
                fetch_k();
                if constexpr (sizeof(In) == 2) fetch_v();
            }
            // weights in base 2 against a reference that moves only when it is passed by more than 10 (see ada_attn.hpp's kernels)
            float mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[i][e] = (i ? p1 : p0) + 4 * g + e < limit ? s[i][e] * a.sc2 : -INFINITY;
                    mx = fmaxf(mx, s[i][e]);
                }
            mx = max_over_groups(mx);
            const bool grow = mx > m_run + 10.f;
            if (__builtin_amdgcn_ballot_w64(grow) != 0ull) {
                const float f = grow ? __builtin_amdgcn_exp2f(m_run - mx) : 1.f;
                m_run = grow ? mx : m_run;
                l_run *= f;
#pragma unroll
                for (int i = 0; i < NB; ++i) acc[i] *= f;
            }
            const float m_use = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[i][e] = __builtin_amdgcn_exp2f(s[i][e] - m_use);
                    l_run += s[i][e];
                }
            if constexpr (sizeof(In) == 2) {
                u32x4 hi, lo;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float w0 = s[w >> 1][2 * (w & 1)], w1 = s[w >> 1][2 * (w & 1) + 1];
                    hi[w] = bf16_pair(w0, w1);
                    lo[w] = bf16_pair(w0 - bf16_lo(hi[w]), w1 - bf16_hi(hi[w]));
                }
                // lane (g, l16) reads 4 columns of key 4 g + l16 / 4 and gets column l16 of keys 4 g .. 4 g + 3, as the weights lie
                char* vr = vbuf + (4 * g + l16 / 4) * R::PITCH + (l16 % 4) * 8;
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    typedef __attribute__((address_space(3))) s16x4* At;
                    const u32x2 v0 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(vr + i * 32)));
                    const u32x2 v1 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(vr + 16 * R::PITCH + i * 32)));
                    const u32x4 v = {v0[0], v0[1], v1[0], v1[1]};
                    acc[i] = mfma16(v, hi, acc[i]);
                    acc[i] = mfma16(v, lo, acc[i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int c = 0; c < NB; ++c)
                            acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[(i * 4 + e) * (DH / 64) + c / 4][c % 4]), s[i][e], acc[c], 0, 0, 0);
                if (have) fetch_v();
            }
        }
        // ---- the four waves' sums, brought to the common maximum
        l_run = sum_over_groups(l_run);
        if (g == 0) { mbuf[wave * TILE_ROWS + l16] = m_run; lbuf[wave * TILE_ROWS + l16] = l_run; }
        __syncthreads();                                   // (and nobody reads values from LDS any more)
        float m_all = mbuf[l16];
#pragma unroll
        for (int w = 1; w < 4; ++w) m_all = fmaxf(m_all, mbuf[w * TILE_ROWS + l16]);
        const float f = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_all);
        float* ob = obuf + (wave * TILE_ROWS + l16) * (DH + 4);
        if constexpr (sizeof(In) == 2) {
#pragma unroll
            for (int i = 0; i < NB; ++i) *reinterpret_cast<f32x4*>(ob + 16 * i + 4 * g) = acc[i] * f;
        } else {                                           // row 4 g + e of block i is column (4 g + e) DH / 16 + i
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < NB; i += 4)
                    *reinterpret_cast<f32x4*>(ob + (4 * g + e) * NB + i) = f32x4{acc[i][e], acc[i + 1][e], acc[i + 2][e], acc[i + 3][e]} * f;
        }
        __syncthreads();
        {
            const int r = tid >> 4, c0 = (tid & 15) * (DH / 16);
            float o[DH / 16], m = -INFINITY, l = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) m = fmaxf(m, mbuf[w * TILE_ROWS + r]);
#pragma unroll
            for (int c = 0; c < DH / 16; ++c) o[c] = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float mw = mbuf[w * TILE_ROWS + r];
                l += mw == -INFINITY ? 0.f : lbuf[w * TILE_ROWS + r] * __builtin_amdgcn_exp2f(mw - m);
#pragma unroll
                for (int c = 0; c < DH / 16; ++c) o[c] += obuf[(w * TILE_ROWS + r) * (DH + 4) + c0 + c];
            }
            int orow, ohead, otoken;
            const bool stored = tile_row<MODE, TILE_ROWS>(a, t, r, orow, ohead, otoken);
            In* to = reinterpret_cast<In*>(a.out) + orow * a.ld_out + (long long)(t.kvh * p.G + ohead) * DH + c0;
            if (part.whole(t)) {
                if (stored) store_out<In, DH>(to, o, l > 0.f ? 1.f / l : 0.f);
            } else {
                const long long slot = part.slot(piece);
                float* po = a.part_o + (slot * TILE_ROWS + r) * DH + c0;
#pragma unroll
                for (int c = 0; c < DH / 16; c += 2) put(po + c, o[c], o[c + 1]);
                if ((tid & 15) == 0) put(a.part_ml + (slot * TILE_ROWS + r) * 2, m, l);
                int first, last;
                if (comes_last(a, piece, t, first, last, flag) && stored) {
                    m = -INFINITY;
                    l = 0.f;
#pragma unroll
                    for (int c = 0; c < DH / 16; ++c) o[c] = 0.f;
#pragma unroll 4
                    for (int w = first; w <= last; ++w) {
                        const long long s2 = (2LL * w + (w == first ? 1 : 0)) * TILE_ROWS + r;
                        const f32x2 ml = get(a.part_ml + s2 * 2);
                        f32x2 v[DH / 32];
#pragma unroll
                        for (int c = 0; c < DH / 32; ++c) v[c] = get(a.part_o + s2 * DH + c0 + 2 * c);
                        const float mn = fmaxf(m, ml[0]), f0 = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn), f1 = ml[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[0] - mn);
                        m = mn;
                        l = l * f0 + ml[1] * f1;
#pragma unroll
                        for (int c = 0; c < DH / 16; ++c) o[c] = o[c] * f0 + v[c / 2][c % 2] * f1;
                    }
                    store_out<In, DH>(to, o, l > 0.f ? 1.f / l : 0.f);
                }
            }
        }
        __syncthreads();                                   // the next tile's values take the same place
    }
}

#include "ada_paged_tile.hpp"

// ------------------------------------------------------------------------------------------------ host
struct AttendWs { size_t tiles, prefix, tile, part_o, part_ml, bytes; int room; };

// Chunks in bf16 go to ada_paged_tile.hpp's kernel where they have more than 16 rows a sequence and 16-row tiles enough for half of the CUs (heads of 256,
// whose 16-row tiles take twice the registers: a sixth): with fewer, no tile of 128 rows has work for a CU that its parts' join does not cost
// again.  us a call with 16-row and 128-row tiles, 32 x 128 over 8 at 8000 keys: 64 16-row tiles in one sequence 36 and 48, 128 57 and 50; 256 in eight
// 96 and 71; 1536 in 24 413 and 173; at 1000 keys 128 in one 18 and 27, 768 in 24 52 and 36.  16 x 256 over 8 at 8000 keys: 32 in one 56 and 77, 64 104 and 80.
inline bool may_take_tiles(const PagedArgs& p, int dtype) { return dtype == ADA_BF16 && (long long)p.longest * p.G > TILE_ROWS; }   // (what grows with the chunk)
inline bool takes_tiles(const PagedArgs& p, int d_h, int dtype) {
    const long long rows = (long long)p.rows * p.G;
    return may_take_tiles(p, dtype) && rows > (long long)TILE_ROWS * p.B &&
           rows / TILE_ROWS * p.H_kv > ada_hook_cus() / (d_h > 128 ? 6 : 2);
}

// Two workgroups per CU: 64 single tokens at 100 to 8191 keys, 32 x 128 over 8, us a call with 1, 2, 3, 4 of them: 101, 102, 118, 111 (registers hold two at
// once); 1024 tokens with 16 listed pages of 64: 597, 422, 477, 422.
inline int rows_pieces() { return 2 * ada_hook_cus() < ADA_PAGED_ZERO_BYTES / 4 ? 2 * ada_hook_cus() : ADA_PAGED_ZERO_BYTES / 4; }
inline int tile_pieces(int d_h) { const int n = (d_h > 128 ? 1 : 2) * ada_hook_cus(); return n < rows_pieces() ? n : rows_pieces(); }

inline AttendWs attend_ws(const PagedArgs& p, int d_h, int dtype) {
    const size_t tiles = (size_t)((long long)p.rows * p.G / TILE_ROWS + p.B);
    const size_t rows = (size_t)rows_pieces() * TILE_ROWS, tile_rows = may_take_tiles(p, dtype) ? (size_t)tile_pieces(d_h) * 128 : 0;
    const size_t parts = 2 * (rows > tile_rows ? rows : tile_rows);           // rows of cut tiles (listed pages always take 16-row ones)
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    AttendWs w;
    w.room = (int)tiles;
    w.tiles = ADA_PAGED_ZERO_BYTES;                        // behind what is zero between calls
    w.prefix = w.tiles + 256;
    w.tile = w.prefix + up((tiles + 1) * 8);
    w.part_ml = w.tile + up(tiles * 8);
    w.part_o = w.part_ml + up(parts * 2 * 4);
    w.bytes = w.part_o + up(parts * (size_t)d_h * 4);
    return w;
}

// A kernel that needs more LDS than a launch gets unasked.
template <typename Kernel>
hipError_t launch_pieces(Kernel kernel, std::once_flag& once, hipError_t& attr_err, int pieces, int threads, int lds, const AttendArgs& a, hipStream_t st) {
    std::call_once(once, [&] { attr_err = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds); });
    if (attr_err != hipSuccess) return attr_err;
    ProfHook ps(ADA_K_ATTN, st);
    hipLaunchKernelGGL(kernel, dim3(pieces), dim3(threads), lds, st, a);
    return hipGetLastError();
}

template <typename In, int DH, int MODE>
hipError_t launch_rows(const AttendArgs& a, hipStream_t st) {
    static std::once_flag once;
    static hipError_t attr_err = hipSuccess;
    return launch_pieces(&k_paged_rows<In, DH, MODE>, once, attr_err, rows_pieces(), 256, rows_lds<In, DH>(), a, st);
}

template <int DH>
hipError_t launch_tiles(const AttendArgs& a, hipStream_t st) {
    static std::once_flag once;
    static hipError_t attr_err = hipSuccess;
    return launch_pieces(&k_paged_tile<DH>, once, attr_err, tile_pieces(DH), 64 * TileGeom<DH>::WAVES, TileGeom<DH>::LDS, a, st);
}

template <typename In, int DH>
hipError_t launch_attend(AttendArgs a, void* ws, hipStream_t st) {
    constexpr int dtype = sizeof(In) == 2 ? ADA_BF16 : ADA_F32;
    const AttendWs w = attend_ws(a.p, DH, dtype);
    char* at = reinterpret_cast<char*>(ws);
    int* tiles = reinterpret_cast<int*>(at + w.tiles);
    long long* prefix = reinterpret_cast<long long*>(at + w.prefix);
    int2* tile = reinterpret_cast<int2*>(at + w.tile);
    a.arrived = reinterpret_cast<int*>(at);
    a.tiles = tiles; a.prefix = prefix; a.tile = tile;
    a.part_o = reinterpret_cast<float*>(at + w.part_o);
    a.part_ml = reinterpret_cast<float*>(at + w.part_ml);
    if (a.list) return launch_rows<In, DH, LISTED>(a, st);
    const bool chunks = takes_tiles(a.p, DH, dtype);
    if (!chunks && (long long)a.p.longest * a.p.G <= TILE_ROWS) return launch_rows<In, DH, TOKENS>(a, st);
    {
        ProfHook ps(ADA_K_ATTN, st);
        const int tile_rows = chunks ? TileGeom<DH>::ROWS : TILE_ROWS, unit = chunks ? TileGeom<DH>::KEYS : UNIT;
        if (a.p.B <= 64 && (long long)a.p.rows * a.p.G / tile_rows + a.p.B <= 1024)
            hipLaunchKernelGGL(k_paged_plan_few, dim3(1), dim3(64), 0, st, a.p, tile_rows, unit, w.room, prefix, tile, tiles);
        else
            hipLaunchKernelGGL(k_paged_plan, dim3(1), dim3(1024), 0, st, a.p, tile_rows, unit, w.room, prefix, tile, tiles);
    }
    if (hipError_t e = hipGetLastError()) return e;
    if constexpr (dtype == ADA_BF16)
        if (chunks) return launch_tiles<DH>(a, st);
    return launch_rows<In, DH, CHUNKS>(a, st);
}
