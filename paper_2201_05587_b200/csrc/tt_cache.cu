// A paged cache of keys and values in e4m3, a scale for each page and head: new tokens into it, and attention over it.
#include <cuda_runtime.h>
#include <climits>
#include <cstring>
#include <type_traits>
#include "tt_cache.cuh"

namespace tt {

// ---- append ---------------------------------------------------------------------------------------------------------------
//
// The new tokens of one page and head, of the keys or of the values, are a CTA's, or a warp's where there are few of them: read once into registers
// (what is more than kHeld pieces a thread is read again, from the caches), their maximum, their conversion; where the page holds
// tokens already and the scale has to rise, those are brought to it.
//   Bytes are the bound, but a page is only some thousands of values, so what each thread does once counts as much: addresses are stepped, not
// divided for.  (Four prompts of up to 2048 tokens, 8 heads of 128, pages of 64: 8.8 us, 3.3 TB/s; with divisions, 64-bit ones for the sequences, and 256
// threads 13.3.  64 single tokens 3.4 us.)
constexpr int kAppendThreads = 128;         // of a CTA that has a page
template <int TYPE, bool WIDE, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : kAppendThreads, WARP ? 3 : 7) tt_cache_append_kernel(const tt_cache_append_args a) {
    __shared__ float warp_most[kAppendThreads / 32];
    typedef typename Element<TYPE>::type T;
    pdl_allow_next();
    pdl_wait_prev();
    const tt_cache& c = a.cache;
    const int which = WARP ? (int)blockIdx.y * 8 + ((int)threadIdx.x >> 5) : (int)blockIdx.y, head = which >> 1, w = which & 1;
    const int me = WARP ? (int)threadIdx.x & 31 : (int)threadIdx.x;
    constexpr int kThreads = WARP ? 32 : kAppendThreads;
    if (WARP && head >= c.heads) return;
    const int shift = 31 - __clz(c.block);                  // (a power of two)
    long long first_unit;
    int b;
    const bool found = sequence_of(a.starts, c.batch, [&](int start, int i) { return (start >> shift) + 2 * i; }, blockIdx.x, b, first_unit);
    const int start = a.starts[b], count = a.starts[b + 1] - start, length = a.lengths[b];
    if (found && count == 0) return;
    if (!found || count < 0 || start < 0 || start + (long long)count > a.tokens || length < count || length > (long long)c.max_pages * c.block) {
        if (me == 0) report_invalid(a.status);
        return;
    }
    const int first = length - count;                       // position of the first new token
    const long long index = (first >> shift) + ((long long)blockIdx.x - first_unit);
    if (index << shift >= length) return;
    const int lo = max(first, (int)index << shift), hi = (int)min((long long)length, (index + 1) << shift);
    const int held = lo - ((int)index << shift);            // tokens that the page holds already
    constexpr int kPiece = WIDE ? 8 : 1, kHeld = WIDE ? (WARP || TYPE == TT_TYPE_F32 ? 4 : 8) : 16;      // values a thread takes at a time, and how often it keeps them
    const int pieces = c.d / kPiece;
    // A thread's pieces are kThreads apart: value i of token t, then di values and dt tokens further on.
    const int t0 = me / pieces, i0 = (me - t0 * pieces) * kPiece, dt = kThreads / pieces, di = (kThreads - dt * pieces) * kPiece;
    const int n = ((hi - lo) * pieces - me + kThreads - 1) / kThreads;      // of them
    const T* const x = static_cast<const T*>(a.x[w]) + ((long long)(start + (lo - first)) * a.x_token[w] + (long long)head * a.x_head[w]);
    struct Walk {
        int i; long long at;                                // the value of its token, and its place
        __device__ __forceinline__ void next(int d, int di, long long step, long long wrap) {
            i += di; at += step;
            if (i >= d) { i -= d; at += wrap; }
        }
    };
    const long long x_token = a.x_token[w], x_step = dt * x_token + di, x_wrap = x_token - c.d;
    struct One { float v; };
    typedef typename std::conditional<WIDE, Eights<TYPE, 1>, One>::type Piece;
    const auto load = [&](const Walk& p, Piece& u) {
        if constexpr (WIDE) u.load(x + p.at, 0, 0, 8, true);
        else u.v = Element<TYPE>::up(x[p.at]);
    };
    // the largest finite magnitude of u and m; nan: whether there is one that is not
    const auto more = [&](const Piece& u, float m, bool& odd) {
        if constexpr (WIDE) {
            const float n = u.most();
            if (n < INFINITY) return fmaxf(m, n);
            odd = true;
            return fmaxf(m, u.finite_most());
        } else {
            odd = odd || !(fabsf(u.v) < INFINITY);
            return finite_max(m, u.v);
        }
    };
    Piece v[kHeld];
    Walk p{i0, t0 * x_token + i0};
#pragma unroll
    for (int k = 0; k < kHeld; ++k, p.next(c.d, di, x_step, x_wrap)) if (k < n) load(p, v[k]);      // (on their way while the page is looked up)
    const int page = c.table[b * c.table_row + index];
    if (page < 0 || page >= c.pages) {
        if (me == 0) report_invalid(a.status);
        return;
    }
    float* scale = c.scale[w] + page * c.s_page[w] + head * c.s_head[w];
    const float old = held > 0 ? *scale : 0.f;
    float most = 0.f;
    bool odd = false;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) if (k < n) most = more(v[k], most, odd);
    if (n > kHeld) {
        Walk more_of = p;
        for (int k = kHeld; k < n; ++k, more_of.next(c.d, di, x_step, x_wrap)) {
            Piece u;
            load(more_of, u);
            most = more(u, most, odd);
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
    if constexpr (WARP) __syncwarp();                       // (every thread has read the old scale)
    else {
        if ((me & 31) == 0) warp_most[me >> 5] = most;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kAppendThreads / 32; ++k) most = fmaxf(most, warp_most[k]);
    }
    float s = power_scale(most);
    if (held > 0 && old >= s) s = old;
    if (me == 0 && (held == 0 || s != old)) *scale = s;
    uint8_t* const data = static_cast<uint8_t*>(c.data[w]) + page * c.page[w] + head * c.head[w];
    if (held > 0 && s != old) {
        // (a ratio of powers of two as the calls here leave them; a scale of another origin is taken as it is)
        const float ratio = __fdiv_rn(old, s);
        const int words = c.d / 4;
        for (int e = me; e < held * words; e += kThreads) {
            const int row = e / words;
            uint32_t* q = reinterpret_cast<uint32_t*>(data + row * c.token[w]) + (e - row * words);
            const uint32_t n = *q;
            *q = to_e4m3x4(float_of_e4m3(n) * ratio, float_of_e4m3(n >> 8) * ratio, float_of_e4m3(n >> 16) * ratio, float_of_e4m3(n >> 24) * ratio);
        }
    }
    const bool power = (__float_as_int(s) & 0x7fffff) == 0 && s >= 1.17549435e-38f && s <= 1.329227996e36f;      // 2^-126 .. 2^120
    const float inv = power ? power_inverse(s) : 0.f;
    uint8_t* const to = data + held * c.token[w];
    const auto put = [&](const Walk& p, const Piece& u) {
        if constexpr (WIDE) {
            uint2 out;
            if (power) out = odd ? u.template bytes<false>(0, inv) : u.template bytes<true>(0, inv);
            else {
                const float2 p0 = u.pair(0), p1 = u.pair(1), p2 = u.pair(2), p3 = u.pair(3);
                out.x = to_e4m3x4(__fdiv_rn(p0.x, s), __fdiv_rn(p0.y, s), __fdiv_rn(p1.x, s), __fdiv_rn(p1.y, s));
                out.y = to_e4m3x4(__fdiv_rn(p2.x, s), __fdiv_rn(p2.y, s), __fdiv_rn(p3.x, s), __fdiv_rn(p3.y, s));
            }
            *reinterpret_cast<uint2*>(to + p.at) = out;
        } else to[p.at] = (uint8_t)to_e4m3x4(power ? u.v * inv : __fdiv_rn(u.v, s), 0.f, 0.f, 0.f);
    };
    Walk q{i0, t0 * c.token[w] + i0};
    const long long q_step = dt * c.token[w] + di, q_wrap = c.token[w] - c.d;
#pragma unroll
    for (int k = 0; k < kHeld; ++k, q.next(c.d, di, q_step, q_wrap)) if (k < n) put(q, v[k]);
    for (int k = kHeld; k < n; ++k, q.next(c.d, di, q_step, q_wrap), p.next(c.d, di, x_step, x_wrap)) {
        Piece u;
        load(p, u);
        put(q, u);
    }
}

// ---- attention ------------------------------------------------------------------------------------------------------------
//
// One pass over the visible keys and values with a running maximum and sum of each row (a query of one head).  The heads that share a key
// head are rows of one tile, so a key is read once for all of them.
//
// Tiles of 8 to 32 rows: the cache's bytes are the bound.  A warp takes runs of 64 tokens, 16 or 32 at a time, as the rows of m16n8k16
// products: scores^T = K Q^T and o^T = V^T P^T, so eight query rows cost half of what they would as rows.  The order of a reduction is free as
// long as both factors have it, so lane (g, c) takes 16 bytes in a row of the keys g and g + 8, and of four values 16 bytes in a row of
// columns; which keys, and which columns, is chosen so that the swizzled lines of a box are read without bank conflicts.  Boxes arrive by TMA in
// a ring of the warp's own, so the loop has no barrier but theirs.  (Copied by the lanes, 16 bytes each, they were bound by what the load
// unit takes, 4 TB/s.)
//   e4m3 -> 16-bit floating point is exact, and so is a row of queries but for what is below 2^-29 of its largest: brought to a maximum of 2^14..2^15
// by a power of two, which the scores' factor takes back.  What a probability is rounded to 11 bits as has the scale of the page's values in it, and the running maximum is one of
// scores with those scales: it is of each row's own tokens, so that no page that only another row sees takes bits from it. 2^-29 of the
// largest still has all of them; sums are in 32 bits.
//   The keys of a sequence are split over CTAs, of which the last to finish adds up what all have left in the workspace, in their order.
//   (64 sequences of up to 8192 tokens, 32 heads over 8 of 128: 119 us, 5.1 TB/s, 0.79 of a copy's rate; one of 131072 tokens: 54 us, 0.76.)

constexpr int kRun = 64;                    // tokens that a warp takes in a row
constexpr int kAttendWarps = 4;
constexpr unsigned long long kAttendWait = 1000000000ull;   // nanoseconds that a wait takes at most
constexpr int kFewRows = 32;                // rows of a tile at most
constexpr int kMostSplits = 256;            // of a sequence: the last CTA has the maxima and sums of all of them in shared memory

__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of 16-bit values, a row's pair in lane (row, pair), transposed.
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
    uint32_t t;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(t) : "r"(v));
    return t;
}
constexpr int widest(int bytes) { return bytes % 16 == 0 ? 16 : bytes % 8 == 0 ? 8 : 4; }
// Over the eight lanes that have the same pair of rows.
__device__ __forceinline__ float octet_max(float v) {
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
__device__ __forceinline__ float octet_sum(float v) {
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
// Groups of 16 tokens that a step takes: two, where the registers hold them, so that the latencies of one group's products, maxima and
// exponentials are behind the other's.
constexpr int attend_groups(int d, int nt) { return nt * d <= 128 ? 2 : 1; }
// CTAs that their registers leave room for on an SM.
constexpr int attend_ctas(int d, int nt) { return nt <= 2 && nt * d <= 256 ? 3 : 2; }

template <int D, int NT>
struct AttendShape {
    static constexpr int kKey = widest(D / 4), kKeyPieces = D / 4 / kKey;           // bytes of a key that a lane fetches at a time, and how often
    static constexpr int kVal = widest(D / 8), kValPieces = D / 8 / kVal;
    static constexpr int kRows = 8 * NT;
    static constexpr int kGroups = attend_groups(D, NT), kTokens = kStep * kGroups; // ... and the tokens of a step
    static constexpr bool kQueryRegs = NT == 1 || NT * D <= 128;                     // the queries' fragments stay in registers
    // A step's keys, and its values: boxes of kTokens lines of kLine bytes, swizzled as the tensor map has it.
    static constexpr int kLine = 8 * kVal, kBoxes = D / kLine;
    static constexpr uint32_t kBox = kTokens * kLine, kStage = 2u * kTokens * D;
    static constexpr uint32_t kQuery = kQueryRegs ? 0u : NT * (D / 16) * 256u;
    static constexpr int kCtas = attend_ctas(D, NT);
    static constexpr int kFits = (int)((227u * 1024u / kCtas - 3u * 1024u - kQuery) / (kAttendWarps * kStage));
    static constexpr int kStages = kFits > 6 ? 6 : kFits;                            // steps in shared memory: one is worked on, the others are under way
    static constexpr uint32_t kRing = kAttendWarps * kStages * kStage;
    static constexpr uint32_t kJoin = kAttendWarps * kRows * (D + 4) * 4u;           // the warps' results (over the ring)
    static constexpr uint32_t kLists = kMostSplits * kRows * 8u;                     // ... the splits' maxima and sums
    static constexpr uint32_t kMore = kRing > kJoin ? (kRing > kLists ? kRing : kLists) : (kJoin > kLists ? kJoin : kLists);
    static constexpr uint32_t kBytes = 1024u + kQuery + kMore;                       // (the ring on 1024 bytes)
    // The key of a group that row g of the products is (and g + 8), and the place in a line of what lane g takes of a value.
    static __device__ __forceinline__ int key_of(int g) { return kLine == 128 ? (g & 1) * 4 + (g >> 1) : kLine == 64 ? g ^ ((g >> 1) & 1) : g; }
    static __device__ __forceinline__ int column_of(int g) { return (kLine == 128 ? (g & 1) * 4 + (g >> 1) : g) * kVal; }
    static __device__ __forceinline__ uint32_t place(int row, int byte) {            // of a byte of a line in its box
        const int swz = kLine == 128 ? row & 7 : kLine == 64 ? (row >> 1) & 3 : (row >> 2) & 1;
        return (uint32_t)(row * kLine + (((byte >> 4) ^ swz) << 4) + (byte & 15));
    }
    static_assert(kStages >= 2, "copies run ahead");
};

// The tokens of a split.  Only the device knows the lengths: the split that deals all sequences' tokens to the CTAs that the SMs hold at once, less a
// fifth, as every sequence has a last split that is not full.  (8 sequences of up to 16384 tokens: 34 us so; by the longest that there may be 42.)  No
// less than what the grid has room for, nor than what makes the join, which reads 14 bytes a cycle, as long as a split, whose warps take some
// 8 + 6 NT cycles a token.  (One sequence of 14353 tokens, 8 rows of 128: 19 splits 16 us, 57 of them 19.)
struct Lane { int start, next, length; };                    // of sequence `lane`
__device__ __forceinline__ Lane lane_of(const Attend& g) {
    const int b = threadIdx.x & 31;
    if (g.splits == 1 || b >= g.a.cache.batch) return Lane{0, 0, 0};
    return Lane{g.a.starts[b], g.a.starts[b + 1], g.a.lengths[b]};
}
// `tokens` that the tile sees, `bytes` of a split's part
template <int ROWS>
__device__ __forceinline__ int split_tokens(const Attend& g, const Lane& mine, float tokens, float bytes) {
    constexpr int kGrain = kAttendWarps * kRun;
    const tt_cache& c = g.a.cache;
    if (g.splits == 1 || c.batch > 1024) return g.chunk;       // (so many have no need of splits)
    unsigned runs = 0u;                                      // of all sequences' tiles
    const auto add = [&](int start, int next, int length) {
        const long long rows = (long long)(next - start) * g.group;
        if (rows >= g.least && rows <= g.most) runs += (unsigned)min((long long)((unsigned)min(max(length, 0), g.span) + kRun - 1) / kRun * ((unsigned)(rows + ROWS - 1) / ROWS), 1ll << 20);
    };
    add(mine.start, mine.next, mine.length);
    for (int b = (threadIdx.x & 31) + 32; b < c.batch; b += 32) add(g.a.starts[b], g.a.starts[b + 1], g.a.lengths[b]);
    // (in 32-bit floating point: whatever it is rounded to, all CTAs have the same)
    const float all = (float)__reduce_add_sync(0xffffffffu, min(runs, 1u << 26));
    const float join = sqrtf(tokens * bytes * (1.f / (14.f * (8.f + 0.75f * ROWS))));
    const float share = fminf(fmaxf(join, all * ((float)(c.heads * kRun) / (float)g.share)), 1073741824.f);
    return max(g.chunk, ((int)share + kGrain) / kGrain * kGrain);
}

template <int D, int NT>
__global__ void __launch_bounds__(kAttendWarps * 32, (AttendShape<D, NT>::kCtas)) tt_attend_few_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ Attend g) {
    typedef AttendShape<D, NT> S;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full_bar[kAttendWarps][S::kStages];
    __shared__ int last_one, abort_flag;
    __shared__ long long y_at[S::kRows];
    __shared__ int2 seen[S::kRows];
    volatile int* abortp = &abort_flag;
    if (threadIdx.x < kAttendWarps * S::kStages) mbar_init(smem_u32(&full_bar[0][0] + threadIdx.x), 1u);
    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_v) : "memory");
        abort_flag = 0;
    }
    fence_mbar_init();
    fence_proxy_async_shared();
    __syncthreads();
    pdl_allow_next();
    pdl_wait_prev();
    const tt_cache& c = g.a.cache;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gq = lane >> 2, cq = lane & 3, head = blockIdx.y;
    const Lane mine = lane_of(g);                            // (under way while the tile is looked up)
    TileView view;
    if (!view_tile(g, S::kRows, blockIdx.x, view)) return;
    const int b = view.b, start = view.start, rows = view.rows, t0 = view.t0, h0 = view.h0, before = view.before, lo = view.lo, hi = view.hi;
    const int base = lo / kRun * kRun, chunk = split_tokens<S::kRows>(g, mine, (float)(hi - lo), 4.f * rows * D);
    const int active = hi > lo ? (int)((unsigned)(hi - base + chunk - 1) / (unsigned)chunk) : 1;
    if ((int)blockIdx.z >= active) return;
    const int from = base + (int)blockIdx.z * chunk, to = hi - from > chunk ? from + chunk : hi;

    const uint32_t base_s = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base_s - smem_u32(smem_raw));
    const uint32_t ring = base_s + (uint32_t)warp * S::kStages * S::kStage, query = base_s + S::kMore;
    // ---- the copies of a step: groups of 16 tokens, each of one page ----
    const int groups = [&] {                                 // of this warp
        const int runs = to > from ? (to - from + kRun - 1) / kRun : 0;
        if (warp >= runs) return 0;
        const int mine = (runs - warp + kAttendWarps - 1) / kAttendWarps;
        const int last = from + ((mine - 1) * kAttendWarps + warp) * kRun;
        return (mine - 1) * (kRun / kStep) + (min(kRun, to - last) + kStep - 1) / kStep;
    }();
    const int steps = (groups + S::kGroups - 1) / S::kGroups;
    const auto token_of = [&](int group) { return from + ((group >> 2) * kAttendWarps + warp) * kRun + (group & 3) * kStep; };
    // Lane l has the page and the scales of group 32 i + l, and of the set of 32 behind it.  A split's first groups may be of pages in front of what any
    // row sees, which the sequence need not have any more: zeros, as behind the last group.
    const int* table = c.table + b * c.table_row;
    const int shift = 31 - __clz(c.block);
    struct Set { int page; float ks, lg; };                  // lg: of the values' scale, a power of two (0 is 2^-126)
    const auto look_up = [&](int set) {
        const int group = 32 * set + lane;
        Set x{-1, 0.f, -126.f};
        if (group < groups && (token_of(group) | (c.block - 1)) >= lo) {
            x.page = table[token_of(group) >> shift];
            if ((unsigned)x.page >= (unsigned)c.pages) {
                report_invalid(g.a.status);
                x.page = -1;                                  // (a box outside of the tensor is zeros)
            } else {
                x.ks = c.scale[0][x.page * c.s_page[0] + head * c.s_head[0]];
                const float vs = c.scale[1][x.page * c.s_page[1] + head * c.s_head[1]];
                if (!(vs <= 1.17549435e-38f)) x.lg = vs < INFINITY ? log2f(vs) : __int_as_float(0x7fffffff);
            }
        }
        return x;
    };
    Set now = look_up(0), then = look_up(1);
    int set = 0;                                             // of the step that is worked on
    const bool whole_boxes = c.block >= S::kTokens;          // a step's tokens are of one page
    const auto fetch = [&](int step, uint32_t slot, int stage) {
        if (step >= steps) return;
        int pages[S::kGroups];
#pragma unroll
        for (int i = 0; i < S::kGroups; ++i) {
            const int group = step * S::kGroups + i;
            pages[i] = __shfl_sync(0xffffffffu, (group >> 5) == set ? now.page : then.page, group & 31);
        }
        if (lane == 0) {
            const uint32_t bar = smem_u32(&full_bar[warp][stage]);
            mbar_expect_tx(bar, S::kStage);
            const int t = token_of(step * S::kGroups) & (c.block - 1);
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
                for (int x = 0; x < S::kBoxes; ++x) {
                    const uint32_t dst = slot + (uint32_t)(w * S::kBoxes + x) * S::kBox;
                    const CUtensorMap* map = w ? &tmap_v : &tmap_k;
                    if (S::kGroups == 1 || whole_boxes) tma_load_4d(dst, map, bar, x * S::kLine, t, head, pages[0]);
                    else {
#pragma unroll
                        for (int i = 0; i < S::kGroups; ++i)
                            tma_load_4d(dst + (uint32_t)(i * kStep * S::kLine), map, bar, x * S::kLine, token_of(step * S::kGroups + i) & (c.block - 1), head, pages[i]);
                    }
                }
        }
    };
#pragma unroll
    for (int i = 0; i < S::kStages - 1; ++i) fetch(i, ring + (uint32_t)i * S::kStage, i);

    // ---- of each row: where its output is, and the tokens that it sees ----
    const auto q_row = [&](int r) { const int t = (h0 + r) / g.group; return make_int2(start + t0 + t, head * g.group + (h0 + r - t * g.group)); };
    if ((int)threadIdx.x < S::kRows) {
        const int2 at = q_row((int)threadIdx.x);
        const int pos = before + (at.x - start);
        y_at[threadIdx.x] = at.x * g.a.y_token + at.y * g.a.y_head;
        seen[threadIdx.x] = make_int2(g.a.window > 0 ? pos - g.a.window + 1 : INT_MIN, g.a.causal ? min(to, pos + 1) : to);
    }
    __syncthreads();

    // ---- queries: lane (g, c) has of rows g, g + 8, ... what it has of the keys ----
    uint32_t q[S::kQueryRegs ? NT : 1][D / 16][2];
    float factor[NT][2];                                     // of the rows 2c, 2c + 1: what turns a product into a score in powers of two
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = 8 * n + gq;
        float f = 0.f;
        if (S::kQueryRegs || warp == n % kAttendWarps) {
            float v[D / 16][4], most = 0.f;
            if (r < rows) {
                const int2 at = q_row(r);
                const long long first = at.x * g.a.q_token + at.y * g.a.q_head + cq * S::kKey;
                uint2 raw[D / 16];
                const auto load = [&](auto wide) {
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) raw[i] = raw_four(g.a.q, first + i / (S::kKey / 4) * 4 * S::kKey + i % (S::kKey / 4) * 4, decltype(wide)::value);
                };
                // (a branch for all loads: one for each makes them wait for each other)
                if (g.q_wide) load(std::integral_constant<int, 1>());
                else load(std::integral_constant<int, 0>());
#pragma unroll
                for (int i = 0; i < D / 16; ++i) four_of(raw[i], g.a.type, v[i]);
            } else {
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[i][e] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) most = finite_max(most, v[i][e]);
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            const int ex = most > 0.f ? (__float_as_int(most) >> 23) : 127 + 14;      // (a subnormal: 0, as good as 1)
            const float up = __int_as_float((min(254, max(1, 127 + 14 + 127 - ex))) << 23);
            f = g.scale_log2 / up;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const uint32_t x = down2<TT_TYPE_F16>(v[i][0] * up, v[i][1] * up), y = down2<TT_TYPE_F16>(v[i][2] * up, v[i][3] * up);
                if constexpr (S::kQueryRegs) { q[n][i][0] = x; q[n][i][1] = y; }
                else {
                    const uint32_t at = query + (uint32_t)(((n * (D / 16) + i) * 32 + lane) * 8);
                    st_shared_u32(at, x);
                    st_shared_u32(at + 4u, y);
                }
            }
        }
        if constexpr (!S::kQueryRegs) {
            // (the warp that has the rows tells the others, through the place that the join takes later)
            __shared__ float factors[S::kRows];
            if (warp == n % kAttendWarps && cq == 0) factors[8 * n + gq] = f;
            if (n == NT - 1) {
                __syncthreads();
#pragma unroll
                for (int m = 0; m < NT; ++m)
#pragma unroll
                    for (int e = 0; e < 2; ++e) factor[m][e] = factors[8 * m + 2 * cq + e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) factor[n][e] = __shfl_sync(0xffffffffu, f, 4 * (2 * cq + e));
        }
    }

    float o[NT][D / 16][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][j][e] = 0.f;
    float top[NT][2], sum[NT][2], ref = -50.f;               // ref: the largest scale of values so far, as a power of two; the unit of o is 2^(ref - 15)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) { top[n][e] = -INFINITY; sum[n][e] = 0.f; }
    const auto sees = [&](int r, int tok) { const int2 s = seen[r]; return tok >= s.x && tok < s.y; };

    // what a lane reads of a step's boxes
    const int row0 = S::key_of(gq), rows_v[2] = {S::key_of(2 * cq), S::key_of(2 * cq + 1)};
    const uint32_t k_at = S::place(row0, cq * S::kKey), v_at[2] = {S::place(rows_v[0], S::column_of(gq)), S::place(rows_v[1], S::column_of(gq))};
    const auto key_at = [&](int p) {                        // piece p, a line's second 64 bytes or the next box
        return S::kLine == 128 ? (uint32_t)(p >> 1) * S::kBox + (k_at ^ ((uint32_t)(p & 1) << 6)) : (uint32_t)p * S::kBox + k_at;
    };
    int stage = 0, ahead = S::kStages - 1;                   // of this step, of the one that is fetched
    uint32_t phase = 0u;
#pragma unroll 1
    for (int step = 0; step < steps; ++step) {
        if ((step * S::kGroups) >> 5 != set) {
            ++set;
            now = then;
            then = look_up(set + 1);
        }
        __syncwarp();                                        // (every lane has read what lay where the next copies go)
        fetch(step + S::kStages - 1, ring + (uint32_t)ahead * S::kStage, ahead);
        if (++ahead == S::kStages) ahead = 0;
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&full_bar[warp][stage]), phase, abortp, g.a.status, 40u, kAttendWait))) break;
        const uint32_t at = ring + (uint32_t)stage * S::kStage;
        if (++stage == S::kStages) { stage = 0; phase ^= 1u; }
        const int t = token_of(step * S::kGroups);
        const bool whole = t >= view.whole_lo && t + S::kTokens <= view.whole_hi && step * S::kGroups + S::kGroups <= groups;
        float ks[S::kGroups], lg[S::kGroups], new_ref = ref;
#pragma unroll
        for (int i = 0; i < S::kGroups; ++i) {
            const int group = step * S::kGroups + i;         // (a last step may have fewer: zeros)
            ks[i] = __shfl_sync(0xffffffffu, now.ks, group & 31);
            lg[i] = __shfl_sync(0xffffffffu, now.lg, group & 31);
            new_ref = fmaxf(new_ref, lg[i]);
        }
        if (new_ref != ref) {                                // o stays as it is: what it is relative to is lower by as much as its unit is higher
            const float more = exp2_fast(fminf(new_ref - ref, 120.f));      // (not infinite: the first time the sum is 0)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) { top[n][e] -= new_ref - ref; sum[n][e] *= more; }
            ref = new_ref;
        }
        // A page's scale over the largest, which is added to its scores, and what takes it (and the 2^15) out of the sum again.  (2^-80 at least, so that
        // all probabilities of 2^-46 and more are in the sum; NaN stays, but for the sum, whose rows need not see it.)
        float back[S::kGroups];
#pragma unroll
        for (int i = 0; i < S::kGroups; ++i) {
            lg[i] = lg[i] < ref - 80.f ? -80.f : lg[i] - ref;
            back[i] = exp2_fast(fminf(-lg[i], 80.f) - 15.f);
        }
        // scores of 16 tokens x rows: tokens g, g + 8 and rows 2c, 2c + 1 of each eight (in two sums, a chain of products half as long)
        float s[S::kGroups][NT][2][4];
#pragma unroll
        for (int i = 0; i < S::kGroups; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[i][n][0][e] = s[i][n][1][e] = 0.f;
#pragma unroll
        for (int p = 0; p < S::kKeyPieces; ++p) {
            uint32_t k[S::kGroups][2][S::kKey / 4];
#pragma unroll
            for (int i = 0; i < S::kGroups; ++i)
#pragma unroll
                for (int n = 0; n < 2; ++n) read_shared<S::kKey>(at + key_at(p) + (uint32_t)((i * kStep + 8 * n) * S::kLine), k[i][n]);
#pragma unroll
            for (int w = 0; w < S::kKey / 4; ++w) {
                const int j = p * (S::kKey / 4) + w;
#pragma unroll
                for (int i = 0; i < S::kGroups; ++i) {
                    uint32_t a0, a1, a2, a3;
                    f16_pairs_of_e4m3(k[i][0][w], a0, a2);
                    f16_pairs_of_e4m3(k[i][1][w], a1, a3);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        if constexpr (S::kQueryRegs) mma_16x8x16(s[i][n][j & 1], a0, a1, a2, a3, q[n][j][0], q[n][j][1]);
                        else {
                            uint32_t qq[2];
                            read_shared<8>(query + (uint32_t)(((n * (D / 16) + j) * 32 + lane) * 8), qq);
                            mma_16x8x16(s[i][n][j & 1], a0, a1, a2, a3, qq[0], qq[1]);
                        }
                    }
                }
            }
        }
        // the running maximum, in powers of two
        bool moved = false;
        float alpha[NT][2];
        uint32_t pb[S::kGroups][NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float v[S::kGroups][4];
#pragma unroll
            for (int i = 0; i < S::kGroups; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[i][e] = fmaf(s[i][n][0][e] + s[i][n][1][e], factor[n][e & 1] * ks[i], lg[i]);
                    if (!whole) v[i][e] = sees(8 * n + 2 * cq + (e & 1), t + kStep * i + row0 + 8 * (e >> 1)) ? v[i][e] : -INFINITY;
                }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float mx = fmaxf(v[0][e], v[0][e + 2]);
#pragma unroll
                for (int i = 1; i < S::kGroups; ++i) mx = fmaxf(mx, fmaxf(v[i][e], v[i][e + 2]));
                mx = fmaxf(top[n][e], octet_max(mx) - 15.f);      // (P is 2^15 at most)
                const float ref_max = mx == -INFINITY ? 0.f : mx;
                const float keep = exp2_fast(top[n][e] - ref_max);
                moved = moved || mx != top[n][e];
                top[n][e] = mx;
                float add = 0.f;
#pragma unroll
                for (int i = 0; i < S::kGroups; ++i) {
                    v[i][e] = exp2_fast(v[i][e] - ref_max);
                    v[i][e + 2] = exp2_fast(v[i][e + 2] - ref_max);
                    add = fmaf(v[i][e] + v[i][e + 2], back[i], add);
                }
                sum[n][e] = fmaf(sum[n][e], keep, add);
                alpha[n][e] = keep;
            }
#pragma unroll
            for (int i = 0; i < S::kGroups; ++i) {
                pb[i][n][0] = transpose_8x8(down2<TT_TYPE_F16>(v[i][0], v[i][1]));
                pb[i][n][1] = transpose_8x8(down2<TT_TYPE_F16>(v[i][2], v[i][3]));
            }
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < D / 16; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[n][j][e] *= alpha[n][e & 1];
        }
        // values
#pragma unroll
        for (int i = 0; i < S::kGroups; ++i)
#pragma unroll
            for (int p = 0; p < S::kValPieces; ++p) {
                uint32_t v[4][S::kVal / 4];
#pragma unroll
                for (int n = 0; n < 4; ++n) read_shared<S::kVal>(at + (uint32_t)(S::kBoxes + p) * S::kBox + v_at[n & 1] + (uint32_t)((i * kStep + 8 * (n >> 1)) * S::kLine), v[n]);
                if (!whole) {
                    // What no row of the tile sees is not multiplied (it may be anything), and a NaN that only some rows see reaches just those: it is
                    // replaced by 0 in the product, and another product counts for each row how many of a column's it sees.
                    uint32_t nans = 0u;
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const int tok = t + kStep * i + rows_v[n & 1] + 8 * (n >> 1);
                        const bool any = tok >= lo && tok < min(hi, to);
#pragma unroll
                        for (int w = 0; w < S::kVal / 4; ++w) {
                            v[n][w] = any ? v[n][w] : 0u;
                            nans |= nan_bytes(v[n][w]);
                        }
                    }
                    if (__any_sync(0xffffffffu, nans != 0u)) {
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            uint32_t see[2];
#pragma unroll
                            for (int r = 0; r < 2; ++r)
                                see[r] = (sees(8 * n + gq, t + kStep * i + 8 * r + rows_v[0]) ? 0x3c00u : 0u) | (sees(8 * n + gq, t + kStep * i + 8 * r + rows_v[1]) ? 0x3c000000u : 0u);
#pragma unroll
                            for (int j = 0; j < S::kVal; j += 2) {
                                const auto is_nan = [&](int m, int x) { return ((v[m][x >> 2] >> (8 * (x & 3))) & 0x7fu) == 0x7fu; };
                                uint32_t a[4];
#pragma unroll
                                for (int r = 0; r < 4; ++r) a[r] = (is_nan(r & 2, j + (r & 1)) ? 0x3c00u : 0u) | (is_nan((r & 2) + 1, j + (r & 1)) ? 0x3c000000u : 0u);
                                float hit[4] = {0.f, 0.f, 0.f, 0.f};
                                mma_16x8x16(hit, a[0], a[1], a[2], a[3], see[0], see[1]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) if (hit[e] > 0.f) o[n][(p * S::kVal + j) / 2][e] = __int_as_float(0x7fffffff);
                            }
                        }
#pragma unroll
                        for (int n = 0; n < 4; ++n)
#pragma unroll
                            for (int w = 0; w < S::kVal / 4; ++w) v[n][w] &= ~((nan_bytes(v[n][w]) >> 7) * 0xffu);
                    }
                }
#pragma unroll
                for (int j = 0; j < S::kVal; j += 2) {
                    // bytes j, j + 1 of two tokens side by side: the pairs of the reduction, two columns of them
                    const uint32_t sel = (j & 2) ? 0x7362u : 0x5140u;
                    uint32_t a0, a1, a2, a3;
                    f16_pairs_of_e4m3(__byte_perm(v[0][j >> 2], v[1][j >> 2], sel), a0, a1);
                    f16_pairs_of_e4m3(__byte_perm(v[2][j >> 2], v[3][j >> 2], sel), a2, a3);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma_16x8x16(o[n][(p * S::kVal + j) / 2], a0, a1, a2, a3, pb[i][n][0], pb[i][n][1]);
                }
            }
    }
    // a wait that gave up: the copies under way land before the shared memory is used again (bounded)
    if (*abortp && lane == 0) {
        const unsigned long long t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 2000000ull) { }
    }

    // ---- the warps' results together: maximum, sum and o of every row, through shared memory ----
    __syncthreads();                                         // (the ring is idle)
    constexpr int kLine = D + 4;                             // floats of a row: o, then maximum, sum
    float* join = reinterpret_cast<float*>(smem);
    const float to_real = exp2f(ref - 15.f);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float* line = join + (warp * S::kRows + 8 * n + 2 * cq + e) * kLine;
            const float total = octet_sum(sum[n][e]);
#pragma unroll
            for (int p = 0; p < S::kValPieces; ++p)
#pragma unroll
                for (int j = 0; j < S::kVal; j += 2)
                    *reinterpret_cast<float2*>(line + p * S::kLine + S::column_of(gq) + j) = make_float2(o[n][(p * S::kVal + j) / 2][e] * to_real, o[n][(p * S::kVal + j) / 2][e + 2] * to_real);
            if (gq == 0) *reinterpret_cast<float2*>(line + D) = make_float2(top[n][e], total);
        }
    __syncthreads();
    const auto store = [&](int r, int i, const float (&v)[4]) { store_four(g.a.y, y_at[r] + i, g.a.type, g.y_wide, v); };
    const long long tile = (long long)blockIdx.x * c.heads + head;
    constexpr int kPart = S::kRows * (D + 2);
    float* left = g.partial + (tile * g.splits + blockIdx.z) * kPart;
    for (int e = threadIdx.x; e < rows * (D / 4); e += kAttendWarps * 32) {
        const int r = e / (D / 4), i = 4 * (e - r * (D / 4));
        float2 ml[kAttendWarps];
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < kAttendWarps; ++w) {
            ml[w] = *reinterpret_cast<const float2*>(join + (w * S::kRows + r) * kLine + D);
            mx = fmaxf(mx, ml[w].x);
        }
        const float ref_max = mx == -INFINITY ? 0.f : mx;
        float v[4] = {0.f, 0.f, 0.f, 0.f}, l = 0.f;
#pragma unroll
        for (int w = 0; w < kAttendWarps; ++w) {
            const float k = exp2_fast(ml[w].x - ref_max);
            if (ml[w].y != 0.f) {                            // (a warp without tokens has nothing)
                const float4 f = *reinterpret_cast<const float4*>(join + (w * S::kRows + r) * kLine + i);
                v[0] += f.x * k; v[1] += f.y * k; v[2] += f.z * k; v[3] += f.w * k;
                l += ml[w].y * k;
            }
        }
        if (active == 1) {
            const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] *= inv;
            store(r, i, v);
        } else {
            *reinterpret_cast<float4*>(left + r * D + i) = make_float4(v[0], v[1], v[2], v[3]);
            if (i == 0) *reinterpret_cast<float2*>(left + S::kRows * D + 2 * r) = make_float2(mx, l);
        }
    }
    if (active == 1) return;

    // ---- the splits together, by the last CTA of the tile ----
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last_one = atomicAdd(g.counters + tile, 1u) == (unsigned)active - 1u;
    __syncthreads();
    if (!last_one) return;
    __threadfence();
    const float* parts = g.partial + tile * g.splits * kPart;
    float2* lists = reinterpret_cast<float2*>(join);         // [split][row]: maximum and sum, then the split's share
    constexpr int kThreads = kAttendWarps * 32;
    for (int e0 = threadIdx.x; e0 < active * S::kRows; e0 += 8 * kThreads) {
        float2 ml[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int e = e0 + k * kThreads, z = e / S::kRows, r = e % S::kRows;
            ml[k] = make_float2(0.f, 0.f);
            if (z < active && r < rows) ml[k] = __ldcg(reinterpret_cast<const float2*>(parts + (long long)z * kPart + S::kRows * D + 2 * r));
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) if (e0 + k * kThreads < active * S::kRows) lists[e0 + k * kThreads] = ml[k];
    }
    __syncthreads();
    for (int r = warp; r < rows; r += kAttendWarps) {
        float mx = -INFINITY, l = 0.f;
        for (int z = lane; z < active; z += 32) mx = fmaxf(mx, lists[z * S::kRows + r].x);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        const float ref_max = mx == -INFINITY ? 0.f : mx;
        for (int z = lane; z < active; z += 32) {
            const float2 ml = lists[z * S::kRows + r];
            if (ml.y != 0.f) l += ml.y * exp2_fast(ml.x - ref_max);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
        const float inv = l != 0.f ? 1.f / l : 0.f;
        for (int z = lane; z < active; z += 32) {
            const float2 ml = lists[z * S::kRows + r];
            lists[z * S::kRows + r].x = ml.y != 0.f ? exp2_fast(ml.x - ref_max) * inv : 0.f;
        }
    }
    __syncthreads();
    join_splits<kAttendWarps * 32>(rows * (D / 4), active,
        [&](int e, int z) { return reinterpret_cast<const float4*>(parts + (long long)z * kPart + 4 * e); },
        [&](int e, int z) { return lists[z * S::kRows + e / (D / 4)].x; },
        [&](int e, const float (&v)[4]) { store(e / (D / 4), 4 * (e % (D / 4)), v); });
    if (threadIdx.x == 0) g.counters[tile] = 0u;             // ready for the next call
}

// ---- host ----

static tt_status check_cache(const tt_cache& c) {
    if (c.pages < 0 || c.heads < 0 || c.batch < 0 || c.max_pages < 0 || c.d < 0 || c.block < 0) return TT_ERR_INVALID_ARG;
    if (c.block != 16 && c.block != 32 && c.block != 64 && c.block != 128) return TT_ERR_NOT_IMPLEMENTED;
    if (c.d == 0 || c.d % 32 || c.d > 256) return TT_ERR_NOT_IMPLEMENTED;
    if (c.heads > 32767 || (long long)c.max_pages * c.block > 0x7fffff00ll || c.batch > (1 << 24)) return TT_ERR_INVALID_ARG;
    return TT_OK;
}
static tt_status check_cache_memory(const tt_cache& c) {
    if (!c.table || c.table_row < c.max_pages || reinterpret_cast<uintptr_t>(c.table) % 4) return TT_ERR_INVALID_ARG;
    for (int w = 0; w < 2; ++w) {
        if (!c.data[w] || !c.scale[w] || reinterpret_cast<uintptr_t>(c.scale[w]) % 4 || !on16(c.data[w])) return TT_ERR_INVALID_ARG;
        if (c.page[w] < 0 || c.head[w] < 0 || c.token[w] < 0 || c.page[w] % 16 || c.head[w] % 16 || c.token[w] % 16 || c.s_page[w] < 0 || c.s_head[w] < 0) return TT_ERR_INVALID_ARG;
        if (c.page[w] >= 1ll << 40 || c.head[w] >= 1ll << 40 || c.token[w] >= 1ll << 40) return TT_ERR_INVALID_ARG;      // (a tensor map takes no more)
    }
    return TT_OK;
}

// The layout of an attention call: the kernels that it takes and what they split over how many CTAs.
struct AttendPlan {
    Attend few{}, prompt{};
    long long few_units = 0, prompt_units = 0;              // 0: the kernel is not needed
    long long bytes = 0, prompt_at = 0;                     // of the workspace; where the prompts' part begins
};
// The workspace begins with the counters of tt_attend_few_kernel, in a place that is theirs whatever the sizes of a call: they are zeros between calls
// of any sizes.  (A tile has splits where there are no more than 2 * slots of them, see plan_attend.)
constexpr int kCounterBytes = 4096;
static_assert(2 * kSms * 3 * 4 <= kCounterBytes, "a counter for each tile that is split");
// The sums behind them.  d: of a head, as the kernel is built for it
static long long workspace_part(const Attend& g, long long units, int d) {
    return g.splits > 1 ? units * g.a.cache.heads * g.splits * g.rows * (d + 2) * 4 : 0;
}
static tt_status plan_attend(const tt_cache_attention_args& a, AttendPlan& plan) {
    const tt_cache& c = a.cache;
    plan = AttendPlan{};
    const tt_status s = check_cache(c);
    if (s != TT_OK) return s;
    if ((a.type != TT_TYPE_F16 && a.type != TT_TYPE_BF16) || a.tokens < 0 || a.heads_q < 0 || a.window < 0 || a.max_count < 0 || a.max_length < 0 || !(a.scale == a.scale)) return TT_ERR_INVALID_ARG;
    if (c.heads == 0 ? a.heads_q != 0 : a.heads_q % c.heads) return TT_ERR_INVALID_ARG;
    if (a.window > 0 && !a.causal) return TT_ERR_INVALID_ARG;
    if (a.tokens == 0 || a.heads_q == 0 || c.batch == 0) return TT_OK;
    Attend g{};
    g.a = a;
    g.group = a.heads_q / c.heads;
    g.least = 1; g.most = 0x7fffffff;
    g.scale_log2 = a.scale * 1.4426950408889634f;
    g.max_length = c.pages > 0 ? c.max_pages * c.block : 0;
    if (a.max_length > 0 && a.max_length < g.max_length) g.max_length = a.max_length;
    if (a.window >= g.max_length) g.a.window = 0;             // (it hides nothing, and the first token of such a window need not be a 32-bit number)
    const auto wide = [](const void* p, long long token, long long head) {
        const auto at = [&](int n) { return reinterpret_cast<uintptr_t>(p) % (2 * n) == 0 && token % n == 0 && head % n == 0; };
        return at(8) ? 2 : at(4) ? 1 : 0;
    };
    g.q_wide = wide(a.q, a.q_token, a.q_head);
    g.y_wide = wide(a.y, a.y_token, a.y_head);
    const int count = c.batch > 1 && a.max_count > 0 && a.max_count < a.tokens ? a.max_count : a.tokens;
    const long long most_rows = (long long)count * g.group;
    if (most_rows > 0x7fffffff) return TT_ERR_INVALID_ARG;
    const auto span_of = [&](int rows) {
        const long long span = g.max_length, tokens = rows / g.group + 2;
        return g.a.window > 0 && g.a.window + tokens < span ? g.a.window + tokens : span;
    };
    // More than kFewRows rows of a sequence are a prompt's: its tiles take the tensor cores, whose minimum is 128 rows.  (A window must be longer than
    // what a tile's rows and a step span, so that no step is at both ends of it.)
    const bool prompts = most_rows > kFewRows && prompt_built_for(c.d) && (g.a.window == 0 || g.a.window > kPromptRows / g.group + 2 * kPromptTokens + 2);
    const bool few = !prompts || c.batch > 1;
    long long few_bytes = 0, prompt_bytes = 0;
    if (few) {
        Attend& f = plan.few;
        f = g;
        // As many rows as a sequence has, up to what the registers hold: a key that is fetched and converted serves all of them.
        f.rows = most_rows <= 8 ? 8 : most_rows <= 16 || c.d > 128 ? 16 : 32;
        f.by_sequence = prompts || ((a.max_count > 0 || c.batch == 1) && most_rows <= f.rows);      // (no more than a tile each)
        if (prompts) f.most = kFewRows;
        plan.few_units = f.by_sequence ? c.batch : (long long)a.tokens * g.group / f.rows + c.batch;
        const long long tiles = plan.few_units * c.heads, span = span_of(f.rows) + kRun;      // (splits begin at multiples of kRun)
        if (tiles > 0x7fffffffll) return TT_ERR_INVALID_ARG;
        // The CTAs that the SMs hold at once share all tokens (split_tokens); the grid has room for as many splits of a sequence as four rounds of
        // them allow, most of which find nothing to do where there are many sequences.
        const long long slots = (long long)kSms * attend_ctas(c.d, f.rows / 8);
        constexpr int kGrain = kAttendWarps * kRun;
        f.span = (int)(span - kRun);
        f.share = (int)(c.batch > 1 ? slots * 4 / 5 : slots);
        long long splits = 4 * slots / tiles;
        if (splits > kMostSplits) splits = kMostSplits;
        if (splits < 1) splits = 1;
        long long chunk = (span + splits - 1) / splits;
        chunk = (chunk + kGrain - 1) / kGrain * kGrain;
        if (chunk < kGrain) chunk = kGrain;
        f.chunk = (int)chunk;
        f.splits = (int)((span + chunk - 1) / chunk);
        if (f.splits < 1) f.splits = 1;
        few_bytes = workspace_part(f, plan.few_units, c.d);
    }
    if (prompts) {
        Attend& p = plan.prompt;
        p = g;
        p.rows = kPromptRows;
        if (few) p.least = kFewRows + 1;
        plan.prompt_units = (long long)a.tokens * g.group / kPromptRows + c.batch;
        const long long tiles = plan.prompt_units * c.heads, span = span_of(kPromptRows) + kPromptTokens;
        if (tiles > 0x7fffffffll) return TT_ERR_INVALID_ARG;
        // Few tiles: the keys are split as well, into shares of 256 tokens at least, for 128 CTAs at most (144 of heads of 128 values are slower than
        // 104: 64 tokens over 16000, 8 heads, 50 us and 38) and 16 shares, which the join has under way at once.  Short ones are not worth it (300
        // tokens, 8 heads: 14 us whole, 18 in two).
        long long chunk = span;
        if (2 * tiles <= kPromptCtas && span >= 6 * kPromptTokens) {
            const long long shares = kPromptCtas / tiles < kPromptSplits ? kPromptCtas / tiles : kPromptSplits;
            chunk = (span + shares - 1) / shares;
            chunk = (chunk + kPromptTokens - 1) / kPromptTokens * kPromptTokens;
            if (chunk < 2 * kPromptTokens) chunk = 2 * kPromptTokens;
        }
        p.chunk = (int)(chunk < span ? chunk : (span + kPromptTokens - 1) / kPromptTokens * kPromptTokens);
        p.splits = (int)((span + p.chunk - 1) / p.chunk);
        prompt_bytes = workspace_part(p, plan.prompt_units, prompt_head(c.d));
    }
    plan.prompt_at = kCounterBytes + (few_bytes + 15) / 16 * 16;
    plan.bytes = few_bytes + prompt_bytes > 0 ? plan.prompt_at + prompt_bytes : 0;
    return TT_OK;
}
static void place(Attend& g, void* workspace, long long at) {
    g.counters = static_cast<unsigned*>(workspace);
    g.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + (g.splits > 1 ? at : 0));
}

template <int D, int NT>
static cudaError_t launch_attend(const Attend& g, long long units, void* stream) {
    typedef AttendShape<D, NT> S;
    static OncePerDevice raised;
    const cudaError_t ready = raised([] { return cudaFuncSetAttribute(tt_attend_few_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kBytes); });
    if (ready != cudaSuccess) return ready;
    CUtensorMap maps[2];
    for (int w = 0; w < 2; ++w) {
        const tt_cache& c = g.a.cache;
        const int box = c.block >= S::kTokens ? S::kTokens : kStep;
        // (without pages nothing is read: the map is of any memory)
        const tt_status st = g.max_length > 0 ? encode_pages(&maps[w], c.data[w], c.d, c.block, c.heads, c.pages, c.token[w], c.head[w], c.page[w], S::kLine, true, box)
                                              : encode_pages(&maps[w], reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(g.a.y) & ~uintptr_t(15)), c.d, c.block, 1, 1, c.d, c.d, c.d, S::kLine, true, box);
        if (st != TT_OK) return cudaErrorInvalidValue;
    }
    return launch(tt_attend_few_kernel<D, NT>, dim3((unsigned)units, (unsigned)g.a.cache.heads, (unsigned)g.splits), kAttendWarps * 32, S::kBytes, 1, stream, maps[0], maps[1], g);
}
template <int D>
static cudaError_t launch_attend_rows(const Attend& g, long long units, void* stream) {
    if (g.rows == 8) return launch_attend<D, 1>(g, units, stream);
    if constexpr (D <= 128) if (g.rows == 32) return launch_attend<D, 4>(g, units, stream);
    return launch_attend<D, 2>(g, units, stream);
}

}  // namespace tt

using namespace tt;

extern "C" tt_status tt_cache_append(const tt_cache_append_args* a, void* stream) {
    if (!a || !known_type(a->type) || a->tokens < 0) return TT_ERR_INVALID_ARG;
    const tt_cache& c = a->cache;
    tt_status s = check_cache(c);
    if (s != TT_OK) return s;
    if (a->tokens == 0 || c.batch == 0 || c.heads == 0) return TT_OK;
    s = check_cache_memory(c);
    if (s != TT_OK) return s;
    const int bytes = type_bytes(a->type);
    if (!a->starts || !a->lengths || !a->status || reinterpret_cast<uintptr_t>(a->starts) % 4 || reinterpret_cast<uintptr_t>(a->lengths) % 4 || reinterpret_cast<uintptr_t>(a->status) % 4)
        return TT_ERR_INVALID_ARG;
    bool wide = true;
    for (int w = 0; w < 2; ++w) {
        if (!a->x[w] || reinterpret_cast<uintptr_t>(a->x[w]) % (uintptr_t)bytes || a->x_token[w] < 0 || a->x_head[w] < 0) return TT_ERR_INVALID_ARG;
        wide = wide && on16(a->x[w]) && a->x_token[w] * bytes % 16 == 0 && a->x_head[w] * bytes % 16 == 0;
    }
    const long long units = a->tokens / c.block + 2ll * c.batch;
    if (units > 0x7fffffff) return TT_ERR_INVALID_ARG;
    // A warp has a page's tokens where there is hardly more than one of them, a CTA where there are many.
    const bool warp = (long long)(a->tokens / c.batch < c.block ? a->tokens / c.batch : c.block) * c.d <= 1024;
    const dim3 grid((unsigned)units, warp ? (2u * (unsigned)c.heads + 7u) / 8u : 2u * (unsigned)c.heads, 1);
    const auto go = [&](auto by_warp, auto by_cta) { return status_of(launch(warp ? by_warp : by_cta, grid, warp ? 256 : kAppendThreads, 0, 1, stream, *a)); };
#define TT_APPEND(TYPE) (wide ? go(tt_cache_append_kernel<TYPE, true, true>, tt_cache_append_kernel<TYPE, true, false>) : go(tt_cache_append_kernel<TYPE, false, true>, tt_cache_append_kernel<TYPE, false, false>))
    return a->type == TT_TYPE_F32 ? TT_APPEND(TT_TYPE_F32) : a->type == TT_TYPE_F16 ? TT_APPEND(TT_TYPE_F16) : TT_APPEND(TT_TYPE_BF16);
#undef TT_APPEND
}

extern "C" tt_status tt_cache_attention_workspace(const tt_cache_attention_args* a, int64_t* bytes) {
    if (!a || !bytes) return TT_ERR_INVALID_ARG;
    AttendPlan plan;
    const tt_status s = plan_attend(*a, plan);
    *bytes = s == TT_OK ? plan.bytes : 0;
    return s;
}

extern "C" tt_status tt_cache_attention(const tt_cache_attention_args* a, void* stream) {
    if (!a) return TT_ERR_INVALID_ARG;
    AttendPlan plan;
    tt_status s = plan_attend(*a, plan);
    if (s != TT_OK || (plan.few_units == 0 && plan.prompt_units == 0)) return s;
    const tt_cache& c = a->cache;
    if (c.pages > 0 && c.max_pages > 0) s = check_cache_memory(c);
    if (s != TT_OK) return s;
    if (!a->q || !a->y || !a->starts || !a->lengths || !a->status || a->q_token < 0 || a->q_head < 0 || a->y_token < 0 || a->y_head < 0) return TT_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(a->q) % 2 || reinterpret_cast<uintptr_t>(a->y) % 2 || reinterpret_cast<uintptr_t>(a->starts) % 4 || reinterpret_cast<uintptr_t>(a->lengths) % 4 ||
        reinterpret_cast<uintptr_t>(a->status) % 4) return TT_ERR_INVALID_ARG;
    if (plan.bytes > 0 && (!a->workspace || !on16(a->workspace) || a->workspace_bytes < plan.bytes)) return TT_ERR_INVALID_ARG;
    if (plan.prompt_units > 0) {
        place(plan.prompt, a->workspace, plan.prompt_at);
        s = status_of(launch_attend_prompt(plan.prompt, plan.prompt_units, stream));
        if (s != TT_OK || plan.few_units == 0) return s;
    }
    const Attend& g = plan.few;
    const long long units = plan.few_units;
    place(plan.few, a->workspace, kCounterBytes);
    switch (c.d) {
        case 32: return status_of(launch_attend_rows<32>(g, units, stream));
        case 64: return status_of(launch_attend_rows<64>(g, units, stream));
        case 96: return status_of(launch_attend_rows<96>(g, units, stream));
        case 128: return status_of(launch_attend_rows<128>(g, units, stream));
        case 160: return status_of(launch_attend_rows<160>(g, units, stream));
        case 192: return status_of(launch_attend_rows<192>(g, units, stream));
        case 224: return status_of(launch_attend_rows<224>(g, units, stream));
        default: return status_of(launch_attend_rows<256>(g, units, stream));
    }
}
