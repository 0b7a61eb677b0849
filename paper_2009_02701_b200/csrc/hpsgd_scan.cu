// A gated linear recurrence over sequences, and its gradients.
//
// Per channel h_t = a_t h_(t-1) + (1 - a_t) v_t with a = sigmoid(f): an affine map of the state, and maps compose, so rows need not be gone through
// one by one: (A, H) then (A', H') is (A' A, A' H + H').  A thread takes two neighbouring channels over a group of consecutive rows: it composes its
// rows' maps, the groups' maps are exchanged, and with the state that reaches its first row it goes through its rows again.  So everything is
// read once and written once.  A block's warps have consecutive rows (each of its half warps a group of them), the blocks of a cluster consecutive
// pieces of a chunk of rows, and chunks follow one another; a warp's next rows come to its part of shared memory meanwhile (cp.async, of
// its own, so that no barrier is needed for them).  Sequences need no division of work of their own: the rows are one long sequence, in which a
// map that forgets stands where one begins.
//
// The gradient runs the other way with the same maps: what reaches h_(t-1) is M_t = a_t (g_t + M_(t+1)).  It needs h, which is computed
// again from the state that the forward pass keeps for each eight rows.
//
// Bytes: 8 an element forward and 14 backward in bf16 with output gates, and half a byte each for the kept states.  What bounds it now is the chain of a
// warp's instructions (an instruction every 6.5 cycles of a warp; the unit for powers and quotients, four an element, is 55 % busy forward and 47 % backward):
// 16384 x 2048 of 16 sequences 64 us forward, 104 backward (HBM would allow 43 and 75); 65536 x 1024 of one sequence 150 us (82).  Measured and
// not kept: a chunk's second pass interleaved with the next one's first in the same registers (64 -> 84 us), three and four stages (fewer blocks:
// 82), maps that say in one flag for a block that none forgets (no change).
#include "hpsgd_ops_common.cuh"

#include <algorithm>
#include <type_traits>

namespace hpsgd {
namespace ops {
namespace {

constexpr int kSlab = 32;                           // channels of a block: two for each of 16 lanes
constexpr int kSaved = 8;                           // rows that share a kept state
constexpr int kMaxCluster = 8;

// What a kernel holds: R rows a thread, W warps, S stages of A arrays in shared memory; PER_SM warps on an SM.
template <typename T, int ROWS, int ARRAYS, int WARPS, int PER_SM>
struct Form {
    static constexpr int R = ROWS, A = ARRAYS, W = WARPS, S = 2;
    static constexpr int kThreads = 32 * W, kRows = 2 * R * W;                       // rows of a block's piece of a chunk
    static constexpr int kLine = 2 * kSlab * (int)sizeof(T);                         // a row of each half warp's group, side by side
    static constexpr int kWarpBytes = A * R * kLine, kStageBytes = W * kWarpBytes;
    static constexpr int kPerSm = PER_SM / W;
};

struct Sequences {
    int rows, cols, count, each;                    // each: rows of a sequence where there are no offsets
    int walkers, share;                             // rows of a walker's share
    const int64_t* offsets;

    // First row of sequence s; s = count gives the end of the last one.
    __device__ __forceinline__ int begin(int s) const
    {
        if (!offsets) return s * each;
        const int64_t x = offsets[s];
        return (int)(x < 0 ? 0 : x > rows ? rows : x);
    }

    // The first sequence that begins at row r or behind it (count if none does).  All lanes of a warp come here: 32 places are looked at at once.
    __device__ __forceinline__ int at_or_behind(int r) const
    {
        if (!offsets) return min(count, (int)(((unsigned)r + (unsigned)each - 1u) / (unsigned)max(1, each)));
        int lo = 0, hi = count;
        const int lane = threadIdx.x & 31;
        while (lo < hi) {
            const int step = (hi - lo + 31) / 32, i = lo + lane * step;
            const int less = __popc(__ballot_sync(0xFFFFFFFFu, i < hi && begin(i) < r));
            hi = less ? min(hi, lo + less * step) : lo;
            lo = less ? lo + (less - 1) * step + 1 : lo;
        }
        return lo;
    }
};

// The sequences of a walker: those that begin in its equal share of the rows.  All threads of the block come here.
struct Share {
    int first, last, row0, row1;                    // sequences [first, last), rows [row0, row1)
    __device__ __forceinline__ Share(const Sequences& q, int walker)
    {
        const auto border = [&](int w) { return min(q.rows, w * q.share); };
        first = walker == 0 ? 0 : q.at_or_behind(border(walker));
        last = walker + 1 == q.walkers ? q.count : q.at_or_behind(border(walker + 1));
        last = max(first, last);
        row0 = first < last ? q.begin(first) : 0;
        row1 = first < last ? max(row0, q.begin(last)) : 0;
    }
};

// Where sequences begin and end among the rows [r0, r0 + R) of a warp: a bit for each row, and which sequence it is.  The last sequence seen is
// remembered, so that rows inside of it are not looked up.
struct Marks {
    uint32_t begins, ends;
    int from, to;                                   // a sequence that is known
};
template <int R>
__device__ __forceinline__ void find_marks(const Sequences& q, int r0, int (*which)[32], Marks& m)
{
    m.begins = m.ends = 0u;
    if (m.from < r0 && m.to > r0 + R) return;
    const int lane = threadIdx.x & 31;
    __syncwarp();
    for (int k = max(0, q.at_or_behind(r0) - 1);; k += 32) {
        const int i = k + lane, b = i < q.count ? q.begin(i) : 0x7FFFFFFF, e = i < q.count ? q.begin(i + 1) : 0;
        if (b < e) {
            if (b >= r0 && b < r0 + R) m.begins |= 1u << (b - r0), which[0][b - r0] = i;
            if (e > r0 && e <= r0 + R) m.ends |= 1u << (e - 1 - r0), which[1][e - 1 - r0] = i;
        }
        const uint32_t wide = __ballot_sync(0xFFFFFFFFu, b < e && e - b > R);
        if (wide) m.from = __shfl_sync(0xFFFFFFFFu, b, 31 - __clz(wide)), m.to = __shfl_sync(0xFFFFFFFFu, e, 31 - __clz(wide));
        if (!__all_sync(0xFFFFFFFFu, i < q.count && b < r0 + R)) break;
    }
    m.begins = __reduce_or_sync(0xFFFFFFFFu, m.begins);
    m.ends = __reduce_or_sync(0xFFFFFFFFu, m.ends);
    __syncwarp();
}

// ---------------------------------------------------------------------------- two channels
__device__ __forceinline__ pair load_two(const float* p, int left) { return make_pair(left > 0 ? p[0] : 0.f, left > 1 ? p[1] : 0.f); }
__device__ __forceinline__ pair load_two(const __nv_bfloat16* p, int left) { return make_pair(left > 0 ? load1(p) : 0.f, left > 1 ? load1(p + 1) : 0.f); }
__device__ __forceinline__ pair load_pair(const float* p)
{
    const float2 x = *reinterpret_cast<const float2*>(p);
    return make_pair(x.x, x.y);
}
__device__ __forceinline__ pair load_pair(const __nv_bfloat16* p)
{
    float lo, hi;
    widen_pair(*reinterpret_cast<const uint32_t*>(p), lo, hi);
    return make_pair(lo, hi);
}
// (written so that what is read from shared memory behind a store may be requested in front of it)
__device__ __forceinline__ void store_pair(float* p, float lo, float hi) { asm volatile("st.global.v2.f32 [%0], {%1, %2};" ::"l"(p), "f"(lo), "f"(hi)); }
__device__ __forceinline__ void store_pair(__nv_bfloat16* p, float lo, float hi) { asm volatile("st.global.b32 [%0], %1;" ::"l"(p), "r"(pack_bf16(lo, hi))); }

// WIDE: the address allows both in one access.  `left` of them are there; ALL: both are.
template <bool WIDE, bool ALL = false, typename T>
__device__ __forceinline__ void store_two(T* p, pair v, int left)
{
    float lo, hi;
    split(v, lo, hi);
    if (WIDE && (ALL || left > 1)) store_pair(p, lo, hi);
    else {
        if (left > 0) store1(p, lo);
        if (left > 1) store1(p + 1, hi);
    }
}

__device__ __forceinline__ void copy_async16(uint32_t to, const void* from, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
// s = sigmoid(x) and 1 - s: e = 2^(-x log2 e), s = 1 / (1 + e), 1 - s = e s.  The exponent is rounded with its product, so e is right to |x| 2^-23 + 2^-22 of
// itself, and so is the smaller of the two; the one next to 1 to a few 2^-24.  e is held to 2^126, so that s is not 0 where e s has to be 1; a NaN stays one.
__device__ __forceinline__ void sigmoid(pair x, pair& s, pair& rest)
{
    float lo, hi;
    split(mul2(x, both(-kLog2e)), lo, hi);
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(lo) : "f"(126.f));
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(hi) : "f"(126.f));
    const pair e = make_pair(exp2_of(lo), exp2_of(hi));
    float d0, d1;
    split(add2(e, both(1.f)), d0, d1);
    s = make_pair(reciprocal(d0), reciprocal(d1));
    rest = mul2(e, s);
}
__device__ __forceinline__ pair sigmoid(pair x)
{
    float lo, hi;
    split(mul2(x, both(-kLog2e)), lo, hi);
    float d0, d1;
    split(add2(make_pair(exp2_of(lo), exp2_of(hi)), both(1.f)), d0, d1);
    return make_pair(reciprocal(d0), reciprocal(d1));
}

// ---------------------------------------------------------------------------- maps
// h -> A h + H.  A map that forgets what comes in (a sequence begins in it) has A = -1, which no product of gates is: what came in may
// be infinite or NaN, and 0 times it would not be 0.
struct Map {
    pair A, H;
    __device__ __forceinline__ pair of(pair h) const
    {
        float a0, a1;
        split(A, a0, a1);
        return a0 == -1.f ? H : fma2(A, h, H);      // (both channels forget, or neither)
    }
    // this one behind m
    __device__ __forceinline__ Map behind(const Map& m) const
    {
        float a0, a1, m0, m1;
        split(A, a0, a1);
        split(m.A, m0, m1);
        Map r;
        r.A = a0 == -1.f ? A : m0 == -1.f ? m.A : mul2(A, m.A);
        r.H = a0 == -1.f ? H : fma2(A, m.H, H);
        return r;
    }
};
__device__ __forceinline__ Map identity() { return Map{both(1.f), both(0.f)}; }

__device__ __forceinline__ void map_to_block(const ulonglong2* at, int rank, const Map& m)
{
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(shared_address(at)), "r"(rank));
    asm volatile("st.shared::cluster.v2.u64 [%0], {%1, %2};" ::"r"(there), "l"(m.A), "l"(m.H) : "memory");
}

// What the maps are exchanged through; two of each in turn, so that one barrier a chunk is enough.
template <int W>
struct Exchange {
    ulonglong2 warp[2][W][16];                      // of this block's warps
    ulonglong2 block[2][kMaxCluster][16];           // of the cluster's blocks
};

// The state that reaches this thread's group, given the state in front of the chunk (`carry`, which becomes the one behind it).  `half`, `warp` and
// `rank` count in the direction of the recurrence.  All threads of the cluster come here.
template <int W, bool CLUSTER>
__device__ __forceinline__ pair exchange(Exchange<W>& x, int turn, const Map& mine, pair& carry, int half, int warp, int rank, int blocks)
{
    const int lane = threadIdx.x & 15;
    const Map other{__shfl_xor_sync(0xFFFFFFFFu, mine.A, 16), __shfl_xor_sync(0xFFFFFFFFu, mine.H, 16)};
    if (half == 1) {
        const Map both_halves = mine.behind(other);
        x.warp[turn][warp][lane] = make_ulonglong2(both_halves.A, both_halves.H);
    }
    __syncthreads();
    const auto of_warp = [&](int w) {
        const ulonglong2 m = x.warp[turn][w][lane];
        return Map{m.x, m.y};
    };
    pair in;
    if constexpr (!CLUSTER) {
        pair h = in = carry;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (w == warp) in = h;
            h = of_warp(w).of(h);
        }
        carry = h;
    } else {
        if (warp == 0) {                            // the block's own map to all blocks
            Map all = of_warp(0);
#pragma unroll
            for (int w = 1; w < W; ++w) all = of_warp(w).behind(all);
            for (int r = half; r < blocks; r += 2) map_to_block(&x.block[turn][rank][lane], r, all);
            // Only this warp has something to publish; a release by all of them waits for every store of theirs to device memory as well.
            asm volatile("fence.acq_rel.cluster;" ::: "memory");
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
        Map before = identity();
        for (int w = 0; w < warp; ++w) before = of_warp(w).behind(before);
        cluster_wait();
        pair h = in = carry;
        for (int r = 0; r < blocks; ++r) {
            if (r == rank) in = h;
            const ulonglong2 m = x.block[turn][r][lane];
            h = Map{m.x, m.y}.of(h);
        }
        carry = h;
        in = before.of(in);
    }
    return half == 1 ? other.of(in) : in;
}

// ---------------------------------------------------------------------------- where a thread stands
// Rows r .. r + R - 1 of a group.  in: those that are the walker's; begins, ends: of those, where a sequence does.
struct Group {
    uint32_t in, begins, ends;
    bool plain;                                     // all rows of the warp's groups are, nothing begins or ends, and all of the slab's columns are there
};
template <int R>
__device__ __forceinline__ Group group_of(const Share& mine, const Marks& m, int warp_row, int half, bool whole)
{
    constexpr uint32_t kAll = (1u << R) - 1u;
    const int r = warp_row + half * R;
    Group g;
    g.plain = whole && warp_row >= mine.row0 && warp_row + 2 * R <= mine.row1 && (m.begins | m.ends) == 0u;
    const uint32_t below = r >= mine.row0 ? 0u : r + R <= mine.row0 ? kAll : (1u << (mine.row0 - r)) - 1u;
    g.in = kAll & ~below & (r + R <= mine.row1 ? kAll : r >= mine.row1 ? 0u : (1u << (mine.row1 - r)) - 1u);
    g.begins = m.begins >> (half * R) & g.in;
    g.ends = m.ends >> (half * R) & g.in;
    return g;
}

// The rows of one array that a warp requests (two groups of R, side by side in shared memory), chunk after chunk: a lane has 16 bytes of every
// kAtOnce-th row.
template <typename T, int R>
struct Requests {
    static constexpr int kLine = 2 * kSlab * (int)sizeof(T), kPieces = kLine / 16, kAtOnce = 32 / kPieces;      // rows of both groups in one instruction
    const char* at;                                 // of the rows that come next
    const void* base;
    int64_t step, next;                             // bytes: kAtOnce rows, a chunk

    __device__ __forceinline__ Requests(const T* p, int64_t ld, int warp_row, int slab, int64_t chunk)
    {
        const int lane = threadIdx.x & 31, piece = lane % kPieces, half = piece / (kPieces / 2);
        base = p;
        at = reinterpret_cast<const char*>(p) + ((warp_row + half * R + lane / kPieces) * ld + slab * kSlab) * (int)sizeof(T) + piece % (kPieces / 2) * 16;
        step = kAtOnce * ld * (int)sizeof(T);
        next = chunk * ld * (int)sizeof(T);
    }
    __device__ __forceinline__ void skip() { at += next; }
    // all rows and columns are there
    __device__ __forceinline__ void all(uint32_t to)
    {
        const uint32_t mine = to + (threadIdx.x & 31) * 16;
        const char* from = at;
#pragma unroll
        for (int i = 0; i < R; i += kAtOnce, from += step) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(mine + i * kLine), "l"(from) : "memory");
        at += next;
    }
    // rows that are not the walker's and columns behind the last become zeros
    __device__ __forceinline__ void some(uint32_t to, int warp_row, int slab, int cols, const Share& mine)
    {
        const int lane = threadIdx.x & 31, piece = lane % kPieces, half = piece / (kPieces / 2);
        const int bytes = min(16, max(0, (cols - slab * kSlab) * (int)sizeof(T) - piece % (kPieces / 2) * 16));
        const char* from = at;
#pragma unroll
        for (int i = 0; i < R; i += kAtOnce, from += step) {
            const int row = warp_row + half * R + i + lane / kPieces;
            const bool there = row >= mine.row0 && row < mine.row1 && bytes > 0;
            copy_async16(to + i * kLine + lane * 16, there ? from : base, there ? bytes : 0);
        }
        at += next;
    }
};

// ---------------------------------------------------------------------------- forward
struct ScanForward {
    Sequences q;
    int slabs, blocks;                              // blocks of a cluster
    const void* f;
    const void* v;
    const void* o;
    const float* h0;
    float* h_last;
    void* y;
    float* saved;
    int64_t ldf, ldv, ldo, ldy, ldh0, ldlast, ldsaved;
};

// Blocks of a cluster wait for one another, and longest for the cluster's barrier: there a chunk is 16 rows a thread (8 in fp32) of eight warps.  By
// themselves they are many, and small: eight rows a thread of four warps, so that there are twice as many warps to wait with.
template <typename T, bool GATE, bool CLUSTER>
using ForwardForm = Form<T, CLUSTER && sizeof(T) == 2 ? 16 : 8, GATE ? 3 : 2, CLUSTER || sizeof(T) == 4 ? 8 : 4, !CLUSTER && sizeof(T) == 2 ? 32 : 16>;

// STAGED: rows of the inputs start on 16-byte boundaries and two outputs can be stored at once; else both are taken one by one, without a stage.
template <typename T, bool GATE, bool STAGED, bool CLUSTER>
__global__ void __launch_bounds__(ForwardForm<T, GATE, CLUSTER>::kThreads, ForwardForm<T, GATE, CLUSTER>::kPerSm) scan_forward_kernel(const ScanForward a)
{
    using F = ForwardForm<T, GATE, CLUSTER>;
    constexpr int R = F::R;
    extern __shared__ __align__(16) uint8_t stages[];
    __shared__ alignas(16) Exchange<F::W> ex;
    __shared__ int which_of[F::W][2][32];
    const Sequences& q = a.q;
    const int warp = threadIdx.x >> 5, half = (threadIdx.x >> 4) & 1, lane = threadIdx.x & 15;
    const int rank = CLUSTER ? (int)(blockIdx.x % (unsigned)a.blocks) : 0, unit = CLUSTER ? (int)(blockIdx.x / (unsigned)a.blocks) : (int)blockIdx.x;
    const int slab = unit % a.slabs, c = slab * kSlab + lane * 2, left = max(0, min(2, q.cols - c));
    int(*const which)[32] = which_of[warp];
    after_previous();
    if constexpr (CLUSTER) cluster_arrive();        // the others' shared memory is there to be written; waited for below
    const Share mine(q, unit / a.slabs);
    const int start = mine.row0 / R * R, chunk = a.blocks * F::kRows;
    int r = start + (rank * F::W + warp) * 2 * R;   // the warp's first row
    const T* const f = static_cast<const T*>(a.f);
    const T* const v = static_cast<const T*>(a.v);
    const T* const o = static_cast<const T*>(a.o);
    T* const y = static_cast<T*>(a.y) + c;
    const uint32_t room = shared_address(stages) + warp * F::kWarpBytes;
    const bool whole = q.cols - slab * kSlab >= kSlab;
    Requests<T, R> rf(f, a.ldf, r, slab, chunk), rv(v, a.ldv, r, slab, chunk), ro(o, a.ldo, r, slab, chunk);
    const auto request = [&](int row, int stage) {  // (rows one chunk behind those of the last call)
        if constexpr (STAGED) {
            const uint32_t to = room + stage * F::kStageBytes;
            if (whole && row >= mine.row0 && row + 2 * R <= mine.row1) {
                rf.all(to);
                rv.all(to + R * F::kLine);
                if (GATE) ro.all(to + 2 * R * F::kLine);
            } else if (row < mine.row1) {
                rf.some(to, row, slab, q.cols, mine);
                rv.some(to + R * F::kLine, row, slab, q.cols, mine);
                if (GATE) ro.some(to + 2 * R * F::kLine, row, slab, q.cols, mine);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    request(r, 0);
    // sequences without rows: their state goes through
    if (a.h_last && rank == 0)
        for (int s = mine.first + (int)(threadIdx.x >> 4); s < mine.last; s += 2 * F::W)
            if (q.begin(s) >= q.begin(s + 1)) store_two<false>(a.h_last + s * a.ldlast + c, a.h0 ? load_two(a.h0 + s * a.ldh0 + c, left) : both(0.f), left);
    if constexpr (CLUSTER) {
        __syncwarp();
        cluster_wait();
    }

    Marks m{0u, 0u, 0, 0};
    pair carry = both(0.f);
    int turn = 0;
    for (int base = start; base < mine.row1; base += chunk, r += chunk, turn ^= 1) {
        request(r + chunk, turn ^ 1);
        find_marks<2 * R>(q, r, which, m);
        const Group w = group_of<R>(mine, m, r, half, whole);
        if constexpr (STAGED) {
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            __syncwarp();
        }
        const T* const staged = reinterpret_cast<const T*>(stages + turn * F::kStageBytes + warp * F::kWarpBytes) + half * kSlab + lane * 2;
        const int64_t row = r + half * R;
        const auto value = [&](int array, const T* p, int64_t ld, int t) {
            if constexpr (STAGED) return load_pair(staged + (array * R + t) * 2 * kSlab);
            else return load_two(p + (row + t) * ld + c, w.in >> t & 1u ? left : 0);
        };
        pair g[R], b[R];                            // the gates, and what they let in
        Map map = identity();
        if (w.plain) {
#pragma unroll
            for (int t = 0; t < R; ++t) {
                pair rest;
                sigmoid(value(0, f, a.ldf, t), g[t], rest);
                b[t] = mul2(rest, value(1, v, a.ldv, t));
                map.H = fma2(g[t], map.H, b[t]);
                map.A = mul2(map.A, g[t]);
            }
        } else {
            bool forgets = false;
#pragma unroll
            for (int t = 0; t < R; ++t) {
                pair rest;
                sigmoid(value(0, f, a.ldf, t), g[t], rest);
                b[t] = mul2(rest, value(1, v, a.ldv, t));
                if (!(w.in >> t & 1u)) g[t] = both(1.f), b[t] = both(0.f);
                if (w.begins >> t & 1u) {
                    if (a.h0) b[t] = fma2(g[t], load_two(a.h0 + which[0][half * R + t] * a.ldh0 + c, left), b[t]);
                    map.H = b[t];
                    forgets = true;
                } else {
                    map.H = fma2(g[t], map.H, b[t]);
                    map.A = mul2(map.A, g[t]);
                }
            }
            if (forgets) map.A = both(-1.f);
            __syncwarp();
        }
        pair h = exchange<F::W, CLUSTER>(ex, turn, map, carry, half, warp, rank, a.blocks);
        float* const keep = a.saved ? a.saved + row / kSaved * a.ldsaved + c : nullptr;
        T* to = y + row * a.ldy;
        if (w.plain) {
#pragma unroll
            for (int t = 0; t < R; ++t, to += a.ldy) {
                if (t % kSaved == 0 && keep) store_two<true, true>(keep + t / kSaved * a.ldsaved, h, left);
                h = fma2(g[t], h, b[t]);
                store_two<STAGED, true>(to, GATE ? mul2(h, sigmoid(value(2, o, a.ldo, t))) : h, 2);
            }
        } else {
#pragma unroll
            for (int t = 0; t < R; ++t, to += a.ldy) {
                if (t % kSaved == 0 && keep && (w.in >> t & 1u)) store_two<true>(keep + t / kSaved * a.ldsaved, h, left);
                h = w.begins >> t & 1u ? b[t] : fma2(g[t], h, b[t]);
                if (w.ends >> t & 1u)
                    if (a.h_last) store_two<false>(a.h_last + which[1][half * R + t] * a.ldlast + c, h, left);
                if (w.in >> t & 1u) store_two<STAGED>(to, GATE ? mul2(h, sigmoid(value(2, o, a.ldo, t))) : h, left);
            }
        }
        __syncwarp();                               // the stage has been read, and may be filled again
    }
}

// One token for each sequence: no row depends on another.
template <typename T, bool GATE, bool WIDE>
__global__ void __launch_bounds__(128) scan_step_kernel(const ScanForward a)
{
    const int row = blockIdx.y, c = ((int)blockIdx.x * 128 + (int)threadIdx.x) * 2, left = min(2, a.q.cols - c);
    if (left <= 0) return;
    const T* const f = static_cast<const T*>(a.f) + row * a.ldf + c;
    const T* const v = static_cast<const T*>(a.v) + row * a.ldv + c;
    const T* const o = static_cast<const T*>(a.o) + row * a.ldo + c;
    after_previous();
    const auto load = [&](const T* p) { return WIDE && left == 2 ? load_pair(p) : load_two(p, left); };
    const pair fx = load(f), vx = load(v), ox = GATE ? load(o) : both(0.f), h0 = a.h0 ? load_two(a.h0 + row * a.ldh0 + c, left) : both(0.f);
    pair g, rest;
    sigmoid(fx, g, rest);
    const pair h = fma2(g, h0, mul2(rest, vx));
    if (a.h_last) store_two<false>(a.h_last + row * a.ldlast + c, h, left);
    store_two<WIDE>(static_cast<T*>(a.y) + row * a.ldy + c, GATE ? mul2(h, sigmoid(ox)) : h, left);
}

// ---------------------------------------------------------------------------- backward
struct ScanBackward {
    Sequences q;
    int slabs, blocks;
    const void* f;
    const void* v;
    const void* o;
    const float* h0;
    const float* saved;
    const void* dy;
    const float* dh_last;
    void* df;
    void* dv;
    void* d_o;
    float* dh0;
    int64_t ldf, ldv, ldo, ldh0, lddy, lddlast, lddf, lddv, lddo, lddh0, ldsaved;
};

template <typename T, bool GATE, bool CLUSTER>
using BackwardForm = Form<T, kSaved, GATE ? 4 : 3, CLUSTER ? 8 : 4, sizeof(T) == 2 ? 16 : CLUSTER ? 8 : 12>;

template <typename T, bool GATE, bool STAGED, bool CLUSTER>
__global__ void __launch_bounds__(BackwardForm<T, GATE, CLUSTER>::kThreads, BackwardForm<T, GATE, CLUSTER>::kPerSm) scan_backward_kernel(const ScanBackward a)
{
    using F = BackwardForm<T, GATE, CLUSTER>;
    constexpr int R = F::R;
    extern __shared__ __align__(16) uint8_t stages[];
    __shared__ alignas(16) Exchange<F::W> ex;
    __shared__ alignas(16) float kept[2][F::W][2 * kSlab];      // the states in front of the groups' first rows
    __shared__ int which_of[F::W][2][32];
    const Sequences& q = a.q;
    const int warp = threadIdx.x >> 5, half = (threadIdx.x >> 4) & 1, lane = threadIdx.x & 15;
    const int rank = CLUSTER ? (int)(blockIdx.x % (unsigned)a.blocks) : 0, unit = CLUSTER ? (int)(blockIdx.x / (unsigned)a.blocks) : (int)blockIdx.x;
    const int slab = unit % a.slabs, c = slab * kSlab + lane * 2, left = max(0, min(2, q.cols - c));
    int(*const which)[32] = which_of[warp];
    after_previous();
    if constexpr (CLUSTER) cluster_arrive();
    const Share mine(q, unit / a.slabs);
    // chunks from the last to the first; in a chunk as well the first warp of the first block has the last rows
    const int start = mine.row0 / R * R, chunk = a.blocks * F::kRows;
    const int chunks = (mine.row1 - start + chunk - 1) / chunk;
    int r = start + (chunks - 1) * chunk + ((a.blocks - 1 - rank) * F::W + (F::W - 1 - warp)) * 2 * R;
    const T* const f = static_cast<const T*>(a.f);
    const T* const v = static_cast<const T*>(a.v);
    const T* const o = static_cast<const T*>(a.o);
    const T* const dy = static_cast<const T*>(a.dy);
    T* const df = static_cast<T*>(a.df) + c;
    T* const dv = static_cast<T*>(a.dv) + c;
    T* const d_o = static_cast<T*>(a.d_o) + c;
    const uint32_t room = shared_address(stages) + warp * F::kWarpBytes;
    const bool whole = q.cols - slab * kSlab >= kSlab;
    Requests<T, R> rf(f, a.ldf, r, slab, -chunk), rv(v, a.ldv, r, slab, -chunk), rd(dy, a.lddy, r, slab, -chunk), ro(o, a.ldo, r, slab, -chunk);
    const auto request = [&](int row, int stage) {
        if constexpr (STAGED) {
            const uint32_t to = room + stage * F::kStageBytes;
            if (whole && row >= mine.row0 && row + 2 * R <= mine.row1) {
                rf.all(to);
                rv.all(to + R * F::kLine);
                rd.all(to + 2 * R * F::kLine);
                if (GATE) ro.all(to + 3 * R * F::kLine);
            } else if (row >= start && row < mine.row1) {
                rf.some(to, row, slab, q.cols, mine);
                rv.some(to + R * F::kLine, row, slab, q.cols, mine);
                rd.some(to + 2 * R * F::kLine, row, slab, q.cols, mine);
                if (GATE) ro.some(to + 3 * R * F::kLine, row, slab, q.cols, mine);
            } else {                                // behind the last row, in the last chunk, which comes first
                rf.skip();
                rv.skip();
                rd.skip();
                ro.skip();
            }
        }
        // (the kept rows are padded to whole pieces of four)
        const int piece = lane % 8, group = row + half * R;
        if (lane < 8 && row >= start && group < mine.row1 && slab * kSlab + piece * 4 < a.ldsaved)
            copy_async16(shared_address(&kept[stage][warp][half * kSlab + piece * 4]), a.saved + (int64_t)(group / kSaved) * a.ldsaved + slab * kSlab + piece * 4, 16);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    request(r, 0);
    if (a.dh0 && rank == 0)
        for (int s = mine.first + (int)(threadIdx.x >> 4); s < mine.last; s += 2 * F::W)
            if (q.begin(s) >= q.begin(s + 1)) store_two<false>(a.dh0 + s * a.lddh0 + c, a.dh_last ? load_two(a.dh_last + s * a.lddlast + c, left) : both(0.f), left);
    if constexpr (CLUSTER) {
        __syncwarp();
        cluster_wait();
    }

    Marks m{0u, 0u, 0, 0};
    pair carry = both(0.f);
    int turn = 0;
    for (int k = chunks - 1; k >= 0; --k, r -= chunk, turn ^= 1) {
        request(r - chunk, turn ^ 1);
        find_marks<2 * R>(q, r, which, m);
        const Group w = group_of<R>(mine, m, r, half, whole);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncwarp();
        const T* const staged = reinterpret_cast<const T*>(stages + turn * F::kStageBytes + warp * F::kWarpBytes) + half * kSlab + lane * 2;
        const int64_t row = r + half * R;
        const auto value = [&](int array, const T* p, int64_t ld, int t) {
            if constexpr (STAGED) return load_pair(staged + (array * R + t) * 2 * kSlab);
            else return load_two(p + (row + t) * ld + c, w.in >> t & 1u ? left : 0);
        };
        pair h = w.in ? load_pair(&kept[turn][warp][half * kSlab + lane * 2]) : both(0.f);
        pair g[R], rest[R], step[R], dh[R];         // a, 1 - a, h_(t-1) - v, the gradient that reaches h_t through y
        const auto gather = [&](auto tag) {
            constexpr bool plain = decltype(tag)::value;
            T* to = d_o + row * a.lddo;
#pragma unroll
            for (int t = 0; t < R; ++t, to += a.lddo) {
                const pair vt = value(1, v, a.ldv, t), dt = value(2, dy, a.lddy, t);
                sigmoid(value(0, f, a.ldf, t), g[t], rest[t]);
                if constexpr (!plain)
                    if (w.begins >> t & 1u) h = a.h0 ? load_two(a.h0 + which[0][half * R + t] * a.ldh0 + c, left) : both(0.f);
                step[t] = fma2(vt, both(-1.f), h);
                h = fma2(g[t], h, mul2(rest[t], vt));
                dh[t] = dt;
                if (GATE) {
                    pair s, s1;
                    sigmoid(value(3, o, a.ldo, t), s, s1);
                    dh[t] = mul2(dt, s);
                    if (plain || (w.in >> t & 1u)) store_two<STAGED, plain>(to, mul2(mul2(dh[t], h), s1), left);
                }
                if constexpr (!plain)
                    if (w.ends >> t & 1u)
                        if (a.dh_last) dh[t] = add2(dh[t], load_two(a.dh_last + which[1][half * R + t] * a.lddlast + c, left));
            }
        };
        // M -> a (dh + M), rows from the last to the first; nothing comes into a sequence's last row
        Map map = identity();
        if (w.plain) {
            gather(std::true_type{});
#pragma unroll
            for (int t = R - 1; t >= 0; --t) {
                map.H = mul2(g[t], add2(dh[t], map.H));
                map.A = mul2(map.A, g[t]);
            }
        } else {
            gather(std::false_type{});
            bool forgets = false;
#pragma unroll
            for (int t = R - 1; t >= 0; --t) {
                if (!(w.in >> t & 1u)) continue;
                map.H = mul2(g[t], w.ends >> t & 1u ? dh[t] : add2(dh[t], map.H));
                map.A = mul2(map.A, g[t]);
                forgets = forgets || (w.ends >> t & 1u);
            }
            if (forgets) map.A = both(-1.f);
            __syncwarp();
        }
        pair M = exchange<F::W, CLUSTER>(ex, turn, map, carry, 1 - half, warp, rank, a.blocks);
        T* to_v = dv + (row + R - 1) * a.lddv;
        T* to_f = df + (row + R - 1) * a.lddf;
        if (w.plain) {
#pragma unroll
            for (int t = R - 1; t >= 0; --t, to_v -= a.lddv, to_f -= a.lddf) {
                const pair G = add2(dh[t], M), p = mul2(G, rest[t]);
                M = mul2(G, g[t]);
                store_two<STAGED, true>(to_v, p, 2);
                store_two<STAGED, true>(to_f, mul2(mul2(p, g[t]), step[t]), 2);
            }
        } else {
#pragma unroll
            for (int t = R - 1; t >= 0; --t, to_v -= a.lddv, to_f -= a.lddf) {
                if (!(w.in >> t & 1u)) continue;
                const pair G = w.ends >> t & 1u ? dh[t] : add2(dh[t], M), p = mul2(G, rest[t]);
                M = mul2(G, g[t]);
                store_two<STAGED>(to_v, p, left);
                store_two<STAGED>(to_f, mul2(mul2(p, g[t]), step[t]), left);
                if (w.begins >> t & 1u)
                    if (a.dh0) store_two<false>(a.dh0 + which[0][half * R + t] * a.lddh0 + c, M, left);
            }
        }
        __syncwarp();
    }
}

// ---------------------------------------------------------------------------- host side
// rows of a chunk and columns of a block that reach past the end are counted too
constexpr int64_t kMostRows = 0x7FFFFFFF - 65536, kMostCols = 0x7FFFFFFF - 512;

int check_sequences(const char* what, int64_t rows, int64_t cols, int64_t sequences, int dtype, const int64_t* offsets)
{
    if (rows < 0 || cols < 0 || sequences < 0) return report(HPSGD_E_BADARG, "%s: a size is negative", what);
    if (dtype != HPSGD_F32 && dtype != HPSGD_BF16) return report(HPSGD_E_BADARG, "%s: unknown dtype %d", what, dtype);
    if (rows > kMostRows || cols > kMostCols || sequences > 0x7FFFFFFF - 64) return report(HPSGD_E_UNSUPPORTED, "%s: a size is too large", what);
    if (!offsets && sequences > 0 && rows % sequences) return report(HPSGD_E_BADARG, "%s: without offsets rows must be a multiple of sequences", what);
    if (!aligned(offsets, 8)) return report(HPSGD_E_BADARG, "%s: offsets is not 8-byte aligned", what);
    return HPSGD_OK;
}

// A matrix of the call's columns: its stride, its alignment, and whether its rows start on `unit` bytes.
int check_rows(const char* what, const char* name, const void* p, int64_t* ld, int64_t cols, int64_t esz, int64_t unit, bool* all)
{
    if (*ld == 0) *ld = cols;
    if (!p) return HPSGD_OK;
    if (*ld < cols) return report(HPSGD_E_BADARG, "%s: the stride of %s is below cols", what, name);
    if (!aligned(p, esz)) return report(HPSGD_E_BADARG, "%s: %s is not aligned to its elements", what, name);
    if (all) *all = *all && aligned(p, unit) && *ld * esz % unit == 0;
    return HPSGD_OK;
}

struct Plan {
    int slabs, walkers, blocks;
};

// Walkers first: they wait for nobody (16384 x 2048 bf16 of 16 sequences: 66 and 107 us with 16 walkers; clusters of eight 117 and 170), but what a sequence
// that is longer than a walker's share has more is waited for at the end, so without equal sequences each has two on the average.  Where they do not
// fill half of the SMs' places, clusters, whose blocks share rows whatever the sequences are, as many as the device holds at once (65536 x 1024
// of one sequence: 150 us with clusters of eight, 195 with four, 445 with two).
template <int ALONE, int TOGETHER>
Plan plan_of(int64_t rows, int64_t cols, int64_t sequences, bool equal)
{
    constexpr int64_t kAlone = 148 * 8, kTogether = 148 * 2;
    Plan p{};
    p.slabs = (int)((cols + kSlab - 1) / kSlab);
    p.walkers = p.blocks = 1;
    const int64_t most = equal ? sequences : (sequences + 1) / 2;
    while ((int64_t)p.slabs * p.walkers * 2 <= kAlone && p.walkers * 2 <= most && rows > ALONE * p.walkers) p.walkers *= 2;
    if ((int64_t)p.slabs * p.walkers * 2 > kAlone / 2 || rows <= ALONE * p.walkers * 2) return p;
    p.walkers = 1;
    while ((int64_t)p.slabs * p.blocks * 2 <= kTogether && p.blocks < kMaxCluster && rows > TOGETHER * p.blocks) p.blocks *= 2;
    while ((int64_t)p.slabs * p.blocks * p.walkers * 2 <= kTogether && p.walkers * 2 <= most && rows > TOGETHER * p.blocks * p.walkers) p.walkers *= 2;
    return p;
}

template <typename F, bool STAGED, auto kernel, typename Args>
int launch_scan(const char* what, const Args& a, const Plan& p, cudaStream_t s)
{
    static bool ready[64] = {};
    const size_t smem = STAGED ? F::S * F::kStageBytes : 0;
    int dev = 0;
    OPS_CUDA(cudaGetDevice(&dev));
    if (dev >= 64 || !ready[dev]) {
        OPS_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        if (dev < 64) ready[dev] = true;
    }
    return launch_clusters(what, kernel, dim3((unsigned)(p.slabs * p.walkers * p.blocks)), F::kThreads, smem, p.blocks, s, a);
}

template <typename T, bool GATE, bool STAGED>
int forward_launch(ScanForward& a, bool equal, cudaStream_t s)
{
    const char* what = "hpsgd_gated_scan_forward";
    using Alone = ForwardForm<T, GATE, false>;
    using Together = ForwardForm<T, GATE, true>;
    const Plan p = plan_of<Alone::kRows, Together::kRows>(a.q.rows, a.q.cols, a.q.count, equal);
    a.slabs = p.slabs; a.blocks = p.blocks; a.q.walkers = p.walkers; a.q.share = (a.q.rows + p.walkers - 1) / p.walkers;
    return p.blocks > 1 ? launch_scan<Together, STAGED, scan_forward_kernel<T, GATE, STAGED, true>>(what, a, p, s)
                        : launch_scan<Alone, STAGED, scan_forward_kernel<T, GATE, STAGED, false>>(what, a, p, s);
}
template <typename T, bool GATE>
int forward_gate(ScanForward& a, bool equal, bool staged, bool wide, cudaStream_t s)
{
    const char* what = "hpsgd_gated_scan_forward";
    if (equal && a.q.rows == a.q.count && a.q.rows <= 65535) {
        const dim3 grid((unsigned)((a.q.cols + 255) / 256), (unsigned)a.q.rows);
        return wide ? launch_early(what, scan_step_kernel<T, GATE, true>, grid, 128, 0, s, a) : launch_early(what, scan_step_kernel<T, GATE, false>, grid, 128, 0, s, a);
    }
    return staged ? forward_launch<T, GATE, true>(a, equal, s) : forward_launch<T, GATE, false>(a, equal, s);
}
template <typename T>
int forward_types(ScanForward& a, bool equal, bool staged, bool wide, cudaStream_t s)
{
    return a.o ? forward_gate<T, true>(a, equal, staged, wide, s) : forward_gate<T, false>(a, equal, staged, wide, s);
}

template <typename T, bool GATE, bool STAGED>
int backward_launch(ScanBackward& a, bool equal, cudaStream_t s)
{
    const char* what = "hpsgd_gated_scan_backward";
    using Alone = BackwardForm<T, GATE, false>;
    using Together = BackwardForm<T, GATE, true>;
    const Plan p = plan_of<Alone::kRows, Together::kRows>(a.q.rows, a.q.cols, a.q.count, equal);
    a.slabs = p.slabs; a.blocks = p.blocks; a.q.walkers = p.walkers; a.q.share = (a.q.rows + p.walkers - 1) / p.walkers;
    return p.blocks > 1 ? launch_scan<Together, STAGED, scan_backward_kernel<T, GATE, STAGED, true>>(what, a, p, s)
                        : launch_scan<Alone, STAGED, scan_backward_kernel<T, GATE, STAGED, false>>(what, a, p, s);
}
template <typename T, bool GATE>
int backward_gate(ScanBackward& a, bool equal, bool staged, cudaStream_t s)
{
    return staged ? backward_launch<T, GATE, true>(a, equal, s) : backward_launch<T, GATE, false>(a, equal, s);
}
template <typename T>
int backward_types(ScanBackward& a, bool equal, bool staged, cudaStream_t s)
{
    return a.o ? backward_gate<T, true>(a, equal, staged, s) : backward_gate<T, false>(a, equal, staged, s);
}

int64_t saved_stride(int64_t cols) { return (cols + 3) / 4 * 4; }

}  // namespace
}  // namespace ops
}  // namespace hpsgd

using namespace hpsgd;
using namespace hpsgd::ops;

extern "C" {

size_t hpsgd_gated_scan_saved_bytes(int64_t rows, int64_t cols)
{
    if (rows <= 0 || cols <= 0 || rows > kMostRows || cols > kMostCols) return 0;
    return (size_t)((rows + kSaved - 1) / kSaved) * (size_t)saved_stride(cols) * sizeof(float);
}

int hpsgd_gated_scan_forward(const hpsgd_gated_scan_forward_args* args, void* stream)
{
    const char* what = "hpsgd_gated_scan_forward";
    if (!args) return report(HPSGD_E_BADARG, "%s: args is NULL", what);
    hpsgd_gated_scan_forward_args p = *args;
    OPS_TRY(check_sequences(what, p.rows, p.cols, p.sequences, p.dtype, p.offsets));
    if (p.cols == 0 || p.sequences == 0) return HPSGD_OK;
    const int64_t esz = p.dtype == HPSGD_F32 ? 4 : 2;
    if (p.rows > 0 && (!p.f || !p.v || !p.y)) return report(HPSGD_E_BADARG, "%s: f, v or y is NULL", what);
    bool staged = true, wide = true;                // rows of the inputs on 16 bytes; two elements of everything at once
    OPS_TRY(check_rows(what, "f", p.f, &p.ldf, p.cols, esz, 16, &staged));
    OPS_TRY(check_rows(what, "v", p.v, &p.ldv, p.cols, esz, 16, &staged));
    OPS_TRY(check_rows(what, "o", p.o, &p.ldo, p.cols, esz, 16, &staged));
    OPS_TRY(check_rows(what, "f", p.f, &p.ldf, p.cols, esz, 2 * esz, &wide));
    OPS_TRY(check_rows(what, "v", p.v, &p.ldv, p.cols, esz, 2 * esz, &wide));
    OPS_TRY(check_rows(what, "o", p.o, &p.ldo, p.cols, esz, 2 * esz, &wide));
    OPS_TRY(check_rows(what, "y", p.y, &p.ldy, p.cols, esz, 2 * esz, &wide));
    OPS_TRY(check_rows(what, "h0", p.h0, &p.ldh0, p.cols, 4, 4, nullptr));
    OPS_TRY(check_rows(what, "h_last", p.h_last, &p.ldlast, p.cols, 4, 4, nullptr));
    staged = staged && wide;
    if (!aligned(p.saved, 16)) return report(HPSGD_E_BADARG, "%s: saved is not 16-byte aligned", what);
    if (p.h0 && p.h0 == p.h_last && p.ldh0 != p.ldlast) return report(HPSGD_E_BADARG, "%s: h0 and h_last are the same memory with different strides", what);
    if (p.rows == 0 && !p.h_last) return HPSGD_OK;
    int sms = 0;
    OPS_TRY(device_sms(&sms));
    ScanForward a{};
    a.q = Sequences{(int)p.rows, (int)p.cols, (int)p.sequences, (int)(p.rows / p.sequences), 1, 0, p.offsets};
    a.f = p.f; a.v = p.v; a.o = p.o; a.h0 = p.h0; a.h_last = p.h_last; a.y = p.y; a.saved = p.saved;
    a.ldf = p.ldf; a.ldv = p.ldv; a.ldo = p.ldo; a.ldy = p.ldy; a.ldh0 = p.ldh0; a.ldlast = p.ldlast; a.ldsaved = saved_stride(p.cols);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool equal = !p.offsets;
    return p.dtype == HPSGD_F32 ? forward_types<float>(a, equal, staged, wide, s) : forward_types<__nv_bfloat16>(a, equal, staged, wide, s);
}

int hpsgd_gated_scan_backward(const hpsgd_gated_scan_backward_args* args, void* stream)
{
    const char* what = "hpsgd_gated_scan_backward";
    if (!args) return report(HPSGD_E_BADARG, "%s: args is NULL", what);
    hpsgd_gated_scan_backward_args p = *args;
    OPS_TRY(check_sequences(what, p.rows, p.cols, p.sequences, p.dtype, p.offsets));
    if (p.cols == 0 || p.sequences == 0) return HPSGD_OK;
    const int64_t esz = p.dtype == HPSGD_F32 ? 4 : 2;
    if (p.rows > 0 && (!p.f || !p.v || !p.saved || !p.dy || !p.df || !p.dv)) return report(HPSGD_E_BADARG, "%s: f, v, saved, dy, df or dv is NULL", what);
    if (!p.o != !p.d_o) return report(HPSGD_E_BADARG, "%s: o and its gradient go together", what);
    bool staged = true;                             // rows of the inputs on 16 bytes, of the results on two elements
    OPS_TRY(check_rows(what, "f", p.f, &p.ldf, p.cols, esz, 16, &staged));
    OPS_TRY(check_rows(what, "v", p.v, &p.ldv, p.cols, esz, 16, &staged));
    OPS_TRY(check_rows(what, "o", p.o, &p.ldo, p.cols, esz, 16, &staged));
    OPS_TRY(check_rows(what, "dy", p.dy, &p.lddy, p.cols, esz, 16, &staged));
    OPS_TRY(check_rows(what, "df", p.df, &p.lddf, p.cols, esz, 2 * esz, &staged));
    OPS_TRY(check_rows(what, "dv", p.dv, &p.lddv, p.cols, esz, 2 * esz, &staged));
    OPS_TRY(check_rows(what, "do", p.d_o, &p.lddo, p.cols, esz, 2 * esz, &staged));
    OPS_TRY(check_rows(what, "h0", p.h0, &p.ldh0, p.cols, 4, 4, nullptr));
    OPS_TRY(check_rows(what, "dh_last", p.dh_last, &p.lddlast, p.cols, 4, 4, nullptr));
    OPS_TRY(check_rows(what, "dh0", p.dh0, &p.lddh0, p.cols, 4, 4, nullptr));
    if (!aligned(p.saved, 16)) return report(HPSGD_E_BADARG, "%s: saved is not 16-byte aligned", what);
    if (p.rows == 0 && !p.dh0) return HPSGD_OK;
    int sms = 0;
    OPS_TRY(device_sms(&sms));
    ScanBackward a{};
    a.q = Sequences{(int)p.rows, (int)p.cols, (int)p.sequences, (int)(p.rows / p.sequences), 1, 0, p.offsets};
    a.f = p.f; a.v = p.v; a.o = p.o; a.h0 = p.h0; a.saved = p.saved; a.dy = p.dy; a.dh_last = p.dh_last;
    a.df = p.df; a.dv = p.dv; a.d_o = p.d_o; a.dh0 = p.dh0;
    a.ldf = p.ldf; a.ldv = p.ldv; a.ldo = p.ldo; a.ldh0 = p.ldh0; a.lddy = p.lddy; a.lddlast = p.lddlast;
    a.lddf = p.lddf; a.lddv = p.lddv; a.lddo = p.lddo; a.lddh0 = p.lddh0; a.ldsaved = saved_stride(p.cols);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool equal = !p.offsets;
    return p.dtype == HPSGD_F32 ? backward_types<float>(a, equal, staged, s) : backward_types<__nv_bfloat16>(a, equal, staged, s);
}

}  // extern "C"
