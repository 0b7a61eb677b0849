// A gated linear recurrence over sequences, and its gradients.
//
// Per channel h_t = a_t h_(t-1) + (1 - a_t) v_t with a = sigmoid(f): an affine map of the state, and maps compose, so rows need not be gone through
// one by one: (A, H) then (A', H') is (A' A, A' H + H').  A thread takes two neighbouring channels over a group of consecutive rows, whose
// values it holds in registers: it composes its rows' maps, the groups' maps are exchanged, and with the state that reaches its first row it
// goes through its rows again.  So everything is read once and written once.  A block's warps have consecutive groups, the blocks of a cluster
// consecutive pieces of a chunk of rows, and chunks follow one another.  Sequences need no division of work of their own: the rows are one
// long sequence, in which a map that forgets stands where one begins.
//
// The gradient runs the other way with the same maps: what reaches h_(t-1) is M_t = a_t (g_t + M_(t+1)).  It needs h, which is computed
// again from the state that the forward pass keeps for each eight rows.
#include "hpsgd_ops_common.cuh"

#include <algorithm>

namespace hpsgd {
namespace ops {
namespace {

constexpr int kLanes = 32, kSlab = 2 * kLanes;      // channels of a block
constexpr int kWarps = 8, kScanThreads = 32 * kWarps;
constexpr int kRowsF = 16, kRowsB = 8;              // rows of a thread, forward and backward
constexpr int kSaved = 8;                           // rows that share a kept state
constexpr int kMaxCluster = 8;

struct Sequences {
    int rows, cols, count, each;                    // each: rows of a sequence where there are no offsets
    int walkers;
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
        const auto border = [&](int w) { return (int)((int64_t)q.rows * w / q.walkers); };
        first = walker == 0 ? 0 : q.at_or_behind(border(walker));
        last = walker + 1 == q.walkers ? q.count : q.at_or_behind(border(walker + 1));
        last = max(first, last);
        row0 = first < last ? q.begin(first) : 0;
        row1 = first < last ? max(row0, q.begin(last)) : 0;
    }
};

// Where sequences begin and end among the rows [r0, r0 + R) of a warp: a bit for each row, and which sequence it is.
struct Marks {
    uint32_t begins, ends;
};
template <int R>
__device__ __forceinline__ Marks find_marks(const Sequences& q, int r0, int (*which)[32])
{
    Marks m{0u, 0u};
    const int lane = threadIdx.x & 31;
    __syncwarp();
    for (int k = max(0, q.at_or_behind(r0) - 1);; k += 32) {
        const int i = k + lane, b = i < q.count ? q.begin(i) : 0x7FFFFFFF, e = i < q.count ? q.begin(i + 1) : 0;
        if (b < e) {
            if (b >= r0 && b < r0 + R) m.begins |= 1u << (b - r0), which[0][b - r0] = i;
            if (e > r0 && e <= r0 + R) m.ends |= 1u << (e - 1 - r0), which[1][e - 1 - r0] = i;
        }
        if (!__all_sync(0xFFFFFFFFu, i < q.count && b < r0 + R)) break;
    }
    m.begins = __reduce_or_sync(0xFFFFFFFFu, m.begins);
    m.ends = __reduce_or_sync(0xFFFFFFFFu, m.ends);
    __syncwarp();
    return m;
}

// ---------------------------------------------------------------------------- two channels
// As they are stored.  WIDE: both in one access; else one by one, `left` of them there.
template <typename T, bool WIDE>
struct Two;
template <bool WIDE>
struct Two<float, WIDE> {
    float2 x;
    __device__ __forceinline__ void load(const float* p, int left)
    {
        if (WIDE) x = left > 0 ? *reinterpret_cast<const float2*>(p) : make_float2(0.f, 0.f);
        else x = make_float2(left > 0 ? p[0] : 0.f, left > 1 ? p[1] : 0.f);
    }
    __device__ __forceinline__ pair values() const { return make_pair(x.x, x.y); }
};
template <bool WIDE>
struct Two<__nv_bfloat16, WIDE> {
    uint32_t x;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int left)
    {
        const unsigned short* const h = reinterpret_cast<const unsigned short*>(p);
        if (WIDE) x = left > 0 ? *reinterpret_cast<const uint32_t*>(p) : 0u;
        else x = (left > 0 ? (uint32_t)h[0] : 0u) | (left > 1 ? (uint32_t)h[1] << 16 : 0u);
    }
    __device__ __forceinline__ pair values() const
    {
        float lo, hi;
        widen_pair(x, lo, hi);
        return make_pair(lo, hi);
    }
};
template <bool WIDE>
__device__ __forceinline__ void store_two(float* p, pair v, int left)
{
    float lo, hi;
    split(v, lo, hi);
    if (WIDE) {
        if (left > 0) *reinterpret_cast<float2*>(p) = make_float2(lo, hi);
    } else {
        if (left > 0) p[0] = lo;
        if (left > 1) p[1] = hi;
    }
}
template <bool WIDE>
__device__ __forceinline__ void store_two(__nv_bfloat16* p, pair v, int left)
{
    float lo, hi;
    split(v, lo, hi);
    if (WIDE) {
        if (left > 0) *reinterpret_cast<uint32_t*>(p) = pack_bf16(lo, hi);
    } else {
        if (left > 0) p[0] = __float2bfloat16_rn(lo);
        if (left > 1) p[1] = __float2bfloat16_rn(hi);
    }
}

// s = sigmoid(x) and 1 - s, each to a few units of its own last place: e = 2^(-x log2 e), s = 1 / (1 + e), 1 - s = e s.  e is held to 2^126, so that s
// is not 0 where e s has to be 1; a NaN stays one.
__device__ __forceinline__ void sigmoid(pair x, pair& s, pair& rest)
{
    float lo, hi;
    split(x, lo, hi);
    lo = __fmul_rn(lo, -kLog2e), hi = __fmul_rn(hi, -kLog2e);
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
    split(x, lo, hi);
    float d0, d1;
    split(add2(make_pair(exp2_of(__fmul_rn(lo, -kLog2e)), exp2_of(__fmul_rn(hi, -kLog2e))), both(1.f)), d0, d1);
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

// What the groups' maps are exchanged through; two of each in turn, so that one barrier a chunk is enough.
struct Exchange {
    ulonglong2 group[2][kWarps][kLanes];            // of this block's warps
    ulonglong2 block[2][kMaxCluster][kLanes];       // of the cluster's blocks
};

// The state that reaches this thread's group, given the state in front of the chunk (`carry`, which becomes the one behind it).  `warp` and
// `rank` count in the direction of the recurrence.  All threads of the cluster come here.
template <bool CLUSTER>
__device__ __forceinline__ pair exchange(Exchange& x, int turn, const Map& mine, pair& carry, int warp, int rank, int blocks)
{
    const int lane = threadIdx.x & 31;
    x.group[turn][warp][lane] = make_ulonglong2(mine.A, mine.H);
    __syncthreads();
    const auto group = [&](int w) {
        const ulonglong2 m = x.group[turn][w][lane];
        return Map{m.x, m.y};
    };
    if constexpr (!CLUSTER) {
        pair h = carry, in = carry;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w == warp) in = h;
            h = group(w).of(h);
        }
        carry = h;
        return in;
    } else {
        if (warp == 0) {                            // the block's own map to all blocks
            Map all = group(0);
#pragma unroll
            for (int w = 1; w < kWarps; ++w) all = group(w).behind(all);
            for (int r = 0; r < blocks; ++r) map_to_block(&x.block[turn][rank][lane], r, all);
        }
        cluster_arrive();
        Map before = identity();
        for (int w = 0; w < warp; ++w) before = group(w).behind(before);
        cluster_wait();
        pair h = carry, in = carry;
        for (int r = 0; r < blocks; ++r) {
            if (r == rank) in = h;
            const ulonglong2 m = x.block[turn][r][lane];
            h = Map{m.x, m.y}.of(h);
        }
        carry = h;
        return before.of(in);
    }
}

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
    int64_t ldf, ldv, ldo, ldy, ldh0, ldlast;
};

__device__ __forceinline__ pair load_state(const float* p, int left) { return make_pair(left > 0 ? p[0] : 0.f, left > 1 ? p[1] : 0.f); }
__device__ __forceinline__ void store_state(float* p, pair h, int left)
{
    float lo, hi;
    split(h, lo, hi);
    if (left > 0) p[0] = lo;
    if (left > 1) p[1] = hi;
}

template <typename T, bool GATE, bool WIDE, bool CLUSTER>
__global__ void __launch_bounds__(kScanThreads) scan_forward_kernel(const ScanForward a)
{
    constexpr int R = kRowsF;
    __shared__ alignas(16) Exchange ex;
    __shared__ int which_of[kWarps][2][32];
    const Sequences& q = a.q;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = CLUSTER ? (int)(blockIdx.x % (unsigned)a.blocks) : 0, unit = CLUSTER ? (int)(blockIdx.x / (unsigned)a.blocks) : (int)blockIdx.x;
    const int slab = unit % a.slabs, c = slab * kSlab + lane * 2, left = min(2, q.cols - c);
    int(*const which)[32] = which_of[warp];
    after_previous();
    if constexpr (CLUSTER) cluster_arrive();        // the others' shared memory is there to be written; waited for below
    const Share mine(q, unit / a.slabs);
    // sequences without rows: their state goes through
    if (a.h_last && rank == 0)
        for (int s = mine.first + warp; s < mine.last; s += kWarps)
            if (q.begin(s) >= q.begin(s + 1)) store_state(a.h_last + s * a.ldlast + c, a.h0 ? load_state(a.h0 + s * a.ldh0 + c, left) : both(0.f), left);
    if constexpr (CLUSTER) cluster_wait();

    const T* const f = static_cast<const T*>(a.f) + c;
    const T* const v = static_cast<const T*>(a.v) + c;
    const T* const o = static_cast<const T*>(a.o) + c;
    T* const y = static_cast<T*>(a.y) + c;
    const int chunk = a.blocks * kWarps * R;
    pair carry = both(0.f);
    int turn = 0;
    for (int r = mine.row0 / R * R + (rank * kWarps + warp) * R, base = mine.row0 / R * R; base < mine.row1; base += chunk, r += chunk, turn ^= 1) {
        Two<T, WIDE> fx[R], vx[R], ox[R];
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const int here = r + t >= mine.row0 && r + t < mine.row1 ? left : 0;
            fx[t].load(f + (r + t) * a.ldf, here);
            vx[t].load(v + (r + t) * a.ldv, here);
            if (GATE) ox[t].load(o + (r + t) * a.ldo, here);
        }
        const Marks m = find_marks<R>(q, r, which);
        const uint32_t below = r >= mine.row0 ? 0u : r + R <= mine.row0 ? 0xFFFFu : (1u << (mine.row0 - r)) - 1u;
        const uint32_t in = 0xFFFFu & ~below & (r + R <= mine.row1 ? 0xFFFFu : r >= mine.row1 ? 0u : (1u << (mine.row1 - r)) - 1u);
        const uint32_t begins = m.begins & in, ends = m.ends & in;
        pair g[R], b[R];                            // the gates, and what they let in
        Map map = identity();
#pragma unroll
        for (int t = 0; t < R; ++t) {
            pair rest;
            sigmoid(fx[t].values(), g[t], rest);
            b[t] = mul2(rest, vx[t].values());
            if (!(in >> t & 1u)) g[t] = both(1.f), b[t] = both(0.f);
            if (begins >> t & 1u) {
                if (a.h0) b[t] = fma2(g[t], load_state(a.h0 + which[0][t] * a.ldh0 + c, left), b[t]);
                map.H = b[t];
                map.A = both(-1.f);
            } else {
                map.H = fma2(g[t], map.H, b[t]);
                float a0, a1;
                split(map.A, a0, a1);
                if (a0 != -1.f) map.A = mul2(map.A, g[t]);
            }
        }
        pair h = exchange<CLUSTER>(ex, turn, map, carry, warp, rank, a.blocks);
#pragma unroll
        for (int t = 0; t < R; ++t) {
            if (t % kSaved == 0 && a.saved && (in >> t & 1u)) store_state(a.saved + (int64_t)((r + t) / kSaved) * q.cols + c, h, left);
            h = begins >> t & 1u ? b[t] : fma2(g[t], h, b[t]);
            if (ends >> t & 1u)
                if (a.h_last) store_state(a.h_last + which[1][t] * a.ldlast + c, h, left);
            if (in >> t & 1u) store_two<WIDE>(y + (r + t) * a.ldy, GATE ? mul2(h, sigmoid(ox[t].values())) : h, left);
        }
    }
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
    int64_t ldf, ldv, ldo, ldh0, lddy, lddlast, lddf, lddv, lddo, lddh0;
};

template <typename T, bool GATE, bool WIDE, bool CLUSTER>
__global__ void __launch_bounds__(kScanThreads) scan_backward_kernel(const ScanBackward a)
{
    constexpr int R = kRowsB;
    __shared__ alignas(16) Exchange ex;
    __shared__ int which_of[kWarps][2][32];
    const Sequences& q = a.q;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = CLUSTER ? (int)(blockIdx.x % (unsigned)a.blocks) : 0, unit = CLUSTER ? (int)(blockIdx.x / (unsigned)a.blocks) : (int)blockIdx.x;
    const int slab = unit % a.slabs, c = slab * kSlab + lane * 2, left = min(2, q.cols - c);
    int(*const which)[32] = which_of[warp];
    after_previous();
    if constexpr (CLUSTER) cluster_arrive();
    const Share mine(q, unit / a.slabs);
    if (a.dh0 && rank == 0)
        for (int s = mine.first + warp; s < mine.last; s += kWarps)
            if (q.begin(s) >= q.begin(s + 1)) store_state(a.dh0 + s * a.lddh0 + c, a.dh_last ? load_state(a.dh_last + s * a.lddlast + c, left) : both(0.f), left);
    if constexpr (CLUSTER) cluster_wait();

    const T* const f = static_cast<const T*>(a.f) + c;
    const T* const v = static_cast<const T*>(a.v) + c;
    const T* const o = static_cast<const T*>(a.o) + c;
    const T* const dy = static_cast<const T*>(a.dy) + c;
    T* const df = static_cast<T*>(a.df) + c;
    T* const dv = static_cast<T*>(a.dv) + c;
    T* const d_o = static_cast<T*>(a.d_o) + c;
    const int chunk = a.blocks * kWarps * R;
    const int start = mine.row0 / R * R;
    pair carry = both(0.f);
    int turn = 0;
    // chunks from the last to the first; in a chunk as well the first warp of the first block has the last rows
    for (int k = (mine.row1 - start + chunk - 1) / chunk - 1; k >= 0; --k, turn ^= 1) {
        const int r = start + k * chunk + ((a.blocks - 1 - rank) * kWarps + (kWarps - 1 - warp)) * R;
        Two<T, WIDE> fx[R], vx[R], ox[R], dx[R];
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const int here = r + t >= mine.row0 && r + t < mine.row1 ? left : 0;
            fx[t].load(f + (r + t) * a.ldf, here);
            vx[t].load(v + (r + t) * a.ldv, here);
            dx[t].load(dy + (r + t) * a.lddy, here);
            if (GATE) ox[t].load(o + (r + t) * a.ldo, here);
        }
        pair h = r >= mine.row0 && r < mine.row1 ? load_state(a.saved + (int64_t)(r / kSaved) * q.cols + c, left) : both(0.f);
        const Marks m = find_marks<R>(q, r, which);
        const uint32_t below = r >= mine.row0 ? 0u : r + R <= mine.row0 ? 0xFFu : (1u << (mine.row0 - r)) - 1u;
        const uint32_t in = 0xFFu & ~below & (r + R <= mine.row1 ? 0xFFu : r >= mine.row1 ? 0u : (1u << (mine.row1 - r)) - 1u);
        const uint32_t begins = m.begins & in, ends = m.ends & in;
        pair g[R], rest[R], step[R], dh[R];         // a, 1 - a, h_(t-1) - v, the gradient that reaches h_t through y
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const pair vt = vx[t].values(), dt = dx[t].values();
            sigmoid(fx[t].values(), g[t], rest[t]);
            if (begins >> t & 1u) h = a.h0 ? load_state(a.h0 + which[0][t] * a.ldh0 + c, left) : both(0.f);
            step[t] = fma2(vt, both(-1.f), h);
            h = fma2(g[t], h, mul2(rest[t], vt));
            dh[t] = dt;
            if (GATE) {
                pair s, s1;
                sigmoid(ox[t].values(), s, s1);
                dh[t] = mul2(dt, s);
                if (in >> t & 1u) store_two<WIDE>(d_o + (r + t) * a.lddo, mul2(mul2(dh[t], h), s1), left);
            }
            if (ends >> t & 1u)
                if (a.dh_last) dh[t] = add2(dh[t], load_state(a.dh_last + which[1][t] * a.lddlast + c, left));
        }
        // M -> a (dh + M), rows from the last to the first; nothing comes into a sequence's last row
        Map map = identity();
#pragma unroll
        for (int t = R - 1; t >= 0; --t) {
            const pair gt = in >> t & 1u ? g[t] : both(1.f), x = in >> t & 1u ? mul2(g[t], dh[t]) : both(0.f);
            float a0, a1;
            split(map.A, a0, a1);
            if (ends >> t & 1u) map = Map{both(-1.f), x};
            else map = Map{a0 == -1.f ? map.A : mul2(map.A, gt), fma2(gt, map.H, x)};
        }
        pair M = exchange<CLUSTER>(ex, turn, map, carry, warp, rank, a.blocks);
#pragma unroll
        for (int t = R - 1; t >= 0; --t) {
            if (!(in >> t & 1u)) continue;
            const pair G = ends >> t & 1u ? dh[t] : add2(dh[t], M);
            const pair p = mul2(G, rest[t]);
            M = mul2(G, g[t]);
            store_two<WIDE>(dv + (r + t) * a.lddv, p, left);
            store_two<WIDE>(df + (r + t) * a.lddf, mul2(mul2(p, g[t]), step[t]), left);
            if (begins >> t & 1u)
                if (a.dh0) store_state(a.dh0 + which[0][t] * a.lddh0 + c, M, left);
        }
    }
}

// ---------------------------------------------------------------------------- host side
constexpr int64_t kMostRows = 0x7FFFFFFF - 65536;   // rows of a chunk that reaches past the end are counted too

int check_sequences(const char* what, int64_t rows, int64_t cols, int64_t sequences, int dtype, const int64_t* offsets)
{
    if (rows < 0 || cols < 0 || sequences < 0) return report(HPSGD_E_BADARG, "%s: a size is negative", what);
    if (dtype != HPSGD_F32 && dtype != HPSGD_BF16) return report(HPSGD_E_BADARG, "%s: unknown dtype %d", what, dtype);
    if (rows > kMostRows || cols > 0x7FFFFFFF - 64 || sequences > 0x7FFFFFFF - 64) return report(HPSGD_E_UNSUPPORTED, "%s: a size is too large", what);
    if (!offsets && sequences > 0 && rows % sequences) return report(HPSGD_E_BADARG, "%s: without offsets rows must be a multiple of sequences", what);
    if (!aligned(offsets, 8)) return report(HPSGD_E_BADARG, "%s: offsets is not 8-byte aligned", what);
    return HPSGD_OK;
}

// A matrix of `rows` rows of the call's columns: its stride, its alignment, and whether two channels can be taken at once.
int check_rows(const char* what, const char* name, const void* p, int64_t* ld, int64_t cols, int64_t esz, bool* wide)
{
    if (*ld == 0) *ld = cols;
    if (!p) return HPSGD_OK;
    if (*ld < cols) return report(HPSGD_E_BADARG, "%s: the stride of %s is below cols", what, name);
    if (!aligned(p, esz)) return report(HPSGD_E_BADARG, "%s: %s is not aligned to its elements", what, name);
    if (wide) *wide = *wide && aligned(p, 2 * esz) && *ld % 2 == 0;
    return HPSGD_OK;
}

struct Plan {
    int slabs, walkers, blocks;
};

Plan plan_of(int64_t rows, int64_t cols, int64_t sequences, int R)
{
    Plan p{};
    p.slabs = (int)((cols + kSlab - 1) / kSlab);
    p.walkers = p.blocks = 1;
    const int64_t want = 2 * 148, piece = kWarps * R;
    while ((int64_t)p.slabs * p.blocks * 2 <= want && p.blocks < kMaxCluster && rows > piece * p.blocks) p.blocks *= 2;
    while ((int64_t)p.slabs * p.blocks * p.walkers * 2 <= want && p.walkers * 2 <= sequences && rows > piece * p.blocks * p.walkers) p.walkers *= 2;
    return p;
}

template <typename Kernel, typename Args>
int launch_scan(const char* what, Kernel kernel, const Args& a, const Plan& p, cudaStream_t s)
{
    return launch_clusters(what, kernel, dim3((unsigned)(p.slabs * p.walkers * p.blocks)), kScanThreads, 0, p.blocks, s, a);
}

template <typename T, bool GATE, bool WIDE>
int forward_launch(const ScanForward& a, const Plan& p, cudaStream_t s)
{
    const char* what = "hpsgd_gated_scan_forward";
    return p.blocks > 1 ? launch_scan(what, scan_forward_kernel<T, GATE, WIDE, true>, a, p, s) : launch_scan(what, scan_forward_kernel<T, GATE, WIDE, false>, a, p, s);
}
template <typename T>
int forward_types(const ScanForward& a, const Plan& p, bool wide, cudaStream_t s)
{
    if (a.o) return wide ? forward_launch<T, true, true>(a, p, s) : forward_launch<T, true, false>(a, p, s);
    return wide ? forward_launch<T, false, true>(a, p, s) : forward_launch<T, false, false>(a, p, s);
}

template <typename T, bool GATE, bool WIDE>
int backward_launch(const ScanBackward& a, const Plan& p, cudaStream_t s)
{
    const char* what = "hpsgd_gated_scan_backward";
    return p.blocks > 1 ? launch_scan(what, scan_backward_kernel<T, GATE, WIDE, true>, a, p, s) : launch_scan(what, scan_backward_kernel<T, GATE, WIDE, false>, a, p, s);
}
template <typename T>
int backward_types(const ScanBackward& a, const Plan& p, bool wide, cudaStream_t s)
{
    if (a.o) return wide ? backward_launch<T, true, true>(a, p, s) : backward_launch<T, true, false>(a, p, s);
    return wide ? backward_launch<T, false, true>(a, p, s) : backward_launch<T, false, false>(a, p, s);
}

}  // namespace
}  // namespace ops
}  // namespace hpsgd

using namespace hpsgd;
using namespace hpsgd::ops;

extern "C" {

size_t hpsgd_gated_scan_saved_bytes(int64_t rows, int64_t cols)
{
    if (rows <= 0 || cols <= 0 || rows > kMostRows || cols > 0x7FFFFFFF - 64) return 0;
    return (size_t)((rows + kSaved - 1) / kSaved) * (size_t)cols * sizeof(float);
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
    bool wide = p.cols % 2 == 0;
    OPS_TRY(check_rows(what, "f", p.f, &p.ldf, p.cols, esz, &wide));
    OPS_TRY(check_rows(what, "v", p.v, &p.ldv, p.cols, esz, &wide));
    OPS_TRY(check_rows(what, "o", p.o, &p.ldo, p.cols, esz, &wide));
    OPS_TRY(check_rows(what, "y", p.y, &p.ldy, p.cols, esz, &wide));
    OPS_TRY(check_rows(what, "h0", p.h0, &p.ldh0, p.cols, 4, nullptr));
    OPS_TRY(check_rows(what, "h_last", p.h_last, &p.ldlast, p.cols, 4, nullptr));
    if (!aligned(p.saved, 4)) return report(HPSGD_E_BADARG, "%s: saved is not aligned to its elements", what);
    if (p.h0 && p.h0 == p.h_last && p.ldh0 != p.ldlast) return report(HPSGD_E_BADARG, "%s: h0 and h_last are the same memory with different strides", what);
    if (p.rows == 0 && !p.h_last) return HPSGD_OK;
    int sms = 0;
    OPS_TRY(device_sms(&sms));
    const Plan plan = plan_of(p.rows, p.cols, p.sequences, kRowsF);
    ScanForward a{};
    a.q = Sequences{(int)p.rows, (int)p.cols, (int)p.sequences, (int)(p.rows / p.sequences), plan.walkers, p.offsets};
    a.slabs = plan.slabs; a.blocks = plan.blocks;
    a.f = p.f; a.v = p.v; a.o = p.o; a.h0 = p.h0; a.h_last = p.h_last; a.y = p.y; a.saved = p.saved;
    a.ldf = p.ldf; a.ldv = p.ldv; a.ldo = p.ldo; a.ldy = p.ldy; a.ldh0 = p.ldh0; a.ldlast = p.ldlast;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return p.dtype == HPSGD_F32 ? forward_types<float>(a, plan, wide, s) : forward_types<__nv_bfloat16>(a, plan, wide, s);
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
    bool wide = p.cols % 2 == 0;
    OPS_TRY(check_rows(what, "f", p.f, &p.ldf, p.cols, esz, &wide));
    OPS_TRY(check_rows(what, "v", p.v, &p.ldv, p.cols, esz, &wide));
    OPS_TRY(check_rows(what, "o", p.o, &p.ldo, p.cols, esz, &wide));
    OPS_TRY(check_rows(what, "dy", p.dy, &p.lddy, p.cols, esz, &wide));
    OPS_TRY(check_rows(what, "df", p.df, &p.lddf, p.cols, esz, &wide));
    OPS_TRY(check_rows(what, "dv", p.dv, &p.lddv, p.cols, esz, &wide));
    OPS_TRY(check_rows(what, "do", p.d_o, &p.lddo, p.cols, esz, &wide));
    OPS_TRY(check_rows(what, "h0", p.h0, &p.ldh0, p.cols, 4, nullptr));
    OPS_TRY(check_rows(what, "dh_last", p.dh_last, &p.lddlast, p.cols, 4, nullptr));
    OPS_TRY(check_rows(what, "dh0", p.dh0, &p.lddh0, p.cols, 4, nullptr));
    if (!aligned(p.saved, 4)) return report(HPSGD_E_BADARG, "%s: saved is not aligned to its elements", what);
    if (p.rows == 0 && !p.dh0) return HPSGD_OK;
    int sms = 0;
    OPS_TRY(device_sms(&sms));
    const Plan plan = plan_of(p.rows, p.cols, p.sequences, kRowsB);
    ScanBackward a{};
    a.q = Sequences{(int)p.rows, (int)p.cols, (int)p.sequences, (int)(p.rows / p.sequences), plan.walkers, p.offsets};
    a.slabs = plan.slabs; a.blocks = plan.blocks;
    a.f = p.f; a.v = p.v; a.o = p.o; a.h0 = p.h0; a.saved = p.saved; a.dy = p.dy; a.dh_last = p.dh_last;
    a.df = p.df; a.dv = p.dv; a.d_o = p.d_o; a.dh0 = p.dh0;
    a.ldf = p.ldf; a.ldv = p.ldv; a.ldo = p.ldo; a.ldh0 = p.ldh0; a.lddy = p.lddy; a.lddlast = p.lddlast;
    a.lddf = p.lddf; a.lddv = p.lddv; a.lddo = p.lddo; a.lddh0 = p.lddh0;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return p.dtype == HPSGD_F32 ? backward_types<float>(a, plan, wide, s) : backward_types<__nv_bfloat16>(a, plan, wide, s);
}

}  // extern "C"
