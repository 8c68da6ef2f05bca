// Rows of the states of beams in the order of the beams that have been chosen (kan_net.h).
//
// A copy, bound by HBM: each row that moves is written once, the row in whose place it comes is read.  In place the rows of a search can
// change places with one another, so whoever writes a byte of one of them has to have read that byte of all: a thread has one piece of 16
// bytes (8 for more than 16 rows, 4 for more than 32) of every row of a search, reads it from the parents' rows, and writes it then.  Pieces of different threads do not overlap, a run's
// last bytes are read and written as they are, hence no wait between threads, no buffer, and no order of the rows to find.  Rows that
// stay are left out.  A launch takes up to kMost tensors from its arguments.  What is written goes past the caches (24 x 6 rows of 117 x 771 bf16 into other buffers 68 us,
// 75 through them; of 117 x 768, six rows read, 56 and 82).  Measured: caches of 4 x 8 rows of 8 heads, 2000 of 2304 x 128 bf16, 16 of them, 2.1 GB to move, 355 us (5.9 TB/s); the
// 24 x 6 x 117 x 771 above, 312 MB, 56 on the same states again and 66 on others (4.7 TB/s: rows that start anywhere in a line).
#include <algorithm>
#include "net_device.hpp"

namespace kannet {
namespace {

constexpr int kMost = 32;               // tensors of a launch
constexpr int kThreads = 256;
constexpr int64_t kBlocks = 1 << 23;    // of a launch

struct State {
    const char *data;                   // the first search's
    char *out;
    int64_t stride[3], out_stride[3];
    uint32_t blocks;                    // of a search
    uint32_t items, inner, pieces;      // outer * inner * pieces a run
    uint32_t whole, tail;               // pieces of a run that are whole, and bytes behind them
    bool place;
};

struct ReorderCall {
    State state[kMost];
    uint32_t first[kMost + 1];          // workgroups of the tensors before
    int64_t search[kMost];              // the first one
    const int64_t *parents;
    int n, B, top;
};
static_assert(sizeof(ReorderCall) <= 4096, "kernel arguments");

typedef uint16_t u16_a1 __attribute__((aligned(1)));
typedef uint32_t u32_a1 __attribute__((aligned(1)));
typedef u32x2 u32x2_a1 __attribute__((aligned(1)));
typedef u32x4 u32x4_a1 __attribute__((aligned(1)));

// Rows that move, into[k] <- from[k], k < count <= K; the same for the whole workgroup.  Behind the last one everybody reads the same few bytes, which are
// not written (loads under a condition cost the registers of five of each).
template <int K>
struct Moves {
    int from[K], into[K], count;
};

template <int K>
__device__ __forceinline__ Moves<K> moves_of(int source)
{
    Moves<K> m;
    uint64_t open = __ballot(source >= 0);
    m.count = __popcll(open);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        m.into[k] = open ? __ffsll((unsigned long long)open) - 1 : 0;
        m.from[k] = __builtin_amdgcn_readlane(source, m.into[k]);
        open &= open - 1;
    }
    return m;
}

template <int K, bool STREAM, class P>
__device__ __forceinline__ void move(const Moves<K> &m, const char *idle, const char *from, int64_t stride, char *to, int64_t out_stride)
{
    typedef const P *From;
    typedef P *To;
    P v[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const From p = (From)(k < m.count ? from + m.from[k] * stride : idle);
        if constexpr (STREAM) v[k] = __builtin_nontemporal_load(p);
        else v[k] = *p;
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (k < m.count) __builtin_nontemporal_store(v[k], (To)(to + m.into[k] * out_stride));
}

template <int K, bool STREAM, class P>
__device__ __forceinline__ void move_item(const State &s, const ReorderCall &a, int64_t search, uint32_t item, int source)
{
    const Moves<K> m = moves_of<K>(source);
    if (item >= s.items) return;
    const uint32_t piece = item % s.pieces, run = item / s.pieces, in = run % s.inner, block = run / s.inner;
    const char *from = s.data + search * a.B * s.stride[1] + block * s.stride[0] + in * s.stride[2] + (int64_t)piece * (int)sizeof(P);
    char *to = s.out + search * a.top * s.out_stride[1] + block * s.out_stride[0] + in * s.out_stride[2] + (int64_t)piece * (int)sizeof(P);
    if (piece < s.whole) {
        move<K, STREAM, P>(m, s.data, from, s.stride[1], to, s.out_stride[1]);
        return;
    }
    // a run's last bytes
    if (sizeof(P) > 8 && (s.tail & 8)) {
        move<K, STREAM, u32x2_a1>(m, s.data, from, s.stride[1], to, s.out_stride[1]);
        from += 8, to += 8;
    }
    if (sizeof(P) > 4 && (s.tail & 4)) {
        move<K, STREAM, u32_a1>(m, s.data, from, s.stride[1], to, s.out_stride[1]);
        from += 4, to += 4;
    }
    if (s.tail & 2) {
        move<K, STREAM, u16_a1>(m, s.data, from, s.stride[1], to, s.out_stride[1]);
        from += 2, to += 2;
    }
    if (s.tail & 1) move<K, STREAM, uint8_t>(m, s.data, from, s.stride[1], to, s.out_stride[1]);
}

// MOST: rows of a search; P: a piece; STREAM: states that the caches do not hold anyway
template <int MOST, bool STREAM, class P>
__global__ __launch_bounds__(kThreads) void reorder_kernel(ReorderCall a)
{
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const State &s = a.state[lo];
    const uint32_t here = blockIdx.x - a.first[lo];
    const int64_t search = here / s.blocks;
    const int lane = threadIdx.x & 63;
    int source = -1;
    if (lane < a.top) {
        const int64_t p = a.parents[(a.search[lo] + search) * a.top + lane];
        if (p >= 0 && p < a.B && !(s.place && p == lane)) source = (int)p;
    }
    const int count = __popcll(__ballot(source >= 0));
    const uint32_t item = here % s.blocks * kThreads + threadIdx.x;
    if (count == 0) return;
    if (count == 1) move_item<1, STREAM, P>(s, a, search, item, source);
    else if (count <= 4) move_item<4, STREAM, P>(s, a, search, item, source);
    else if (MOST <= 8 || count <= 8) move_item<8, STREAM, P>(s, a, search, item, source);
    else if (MOST <= 16 || count <= 16) move_item<(MOST < 16 ? MOST : 16), STREAM, P>(s, a, search, item, source);
    else if (MOST <= 32 || count <= 32) move_item<(MOST < 32 ? MOST : 32), STREAM, P>(s, a, search, item, source);
    else move_item<MOST, STREAM, P>(s, a, search, item, source);
}

// whether no two runs overlap
bool apart(const int64_t (&count)[3], const int64_t (&stride)[3], int64_t bytes)
{
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (stride[order[j]] > stride[order[j + 1]]) {
                const int t = order[j];
                order[j] = order[j + 1];
                order[j + 1] = t;
            }
    __int128 extent = bytes;
    for (int i : order) {
        if (count[i] <= 1) continue;
        if (stride[i] < extent) return false;
        extent += (__int128)stride[i] * (count[i] - 1);
    }
    return true;
}

int piece_of(int top) { return top <= 16 ? 16 : top <= 32 ? 8 : 4; }

int64_t pieces_of(const kan_state_ref &t, int piece) { return t.bytes / piece + (t.bytes % piece ? 1 : 0); }

// What an entry reads or writes: runs of `bytes` bytes, `count` of them `stride` apart in each dimension, from the lowest address on
struct Region {
    uint64_t first, last;               // bytes from the first one to behind the last one
    int64_t count[3], stride[3], bytes;
};

// false: no memory is like that
bool region_of(const void *at, const int64_t (&count)[3], const int64_t (&stride)[3], int64_t bytes, Region &r)
{
    __int128 first = (uintptr_t)at, extent = bytes;
    for (int d = 0; d < 3; ++d) {
        const int64_t n = stride[d] ? count[d] : 1;     // rows that are one and the same
        r.count[d] = n;
        r.stride[d] = n > 1 ? stride[d] : 0;
        const __int128 reach = (__int128)r.stride[d] * (n - 1);
        if (reach <= -((__int128)1 << 62)) return false;
        if (reach < 0) {
            first += reach;
            r.stride[d] = -r.stride[d];
        }
        extent += reach < 0 ? -reach : reach;
    }
    r.bytes = bytes;
    if (first < 0 || extent >= (__int128)1 << 62 || first + extent > (__int128)UINT64_MAX) return false;
    r.first = (uint64_t)first;
    r.last = (uint64_t)(first + extent);
    return true;
}

// Whether two regions have a byte in common: a run of one and a run of the other begin at a distance from -bytes to +bytes of one another.  The distances are sums of multiples of the strides, one
// range of factors for each different stride; for the largest one only the factors are looked at that the others can make up for, and so on.  Strides that lie within one another, as those of
// views of one buffer do, leave one or two factors each.  `left` bounds what is tried; -1: it did not do.
struct Steps {
    int n;
    int64_t stride[6], lo[6], hi[6];    // largest stride first
    int64_t least[7], most[7];          // what the strides from here on can make
};

int reaches(const Steps &s, int d, int64_t least, int64_t most, int &left)
{
    if (d == s.n) return least <= 0 && most >= 0;
    const int64_t stride = s.stride[d], from = least - s.most[d + 1], to = most - s.least[d + 1];
    const int64_t lo = std::max(s.lo[d], from / stride + (from % stride > 0)), hi = std::min(s.hi[d], to / stride - (to % stride < 0));
    for (int64_t k = lo; k <= hi; ++k) {
        if (--left < 0) return -1;
        const int found = reaches(s, d + 1, least - k * stride, most - k * stride, left);
        if (found) return found;
    }
    return 0;
}

int meet(const Region &a, const Region &b)
{
    Steps s;
    s.n = 0;
    const auto add = [&](int64_t stride, int64_t lo, int64_t hi) {
        if (!stride) return;
        int at = 0;
        while (at < s.n && s.stride[at] > stride) ++at;
        if (at == s.n || s.stride[at] != stride) {
            for (int k = s.n++; k > at; --k) s.stride[k] = s.stride[k - 1], s.lo[k] = s.lo[k - 1], s.hi[k] = s.hi[k - 1];
            s.stride[at] = stride, s.lo[at] = s.hi[at] = 0;
        }
        s.lo[at] += lo, s.hi[at] += hi;
    };
    for (int d = 0; d < 3; ++d) {
        add(a.stride[d], 0, a.count[d] - 1);
        add(b.stride[d], 1 - b.count[d], 0);
    }
    s.least[s.n] = s.most[s.n] = 0;
    for (int d = s.n; d-- > 0;) s.least[d] = s.least[d + 1] + s.lo[d] * s.stride[d], s.most[d] = s.most[d + 1] + s.hi[d] * s.stride[d];
    int left = 1 << 16;
    const int64_t apart = (int64_t)(b.first - a.first);
    return reaches(s, 0, apart - a.bytes + 1, apart + b.bytes - 1, left);
}

// Whether anything that is written lies where something else is read or written: in the order of their first bytes, each against those that begin before it ends.  kTogether entries at a
// time, and two times as many for the pairs among them, so that nothing is allocated.
constexpr int kTogether = 128;

struct Part {
    Region region;
    int entry;
    bool written;
};

bool empty(const kan_state_ref &t) { return t.outer == 0 || t.inner == 0 || t.bytes == 0; }

int overlaps(int64_t N, int32_t B, int32_t top, int32_t n, const kan_state_ref *list)
{
    Part part[4 * kTogether];
    uint16_t order[4 * kTogether];
    for (int one = 0; one < n; one += kTogether)
        for (int other = one; other < n; other += kTogether) {
            int m = 0;
            const auto gather = [&](int first) {
                for (int i = first; i < n && i < first + kTogether; ++i) {
                    const kan_state_ref &t = list[i];
                    if (empty(t)) continue;
                    const int64_t rows[3] = {t.outer, N * top, t.inner}, from[3] = {t.outer, N * B, t.inner};
                    part[m].entry = i;
                    part[m].written = true;
                    if (!region_of(t.out, rows, t.out_stride, t.bytes, part[m++].region)) return false;
                    if (t.data == t.out) continue;      // in place
                    part[m].entry = i;
                    part[m].written = false;
                    if (!region_of(t.data, from, t.stride, t.bytes, part[m++].region)) return false;
                }
                return true;
            };
            if (!gather(one) || (other != one && !gather(other))) return KAN_ERR_INVALID_ARG;
            for (int i = 0; i < m; ++i) order[i] = (uint16_t)i;
            std::sort(order, order + m, [&](uint16_t a, uint16_t b) { return part[a].region.first < part[b].region.first; });
            for (int i = 0; i < m; ++i)
                for (int k = i + 1; k < m && part[order[k]].region.first < part[order[i]].region.last; ++k) {
                    const Part &a = part[order[i]], &b = part[order[k]];
                    if ((!a.written && !b.written) || (other != one && a.entry / kTogether == b.entry / kTogether)) continue;
                    const int found = meet(a.region, b.region);
                    if (found) return found < 0 ? KAN_ERR_UNSUPPORTED : KAN_ERR_INVALID_ARG;
                }
        }
    return KAN_OK;
}

int check(int64_t N, int32_t B, int32_t top, const int64_t *parents, int32_t n, const kan_state_ref *list)
{
    if (N < 0 || B < 1 || top < 1 || n < 0 || (n > 0 && !list)) return KAN_ERR_INVALID_ARG;
    if (B > KAN_BEAM_MAX || top > KAN_BEAM_MAX || N >= (1ll << 31) / KAN_BEAM_MAX) return KAN_ERR_UNSUPPORTED;
    for (int i = 0; i < n; ++i) {
        const kan_state_ref &t = list[i];
        if (t.outer < 0 || t.inner < 0 || t.bytes < 0) return KAN_ERR_INVALID_ARG;
        if (empty(t) || N == 0) continue;
        if (!t.data || !t.out) return KAN_ERR_INVALID_ARG;
        const int64_t rows[3] = {t.outer, N * top, t.inner};
        if (!apart(rows, t.out_stride, t.bytes)) return KAN_ERR_INVALID_ARG;
        // the parents are read while rows are written
        Region out;
        if (!region_of(t.out, rows, t.out_stride, t.bytes, out)) return KAN_ERR_INVALID_ARG;
        const uint64_t order = (uintptr_t)parents;
        if (parents && order < out.last && out.first < order + (uint64_t)N * top * 8) return KAN_ERR_INVALID_ARG;
        if (t.data == t.out) {
            if (top != B) return KAN_ERR_INVALID_ARG;
            for (int d = 0; d < 3; ++d)
                if (rows[d] > 1 && t.stride[d] != t.out_stride[d]) return KAN_ERR_INVALID_ARG;
        }
        if ((__int128)t.outer * t.inner * pieces_of(t, piece_of(top > B ? top : B)) >= (1ll << 31)) return KAN_ERR_UNSUPPORTED;
    }
    return N == 0 ? KAN_OK : overlaps(N, B, top, n, list);
}

template <bool STREAM>
void launch_kernel(const ReorderCall &a, unsigned grid, hipStream_t st)
{
    if (a.top <= 8) reorder_kernel<8, STREAM, u32x4_a1><<<grid, kThreads, 0, st>>>(a);
    else if (a.top <= 16) reorder_kernel<16, STREAM, u32x4_a1><<<grid, kThreads, 0, st>>>(a);
    else if (a.top <= 32) reorder_kernel<32, STREAM, u32x2_a1><<<grid, kThreads, 0, st>>>(a);
    else reorder_kernel<64, STREAM, u32_a1><<<grid, kThreads, 0, st>>>(a);
}

hipError_t launch(const ReorderCall &a, bool past, hipStream_t st)
{
    prof::Timed timed("beam_reorder", st);
    if (past) launch_kernel<true>(a, a.first[a.n], st);
    else launch_kernel<false>(a, a.first[a.n], st);
    return hipGetLastError();
}

}  // namespace
}  // namespace kannet

using namespace kannet;

extern "C" int kan_beam_reorder(int64_t N, int32_t B, int32_t top, const int64_t *parents, int32_t n, const kan_state_ref *list, void *stream)
{
    const int rc = check(N, B, top, parents, n, list);
    if (rc != KAN_OK) return rc;
    if (N == 0 || n == 0) return KAN_OK;
    if (!parents || misplaced8(parents)) return KAN_ERR_INVALID_ARG;
    const int piece = piece_of(top);
    double bytes = 0.0;
    for (int i = 0; i < n; ++i) bytes += (double)list[i].outer * (double)list[i].inner * (double)list[i].bytes * (double)N * B;
    const bool past = bytes >= kLastCache;
    ReorderCall a = {};
    a.parents = parents;
    a.B = B;
    a.top = top;
    const auto flush = [&]() {
        const hipError_t e = a.n ? launch(a, past, (hipStream_t)stream) : hipSuccess;
        a.n = 0;
        return e;
    };
    for (int i = 0; i < n; ++i) {
        const kan_state_ref &t = list[i];
        if (t.outer == 0 || t.inner == 0 || t.bytes == 0) continue;
        State s = {};
        for (int d = 0; d < 3; ++d) s.stride[d] = t.stride[d], s.out_stride[d] = t.out_stride[d];
        s.inner = (uint32_t)t.inner;
        s.pieces = (uint32_t)pieces_of(t, piece);
        s.whole = (uint32_t)(t.bytes / piece);
        s.tail = (uint32_t)(t.bytes % piece);
        s.items = (uint32_t)(t.outer * t.inner) * s.pieces;
        s.blocks = div_up(s.items, (uint32_t)kThreads);
        s.place = t.data == t.out;
        const int64_t most = kBlocks / s.blocks;
        for (int64_t search = 0; search < N; search += most) {
            const int64_t here = N - search < most ? N - search : most;
            if ((a.n == kMost || (a.n && a.first[a.n] + here * s.blocks > kBlocks)) && flush() != hipSuccess) return KAN_ERR_HIP;
            s.data = (const char *)t.data + search * B * t.stride[1];
            s.out = (char *)t.out + search * top * t.out_stride[1];
            a.state[a.n] = s;
            a.search[a.n] = search;
            a.first[a.n + 1] = a.first[a.n] + (uint32_t)(here * s.blocks);
            ++a.n;
        }
    }
    return status_of(flush());
}
