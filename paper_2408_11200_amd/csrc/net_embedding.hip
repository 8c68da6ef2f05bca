// Embedding rows and their gradient (kan_net.h).
//
// Forward: a copy of rows, bound by HBM (by latency for a few tokens).
//
// Backward: tokens are sorted by id, stably (least significant digit first, up to ten bits a pass), and each table row adds up its run of the
// sorted list: no atomics on values, so a row's sum has one order, and rows without a token are written as zeros in the same pass, so the
// table's gradient is written once.  A run may hold a good part of the batch (frequent tokens): pieces of 32 sorted places that lie
// wholly within a run are summed beforehand by workgroups of their own, and pieces of 32 such pieces again, so that a run of N tokens
// takes at most about 62 rows, 62 sums of 32 and N / 1024 sums of 1024, from as many workgroups as there are pieces.
#include "net_device.hpp"

namespace kannet {
namespace {

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMaxDigit = 10;
constexpr int kMaxBlocks = 64;        // of a sort pass: every block reads all blocks' counts
constexpr int kPiece = 32;

template <class T, class Y>
__global__ __launch_bounds__(256) void embedding_rows_kernel(const int64_t *ids, const T *table, Y *y, int64_t T_, int64_t V, int n, int pieces, float scale)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, t = i / pieces;
    if (t >= T_) return;
    const int c = (int)(i - t * pieces) * 8;
    const int64_t id = ids[t];
    float v[8];
    if (id >= 0 && id < V) {
        load_at(table + id * n, c, n, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= scale;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 0.0f;
    }
    store_at(y + t * n, c, n, v);
}

// ---- the sort -------------------------------------------------------------------------------

struct SortPass {
    const int64_t *ids;                 // first pass: keys come from here (ids outside the table: V), places are 0, 1, 2, ...
    const uint32_t *key_in, *place_in;
    uint32_t *key_out, *place_out;
    uint32_t *counts;                   // [blocks][digits]
    int64_t V;
    uint32_t T, per_block;
    int blocks, shift, bits;
};

__device__ __forceinline__ uint32_t key_at(const SortPass &a, uint32_t i)
{
    if (!a.ids) return a.key_in[i];
    const int64_t id = a.ids[i];
    return id >= 0 && id < a.V ? (uint32_t)id : (uint32_t)a.V;
}

__global__ __launch_bounds__(kSortThreads) void embedding_count_kernel(SortPass a)
{
    __shared__ uint32_t count[1 << kMaxDigit];
    const uint32_t digits = 1u << a.bits;
    for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) count[d] = 0;
    __syncthreads();
    const uint32_t from = blockIdx.x * a.per_block, to = from + a.per_block < a.T ? from + a.per_block : a.T;
    for (uint32_t i = from + threadIdx.x; i < to; i += kSortThreads) atomicAdd(&count[key_at(a, i) >> a.shift & (digits - 1)], 1u);
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) a.counts[blockIdx.x * digits + d] = count[d];
}

__global__ __launch_bounds__(kSortThreads) void embedding_place_kernel(SortPass a)
{
    __shared__ uint32_t cursor[kSortWaves][1 << kMaxDigit];      // a wave's counts, then where its next entry of a digit goes
    __shared__ uint32_t wave_total[kSortWaves];
    const uint32_t digits = 1u << a.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (uint32_t d = threadIdx.x; d < kSortWaves * (1u << kMaxDigit); d += kSortThreads) (&cursor[0][0])[d] = 0;
    __syncthreads();
    // a wave has consecutive entries, so that waves in turn are the order of the list
    const uint32_t per_wave = a.per_block / kSortWaves;
    uint32_t from = blockIdx.x * a.per_block + wave * per_wave;
    const uint32_t to = from + per_wave < a.T ? from + per_wave : a.T;
    for (uint32_t i = from + lane; i < to; i += 64) atomicAdd(&cursor[wave][key_at(a, i) >> a.shift & (digits - 1)], 1u);
    // of each digit (one a thread): entries in all blocks, and in the blocks before this one
    uint32_t all = 0, before = 0;
    if (threadIdx.x < digits) {
        const uint32_t *column = a.counts + threadIdx.x;
#pragma unroll 8
        for (uint32_t b = 0; b < (uint32_t)a.blocks; ++b) {
            const uint32_t v = column[b * digits];
            all += v;
            before += b < blockIdx.x ? v : 0u;
        }
    }
    // entries of smaller digits: a running sum over the threads
    uint32_t sum = all;
    for (int step = 1; step < 64; step *= 2) {
        const uint32_t o = __shfl_up(sum, step, 64);
        if ((int)lane >= step) sum += o;
    }
    if (lane == 63) wave_total[wave] = sum;
    __syncthreads();
    uint32_t base = sum - all + before;
    for (uint32_t w = 0; w < wave; ++w) base += wave_total[w];
    if (threadIdx.x < digits)
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = cursor[w][threadIdx.x];
            cursor[w][threadIdx.x] = base;
            base += c;
        }
    __syncthreads();
    for (; from < to; from += 64) {
        const uint32_t i = from + lane;
        const bool in = i < to;
        const uint32_t key = in ? key_at(a, i) : 0u, digit = key >> a.shift & (digits - 1);
        // lanes with the same digit; the first of them moves the cursor on for all
        uint64_t same = __ballot(in);
        for (int b = 0; b < a.bits; ++b) {
            const bool bit = (digit >> b & 1u) != 0;
            const uint64_t set = __ballot(bit);
            same &= bit ? set : ~set;
        }
        const int first = __ffsll((unsigned long long)same) - 1;
        uint32_t at = 0;
        if (in && (int)lane == first) at = atomicAdd(&cursor[wave][digit], (uint32_t)__popcll(same));
        at = __shfl(at, first < 0 ? 0 : first, 64) + (uint32_t)__popcll(same & ((1ull << lane) - 1));
        if (in) {
            a.key_out[at] = key;
            a.place_out[at] = a.ids ? i : a.place_in[i];
        }
    }
}

// ---- sums -----------------------------------------------------------------------------------

// Adds eight channels of `count` rows to t, one after the other, as many of them in flight as fit the registers: the rows `first`, first + 1, ...
// of a table, or those that `places` names.
template <int AHEAD, class Y>
__device__ __forceinline__ void add_rows(const Y *rows, const uint32_t *places, uint32_t first, uint32_t count, int n, int c, float (&t)[8])
{
    uint32_t i = 0;
    for (; i + AHEAD <= count; i += AHEAD) {
        Raw<Y> r[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) r[k] = raw_at(rows + (int64_t)(places ? places[first + i + k] : first + i + k) * n, c, n);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            float v[8];
            settle(r[k], c, n);
            unpack(r[k], v);
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] += v[j];
        }
    }
    for (; i < count; ++i) {
        float v[8];
        load_at(rows + (int64_t)(places ? places[first + i] : first + i) * n, c, n, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] += v[j];
    }
}

// Pieces of 32 consecutive entries that have one id: of the sorted list (`places` names rows of gy), or of the pieces themselves (`step` = 32
// entries of the list each).  Narrow rows leave the workgroup several workers, which take a share of the 32 each.
template <class Y>
__global__ __launch_bounds__(256) void embedding_piece_kernel(const uint32_t *keys, const uint32_t *places, const Y *rows, float *sums, int64_t V, int n, int lanes,
                                                              int step)
{
    __shared__ float lds[256 * 8];
    const uint32_t p = blockIdx.x, width = kPiece * step;
    const uint32_t id = keys[p * width];
    if (id >= V || keys[(p + 1) * width - 1] != id) return;
    const int workers = 256 / lanes < kPiece ? 256 / lanes : kPiece, each = kPiece / workers;
    const int w = threadIdx.x / lanes, lane = threadIdx.x % lanes, c = (blockIdx.y * lanes + lane) * 8;
    float t[8] = {};
    if (w < workers) add_rows<8>(rows, places, p * kPiece + w * each, each, n, c, t);
    if (workers > 1) {
#pragma unroll
        for (int k = 0; k < 8; ++k) lds[k * 256 + threadIdx.x] = t[k];
        __syncthreads();
        if (w > 0) return;
        for (int o = 1; o < workers; ++o)
#pragma unroll
            for (int k = 0; k < 8; ++k) t[k] += lds[k * 256 + o * lanes + lane];
    }
    store_at(sums + (int64_t)p * n, c, n, t);
}

constexpr int kRows = 32;       // table rows of a workgroup

// the number of keys below `row` among `count` of them, by the whole workgroup: 256 samples at a time
__device__ __forceinline__ uint32_t keys_below(const uint32_t *keys, uint32_t count, int64_t row, uint32_t *lds)
{
    uint32_t from = 0;
    while (count > 0) {
        // a sample ends each of (up to) 256 equal stretches: those whose last key is below lie in front
        const uint32_t stretch = (count + 255) / 256, at = (threadIdx.x + 1) * stretch - 1;
        const bool below = at < count && (int64_t)keys[from + at] < row;
        const uint64_t votes = __ballot(below);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = (uint32_t)__popcll(votes);
        __syncthreads();
        const uint32_t skip = (lds[0] + lds[1] + lds[2] + lds[3]) * stretch;
        from += skip;
        count = count - skip < stretch - 1 ? count - skip : stretch - 1;
    }
    return from;
}

template <class Y, class G>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const uint32_t *keys, const uint32_t *places, const Y *gy, const float *sums, const float *sums2,
                                                            G *gtable, uint32_t T, int64_t V, int n, int lanes, float scale)
{
    __shared__ uint32_t start[kRows + 1], lds[4];
    const int64_t first = (int64_t)blockIdx.x * kRows;
    const uint32_t begin = keys_below(keys, T, first, lds), rest = keys_below(keys + begin, T - begin, first + kRows, lds);
    if (threadIdx.x <= kRows) {
        // the first sorted place whose id is not below this row
        const int64_t row = first + threadIdx.x;
        uint32_t lo = begin, hi = begin + rest;
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if ((int64_t)keys[mid] < row) lo = mid + 1;
            else hi = mid;
        }
        start[threadIdx.x] = lo;
    }
    __syncthreads();
    const int workers = 256 / lanes;
    for (int r = threadIdx.x / lanes; r < kRows && first + r < V; r += workers) {
        const uint32_t from = start[r], to = start[r + 1];
        // the run in whole pieces and what lies before and behind them, and these again in pieces of pieces
        uint32_t p0 = (from + kPiece - 1) / kPiece, p1 = to / kPiece;
        if (p1 <= p0) p0 = p1 = 0;
        uint32_t q0 = (p0 + kPiece - 1) / kPiece, q1 = p1 / kPiece;
        if (!sums2 || q1 <= q0) q0 = q1 = 0;
        for (int c = threadIdx.x % lanes * 8; c < n; c += lanes * 8) {
            float t[8] = {};
            if (p1 > 0) {
                add_rows<4>(gy, places, from, p0 * kPiece - from, n, c, t);
                if (q1 > 0) {
                    add_rows<4>(sums, nullptr, p0, q0 * kPiece - p0, n, c, t);
                    add_rows<4>(sums2, nullptr, q0, q1 - q0, n, c, t);
                    add_rows<4>(sums, nullptr, q1 * kPiece, p1 - q1 * kPiece, n, c, t);
                } else {
                    add_rows<4>(sums, nullptr, p0, p1 - p0, n, c, t);
                }
                add_rows<4>(gy, places, p1 * kPiece, to - p1 * kPiece, n, c, t);
            } else {
                add_rows<4>(gy, places, from, to - from, n, c, t);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) t[k] *= scale;
            store_at<true>(gtable + (first + r) * n, c, n, t);
        }
    }
}

// ---- workspace ------------------------------------------------------------------------------

struct Layout {
    int passes, bits, blocks;
    uint32_t per_block;
    size_t counts, keys[2], places[2], sums, sums2, bytes;
    bool second;
};

Layout layout_of(int64_t T, int64_t V, int n)
{
    Layout l = {};
    int bits = 1;
    while ((V >> bits) != 0) ++bits;                    // V itself stands for ids outside
    l.passes = div_up(bits, kMaxDigit);
    l.bits = div_up(bits, l.passes);
    int64_t per = div_up(T, (int64_t)kMaxBlocks);
    per = per < 1 ? kSortThreads : div_up(per, (int64_t)kSortThreads) * kSortThreads;
    l.per_block = (uint32_t)per;
    l.blocks = (int)div_up(T, per);
    l.second = T >= 4 * kPiece * kPiece;
    size_t at = 0;
    const auto take = [&at](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes);
        return here;
    };
    l.counts = take((size_t)l.blocks * ((size_t)4 << l.bits));
    for (int i = 0; i < 2; ++i) {
        l.keys[i] = take((size_t)T * 4);
        l.places[i] = take((size_t)T * 4);
    }
    l.sums = take((size_t)(T / kPiece) * n * 4);
    l.sums2 = l.second ? take((size_t)(T / (kPiece * kPiece)) * n * 4) : at;
    l.bytes = at;
    return l;
}

int check(int64_t T, int64_t V, int32_t n)
{
    if (T < 0 || V <= 0 || n <= 0) return KAN_ERR_INVALID_ARG;
    if (T >= (1ll << 31) - 65536 || V >= (1ll << 31) - 1) return KAN_ERR_UNSUPPORTED;
    return KAN_OK;
}

int check_types(int table_type, int y_type)
{
    if (!known_type(table_type) || !known_type(y_type) || (table_type == KAN_F32 && y_type != KAN_F32)) return KAN_ERR_UNSUPPORTED;
    return KAN_OK;
}

template <class T, class Y>
hipError_t launch_rows(int64_t count, int64_t V, int n, const int64_t *ids, const void *table, float scale, void *y, hipStream_t st)
{
    const int pieces = div_up(n, 8);
    prof::Timed timed("embedding_rows", st);
    embedding_rows_kernel<T, Y><<<(unsigned)div_up(count * pieces, (int64_t)256), 256, 0, st>>>(ids, (const T *)table, (Y *)y, count, V, n, pieces, scale);
    return hipGetLastError();
}

template <class Y, class G>
hipError_t launch_sums(const Layout &l, int64_t T, int64_t V, int n, const uint32_t *keys, const uint32_t *places, const void *gy, float scale, void *gtable,
                       char *ws, hipStream_t st)
{
    const int lanes = lanes_of_row(n) < 256 ? lanes_of_row(n) : 256;
    const unsigned wide = (unsigned)div_up(n, lanes * 8);
    float *sums = (float *)(ws + l.sums), *sums2 = (float *)(ws + l.sums2);
    hipError_t e = hipSuccess;
    if (T >= kPiece) {
        prof::Timed timed("embedding_pieces", st);
        embedding_piece_kernel<Y><<<dim3((unsigned)(T / kPiece), wide), 256, 0, st>>>(keys, places, (const Y *)gy, sums, V, n, lanes, 1);
        e = hipGetLastError();
    }
    if (e == hipSuccess && l.second) {
        prof::Timed timed("embedding_pieces", st);
        embedding_piece_kernel<float><<<dim3((unsigned)(T / (kPiece * kPiece)), wide), 256, 0, st>>>(keys, nullptr, sums, sums2, V, n, lanes, kPiece);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    prof::Timed timed("embedding_sum", st);
    embedding_sum_kernel<Y, G><<<(unsigned)div_up(V, (int64_t)kRows), 256, 0, st>>>(keys, places, (const Y *)gy, sums, l.second ? sums2 : nullptr, (G *)gtable,
                                                                                   (uint32_t)T, V, n, lanes, scale);
    return hipGetLastError();
}

}  // namespace
}  // namespace kannet

using namespace kannet;

extern "C" int kan_embedding_forward(int64_t T, int64_t V, int32_t n, const int64_t *ids, const void *table, int32_t table_type, float scale,
                                     void *y, int32_t y_type, void *stream)
{
    int rc = check(T, V, n);
    if (rc == KAN_OK) rc = check_types(table_type, y_type);
    if (rc != KAN_OK) return rc;
    if (T == 0) return KAN_OK;
    if (!ids || !table || !y || misplaced8(ids) || misplaced(table, table_type) || misplaced(y, y_type)) return KAN_ERR_INVALID_ARG;
    if (T * div_up(n, 8) >= (1ll << 31) * 256) return KAN_ERR_UNSUPPORTED;
    hipStream_t st = (hipStream_t)stream;
    return status_of(table_type == KAN_F32 ? launch_rows<float, float>(T, V, n, ids, table, scale, y, st)
                     : y_type == KAN_F32   ? launch_rows<bf16, float>(T, V, n, ids, table, scale, y, st)
                                           : launch_rows<bf16, bf16>(T, V, n, ids, table, scale, y, st));
}

extern "C" size_t kan_embedding_workspace_bytes(int64_t T, int64_t V, int32_t n)
{
    return check(T, V, n) == KAN_OK ? layout_of(T, V, n).bytes : 0;
}

extern "C" int kan_embedding_backward(int64_t T, int64_t V, int32_t n, const int64_t *ids, const void *gy, int32_t y_type, float scale,
                                      void *gtable, int32_t table_type, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check(T, V, n);
    if (rc == KAN_OK) rc = check_types(table_type, y_type);
    if (rc != KAN_OK) return rc;
    if (!gtable || misplaced(gtable, table_type)) return KAN_ERR_INVALID_ARG;
    if (T > 0 && (!ids || !gy || misplaced8(ids) || misplaced(gy, y_type))) return KAN_ERR_INVALID_ARG;
    const Layout l = layout_of(T, V, n);
    if (bad_workspace(ws, ws_bytes, l.bytes)) return KAN_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    char *at = (char *)ws;
    int from = 0;
    for (int pass = 0; pass < l.passes && T > 0; ++pass) {
        SortPass a = {};
        a.ids = pass == 0 ? ids : nullptr;
        a.key_in = (const uint32_t *)(at + l.keys[from]);
        a.place_in = (const uint32_t *)(at + l.places[from]);
        a.key_out = (uint32_t *)(at + l.keys[1 - from]);
        a.place_out = (uint32_t *)(at + l.places[1 - from]);
        a.counts = (uint32_t *)(at + l.counts);
        a.V = V;
        a.T = (uint32_t)T;
        a.per_block = l.per_block;
        a.blocks = l.blocks;
        a.shift = pass * l.bits;
        a.bits = l.bits;
        from = 1 - from;
        {
            prof::Timed timed("embedding_sort", st);
            embedding_count_kernel<<<l.blocks, kSortThreads, 0, st>>>(a);
        }
        if (hipGetLastError() != hipSuccess) return KAN_ERR_HIP;
        prof::Timed timed("embedding_sort", st);
        embedding_place_kernel<<<l.blocks, kSortThreads, 0, st>>>(a);
        if (hipGetLastError() != hipSuccess) return KAN_ERR_HIP;
    }
    const uint32_t *keys = (const uint32_t *)(at + l.keys[from]), *places = (const uint32_t *)(at + l.places[from]);
    return status_of(table_type == KAN_F32 ? launch_sums<float, float>(l, T, V, n, keys, places, gy, scale, gtable, at, st)
                     : y_type == KAN_F32   ? launch_sums<float, bf16>(l, T, V, n, keys, places, gy, scale, gtable, at, st)
                                           : launch_sums<bf16, bf16>(l, T, V, n, keys, places, gy, scale, gtable, at, st));
}
