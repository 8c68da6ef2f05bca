// Embedding rows and their gradient (kan_net.h).
//
// Forward: a copy of rows, bound by HBM (by latency for a few tokens: 8 x 512 2.0 us).  65536 rows of 2048 bf16 87 us (441 MB with what of the table
// comes from memory, 5.1 TB/s), 16384 of 512 fp32 10.2.
//
// Backward: tokens are sorted by id, stably (least significant digit first, up to ten bits a pass), and the sorted list is cut into pieces
// of 16 entries, each worked on by the lanes of one row with its sixteen rows of gy in flight together.  A run of equal ids within a piece is a
// row of the table, written at once; a run that goes on into the next piece leaves its sum there as a fragment, and a workgroup for
// the piece it starts in joins them (of long runs, sixteen pieces at a time have been added before).  Rows without a token are zeroed by
// other workgroups of the same launch.  So the work is cut by places of the list, however often a token occurs, every row of the
// table is written once, and a row's sum has one order: no atomics on values.  Bound by HBM behind the sort: 65536 tokens, table of 131072 x 2048 bf16,
// sort 27 us, pieces 179 (805 MB, 4.5 TB/s), groups and joins 31-34; 16384 tokens, 50001 x 512 fp32, 14, 26 (136 MB, 5.2 TB/s) and 8.
#include "net_device.hpp"

namespace kannet {
namespace {

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMaxDigit = 10;
constexpr int kMaxBlocks = 64;        // of a sort pass: every block reads all blocks' counts
constexpr int kPiece = 16;
constexpr int kMaxChannels = 1 << 30;

template <class T, class Y>
__global__ __launch_bounds__(256) void embedding_rows_kernel(const int64_t *ids, const T *table, Y *y, int64_t T_, int64_t V, int n, int pieces, float scale)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, t = i / pieces;
    if (t >= T_) return;
    constexpr bool PAIR = is_float<T> || is_float<Y>;
    const int lane = (int)(i - t * pieces);
    const int64_t id = ids[t];
    float v[8];
    if (id >= 0 && id < V) {
        load_eight<PAIR>(table + id * n, 0, lane, pieces, n, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= scale;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 0.0f;
    }
    store_eight<PAIR>(y + t * n, 0, lane, pieces, n, v);
}

// ---- the sort -------------------------------------------------------------------------------

struct SortPass {
    const int64_t *ids;                 // first pass: keys come from here (ids outside the table: V), places are 0, 1, 2, ...
    const uint32_t *key_in, *place_in;
    uint32_t *key_out, *place_out;
    uint32_t *counts;                   // [blocks][digits]
    uint32_t *starts;                   // set to 0 by the first pass
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
    if (a.ids && blockIdx.x == 0 && threadIdx.x == 0) *a.starts = 0;
}

// entries of smaller digits, where each thread brings those of its own: a running sum over the threads
__device__ __forceinline__ uint32_t smaller_digits(uint32_t mine, uint32_t *wave_total)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t sum = mine;
    for (int step = 1; step < 64; step *= 2) {
        const uint32_t o = __shfl_up(sum, step, 64);
        if ((int)lane >= step) sum += o;
    }
    if (lane == 63) wave_total[wave] = sum;
    __syncthreads();
    uint32_t before = sum - mine;
    for (uint32_t w = 0; w < wave; ++w) before += wave_total[w];
    return before;
}

// Where a wave's entry of a digit goes: the cursor of the digit moves on by as many lanes as have it, which keep their order.
__device__ __forceinline__ uint32_t take_place(uint32_t *cursor, uint32_t digit, int bits, bool in)
{
    const uint32_t lane = threadIdx.x & 63;
    uint64_t same = __ballot(in);
    for (int b = 0; b < bits; ++b) {
        const bool bit = (digit >> b & 1u) != 0;
        const uint64_t set = __ballot(bit);
        same &= bit ? set : ~set;
    }
    const int first = __ffsll((unsigned long long)same) - 1;
    uint32_t at = 0;
    if (in && (int)lane == first) at = atomicAdd(&cursor[digit], (uint32_t)__popcll(same));
    return __shfl(at, first < 0 ? 0 : first, 64) + (uint32_t)__popcll(same & ((1ull << lane) - 1));
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
    uint32_t base = smaller_digits(all, wave_total) + before;
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
        const uint32_t key = in ? key_at(a, i) : 0u;
        const uint32_t at = take_place(cursor[wave], key >> a.shift & (digits - 1), a.bits, in);
        if (in) {
            a.key_out[at] = key;
            a.place_out[at] = a.ids ? i : a.place_in[i];
        }
    }
}

// The whole sort of up to 16384 tokens in one launch: a workgroup for each range of 2^bits ids goes through all tokens, a wave through consecutive
// ones; it keeps those of its range, in their order, in LDS, counts those below, and places what it kept.  The tokens come from L2, so that the
// launches saved (two a digit, some 9 us) are worth it while the ranges' workgroups are hardly more than the CUs.  By digits and so, us: 16384 tokens
// of 50001 ids 18.2 and 14.0, 4096 of 8000 17.4 and 6.5; one digit, 256 ids, 16384 tokens 8.7 and 13.2.
constexpr int kRangeRounds = 16;                                  // of 64 tokens a wave
constexpr int64_t kRangeTokens = (int64_t)kRangeRounds * kSortThreads;
constexpr int64_t kRanges = 512;

__global__ __launch_bounds__(kSortThreads) void embedding_range_sort_kernel(SortPass a)
{
    __shared__ uint32_t cursor[kSortWaves][1 << kMaxDigit];
    __shared__ uint32_t kept[kSortWaves][kRangeRounds * 64];         // id in the range, and which of the wave's tokens it is
    __shared__ uint32_t wave_total[kSortWaves], wave_below[kSortWaves];
    constexpr uint32_t kNone = 0xFFFFFFFFu;
    const uint32_t digits = 1u << a.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, start = blockIdx.x << a.bits;
    const uint32_t per_wave = (a.T + kSortThreads - 1) / kSortThreads * 64, from = wave * per_wave;
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.starts = 0;
    uint32_t key[kRangeRounds];
#pragma unroll
    for (int u = 0; u < kRangeRounds; ++u) {
        const uint32_t i = from + u * 64 + lane;
        key[u] = (uint32_t)u * 64 < per_wave && i < a.T ? key_at(a, i) : kNone;
    }
    for (uint32_t d = threadIdx.x; d < kSortWaves * digits; d += kSortThreads) cursor[d >> a.bits][d & (digits - 1)] = 0;
    uint32_t below = 0, count = 0;
#pragma unroll
    for (int u = 0; u < kRangeRounds; ++u) {
        below += (uint32_t)__popcll(__ballot(key[u] < start));
        const bool in = key[u] - start < digits;
        const uint64_t those = __ballot(in);
        if (in) kept[wave][count + (uint32_t)__popcll(those & ((1ull << lane) - 1))] = (key[u] - start) << 16 | (uint32_t)(u * 64 + lane);
        count += (uint32_t)__popcll(those);
    }
    if (lane == 0) wave_below[wave] = below;
    __syncthreads();
    for (uint32_t e = lane; e < count; e += 64) atomicAdd(&cursor[wave][kept[wave][e] >> 16], 1u);
    __syncthreads();
    uint32_t all = 0;
    if (threadIdx.x < digits)
        for (int w = 0; w < kSortWaves; ++w) all += cursor[w][threadIdx.x];
    uint32_t base = smaller_digits(all, wave_total);
    for (int w = 0; w < kSortWaves; ++w) base += wave_below[w];
    if (threadIdx.x < digits)
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = cursor[w][threadIdx.x];
            cursor[w][threadIdx.x] = base;
            base += c;
        }
    __syncthreads();
    for (uint32_t first = 0; first < count; first += 64) {
        const bool in = first + lane < count;
        const uint32_t k = in ? kept[wave][first + lane] : 0u;
        const uint32_t at = take_place(cursor[wave], k >> 16, a.bits, in);
        if (in) {
            a.key_out[at] = start + (k >> 16);
            a.place_out[at] = from + (k & 0xFFFFu);
        }
    }
}

// ---- sums -----------------------------------------------------------------------------------

// Adds a lane's eight channels of the rows first .. first + count - 1, `stride` floats apart, to t, one after the other, AHEAD of them in flight.
template <int AHEAD>
__device__ __forceinline__ void add_rows(const float *rows, int64_t stride, uint32_t first, uint32_t count, int n, int base, int lane, int lanes, float (&t)[8])
{
    for (uint32_t i = 0; i < count; i += AHEAD) {
        Eight<float, true> r[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) r[k] = eight_at<true>(rows + (int64_t)(first + i + k) * stride, base, lane, lanes, i + k < count ? n : 0);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            float v[8];
            unpack_at<true>(r[k], base, lane, lanes, n, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] += v[j];
        }
    }
}

constexpr int kRows = 256;      // most table rows of a workgroup that looks for rows without tokens

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

struct SumCall {
    const uint32_t *keys, *places;
    float *fragments;       // [pieces][2][n]: of the run a piece begins with (all of the piece, or as far as the run goes), and of the one it ends with
    float *groups;          // [pieces / 16][n]: sixteen pieces of one id; null: too few entries for that
    uint32_t *starts;       // [0]: how many runs leave the piece they start in; then those pieces, in any order
    uint32_t T, pieces;     // keys and places are readable up to whole pieces
    int64_t V;
    int n, lanes;
    unsigned piece_blocks;
    int zero_rows;
    float scale;
};

// The first piece_blocks workgroups have the pieces, 256 / lanes each; the others zero_rows table rows each (32 KB, 32 rows at least), which they zero
// where no token names them.
// WAVES: a row takes whole waves (64 lanes and more): ids and places of a piece are then in scalar registers.
template <class Y, class G, bool WAVES>
__global__ __launch_bounds__(256) void embedding_piece_kernel(SumCall a, const Y *gy, G *gtable)
{
    __shared__ uint32_t lds[4], here[kRows];
    const int n = a.n, lanes = a.lanes, worker = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    if (blockIdx.x >= a.piece_blocks) {
        const int rows = a.zero_rows;
        const int64_t first = (int64_t)(blockIdx.x - a.piece_blocks) * rows;
        const uint32_t begin = keys_below(a.keys, a.T, first, lds), rest = keys_below(a.keys + begin, a.T - begin, first + rows, lds);
        if ((int)threadIdx.x < rows) {
            uint32_t lo = begin, hi = begin + rest;
            while (lo < hi) {
                const uint32_t mid = lo + (hi - lo) / 2;
                if ((int64_t)a.keys[mid] < first + threadIdx.x) lo = mid + 1;
                else hi = mid;
            }
            here[threadIdx.x] = lo < begin + rest && (int64_t)a.keys[lo] == first + threadIdx.x;
        }
        __syncthreads();
        const float zeros[8] = {};
        constexpr bool kPairZero = is_float<G>;
        for (int r = worker; r < rows && first + r < a.V; r += 256 / lanes)
            if (!here[r])
                for (int base = 0; base < n; base += lanes * 8) store_eight<kPairZero, true>(gtable + (first + r) * n, base, lane, lanes, n, zeros);
        return;
    }
    uint32_t p = blockIdx.x * (256 / lanes) + worker;
    if (WAVES) p = __builtin_amdgcn_readfirstlane(p);
    if (p >= a.pieces) return;
    uint32_t key[kPiece], place[kPiece];
#pragma unroll
    for (int i = 0; i < kPiece; i += 4) {
        const u32x4 k = *(const u32x4 *)(a.keys + p * kPiece + i), q = *(const u32x4 *)(a.places + p * kPiece + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool in = p * kPiece + i + j < a.T;
            key[i + j] = in ? k[j] : 0xFFFFFFFFu;
            place[i + j] = q[j];
        }
    }
    const uint32_t V = (uint32_t)a.V;
    constexpr bool PAIR = is_float<Y> || is_float<G>;
    const bool from_before = p > 0 && a.keys[p * kPiece - 1] == key[0];
    const bool goes_on = (p + 1) * kPiece < a.T && a.keys[(p + 1) * kPiece] == key[kPiece - 1];
    if (lane == 0 && goes_on && key[kPiece - 1] < V && !(from_before && key[0] == key[kPiece - 1])) a.starts[1 + atomicAdd(a.starts, 1u)] = p;
    for (int base = 0; base < n; base += lanes * 8) {
        float t[8] = {};
        bool first_run = true;
#pragma unroll
        for (int b = 0; b < kPiece; b += 8) {
            Eight<Y, PAIR> r[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) r[j] = eight_at<PAIR>(gy + (int64_t)place[b + j] * n, base, lane, lanes, key[b + j] < V ? n : 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v[8];
                unpack_at<PAIR>(r[j], base, lane, lanes, n, v);
#pragma unroll
                for (int k = 0; k < 8; ++k) t[k] += v[k];
                const bool last = b + j == kPiece - 1;
                if (last || key[b + j] != key[b + j + 1 < kPiece ? b + j + 1 : 0]) {
                    if (key[b + j] < V) {
                        const bool left = first_run && from_before, right = last && goes_on;
                        if (left || right) {
                            float *to = a.fragments + ((int64_t)p * 2 + (first_run ? 0 : 1)) * n;
                            if constexpr (PAIR) {
                                store_eight<true>(to, base, lane, lanes, n, t);
                            } else {
                                store_at<4>(to, base + 8 * lane, n, t);
                                store_at<4>(to, base + 8 * lane + 4, n, t + 4);
                            }
                        } else {
#pragma unroll
                            for (int k = 0; k < 8; ++k) t[k] *= a.scale;
                            store_eight<PAIR, true>(gtable + (int64_t)key[b + j] * n, base, lane, lanes, n, t);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) t[k] = 0.0f;
                    first_run = false;
                }
            }
        }
    }
}

// Sixteen pieces of one id, a workgroup each: a run of 10000 places would be 625 fragments one behind the other for the join
__global__ __launch_bounds__(256) void embedding_group_kernel(SumCall a)
{
    const uint32_t q = blockIdx.x, width = kPiece * kPiece;
    if (a.keys[q * width] >= (uint32_t)a.V || a.keys[(q + 1) * width - 1] != a.keys[q * width]) return;
    for (int base = 0; base < a.n; base += 256 * 8) {
        float t[8] = {};
        add_rows<8>(a.fragments + (int64_t)q * kPiece * 2 * a.n, 2ll * a.n, 0, kPiece, a.n, base, threadIdx.x, 256, t);
        store_eight<true>(a.groups + (int64_t)q * a.n, base, threadIdx.x, 256, a.n, t);
    }
}

template <class G>
__device__ __forceinline__ void join_run(const SumCall &a, G *gtable, uint32_t p)
{
    __shared__ float lds[256 * 8];
    __shared__ uint32_t votes[4];
    const uint32_t id = a.keys[p * kPiece + kPiece - 1];
    const bool whole = a.keys[p * kPiece] == id;
    // pieces behind this one that begin with the id
    uint32_t more = 0;
    for (;;) {
        const uint64_t at = (uint64_t)(p + 1 + more + threadIdx.x) * kPiece;
        const uint64_t yes = __ballot(at < a.T && a.keys[at < a.T ? at : 0] == id);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) votes[threadIdx.x >> 6] = (uint32_t)__popcll(yes);       // the list is sorted: those that do come first
        __syncthreads();
        const uint32_t all = votes[0] + votes[1] + votes[2] + votes[3];
        more += all;
        if (all < 256) break;
    }
    // rows wider than a wave's 512 channels are shared by workgroups of as many workers
    const int n = a.n, lanes = a.lanes < 64 ? a.lanes : 64, workers = 256 / lanes, w = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    // pieces p + 1 .. end - 1; the groups q0 .. q1 - 1 lie wholly among those that hold nothing but the id
    const uint32_t begin = p + 1, end = begin + more;
    const uint64_t full_end = (uint64_t)end * kPiece <= a.T && a.keys[(uint64_t)end * kPiece - 1] == id ? end : end - 1;
    uint32_t q0 = (begin + kPiece - 1) / kPiece, q1 = (uint32_t)(full_end / kPiece);
    if (!a.groups || q1 <= q0) q0 = q1 = 0;
    const uint32_t cut0 = q1 > 0 ? q0 * kPiece : end, cut1 = q1 > 0 ? q1 * kPiece : end;
    const auto part = [&](uint32_t from, uint32_t count, int which) { return from + (uint32_t)((uint64_t)count * which / workers); };
    for (int base = blockIdx.y * lanes * 8; base < n; base += gridDim.y * lanes * 8) {
        float t[8] = {};
        if (w == 0) add_rows<1>(a.fragments + ((int64_t)p * 2 + (whole ? 0 : 1)) * n, 0, 0, 1, n, base, lane, lanes, t);
        const uint32_t b0 = part(begin, cut0 - begin, w), b1 = part(begin, cut0 - begin, w + 1);
        add_rows<8>(a.fragments, 2ll * n, b0, b1 - b0, n, base, lane, lanes, t);
        const uint32_t g0 = part(q0, q1 - q0, w), g1 = part(q0, q1 - q0, w + 1);
        add_rows<8>(a.groups, n, g0, g1 - g0, n, base, lane, lanes, t);
        const uint32_t e0 = part(cut1, end - cut1, w), e1 = part(cut1, end - cut1, w + 1);
        add_rows<8>(a.fragments, 2ll * n, e0, e1 - e0, n, base, lane, lanes, t);
        if (workers > 1) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 8; ++k) lds[k * 256 + threadIdx.x] = t[k];
            __syncthreads();
            if (w == 0)
                for (int o = 1; o < workers; ++o)
#pragma unroll
                    for (int k = 0; k < 8; ++k) t[k] += lds[k * 256 + o * lanes + lane];
        }
        if (w == 0) {
#pragma unroll
            for (int k = 0; k < 8; ++k) t[k] *= a.scale;
            store_eight<true>(gtable + (int64_t)id * n, base, lane, lanes, n, t);
        }
    }
}

// The runs that leave the piece they start in, a workgroup each: its workers share the run's fragments.  Latency (a list entry, ids, fragments):
// 7.6 us for 16384 tokens, 26-28 for 65536.
template <class G>
__global__ __launch_bounds__(256) void embedding_join_kernel(SumCall a, G *gtable)
{
    const uint32_t runs = a.starts[0];
    for (uint32_t i = blockIdx.x; i < runs; i += gridDim.x) join_run(a, gtable, a.starts[1 + i]);
}

// ---- workspace ------------------------------------------------------------------------------

struct Layout {
    int ranges, range_bits;     // of ids, where one launch sorts; 0: by digits
    int passes, bits, blocks;
    uint32_t per_block;
    size_t counts, starts, keys[2], places[2], fragments, groups, bytes;
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
    // about 64 ranges, of 16 .. 1024 ids
    l.range_bits = bits - 6 < 4 ? 4 : bits - 6 > kMaxDigit ? kMaxDigit : bits - 6;
    const int64_t ranges = (V >> l.range_bits) + 1;
    l.ranges = T <= (l.passes > 1 ? kRangeTokens : kRangeTokens / 2) && ranges <= kRanges ? (int)ranges : 0;
    l.second = T >= 128 * kPiece * kPiece;
    size_t at = 0;
    const auto take = [&at](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes);
        return here;
    };
    l.counts = take((size_t)l.blocks * ((size_t)4 << l.bits));
    l.starts = take(T > 0 ? ((size_t)div_up(T, (int64_t)kPiece) + 1) * 4 : 0);
    for (int i = 0; i < 2; ++i) {
        l.keys[i] = take((size_t)div_up(T, (int64_t)kPiece) * kPiece * 4);
        l.places[i] = take((size_t)div_up(T, (int64_t)kPiece) * kPiece * 4);
    }
    l.fragments = take((size_t)div_up(T, (int64_t)kPiece) * 2 * n * 4);
    l.groups = l.second ? take((size_t)(T / (kPiece * kPiece)) * n * 4) : at;
    l.bytes = at;
    return l;
}

int check(int64_t T, int64_t V, int32_t n)
{
    if (T < 0 || V <= 0 || n <= 0) return KAN_ERR_INVALID_ARG;
    // channels are counted in 32 bits, up to two workgroups' width past a row's end
    if (T >= (1ll << 31) - 65536 || V >= (1ll << 31) - 1 || n > kMaxChannels) return KAN_ERR_UNSUPPORTED;
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
    // a launch has less than 2^32 threads: of more, HIP starts what is left of their number in 32 bits, and reports nothing
    const int64_t most = (1ll << 31) / pieces;
    for (int64_t first = 0; first < count; first += most) {
        const int64_t here = count - first < most ? count - first : most;
        prof::Timed timed("embedding_rows", st);
        embedding_rows_kernel<T, Y><<<(unsigned)div_up(here * pieces, (int64_t)256), 256, 0, st>>>(ids + first, (const T *)table, (Y *)y + first * n, here, V, n, pieces,
                                                                                                   scale);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class Y, class G>
hipError_t launch_sums(const Layout &l, int64_t T, int64_t V, int n, const uint32_t *keys, const uint32_t *places, const void *gy, float scale, void *gtable,
                       char *ws, hipStream_t st)
{
    SumCall a = {};
    a.keys = keys;
    a.places = places;
    a.fragments = (float *)(ws + l.fragments);
    a.groups = l.second ? (float *)(ws + l.groups) : nullptr;
    a.starts = (uint32_t *)(ws + l.starts);
    a.T = (uint32_t)T;
    a.pieces = (uint32_t)div_up(T, (int64_t)kPiece);
    a.V = V;
    a.n = n;
    a.lanes = lanes_of_row(n) < 256 ? lanes_of_row(n) : 256;
    a.piece_blocks = div_up(a.pieces, 256u / (unsigned)a.lanes);
    const int64_t zero_rows = 32768 / ((int64_t)n * (int64_t)sizeof(G));
    a.zero_rows = zero_rows < 32 ? 32 : zero_rows > kRows ? kRows : (int)zero_rows;
    a.scale = scale;
    {
        prof::Timed timed("embedding_pieces", st);
        const unsigned blocks = a.piece_blocks + (unsigned)div_up(V, (int64_t)a.zero_rows);
        if (a.lanes >= 64) embedding_piece_kernel<Y, G, true><<<blocks, 256, 0, st>>>(a, (const Y *)gy, (G *)gtable);
        else embedding_piece_kernel<Y, G, false><<<blocks, 256, 0, st>>>(a, (const Y *)gy, (G *)gtable);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || T <= kPiece) return e;
    if (l.second) {
        prof::Timed timed("embedding_groups", st);
        embedding_group_kernel<<<(unsigned)(T / (kPiece * kPiece)), 256, 0, st>>>(a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    prof::Timed timed("embedding_join", st);
    embedding_join_kernel<G><<<dim3(a.pieces < 1024 ? a.pieces : 1024, (unsigned)div_up(n, 512)), 256, 0, st>>>(a, (G *)gtable);
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
    if (T > 0 && l.ranges) {
        SortPass a = {};
        a.ids = ids;
        a.key_out = (uint32_t *)(at + l.keys[0]);
        a.place_out = (uint32_t *)(at + l.places[0]);
        a.starts = (uint32_t *)(at + l.starts);
        a.V = V;
        a.T = (uint32_t)T;
        a.bits = l.range_bits;
        prof::Timed timed("embedding_sort", st);
        embedding_range_sort_kernel<<<l.ranges, kSortThreads, 0, st>>>(a);
        if (hipGetLastError() != hipSuccess) return KAN_ERR_HIP;
    }
    for (int pass = 0; pass < l.passes && T > 0 && !l.ranges; ++pass) {
        SortPass a = {};
        a.ids = pass == 0 ? ids : nullptr;
        a.key_in = (const uint32_t *)(at + l.keys[from]);
        a.place_in = (const uint32_t *)(at + l.places[from]);
        a.key_out = (uint32_t *)(at + l.keys[1 - from]);
        a.place_out = (uint32_t *)(at + l.places[1 - from]);
        a.counts = (uint32_t *)(at + l.counts);
        a.starts = (uint32_t *)(at + l.starts);
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
