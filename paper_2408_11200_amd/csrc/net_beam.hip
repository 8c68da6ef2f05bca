// One step of beam searches: the best continuations over a search's beams and the vocabulary (kan_net.h).
//
// Of one beam no more than `top` tokens can be among the search's `top` best, and they are its `top` largest logits.  So a first launch goes through the rows
// once, each on its own (few rows cut into parts): the sum of the exponentials, and the keys of the largest logits, in order.  The second one has a
// workgroup for each search: it adds the beams' scores, in 64 bits, and takes the `top` best of what the rows have left.  Rows of beams that have ended
// or are not there are not read.
//
// The largest logits come out of the one read: the `top`-th largest of the threads' largest ones is a bound that `top` logits reach.  Of the first round's pieces
// and of every later one that reach the bound after the first round (taken anew behind rounds 2, 4, 8, ... where as many would not fit), a wave notes which they are, with their largest
// logits; behind the row those that reach the bound of all of it, hardly more than `top` of them, are read again, and their logits that do are put in order.
// (Logits picked from each piece as it passed took the waves through some hundred instructions a piece more where no tokens stand out: 64 x 8 x 131072 bf16 48 us.)
//
// Measured: 128 x 8 x 131072 bf16 with sixteen 50-53 us for the rows (268 MB, 5.1-5.3 TB/s; half of the workgroups wait 5 us for their first logits, as all begin together, and
// each has 4 left after its last ones) and 5.3 for the second launch; 4 x 32 x 131072 with 64 16.4 and 10.7; 1 x 4 x 32768 with four 6.2 and 4.4, one latency after another.
#include "net_softmax.hpp"

namespace kannet {
namespace {

struct BeamCall {
    const void *logits;
    int64_t row_stride, V;
    uint32_t rows;          // N * B
    int B, top;
    const float *scores, *rank_scale;
    const uint8_t *ended;
    int64_t end_id;
    Temperature t;
    float *out_scores;
    int64_t *tokens, *parents;
    uint8_t *out_ended;
    int parts;              // of a row
    uint32_t part_pieces;   // pieces of 16 bytes of a part
    Mass *sums;             // [rows][parts]
    uint64_t *keys;         // [rows][parts][top], best first; 0: none
};

__device__ __forceinline__ bool finite(float v) { return v - v == 0.0f; }

// whether a beam's logits are looked at
__device__ __forceinline__ bool goes_on(const BeamCall &a, uint32_t row)
{
    const bool ended = a.ended && a.ended[row];
    return finite(a.scores[row]) && !ended;
}

// A row, or part blockIdx.x % a.parts of it
template <class T, int NT, bool STREAM>
__global__ __launch_bounds__(NT) void beam_rows_kernel(BeamCall a)
{
    constexpr int N = 16 / sizeof(T);
    constexpr uint32_t kCandidates = 4 * NT, kNotes = 512, kWaves = NT / 64;
    struct Note {
        float most;
        uint32_t piece;
    };
    __shared__ Mass wave_sums[kWaves];
    __shared__ Note notes[kWaves][kNotes];
    __shared__ uint64_t best[kCandidates];
    __shared__ uint32_t candidates, sources;
    __shared__ uint16_t source[NT];
    __shared__ float thread_most[NT];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    if (!goes_on(a, row)) return;
    const T *z = (const T *)a.logits + (int64_t)row * a.row_stride;
    const uint32_t V = (uint32_t)a.V, pieces = (V + N - 1) / N;
    const uint32_t begin = part * a.part_pieces, end = pieces - begin < a.part_pieces ? pieces : begin + a.part_pieces;
    const float scale = a.t.scale;
    Tally tally = no_tally();
    float most = -INFINITY, bound = NAN;
    uint32_t noted = 0;             // by this wave
    const auto note = [&](float m, uint32_t p) {
        const uint64_t which = __ballot(m >= bound && m > -INFINITY);
        if (!which) return;
        const uint32_t at = noted + __builtin_amdgcn_mbcnt_hi((uint32_t)(which >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)which, 0));
        if ((which >> lane & 1) && at < kNotes) notes[wave][at] = Note{m, p};
        noted += __popcll(which);
    };
    if (tid == 0) candidates = sources = 0;
    Round<T, NT> next;
    read_round<STREAM>(next, z, begin, end, V);
    const uint32_t rounds = (end - begin + kRound * NT - 1) / (kRound * NT);
    const bool tighten = (uint32_t)a.top * rounds > kNotes * kWaves / 4;
    uint32_t round = 0, again = 2;
    for (uint32_t first = begin; first < end; first += kRound * NT) {
        const Round<T, NT> now = next;
        read_round<STREAM>(next, z, first + kRound * NT, end, V);
        float piece_most[kRound] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        each_piece(now, first, end, V, [&](const float (&v)[N], uint32_t, int u) {
            const float m = add_piece<N>(v, scale, tally);
            most = fmaxf(most, m);
            if (u == 0) piece_most[0] = m;
            else if (u == 1) piece_most[1] = m;
            else if (u == 2) piece_most[2] = m;
            else piece_most[3] = m;
        });
        if (++round == 1 || (tighten && round == again)) {
            if (round > 1) {
                __syncthreads();
                again *= 2;
            }
            bound = value_of_rank<NT>(most, a.top, lane, thread_most);
        }
#pragma unroll
        for (int u = 0; u < kRound; ++u) note(piece_most[u], first + tid + u * NT);
    }
    const Mass sum = join_mass<NT>(mass_of(tally, scale), scale, wave_sums);
    uint64_t found = 0;
    uint32_t n = 0;
    if (sum.s == sum.s && sum.s > 0.0f) {           // the same in all threads; a NaN's beam has no candidates
        __syncthreads();
        if (rounds > 1) bound = value_of_rank<NT>(most, a.top, lane, thread_most);
        for (uint32_t i = lane; i < (noted < kNotes ? noted : kNotes); i += 64) {
            const Note from = notes[wave][i];
            if (from.most < bound) continue;
            float v[N];
            piece_logits<N>(raw_at<N>(z, (int64_t)from.piece * N, (int64_t)V), from.piece, V, v);
            uint32_t which = 0;
#pragma unroll
            for (int k = 0; k < N; ++k) which |= v[k] >= bound && v[k] > -INFINITY ? 1u << k : 0u;
            uint32_t slot = atomicAdd(&candidates, (uint32_t)__popc(which));
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (which >> k & 1) {
                    if (slot < kCandidates) best[slot] = key_of(v[k], from.piece * N + k);
                    ++slot;
                }
        }
        if (lane == 0 && noted > kNotes) atomicAdd(&candidates, kCandidates + 1u);
        __syncthreads();
        n = candidates;
        if (n > kCandidates) {
            // more than there is room for (many equal logits, rising ones): the pieces of the threads whose largest logit reaches the bound are read
            // again, by every wave into a sorted list of its own
            if (begin + tid < end && most >= bound && most > -INFINITY) source[atomicAdd(&sources, 1u)] = (uint16_t)tid;
            __syncthreads();
            const uint32_t each = (end - begin + NT - 1) / NT, count = sources * each;
            for (uint32_t first = 64 * wave; first < count; first += NT) {
                const uint32_t i = first + lane, p = i < count ? begin + source[i / each] + i % each * NT : end;
                float v[N];
                piece_logits<N>(raw_at<N>(z, (int64_t)p * N, (int64_t)(p < end ? V : 0)), p, V, v);
#pragma unroll 1
                for (int k = 0; k < N; ++k) put_in(found, p < end && v[k] >= bound && v[k] > -INFINITY ? key_of(v[k], p * N + k) : 0, a.top, lane);
            }
        } else if (n > 64) {
            for (uint32_t first = 64 * wave; first < n; first += NT) {
                const uint64_t k = first + lane < n ? best[first + lane] : 0;
                found = best_of(found, of_partner<63>(sorted(k, lane), lane), lane);
            }
        }
        // two waves' lists at a time, to the first wave
#pragma unroll 1
        for (uint32_t half = n > 64 ? kWaves / 2 : 0; half >= 1; half /= 2) {
            __syncthreads();
            if (wave >= half && wave < 2 * half) best[wave * 64 + lane] = found;
            __syncthreads();
            if (wave < half) found = best_of(found, best[(wave + half) * 64 + 63 - lane], lane);
        }
    }
    if (wave != 0) return;
    const uint32_t slot = row * a.parts + part;
    if (lane == 0) a.sums[slot] = sum;
    uint64_t *to = a.keys + (uint64_t)slot * a.top;
    if (n > 64) {
        if (lane < (uint32_t)a.top) to[lane] = found;
        return;
    }
    // few: each one's place is the number of those above it
    const uint64_t mine = lane < n ? best[lane] : 0;
    uint32_t place = 0;
    for (uint32_t i = 0; i < n; ++i) place += of_lane(mine, i) > mine ? 1 : 0;
    if (lane >= n) place = lane;
    if (place < (uint32_t)a.top) to[place] = mine;
}

// A candidate: larger ones first.  Its rank in all 64 bits, ordered like the values; of equal ones the lower beam, of one beam the larger logit (at a high temperature, or beside
// a large score, logits that differ can have one rank), and of equal logits the place in the rows' lists, which lie in the order of a beam's parts and so of its tokens.  Rank 0: none.
__device__ __forceinline__ Ranked candidate_of(double rank, uint32_t beam, uint32_t logit, uint32_t place)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, rank + 0.0);        // both zeros are one value
    return Ranked{(b >> 63) ? ~b : b | 0x8000000000000000ull, (uint64_t)(KAN_BEAM_MAX - 1 - beam) << 48 | (uint64_t)logit << 16 | (0xFFFFu - place)};
}

enum { kOut = 0, kGoesOn = 1, kEnded = 2 };

struct Beam {
    double score, log_sum;          // of the log probability: score + ((z - most) / temperature - log_sum)
    float most, rank_scale;
    int state;
};

constexpr uint32_t kLists = 1024;       // of a search: parts of its rows, or rows; an entry's place is below kLists * KAN_TOP_MAX = 2^16

// A workgroup for each search: 256 threads where each has one of the lists' entries at most, 1024 otherwise.  What counts is latency: all there is to read
// is on its way before any of it is looked at, and instead of counting for each candidate how many are above it (128 of them: 7 us) waves sort theirs in
// registers and join them.  Ranks cut to 48 bits beside the place, half the registers a candidate, took 0.5 to 0.7 us less (2.7 of 4 x 32 x 131072 with 64), and were equal where they are not;
// compared as 64-bit floats they take as long.
template <int NT>
__global__ __launch_bounds__(NT) void beam_join_kernel(BeamCall a)
{
    constexpr uint32_t kWaves = NT / 64;
    __shared__ Mass sums[kLists];
    __shared__ Beam beams[KAN_BEAM_MAX];
    __shared__ Ranked waves_best[kWaves][64];
    __shared__ Ranked bound;
    __shared__ uint16_t open[kLists];
    __shared__ uint32_t count;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), top = a.top, parts = a.parts, lists = a.B * parts;
    const uint32_t first_row = blockIdx.x * a.B;
    const uint64_t *keys = a.keys + (uint64_t)first_row * parts * top;
    // A wave looks at 64 entries, of as many lists as there are up to 64 and as many layers as fit beside one another: groups of lists, and of
    // every group the `step` first layers, dealt out to the waves.
    const uint32_t width = lists < 64 ? lists : 64, layers = 64 / width, groups = (lists + 63) / 64, group = wave % groups;
    const uint32_t l = group * 64 + lane % width, step = kWaves / groups * layers;
    const uint32_t j = wave / groups * layers + lane / width;
    const bool takes = l < lists && lane < width * layers && wave / groups < kWaves / groups;
    uint64_t key = takes && j < top ? keys[l * top + j] : 0;
    Beam mine = {0.0, 0.0, 0.0f, 1.0f, kOut};
    if (tid < (uint32_t)a.B) {
        const float score = a.scores[first_row + tid];
        if (a.rank_scale) mine.rank_scale = a.rank_scale[first_row + tid];
        const bool ended = a.ended && a.ended[first_row + tid];
        mine.score = (double)score;
        if (finite(score) && mine.rank_scale > 0.0f && finite(mine.rank_scale)) mine.state = ended ? kEnded : kGoesOn;
    }
    for (uint32_t i = tid; i < lists; i += NT) sums[i] = a.sums[(uint64_t)first_row * parts + i];
    __syncthreads();
    if (tid < (uint32_t)a.B) {
        const Mass *part = sums + tid * parts;
        float m = kLowest;
#pragma unroll 4
        for (uint32_t p = 0; p < parts; ++p) m = fmaxf(m, part[p].m);
        double s = 0.0;
#pragma unroll 4
        for (uint32_t p = 0; p < parts; ++p) s += (double)(part[p].s * power(part[p].m, m, a.t.scale));
        mine.most = m;
        mine.log_sum = log_of(s);
        if (mine.state == kGoesOn && !(s > 0.0 && s < (double)INFINITY)) mine.state = kOut;
        beams[tid] = mine;
    }
    __syncthreads();
    // the score of entry j of list l, `key` of it; -infinity: none
    const auto score_of = [&](const Beam &beam, uint32_t j, bool first_part, uint64_t key) {
        double score = beam.score;
        bool there = beam.state == kGoesOn && key;
        if (beam.state == kEnded) there = first_part && j == 0;
        else score += ((double)logit_of(key) - (double)beam.most) * a.t.inverse - beam.log_sum;
        return there && finite((float)score) ? score : -(double)INFINITY;
    };
    // entry j of list l as a candidate
    const Ranked none = {0, 0};
    const auto entry = [&](uint32_t l, uint32_t j, uint64_t key) {
        const uint32_t b = l / parts;
        const Beam beam = beams[b];
        const double score = score_of(beam, j, l == b * parts, key);
        return score > -(double)INFINITY ? candidate_of(score * (double)beam.rank_scale, b, (uint32_t)(key >> 32), l * top + j) : none;
    };
    const Ranked first = takes && j < top ? entry(l, j, key) : none;
    Ranked best = sorted(first, lane);
    // two waves' lists at a time, to the first wave
    const auto join = [&]() {
#pragma unroll 1
        for (uint32_t half = kWaves / 2; half >= 1; half /= 2) {
            if (wave >= half && wave < 2 * half) waves_best[wave][lane] = best;
            __syncthreads();
            if (wave < half) best = best_of(best, waves_best[wave + half][63 - lane], lane);
        }
    };
    join();
    if (step < top) {
        // What is below `top` others, or below an entry of its list that is, leads to none: left are the rests of the lists whose layers reach the `top`-th best of
        // these, a wave each.  (All lists layer by layer: 34 us for 256 lists of 64, whose likely tokens are in every eighth one.)
        const Ranked seen = of_lane(best, top - 1);
        if (tid == 0) {
            bound = seen;
            count = 0;
        }
        __syncthreads();
        if (takes && j == step - 1 && above(first, bound)) open[atomicAdd(&count, 1u)] = (uint16_t)l;
        __syncthreads();
        if (wave != 0) best = none;
        for (uint32_t i = wave; i < count; i += kWaves) {
            const uint32_t l = open[i], j = step + lane;
            const Ranked c = j < top ? entry(l, j, keys[l * top + j]) : none;
            best = best_of(best, of_partner<63>(c, lane), lane);
        }
        join();
    }
    if (wave != 0 || lane >= top) return;
    const int64_t at = (int64_t)blockIdx.x * top + lane;
    const bool there = best.rank != 0;
    const uint32_t place = there ? 0xFFFFu - (uint32_t)(best.tie & 0xFFFF) : 0, list = place / top, b = list / parts;
    const Beam parent = beams[b];
    const uint64_t found = keys[place];
    const int64_t token = parent.state == kEnded ? a.end_id : (int64_t)(uint32_t)~(uint32_t)found;
    a.out_scores[at] = there ? (float)score_of(parent, place % top, list == b * parts, found) : -INFINITY;
    a.tokens[at] = there ? token : -1;
    a.parents[at] = there ? b : 0;
    if (a.out_ended) a.out_ended[at] = there && (parent.state == kEnded || token == a.end_id);
}

// How rows are cut: few rows are shared among workgroups, two a CU, of a round of pieces (16 KB) at least.  Both launches, us, whole rows, two workgroups
// a CU and four (all with a second launch of 0.6 us less than now): 1 x 4 x 16384 bf16 11.1, 9.6, 9.5; 32 x 4 x 16384 12.3, 10.8, 10.8; 24 x 4 x 50001 fp32 with twelve -, 15.0, 18.4; 16 x 8 x 131072 bf16 with sixteen -, 19.3, 21.3; half
// a round: 1 x 4 x 32768 bf16 10.3 for 9.7, 1 x 8 x 131072 16.5 for 14.7.
int parts_of(int64_t rows, int64_t V, size_t size)
{
    const int64_t rounds = V / (int64_t)(16384 / size);
    if (rows <= 0 || rows > 256 || rounds < 2) return 1;
    const int64_t parts = 512 / rows < rounds ? 512 / rows : rounds;
    return (int)(parts > 64 ? 64 : parts);
}

template <class T>
hipError_t launch(BeamCall &a, int64_t N, hipStream_t st)
{
    constexpr uint32_t per = 16 / sizeof(T);
    const uint32_t pieces = (uint32_t)div_up(a.V, (int64_t)per);
    a.part_pieces = div_up(pieces, (uint32_t)a.parts);
    a.parts = (int)div_up(pieces, a.part_pieces);
    const unsigned grid = a.rows * (unsigned)a.parts;
    {
        prof::Timed timed("beam_rows", st);
        const bool past = (double)a.rows * (double)a.V * sizeof(T) >= kLastCache;
        if (a.V <= 4096) beam_rows_kernel<T, 64, false><<<grid, 64, 0, st>>>(a);
        else if (past) beam_rows_kernel<T, 256, true><<<grid, 256, 0, st>>>(a);
        else beam_rows_kernel<T, 256, false><<<grid, 256, 0, st>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    prof::Timed timed("beam_join", st);
    if ((int64_t)a.B * a.parts * a.top <= 256) beam_join_kernel<256><<<(unsigned)N, 256, 0, st>>>(a);
    else beam_join_kernel<1024><<<(unsigned)N, 1024, 0, st>>>(a);
    return hipGetLastError();
}

int check(int64_t N, int32_t B, int64_t V, int32_t top)
{
    if (N < 0 || B < 1 || V <= 0 || top < 1) return KAN_ERR_INVALID_ARG;
    if (B > KAN_BEAM_MAX || top > KAN_TOP_MAX || V >= (1ll << 31) - 1 || N >= (1ll << 24) / B) return KAN_ERR_UNSUPPORTED;
    return top > B * V ? KAN_ERR_INVALID_ARG : KAN_OK;
}

// for the type whose rows are cut into more parts
size_t sums_bytes(int64_t N, int32_t B, int64_t V) { return align_up((size_t)(N * B) * parts_of(N * B, V, 4) * sizeof(Mass)); }

}  // namespace
}  // namespace kannet

using namespace kannet;

extern "C" size_t kan_beam_select_workspace_bytes(int64_t N, int32_t B, int64_t V, int32_t top)
{
    if (check(N, B, V, top) != KAN_OK || N == 0) return 0;
    return sums_bytes(N, B, V) + align_up((size_t)(N * B) * parts_of(N * B, V, 4) * top * sizeof(uint64_t));
}

extern "C" int kan_beam_select(int64_t N, int32_t B, int64_t V, const void *logits, int32_t type, int64_t row_stride, const float *scores,
                               const uint8_t *ended, const float *rank_scale, int64_t end_id, float temperature, int32_t top, float *out_scores,
                               int64_t *tokens, int64_t *parents, uint8_t *out_ended, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = check(N, B, V, top);
    if (rc != KAN_OK) return rc;
    if (row_stride < V || !(temperature >= 1e-30f && temperature <= 1e30f) || end_id < -1 || end_id >= V || (ended && end_id < 0)) return KAN_ERR_INVALID_ARG;
    if (!known_type(type)) return KAN_ERR_UNSUPPORTED;
    if (N == 0) return KAN_OK;
    if (!logits || !scores || !out_scores || !tokens || !parents) return KAN_ERR_INVALID_ARG;
    if (misplaced(logits, type) || misplaced(scores, KAN_F32) || misplaced(rank_scale, KAN_F32) || misplaced(out_scores, KAN_F32) || misplaced8(tokens) ||
        misplaced8(parents))
        return KAN_ERR_INVALID_ARG;
    if (bad_workspace(ws, ws_bytes, kan_beam_select_workspace_bytes(N, B, V, top))) return KAN_ERR_WORKSPACE;
    BeamCall a = {};
    a.logits = logits;
    a.row_stride = row_stride;
    a.V = V;
    a.rows = (uint32_t)(N * B);
    a.B = B;
    a.top = top;
    a.scores = scores;
    a.rank_scale = rank_scale;
    a.ended = ended;
    a.end_id = end_id;
    a.t = temperature_of(temperature);
    a.out_scores = out_scores;
    a.tokens = tokens;
    a.parents = parents;
    a.out_ended = out_ended;
    a.parts = parts_of(N * B, V, size_of(type));
    a.sums = (Mass *)ws;
    a.keys = (uint64_t *)((char *)ws + sums_bytes(N, B, V));
    return status_of(type == KAN_F32 ? launch<float>(a, N, (hipStream_t)stream) : launch<bf16>(a, N, (hipStream_t)stream));
}
