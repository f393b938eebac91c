// Rows of a table looked up by id, and the gradient of the table.
//   y[i] = scale * table[id[i]],   g_table[v] = scale * (sum over the i with id[i] = v of g_y[i])
// An id equal to `padding` gives a row of zeros, one outside the table a row of NaN; neither sends a gradient.
// The gradient sorts the tokens by id (stable, so that equal ids stay in their order and every sum has one fixed order), cuts the sorted list into equal pieces
// whatever the ids are, and adds up runs of equal ids: a piece's inner runs are rows of g_table, runs that cross pieces are joined afterwards.
#include "hag_elem.hpp"

namespace hag {

// ------------------------------------------------------------------------------------------------------------------ lookup

struct EmbedArgs {
    const void *table, *ids;
    void *y;
    int64_t stride, extent;          // of the table: elements to the next row, to the end of the last one
    int64_t n, rows, padding;
    int32_t d;
    float scale;
};

// Bound by writing y (and by reading the table where it exceeds the caches).  LPR lanes move a row, 16 bytes each, four rows at a time: the ids first, then the rows they name.
// Streaming stores leave the caches to the table: 524288 rows of 232965, 128 columns, ids spread evenly / some rows in demand: fp32 88 -> 83 us, 84 -> 53, bf16 40.7 -> 37.8, 29.9 -> 27.8.  What
// reads y next finds less of it there: with a layer norm after it fp32 186 -> 181, but bf16 84 -> 90, and 56944 rows of as many, fp32, 21.8 -> 23.9, 370000 x 64 of 74 47 -> 52.
// 370000 rows of 74, 64 fp32 columns: 16.4 us, 5.8 TB/s written (a fill: 6.4); a call on 74 rows 7.5 us, which is the host's.
constexpr int kEmbedRows = 4;
template <typename T, typename I, int LPR, bool TAIL>
__global__ __launch_bounds__(kBlock) void embed_kernel(EmbedArgs a) {
    constexpr int V = kVec<T>, R = kEmbedRows;
    const int l = threadIdx.x % LPR;
    const int64_t row0 = ((int64_t)blockIdx.x * (kBlock / LPR) + threadIdx.x / kWave * (kWave / LPR)) * R + threadIdx.x % kWave / LPR;
    const T *table = (const T *)a.table;
    const I *ids = (const I *)a.ids;
    int64_t id[R];
    float other[R];                                        // what an id that names no row gives
#pragma unroll
    for (int t = 0; t < R; ++t) id[t] = ids[min(row0 + t * (kWave / LPR), a.n - 1)];
#pragma unroll
    for (int t = 0; t < R; ++t) {
        other[t] = id[t] == a.padding && a.padding != HAG_NO_PADDING ? 0.f : NAN;   // (HAG_NO_PADDING is a number that an id can be)
        if (id[t] < 0 || id[t] >= a.rows || id[t] == a.padding) id[t] = -1;
    }
    for (int col = l * V; col < a.d; col += LPR * V) {
        typename VecOf<T>::type raw[R] = {};
        if (a.rows > 0) {
#pragma unroll
            for (int t = 0; t < R; ++t) raw[t] = load_columns<T, TAIL>(table, (id[t] < 0 ? 0 : id[t]) * a.stride, col, a.d, a.extent);
        }
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const int64_t row = row0 + t * (kWave / LPR);
            if (row >= a.n) continue;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = id[t] < 0 ? other[t] : a.scale * (float)raw[t][e];
            store_vec<true>((T *)a.y + row * a.d + col, TAIL ? a.d - col : V, v);
        }
    }
}

// ------------------------------------------------------------------------------------------------------------------ order of the tokens

// A token's key is its id, `rows` where it names no row: those come last and are left out.  Radix sort, low digits first, with stable passes of up to 10 bits:
// counts per piece of the list, then every piece finds where each of its digits begins (the counts of smaller digits and of earlier pieces) and writes its tokens there.
// Few bytes, so what it costs is the way of a piece through the steps of a pass: many loads at a time, few pieces to look back at.  524288 tokens, 9 bits: counts 5 us, places 12; a
// gradient with pieces of 2048 tokens 121 us, of 4096 (half of the compute units idle) 123, of 1024 (twice as many to look back at) 137.
// Up to kSortShort tokens the tiles are half as long: twice as many compute units have one (12000 tokens of 64 columns 30.5 -> 28.6 us, 30000 34.9 -> 33.5; 370000 36 -> 43).
constexpr int kSortBlock = 1024, kSortWaves = kSortBlock / kWave, kSortBits = 10, kSortPieces = 256;
constexpr int64_t kSortShort = 128 * kSortBlock, kSortAlone = 16 * kSortBlock;     // (so few tokens every piece counts itself)
template <int ROUNDS>                // of 64 tokens that a wavefront takes of a tile
constexpr int kSortTile = kSortBlock * ROUNDS;
template <int ROUNDS>
constexpr int kSortGroup = 8 / ROUNDS;   // pieces that are counted together
template <int ROUNDS>
constexpr int kSortSpace = std::max(2 * kSortTile<ROUNDS>, (kSortWaves << kSortBits) / 2);   // words
static int sort_rounds(int64_t n) { return n <= kSortShort ? 1 : 2; }
struct SortArgs {
    const void *ids;                 // first pass: the tokens' ids
    const uint32_t *keys, *tokens;   // later passes: what the one before wrote
    uint32_t *keys_out, *tokens_out, *counts, *group_counts;
    int64_t n, rows, padding, piece; // tokens of a piece, a multiple of the tile
    int32_t pieces, shift, bits;
};

template <typename I, bool FIRST>
__device__ __forceinline__ uint32_t sort_key(const SortArgs &a, int64_t i) {
    if (!FIRST) return a.keys[i];
    const int64_t id = ((const I *)a.ids)[i];
    return id >= 0 && id < a.rows && id != a.padding ? (uint32_t)id : (uint32_t)a.rows;
}

// lanes whose digit is this lane's, among those of `active`
__device__ __forceinline__ uint64_t equal_digits(uint32_t digit, int bits, uint64_t active) {
    uint32_t lo = (uint32_t)active, hi = (uint32_t)(active >> 32);
#pragma unroll
    for (int b = 0; b < kSortBits; ++b) {
        if (b < bits) {
            const uint32_t set = (uint32_t)((int32_t)(digit << (31 - b)) >> 31);   // all bits of it are bit b
            const uint64_t with = __ballot(set != 0);
            lo &= ~((uint32_t)with ^ set);
            hi &= ~((uint32_t)(with >> 32) ^ set);
        }
    }
    return (uint64_t)hi << 32 | lo;
}

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_zero(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false); }

// sum over the threads before this one; all threads of the workgroup take part
__device__ __forceinline__ uint32_t threads_before(uint32_t v, uint32_t *wave_sum) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    uint32_t sum = v;                                      // of the lanes up to this one: shifts within rows of 16, then the last lanes of rows and of halves
    sum += dpp_or_zero<0x111, 0xf>(sum);
    sum += dpp_or_zero<0x112, 0xf>(sum);
    sum += dpp_or_zero<0x114, 0xf>(sum);
    sum += dpp_or_zero<0x118, 0xf>(sum);
    sum += dpp_or_zero<0x142, 0xa>(sum);
    sum += dpp_or_zero<0x143, 0xc>(sum);
    if (lane == kWave - 1) wave_sum[wave] = sum;
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) before += w < wave ? wave_sum[w] : 0;
    return before + sum - v;
}

// count[digit] of the tokens begin .. end, which `threads` threads share.  The lanes that have the first lane's digit add once: an id that is named most of the time would
// have all 64 wait for each other (370000 tokens of one id: 12 us, so 7).
template <typename I, bool FIRST>
__device__ __forceinline__ void count_digits(const SortArgs &a, int64_t begin, int64_t end, int thread, int threads, uint32_t *count) {
    constexpr int kAsk = 8;
    for (int64_t at = begin + thread; at < end; at += kAsk * threads) {
        uint32_t key[kAsk];
#pragma unroll
        for (int r = 0; r < kAsk; ++r) key[r] = sort_key<I, FIRST>(a, min(at + r * threads, end - 1));
#pragma unroll
        for (int r = 0; r < kAsk; ++r) {
            if (at + r * threads >= end) continue;
            const uint32_t digit = key[r] >> a.shift & ((1u << a.bits) - 1), first = __builtin_amdgcn_readfirstlane(digit);
            const uint64_t same = __ballot(digit == first);
            if (digit != first) atomicAdd(&count[digit], 1u);
            else if ((int)(threadIdx.x % kWave) == __builtin_ctzll(same)) atomicAdd(&count[digit], (uint32_t)__popcll(same));
        }
    }
}

// A workgroup counts a group of pieces, some wavefronts each: `counts` gets the tokens of every digit in the earlier pieces of the group, `group_counts` those of the group.
template <typename I, bool FIRST, int ROUNDS>
__global__ __launch_bounds__(kSortBlock) void sort_count_kernel(SortArgs a) {
    constexpr int kGroup = kSortGroup<ROUNDS>;
    __shared__ uint32_t count[kGroup][1 << kSortBits];
    constexpr int kThreads = kSortBlock / kGroup;
    const int digits = 1 << a.bits, mine = threadIdx.x, k = mine / kThreads;
    if (mine < digits)
#pragma unroll
        for (int q = 0; q < kGroup; ++q) count[q][mine] = 0;
    __syncthreads();
    const int64_t begin = ((int64_t)blockIdx.x * kGroup + k) * a.piece;
    count_digits<I, FIRST>(a, begin, min(begin + a.piece, a.n), mine % kThreads, kThreads, count[k]);
    __syncthreads();
    if (mine >= digits) return;
    uint32_t sum = 0;
#pragma unroll
    for (int q = 0; q < kGroup; ++q) {
        const int p = blockIdx.x * kGroup + q;
        if (p < a.pieces) a.counts[(int64_t)p * digits + mine] = sum;
        sum += count[q][mine];
    }
    a.group_counts[(int64_t)blockIdx.x * digits + mine] = sum;
}

// Within a tile a wavefront takes its tokens in their order, 64 at a time; a token's place in the tile is where its digit begins, plus the tokens of that digit in earlier wavefronts, in
// earlier rounds of its own, and in lower lanes.  The tile is put in that order in LDS first, so that neighbours are written side by side.
template <typename I, bool FIRST, int ROUNDS>
__global__ __launch_bounds__(kSortBlock) void sort_place_kernel(SortArgs a) {
    constexpr int kTile = kSortTile<ROUNDS>, kGroup = kSortGroup<ROUNDS>;
    __shared__ uint32_t space[kSortSpace<ROUNDS>];                 // counts per wavefront and digit, 16 bits each; then the tile's keys and tokens in order
    __shared__ uint32_t base[1 << kSortBits], total[1 << kSortBits], wave_sum[2][kSortWaves];
    uint16_t *count = (uint16_t *)space;
    const int digits = 1 << a.bits, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, mine = threadIdx.x;
    const int64_t begin = (int64_t)blockIdx.x * a.piece, end = min(begin + a.piece, a.n);
    uint32_t key[ROUNDS], token[ROUNDS];
    auto request = [&](int64_t tile) {
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int64_t i = min(tile + (wave * ROUNDS + r) * kWave + lane, end - 1);
            key[r] = sort_key<I, FIRST>(a, i);
            token[r] = FIRST ? (uint32_t)i : a.tokens[i];
        }
    };
    request(begin);
    if (mine < digits) base[mine] = total[mine] = 0;
    __syncthreads();
    // total: tokens of every digit; base: those of earlier pieces
    if (a.n <= kSortAlone) {
        count_digits<I, FIRST>(a, 0, begin, mine, kSortBlock, base);
        count_digits<I, FIRST>(a, begin, a.n, mine, kSortBlock, total);
        __syncthreads();
        if (mine < digits) total[mine] += base[mine];
    } else {
        const int slices = kSortBlock >> a.bits, digit = mine & (digits - 1), groups = (a.pieces + kGroup - 1) / kGroup, own = (int)blockIdx.x / kGroup;
        uint32_t all = 0, before = mine < digits ? a.counts[(int64_t)blockIdx.x * digits + mine] : 0;
        for (int g0 = mine >> a.bits; g0 < groups; g0 += 32 * slices) {
            uint32_t v[32];
#pragma unroll
            for (int u = 0; u < 32; ++u) v[u] = a.group_counts[(int64_t)min(g0 + u * slices, groups - 1) * digits + digit];
#pragma unroll
            for (int u = 0; u < 32; ++u) {
                const int g = g0 + u * slices;
                all += g < groups ? v[u] : 0;
                before += g < own ? v[u] : 0;
            }
        }
        atomicAdd(&total[digit], all);
        atomicAdd(&base[digit], before);
        __syncthreads();
    }
    {
        const uint32_t smaller = threads_before(mine < digits ? total[mine] : 0, wave_sum[0]);
        if (mine < digits) base[mine] += smaller;
    }
    for (int64_t tile = begin; tile < end; tile += kTile) {
        if (tile > begin) request(tile);
        for (int c = mine; c < (kSortWaves << a.bits) / 2; c += kSortBlock) space[c] = 0;
        __syncthreads();
        uint32_t place[ROUNDS];
        uint64_t same[ROUNDS];                        // lanes of the same digit
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
            same[r] = equal_digits(key[r] >> a.shift & (digits - 1), a.bits, __ballot(tile + (wave * ROUNDS + r) * kWave + lane < end));
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {            // the first of them adds them all to the wavefront's count
            const uint32_t at = (uint32_t)wave << a.bits | (key[r] >> a.shift & (digits - 1));
            place[r] = 0;
            if (same[r] && lane == __builtin_ctzll(same[r])) place[r] = atomicAdd(&space[at >> 1], (uint32_t)__popcll(same[r]) << (at & 1) * 16) >> (at & 1) * 16 & 0xffff;
        }
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
            place[r] = __shfl(place[r], same[r] ? __builtin_ctzll(same[r]) : lane) + __popcll(same[r] & ((1ull << lane) - 1));
        __syncthreads();
        uint32_t here = 0;                                 // the tile's tokens of digit `mine`
        if (mine < digits) {
            uint32_t v[kSortWaves];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) v[w] = count[w << a.bits | mine];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                count[w << a.bits | mine] = (uint16_t)here;
                here += v[w];
            }
        }
        const uint32_t smaller = threads_before(here, wave_sum[1]);
        if (mine < digits) {
            total[mine] = smaller;                         // (where the digit begins in the tile)
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const uint32_t digit = key[r] >> a.shift & (digits - 1);
            place[r] += total[digit] + count[wave << a.bits | digit];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
            if (tile + (wave * ROUNDS + r) * kWave + lane < end) {
                space[place[r]] = key[r];
                space[kTile + place[r]] = token[r];
            }
        __syncthreads();
        const int filled = (int)min((int64_t)kTile, end - tile);
        for (int j = mine; j < filled; j += kSortBlock) {
            const uint32_t k = space[j], digit = k >> a.shift & (digits - 1), to = base[digit] + (uint32_t)j - total[digit];
            a.keys_out[to] = k;
            a.tokens_out[to] = space[kTile + j];
        }
        __syncthreads();
        if (mine < digits) base[mine] += here;
    }
}

// Up to kRankMost tokens are put in order by one launch instead of two passes: a token's place is the number of tokens that come before it, counted by comparing it with all of them (2 vector
// instructions for 64 pairs, and LDS for the keys: a gradient of 8192 tokens of 30000 rows 19.7 us where two passes make it 23.3, of 16384 38 and 27; of 300 rows, which take one pass, 4096
// tokens 15.3 both ways, 8192 18.5 and 15.5).  A workgroup places 32 tokens, 16 lanes each, out of all keys in LDS.
constexpr int kRankMost = 8192, kRankTokens = 32, kRankBlock = 512, kRankStreams = kRankBlock / kRankTokens, kRankAsk = kRankMost / kRankBlock;
template <typename I>
__global__ __launch_bounds__(kRankBlock) void sort_rank_kernel(SortArgs a) {
    __shared__ uint4 keys[kRankMost / 4];
    __shared__ uint32_t count[kRankTokens];
    uint32_t *key = (uint32_t *)keys;
    const int n = (int)a.n, vectors = (n + 3) / 4, first = blockIdx.x * kRankTokens, token = threadIdx.x % kRankTokens, stream = threadIdx.x / kRankTokens, i = first + token;
    {
        uint32_t k[kRankAsk];
#pragma unroll
        for (int r = 0; r < kRankAsk; ++r) k[r] = sort_key<I, true>(a, min(r * kRankBlock + (int)threadIdx.x, n - 1));
#pragma unroll
        for (int r = 0; r < kRankAsk; ++r)
            if (r * kRankBlock < 4 * vectors) key[r * kRankBlock + threadIdx.x] = r * kRankBlock + (int)threadIdx.x < n ? k[r] : 0xffffffffu;
    }
    if (threadIdx.x < kRankTokens) count[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t mine = i < n ? key[i] : 0;
    uint32_t before = 0;
#pragma unroll 4
    for (int v = stream; v < vectors; v += kRankStreams) {
        const uint4 k = keys[v];
        const uint32_t limit = mine + (4 * v < first ? 1 : 0);                     // equal keys of the workgroups before this one come first
        before += k.x < limit;
        before += k.y < limit;
        before += k.z < limit;
        before += k.w < limit;
    }
    for (int q = stream; q < token; q += kRankStreams) before += key[first + q] == mine;                 // and those before it in its own
    before += __shfl_xor(before, kRankTokens);
    if (threadIdx.x % kWave < kRankTokens) atomicAdd(&count[token], before);
    __syncthreads();
    if (threadIdx.x < kRankTokens && i < n) {
        a.keys_out[count[token]] = mine;
        a.tokens_out[count[token]] = (uint32_t)i;
    }
}

// ------------------------------------------------------------------------------------------------------------------ sums of sorted tokens

struct GradArgs {
    const void *gy;
    int64_t stride, extent;
    const uint32_t *keys, *tokens;   // sorted
    void *out;
    uint32_t *where;                 // [rows]: for every row that is named, an entry that names it; for others anything
    float *part;                     // [workgroups][2][d]: sums of runs that began before the workgroup's entries, that go on after them
    int64_t n, rows;
    int32_t d, each;                 // entries of a group of lanes
    int32_t groups;                  // workgroups of the sums
    int32_t first;                   // workgroup that this launch begins with
    float scale;
};

// Adds up runs of equal keys among `count` entries in LDS (sorted; keys[-1] is the key before them, keys[count] the one after, kNone where there is none).  Groups of LPR lanes take
// `each` entries one after the other, requesting eight rows ahead; a run inside a group's entries is done there (store), those that cross groups go through LDS
// (edge: [groups of lanes][LPR * V] sums of the run that began earlier and ends in the group or covers it) and are added up by
// the group in which they begin.  open(first, sum): a run that began before the entries (first) or goes on after them.
// Equal pieces keep every lane busy whatever the ids are; a sum for each row of the table would last as long as the id that is named most.
constexpr uint32_t kNone = 0xffffffffu;
template <typename T, int LPR, bool TAIL, typename Store, typename Open>
__device__ __forceinline__ void sum_runs(const T *gy, int64_t stride, int64_t extent, int d, int col, const uint32_t *keys, const uint32_t *tokens, int count, int each, uint32_t rows,
                                         float (*edge)[LPR * kVec<T>], uint8_t *flags, Store store, Open open) {
    constexpr int V = kVec<T>, G = kBlock / LPR, kAhead = 8;
    const int l = threadIdx.x % LPR, g = threadIdx.x / LPR;
    const int begin = min(g * each, count), end = min(begin + each, count);
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.f;
    uint32_t run = begin < end ? keys[begin] : kNone;
    bool inherited = begin < end && keys[begin - 1] == run;         // the run at hand began before this group
    for (int i = begin; i < end; i += kAhead) {
        typename VecOf<T>::type raw[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int at = min(i + u, end - 1);
            raw[u] = load_columns<T, TAIL>(gy, (int64_t)tokens[at] * stride, col, d, extent);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= end) break;
            const uint32_t key = keys[i + u];
            if (key != run) {
                if (inherited) {
#pragma unroll
                    for (int e = 0; e < V; ++e) edge[g][l * V + e] = sum[e];
                } else if (run != rows) {
                    store(run, sum);
                }
                run = key;
                inherited = false;
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += (float)raw[u][e];
        }
    }
    const bool covers = begin < end && inherited;          // one run throughout, which began earlier
    if (covers) {
#pragma unroll
        for (int e = 0; e < V; ++e) edge[g][l * V + e] = sum[e];
    }
    // bit 0: the group's first entry goes on with the run before it; bit 1: one such run covers the group
    if (l == 0) flags[g] = (uint8_t)((begin < end && keys[begin - 1] == keys[begin] ? 1 : 0) | (covers ? 2 : 0));
    __syncthreads();
    const int lane = threadIdx.x % kWave;
    const uint8_t flag = lane < G ? flags[lane] : 0;
    const uint64_t goes_on = __ballot(flag & 1), through = __ballot(flag & 2);
    // the runs that are not done: one that begins in this group and reaches its end, and, for the first group, one that began before all entries
    auto follow = [&](int from, float (&s)[V]) {           // adds groups from, from + 1, ... as far as the run reaches; true: it goes on after the last entry
        // the first group that begins another run, and the first where the run ends inside
        const uint64_t other = from < 64 ? ~goes_on >> from : 1, inside = from < 64 ? ~through >> from : 1;
        const int until = min(from + (other ? __builtin_ctzll(other) : 64), G), last = from + (inside ? __builtin_ctzll(inside) : 64);
        const int stop = min(until, last + 1);
#pragma unroll 4
        for (int h = from; h < stop; ++h)
#pragma unroll
            for (int e = 0; e < V; ++e) s[e] += edge[h][l * V + e];
        return stop == until && until * each >= count && last >= until;
    };
    if (g == 0 && count > 0 && keys[-1] == keys[0] && keys[0] != rows) {
        float s[V];
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] = 0.f;
        follow(0, s);
        open(true, s);
    }
    if (begin < end && !inherited && run != rows) {
        if (follow(g + 1, sum) && keys[count] == run) open(false, sum);
        else store(run, sum);
    }
}

// Bound by reading g_y in the order of the ids: 370000 x 64 fp32 into 74 rows 18 us (5.3 TB/s, what a copy moves), 524288 x 128 into 232965 rows, 512 bytes here and there, 74 to 78 us
// (245 MB in, 105 out, 4.5 TB/s); 4 or 16 rows ahead instead of 8, 16 entries instead of 32: the same.
constexpr int kEachMost = 32;
template <typename T, typename O, int LPR, bool TAIL>
__global__ __launch_bounds__(kBlock) void embed_sum_kernel(GradArgs a) {
    constexpr int V = kVec<T>, G = kBlock / LPR, kMost = G * kEachMost;
    __shared__ uint32_t key_store[kMost + 2], tokens[kMost];
    __shared__ float edge[G][LPR * V];
    __shared__ uint8_t flags[G];
    uint32_t *keys = key_store + 1;
    const int l = threadIdx.x % LPR, col = ((int)blockIdx.y * LPR + l) * V;
    const int64_t block = a.first + (int64_t)blockIdx.x, begin = block * G * a.each;
    const int count = (int)min((int64_t)G * a.each, a.n - begin);
    for (int i = threadIdx.x; i < count; i += 2 * kBlock) {
        const int64_t at = begin + i, then = begin + min(i + kBlock, count - 1);
        const uint32_t k0 = a.keys[at], k1 = a.keys[then], t0 = a.tokens[at], t1 = a.tokens[then];
        keys[i] = k0;
        tokens[i] = t0;
        if (i + kBlock < count) {
            keys[i + kBlock] = k1;
            tokens[i + kBlock] = t1;
        }
    }
    if (threadIdx.x == 0) keys[-1] = begin > 0 ? a.keys[begin - 1] : kNone;
    if (threadIdx.x == kBlock - 1) keys[count] = begin + count < a.n ? a.keys[begin + count] : kNone;
    __syncthreads();
    if (keys[0] == (uint32_t)a.rows) return;               // nothing here names a row
    if (blockIdx.y == 0) {
        for (int i = threadIdx.x; i < count; i += kBlock)
            if (keys[i] != keys[i - 1] && keys[i] != (uint32_t)a.rows) a.where[keys[i]] = (uint32_t)(begin + i);
    }
    sum_runs<T, LPR, TAIL>((const T *)a.gy, a.stride, a.extent, a.d, col, keys, tokens, count, a.each, (uint32_t)a.rows, edge, flags,
        [&](uint32_t row, float (&s)[V]) {
            if (col >= a.d) return;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = a.scale * s[e];
            store_cols((O *)a.out + (int64_t)row * a.d + col, TAIL ? a.d - col : V, v);
        },
        [&](bool first, float (&s)[V]) {
            if (col >= a.d) return;
            store_cols(a.part + (block * 2 + (first ? 0 : 1)) * a.d + col, TAIL ? a.d - col : V, s);
        });
}

// 8 us for those 232965 rows, 4 for 74; 5 us for 232965 rows of 16 columns most of which are zeros.
// The first `groups` - 1 workgroups: the run that begins among the entries of workgroup b of the sums and goes on after them.  The others: 64 rows of g_table for each wavefront, zeros
// where no token names them.
template <typename T, typename O, int LPR, bool TAIL>
__global__ __launch_bounds__(kBlock) void embed_join_kernel(GradArgs a) {
    constexpr int V = kVec<T>, G = kBlock / LPR;
    __shared__ float lds[G][LPR * V];
    const int l = threadIdx.x % LPR, g = threadIdx.x / LPR;
    const int64_t block = a.first + (int64_t)blockIdx.x;
    if (block < a.groups - 1) {
        const int64_t per = (int64_t)G * a.each, begin = block * per, next = begin + per;
        const uint32_t run = a.keys[next - 1], first = a.keys[begin], before = begin > 0 ? a.keys[begin - 1] : kNone, after = a.keys[next];
        // the last workgroup that it reaches: those whose first entry is of this run, 256 looked at a time (the first of them with the loads above)
        int64_t lo = block;
        uint32_t probe = a.keys[min(lo + 1 + threadIdx.x, (int64_t)a.groups - 1) * per];
        if (run == (uint32_t)a.rows || after != run || (first == run && before == run)) return;          // padding; done; began earlier
        for (;;) {
            const int found = __syncthreads_count(lo + 1 + threadIdx.x < a.groups && probe == run);
            lo += found;
            if (found < kBlock) break;
            probe = a.keys[min(lo + 1 + threadIdx.x, (int64_t)a.groups - 1) * per];
        }
        const int col = ((int)blockIdx.y * LPR + l) * V;
        float s[V];
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] = 0.f;
        if (col < a.d) {
            for (int64_t b0 = block + g; b0 <= lo; b0 += 4 * G) {
                float p[4][V];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int64_t b = min(b0 + u * G, lo);
                    const float *q = a.part + (b * 2 + (b == block ? 1 : 0)) * a.d;
#pragma unroll
                    for (int e = 0; e < V; ++e) p[u][e] = q[TAIL ? min(col + e, a.d - 1) : col + e];
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int e = 0; e < V; ++e) s[e] += b0 + u * G <= lo ? p[u][e] : 0.f;
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) lds[g][l * V + e] = s[e];
        __syncthreads();
        if (g > 0 || col >= a.d) return;
        for (int h = 1; h < G && block + h <= lo; ++h)
#pragma unroll
            for (int e = 0; e < V; ++e) s[e] += lds[h][l * V + e];
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] *= a.scale;
        store_cols((O *)a.out + (int64_t)run * a.d + col, TAIL ? a.d - col : V, s);
        return;
    }
    if (blockIdx.y > 0) return;
    const int lane = threadIdx.x % kWave;
    const int64_t row0 = ((block - max(a.groups - 1, 0)) * (kBlock / kWave) + threadIdx.x / kWave) * kWave, row = row0 + lane;
    bool empty = row < a.rows;
    if (empty && a.n > 0) {
        const uint32_t at = a.where[row];
        empty = at >= (uint64_t)a.n || a.keys[at] != (uint32_t)row;
    }
    const float zero[V] = {};
    uint64_t rest = __ballot(empty);
    if (!TAIL && __popcll(rest) >= kWave / 2) {           // most of the rows: as one piece of memory, without the vectors of rows that are named
        O *p = (O *)a.out + row0 * a.d;
        for (uint32_t c = lane * V; c < (uint32_t)(kWave * a.d) && rest; c += kWave * V)
            if (rest >> (c / (uint32_t)a.d) & 1) store_cols(p + c, V, zero);
        return;
    }
    for (; rest; ) {                                       // kWave / LPR of them at a time
        uint64_t mine = rest;
        for (int k = 0; k < lane / LPR; ++k) mine &= mine - 1;
        if (mine) {
            O *p = (O *)a.out + (row0 + __builtin_ctzll(mine)) * a.d;
            for (int col = l * V; col < a.d; col += LPR * V) store_cols(p + col, a.d - col, zero);
        }
        for (int k = 0; k < kWave / LPR; ++k) rest &= rest - 1;
    }
}

// ------------------------------------------------------------------------------------------------------------------ few tokens

// Few tokens: one launch.  A workgroup looks through all ids for those of its 32 rows, sorts them by row in LDS and adds up their runs, which are whole.
// Bound by the busiest workgroup: 9 us (a launch and the host) and 1 us for each 8000 to 10000 elements that its rows get (4000 where d is no multiple of a vector), whatever the other
// compute units do; the path above takes 14 to 16 us, 20 to 35 where many wide rows are empty.  Fewer rows than tokens are categories, of which some are in demand: few tokens of those are what one workgroup
// can take in that time.  As many rows as tokens are names, most of them given once: a workgroup gets few tokens, unless nearly all of them name one row.  fp32, us by this path / that, for ids
// spread evenly and for all of one row:
//   2000 x 64 of 16 rows 19 / 16, 19 / 16    2000 x 128 of 300 10 / 16, 32 / 16     2000 x 1024 of 16 247 / 14, 251 / 17    2000 x 1024 of 300 42 / 16, 249 / 34
//   1000 x 37 of 4096 9.3 / 16, 16 / 17      1000 x 250 of 4096 9.5 / 20, 50 / 21   250 x 1024 of 4096 12 / 33, 40 / 32     2000 x 1024 of 4096 16 / 35, 252 / 35 (a tenth of them one row: 32 / 35)
constexpr int kFew = 2048, kFewRows = 32, kFewRounds = kFew / kBlock;
static bool few_tokens(int64_t n, int64_t rows, int64_t d) { return n <= kFew && (rows >= n || n * d <= 1 << 17); }
template <typename T, typename O, typename I, int LPR, bool TAIL>
__global__ __launch_bounds__(kBlock) void embed_few_kernel(GradArgs a, const I *ids, int64_t padding) {
    constexpr int V = kVec<T>, G = kBlock / LPR, kWaves = kBlock / kWave;
    __shared__ uint32_t key_store[kFew + 2], tokens[kFew], count[kWaves][kFewRows], begins[kFewRows + 1];
    __shared__ float edge[G][LPR * V];
    __shared__ uint8_t flags[G];
    uint32_t *keys = key_store + 1;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, l = threadIdx.x % LPR, g = threadIdx.x / LPR;
    const int64_t row0 = (a.first + (int64_t)blockIdx.x) * kFewRows;
    for (int c = threadIdx.x; c < kWaves * kFewRows; c += kBlock) count[c / kFewRows][c % kFewRows] = 0;
    __syncthreads();
    uint32_t row[kFewRounds], rank[kFewRounds];
    const int n = (int)a.n, rounds = (n + kBlock - 1) / kBlock;    // a wavefront takes so many times 64 tokens
    if (n > 0) {
        int64_t id[kFewRounds];
#pragma unroll
        for (int r = 0; r < kFewRounds; ++r) id[r] = ids[min((wave * rounds + min(r, rounds - 1)) * kWave + lane, n - 1)];
#pragma unroll
        for (int r = 0; r < kFewRounds; ++r) {
            const bool here = r < rounds && (wave * rounds + r) * kWave + lane < n;
            row[r] = here && id[r] >= row0 && id[r] < a.rows && id[r] != padding && id[r] - row0 < kFewRows ? (uint32_t)(id[r] - row0) : kNone;
        }
    } else {
#pragma unroll
        for (int r = 0; r < kFewRounds; ++r) row[r] = kNone;
    }
#pragma unroll
    for (int r = 0; r < kFewRounds; ++r) {
        const bool here = row[r] != kNone;
        const uint64_t any = __ballot(here);
        rank[r] = 0;
        if (!any) continue;
        const uint64_t same = equal_digits(row[r], 5, any);
        const int leader = here ? __builtin_ctzll(same) : lane;
        uint32_t before = 0;
        if (here && lane == leader) before = atomicAdd(&count[wave][row[r]], (uint32_t)__popcll(same));
        rank[r] = __shfl(before, leader) + __popcll(same & ((1ull << lane) - 1));
    }
    __syncthreads();
    if (wave == 0) {
        uint32_t sum = 0;
        if (lane < kFewRows)
            for (int w = 0; w < kWaves; ++w) sum += count[w][lane];
        const uint32_t mine = sum;
#pragma unroll
        for (int off = 1; off < kFewRows; off <<= 1) {
            const uint32_t v = __shfl_up(sum, off);
            sum += lane >= off ? v : 0;
        }
        if (lane < kFewRows) {
            begins[lane + 1] = sum;
            if (lane == 0) begins[0] = 0;
            uint32_t at = sum - mine;
            for (int w = 0; w < kWaves; ++w) {
                const uint32_t v = count[w][lane];
                count[w][lane] = at;
                at += v;
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kFewRounds; ++r)
        if (row[r] != kNone) {
            const uint32_t to = count[wave][row[r]] + rank[r];
            keys[to] = row[r];
            tokens[to] = (uint32_t)((wave * rounds + r) * kWave + lane);
        }
    const int found = (int)begins[kFewRows];
    if (threadIdx.x == 0) keys[-1] = keys[found] = kNone;
    __syncthreads();
    O *out = (O *)a.out + row0 * a.d;
    const float zero[V] = {};
    for (int r = g; r < kFewRows && row0 + r < a.rows; r += G)
        if (begins[r] == begins[r + 1])
            for (int col = l * V; col < a.d; col += LPR * V) store_cols(out + (int64_t)r * a.d + col, a.d - col, zero);
    if (found == 0) return;
    const int each = (found + G - 1) / G;
    for (int col0 = 0; col0 < a.d; col0 += LPR * V) {
        const int col = col0 + l * V;
        sum_runs<T, LPR, TAIL>((const T *)a.gy, a.stride, a.extent, a.d, col, keys, tokens, found, each, kNone, edge, flags,
            [&](uint32_t r, float (&s)[V]) {
                if (col >= a.d) return;
                float v[V];
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = a.scale * s[e];
                store_cols(out + (int64_t)r * a.d + col, TAIL ? a.d - col : V, v);
            },
            [&](bool, float (&)[V]) {});
        __syncthreads();                                   // (edge is used again)
    }
}

// ------------------------------------------------------------------------------------------------------------------ sizes

static int embed_lanes(int64_t d, int vec) {
    int lpr = 4;
    while (lpr < kWave && lpr * vec < d) lpr *= 2;
    return lpr;
}
template <typename F>
static int lanes_switch(int lpr, bool tail, F f) {
    auto with = [&](auto n) { return tail ? f(n, std::true_type()) : f(n, std::false_type()); };
    return lpr == 4    ? with(std::integral_constant<int, 4>())
           : lpr == 8  ? with(std::integral_constant<int, 8>())
           : lpr == 16 ? with(std::integral_constant<int, 16>())
           : lpr == 32 ? with(std::integral_constant<int, 32>())
                       : with(std::integral_constant<int, 64>());
}

// The parts of a gradient's workspace.
struct GradPlan {
    int64_t piece;               // sort
    int32_t pieces, passes, bits;
    int32_t each, groups;        // sums
    size_t lists, counts, where, part, bytes;      // offsets; four lists of n words begin at `lists`
};
template <int ROUNDS>
static int launch_sort_pass(const SortArgs &sort, const GradPlan &p, bool first, hag_dtype_t id_type, hipStream_t s) {
    typedef void (*kernel_t)(SortArgs);
    const bool wide = id_type == HAG_I64;
    const kernel_t count = !first ? (kernel_t)sort_count_kernel<int32_t, false, ROUNDS> : wide ? (kernel_t)sort_count_kernel<int64_t, true, ROUNDS> : (kernel_t)sort_count_kernel<int32_t, true, ROUNDS>;
    const kernel_t place = !first ? (kernel_t)sort_place_kernel<int32_t, false, ROUNDS> : wide ? (kernel_t)sort_place_kernel<int64_t, true, ROUNDS> : (kernel_t)sort_place_kernel<int32_t, true, ROUNDS>;
    if (sort.n > kSortAlone) hipLaunchKernelGGL(count, dim3((unsigned)((p.pieces + kSortGroup<ROUNDS> - 1) / kSortGroup<ROUNDS>)), dim3(kSortBlock), 0, s, sort);
    HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL(place, dim3((unsigned)p.pieces), dim3(kSortBlock), 0, s, sort);
    HIP_TRY(hipGetLastError());
    return HAG_OK;
}
static GradPlan grad_plan(int64_t n, int64_t rows, int64_t d, int vec) {
    GradPlan p = {};
    int key_bits = 1;
    while ((rows >> key_bits) > 0) ++key_bits;
    p.passes = (key_bits + kSortBits - 1) / kSortBits;
    p.bits = (key_bits + p.passes - 1) / p.passes;
    const int64_t tile = (int64_t)kSortBlock * sort_rounds(n), group = 8 / sort_rounds(n);
    p.piece = std::max<int64_t>(1, (n + kSortPieces * tile - 1) / (kSortPieces * tile)) * tile;
    p.pieces = (int32_t)((n + p.piece - 1) / p.piece);
    const int64_t side = kBlock / embed_lanes(d, vec);
    p.each = kEachMost;
    while (p.each > 8 && n < side * p.each * 512) p.each /= 2;
    p.groups = (int32_t)((n + side * p.each - 1) / (side * p.each));
    auto take = [&](size_t bytes) { const size_t at = p.bytes; p.bytes += (bytes + 255) / 256 * 256; return at; };
    p.lists = take((size_t)n * 4 * 4);
    p.counts = take((size_t)(p.pieces + (p.pieces + group - 1) / group) * 4 << p.bits);
    p.where = take((size_t)rows * 4);
    p.part = take((size_t)p.groups * 2 * d * 4);
    return p;
}

}  // namespace hag

using namespace hag;

extern "C" {

// what both calls ask of their sizes
static const char *embed_refusal(int64_t n, int64_t rows, int64_t d, hag_dtype_t id_type, int64_t stride) {
    if (n < 0 || rows < 0 || d <= 0) return "n < 0, rows < 0 or d <= 0";
    if (n > 0x7fffffffLL || rows > 0x7fffffffLL || d > (1 << 20)) return "n and rows must be below 2^31, d at most 2^20";
    if (id_type != HAG_I32 && id_type != HAG_I64) return "ids are HAG_I32 or HAG_I64";
    if (stride < 0) return "negative row stride";
    return nullptr;
}

int hag_embedding(int64_t n, int64_t rows, int64_t d, hag_dtype_t dtype, const void *table, int64_t table_stride, hag_dtype_t id_type, const void *ids,
                  int64_t padding, float scale, void *y, void *stream) {
    if (const char *why = embed_refusal(n, rows, d, id_type, table_stride)) { set_error(why); return HAG_EINVAL; }
    if (!elem_type(dtype)) { set_error("elements are HAG_F32, HAG_BF16 or HAG_F16"); return HAG_EINVAL; }
    if (n == 0) return HAG_OK;
    if ((rows > 0 && !table) || !ids || !y) { set_error("NULL pointer"); return HAG_EINVAL; }
    const EmbedArgs a = {table, ids, y, table_stride, rows > 0 ? (rows - 1) * table_stride + d : 0, n, rows, padding, (int32_t)d, scale};
    return elem_switch(dtype, [&](auto e) {
        return id_switch(id_type, [&](auto k) {
            using T = decltype(e);
            using I = decltype(k);
            return lanes_switch(embed_lanes(d, kVec<T>), d % kVec<T> != 0, [&](auto lanes, auto tail) {
                constexpr int LPR = decltype(lanes)::value;
                constexpr int64_t kRows = kBlock / LPR * kEmbedRows;
                return launch_parts((n + kRows - 1) / kRows, kBlock, [&](int64_t first, int64_t count) {
                    EmbedArgs part = a;
                    part.ids = (const I *)ids + first * kRows;
                    part.y = (T *)y + first * kRows * d;
                    part.n = std::min(count * kRows, n - first * kRows);
                    hipLaunchKernelGGL((embed_kernel<T, I, LPR, decltype(tail)::value>), dim3((unsigned)count), dim3(kBlock), 0, (hipStream_t)stream, part);
                });
            });
        });
    });
}

size_t hag_embedding_grad_workspace_bytes(int64_t n, int64_t rows, int64_t d) {
    if (embed_refusal(n, rows, d, HAG_I64, 0)) return 0;
    return few_tokens(n, rows, d) ? 16 : std::max(grad_plan(n, rows, d, 4).bytes, grad_plan(n, rows, d, 8).bytes);
}

int hag_embedding_grad(int64_t n, int64_t rows, int64_t d, hag_dtype_t dtype, const void *g_y, int64_t g_y_stride, hag_dtype_t id_type, const void *ids, int64_t padding,
                       float scale, hag_dtype_t out_dtype, void *g_table, void *workspace, void *stream) {
    if (const char *why = embed_refusal(n, rows, d, id_type, g_y_stride)) { set_error(why); return HAG_EINVAL; }
    if (!elem_type(dtype) || (out_dtype != dtype && out_dtype != HAG_F32)) {
        set_error("elements are HAG_F32, HAG_BF16 or HAG_F16, those of g_table the same or HAG_F32");
        return HAG_EINVAL;
    }
    if (rows == 0) return HAG_OK;
    if ((n > 0 && (!g_y || !ids)) || !g_table || !workspace) { set_error("NULL pointer"); return HAG_EINVAL; }
    if ((uintptr_t)workspace & 15) { set_error("workspace must be 16-byte aligned"); return HAG_EINVAL; }
    hipStream_t s = (hipStream_t)stream;
    GradArgs a = {};
    a.gy = g_y;
    a.stride = g_y_stride;
    a.extent = n > 0 ? (n - 1) * g_y_stride + d : 0;
    a.out = g_table;
    a.n = n;
    a.rows = rows;
    a.d = (int32_t)d;
    a.scale = scale;
    const int vec = 16 / elem_size(dtype), lpr = embed_lanes(d, vec);
    const bool tail = d % vec != 0;
    const unsigned chunks = (unsigned)((d + lpr * vec - 1) / (lpr * vec));
    // f(type of g_y, of g_table, lanes, tail)
    auto pick = [&](auto f) {
        return elem_switch(dtype, [&](auto e) {
            return lanes_switch(lpr, tail, [&](auto lanes, auto tails) { return out_dtype == dtype ? f(e, e, lanes, tails) : f(e, float(), lanes, tails); });
        });
    };
    if (few_tokens(n, rows, d))
        return pick([&](auto e, auto o, auto lanes, auto tails) {
            return id_switch(id_type, [&](auto k) {
                using I = decltype(k);
                return launch_parts((rows + kFewRows - 1) / kFewRows, kBlock, [&](int64_t first, int64_t count) {
                    a.first = (int32_t)first;
                    hipLaunchKernelGGL((embed_few_kernel<decltype(e), decltype(o), I, decltype(lanes)::value, decltype(tails)::value>), dim3((unsigned)count), dim3(kBlock), 0, s, a,
                                       (const I *)ids, padding);
                });
            });
        });
    const GradPlan p = grad_plan(n, rows, d, vec);
    char *ws = (char *)workspace;
    uint32_t *lists = (uint32_t *)(ws + p.lists);
    SortArgs sort = {};
    sort.ids = ids;
    sort.counts = (uint32_t *)(ws + p.counts);
    sort.group_counts = sort.counts + ((size_t)p.pieces << p.bits);
    sort.n = n;
    sort.rows = rows;
    sort.padding = padding;
    sort.piece = p.piece;
    sort.pieces = p.pieces;
    sort.bits = p.bits;
    if (n <= kRankMost) {
        sort.keys_out = lists;
        sort.tokens_out = lists + n;
        const dim3 grid((unsigned)((n + kRankTokens - 1) / kRankTokens));
        if (id_type == HAG_I64) hipLaunchKernelGGL(sort_rank_kernel<int64_t>, grid, dim3(kRankBlock), 0, s, sort);
        else hipLaunchKernelGGL(sort_rank_kernel<int32_t>, grid, dim3(kRankBlock), 0, s, sort);
        HIP_TRY(hipGetLastError());
    }
    for (int pass = 0; n > kRankMost && pass < p.passes; ++pass) {
        sort.shift = pass * p.bits;
        sort.keys = sort.keys_out;
        sort.tokens = sort.tokens_out;
        sort.keys_out = lists + (pass & 1) * 2 * n;
        sort.tokens_out = sort.keys_out + n;
        if (const int rc = sort_rounds(n) == 1 ? launch_sort_pass<1>(sort, p, pass == 0, id_type, s) : launch_sort_pass<2>(sort, p, pass == 0, id_type, s)) return rc;
    }
    a.keys = sort.keys_out;
    a.tokens = sort.tokens_out;
    a.where = (uint32_t *)(ws + p.where);
    a.part = (float *)(ws + p.part);
    a.each = p.each;
    a.groups = p.groups;
    const int64_t joins = p.groups - 1 + (rows + kBlock - 1) / kBlock;
    return pick([&](auto e, auto o, auto lanes, auto tails) {
        using T = decltype(e);
        using O = decltype(o);
        constexpr int LPR = decltype(lanes)::value;
        constexpr bool TAIL = decltype(tails)::value;
        const int rc = launch_parts(p.groups, kBlock, [&](int64_t first, int64_t count) {
            a.first = (int32_t)first;
            hipLaunchKernelGGL((embed_sum_kernel<T, O, LPR, TAIL>), dim3((unsigned)count, chunks), dim3(kBlock), 0, s, a);
        });
        if (rc != HAG_OK) return rc;
        return launch_parts(joins, kBlock, [&](int64_t first, int64_t count) {
            a.first = (int32_t)first;
            hipLaunchKernelGGL((embed_join_kernel<T, O, LPR, TAIL>), dim3((unsigned)count, chunks), dim3(kBlock), 0, s, a);
        });
    });
}

}  // extern "C"
