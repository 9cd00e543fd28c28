// Rows of an embedding table for a batch of tokens, and the table's gradient: the rows of equal tokens summed.
//
// The gradient of a few tokens is one launch, in which every workgroup looks for its token among all of them.  More are sorted by row first (stable, so
// that equal tokens stand in the order of the batch), cut into pieces of a few tokens whatever rows they belong to (a text's most frequent token may be a tenth of
// it), and the sums of rows that go over the end of a piece are joined in a launch of their own.  No sum is formed by atomics.
#include "rdk_vec.hpp"

namespace rdk {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kCols = 8;                 // columns of a thread
constexpr int kAhead = 8;                // rows on their way at a time

// ---- eight columns of a row of either type

template <int TYPE>
struct Cols {
    typedef Vec<TYPE> V;
    static constexpr int kVecs = kCols / V::kLen;
    u32x4 r[kVecs];

    // columns col .. of a row, of which `left` belong to it (what stands for the others is not used)
    __device__ __forceinline__ void load(const void *row, int col, int left)
    {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) r[i] = left > i * V::kLen ? V::load_at((const char *)row + (int64_t)col * V::kSize, i * 16, left - i * V::kLen) : V::fill();
    }
    __device__ __forceinline__ void to(float (&v)[kCols]) const
    {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            float part[V::kLen];
            V::to(r[i], part);
#pragma unroll
            for (int e = 0; e < V::kLen; ++e) v[i * V::kLen + e] = part[e];
        }
    }
    static __device__ __forceinline__ void store(void *row, int col, int left, const float (&v)[kCols])
    {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            float part[V::kLen];
#pragma unroll
            for (int e = 0; e < V::kLen; ++e) part[e] = v[i * V::kLen + e];
            if (left > i * V::kLen) V::store_at((char *)row + (int64_t)col * V::kSize, i * 16, left - i * V::kLen, V::from(part));
        }
    }
};

// The table's row of a token, -1 for one that it does not hold.
struct Rows {
    const int32_t *slot_of;   // or NULL: ids are rows
    int ids;                  // ids below this are known there
    __device__ __forceinline__ int of(int id) const { return id < 0 || id >= ids ? -1 : slot_of ? max(slot_of[id], -1) : id; }
};

// ---- lookup

struct EmbedArgs {
    Rows rows;
    const int32_t *ids;
    const void *table;
    void *out;
    int64_t ldt, ldo;
    int B, d, shift;          // 2^shift threads side by side on a row
    float scale;
};

// Every thread takes its eight columns of ROWS rows, all of which are asked for before the first is written.
template <int TABLE, int OUT, int ROWS>
__global__ __launch_bounds__(kThreads) void embed_kernel(EmbedArgs a)
{
    const int across = 1 << a.shift, down = kThreads >> a.shift;
    const int col = ((int)blockIdx.y * across + (int)(threadIdx.x & (across - 1))) * kCols, left = a.d - col;
    const int first = (int)blockIdx.x * (down * ROWS) + (int)(threadIdx.x >> a.shift);   // (B < 2^24: no overflow)
    if (left <= 0) return;
    int row[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) row[j] = first + j * down < a.B ? a.rows.of(a.ids[first + j * down]) : -1;
    Cols<TABLE> raw[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j)
        if (row[j] >= 0) raw[j].load(row_ptr<TABLE>(a.table, a.ldt, row[j]), col, left);
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        if (first + j * down >= a.B) break;
        float v[kCols];
        raw[j].to(v);
#pragma unroll
        for (int e = 0; e < kCols; ++e) v[e] = row[j] >= 0 ? v[e] * a.scale : 0.f;
        Cols<OUT>::store(const_cast<void *>(row_ptr<OUT>(a.out, a.ldo, first + j * down)), col, left, v);
    }
}

// ---- gradient

constexpr int kShares = 256;      // of the tokens that are sorted, a workgroup each

// What stands for a row among 0 .. V (V: a token that the table does not hold, behind all others) when rows are sorted; bits: of V.
struct SortOrder {
    int high;                 // bits above the lowest eight
    uint32_t V;
    __host__ __device__ __forceinline__ uint32_t of(uint32_t row) const
    {
        return row >= V ? (uint32_t)kShares << high : (row & (kShares - 1)) << high | row >> 8;
    }
    __device__ __forceinline__ uint32_t row(uint32_t key) const { return key >> high >= (uint32_t)kShares ? V : (key & ((1u << high) - 1)) << 8 | key >> high; }
};

struct EmbedGradArgs {
    Rows rows;
    const int32_t *ids;
    const void *d_out;
    void *d_table;
    int64_t ldo, ldt;
    int B, V, d, accumulate;
    float scale;
    int blocks, shift;        // workgroups along a row; 2^shift threads side by side on a row
    int fill_rows, fills;     // rows of the table that a workgroup sets to 0 where no token names them, and workgroups that do
    // sorted: tokens by row
    SortOrder order;
    const uint32_t *key;      // [B] what stands for the row
    const int32_t *at;        // [B] the token
    int piece, pieces;        // tokens of a piece
    float *partial;           // [pieces, 2, d]: sums of a row that begins before the piece; of one that begins in it and goes on behind it
};

// A sum into the table.
template <int TABLE>
__device__ __forceinline__ void write_sum(const EmbedGradArgs &a, int row, int col, int left, float (&v)[kCols])
{
    void *to = const_cast<void *>(row_ptr<TABLE>(a.d_table, a.ldt, row));
    float old[kCols];
    if (a.accumulate) {
        Cols<TABLE> raw;
        raw.load(to, col, left);
        raw.to(old);
    }
#pragma unroll
    for (int e = 0; e < kCols; ++e) v[e] = a.accumulate ? fmaf(v[e], a.scale, old[e]) : v[e] * a.scale;
    Cols<TABLE>::store(to, col, left, v);
}

// Sets rows first .. first + count - 1 (at most 64) of the table to 0 where `named` has no bit, by the threads of a workgroup.
template <int TABLE>
__device__ __forceinline__ void clear_rows(const EmbedGradArgs &a, int first, int count, uint64_t named)
{
    const float zero[kCols] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int units = (a.d - 1) / kCols + 1;
    int r = 0, u = threadIdx.x;
    while (true) {   // all units of the rows one behind the other
        while (u >= units && r < count) {
            u -= units;
            ++r;
        }
        if (r >= count) break;
        if (!(named >> r & 1)) Cols<TABLE>::store(const_cast<void *>(row_ptr<TABLE>(a.d_table, a.ldt, first + r)), u * kCols, a.d - u * kCols, zero);
        u += kThreads;
    }
}

constexpr int kFewTokens = 1024;   // that a workgroup looks through
constexpr int kFewEach = kFewTokens / kThreads;

struct FewShared {
    int list[kFewTokens];
    int count[kFewEach * kWaves];
    unsigned long long named;
};

// The gradient of a few tokens in one launch.  A workgroup to a token: it sums the rows of all tokens like its own if it is the first of them.  The
// workgroups behind these set the rows that no token names to 0.
template <int OUT, int TABLE>
__global__ __launch_bounds__(kThreads) void embed_grad_few_kernel(EmbedGradArgs a)
{
    __shared__ FewShared sh;
    __shared__ float sums[kThreads][kCols + 1];
    const int tid = threadIdx.x;
    int mine[kFewEach];
#pragma unroll
    for (int j = 0; j < kFewEach; ++j) mine[j] = j * kThreads + tid < a.B ? a.ids[j * kThreads + tid] : -1;
    if ((int)blockIdx.x >= a.B) {
        const int first = ((int)blockIdx.x - a.B) * a.fill_rows, count = min(a.fill_rows, a.V - first);
        if (tid == 0) sh.named = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kFewEach; ++j) {
            const int r = a.rows.of(mine[j]) - first;
            if (r >= 0 && r < count) atomicOr(&sh.named, 1ull << r);
        }
        __syncthreads();
        clear_rows<TABLE>(a, first, count, sh.named);
        return;
    }
    const int b = blockIdx.x, id = a.ids[b], row = a.rows.of(id);
    if (row < 0) return;
    // the tokens like it in the order of the batch
    uint64_t like[kFewEach];
    int n = 0, before = 0;
#pragma unroll
    for (int j = 0; j < kFewEach; ++j) {
        like[j] = __ballot(j * kThreads + tid < a.B && mine[j] == id);
        if (lane_id() == 0) sh.count[j * kWaves + tid / kWave] = __popcll(like[j]);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kFewEach; ++j) {
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w == tid / kWave) {
                before = n;
                if (like[j] >> lane_id() & 1) sh.list[before + __popcll(like[j] & (((uint64_t)1 << lane_id()) - 1))] = j * kThreads + tid;
            }
            n += sh.count[j * kWaves + w];
        }
    }
    __syncthreads();
    if (sh.list[0] != b) return;
    const int across = 1 << a.shift, down = kThreads >> a.shift, x = tid & (across - 1), y = tid >> a.shift;
    const int units = (a.d - 1) / kCols + 1;
    for (int u0 = 0; u0 < units; u0 += across) {
        const int col = (u0 + x) * kCols, left = a.d - col;
        float acc[kCols] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (left > 0) {
#pragma unroll 1
            for (int i = y; i < n; i += down * kAhead) {
                Cols<OUT> raw[kAhead];
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (i + j * down < n) raw[j].load(row_ptr<OUT>(a.d_out, a.ldo, sh.list[i + j * down]), col, left);
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (i + j * down < n) {
                        float v[kCols];
                        raw[j].to(v);
#pragma unroll
                        for (int e = 0; e < kCols; ++e) acc[e] += v[e];
                    }
            }
        }
        if (down > 1 && n > 1) {   // (alike for the workgroup)
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kCols; ++e) sums[tid][e] = acc[e];
            __syncthreads();
            if (y == 0)
                for (int w = 1; w < min(down, n); ++w)
#pragma unroll
                    for (int e = 0; e < kCols; ++e) acc[e] += sums[w * across + x][e];
        }
        if (y == 0 && left > 0) write_sum<TABLE>(a, row, col, left, acc);
    }
}

// ---- tokens sorted by row, each row's in the order of the batch
//
// Rows are ordered by their lowest eight bits first (SortOrder), whatever order the table has: where frequent tokens have neighbouring ids, as
// tokenizers give them, the workgroups that sort by these bits have shares of one size.

constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr int kSortRounds = 20;                       // tokens of a thread
constexpr int kSortTokens = kSortThreads * kSortRounds;
// The place of a token: places[digit] is that of the wavefront's next token of a digit, and grows by those of the round.
__device__ __forceinline__ uint32_t place_next(uint32_t digit, volatile uint32_t *places)
{
    uint32_t lo = ~0u, hi = ~0u;
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
        const uint64_t on = __ballot(digit >> b & 1);
        const uint32_t other = (uint32_t)__builtin_amdgcn_sbfe((int)~digit, b, 1);   // all ones where the lane's bit is 0
        lo &= (uint32_t)on ^ other;
        hi &= (uint32_t)(on >> 32) ^ other;
    }
    const uint64_t like = (uint64_t)hi << 32 | lo;
    const uint32_t first = places[digit], before = (uint32_t)__popcll(like & (((uint64_t)1 << lane_id()) - 1));
    __builtin_amdgcn_wave_barrier();
    if (before == 0) places[digit] = first + (uint32_t)__popcll(like);   // one lane of those alike
    __builtin_amdgcn_wave_barrier();
    return first + before;
}

__device__ __forceinline__ uint32_t wave_scan(uint32_t v)   // inclusive
{
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t u = __shfl_up(v, o);
        if (lane_id() >= o) v += u;
    }
    return v;
}

// counts[w][digit] of the wavefronts become the places where their tokens of that digit begin: behind `base` (the digit's; NULL: all tokens of the
// lower digits) and the wavefronts before.  All threads call it.
template <int WAVES>
__device__ __forceinline__ void place_counts(uint32_t (*counts)[kDigits], uint32_t *totals, const uint32_t *base, int base_stride)
{
    const int tid = threadIdx.x;
    constexpr int kT = WAVES * kWave;
    static_assert(kDigits == 8 * kWave, "eight digits to a lane");
    if (!base) {
        for (int g = tid; g < kDigits; g += kT) {
            uint32_t sum = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) sum += counts[w][g];
            totals[g] = sum;
        }
        __syncthreads();
        if (tid < kWave) {   // eight digits a lane
            uint32_t own[8], sum = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                own[e] = totals[tid * 8 + e];
                sum += own[e];
            }
            uint32_t before = wave_scan(sum) - sum;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                totals[tid * 8 + e] = before;
                before += own[e];
            }
        }
        __syncthreads();
    }
    for (int g = tid; g < kDigits; g += kT) {
        uint32_t own[WAVES], at = base ? base[(int64_t)g * base_stride] : totals[g];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) own[w] = counts[w][g];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            counts[w][g] = at;
            at += own[w];
        }
    }
    __syncthreads();
}

struct SortArgs {
    Rows rows;
    const int32_t *ids;
    int B, passes;
    SortOrder order;
    uint32_t *key;
    int32_t *at;
    // of more tokens than one workgroup holds
    const uint32_t *key_in;   // NULL: from ids
    const int32_t *at_in;
    int shift, tiles;
    uint32_t *table;          // [digits, tiles]
};

__device__ __forceinline__ uint32_t key_of(const SortArgs &a, int b)
{
    const int row = a.rows.of(a.ids[b]);
    return a.order.of(row < 0 ? a.order.V : (uint32_t)row);
}

struct SortShared {
    uint32_t key[kSortTokens];
    uint16_t at[kSortTokens];
    uint32_t counts[kSortWaves][kDigits];
    uint32_t totals[kDigits];
    uint32_t waves[kSortWaves][2];
};

// Up to 20480 tokens in one launch.  Every workgroup reads the keys of all, takes those of its share (the highest bits of the key) in their order, counts those
// of lower shares, which come before them, and sorts its own by the bits that are left: a pass of nine bits for tables of up to 2^17 rows.  Tokens that the
// table does not hold are a share of their own, in order already.
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(SortArgs a)
{
    extern __shared__ __align__(16) char lds[];
    SortShared &sh = *(SortShared *)lds;
    const int tid = threadIdx.x, wid = tid / kWave, rounds = (a.B - 1) / kSortThreads + 1;
    const int first = wid * rounds * kWave + lane_id();   // a wavefront's tokens stand together
    const uint32_t share = blockIdx.x;
    uint32_t key[kSortRounds];
    uint32_t mine = 0, lower = 0;
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
        if (r < rounds) {
            const int b = first + r * kWave;
            key[r] = b < a.B ? key_of(a, b) : 0xFFFFFFFFu;
        }
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
        if (r < rounds) {
            mine += key[r] >> a.order.high == share;
            lower += key[r] >> a.order.high < share;
        }
    mine = (uint32_t)wave_sum((float)mine);   // (at most 1280 a wavefront: exact)
    lower = (uint32_t)wave_sum((float)lower);
    if (lane_id() == 0) {
        sh.waves[wid][0] = mine;
        sh.waves[wid][1] = lower;
    }
    __syncthreads();
    uint32_t before = 0, n = 0, base = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        if (w < wid) before += sh.waves[w][0];
        n += sh.waves[w][0];
        base += sh.waves[w][1];
    }
    if (n == 0) return;
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
        if (r < rounds) {
            const uint64_t who = __ballot(key[r] >> a.order.high == share);
            if (who >> lane_id() & 1) {
                const uint32_t to = before + __popcll(who & (((uint64_t)1 << lane_id()) - 1));
                sh.key[to] = key[r];
                sh.at[to] = (uint16_t)(first + r * kWave);
            }
            before += __popcll(who);
        }
    __syncthreads();
    if (share >= (uint32_t)kShares || a.passes == 0) {
        for (int i = tid; i < (int)n; i += kSortThreads) {
            a.key[base + i] = sh.key[i];
            a.at[base + i] = sh.at[i];
        }
        return;
    }
    const int own_rounds = ((int)n - 1) / kSortThreads + 1, own_first = wid * own_rounds * kWave + lane_id();
#pragma unroll 1
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * kDigitBits, bits = min(a.order.high - shift, kDigitBits);
        const uint32_t mask = (1u << bits) - 1;
        for (int i = tid; i < kSortWaves * kDigits; i += kSortThreads) (&sh.counts[0][0])[i] = 0;
        __syncthreads();
#pragma unroll 1
        for (int r = 0; r < own_rounds; ++r) {
            const int i = own_first + r * kWave;
            if (i < (int)n) atomicAdd(&sh.counts[wid][sh.key[i] >> shift & mask], 1u);
        }
        __syncthreads();
        place_counts<kSortWaves>(sh.counts, sh.totals, nullptr, 0);
#pragma unroll 1
        for (int r = 0; r < own_rounds; ++r) {
            const int i = own_first + r * kWave;
            const uint32_t k = i < (int)n ? sh.key[i] : 0xFFFFFFFFu;
            const uint32_t to = base + place_next(k >> shift & mask, sh.counts[wid]);   // (those behind the last token come last, and are not written)
            if (i < (int)n) {
                a.key[to] = k;
                a.at[to] = sh.at[i];
            }
        }
        __syncthreads();
        if (pass + 1 == a.passes) return;
        for (int i = tid; i < (int)n; i += kSortThreads) {   // (what this workgroup wrote)
            sh.key[i] = a.key[base + i];
            sh.at[i] = (uint16_t)a.at[base + i];
        }
        __syncthreads();
    }
}

constexpr int kTileRounds = 16, kTile = kThreads * kTileRounds;

// Tokens of every digit in a tile.
__global__ __launch_bounds__(kThreads) void embed_count_kernel(SortArgs a)
{
    __shared__ uint32_t counts[kDigits];
    const int tile = blockIdx.x;
    for (int g = threadIdx.x; g < kDigits; g += kThreads) counts[g] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kTileRounds; ++r) {
        const int b = tile * kTile + r * kThreads + (int)threadIdx.x;
        if (b < a.B) atomicAdd(&counts[(a.key_in ? a.key_in[b] : key_of(a, b)) >> a.shift & (kDigits - 1)], 1u);
    }
    __syncthreads();
    for (int g = threadIdx.x; g < kDigits; g += kThreads) a.table[(int64_t)g * a.tiles + tile] = counts[g];
}

// Counts become places: exclusive sums over [digits, tiles], by one workgroup.
__global__ __launch_bounds__(kSortThreads) void embed_scan_kernel(SortArgs a)
{
    __shared__ uint32_t waves[kSortWaves];
    const int total = kDigits * a.tiles, each = (total - 1) / kSortThreads + 1;   // (B < 2^24: at most 2^21)
    const int begin = min((int)threadIdx.x * each, total), end = min(begin + each, total);
    uint32_t sum = 0;
#pragma unroll 8
    for (int i = begin; i < end; ++i) sum += a.table[i];
    const uint32_t upto = wave_scan(sum);
    if (lane_id() == kWave - 1) waves[threadIdx.x / kWave] = upto;
    __syncthreads();
    uint32_t before = upto - sum;
    for (int w = 0; w < (int)threadIdx.x / kWave; ++w) before += waves[w];
#pragma unroll 8
    for (int i = begin; i < end; ++i) {
        const uint32_t c = a.table[i];
        a.table[i] = before;
        before += c;
    }
}

// Tokens of a tile to their places.
__global__ __launch_bounds__(kThreads) void embed_place_kernel(SortArgs a)
{
    __shared__ uint32_t counts[kWaves][kDigits], totals[kDigits];
    const int tile = blockIdx.x, wid = threadIdx.x / kWave, first = tile * kTile + wid * kTileRounds * kWave + lane_id();
    for (int i = threadIdx.x; i < kWaves * kDigits; i += kThreads) (&counts[0][0])[i] = 0;
    __syncthreads();
    uint32_t key[kTileRounds];
#pragma unroll
    for (int r = 0; r < kTileRounds; ++r) {
        const int b = first + r * kWave;
        key[r] = b >= a.B ? 0xFFFFFFFFu : a.key_in ? a.key_in[b] : key_of(a, b);
        if (b < a.B) atomicAdd(&counts[wid][key[r] >> a.shift & (kDigits - 1)], 1u);
    }
    __syncthreads();
    place_counts<kWaves>(counts, totals, a.table + tile, a.tiles);
#pragma unroll
    for (int r = 0; r < kTileRounds; ++r) {
        const int b = first + r * kWave;
        const uint32_t to = place_next(key[r] >> a.shift & (kDigits - 1), counts[wid]);   // (those behind the last token come last, and are not written)
        if (b < a.B) {
            a.key[to] = key[r];
            a.at[to] = a.at_in ? a.at_in[b] : b;
        }
    }
}

// ---- sums over sorted tokens

// The rows of a piece of the sorted tokens by the threads side by side on a row; behind the pieces workgroups that set rows without tokens to 0.
template <int OUT, int TABLE>
__global__ __launch_bounds__(kThreads) void embed_grad_sum_kernel(EmbedGradArgs a)
{
    const int across = 1 << a.shift, down = kThreads >> a.shift, tid = threadIdx.x;
    const int sum_blocks = ((a.pieces - 1) / down + 1) * a.blocks;
    if ((int)blockIdx.x >= sum_blocks) {
        __shared__ unsigned long long named;
        const int first = ((int)blockIdx.x - sum_blocks) * a.fill_rows, count = min(a.fill_rows, a.V - first);
        if (tid < kWave) {
            bool is = false;
            if (tid < count) {   // the first token that is not below the row
                const uint32_t key = a.order.of((uint32_t)(first + tid));
                int lo = 0, hi = a.B;
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (a.key[mid] < key) lo = mid + 1;
                    else hi = mid;
                }
                is = lo < a.B && a.key[lo] == key;
            }
            const uint64_t who = __ballot(is);
            if (tid == 0) named = who;
        }
        __syncthreads();
        clear_rows<TABLE>(a, first, count, named);
        return;
    }
    const int piece = (int)blockIdx.x / a.blocks * down + (tid >> a.shift);
    const int col = ((int)blockIdx.x % a.blocks * across + (tid & (across - 1))) * kCols, left = a.d - col;
    if (piece >= a.pieces || left <= 0) return;
    const int begin = piece * a.piece, end = min(begin + a.piece, a.B);
    const uint32_t none = a.order.of(a.order.V);
    uint32_t run = a.key[begin];
    if (run >= none) return;
    bool head = begin > 0 && a.key[begin - 1] == run;   // the run at hand began before the piece
    float acc[kCols] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto keep = [&](int which) {
        float *to = a.partial + ((int64_t)piece * 2 + which) * a.d + col;
#pragma unroll
        for (int e = 0; e < kCols; ++e)
            if (e < left) to[e] = acc[e];
    };
#pragma unroll 1
    for (int i = begin; i < end; i += kAhead) {
        uint32_t key[kAhead];
        Cols<OUT> raw[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            key[j] = i + j < end ? a.key[i + j] : none;
            if (key[j] < none) raw[j].load(row_ptr<OUT>(a.d_out, a.ldo, a.at[i + j]), col, left);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (i + j >= end || run >= none) break;
            if (key[j] != run) {   // the run ends within the piece
                if (head) keep(0);
                else write_sum<TABLE>(a, (int)a.order.row(run), col, left, acc);
                head = false;
                run = key[j];
#pragma unroll
                for (int e = 0; e < kCols; ++e) acc[e] = 0.f;
                if (run >= none) break;
            }
            float v[kCols];
            raw[j].to(v);
#pragma unroll
            for (int e = 0; e < kCols; ++e) acc[e] += v[e];
        }
    }
    if (run >= none) return;
    if (head) keep(0);
    else if (end < a.B && a.key[end] == run) keep(1);
    else write_sum<TABLE>(a, (int)a.order.row(run), col, left, acc);
}

// The sums of a row that goes over the end of a piece, brought together by a workgroup to the piece where it begins: threads side by side on
// the row, in several groups that take every so manieth piece.
template <int TABLE>
__global__ __launch_bounds__(kThreads) void embed_grad_join_kernel(EmbedGradArgs a)
{
    __shared__ float sums[kThreads][kCols + 1];
    const int piece = (int)blockIdx.x / a.blocks, begin = piece * a.piece, end = begin + a.piece, tid = threadIdx.x;
    if (end >= a.B) return;
    const uint32_t run = a.key[end - 1];
    if (run >= a.order.of(a.order.V) || a.key[end] != run) return;
    if (a.key[begin] == run && begin > 0 && a.key[begin - 1] == run) return;   // it begins before this piece
    const int across = 1 << a.shift, down = kThreads >> a.shift, x = tid & (across - 1), y = tid >> a.shift;
    const int col = ((int)blockIdx.x % a.blocks * across + x) * kCols, left = a.d - col;
    int last = piece + 1;   // the last piece that the run reaches
    while (true) {          // (every wavefront for itself: 64 pieces at a time)
        const int next = (last + 1 + lane_id()) * a.piece;   // (B < 2^24 and pieces of at most 32: no overflow)
        const uint64_t on = __ballot(next < a.B && a.key[min(next, a.B - 1)] == run);
        const int more = ~on ? __ffsll((unsigned long long)~on) - 1 : kWave;
        last += more;
        if (more < kWave) break;
    }
    float acc[kCols] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int n = last - piece + 1;
    if (left > 0) {
#pragma unroll 1
        for (int i = y; i < n; i += down * kAhead) {
            Cols<RDK_F32> raw[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int p = i + j * down;
                if (p < n) raw[j].load(a.partial + ((int64_t)(piece + p) * 2 + (p == 0)) * a.d, col, left);
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (i + j * down < n) {
                    float v[kCols];
                    raw[j].to(v);
#pragma unroll
                    for (int e = 0; e < kCols; ++e) acc[e] += v[e];
                }
        }
    }
    if (down > 1) {
#pragma unroll
        for (int e = 0; e < kCols; ++e) sums[tid][e] = acc[e];
        __syncthreads();
        if (y == 0)
            for (int w = 1; w < min(down, n); ++w)
#pragma unroll
                for (int e = 0; e < kCols; ++e) acc[e] += sums[w * across + x][e];
    }
    if (y == 0 && left > 0) write_sum<TABLE>(a, (int)a.order.row(run), col, left, acc);
}

// ---- host

// log2 of the threads side by side on a row: as many as its columns take, up to `most`.
int threads_across(int d, int most)
{
    const int units = (d - 1) / kCols + 1;
    int shift = 0;
    while ((1 << shift) < units && (1 << shift) < most) ++shift;
    return shift;
}

struct GradPlan {
    bool few;
    int shift, blocks;
    int piece, pieces;
    SortOrder order;
    int tiles, passes;
    size_t key, at, key2, at2, table, partial, bytes;   // places in the workspace
};

GradPlan plan_of(const rdk_embed_desc_t &d)
{
    GradPlan p{};
    p.few = d.B <= kFewTokens;
    if (p.few) {
        p.shift = threads_across(d.d, kThreads);
        return p;
    }
    p.shift = threads_across(d.d, kWave);
    p.blocks = (d.d - 1) / ((1 << p.shift) * kCols) + 1;
    // Pieces as long as leaves enough of them to fill the chip.
    const int64_t waves = ((int64_t)d.B * p.blocks << p.shift) / kWave;   // with pieces of one token
    p.piece = 32;
    while (p.piece > 4 && waves / p.piece < 4096) p.piece >>= 1;
    p.pieces = (d.B - 1) / p.piece + 1;
    int bits = 8;
    while (((d.V - 1) >> bits) != 0) ++bits;                             // of rows
    p.order = SortOrder{bits - 8, (uint32_t)d.V};
    // all bits of the keys over tiles, or those that a share is sorted by
    p.passes = d.B > kSortTokens ? bits / kDigitBits + 1 : (bits - 8 + kDigitBits - 1) / kDigitBits;
    p.tiles = d.B > kSortTokens ? (d.B - 1) / kTile + 1 : 0;
    size_t at = 0;
    auto room = [&](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes, 256);
        return here;
    };
    p.key = room((size_t)d.B * 4);
    p.at = room((size_t)d.B * 4);
    if (p.tiles) {
        p.key2 = room((size_t)d.B * 4);
        p.at2 = room((size_t)d.B * 4);
        p.table = room((size_t)kDigits * p.tiles * 4);
    }
    p.partial = room((size_t)p.pieces * 2 * d.d * 4);
    p.bytes = at;
    return p;
}

template <class F>
void with_type(rdk_float_t type, const F &f)
{
    if (type == RDK_F32) f(std::integral_constant<int, RDK_F32>());
    else f(std::integral_constant<int, RDK_BF16>());
}

Rows rows_of(const rdk_embed_desc_t &d, const KernelHandle *h) { return Rows{h ? h->slot_of : nullptr, h ? h->N : d.V}; }

LdsGrant sort_grant;

rdk_status_t launch_sort(SortArgs s, const GradPlan &p, char *ws, hipStream_t st)
{
    if (!p.tiles) {
        const rdk_status_t rc = sort_grant((const void *)embed_sort_kernel, sizeof(SortShared));
        if (rc != RDK_OK) return rc;
        RDK_TIMED_LAUNCH("embed_sort_kernel", embed_sort_kernel, dim3(kShares + 1), dim3(kSortThreads), sizeof(SortShared), st, s);
        RDK_LAUNCH_CHECK("embed_sort_kernel");
        return RDK_OK;
    }
    // passes write to the other buffers in turn, the last one to those that are read later
    uint32_t *const key[2] = {s.key, (uint32_t *)(ws + p.key2)};
    int32_t *const at[2] = {s.at, (int32_t *)(ws + p.at2)};
    s.tiles = p.tiles;
    s.table = (uint32_t *)(ws + p.table);
    for (int pass = 0; pass < p.passes; ++pass) {
        const int to = (p.passes - 1 - pass) & 1;
        s.shift = pass * kDigitBits;
        s.key_in = pass ? key[to ^ 1] : nullptr;
        s.at_in = pass ? at[to ^ 1] : nullptr;
        s.key = key[to];
        s.at = at[to];
        RDK_TIMED_LAUNCH("embed_count_kernel", embed_count_kernel, dim3((unsigned)p.tiles), dim3(kThreads), 0, st, s);
        RDK_TIMED_LAUNCH("embed_scan_kernel", embed_scan_kernel, dim3(1), dim3(kSortThreads), 0, st, s);
        RDK_TIMED_LAUNCH("embed_place_kernel", embed_place_kernel, dim3((unsigned)p.tiles), dim3(kThreads), 0, st, s);
    }
    RDK_LAUNCH_CHECK("embed_place_kernel");
    return RDK_OK;
}

}  // namespace

rdk_status_t launch_embed(const rdk_embed_desc_t &d, const KernelHandle *h, const int32_t *ids, const void *table, rdk_float_t table_type, int64_t ldt,
                          void *out, rdk_float_t out_type, int64_t ldo, hipStream_t st)
{
    EmbedArgs a{};
    a.rows = rows_of(d, h);
    a.ids = ids; a.table = table; a.out = out; a.ldt = ldt; a.ldo = ldo;
    a.B = d.B; a.d = d.d; a.scale = d.scale;
    a.shift = threads_across(d.d, kThreads);
    const int across = 1 << a.shift, down = kThreads >> a.shift;
    const int blocks = (d.d - 1) / (across * kCols) + 1;
    const bool many = (int64_t)d.B * blocks / down >= 4096;
    const int rows = down * (many ? 4 : 1);
    const dim3 grid((unsigned)((d.B - 1) / rows + 1), (unsigned)blocks);
    with_type(table_type, [&](auto t) {
        with_type(out_type, [&](auto o) {
            constexpr int T = decltype(t)::value, O = decltype(o)::value;
            if (many) RDK_TIMED_LAUNCH("embed_kernel", (embed_kernel<T, O, 4>), grid, dim3(kThreads), 0, st, a);
            else RDK_TIMED_LAUNCH("embed_kernel", (embed_kernel<T, O, 1>), grid, dim3(kThreads), 0, st, a);
        });
    });
    RDK_LAUNCH_CHECK("embed_kernel");
    return RDK_OK;
}

size_t embed_grad_workspace_bytes(const rdk_embed_desc_t &d) { return plan_of(d).bytes; }

rdk_status_t launch_embed_grad(const rdk_embed_desc_t &d, const KernelHandle *h, const int32_t *ids, const void *d_out, rdk_float_t out_type,
                               int64_t ldo, void *d_table, rdk_float_t table_type, int64_t ldt, bool accumulate, void *ws, hipStream_t st)
{
    const GradPlan p = plan_of(d);
    EmbedGradArgs a{};
    a.rows = rows_of(d, h);
    a.ids = ids; a.d_out = d_out; a.d_table = d_table; a.ldo = ldo; a.ldt = ldt;
    a.B = d.B; a.V = d.V; a.d = d.d; a.accumulate = accumulate; a.scale = d.scale;
    a.shift = p.shift; a.blocks = p.blocks; a.piece = p.piece; a.pieces = p.pieces;
    a.fill_rows = 64;
    while (a.fill_rows > 8 && (d.V - 1) / a.fill_rows + 1 < 2048) a.fill_rows >>= 1;
    a.fills = accumulate ? 0 : (d.V - 1) / a.fill_rows + 1;
    char *const w = (char *)ws;
    if (!p.few) {
        SortArgs s{};
        s.rows = a.rows;
        s.ids = ids; s.B = d.B; s.order = p.order; s.passes = p.passes;
        s.key = (uint32_t *)(w + p.key);
        s.at = (int32_t *)(w + p.at);
        a.order = p.order; a.key = s.key; a.at = s.at;
        a.partial = (float *)(w + p.partial);
        const rdk_status_t rc = launch_sort(s, p, w, st);
        if (rc != RDK_OK) return rc;
    }
    with_type(out_type, [&](auto o) {
        with_type(table_type, [&](auto t) {
            constexpr int O = decltype(o)::value, T = decltype(t)::value;
            if (p.few) {
                RDK_TIMED_LAUNCH("embed_grad_few_kernel", (embed_grad_few_kernel<O, T>), dim3((unsigned)(d.B + a.fills)), dim3(kThreads), 0, st, a);
                return;
            }
            const int sums = ((p.pieces - 1) / (kThreads >> p.shift) + 1) * p.blocks;
            RDK_TIMED_LAUNCH("embed_grad_sum_kernel", (embed_grad_sum_kernel<O, T>), dim3((unsigned)(sums + a.fills)), dim3(kThreads), 0, st, a);
            RDK_TIMED_LAUNCH("embed_grad_join_kernel", (embed_grad_join_kernel<T>), dim3((unsigned)(p.pieces * p.blocks)), dim3(kThreads), 0, st, a);
        });
    });
    RDK_LAUNCH_CHECK("embed_grad_sum_kernel");
    return RDK_OK;
}

}  // namespace rdk
