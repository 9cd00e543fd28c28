// Rows of an embedding table for a batch of tokens, and the table's gradient: the rows of equal tokens summed.
//
// The gradient of a few tokens is one launch, in which every workgroup looks for its token among all of them.  More are sorted by row first (stable, so
// that equal tokens stand in the order of the batch), cut into pieces of a few tokens whatever rows they belong to (a text's most frequent token may be a tenth of
// it), and the sums of rows that go over the end of a piece are joined in a launch of their own.  No sum is formed by atomics.
#include <algorithm>
#include <cstddef>

#include "rdk_vec.hpp"

namespace rdk {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kAhead = 8;                // rows on their way at a time

// ---- columns of a row, a thread's next to one another: eight where both sides are bf16, four where one is fp32, so that the threads side by side
// read and write whole lines with every access (eight fp32 values a thread, in two accesses of every other 16 bytes: rows of 8192 tokens of 4096 72 us, 36 this way)

template <int A, int B>
constexpr int kColumns = A == RDK_BF16 && B == RDK_BF16 ? 8 : 4;

template <int TYPE, int N>
struct Cols {
    static constexpr int kSize = TYPE == RDK_BF16 ? 2 : 4, kWords = N * kSize / 4;
    typedef uint32_t Words __attribute__((ext_vector_type(kWords)));
    typedef uint32_t WordsAny __attribute__((ext_vector_type(kWords), aligned(kSize)));
    Words r;

    // columns col .. of a row, of which `left` belong to it (the others are 0)
    __device__ __forceinline__ void load(const void *row, int col, int left)
    {
        const char *p = (const char *)row + (int64_t)col * kSize;
        if (left >= N) {
            r = *(const WordsAny *)p;
            return;
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i) r[i] = 0;
#pragma unroll
        for (int e = 0; e < N - 1; ++e)
            if (e < left) {
                if constexpr (TYPE == RDK_BF16) r[e / 2] |= (uint32_t)((const uint16_t *)p)[e] << (e % 2 * 16);
                else r[e] = ((const uint32_t *)p)[e];
            }
    }
    __device__ __forceinline__ void to(float (&v)[N]) const
    {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if constexpr (TYPE == RDK_BF16) v[e] = __uint_as_float(e % 2 ? r[e / 2] & 0xFFFF0000u : r[e / 2] << 16);
            else v[e] = __uint_as_float(r[e]);
        }
    }
    // rounded to the nearest, ties to even; non-temporal: tables are larger than the caches
    static __device__ __forceinline__ void store(void *row, int col, int left, const float (&v)[N])
    {
        Words w;
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (TYPE == RDK_BF16) {
                typedef float f2 __attribute__((ext_vector_type(2)));
                typedef __bf16 b2 __attribute__((ext_vector_type(2)));
                w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{v[2 * i], v[2 * i + 1]}, b2));
            } else {
                w[i] = __float_as_uint(v[i]);
            }
        }
        char *p = (char *)row + (int64_t)col * kSize;
        if (left >= N) {
            __builtin_nontemporal_store(w, (WordsAny *)p);
            return;
        }
#pragma unroll
        for (int e = 0; e < N - 1; ++e)
            if (e < left) {
                if constexpr (TYPE == RDK_BF16) ((uint16_t *)p)[e] = (uint16_t)(w[e / 2] >> (e % 2 * 16));
                else ((uint32_t *)p)[e] = w[e];
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

// Every thread takes its columns of ROWS rows, all of which are asked for before the first is written.  HBM: 8192 bf16 rows of 4096 17.8 us = 6.2 TB/s of what has to
// move (frequent tokens' rows once), fp32 34; 8 rows 3.1 to 3.7 us, a launch.
template <int TABLE, int OUT, int ROWS>
__global__ __launch_bounds__(kThreads) void embed_kernel(EmbedArgs a)
{
    constexpr int N = kColumns<TABLE, OUT>;
    const int across = 1 << a.shift, down = kThreads >> a.shift;
    const int col = ((int)blockIdx.y * across + (int)(threadIdx.x & (across - 1))) * N, left = a.d - col;
    const int first = (int)blockIdx.x * (down * ROWS) + (int)(threadIdx.x >> a.shift);   // (B < 2^24: no overflow)
    if (left <= 0) return;
    int row[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) row[j] = first + j * down < a.B ? a.rows.of(a.ids[first + j * down]) : -1;
    Cols<TABLE, N> raw[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j)
        if (row[j] >= 0) raw[j].load(row_ptr<TABLE>(a.table, a.ldt, row[j]), col, left);
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        if (first + j * down >= a.B) break;
        float v[N];
        raw[j].to(v);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = row[j] >= 0 ? v[e] * a.scale : 0.f;
        Cols<OUT, N>::store(const_cast<void *>(row_ptr<OUT>(a.out, a.ldo, first + j * down)), col, left, v);
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
    int units;                // threads that the columns of a row take
    // sorted: tokens by row
    SortOrder order;
    const uint32_t *key;      // [B] what stands for the row
    const int32_t *at;        // [B] the token
    int piece, pieces;        // tokens of a piece
    float4 *partial;          // [pieces, 2, N / 4, units]: sums of a row that begins before the piece; of one that begins in it and goes on behind it
};

// A sum into the table.
template <int TABLE, int N>
__device__ __forceinline__ void write_sum(const EmbedGradArgs &a, int row, int col, int left, float (&v)[N], const Cols<TABLE, N> *before = nullptr)
{
    void *to = const_cast<void *>(row_ptr<TABLE>(a.d_table, a.ldt, row));
    float old[N];
    if (a.accumulate) {
        Cols<TABLE, N> raw;
        if (before) raw = *before;   // read ahead
        else raw.load(to, col, left);
        raw.to(old);
    }
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = a.accumulate ? fmaf(v[e], a.scale, old[e]) : v[e] * a.scale;
    Cols<TABLE, N>::store(to, col, left, v);
}

// Sets rows first .. first + count - 1 (at most 64) of the table to 0 where `named` has no bit, by the threads of a workgroup.
template <int TABLE>
__device__ __forceinline__ void clear_rows(const EmbedGradArgs &a, int first, int count, uint64_t named)
{
    constexpr int N = kColumns<TABLE, TABLE>;
    float zero[N];
#pragma unroll
    for (int e = 0; e < N; ++e) zero[e] = 0.f;
    const int units = (a.d - 1) / N + 1;
    int r = 0, u = threadIdx.x;
    while (true) {   // all units of the rows one behind the other
        while (u >= units && r < count) {
            u -= units;
            ++r;
        }
        if (r >= count) break;
        if (!(named >> r & 1)) Cols<TABLE, N>::store(const_cast<void *>(row_ptr<TABLE>(a.d_table, a.ldt, first + r)), u * N, a.d - u * N, zero);
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
// workgroups behind these set the rows that no token names to 0.  Bound by its chain for small tables (301 tokens into 7999 x 515 fp32 6.9 us: ids, search and sum one after
// the other) and by HBM's writing for large ones (1024 tokens into 128256 x 2048 bf16 105 us = 5.0 TB/s).
template <int OUT, int TABLE>
__global__ __launch_bounds__(kThreads) void embed_grad_few_kernel(EmbedGradArgs a)
{
    constexpr int N = kColumns<OUT, TABLE>;
    __shared__ FewShared sh;
    __shared__ float sums[kThreads][N + 1];
    const int tid = threadIdx.x;
    int mine[kFewEach];
#pragma unroll
    for (int j = 0; j < kFewEach; ++j) mine[j] = j * kThreads + tid < a.B ? a.ids[j * kThreads + tid] : -1;
    if ((int)blockIdx.x >= a.B * a.blocks) {
        const int first = ((int)blockIdx.x - a.B * a.blocks) * a.fill_rows, count = min(a.fill_rows, a.V - first);
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
    const int b = (int)blockIdx.x / a.blocks, id = a.ids[b], row = a.rows.of(id);
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
    const int col = ((int)blockIdx.x % a.blocks * across + x) * N, left = a.d - col;
    float acc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
    if (left > 0) {
#pragma unroll 1
        for (int i = y; i < n; i += down * kAhead) {
            Cols<OUT, N> raw[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (i + j * down < n) raw[j].load(row_ptr<OUT>(a.d_out, a.ldo, sh.list[i + j * down]), col, left);
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (i + j * down < n) {
                    float v[N];
                    raw[j].to(v);
#pragma unroll
                    for (int e = 0; e < N; ++e) acc[e] += v[e];
                }
        }
    }
    if (n > 1) {   // (alike for the workgroup)
#pragma unroll
        for (int e = 0; e < N; ++e) sums[tid][e] = acc[e];
        __syncthreads();
        if (y == 0)
            for (int w = 1; w < min(down, n); ++w)
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] += sums[w * across + x][e];
    }
    if (y == 0 && left > 0) write_sum<TABLE, N>(a, row, col, left, acc);
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

// counts[w][digit] of the wavefronts become the places where their tokens of that digit begin: behind all tokens of the lower digits, those of the digit in
// tiles before (`before`, NULL: there are none) and in the wavefronts before.  all: tokens of every digit (NULL: those in counts).  All threads call it.
template <int WAVES>
__device__ __forceinline__ void place_counts(uint32_t (*counts)[kDigits], uint32_t *totals, const uint32_t *all, const uint32_t *before, int stride)
{
    const int tid = threadIdx.x;
    constexpr int kT = WAVES * kWave;
    static_assert(kDigits == 8 * kWave, "eight digits to a lane");
    for (int g = tid; g < kDigits; g += kT) {
        uint32_t sum = 0;
        if (all) {
            sum = all[g];
        } else {
#pragma unroll
            for (int w = 0; w < WAVES; ++w) sum += counts[w][g];
        }
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
        uint32_t lower = wave_scan(sum) - sum;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            totals[tid * 8 + e] = lower;
            lower += own[e];
        }
    }
    __syncthreads();
    for (int g = tid; g < kDigits; g += kT) {
        uint32_t own[WAVES], at = totals[g] + (before ? before[(int64_t)g * stride] : 0);
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
    uint32_t *table;          // [digits, tiles], and behind them the digits' sums
};

struct SortShared {
    uint32_t counts[kSortWaves][kDigits];
    uint32_t totals[kDigits];
    uint32_t waves[kSortWaves][2];
    uint32_t key[1];   // of all tokens, and behind them as many 16-bit places in the batch
};
inline size_t sort_bytes(int B) { return offsetof(SortShared, key) + align_up((size_t)B, 8) * 6; }

// Up to 20480 tokens in one launch.  Every workgroup reads the keys of all, takes those of its share (the highest bits of the key) in their order, counts those
// of lower shares, which come before them, and sorts its own by the bits that are left: a pass of nine bits for tables of up to 2^17 rows.  Tokens that the
// table does not hold are a share of their own, in order already.  A chain: 16384 tokens 12 us, whose keys (64 KB) every workgroup reads out of its L2.
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(SortArgs a)
{
    extern __shared__ __align__(16) char lds[];
    SortShared &sh = *(SortShared *)lds;
    uint16_t *const sh_at = (uint16_t *)(sh.key + ((a.B + 7) & ~7));
    const int tid = threadIdx.x, wid = tid / kWave, rounds = (a.B - 1) / kSortThreads + 1;
    const int first = wid * rounds * kWave + lane_id();   // a wavefront's tokens stand together
    const uint32_t share = blockIdx.x;
    uint32_t key[kSortRounds];
    uint32_t mine = 0, lower = 0;
    // (all ids on their way, then all rows: one by one they would be waited for)
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
        if (r < rounds) key[r] = (uint32_t)a.ids[min(first + r * kWave, a.B - 1)];
    if (a.rows.slot_of) {
        int slot[kSortRounds];
#pragma unroll
        for (int r = 0; r < kSortRounds; ++r)
            if (r < rounds) slot[r] = a.rows.slot_of[min(key[r], (uint32_t)a.rows.ids - 1)];
#pragma unroll
        for (int r = 0; r < kSortRounds; ++r)
            if (r < rounds && key[r] < (uint32_t)a.rows.ids) key[r] = (uint32_t)slot[r];   // (a pruned id: a negative number)
    }
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
        if (r < rounds) {
            key[r] = first + r * kWave < a.B ? a.order.of(min(key[r], a.order.V)) : 0xFFFFFFFFu;   // (ids that the table does not hold are V or more, read without a sign)
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
                sh_at[to] = (uint16_t)(first + r * kWave);
            }
            before += __popcll(who);
        }
    __syncthreads();
    if (share >= (uint32_t)kShares || a.passes == 0) {
        for (int i = tid; i < (int)n; i += kSortThreads) {
            a.key[base + i] = sh.key[i];
            a.at[base + i] = sh_at[i];
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
        place_counts<kSortWaves>(sh.counts, sh.totals, nullptr, nullptr, 0);
#pragma unroll 1
        for (int r = 0; r < own_rounds; ++r) {
            const int i = own_first + r * kWave;
            const uint32_t k = i < (int)n ? sh.key[i] : 0xFFFFFFFFu;
            const uint32_t to = base + place_next(k >> shift & mask, sh.counts[wid]);   // (those behind the last token come last, and are not written)
            if (i < (int)n) {
                a.key[to] = k;
                a.at[to] = sh_at[i];
            }
        }
        __syncthreads();
        if (pass + 1 == a.passes) return;
        for (int i = tid; i < (int)n; i += kSortThreads) {   // (what this workgroup wrote)
            sh.key[i] = a.key[base + i];
            sh_at[i] = (uint16_t)a.at[base + i];
        }
        __syncthreads();
    }
}

// More tokens: tiles of them, in three launches a pass.  Small tiles, of which there are enough to fill the chip; larger ones where a wavefront would
// have many of them to go through.  (262144 tokens into 128256 x 512 bf16 153 us, 65536 into 32064 x 4096 212, all launches together.)
constexpr int kSmallRounds = 4, kLargeRounds = 16, kSmallTiles = 512;
inline int tile_rounds(int B) { return B <= kSmallTiles * kThreads * kSmallRounds ? kSmallRounds : kLargeRounds; }

// The keys of a tile, ROUNDS of a thread: those of a wavefront stand together.  (All on their way at once.)
template <int ROUNDS>
__device__ __forceinline__ void tile_keys(const SortArgs &a, uint32_t (&key)[ROUNDS], int first)
{
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int b = min(first + r * kWave, a.B - 1);
        key[r] = a.key_in ? a.key_in[b] : (uint32_t)a.ids[b];
    }
    if (!a.key_in) {
        if (a.rows.slot_of) {
            int slot[ROUNDS];
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r) slot[r] = a.rows.slot_of[min(key[r], (uint32_t)a.rows.ids - 1)];
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r)
                if (key[r] < (uint32_t)a.rows.ids) key[r] = (uint32_t)slot[r];   // (a pruned id: a negative number)
        }
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) key[r] = a.order.of(min(key[r], a.order.V));   // (ids that the table does not hold are V or more, read without a sign)
    }
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
        if (first + r * kWave >= a.B) key[r] = 0xFFFFFFFFu;
}

// Tokens of every digit in a tile.
template <int ROUNDS>
__global__ __launch_bounds__(kThreads) void embed_count_kernel(SortArgs a)
{
    __shared__ uint32_t counts[kDigits];
    const int tile = blockIdx.x, first = tile * kThreads * ROUNDS + (int)threadIdx.x / kWave * ROUNDS * kWave + lane_id();
    for (int g = threadIdx.x; g < kDigits; g += kThreads) counts[g] = 0;
    uint32_t key[ROUNDS];
    tile_keys(a, key, first);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
        if (first + r * kWave < a.B) atomicAdd(&counts[key[r] >> a.shift & (kDigits - 1)], 1u);
    __syncthreads();
    for (int g = threadIdx.x; g < kDigits; g += kThreads) a.table[(int64_t)g * a.tiles + tile] = counts[g];
}

// The tiles' counts of a digit become those of the tiles before, by a wavefront each; the digit's own is kept behind them.
__global__ __launch_bounds__(kWave) void embed_scan_kernel(SortArgs a)
{
    uint32_t *const own = a.table + (int64_t)blockIdx.x * a.tiles;
    uint32_t sum = 0;
    for (int first = 0; first < a.tiles; first += kWave) {
        const int t = first + lane_id();
        const uint32_t c = t < a.tiles ? own[t] : 0, upto = wave_scan(c);
        if (t < a.tiles) own[t] = sum + upto - c;
        sum += (uint32_t)lane_value((int)upto, kWave - 1);
    }
    if (lane_id() == 0) a.table[(int64_t)kDigits * a.tiles + blockIdx.x] = sum;
}

// Tokens of a tile to their places.
template <int ROUNDS>
__global__ __launch_bounds__(kThreads) void embed_place_kernel(SortArgs a)
{
    __shared__ uint32_t counts[kWaves][kDigits], totals[kDigits];
    const int tile = blockIdx.x, wid = threadIdx.x / kWave, first = tile * kThreads * ROUNDS + wid * ROUNDS * kWave + lane_id();
    for (int i = threadIdx.x; i < kWaves * kDigits; i += kThreads) (&counts[0][0])[i] = 0;
    uint32_t key[ROUNDS];
    int at[ROUNDS];
    tile_keys(a, key, first);
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) at[r] = a.at_in ? a.at_in[min(first + r * kWave, a.B - 1)] : first + r * kWave;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
        if (first + r * kWave < a.B) atomicAdd(&counts[wid][key[r] >> a.shift & (kDigits - 1)], 1u);
    __syncthreads();
    place_counts<kWaves>(counts, totals, a.table + (int64_t)kDigits * a.tiles, a.table + tile, a.tiles);
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const uint32_t to = place_next(key[r] >> a.shift & (kDigits - 1), counts[wid]);   // (those behind the last token come last, and are not written)
        if (first + r * kWave < a.B) {
            a.key[to] = key[r];
            a.at[to] = at[r];
        }
    }
}

// ---- sums over sorted tokens

constexpr int kStaged = 1024, kLeastShift = 3, kMostPiece = 32;   // tokens of a workgroup of pieces
static_assert((kThreads >> kLeastShift) * kMostPiece <= kStaged, "what a workgroup's threads side by side on rows sum");

// Where a thread keeps a partial sum: the first four columns of all threads of a row stand together, then the other four.
template <int N>
__device__ __forceinline__ int64_t partial_place(const EmbedGradArgs &a, int64_t piece, int which, int col)
{
    return (piece * 2 + which) * (N / 4) * a.units + col / N;
}

// The rows of a piece of the sorted tokens by the threads side by side on a row; behind the pieces workgroups that set rows without tokens to 0.  HBM: 16384 bf16 rows into
// 128256 x 2048 100 to 106 us = 5.6 to 5.9 TB/s read and written, most of it zeros; added to what
// the table holds 43 with the sort and the join.
template <int OUT, int TABLE, bool ADD>
__global__ __launch_bounds__(kThreads) void embed_grad_sum_kernel(EmbedGradArgs a)
{
    constexpr int N = kColumns<OUT, TABLE>;
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
    // the workgroup's keys and tokens, the keys before and behind them too
    __shared__ uint32_t keys[kStaged + 2];
    __shared__ int tokens[kStaged];
    const int first = (int)blockIdx.x / a.blocks * down, base = first * a.piece, count = min(down * a.piece, a.B - base);
    for (int i = tid; i < count; i += kThreads) {
        keys[i + 1] = a.key[base + i];
        tokens[i] = a.at[base + i];
    }
    if (tid == 0) keys[0] = base > 0 ? a.key[base - 1] : ~0u;
    if (tid == 1) keys[count + 1] = base + count < a.B ? a.key[base + count] : ~0u;
    __syncthreads();
    const int piece = first + (tid >> a.shift);
    const int col = ((int)blockIdx.x % a.blocks * across + (tid & (across - 1))) * N, left = a.d - col;
    if (piece >= a.pieces || left <= 0) return;
    const uint32_t none = a.order.of(a.order.V), *const key = keys + 1;
    const int begin = (tid >> a.shift) * a.piece, end = min(begin + a.piece, count);   // among the workgroup's
    uint32_t run = key[begin];
    if (run >= none) return;
    bool head = key[begin - 1] == run;   // the run at hand began before the piece
    float acc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
    auto keep = [&](int which) __attribute__((always_inline)) {
        float4 *to = a.partial + partial_place<N>(a, piece, which, col);
#pragma unroll
        for (int e = 0; e < N; e += 4) to[(int64_t)(e / 4) * a.units] = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
    };
    // A ring: a row is asked for as soon as the one in its place is added; with ADD so is what the table holds where a run ends.
    Cols<OUT, N> raw[kAhead];
    Cols<TABLE, N> old[ADD ? kAhead : 1];
    auto ask = [&](int j, int i) __attribute__((always_inline)) {
        if (i >= end || key[i] >= none) return;
        raw[j].load(row_ptr<OUT>(a.d_out, a.ldo, tokens[i]), col, left);
        if constexpr (ADD)
            if (key[i + 1] != key[i]) old[j].load(row_ptr<TABLE>(a.d_table, a.ldt, (int)a.order.row(key[i])), col, left);
    };
#pragma unroll
    for (int j = 0; j < kAhead; ++j) ask(j, begin + j);
#pragma unroll 1
    for (int i = begin; i < end; i += kAhead) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (i + j >= end || run >= none) break;
            float v[N];
            raw[j].to(v);
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] += v[e];
            if (key[i + j + 1] != run) {   // the run ends here
                if (head) keep(0);
                else write_sum<TABLE, N>(a, (int)a.order.row(run), col, left, acc, ADD ? &old[j] : nullptr);
                head = false;
                run = i + j + 1 < end ? key[i + j + 1] : none;
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] = 0.f;
            } else if (i + j + 1 == end) {   // or goes on behind the piece
                keep(head ? 0 : 1);
            }
            ask(j, i + j + kAhead);
        }
    }
}

// The sums of a row that goes over the end of a piece, brought together by a workgroup to the piece where it begins: threads side by side on
// the row, in several groups that take every so manieth piece.  (5 us of 16384 tokens by Zipf's law: their first token goes over some dozens of pieces.)
template <int TABLE, int N>
__global__ __launch_bounds__(kThreads) void embed_grad_join_kernel(EmbedGradArgs a)
{
    __shared__ float sums[kThreads][N + 1];
    const int piece = (int)blockIdx.x / a.blocks, begin = piece * a.piece, end = begin + a.piece, tid = threadIdx.x;
    if (end >= a.B) return;
    const uint32_t run = a.key[end - 1];
    if (run >= a.order.of(a.order.V) || a.key[end] != run) return;
    if (a.key[begin] == run && begin > 0 && a.key[begin - 1] == run) return;   // it begins before this piece
    const int across = 1 << a.shift, down = kThreads >> a.shift, x = tid & (across - 1), y = tid >> a.shift;
    const int col = ((int)blockIdx.x % a.blocks * across + x) * N, left = a.d - col;
    int last = piece + 1;   // the last piece that the run reaches
    while (true) {          // (every wavefront for itself: 64 pieces at a time)
        const int next = (last + 1 + lane_id()) * a.piece;   // (B < 2^24 and pieces of at most 32: no overflow)
        const uint64_t on = __ballot(next < a.B && a.key[min(next, a.B - 1)] == run);
        const int more = ~on ? __ffsll((unsigned long long)~on) - 1 : kWave;
        last += more;
        if (more < kWave) break;
    }
    float acc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
    const int n = last - piece + 1;
    if (left > 0) {
#pragma unroll 1
        for (int i = y; i < n; i += down * kAhead) {
            float4 raw[kAhead][N / 4];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int p = i + j * down;
                if (p < n) {
                    const float4 *from = a.partial + partial_place<N>(a, piece + p, p == 0, col);
#pragma unroll
                    for (int e = 0; e < N / 4; ++e) raw[j][e] = from[(int64_t)e * a.units];
                }
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (i + j * down < n) {
#pragma unroll
                    for (int e = 0; e < N / 4; ++e) {
                        acc[4 * e] += raw[j][e].x;
                        acc[4 * e + 1] += raw[j][e].y;
                        acc[4 * e + 2] += raw[j][e].z;
                        acc[4 * e + 3] += raw[j][e].w;
                    }
                }
        }
    }
    if (down > 1) {
#pragma unroll
        for (int e = 0; e < N; ++e) sums[tid][e] = acc[e];
        __syncthreads();
        if (y == 0)
            for (int w = 1; w < min(down, n); ++w)
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] += sums[w * across + x][e];
    }
    if (y == 0 && left > 0) write_sum<TABLE, N>(a, (int)a.order.row(run), col, left, acc);
}

// ---- host

// log2 of the threads side by side on a row: as many as its units take, up to `most`.
int threads_across(int units, int most)
{
    int shift = 0;
    while ((1 << shift) < units && (1 << shift) < most) ++shift;
    return shift;
}

struct GradPlan {
    bool few;
    int units, shift, blocks;
    int piece, pieces;
    SortOrder order;
    int tiles, passes;
    size_t key, at, key2, at2, table, partial, bytes;   // places in the workspace
};

GradPlan plan_of(const rdk_embed_desc_t &d, int columns)
{
    GradPlan p{};
    p.units = (d.d - 1) / columns + 1;
    p.few = d.B <= kFewTokens;
    // Few tokens of wide rows: more columns to a workgroup where there are many more of these than the chip holds, each of which looks for its token (1000 tokens into
    // 32000 x 8192 bf16 117.6 -> 109.2 us, added 24.1 -> 15.2; 844 into 3143 x 2048 8.6 -> 10.1 and so not).
    const bool wide = p.few && (int64_t)d.B * ((p.units - 1) / kWave + 1) > 8192;
    p.shift = std::max(threads_across(p.units, wide ? 2 * kWave : kWave), kLeastShift);
    p.blocks = (p.units - 1) / (1 << p.shift) + 1;
    if (p.few) return p;
    // Pieces as long as leaves enough of them to fill the chip.
    const int64_t waves = ((int64_t)d.B * p.blocks << p.shift) / kWave;   // with pieces of one token
    p.piece = waves / kMostPiece < 2048 ? kMostPiece / 2 : kMostPiece;
    p.pieces = (d.B - 1) / p.piece + 1;
    int bits = 8;
    while (((d.V - 1) >> bits) != 0) ++bits;                             // of rows
    p.order = SortOrder{bits - 8, (uint32_t)d.V};
    // all bits of the keys over tiles, or those that a share is sorted by
    p.passes = d.B > kSortTokens ? bits / kDigitBits + 1 : (bits - 8 + kDigitBits - 1) / kDigitBits;
    p.tiles = d.B > kSortTokens ? (d.B - 1) / (kThreads * tile_rounds(d.B)) + 1 : 0;
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
        p.table = room((size_t)kDigits * (p.tiles + 1) * 4);
    }
    p.partial = room((size_t)p.pieces * 2 * p.units * columns * 4);
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
        const rdk_status_t rc = sort_grant((const void *)embed_sort_kernel, sort_bytes(kSortTokens));
        if (rc != RDK_OK) return rc;
        RDK_TIMED_LAUNCH("embed_sort_kernel", embed_sort_kernel, dim3(kShares + 1), dim3(kSortThreads), sort_bytes(s.B), st, s);
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
        const dim3 grid((unsigned)p.tiles), block(kThreads);
        const bool small = tile_rounds(s.B) == kSmallRounds;
        if (small) RDK_TIMED_LAUNCH("embed_count_kernel", (embed_count_kernel<kSmallRounds>), grid, block, 0, st, s);
        else RDK_TIMED_LAUNCH("embed_count_kernel", (embed_count_kernel<kLargeRounds>), grid, block, 0, st, s);
        RDK_TIMED_LAUNCH("embed_scan_kernel", embed_scan_kernel, dim3(kDigits), dim3(kWave), 0, st, s);
        if (small) RDK_TIMED_LAUNCH("embed_place_kernel", (embed_place_kernel<kSmallRounds>), grid, block, 0, st, s);
        else RDK_TIMED_LAUNCH("embed_place_kernel", (embed_place_kernel<kLargeRounds>), grid, block, 0, st, s);
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
    const int columns = table_type == RDK_BF16 && out_type == RDK_BF16 ? 8 : 4, units = (d.d - 1) / columns + 1;
    a.shift = threads_across(units, kThreads);
    const int across = 1 << a.shift, down = kThreads >> a.shift;
    const int blocks = (units - 1) / across + 1;
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

// (of the types that take more)
size_t embed_grad_workspace_bytes(const rdk_embed_desc_t &d)
{
    const size_t narrow = plan_of(d, 4).bytes, wide = plan_of(d, 8).bytes;
    return narrow > wide ? narrow : wide;
}

rdk_status_t launch_embed_grad(const rdk_embed_desc_t &d, const KernelHandle *h, const int32_t *ids, const void *d_out, rdk_float_t out_type,
                               int64_t ldo, void *d_table, rdk_float_t table_type, int64_t ldt, bool accumulate, void *ws, hipStream_t st)
{
    const GradPlan p = plan_of(d, table_type == RDK_BF16 && out_type == RDK_BF16 ? 8 : 4);
    EmbedGradArgs a{};
    a.rows = rows_of(d, h);
    a.ids = ids; a.d_out = d_out; a.d_table = d_table; a.ldo = ldo; a.ldt = ldt;
    a.B = d.B; a.V = d.V; a.d = d.d; a.accumulate = accumulate; a.scale = d.scale;
    a.units = p.units; a.shift = p.shift; a.blocks = p.blocks; a.piece = p.piece; a.pieces = p.pieces;
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
        a.partial = (float4 *)(w + p.partial);
        const rdk_status_t rc = launch_sort(s, p, w, st);
        if (rc != RDK_OK) return rc;
    }
    with_type(out_type, [&](auto o) {
        with_type(table_type, [&](auto t) {
            constexpr int O = decltype(o)::value, T = decltype(t)::value;
            if (p.few) {
                RDK_TIMED_LAUNCH("embed_grad_few_kernel", (embed_grad_few_kernel<O, T>), dim3((unsigned)(d.B * p.blocks + a.fills)), dim3(kThreads), 0, st, a);
                return;
            }
            const int sums = ((p.pieces - 1) / (kThreads >> p.shift) + 1) * p.blocks;
            if (accumulate) RDK_TIMED_LAUNCH("embed_grad_sum_kernel", (embed_grad_sum_kernel<O, T, true>), dim3((unsigned)sums), dim3(kThreads), 0, st, a);
            else RDK_TIMED_LAUNCH("embed_grad_sum_kernel", (embed_grad_sum_kernel<O, T, false>), dim3((unsigned)(sums + a.fills)), dim3(kThreads), 0, st, a);
            RDK_TIMED_LAUNCH("embed_grad_join_kernel", (embed_grad_join_kernel<T, kColumns<O, T>>), dim3((unsigned)(p.pieces * p.blocks)), dim3(kThreads), 0, st, a);
        });
    });
    RDK_LAUNCH_CHECK("embed_grad_sum_kernel");
    return RDK_OK;
}

}  // namespace rdk
