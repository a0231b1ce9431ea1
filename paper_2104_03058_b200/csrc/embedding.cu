// Learned vertex features: rows of a table looked up by id and scaled, and the table's gradient as sums over the sorted ids.
//
//   out[i, :] = scale * table[ids[i], :]
//   grad[r, :] = scale * (dout rows of the ids i with ids[i] == r, added in ascending i), all rows of the table
//
// Neither does arithmetic worth counting: both are bound by HBM (the lookup reads n rows and writes n rows, the gradient
// reads n rows and writes `vocab` rows), or by latency on small batches.
#include <type_traits>

#include "schedule.cuh"
#include "rows.cuh"

namespace gnnfd {

constexpr int kEmbedBlock = 256;
constexpr unsigned kSms = 148;

// widest vector, in elements, that rows of `in` and of `out` can be read and written in: 16 bytes of `in`, 2 elements or 1
static int embed_vector(const void* in, int64_t ld_in, gnnfd_dtype_t in_type, const void* out, int64_t ld_out, gnnfd_dtype_t out_type)
{
    const int in_size = in_type == GNNFD_F32 ? 4 : 2, out_size = out_type == GNNFD_F32 ? 4 : 2;
    auto fits = [&](int v) {
        const int in_bytes = v * in_size, out_bytes = v * out_size < 16 ? v * out_size : 16;
        return (uintptr_t)in % in_bytes == 0 && (uintptr_t)out % out_bytes == 0 && ld_in * in_size % in_bytes == 0 &&
               ld_out * out_size % out_bytes == 0;
    };
    return fits(16 / in_size) ? 16 / in_size : fits(2) ? 2 : 1;
}
static int lanes_log2(int f, int v)
{
    const int l = ilog2((f + v - 1) / v);
    return l < 5 ? l : 5;
}

// ------------------------------------------------------------------ lookup

constexpr int32_t kMostLookup = 0x7ffff000;      // columns: a row's walk counts on for up to 32 vectors, in 32 bits

struct LookupArgs {
    const void *ids, *table;
    void* out;
    int64_t n, vocab, ldt, ldo;
    int32_t* status;
    float scale;
    int32_t f, lpr_log2;
};

// 2^lpr_log2 lanes per row, U rows of a group in flight together.
template <typename IdT, typename TI, typename TO, int V, int U>
__global__ void __launch_bounds__(kEmbedBlock) embedding_rows(const __grid_constant__ LookupArgs a)
{
    grid_dependency<true>();
    const int lpr = 1 << a.lpr_log2, groups = kEmbedBlock >> a.lpr_log2;
    const int lane = threadIdx.x & (lpr - 1);
    const int64_t row0 = (int64_t)blockIdx.x * (groups * U) + (threadIdx.x >> a.lpr_log2);
    const TI* src[U];
    bool bad = false;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t row = row0 + (int64_t)u * groups;
        src[u] = nullptr;
        if (row < a.n) {
            const int64_t id = (int64_t) static_cast<const IdT*>(a.ids)[row];
            if ((uint64_t)id < (uint64_t)a.vocab) src[u] = static_cast<const TI*>(a.table) + id * a.ldt;
            else bad = true;
        }
    }
    if (bad && a.status) atomicOr(a.status, 1);
    TO* const out = static_cast<TO*>(a.out);
    for (int c = lane * V; c < a.f; c += lpr * V) {
        if (c + V <= a.f) {
            Raw<TI, V> raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (src[u]) raw[u].load(src[u] + c);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t row = row0 + (int64_t)u * groups;
                float x[V];
                raw[u].get(x);
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] = src[u] ? x[i] * a.scale : 0.f;
                if (row < a.n) store_packed<TO, V>(out + row * a.ldo + c, x);
            }
        } else {
            for (int i = c; i < a.f; ++i)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t row = row0 + (int64_t)u * groups;
                    float x[1] = {0.f};
                    if (src[u]) load_packed<TI, 1>(src[u] + i, x);
                    x[0] = src[u] ? x[0] * a.scale : 0.f;
                    if (row < a.n) store_packed<TO, 1>(out + row * a.ldo + i, x);
                }
        }
    }
}

// ------------------------------------------------------------------ gradient

struct GradArgs {
    const void* ids;
    const void* dout;
    void* out;
    int64_t n, vocab, ldd, ldo, padding;
    const unsigned long long* words;       // sorted: id << val_bits | position + 1; ids out of range last
    const BuildCounts* counts;
    float *head, *tail;                    // [blocks, fpad] partial sums of the run that a block starts / ends inside of
    uint8_t* mark;                         // [vocab] rows that get a sum, zeroed (null where the gradient is added to what is there, or nothing is)
    int32_t* status;
    float scale;
    int32_t f, fpad, lpr_log2, val_bits, per_block, n_blocks, wide, accumulate;
};

template <typename TO, int V>
__device__ __forceinline__ void write_row(const GradArgs& a, int64_t row, int c, float (&x)[V])
{
    if (row == a.padding) return;
    TO* const p = static_cast<TO*>(a.out) + row * a.ldo + c;
    const bool add = a.accumulate;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] *= a.scale;
    if (c + V <= a.f) {
        if (add) {
            float old[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float one[1];
                load_packed<TO, 1>(p + i, one);
                old[i] = one[0];
            }
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] += old[i];
        }
        store_packed<TO, V>(p, x);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (c + i < a.f) {
                float one[1];
                one[0] = 0.f;
                if (add) load_packed<TO, 1>(p + i, one);
                one[0] += x[i];
                store_packed<TO, 1>(p + i, one);
            }
    }
}

// Sums over runs of equal ids.  A block takes per_block sorted ids, a group of lanes a consecutive share of them.  The lanes of a group read as many words
// at a time and pass them round; kInFlight rows are loaded together and added until the id changes.  A run that lies inside a group's share is
// written at once; what a group has of a run that goes on before or behind its share meets in shared memory, and is added there in order by the group that
// has the run's beginning; what a block has of a run that goes on in other blocks is left for embedding_grad_finish.
//
// Q: vectors per lane, 32 lanes apart, for rows of more than 32 vectors: narrow vectors would leave little in flight and read the words once per 32 of
// them (300,000 ids, 602 fp32 columns in rows that start on 8 bytes: 8-byte vectors 400 us, four of them a lane 213).
constexpr int kInFlight = 8;
constexpr int wide_lane(int v) { return v == 8 ? 1 : v == 4 ? 2 : 4; }       // the most vectors of a lane

template <typename TI, typename TO, int V, int Q>
__global__ void __launch_bounds__(kEmbedBlock, V == 8 ? 2 : 3) embedding_grad_sums(const __grid_constant__ GradArgs a)
{
    constexpr int U = Q == 1 ? kInFlight : kInFlight / 2, W = V * Q;
    grid_dependency<true>();
    constexpr unsigned kFull = 0xffffffffu;
    __shared__ float ends[2][kEmbedBlock][W];            // a group's first (run begun earlier) and last (run that goes on) sums
    __shared__ bool through[kEmbedBlock];                // of a group: all of its share belongs to a run begun earlier that goes on
    if (a.counts->sort_failed) return;
    const int64_t n_valid = a.counts->n_valid;
    const int lpr = 1 << a.lpr_log2, groups = kEmbedBlock >> a.lpr_log2, g = threadIdx.x >> a.lpr_log2, lane = threadIdx.x & (lpr - 1);
    const int64_t base = (int64_t)blockIdx.x * a.per_block;
    if (base >= n_valid) return;
    const int64_t end = min(base + a.per_block, n_valid);
    const int share = (a.per_block + groups - 1) / groups;
    const int64_t first = min(base + (int64_t)g * share, end);
    const int count = (int)(min(first + share, end) - first);
    const int c = ((int)blockIdx.y * lpr * Q + lane) * V, pitch_q = lpr * V;      // vector q: columns c + q * pitch_q ..
    auto key_of = [&](unsigned long long w) { return (uint32_t)(w >> a.val_bits); };
    const uint32_t pos_mask = (uint32_t)((1ull << a.val_bits) - 1ull);
    const TI* const dout = static_cast<const TI*>(a.dout) + c;
    const uint32_t pitch = (uint32_t)a.ldd;
    auto finish_row = [&](uint32_t key, float (&x)[Q][V]) {
#pragma unroll
        for (int q = 0; q < Q; ++q)
            if (c + q * pitch_q < a.f) write_row<TO, V>(a, key, c + q * pitch_q, x[q]);
        if (a.mark && c == 0 && key != a.padding) a.mark[key] = 1;
    };

    bool head = false, tail = false, passes = false;
    float acc[Q][V];
    auto clear = [&]() {
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) acc[q][i] = 0.f;
    };
    clear();
    uint32_t cur = count > 0 ? key_of(a.words[first]) : 0u;
    bool open = count > 0 && first > 0 && key_of(a.words[first - 1]) == cur;       // the run was begun earlier
    auto flush = [&](bool goes_on) {
        if (open || goes_on) {
#pragma unroll
            for (int i = 0; i < W; ++i) ends[open ? 0 : 1][threadIdx.x][i] = acc[i / V][i % V];
            head |= open;
            tail |= !open;
            passes |= open && goes_on;
        } else {
            finish_row(cur, acc);
        }
        clear();
    };
    unsigned long long word = lane < count ? a.words[first + lane] : 0ull;
    for (int t0 = 0; t0 < share; t0 += lpr) {              // (all groups of a warp make as many turns)
        const uint32_t key = key_of(word), pos = ((uint32_t)word & pos_mask) - 1u;
        const int valid = count - t0;                      // of this turn's ids, where below lpr
        word = t0 + lpr + lane < count ? a.words[first + t0 + lpr + lane] : 0ull;
        for (int j0 = 0; j0 < lpr; j0 += U) {
            if (t0 + j0 >= share) break;
            float x[U][Q][V];
            uint32_t k[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t at = __shfl_sync(kFull, pos, j0 + u, lpr);
                k[u] = __shfl_sync(kFull, key, j0 + u, lpr);
                const TI* const p = dout + (uint64_t)at * pitch;
                if (j0 + u < valid)
#pragma unroll
                    for (int q = 0; q < Q; ++q) {
                        if (c + q * pitch_q + V <= a.f) load_packed<TI, V>(p + q * pitch_q, x[u][q]);
                        else load_row<TI, V>(p + q * pitch_q, a.f - c - q * pitch_q, x[u][q]);
                    }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (j0 + u >= valid) continue;
                if (k[u] != cur) {
                    flush(false);
                    cur = k[u];
                    open = false;
                }
#pragma unroll
                for (int q = 0; q < Q; ++q)
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[q][i] += x[u][q][i];
            }
        }
    }
    if (count > 0) flush(first + count < n_valid && key_of(a.words[first + count]) == cur);
    if (lane == 0) through[g] = passes;
    __syncthreads();

    // which: 0 the run that this group's share begins inside of (asked of the block's first group), 1 the one it ends inside of
    auto join = [&](int which) {
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i / V][i % V] = ends[which][threadIdx.x][i];
        bool goes_on = which == 1 || passes;
        const int used = ((int)(end - base) + share - 1) / share;      // the groups with a share
        for (int h = g + 1; goes_on && h < used; ++h) {
#pragma unroll
            for (int i = 0; i < W; ++i) acc[i / V][i % V] += ends[0][(h << a.lpr_log2) + lane][i];
            goes_on = through[h];
        }
        if (which == 1 && !goes_on) {
            finish_row(cur, acc);
            return;
        }
        float* const part = (which ? a.tail : a.head) + (int64_t)blockIdx.x * a.fpad;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const int col = c + i / V * pitch_q + i % V;
            if (col < a.f) part[col] = acc[i / V][i % V];
        }
        if (which == 1 && a.mark && c == 0 && cur != a.padding) a.mark[cur] = 1;
    };
    if (head && g == 0) join(0);
    if (tail) join(1);
}

// The first n_blocks blocks: a run that begins in block b of the sums and goes on is added up over the blocks it
// reaches, in four interleaved walks.  The others: rows that no id names become zero.

template <typename TO>
__global__ void __launch_bounds__(kEmbedBlock) embedding_grad_finish(const __grid_constant__ GradArgs a, int vec)
{
    grid_dependency<true>();
    __shared__ float sums[kEmbedBlock];
    const int64_t join_blocks = a.n_blocks;                  // 0 where there were no ids, and then no sort
    if (join_blocks > 0 && a.counts->sort_failed) {
        if (blockIdx.x == 0 && threadIdx.x == 0 && a.status) atomicOr(a.status, 2);
        return;
    }
    if (join_blocks > 0 && blockIdx.x == 0 && threadIdx.x == 0 && a.status && a.counts->bad_index) atomicOr(a.status, 1);
    if (blockIdx.x < join_blocks) {
        const int64_t n_valid = a.counts->n_valid;
        const int64_t b = blockIdx.x, begin = b * a.per_block, next = begin + a.per_block;
        auto key_at = [&](int64_t i) { return (int64_t)(a.words[i] >> a.val_bits); };
        if (next >= n_valid) return;
        const int64_t key = key_at(next);
        if (key_at(next - 1) != key || (begin > 0 && key_at(begin - 1) == key)) return;      // nothing goes on, or it was begun earlier
        constexpr int cols = 64, ways = kEmbedBlock / cols;
        const int at_col = threadIdx.x & (cols - 1), way = threadIdx.x / cols;
        for (int c0 = 0; c0 < a.f; c0 += cols) {
            const int c = c0 + at_col;
            float sum = 0.f;
            if (c < a.f) {
                if (way == 0) sum = a.tail[b * a.fpad + c];
                constexpr int kAhead = 8;                // blocks of a walk whose words and sums are read together
                for (int64_t at = b + 1 + way; at < a.n_blocks && at * a.per_block < n_valid;) {
                    float part[kAhead];
                    bool same[kAhead];
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        const int64_t block = at + i * ways;
                        const bool there = block < a.n_blocks && block * a.per_block < n_valid;
                        part[i] = there ? a.head[block * a.fpad + c] : 0.f;      // (of another run it is not used)
                        same[i] = there && key_at(block * a.per_block) == key;
                    }
                    bool on = true;
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        on = on && same[i];
                        if (on) sum += part[i];
                    }
                    if (!on) break;
                    at += kAhead * ways;
                }
            }
            sums[threadIdx.x] = sum;
            __syncthreads();
            if (way == 0 && c < a.f) {
                float x[1] = {sum};
                for (int w = 1; w < ways; ++w) x[0] += sums[w * cols + at_col];
                write_row<TO, 1>(a, key, c, x);
            }
            __syncthreads();
        }
        return;
    }
    // zero rows: 2^lpr_log2 lanes per row, V elements at a time where rows start on such boundaries
    const int lpr = 1 << a.lpr_log2, lane = threadIdx.x & (lpr - 1), groups = kEmbedBlock >> a.lpr_log2;
    const int64_t stride = ((int64_t)gridDim.x - join_blocks) * groups;
    for (int64_t row = (blockIdx.x - join_blocks) * groups + (threadIdx.x >> a.lpr_log2); row < a.vocab; row += stride) {
        if (a.mark && a.mark[row]) continue;
        char* const p = reinterpret_cast<char*>(static_cast<TO*>(a.out) + row * a.ldo);
        const int bytes = a.f * (int)sizeof(TO);
        int at = lane * vec;
        if (vec == 16)
            for (; at + 16 <= bytes; at += lpr * 16) __stcs(reinterpret_cast<uint4*>(p + at), make_uint4(0u, 0u, 0u, 0u));
        else if (vec == 4)
            for (; at + 4 <= bytes; at += lpr * 4) __stcs(reinterpret_cast<unsigned int*>(p + at), 0u);
        else
            for (; at + 2 <= bytes; at += lpr * 2) *reinterpret_cast<unsigned short*>(p + at) = 0;
        for (int i = at; i < bytes && i < at + vec; i += 2) *reinterpret_cast<unsigned short*>(p + i) = 0;      // what is left of a row
    }
}

// ------------------------------------------------------------------ gradient of few ids
//
// One launch in place of the sort's seven (64 columns: 4096 ids 12 to 15 us, 8192 17 to 19, by sorting 27).  Block b has the rows r with r % kClasses == b (a prime number of classes, so that regular ids spread).  It looks through
// all ids, each warp through a share of their places, and lists its own in order; counts them by row; one warp puts the list in the order of the rows, equal
// rows in the order of their places; then a warp takes a row, adds up its places or writes zeros.  Rows of more than kCrowd places
// are added up by the whole block.
constexpr int kFewIds = GNNFD_EMBEDDING_FEW_IDS;
constexpr int kClasses = 443;                                          // three blocks on each of 148 SMs
constexpr int kFewBlock = 512, kFewWarps = kFewBlock / 32;
constexpr int kClassRows = GNNFD_EMBEDDING_FEW_ROWS / kClasses;        // of one class, at most
constexpr int kCrowd = 64;
// shared memory of a block with n ids and so many rows, and the most there can be
constexpr size_t few_bytes(size_t n, size_t rows) { return n * sizeof(uint32_t) + (rows + 1) * sizeof(int) + n * sizeof(uint16_t); }
constexpr int kFewSmem = (int)few_bytes(kFewIds, kClassRows);
static_assert(kFewIds <= kFewWarps * 32 * 32, "a lane keeps one vote per step of its warp's share");
static_assert(kFewIds <= 1 << 16 && kClassRows <= 1 << 16 && GNNFD_EMBEDDING_FEW_ROWS % kClasses == 0, "place and row in one word");

template <typename IdT, typename TI, typename TO, int V, int Q>
__global__ void __launch_bounds__(kFewBlock, 2) embedding_grad_few(const __grid_constant__ GradArgs a, int vec)
{
    grid_dependency<true>();
    extern __shared__ uint32_t few_smem[];
    constexpr unsigned kFull = 0xffffffffu;
    constexpr int U = V * Q >= 8 ? 4 : 8;
    const int n = (int)a.n, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, mine = blockIdx.x;
    const int rows = (int)((a.vocab - mine + kClasses - 1) / kClasses);            // (blocks beyond the last row have none)
    uint32_t* const listed = few_smem;                                 // [n] row << 16 | place, in the order of the places
    int* const first = reinterpret_cast<int*>(listed + n);             // [rows + 1] where each row's places start in `order`
    uint16_t* const order = reinterpret_cast<uint16_t*>(first + rows + 1);         // [n]
    __shared__ int per_warp[kFewWarps], crowded[kFewIds / kCrowd], n_crowded;
    __shared__ float part[kFewWarps][32][V * Q];
    const IdT* const ids = static_cast<const IdT*>(a.ids);

    // the votes of the warp's steps: bit l of step k's vote, which lane k keeps, says that place begin + 32 k + l is this block's
    const int share = (n + kFewBlock - 1) / kFewBlock * 32, begin = warp * share, steps = share / 32;
    unsigned votes = 0u;
    int count = 0;
    bool bad = false;
    constexpr int kLook = 8;
    for (int k0 = 0; k0 < steps; k0 += kLook) {
        int64_t id[kLook];
#pragma unroll
        for (int u = 0; u < kLook; ++u) {
            const int i = begin + (k0 + u) * 32 + lane;
            id[u] = k0 + u < steps && i < n ? (int64_t)ids[i] : 0;
        }
#pragma unroll
        for (int u = 0; u < kLook; ++u) {
            const int i = begin + (k0 + u) * 32 + lane;
            const bool there = k0 + u < steps && i < n, inside = (uint64_t)id[u] < (uint64_t)a.vocab;
            bad = bad || (there && !inside);
            const unsigned vote = __ballot_sync(kFull, there && inside && id[u] != a.padding && (uint32_t)id[u] % kClasses == (uint32_t)mine);
            if (lane == k0 + u) votes = vote;
            count += __popc(vote);
        }
    }
    if (bad && mine == 0 && blockIdx.y == 0 && a.status) atomicOr(a.status, 1);
    if (lane == 0) per_warp[warp] = count;
    for (int r = tid; r <= rows; r += kFewBlock) first[r] = 0;
    if (tid == 0) n_crowded = 0;
    __syncthreads();
    int at = 0, total = 0;
    for (int w = 0; w < kFewWarps; ++w) {
        at += w < warp ? per_warp[w] : 0;
        total += per_warp[w];
    }
    if (count > 0)
        for (int k = 0; k < steps; ++k) {
            const unsigned vote = __shfl_sync(kFull, votes, k);
            if (vote >> lane & 1u) {
                const int place = begin + k * 32 + lane;
                const uint32_t row = (uint32_t)ids[place] / kClasses;
                listed[at + __popc(vote & ((1u << lane) - 1u))] = row << 16 | (uint32_t)place;
                atomicAdd(&first[row + 1], 1);
            }
            at += __popc(vote);
        }
    __syncthreads();
    // counts to starts, then the list in the order of the rows; both by one warp
    if (warp == 0) {
        int sum = 0;
        for (int r0 = 0; r0 < rows; r0 += 32) {
            int v = r0 + lane < rows ? first[r0 + lane + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int t = __shfl_up_sync(kFull, v, o);
                if (lane >= o) v += t;
            }
            if (r0 + lane < rows) first[r0 + lane + 1] = sum + v;
            sum += __shfl_sync(kFull, v, 31);
        }
        __syncwarp();
        for (int j0 = 0; j0 < total; j0 += 32) {                       // first[row] moves on to the row's end
            const uint32_t e = j0 + lane < total ? listed[j0 + lane] : 0xffffffffu;
            const unsigned same = __match_any_sync(kFull, e >> 16 | (j0 + lane < total ? 0u : 0x10000u));
            int to = 0;
            if (j0 + lane < total) to = first[e >> 16] + __popc(same & ((1u << lane) - 1u));
            __syncwarp();
            if (j0 + lane < total) {
                order[to] = (uint16_t)(e & 0xffffu);
                if (lane == __ffs(same) - 1) first[e >> 16] += __popc(same);
            }
            __syncwarp();
        }
    }
    __syncthreads();

    const int c = (int)blockIdx.y * (32 * V * Q) + lane * V;
    float acc[Q][V];
    auto add_places = [&](int from, int to) {
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) acc[q][i] = 0.f;
        for (int j = from; j < to; j += U) {
            float x[U][Q][V];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (j + u < to) {
                    const TI* const p = static_cast<const TI*>(a.dout) + (int64_t)order[j + u] * a.ldd;
#pragma unroll
                    for (int q = 0; q < Q; ++q) load_row<TI, V>(p + c + q * 32 * V, a.f - c - q * 32 * V, x[u][q]);
                }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (j + u < to)
#pragma unroll
                    for (int q = 0; q < Q; ++q)
#pragma unroll
                        for (int i = 0; i < V; ++i) acc[q][i] += x[u][q][i];
        }
    };
    auto write = [&](int r) {
#pragma unroll
        for (int q = 0; q < Q; ++q)
            if (c + q * 32 * V < a.f) write_row<TO, V>(a, mine + (int64_t)r * kClasses, c + q * 32 * V, acc[q]);
    };
    for (int r = warp; r < rows; r += kFewWarps) {
        const int from = r > 0 ? first[r - 1] : 0, to = first[r];      // (row r's start is where row r - 1 ended)
        if (to - from > kCrowd) {
            if (lane == 0) crowded[atomicAdd(&n_crowded, 1)] = r;
        } else if (to > from) {
            add_places(from, to);
            write(r);
        } else if (!a.accumulate) {
            char* const p = reinterpret_cast<char*>(static_cast<TO*>(a.out) + (mine + (int64_t)r * kClasses) * a.ldo);
            const int begin_byte = (int)blockIdx.y * (32 * V * Q) * (int)sizeof(TO), end_byte = min(begin_byte + 32 * V * Q * (int)sizeof(TO), a.f * (int)sizeof(TO));
            for (int k = begin_byte + lane * vec; k < end_byte; k += 32 * vec) {
                if (vec == 16 && k + 16 <= end_byte) __stcs(reinterpret_cast<uint4*>(p + k), make_uint4(0u, 0u, 0u, 0u));
                else if (vec == 4 && k + 4 <= end_byte) __stcs(reinterpret_cast<unsigned int*>(p + k), 0u);
                else
                    for (int m = k; m < k + vec && m < end_byte; m += 2) *reinterpret_cast<unsigned short*>(p + m) = 0;
            }
        }
    }
    __syncthreads();
    for (int k = 0; k < n_crowded; ++k) {                              // (in whatever order: each row's sum is its own)
        const int r = crowded[k], from = r > 0 ? first[r - 1] : 0, length = first[r] - from;
        add_places(from + (int)((int64_t)length * warp / kFewWarps), from + (int)((int64_t)length * (warp + 1) / kFewWarps));
#pragma unroll
        for (int i = 0; i < V * Q; ++i) part[warp][lane][i] = acc[i / V][i % V];
        __syncthreads();
        if (warp == 0) {
            for (int w = 1; w < kFewWarps; ++w)
#pragma unroll
                for (int i = 0; i < V * Q; ++i) acc[i / V][i % V] += part[w][lane][i];
            write(r);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ host side

template <typename IdT, typename TI, typename TO, int V>
static void launch_lookup(const LookupArgs& a, cudaStream_t s)
{
    const int64_t rows = kEmbedBlock >> a.lpr_log2;
    // Four rows in flight per group once that still gives every SM four blocks.  1,000,003 rows of 128 bf16 columns: eight 176 us, four 115, two 101; 200,000
    // of 64: 13.5, 9.7, 12.2; 40,000 of 128 fp32: 9.5, 9.4, 11.8.
    if (a.n >= rows * 4 * 4 * kSms)
        GNNFD_LAUNCH("embedding_rows", s, (embedding_rows<IdT, TI, TO, V, 4>), (unsigned)((a.n + rows * 4 - 1) / (rows * 4)), kEmbedBlock, 0, a);
    else
        GNNFD_LAUNCH("embedding_rows", s, (embedding_rows<IdT, TI, TO, V, 1>), (unsigned)((a.n + rows - 1) / rows), kEmbedBlock, 0, a);
}

template <typename IdT, typename TI, typename TO>
static void lookup_vector(const LookupArgs& a, int v, cudaStream_t s)
{
    if (v == 16 / (int)sizeof(TI)) launch_lookup<IdT, TI, TO, 16 / sizeof(TI)>(a, s);
    else if (v == 2) launch_lookup<IdT, TI, TO, 2>(a, s);
    else launch_lookup<IdT, TI, TO, 1>(a, s);
}

template <typename IdT>
static void lookup_types(const LookupArgs& a, int v, gnnfd_dtype_t tdt, gnnfd_dtype_t odt, cudaStream_t s)
{
    if (tdt == GNNFD_F32) {
        if (odt == GNNFD_F32) lookup_vector<IdT, float, float>(a, v, s);
        else lookup_vector<IdT, float, __nv_bfloat16>(a, v, s);
    } else {
        if (odt == GNNFD_F32) lookup_vector<IdT, __nv_bfloat16, float>(a, v, s);
        else lookup_vector<IdT, __nv_bfloat16, __nv_bfloat16>(a, v, s);
    }
}

// ids per block of the sums: as many as leave every SM sixteen blocks (column tiles counted as tiles of 256), 64 to 1024
static int ids_per_block(int64_t n, int32_t f)
{
    int t = 64;
    while (t < 1024 && (int64_t)t * 2 * kSms * 16 <= n * ((f + 255) / 256)) t *= 2;
    return t;
}

struct GradScratch {
    SortedIds sorted;
    float *head, *tail;
};

static int carve_grad(Carver& c, int64_t n, int64_t vocab, int32_t f, GradScratch* g)
{
    const int rc = carve_sorted_ids(c, n, vocab, (size_t)vocab, &g->sorted);
    if (rc) return rc;
    const size_t blocks = (size_t)((n + ids_per_block(n, f) - 1) / ids_per_block(n, f)), fpad = align_up((size_t)f, 4);
    g->head = c.take<float>(blocks * fpad);
    g->tail = c.take<float>(blocks * fpad);
    return GNNFD_OK;
}

template <typename TI, typename TO, int V>
static int launch_grad(const GradArgs& a, gnnfd_itype_t itype, bool few, bool accumulate, cudaStream_t s)
{
    const uintptr_t bits = (uintptr_t)a.out | (uintptr_t)(a.ldo * sizeof(TO));
    const int vec = bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 2;
    if (few) {
        const size_t smem = few_bytes((size_t)a.n, (size_t)((a.vocab + kClasses - 1) / kClasses));
        auto launch = [&](auto wide, auto id) -> int {
            constexpr int Q = decltype(wide)::value;
            const auto kernel = embedding_grad_few<decltype(id), TI, TO, V, Q>;
            const dim3 grid((unsigned)(a.vocab < kClasses ? a.vocab : kClasses), (unsigned)((a.f + 32 * V * Q - 1) / (32 * V * Q)));
            // Static shared memory counts too: beyond 16 KB the limit is raised, to the same for every call, since it is one for all host threads.
            if (smem > 16 * 1024) GNNFD_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem));
            GNNFD_LAUNCH("embedding_grad_few", s, kernel, grid, kFewBlock, smem, a, vec);
            return GNNFD_OK;
        };
        using One = std::integral_constant<int, 1>;
        using Wide = std::integral_constant<int, wide_lane(V)>;
        const bool wide = a.f > 32 * V;
        const int rc = itype == GNNFD_I32 ? (wide ? launch(Wide(), int32_t()) : launch(One(), int32_t()))
                                          : (wide ? launch(Wide(), (long long)0) : launch(One(), (long long)0));
        if (rc) return rc;
    } else {
        const int per_tile = (V << a.lpr_log2) * (a.wide ? wide_lane(V) : 1);
        const dim3 sums((unsigned)a.n_blocks, (unsigned)((a.f + per_tile - 1) / per_tile));
        if (a.n_blocks == 0) {}                                        // no ids
        else if (a.wide) GNNFD_LAUNCH("embedding_grad_sums", s, (embedding_grad_sums<TI, TO, V, wide_lane(V)>), sums, kEmbedBlock, 0, a);
        else GNNFD_LAUNCH("embedding_grad_sums", s, (embedding_grad_sums<TI, TO, V, 1>), sums, kEmbedBlock, 0, a);
        const int64_t groups = kEmbedBlock >> a.lpr_log2, zero = accumulate ? 0 : (a.vocab + groups - 1) / groups;
        const int64_t grid = (int64_t)a.n_blocks + (zero < 16 * kSms ? zero : 16 * kSms);
        if (grid > 0x7fffffffll) return GNNFD_TOO_LARGE;
        if (grid > 0) GNNFD_LAUNCH("embedding_grad_finish", s, (embedding_grad_finish<TO>), (unsigned)grid, kEmbedBlock, 0, a, vec);
    }
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

template <typename TI, typename TO>
static int grad_vector(const GradArgs& a, int v, gnnfd_itype_t itype, bool few, bool accumulate, cudaStream_t s)
{
    if (v == 16 / (int)sizeof(TI)) return launch_grad<TI, TO, 16 / sizeof(TI)>(a, itype, few, accumulate, s);
    if (v == 2) return launch_grad<TI, TO, 2>(a, itype, few, accumulate, s);
    return launch_grad<TI, TO, 1>(a, itype, few, accumulate, s);
}

static bool few_ids(int64_t n, int64_t vocab) { return n <= kFewIds && vocab <= GNNFD_EMBEDDING_FEW_ROWS; }

static bool known(gnnfd_dtype_t t) { return t == GNNFD_F32 || t == GNNFD_BF16; }

}  // namespace gnnfd

extern "C" {

int gnnfd_embedding(int64_t n, const void* d_ids, gnnfd_itype_t itype, int64_t vocab, const void* d_table, int64_t ldt, gnnfd_dtype_t tdt,
                    int32_t f, float scale, void* d_out, int64_t ldo, gnnfd_dtype_t odt, int32_t* d_status, void* stream)
{
    using namespace gnnfd;
    if (n < 0 || vocab <= 0 || f <= 0 || ldt < f || ldo < f) return GNNFD_INVALID_ARG;
    if (!known(tdt) || !known(odt) || (itype != GNNFD_I32 && itype != GNNFD_I64)) return GNNFD_UNSUPPORTED;
    if (n > 0x7fffffffll || vocab > 0x7fffffffll || f > kMostLookup) return GNNFD_TOO_LARGE;
    if (n == 0) return GNNFD_OK;
    if (!d_ids || !d_table || !d_out) return GNNFD_INVALID_ARG;
    const int v = embed_vector(d_table, ldt, tdt, d_out, ldo, odt);
    const LookupArgs a{d_ids, d_table, d_out, n, vocab, ldt, ldo, d_status, scale, f, lanes_log2(f, v)};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (itype == GNNFD_I32) lookup_types<int32_t>(a, v, tdt, odt, s);
    else lookup_types<long long>(a, v, tdt, odt, s);
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

int gnnfd_embedding_backward_workspace_bytes(int64_t n, int64_t vocab, int32_t f, size_t* scratch_bytes)
{
    using namespace gnnfd;
    if (n < 0 || vocab <= 0 || f <= 0 || !scratch_bytes) return GNNFD_INVALID_ARG;
    if (n > 0x7ffffff0ll || vocab > 0x7ffffff0ll) return GNNFD_TOO_LARGE;
    *scratch_bytes = 0;
    if (n == 0 || few_ids(n, vocab)) return GNNFD_OK;
    Carver c(nullptr, ~size_t(0));
    GradScratch g;
    const int rc = carve_grad(c, n, vocab, f, &g);
    if (rc == GNNFD_OK) *scratch_bytes = c.off;
    return rc;
}

int gnnfd_embedding_backward(int64_t n, const void* d_ids, gnnfd_itype_t itype, const void* d_dout, int64_t ldd, gnnfd_dtype_t ddt,
                             int64_t vocab, int32_t f, float scale, int64_t padding, int accumulate, void* d_grad, int64_t ldg,
                             gnnfd_dtype_t gdt, void* d_scratch, size_t scratch_bytes, int32_t* d_status, void* stream)
{
    using namespace gnnfd;
    const SortDrill drill = take_sort_drill();
    if (n < 0 || vocab <= 0 || f <= 0 || ldd < f || ldd > 0x7fffffffll || ldg < f || !d_grad) return GNNFD_INVALID_ARG;
    if (!known(ddt) || !known(gdt) || (itype != GNNFD_I32 && itype != GNNFD_I64)) return GNNFD_UNSUPPORTED;
    if (n > 0x7ffffff0ll || vocab > 0x7ffffff0ll) return GNNFD_TOO_LARGE;
    if (n > 0 && (!d_ids || !d_dout)) return GNNFD_INVALID_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool few = few_ids(n, vocab);
    if ((few || n == 0) && drill.sweep >= 0) return GNNFD_INVALID_ARG;             // no sort to drill
    int v = embed_vector(d_dout, ldd, ddt, d_grad, ldg, gdt);
    if ((f - 1) / (32 * v * wide_lane(v)) >= 65535) return GNNFD_TOO_LARGE;      // column tiles are a grid's rows
    // a group reads eight words at a time at least: rows narrower than eight vectors are taken in narrower ones
    if (!few && v > 2 && (f + v - 1) / v < kInFlight) v = 2;
    if (!few && (f + v - 1) / v < kInFlight) v = 1;
    GradArgs a{};
    a.ids = d_ids; a.dout = d_dout; a.out = d_grad;
    a.n = n; a.vocab = vocab; a.ldd = ldd; a.ldo = ldg; a.padding = padding;
    a.status = d_status; a.accumulate = accumulate != 0; a.scale = scale; a.f = f; a.fpad = (int32_t)align_up((size_t)f, 4);
    a.lpr_log2 = lanes_log2(f, v);
    if (a.lpr_log2 < 3) a.lpr_log2 = 3;
    a.wide = f > v << a.lpr_log2 && v < 8;
    if (!few && n > 0) {
        if (!d_scratch || ((uintptr_t)d_scratch & 255u)) return GNNFD_INVALID_ARG;
        Carver c(d_scratch, scratch_bytes);
        GradScratch g;
        int rc = carve_grad(c, n, vocab, f, &g);
        if (rc) return rc;
        if (!c.ok) return GNNFD_WORKSPACE_TOO_SMALL;
        rc = sort_ids(n, vocab, d_ids, itype, drill, g.sorted, s);
        if (rc) return rc;
        a.words = g.sorted.words; a.val_bits = g.sorted.val_bits; a.counts = g.sorted.counts;
        a.mark = accumulate ? nullptr : g.sorted.extra;
        a.head = g.head; a.tail = g.tail;
        a.per_block = ids_per_block(n, f);
        a.n_blocks = (int32_t)((n + a.per_block - 1) / a.per_block);
    }
    if (ddt == GNNFD_F32)
        return gdt == GNNFD_F32 ? grad_vector<float, float>(a, v, itype, few, accumulate, s)
                                : grad_vector<float, __nv_bfloat16>(a, v, itype, few, accumulate, s);
    return gdt == GNNFD_F32 ? grad_vector<__nv_bfloat16, float>(a, v, itype, few, accumulate, s)
                            : grad_vector<__nv_bfloat16, __nv_bfloat16>(a, v, itype, few, accumulate, s);
}

}  // extern "C"
