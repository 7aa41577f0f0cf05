// Attention over 16-bit keys and values in pages: of a batch whose sequences share a prefix, and over listed blocks.
//
// Rows, tiles and softmax are those of rows16.h; what differs from contiguous keys is where a tile's positions are.  A tile is made of granules of 16
// positions, each inside a page.  The lanes of a wave look up the pages of its next 64 granules at once (entries of the table, and of the list where there
// is one) and a tile takes its own from there, so that the two dependent reads are paid once for 32 tiles and not for each.
//
// A prefix that all sequences share is work of its own: its rows are those of all sequences together, so its keys and values are read once for as many
// rows as a workgroup holds.  Its partial results, and those of the sequences' own positions, are joined by merge_kernel.
#include "pages.h"
#include "rows16.h"
#include "wave_ops.h"

#include <algorithm>
#include <cmath>

namespace specache {
namespace {

constexpr int kHidden = 1 << 30;      // position of a granule that nobody sees

struct PagedArgs {
    specache_view q, out;
    PageArgs pages;
    const int32_t* q_lengths;
    const int32_t* kv_lengths;
    const int32_t* blocks;            // [batch][KV head][token][slots]
    float* own_o;                     // [unit][row tile][chunk][row][kD], not divided by the sum; a unit is a KV head of a sequence (of a token of it)
    float* own_ml;                    // [unit][row tile][chunk][row][2]: maximum (in powers of two; -infinity where nothing is seen), sum
    float* prefix_o;                  // [KV head][row tile][chunk][row][kD]
    float* prefix_ml;
    int batch, G, q_tokens, kv_tokens, slots;
    int shared;                       // positions of the prefix, whole pages
    int prefix_groups;                // the first workgroups of a launch work on the prefix
    int own_chunks, own_row_tiles, own_rows, prefix_chunks, prefix_row_tiles, prefix_rows;
    int parts;                        // results go to the merge
    int merge_rows;
    float scale;                      // sm_scale in powers of two
};

// What a workgroup works on: rows row0 .. row0 + rows - 1 of a unit or of the prefix, positions begin .. end - 1 or a list's.
struct Job {
    bool prefix;
    int b, h, token, row0, rows, n, N, begin, end, tiles, i_begin, i_end;
    int64_t place;                    // of its first row's partial results
};

// A lane's row of it.
struct Row {
    int b, token, head, last;         // last: the last position seen
};

template <bool LISTED>
__device__ __forceinline__ Row row_of(const PagedArgs& a, const Job& j, int i) {
    const int r = j.row0 + min(i, j.rows - 1);
    Row o;
    if (!LISTED && j.prefix) {
        o.b = r / (a.q_tokens * a.G);
        const int rest = r - o.b * (a.q_tokens * a.G), n = length_of(a.q_lengths, o.b, a.q_tokens), N = length_of(a.kv_lengths, o.b, a.kv_tokens);
        o.token = rest / a.G;
        o.head = j.h * a.G + rest - o.token * a.G;
        o.last = o.token < n ? min(N - n + o.token, j.end - 1) : j.end - 1;   // (of rows that there are not nothing is kept)
        o.token = min(o.token, max(n - 1, 0));
    } else {
        o.b = j.b;
        o.token = LISTED ? j.token : r / a.G;
        o.head = j.h * a.G + r % a.G;
        o.last = j.N - j.n + o.token;
    }
    return o;
}

// Which work the workgroup has; false: none.
template <bool LISTED, int TILE, int ROWS>
__device__ __forceinline__ bool job_of(const PagedArgs& a, bool prefix, Job& j) {
    int chunk, chunks;
    j.prefix = prefix;
    j.token = 0;
    if (j.prefix) {
        const int id = on_one_xcd(blockIdx.x, a.prefix_groups, a.prefix_row_tiles), tile = id % a.prefix_row_tiles;
        chunks = a.prefix_chunks;
        chunk = id / a.prefix_row_tiles % chunks;
        j.h = id / a.prefix_row_tiles / chunks;
        j.b = 0;
        j.row0 = tile * ROWS;
        j.rows = min(ROWS, a.batch * a.q_tokens * a.G - j.row0);
        j.n = j.N = 0;
        j.begin = 0;
        j.end = a.shared;
        j.tiles = (j.end + TILE - 1) / TILE;
        j.place = (((int64_t)j.h * a.prefix_row_tiles + tile) * chunks + chunk) * a.prefix_rows;
    } else {
        const int index = blockIdx.x - a.prefix_groups;
        const int id = TILE == 64 ? on_one_xcd(index, gridDim.x - a.prefix_groups, a.own_row_tiles * a.own_chunks) : index, item = id / a.own_chunks;
        const int tile = a.own_row_tiles - 1 - item % a.own_row_tiles;   // the longest first
        int unit = item / a.own_row_tiles;
        chunks = a.own_chunks;
        chunk = id % chunks;
        j.place = (((int64_t)unit * a.own_row_tiles + tile) * chunks + chunk) * a.own_rows;
        j.h = unit % a.pages.n_kv_heads;
        unit /= a.pages.n_kv_heads;
        if (LISTED) {
            j.token = unit % a.q_tokens;
            unit /= a.q_tokens;
        }
        j.b = unit;
        j.n = length_of(a.q_lengths, j.b, a.q_tokens);
        j.N = length_of(a.kv_lengths, j.b, a.kv_tokens);
        int used = 0;                                                    // of a list's entries: up to the last block that there is
        if (LISTED) {                                                    // (asked for with the lengths)
            const int32_t* list = a.blocks + (((int64_t)j.b * a.pages.n_kv_heads + j.h) * a.q_tokens + j.token) * a.slots;
            const int lane = threadIdx.x % 64;
            for (int at = (a.slots - 1) / 64 * 64; at >= 0; at -= 64) {
                const int32_t block = list[min(at + lane, a.slots - 1)];
                const uint64_t some = __ballot(at + lane < a.slots && block >= 0);
                if (some) {
                    used = at + 64 - __builtin_clzll(some);
                    break;
                }
            }
        }
        j.row0 = tile * ROWS;
        const int all = LISTED ? j.token < j.n ? a.G : 0 : j.n * a.G;
        j.rows = min(ROWS, all - j.row0);
        if (j.rows <= 0) return false;
        j.begin = LISTED ? 0 : a.shared;
        j.end = j.N;
        // (of a sequence without tokens no entry is a block, and there need not be a page whose memory a tile could be taken from)
        if (LISTED) j.tiles = j.N > 0 ? (int)((((int64_t)used << a.pages.log2) + TILE - 1) / TILE) : 0;
        else j.tiles = max(0, (min(j.N, j.N - j.n + (j.row0 + j.rows - 1) / a.G + 1) - j.begin + TILE - 1) / TILE);
    }
    j.i_begin = (int)((int64_t)j.tiles * chunk / chunks);
    j.i_end = (int)((int64_t)j.tiles * (chunk + 1) / chunks);
    return true;
}

// Where the positions of tiles are: tile i_first + k * STEP, its GRANULES granules of 16, for the next 64 granules at a time.
struct Edges {
    uint32_t edge, wave_edge;         // of a tile's granules those that some row (of the wave) does not see all of
};
template <bool LISTED, int GRANULES>
struct Directory {
    static constexpr int kTiles = 64 / GRANULES, kGranules = GRANULES;
    const int32_t* table;
    const int32_t* list;
    int log2, n_pages, slots, begin, end, i_first, step, lane;
    int first, wave_first;            // the first position that is the last one seen of some row (of the wave)
    int k0, page, pos0;
    uint64_t edge, wave_edge;

    __device__ __forceinline__ Directory(const PagedArgs& a, const Job& j, int i_first_, int step_, int lane_, int first_, int wave_first_)
        : table(a.pages.table + (j.prefix ? 0 : j.b * a.pages.table_stride)),
          list(LISTED ? a.blocks + (((int64_t)j.b * a.pages.n_kv_heads + j.h) * a.q_tokens + j.token) * a.slots : nullptr),
          log2(a.pages.log2), n_pages(a.pages.n_pages), slots(a.slots), begin(j.begin), end(j.end), i_first(i_first_), step(step_), lane(lane_),
          first(first_), wave_first(wave_first_) {}
    __device__ __forceinline__ void load(int k) {
        k0 = k;
        const int64_t place = (int64_t)begin + ((int64_t)(i_first + (k + lane / GRANULES) * step) * GRANULES + lane % GRANULES) * 16;
        int64_t position = place;
        bool there = place < end;
        if constexpr (LISTED) {
            const int64_t entry = place >> log2;
            const int block = entry < slots ? list[entry] : -1;
            position = ((int64_t)block << log2) + (place & ((1 << log2) - 1));
            there = block >= 0 && position < end;
        }
        page = -1;
        if (there) page = table[position >> log2];
        there = (uint32_t)page < (uint32_t)n_pages;
        page = there ? page : 0;
        pos0 = there ? (int)position : kHidden;
        edge = __ballot(pos0 + 15 > first);
        wave_edge = __ballot(pos0 + 15 > wave_first);
    }
    __device__ __forceinline__ void one(int k, int granule, int& p, int& x) const {
        const int l = (k - k0) * GRANULES + granule;
        p = __builtin_amdgcn_readlane(page, l);
        x = __builtin_amdgcn_readlane(pos0, l);
    }
    __device__ __forceinline__ void positions(int k, int (&x)[GRANULES]) const {
#pragma unroll
        for (int i = 0; i < GRANULES; ++i) x[i] = __builtin_amdgcn_readlane(pos0, (k - k0) * GRANULES + i);
    }
    __device__ __forceinline__ void tile(int k, int (&p)[GRANULES], int (&x)[GRANULES]) const {
#pragma unroll
        for (int i = 0; i < GRANULES; ++i) one(k, i, p[i], x[i]);
    }
    __device__ __forceinline__ Edges edges(int k) const {
        const int l = (k - k0) * GRANULES;
        constexpr uint32_t kAll = (1u << GRANULES) - 1;
        return Edges{(uint32_t)(edge >> l) & kAll, (uint32_t)(wave_edge >> l) & kAll};
    }
};

// LOADS times 16 bytes to each lane's place (1024 bytes in order of lanes) from `lds` on, from base + at[i].  The compiler is not told which part of LDS this
// writes: it would wait for all that travels in front of some reads of what is there already.  So the kernels wait themselves, and tell it where memory may
// have changed.  (M0, the place in LDS, is left as it was.)
template <int LOADS>
__device__ __forceinline__ void load_to_lds(uint32_t lds, const uint32_t (&at)[LOADS], const char* base) {
    uint32_t m0;
    if constexpr (LOADS == 4)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %6\n\t"
                     "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %6\n\t"
                     "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %6\n\t"
                     "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, %6\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0) : "s"(lds), "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "s"(base) : "memory", "scc");
    else {
        static_assert(LOADS == 2, "two or four loads");
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %4\n\t"
                     "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %4\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0) : "s"(lds), "v"(at[0]), "v"(at[1]), "s"(base) : "memory", "scc");
    }
}
template <int COUNT>
__device__ __forceinline__ void wait_loads() {   // until no more than COUNT loads are on their way
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COUNT) : "memory");
}
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }   // of LDS

// One wave's loads of keys or values of a granule: LOADS times 4 positions from position 4 * LOADS * part of it on, to LDS in the order that Rows reads.
template <bool KEYS, int LOADS>
struct PageFetch {
    const char* base;                 // the head's first place of page 0
    int64_t page_bytes;
    uint32_t place_bytes;
    int part, lane, log2;
    uint32_t at[LOADS];
    __device__ __forceinline__ int position(int i) const { return 4 * (LOADS * part + i) + lane / 16; }
    __device__ __forceinline__ uint32_t piece(int i) const {
        const int r = position(i);
        return ((lane % 16) ^ (KEYS ? key_swizzle(r) : value_swizzle(r))) * 16;
    }
    __device__ __forceinline__ PageFetch(const specache_view& v, int h, int log2_, int part_, int lane_)
        : base((const char*)v.data + h * v.head * 2), page_bytes(v.batch * 2), place_bytes((uint32_t)v.token * 2), part(part_), lane(lane_), log2(log2_) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) at[i] = (uint32_t)position(i) * place_bytes + piece(i);
    }
    __device__ __forceinline__ const char* granule(int page, int pos0) const {
        return base + page * page_bytes + (int64_t)((pos0 & ((1 << log2) - 1)) * (uint64_t)place_bytes);
    }
    // Positions from `end` on are the last one before it again (no row sees them, but they are finite if it is).
    __device__ __forceinline__ void operator()(int page, int pos0, int end, uint32_t lds) const {
        const char* from = granule(page, pos0);
        const uint32_t to = lds + 4 * LOADS * part * kRowBytes16;
        if (pos0 + 16 <= end || pos0 == kHidden) {
            load_to_lds(to, at, from);
        } else {
            uint32_t held[LOADS];
#pragma unroll
            for (int i = 0; i < LOADS; ++i) held[i] = min(position(i), end - 1 - pos0) * place_bytes + piece(i);
            load_to_lds(to, held, from);
        }
    }
};

template <bool BF16, int BLOCKS>
struct PagedRows : Rows<BF16, BLOCKS> {
    using Base = Rows<BF16, BLOCKS>;
    bool saw = false;                 // some position (of this lane's half)
    // hides what the row does not see
    __device__ __forceinline__ void hide(const int (&pos0)[2 * BLOCKS]) {
#pragma unroll
        for (int g = 0; g < 2 * BLOCKS; ++g) {
            const int most = Base::seen.last - pos0[g] - 4 * Base::half;
            saw |= most >= 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (8 * (e / 4) + e % 4 > most) Base::s[g / 2][8 * (g % 2) + e] = -INFINITY;
                if (e % 2) __builtin_amdgcn_sched_barrier(0);   // few conditions at a time: they live in scalar registers
            }
        }
    }
    // what drop_odd_values dropped of a granule
    __device__ void give_odd_granule(const char* values, uint32_t place_bytes, int pos0, int end) {
        for (int j = 0; j < 16 && pos0 + j < end; ++j)
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t x = ((const uint16_t*)(values + (uint64_t)j * place_bytes))[32 * dt + 8 * (i / 4) + 4 * Base::half + i % 4];
                    if ((x & kExponents<BF16> & 0xFFFFu) == (kExponents<BF16> & 0xFFFFu) && pos0 + j <= Base::seen.last) Base::o[dt][i] += widen16<BF16>(x);
                }
    }
    template <class D, class F>
    __device__ void give_odd_values(D& directory, const F& fetch_values, int n, int end) {
        directory.load(0);
        for (int k = 0; k < n; ++k) {
            if (k - directory.k0 >= D::kTiles) directory.load(k);
            if (!directory.edges(k).edge) continue;
            for (int i = 0; i < D::kGranules; ++i) {
                int page, pos0;
                directory.one(k, i, page, pos0);
                if (pos0 != kHidden) give_odd_granule(fetch_values.granule(page, pos0), fetch_values.place_bytes, pos0, end);
            }
        }
    }
    // A wave's sums to their places by way of its kSumsBytes of LDS, so that a row's lines are written whole.  us, straight / by way of LDS: a prefix of 3234 positions
    // for 32 sequences of 27 tokens and 8 heads 61.8 / 58.4, 6517 for 64 of 2 and 32 heads 44.5 / 43.6.  (Results in 16 bits gain nothing from it: 17.1 / 18.9 for 5 sequences
    // of 169 tokens and 64 heads, and go straight.)  place(row) is where a row goes.
    template <typename Place>
    __device__ __forceinline__ void store_sums(char* room, int rows, Place&& place) {
#pragma unroll
        for (int part = 0; part < 2; ++part) {               // 64 channels at a time (a row's turned by 4 per row: no two rows of a group of lanes meet in a bank)
            wait_reads();
#pragma unroll
            for (int dt = 0; dt < 2; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float16v& o = Base::o[2 * part + dt];
                    *(float4*)(room + (Base::lane % 32 * 64 + (32 * dt + 8 * i + 4 * Base::half + 4 * Base::lane) % 64) * 4) = float4{o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]};
                }
            wave_sync();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = 4 * i + Base::lane / 16, c = Base::lane % 16 * 4;
                const float4 x = *(const float4*)(room + (r * 64 + (c + 4 * r) % 64) * 4);
                if (r < rows) *(float4*)(place(r) + 64 * part + c) = x;
            }
            wave_sync();
        }
    }
    // the two halves' sums and what they saw, together
    __device__ __forceinline__ void finish() {
        Base::l += other_half(Base::l);
        const float other = other_half(saw ? 1.0f : 0.0f);   // (by all lanes: a lane that saw nothing asks one that may have)
        if (!saw && other == 0.0f) Base::m = -INFINITY;
    }
};

template <int LANES>
__device__ __forceinline__ int least_of_wave(int v) {
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) v = min(v, __shfl_xor(v, d));
    return __builtin_amdgcn_readfirstlane(v);
}

constexpr int kTileBytes = 64 * kRowBytes16;   // of keys, or of values
constexpr int kSumsBytes = 32 * 64 * 4;         // of a wave's sums, 64 channels at a time
constexpr int kWaveBytes = kTileBytes;         // of a wave by itself: 32 positions, keys and values, or the sums of 32 rows

__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }

template <bool BF16>
__device__ __forceinline__ const uint16_t* query_of(const PagedArgs& a, const Row& row) {
    return (const uint16_t*)a.q.data + row.b * a.q.batch + row.head * a.q.head + row.token * a.q.token;
}

// Rows of more than a wave: the waves of a workgroup have rows of their own and share tiles of 64 positions, which travel to LDS while the one before is worked on.
template <bool BF16, int WAVES>
__device__ __forceinline__ void tile_job(const PagedArgs& a, bool prefix, char* lds, int* least, int* any_dropped) {
    static_assert(WAVES * kSumsBytes <= 4 * kTileBytes, "every wave has a part of the buffers for its sums");
    constexpr int TILE = 64, ROWS = WAVES * kWaveRows, LOADS = 16 / WAVES, PARTS = 4 / LOADS;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    Job j;
    if (!job_of<false, TILE, ROWS>(a, prefix, j)) return;
    const int i_row = wave * kWaveRows + lane % 32;
    const Row row = row_of<false>(a, j, i_row);
    int first, wave_first, wave_last;
    if (threadIdx.x == 0) *any_dropped = 0;
    if (prefix) {
        wave_first = least_of_wave<32>(row.last);
        wave_last = j.end;
        if (lane == 0) least[wave] = wave_first;
        __syncthreads();
        first = least[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) first = min(first, least[w]);
        first = __builtin_amdgcn_readfirstlane(first);
    } else {
        first = j.N - j.n + j.row0 / a.G;
        wave_first = j.N - j.n + (j.row0 + min(wave * kWaveRows, j.rows - 1)) / a.G;
        wave_last = j.N - j.n + (j.row0 + min(wave * kWaveRows + kWaveRows - 1, j.rows - 1)) / a.G;
        __syncthreads();
    }

    PagedRows<BF16, TILE / 32> rs;
    rs.seen = Seen{row.last, 0, 0};
    const int granule = wave / PARTS;      // of a tile, whose keys and values the wave fetches (a part of)
    const uint32_t room = lds_address(lds) + granule * 16 * kRowBytes16;
    Directory<false, 4> directory(a, j, j.i_begin, 1, lane, first, wave_first);
    const PageFetch<true, LOADS> fetch_keys(a.pages.k, j.h, a.pages.log2, wave % PARTS, lane);
    const PageFetch<false, LOADS> fetch_values(a.pages.v, j.h, a.pages.log2, wave % PARTS, lane);
    rs.start(query_of<BF16>(a, row), lane, a.scale);
    const int n = j.i_end - j.i_begin;
    const auto fetch = [&](int k, int buffer) __attribute__((always_inline)) {
        int page, pos0;
        directory.one(k, granule, page, pos0);
        fetch_keys(page, pos0, j.end, room + buffer * kTileBytes);
        fetch_values(page, pos0, j.end, room + (2 + buffer) * kTileBytes);
    };
    Edges here;
    directory.load(0);                     // (and the queries are there when it is)
    if (n > 0) {
        here = directory.edges(0);
        fetch(0, 0);
    }
    const auto step = [&](int k, int buffer) __attribute__((always_inline)) {
        char* keys = lds + buffer * kTileBytes;
        char* values = lds + (2 + buffer) * kTileBytes;
        wait_loads<0>();
        if (here.edge && drop_odd_values<BF16, LOADS>(values, wave, lane)) *any_dropped = 1;
        __syncthreads();
        // some of the wave's rows see the tile
        const bool seen = j.begin + (j.i_begin + k) * TILE <= wave_last;
        const uint32_t wave_edge = here.wave_edge;
        int pos0[4];
        if (wave_edge) directory.positions(k, pos0);
        if (k + 1 < n) {
            if (k + 1 - directory.k0 >= directory.kTiles) directory.load(k + 1);
            here = directory.edges(k + 1);
            fetch(k + 1, buffer ^ 1);
        }
        if (!seen) return;
        rs.scores(keys);
        // the first reads ahead of the products, then one beside each
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
        for (int i = 0; i < 10; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 6, 0);
        if (wave_edge) rs.hide(pos0);
        else rs.saw = true;
        rs.move_maximum(a.scale);
        rs.weights();
        rs.add_values(values);
        // the first step's weights, then the others' beside the products
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 28, 0);
#pragma unroll
        for (int i = 0; i < 12; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 7, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    };
    for (int k = 0; k < n; k += 2) {
        step(k, 0);
        if (k + 1 < n) step(k + 1, 1);
    }
    __syncthreads();
    if (*any_dropped) rs.give_odd_values(directory, fetch_values, n, j.end);
    rs.finish();
    if (prefix || a.parts) {
        __syncthreads();                   // (the buffers have been read)
        const int rows = min(kWaveRows, j.rows - wave * kWaveRows);
        if (rows <= 0) return;
        const int64_t place = j.place + wave * kWaveRows;
        if (lane < rows) *(float2*)((prefix ? a.prefix_ml : a.own_ml) + 2 * (place + lane)) = float2{rs.m, rs.l};
        float* const sums = (prefix ? a.prefix_o : a.own_o) + place * kD;
        if (n > 0) rs.store_sums(lds + wave * kSumsBytes, rows, [&](int r) { return sums + r * kD; });
    } else if (i_row < j.rows) {
        rs.seen.last = rs.m != -INFINITY ? 0 : -1;   // (whether the row saw anything)
        rs.store((uint16_t*)a.out.data + row.b * a.out.batch + row.head * a.out.head + row.token * a.out.token);
    }
}

template <bool BF16, bool LISTED, int WAVES>
__device__ __forceinline__ void step_job(const PagedArgs& a, bool prefix, char* lds, float2 (*joined)[kWaveRows]) {
    constexpr int TILE = 32, HALF = TILE / 2 * kRowBytes16, OWN = kWaveBytes;
    static_assert(OWN >= 2 * TILE * kRowBytes16 && OWN >= kWaveRows * kD * 4, "a wave's part of LDS holds a tile, and its sums");
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    Job j;
    if (!job_of<LISTED, TILE, kWaveRows>(a, prefix, j)) return;
    const Row row = row_of<LISTED>(a, j, lane % 32);
    const int first = least_of_wave<32>(row.last);
    const int n = max(0, (j.i_end - j.i_begin - wave + WAVES - 1) / WAVES);   // tiles of this wave

    PagedRows<BF16, 1> rs;
    rs.seen = Seen{row.last, 0, 0};
    Directory<LISTED, 2> directory(a, j, j.i_begin + wave, WAVES, lane, first, first);
    const PageFetch<true, 4> fetch_keys(a.pages.k, j.h, a.pages.log2, 0, lane);
    const PageFetch<false, 4> fetch_values(a.pages.v, j.h, a.pages.log2, 0, lane);
    char* const keys = lds + wave * OWN;
    char* const values = keys + TILE * kRowBytes16;
    const uint32_t keys_at = lds_address(keys), values_at = lds_address(values);
    bool dropped = false;
    int page[2], pos0[2];
    rs.start(query_of<BF16>(a, row), lane, a.scale);   // (there when the directory is)
    directory.load(0);
    if (n > 0) {
        directory.tile(0, page, pos0);
#pragma unroll
        for (int i = 0; i < 2; ++i) fetch_keys(page[i], pos0[i], j.end, keys_at + i * HALF);
#pragma unroll
        for (int i = 0; i < 2; ++i) fetch_values(page[i], pos0[i], j.end, values_at + i * HALF);
    }
    for (int k = 0; k < n; ++k) {
        const bool more = k + 1 < n;
        const bool edge = directory.edges(k).edge;
        wait_loads<8>();
        rs.scores(keys);
        wait_reads();
        int next_page[2] = {0, 0}, next_pos0[2] = {0, 0};
        if (more) {
            if (k + 1 - directory.k0 >= directory.kTiles) directory.load(k + 1);
            directory.tile(k + 1, next_page, next_pos0);
#pragma unroll
            for (int i = 0; i < 2; ++i) fetch_keys(next_page[i], next_pos0[i], j.end, keys_at + i * HALF);
        }
        if (edge) rs.hide(pos0);
        else rs.saw = true;
        rs.move_maximum(a.scale);
        rs.weights();
        if (more) wait_loads<8>();
        else wait_loads<0>();
        if (edge) dropped |= drop_odd_values<BF16, 8>(values, 0, lane);
        rs.add_values(values);
        wait_reads();
        if (more) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                page[i] = next_page[i], pos0[i] = next_pos0[i];
                fetch_values(page[i], pos0[i], j.end, values_at + i * HALF);
            }
        }
    }
    if (__ballot(dropped)) rs.give_odd_values(directory, fetch_values, n, j.end);
    rs.finish();

    // every wave's sums to its own part of LDS (a row's channels turned by 4 per row: no two rows of a group of lanes meet in a bank), then four channels per thread
    const int mine = lane % 32;
    if (mine < j.rows) {
        if (lane < 32) joined[wave][mine] = float2{rs.m, rs.l};
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(float4*)(keys + (mine * kD + (32 * dt + 8 * i + 4 * rs.half + 4 * mine) % kD) * 4) =
                    float4{rs.o[dt][4 * i], rs.o[dt][4 * i + 1], rs.o[dt][4 * i + 2], rs.o[dt][4 * i + 3]};
    }
    __syncthreads();
    for (int at = threadIdx.x; at < j.rows * (kD / 4); at += 64 * WAVES) {
        const int r = at / (kD / 4), c = at % (kD / 4) * 4;
        float m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, joined[w][r].x);
        float4 o{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float2 ml = joined[w][r];
            const float f = __builtin_amdgcn_exp2f(ml.x - fmaxf(m, kNever));
            const float4 x = *(const float4*)(lds + w * OWN + (r * kD + (c + 4 * r) % kD) * 4);
            l = fmaf(f, ml.y, l);
            o.x = fmaf(f, x.x, o.x), o.y = fmaf(f, x.y, o.y), o.z = fmaf(f, x.z, o.z), o.w = fmaf(f, x.w, o.w);
        }
        if (prefix || a.parts) {
            float* po = prefix ? a.prefix_o : a.own_o;
            float* pm = prefix ? a.prefix_ml : a.own_ml;
            if (c == 0) *(float2*)(pm + 2 * (j.place + r)) = float2{m, l};
            *(float4*)(po + (j.place + r) * kD + c) = o;
        } else {
            const float by = divisor_of(l, m != -INFINITY);
            const Row to = row_of<LISTED>(a, j, r);
            uint16_t* out = (uint16_t*)a.out.data + to.b * a.out.batch + to.head * a.out.head + to.token * a.out.token;
            *(uint2v*)(out + c) = uint2v{pack16<BF16>(o.x * by, o.y * by), pack16<BF16>(o.z * by, o.w * by)};
        }
    }
}

// The prefix's work and the sequences' own in one launch, so that the one fills what the other leaves of the chip.
enum { kSteps, kTilesAndSteps, kTiles };      // of the prefix and the own positions
template <bool BF16, bool LISTED, int KIND, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void paged_kernel(PagedArgs a) {
    __shared__ __align__(1024) char lds[KIND == kTiles ? 4 * kTileBytes : WAVES * kWaveBytes];
    __shared__ union {
        float2 joined[WAVES][kWaveRows];
        struct {
            int any_dropped, least[WAVES];
        };
    } more;
    const bool prefix = !LISTED && (int)blockIdx.x < a.prefix_groups;
    if constexpr (KIND != kSteps) {
        if (KIND == kTiles || prefix) return tile_job<BF16, WAVES>(a, prefix, lds, more.least, &more.any_dropped);
    }
    if constexpr (KIND != kTiles) step_job<BF16, LISTED, WAVES>(a, prefix, lds, more.joined);
}

// The partial results of a row, joined: those of the prefix, then those of its own positions; two channels per lane, the parts dealt to the waves of a
// workgroup (a wave by itself where there are few), every load of a wave's first parts asked for at once.
constexpr int kMergeWaves = 4, kFewParts = 4;
template <bool BF16, bool LISTED, int WAVES>
__global__ __launch_bounds__(64 * kMergeWaves) void paged_merge_kernel(PagedArgs a) {
    __shared__ float part[WAVES][kD];
    __shared__ float3 joined[WAVES];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64 % WAVES;
    const int r = blockIdx.x * (kMergeWaves / WAVES) + threadIdx.x / (64 * WAVES);   // [batch][token][query head]
    if (WAVES < kMergeWaves && r >= a.merge_rows) return;
    const int Hkv = a.pages.n_kv_heads, head = r % (Hkv * a.G), token = r / (Hkv * a.G) % a.q_tokens, b = r / (Hkv * a.G) / a.q_tokens;
    const int h = head / a.G, g = head % a.G;
    const int n_prefix = a.prefix_chunks, parts = n_prefix + a.own_chunks;
    const int prefix_row = (b * a.q_tokens + token) * a.G + g, own_row = LISTED ? g : token * a.G + g;
    const int64_t unit = LISTED ? ((int64_t)b * a.q_tokens + token) * Hkv + h : (int64_t)b * Hkv + h;
    const int64_t prefix0 = n_prefix ? ((int64_t)h * a.prefix_row_tiles + prefix_row / a.prefix_rows) * n_prefix * a.prefix_rows + prefix_row % a.prefix_rows : 0;
    const int64_t own0 = (unit * a.own_row_tiles + own_row / a.own_rows) * a.own_chunks * a.own_rows + own_row % a.own_rows;
    float m = kNever, l = 0.0f, x = 0.0f, y = 0.0f;
    bool sees = false;
    constexpr int kAhead = WAVES == 1 ? kFewParts : 8;
    for (int c0 = wave; c0 < parts; c0 += kAhead * WAVES) {
        float2 one[kAhead], oc[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = min(c0 + i * WAVES, parts - 1);
            const bool shared = c < n_prefix;
            const int64_t at = shared ? prefix0 + (int64_t)c * a.prefix_rows : own0 + (int64_t)(c - n_prefix) * a.own_rows;
            one[i] = ((const float2*)(shared ? a.prefix_ml : a.own_ml))[at];
            oc[i] = *(const float2*)((shared ? a.prefix_o : a.own_o) + at * kD + 2 * lane);
        }
        if (token >= length_of(a.q_lengths, b, a.q_tokens)) return;      // (no row: nothing was stored, and nothing is asked of what was loaded)
        float most = m;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            most = fmaxf(most, one[i].x);
            sees |= one[i].x != -INFINITY;
        }
        const float moved = __builtin_amdgcn_exp2f(m - most);
        l *= moved, x *= moved, y *= moved;
        m = most;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (c0 + i * WAVES >= parts || one[i].y == 0.0f) continue;   // (an empty part stored no sums)
            const float w = __builtin_amdgcn_exp2f(one[i].x - m);
            l = fmaf(w, one[i].y, l);
            x = fmaf(w, oc[i].x, x);
            y = fmaf(w, oc[i].y, y);
        }
    }
    if constexpr (WAVES > 1) {
        *(float2*)&part[wave][2 * lane] = float2{x, y};
        if (lane == 0) joined[wave] = float3{m, l, sees ? 1.0f : 0.0f};
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            m = fmaxf(m, joined[w].x);
            sees |= joined[w].z != 0.0f;
        }
        l = x = y = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(joined[w].x - m);
            const float2 o = *(const float2*)&part[w][2 * lane];
            l = fmaf(f, joined[w].y, l);
            x = fmaf(f, o.x, x);
            y = fmaf(f, o.y, y);
        }
    }
    const float by = divisor_of(l, sees);
    uint16_t* to = (uint16_t*)a.out.data + b * a.out.batch + head * a.out.head + token * a.out.token;
    *(uint32_t*)(to + 2 * lane) = pack16<BF16>(x * by, y * by);
}

constexpr int64_t kMostGroups = INT32_MAX / 512;   // a launch's threads are counted in 32 bits
constexpr int64_t kMostParts = (1 << 30) / (4 * (kD + 2));   // rows of partial results of split walks: of more there is enough to do without (less than kMostGroups / 2)
// how a kind of work (the prefix's, the sequences' own) is laid out
struct Part {
    int row_tiles = 1, item_rows = 1, chunks = 0;
    int64_t items = 0;
    int64_t groups() const { return items * chunks; }
    int64_t places() const { return items * chunks * item_rows; }
};
struct Plan {
    Part prefix, own;
    int shared = 0, kind = kSteps, waves = 4;
    bool parts = false;
    int64_t scratch = 0;
};

// `units` of `rows` rows each over at most `most` positions, in tiles of 64 by workgroups of `waves` waves
Part tiles_of(int64_t units, int64_t rows, int64_t most, int waves, int64_t at_once) {
    Part p;
    p.item_rows = waves * kWaveRows;
    p.row_tiles = (int)((rows + p.item_rows - 1) / p.item_rows);
    p.items = units * p.row_tiles;
    p.chunks = p.items ? (int)std::max<int64_t>(std::min<int64_t>(at_once / p.items, (most + 63) / 64 / 4), 1) : 1;
    return p;
}
// the same by `waves` waves by themselves; joined: the results are joined by a merge anyway
Part steps_of(int64_t units, int64_t rows, int64_t most, int waves, bool joined) {
    Part p;
    p.item_rows = (int)std::min<int64_t>(std::max<int64_t>(rows, 1), kWaveRows);
    p.row_tiles = (int)((rows + kWaveRows - 1) / kWaveRows);
    p.items = units * p.row_tiles;
    const int64_t tiles = (most + 31) / 32, at_once = 2048 / waves;
    int64_t chunks = 1;
    if (p.items && tiles > (joined ? 4 : 6) * waves) {
        chunks = std::max(at_once / p.items, tiles / 64);
        chunks = std::min({chunks, (tiles + waves - 1) / waves, std::max<int64_t>(256, tiles / 64), kMostParts / (p.items * p.item_rows)});
    }
    p.chunks = (int)std::max<int64_t>(chunks, 1);
    return p;
}
// Waves of a workgroup of steps: 2048 waves are what the chip holds, 10 tiles what one has at most where that can be.  us, 2 / 4: 256 tokens of 8 heads over 19 blocks
// of 64 113 / 108; 4 / 8: 64 rows of 19 tiles 11.0 / 9.8, 32 heads of 4 over 5000 positions 13.0 / 11.7, 16 ragged sequences of 8 heads up to 32768 220 / 213;
// 4 / 1: 64 sequences of 32 heads up to 2 positions 22.3 / 8.8, 32 of 20 tokens and 32 heads 15.6 / 10.5
int step_waves(int64_t units, int64_t rows, int64_t most) {
    const int64_t items = units * ((rows + kWaveRows - 1) / kWaveRows), tiles = (most + 31) / 32;
    int waves = 1;
    while (waves < 8 && waves < tiles && (items * waves < 2048 || tiles > 10 * waves)) waves *= 2;
    return waves;
}

// Attention of `batch` sequences of `rows` rows to a KV head over `most` positions, of which `shared` are worked on for all of them together.
struct Work {
    int64_t heads, batch, rows, shared, most;
    // lays it out, and says about how many us it takes
    double plan(Plan& p) const {
        const int64_t units = rows ? batch * heads : 0, own = most - shared;
        p.shared = (int)shared;
        p.prefix = Part();
        if (rows > kWaveRows) {
            p.kind = kTiles;
            p.waves = std::max(shared, own) >= 2048 && rows > 128 ? 8 : 4;
            const int64_t at_once = p.waves == 8 ? 256 : 512;
            if (shared) p.prefix = tiles_of(heads, batch * rows, shared, p.waves, at_once);
            p.own = tiles_of(units, rows, own, p.waves, at_once);
        } else if (shared && batch * rows > kWaveRows) {
            p.kind = kTilesAndSteps;
            p.waves = 4;
            // Two workgroups of the prefix to a compute unit where it is most of the work and their chunks stay long, one beside the sequences' own else.  us, 1 / 2: 31583
            // positions for 64 sequences of 3 tokens and 32 heads 183 / 151, but 6517 for 64 of 2 44 / 47, 15597 for 32 of 2 and 16 heads 30 / 33,
            // and 46783 for 32 of 2 and 64 heads that have 4675 of their own each 234 / 256
            p.prefix = tiles_of(heads, batch * rows, shared, 4, 512);
            if (shared < 2048 * (int64_t)p.prefix.chunks || tile_us(heads, batch * rows, shared, 4) < 2 * step_us(units, own, kOnceRate))
                p.prefix = tiles_of(heads, batch * rows, shared, 4, 256);
            p.own = steps_of(units, rows, own, 4, true);
        } else {
            p.kind = kSteps;
            p.waves = shared ? 4 : step_waves(units, rows, most);   // (joined, us of 4 / 8: 12220 shared by 32 sequences of 32 heads 58.7 / 66.8, 501 21.8 / 30.5)
            if (shared) p.prefix = steps_of(heads, batch * rows, shared, p.waves, true);
            p.own = steps_of(units, rows, own, p.waves, shared != 0);
        }
        const bool parts = shared || p.own.chunks > 1;
        double us = rows > kWaveRows ? tile_us(units, rows, own, p.waves) : step_us(units, own, kAgainRate);
        if (shared) us += kJoinUs + (p.kind == kSteps ? step_us(heads, shared, kOnceRate) : tile_us(heads, batch * rows, shared, p.waves));
        return us + (parts ? 2 * 520 * (double)(p.prefix.places() + p.own.places()) / 3e6 : 0.0);
    }
    // bytes per us: of positions that one sequence reads after another (largely from the caches), and of those read once; us that a prefix by itself costs beside its work
    static constexpr double kAgainRate = 12e6, kOnceRate = 6e6, kJoinUs = 8;
    static double tile_us(int64_t units, int64_t rows, int64_t most, int waves) {   // (whole items of rows, at 0.9 PFLOP/s)
        const int64_t item = waves * kWaveRows;
        return (double)units * ((rows + item - 1) / item * item) * most * 4 * kD / 0.9e9;
    }
    static double step_us(int64_t units, int64_t most, double rate) { return (double)units * ((most + 31) / 32) * 2 * 32 * kRowBytes16 / rate; }
};

int finish_plan(Plan& p, int64_t merge_rows) {
    if (!p.shared && merge_rows >= kMostGroups) p.own.chunks = 1;
    p.parts = p.shared || p.own.chunks > 1;
    if (p.prefix.groups() + p.own.groups() > kMostGroups || (p.parts && merge_rows > kMostGroups)) return fail_without_context(SPECACHE_EINVAL, "too many rows");
    p.scratch = p.parts ? (p.prefix.places() + p.own.places()) * (kD + 2) * (int64_t)sizeof(float) : 0;
    return SPECACHE_OK;
}

int check_counts(const specache_pages& c, int batch, int n_q_heads, int q_tokens, int kv_tokens, float sm_scale) {
    if (batch < 0 || q_tokens < 0 || kv_tokens < 0) return fail_without_context(SPECACHE_EINVAL, "batch, q_tokens and kv_tokens must not be negative");
    if (n_q_heads < 1 || n_q_heads % c.n_kv_heads || n_q_heads / c.n_kv_heads > 64)
        return fail_without_context(SPECACHE_EINVAL, "n_q_heads must be a multiple of n_kv_heads, up to 64 of it");
    if (kv_tokens > (int64_t)c.table_pages * c.page_tokens) return fail_without_context(SPECACHE_EINVAL, "kv_tokens is more than the table holds");
    if (!std::isfinite(sm_scale)) return fail_without_context(SPECACHE_EINVAL, "sm_scale must be finite");
    const int64_t rows = (int64_t)batch * q_tokens;
    if (rows > (1 << 28) || rows * n_q_heads > (1 << 28)) return fail_without_context(SPECACHE_EINVAL, "too many rows");
    return SPECACHE_OK;
}

int plan_of(const specache_pages* cache, const specache_paged_config* c, Plan& p) {
    if (int rc = check_pages(cache)) return rc;
    if (!c) return fail_without_context(SPECACHE_EINVAL, "null configuration");
    if (int rc = check_counts(*cache, c->batch, c->n_q_heads, c->q_tokens, c->kv_tokens, c->sm_scale)) return rc;
    if (c->shared_tokens < 0) return fail_without_context(SPECACHE_EINVAL, "shared_tokens must not be negative");
    const int G = c->n_q_heads / cache->n_kv_heads;
    const int64_t rows = (int64_t)c->q_tokens * G;
    const int64_t units = rows ? (int64_t)c->batch * cache->n_kv_heads : 0;
    // Shared where that takes less time by the estimate.  us, shared / not: 16 sequences of 69 tokens behind 323 positions 33 / 19, 3 steps behind 13424 25 / 20, 64 of one head
    // behind 13559 with 116 tokens 517 / 453; 32 steps of 32 heads behind 12220 59 / 880, 64 of 3 tokens behind 31583 151 / 580.  The 60 calls of several
    // sequences behind a prefix that random.Random(1) to (250) draw in perf/more_operators.py take 36.1 so, 41.2 always shared, 49.3 never (geometric means), 35.2 at best: 6 are off
    // by more than 5 % (one KV head behind 9313 for 32 of 2 23.2 / 25.7; furthest, 64 steps of 32 heads behind 156 with 6 of their own 30.4 / 16.2).
    Work alone{cache->n_kv_heads, c->batch, rows, 0, c->kv_tokens};
    const double us = alone.plan(p);
    if (c->batch > 1 && units && units * rows < kMostGroups / 2) {   // (the prefix's workgroups and the others' are one launch)
        Work joined = alone;
        joined.shared = std::min(c->shared_tokens, c->kv_tokens) / cache->page_tokens * cache->page_tokens;
        Plan q;
        if (joined.shared && joined.plan(q) < us) p = q;
    }
    return finish_plan(p, c->batch * rows * cache->n_kv_heads);
}

}  // namespace

int check_blocks(const specache_pages* cache, const specache_block_config* c) {
    if (int rc = check_pages(cache)) return rc;
    if (!c) return fail_without_context(SPECACHE_EINVAL, "null configuration");
    if (int rc = check_counts(*cache, c->batch, c->n_q_heads, c->q_tokens, c->kv_tokens, c->sm_scale)) return rc;
    const int64_t slots = (int64_t)c->top + c->first + c->recent;
    if (c->top < 0 || c->first < 0 || c->recent < 0 || slots < 1 || slots > (1 << 20))
        return fail_without_context(SPECACHE_EINVAL, "top, first and recent must not be negative, and make up from 1 to 2^20 entries");
    if ((int64_t)c->batch * c->q_tokens * cache->n_kv_heads > kMostGroups) return fail_without_context(SPECACHE_EINVAL, "too many lists");
    return SPECACHE_OK;
}

namespace {

int plan_of_blocks(const specache_pages* cache, const specache_block_config* c, Plan& p) {
    if (int rc = check_blocks(cache, c)) return rc;
    const int64_t slots = (int64_t)c->top + c->first + c->recent, blocks = (c->kv_tokens + cache->page_tokens - 1) / cache->page_tokens;
    const int64_t units = (int64_t)c->batch * c->q_tokens * cache->n_kv_heads;
    const int G = c->n_q_heads / cache->n_kv_heads;
    p.waves = step_waves(units, G, std::min(slots, blocks) * cache->page_tokens);
    p.own = steps_of(units, G, std::min(slots, blocks) * cache->page_tokens, p.waves, false);
    return finish_plan(p, units * G);
}

}  // namespace

int block_attend_scratch(const specache_pages& cache, const specache_block_config& c, int64_t* bytes) {
    Plan p;
    if (int rc = plan_of_blocks(&cache, &c, p)) return rc;
    *bytes = p.scratch;
    return SPECACHE_OK;
}

namespace {

PagedArgs args_of(const specache_pages& cache, const Plan& p, int batch, int n_q_heads, int q_tokens, int kv_tokens, float sm_scale, const specache_view* q,
                  const specache_view* out, const int32_t* q_lengths, const int32_t* kv_lengths, void* scratch) {
    PagedArgs a{};
    a.q = *q;
    a.out = *out;
    a.pages = page_args(cache);
    a.q_lengths = q_lengths;
    a.kv_lengths = kv_lengths;
    a.prefix_o = (float*)scratch;
    a.own_o = a.prefix_o + p.prefix.places() * kD;
    a.prefix_ml = a.own_o + p.own.places() * kD;
    a.own_ml = a.prefix_ml + p.prefix.places() * 2;
    a.batch = batch;
    a.G = n_q_heads / cache.n_kv_heads;
    a.q_tokens = q_tokens;
    a.kv_tokens = cache.n_pages ? kv_tokens : 0;
    a.shared = cache.n_pages ? p.shared : 0;
    a.prefix_groups = (int)p.prefix.groups();
    a.own_chunks = p.own.chunks;
    a.own_row_tiles = p.own.row_tiles;
    a.own_rows = p.own.item_rows;
    a.prefix_chunks = p.prefix.chunks;
    a.prefix_row_tiles = p.prefix.row_tiles;
    a.prefix_rows = p.prefix.item_rows;
    a.parts = p.parts;
    a.merge_rows = batch * q_tokens * n_q_heads;
    a.scale = (sm_scale > 0.0f ? sm_scale : 0.08838834764831845f) * kLog2e;
    return a;
}

template <bool BF16, bool LISTED>
void launch_merge(const Plan& p, const PagedArgs& a, hipStream_t stream) {
    if (!p.parts) return;
    if (a.prefix_chunks + a.own_chunks <= kFewParts)
        hipLaunchKernelGGL((paged_merge_kernel<BF16, LISTED, 1>), dim3((unsigned)((a.merge_rows + kMergeWaves - 1) / kMergeWaves)), dim3(64 * kMergeWaves), 0, stream, a);
    else hipLaunchKernelGGL((paged_merge_kernel<BF16, LISTED, kMergeWaves>), dim3((unsigned)a.merge_rows), dim3(64 * kMergeWaves), 0, stream, a);
}

template <bool BF16, bool LISTED>
void launch(const Plan& p, const PagedArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)(p.prefix.groups() + p.own.groups()));
    const auto steps = p.waves == 8 ? paged_kernel<BF16, LISTED, kSteps, 8> : p.waves == 4 ? paged_kernel<BF16, LISTED, kSteps, 4>
                       : p.waves == 2 ? paged_kernel<BF16, LISTED, kSteps, 2> : paged_kernel<BF16, LISTED, kSteps, 1>;
    const auto kernel = LISTED || p.kind == kSteps ? steps
                        : p.kind == kTilesAndSteps ? paged_kernel<BF16, false, kTilesAndSteps, 4>
                        : p.waves == 8             ? paged_kernel<BF16, false, kTiles, 8>
                                                   : paged_kernel<BF16, false, kTiles, 4>;
    hipLaunchKernelGGL(kernel, grid, dim3(64 * p.waves), 0, stream, a);
    launch_merge<BF16, LISTED>(p, a, stream);
}

int check_call(const specache_pages& cache, const Plan& p, const specache_view* q, const specache_view* out, int batch, int n_q_heads, int q_tokens,
               int kv_tokens, const int32_t* q_lengths, const int32_t* kv_lengths, void* scratch, int64_t scratch_bytes) {
    if (!q || !out) return fail_without_context(SPECACHE_EINVAL, "null view");
    if (!view_fits(*q) || !view_fits(*out)) return fail_without_context(SPECACHE_EINVAL, "a view's address must be 16-byte aligned, its strides multiples of 8");
    if (!rows_apart(*out, batch, n_q_heads, q_tokens)) return fail_without_context(SPECACHE_EINVAL, "the output's rows share memory");
    if ((uintptr_t)q_lengths % 4 || (uintptr_t)kv_lengths % 4) return fail_without_context(SPECACHE_EINVAL, "misaligned lengths");
    if (kv_tokens)
        if (int rc = check_page_views(cache, true, false)) return rc;
    if (p.scratch) {
        if (!scratch || (uintptr_t)scratch % 16) return fail_without_context(SPECACHE_EINVAL, "scratch must be 16-byte aligned");
        if (scratch_bytes < p.scratch) return fail_without_context(SPECACHE_ECAPACITY, "scratch is smaller than the call needs");
    }
    return SPECACHE_OK;
}

}  // namespace
}  // namespace specache

using namespace specache;

extern "C" {

int specache_paged_scratch(const specache_pages* cache, const specache_paged_config* cfg, int64_t* bytes) {
    Plan p;
    if (int rc = plan_of(cache, cfg, p)) return rc;
    if (!bytes) return fail_without_context(SPECACHE_EINVAL, "null output");
    *bytes = p.scratch;
    return SPECACHE_OK;
}

int specache_paged_attend(const specache_pages* cache, const specache_paged_config* cfg, const specache_view* q, const specache_view* out,
                          const int32_t* q_lengths, const int32_t* kv_lengths, void* scratch, int64_t scratch_bytes, void* stream) {
    Plan p;
    if (int rc = plan_of(cache, cfg, p)) return rc;
    if (!p.own.items) return SPECACHE_OK;
    if (int rc = check_call(*cache, p, q, out, cfg->batch, cfg->n_q_heads, cfg->q_tokens, cfg->kv_tokens, q_lengths, kv_lengths, scratch, scratch_bytes)) return rc;
    const PagedArgs a = args_of(*cache, p, cfg->batch, cfg->n_q_heads, cfg->q_tokens, cfg->kv_tokens, cfg->sm_scale, q, out, q_lengths, kv_lengths, scratch);
    if (cache->dtype == SPECACHE_BF16) launch<true, false>(p, a, (hipStream_t)stream);
    else launch<false, false>(p, a, (hipStream_t)stream);
    return launched();
}

int specache_block_attend(const specache_pages* cache, const specache_block_config* cfg, const specache_view* q, const specache_view* out,
                          const int32_t* blocks, const int32_t* q_lengths, const int32_t* kv_lengths, void* scratch, int64_t scratch_bytes, void* stream) {
    Plan p;
    if (int rc = plan_of_blocks(cache, cfg, p)) return rc;
    if (!p.own.items) return SPECACHE_OK;
    if (int rc = check_call(*cache, p, q, out, cfg->batch, cfg->n_q_heads, cfg->q_tokens, cfg->kv_tokens, q_lengths, kv_lengths, scratch, scratch_bytes)) return rc;
    if (!blocks || (uintptr_t)blocks % 4) return fail_without_context(SPECACHE_EINVAL, "null or misaligned blocks");
    PagedArgs a = args_of(*cache, p, cfg->batch, cfg->n_q_heads, cfg->q_tokens, cfg->kv_tokens, cfg->sm_scale, q, out, q_lengths, kv_lengths, scratch);
    a.blocks = blocks;
    a.slots = cfg->top + cfg->first + cfg->recent;
    if (cache->dtype == SPECACHE_BF16) launch<true, true>(p, a, (hipStream_t)stream);
    else launch<false, true>(p, a, (hipStream_t)stream);
    return launched();
}

}  // extern "C"
