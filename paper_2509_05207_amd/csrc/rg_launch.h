// Launch shapes that follow from sizes alone.  Nothing of HIP is used here, so that they can be compiled and tested by themselves.
#pragma once
#include <algorithm>
#include <stdint.h>

namespace rg {

// HIP documents that a launch has fewer than 2^32 work-items along x (the runtime this was tested on also ran 2^32 + 512 of them rightly; nothing promises it).
constexpr uint64_t MAX_WORK_ITEMS = 0xFFFFFFFFull;
// Workgroups for n_groups shares of work, for kernels whose workgroups take a further share where there are more shares than workgroups.
inline uint32_t grid_for(int64_t n_groups, uint32_t threads) { return (uint32_t)std::max<int64_t>(1, std::min<int64_t>(n_groups, (int64_t)(MAX_WORK_ITEMS / threads))); }

// ---------------------------------------------------------------- the O(f) sampler (sample_positions_kernel)
constexpr int POS_THREADS = 256;
constexpr int POS_WAVES = POS_THREADS / 64;
constexpr int POS_DRAWS = 256;           // positions of a wave in LDS (the launch of 25 M draws with 64 / 128 / 256 / 384 / 512: 468 / 346 / 292 / 318 / 328 us)
constexpr int POS_LEAST = 64;            // draws per unit, at least, where there are few
struct PositionUnits {
    uint32_t nodes;                      // of a unit
    int64_t n;
    uint32_t grid;
};
// As many draws to a unit as a wave has room for, or as few as give every wave that the chip holds a unit.  by_place: the units of each of beta batches
// are counted as those of the longest (see ByPlace).  A wave per unit: waves that walk over the units by turns drift apart, and with them what they read (292
// us, so 312); only where a launch cannot have that many waves do they.
// scattered: the waves mark their n_samples in maps of 8.4 M IDs and more.  Every mark is then a line of its own, which the launch waits for, and fewer draws to a
// unit pay up to POS_SCATTERED rounds of waves, as long as a unit has POS_SAMPLES of the samples (15 M nodes, rows of 30 IDs, units of 256 / 128 / 64 draws, us: 150,000 nodes of fan-out 16
// 130 / 119 / 115, 30 212 / 198 / 189; 1,000,000 of 4 198 / 187 / 179, of 10 397 / 388 / 388, of 23 871 / 872 / 917; rows of 100, 150,000 of 50 339 / 315 / 309; 60 M nodes, rows of 8 IDs,
// 1,000,000 of 10 440 / 417 / 401, of 50 406 / 403 / 482).
constexpr int64_t POS_SCATTERED = 16, POS_SAMPLES = 32;
inline PositionUnits position_units(int64_t n_cur, int64_t n_samples, uint32_t fanout, bool by_place, int64_t longest, uint32_t beta, int n_cu, bool scattered)
{
    const int64_t waves = (int64_t)n_cu * 32, all = n_cur * (int64_t)fanout;
    const auto nodes_of = [&](int64_t draws) { return std::max<int64_t>(1, std::min<int64_t>(64, draws / fanout)); };
    int64_t draws = POS_DRAWS;
    while (draws > POS_LEAST && (all < draws * waves || (scattered && all < draws * waves * POS_SCATTERED && nodes_of(draws / 2) * n_samples >= POS_SAMPLES * n_cur))) draws /= 2;
    const int64_t nodes = nodes_of(draws);
    const int64_t n = by_place ? (longest + nodes - 1) / nodes * beta : (n_cur + nodes - 1) / nodes;
    return PositionUnits{(uint32_t)nodes, n, grid_for((n + POS_WAVES - 1) / POS_WAVES, POS_THREADS)};
}

// ---------------------------------------------------------------- remote rows out of pinned memory (gather_remote_kernel)
constexpr int CHUNKS_IN_FLIGHT = 8;      // loads a lane has under way (of both gather kernels)
constexpr int64_t LINK_BYTES = 2 << 20;
struct RemoteShape {
    int per_wave;                        // consecutive rows of a wave's round
    int64_t parts;                       // waves to a row (then per_wave is 1)
    int64_t waves;
};
// n_remote of n_rows rows are remote, pieces to a row, vec bytes to a piece.
inline RemoteShape remote_shape(int64_t n_rows, int64_t n_remote, uint64_t pieces, int vec, int n_cu)
{
    // Two pieces a lane, or a single row, fewer rows where that leaves compute units without waves (rows of 2,408 bytes, 1,971 us at one row a wave
    // and the link's rate, 1,979 at 32; a list of the misses 1,974).
    RemoteShape r{1, 1, 0};
    while (r.per_wave < 64 && r.per_wave * pieces < 128 && n_rows / (2 * r.per_wave) >= (int64_t)n_cu * 8) r.per_wave <<= 1;
    // Few misses of wide rows: a row's pieces are shared out among waves, a round of them (8 KB) or more each (8 rows of 1 MB 440 us with a wave a row, 171 so,
    // 181 with a list of the misses; one 352 / 32 / 39; with parts for 512 waves, not 64, 64 rows of 64 KB 104 us for 88).  Where pieces are single bytes a
    // round has little under way, and more waves of two pieces a lane are the better (500 rows of 9,602 bytes, half of them misses, a wave a row / so / a list 189 / 89 / 93 us;
    // 300 of 3,001, misses alone 76 / 45 / 56; 3,000 of 1,202, a tenth 48 / 37 / 43).
    const uint64_t least = vec == 16 ? 64 * CHUNKS_IN_FLIGHT : 128;
    const int64_t busy = vec == 16 ? 64 : (int64_t)n_cu * 64;
    if (r.per_wave == 1)
        while (n_remote * r.parts < busy && pieces >= (uint64_t)r.parts * 2 * least && n_rows * r.parts <= (int64_t)n_cu * 64) r.parts *= 2;
    // Where all rows would be asked for at once the link is at its best with LINK_BYTES on it, so that the more of its pieces a wave has under way, the fewer
    // waves (a list of misses / all waves / so, us: 1,000 rows of 16 KB, misses alone 326 / 346 / 313; 3,000 of 4 KB 250 / 285 / 244, half of them misses 144 / 160 / 137,
    // a fifth 79 / 70 / 71; 30,000 of 400 bytes 312 / 324 / 300; 20,000 of 2,408 930 / 930 / 922). Where pieces are single bytes fewer waves are slower
    // (20,000 rows of 1,202 bytes, half of them misses 381 / 357 / 390); more rows than the chip holds waves take further rounds anyway.
    const int64_t n_units = (n_rows * r.parts + r.per_wave - 1) / r.per_wave, all_waves = (int64_t)n_cu * 128;
    r.waves = std::min(n_units, all_waves);
    if (vec == 16 && n_units <= all_waves) {
        const double under_way = (double)r.per_wave * (double)pieces / (double)r.parts * (double)n_remote / (double)n_rows;
        r.waves = std::min(r.waves, (int64_t)((double)LINK_BYTES / (16.0 * std::min(64.0 * CHUNKS_IN_FLIGHT, std::max(1.0, under_way)))));
    }
    return r;
}

// ---------------------------------------------------------------- computation blocks
// By ranks (block_ranks_kernel) rather than by tables of positions: where the batches are so many that each has few workgroups to make bitmaps for, and where a
// batch has samples enough to pay for clearing and counting them, some 18 us a round of workgroups at 233,000 nodes (edges: samples of all hops and batches).
// By tables / by ranks, us: 233,000 nodes, 147 batches of 199,000 samples 250 / 176, 31,000 95 / 60, 7,700 53 / 42; 500 of 3,400 74 / 58; 2,000 of 1,400 137 / 163,
// of 300 50 / 157; 100 batches of 200,000 179 / 120, 64 123 / 94, 64 of 7,700 35 / 37; 40 of 200,000 86 / 83, 40 of 31,000 42 / 44, 20 of 200,000 62 / 73, one 32 / 64;
// 30,000 nodes, 64 of 6,000 31 / 26.  Two to eight hops on 20,000 to 160,000 nodes, 64 to 700 batches: 0.34 to 1.05 of the tables' time.
// Behind the first round of workgroups a batch costs 17 ns (two hops) to 28 (four), while the tables of small graphs stay in the L2s, so that there the batch
// has to have the more samples the smaller the graph: 1,000 batches, three hops, 8,000 nodes, 1,000 samples 40 / 45, 2,000 48 / 46; 32,000 nodes, 500
// 40 / 44, 1,000 54 / 46; one hop, 16,000 nodes, 320 27 / 31, 640 34 / 33; 4,000 batches, 8,000 nodes, 1,000 samples 89 / 127, 32,000 nodes 161 / 129;
// 500 batches, two hops, 16,000 nodes, 256 26 / 28, 1,100 33 / 29.
constexpr uint64_t RANK_NODE_SAMPLES = 6000000;          // nodes times samples per batch and bitmap, from which on
inline bool blocks_by_ranks(uint64_t n_nodes, uint32_t L, uint64_t beta, uint64_t edges, int n_cu)
{
    const uint64_t cus = (uint64_t)n_cu, nodes_per_edge = beta * 2 >= cus ? 64 : 16;
    if (beta * 4 < cus || edges * nodes_per_edge < n_nodes * beta) return false;
    const uint64_t least = beta <= cus ? 0 : beta <= 2 * cus ? RANK_NODE_SAMPLES / 4 : RANK_NODE_SAMPLES;
    return edges * n_nodes >= least * (L + 1) * beta;
}

// ---------------------------------------------------------------- layer norm
// Elements of a row in a lane's registers, at most.  The backward pass holds five values to an element (rows of 8,192 bf16, 256 lanes of 32 / 1,024 lanes of 8, us: 150 / 84).
constexpr int norm_elements(bool backward) { return backward ? 16 : 32; }
constexpr int NORM_SUM_COLUMNS = 32, NORM_SUM_THREADS = 1024;
struct NormShape {
    int pack;                            // elements of an access: 16 bytes, or single elements where a row has fewer
    int lanes;                           // of a row: 8 to 64, or a workgroup of 256 or 1,024; 0: the row is longer than that
    int packs;                           // of a lane
    uint32_t grid;                       // workgroups; their waves, or they, take rows by turns
    uint32_t parts;                      // workgroups that share a long row
    uint32_t n_partial;                  // partial sums of every column that the backward pass leaves
    uint32_t column_grid;                // workgroups over the columns of long rows
    uint32_t sum_grid;                   // workgroups that add the partial sums up, NORM_SUM_COLUMNS columns at a time
};
// in_place: the result takes the place of what other workgroups of the row would still read.
inline NormShape norm_shape(int64_t n_rows, int64_t n_cols, int element_bytes, int n_cu, bool backward, bool in_place)
{
    NormShape s{};
    const int v = 16 / element_bytes;
    s.pack = n_cols < v ? 1 : v;
    const int64_t need = (n_cols + s.pack - 1) / s.pack;
    const int64_t most_packs = std::min(4, norm_elements(backward) / s.pack);
    s.lanes = need <= 8 ? 8 : need <= 16 ? 16 : need <= 32 ? 32 : need <= 64 * most_packs ? 64 : need <= 256 * most_packs ? 256 : need <= 1024 * most_packs ? 1024 : 0;
    const int64_t groups = s.lanes == 0 || s.lanes > 64 ? 1 : 256 / s.lanes;
    int64_t most = (int64_t)n_cu * (s.lanes == 1024 || s.lanes == 0 ? 2 : 8);
    if (backward) {
        // As many workgroups as are resident, by the registers that their elements take, so that none waits for another's end; fewer where their partial sums, written and
        // read, would be more than a sixteenth of what the rows are (at least one to a compute unit).
        const int64_t elements = (need + std::max(s.lanes, 1) - 1) / std::max(s.lanes, 1) * s.pack;
        most = std::min((int64_t)n_cu * (s.lanes == 1024 ? 1 : elements <= 4 ? 8 : elements <= 8 ? 4 : 3), std::max<int64_t>(n_cu, n_rows * element_bytes * 3 / 128));
    }
    s.packs = s.lanes ? (int)((need + s.lanes - 1) / s.lanes) : 0;
    s.grid = (uint32_t)std::max<int64_t>(1, std::min(most, (n_rows + groups - 1) / groups));
    s.n_partial = n_rows ? s.grid : 0;
    s.sum_grid = grid_for((n_cols + NORM_SUM_COLUMNS - 1) / NORM_SUM_COLUMNS, NORM_SUM_THREADS);
    s.parts = 1;
    if (s.lanes == 0) {
        while (!in_place && s.parts < 8 && n_rows * s.parts * 2 <= n_cu) s.parts *= 2;
        s.grid = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(n_cu / 4, (n_rows + 7) / 8)) * 8 * s.parts;      // eight rows at a time, one to an XCD
        s.column_grid = (uint32_t)((n_cols + 256 * v - 1) / (256 * v));
        s.n_partial = (uint32_t)std::min<int64_t>(n_rows, std::max<int64_t>(1, (int64_t)n_cu * 4 / s.column_grid));
    }
    return s;
}

// ---------------------------------------------------------------- orthogonalised updates
constexpr int UPDATE_PAD = 64;            // sides are padded to multiples of this: the least tile, and the step along K
inline uint64_t half_tiles(uint64_t n, uint64_t tile)
{
    const uint64_t t = (n + tile - 1) / tile;
    return t * (t + 1) / 2;
}
inline uint64_t whole_tiles(uint64_t n, uint64_t m, uint64_t tile) { return (n + tile - 1) / tile * ((m + tile - 1) / tile); }
// Names of tiles: 64, 96, 128, 192; tiles of 32 and 64 whose blocks have two waves each (32, UPDATE_TILE_SHARED);
// a tile of 128 with less LDS, two of which share a compute unit.
constexpr int UPDATE_TILE_SHARED = 65, UPDATE_TILE_PAIR = 129;
inline int tile_side(int tile) { return tile / 32 * 32; }
// Of the tiles that no waves share the one whose launch is done first: so many tiles to the fullest compute unit, each at what it takes of one that is full (us a step of 64 along K, measured
// on products of 1024 to 4096 a side, of operands in one part and in two), but no less than a tile that has the unit to itself.
template <typename F> inline int update_tile(F &&tiles, int n_cu, bool split)
{
    struct Cost { int tile; double full, alone; };
    static constexpr Cost ONE[] = {{64, 0.20, 0.27}, {96, 0.36, 0.45}, {128, 0.55, 0.53}, {UPDATE_TILE_PAIR, 0.48, 0.85}, {192, 1.0, 0.95}};
    static constexpr Cost TWO[] = {{64, 0.28, 0.45}, {96, 0.60, 0.60}, {128, 0.90, 0.85}, {UPDATE_TILE_PAIR, 0.85, 1.5}, {192, 1.9, 1.9}};
    int best = 64;
    double least = 0;
    for (const Cost &c : split ? TWO : ONE) {
        const double t = std::max(c.alone, c.full * (double)((tiles(c.tile) + n_cu - 1) / n_cu));
        if (least == 0 || t < least) { least = t; best = c.tile; }
    }
    return best;
}

// Of the two shared tiles, which add along K in the same order: that of 32, as long as the chip holds all of them at once.  What a compute unit loads bounds them, and a
// tile of 32 needs half of it (1999 x 517 fp32, us: X X^T by tiles of 64 16.5, of 32 10.8, A^2 9.7 and 6.0).
template <typename F> inline int shared_tile(F &&tiles, int n_cu) { return tiles(32) <= (uint64_t)n_cu * 2 ? 32 : UPDATE_TILE_SHARED; }

// How a matrix' products are made.  Nothing in a result may depend on what else is in the call.  Sums along K are taken in one order by all tiles but the
// shared ones, so that whether tiles are shared goes by the matrix alone.  Operands in two parts have two cross terms, added in an order that is another one in a
// tile's reflection: which elements are reflected, that is the symmetric products' tile, then goes by the matrix alone too.
constexpr uint64_t TINY_WIDE = 256, UPDATE_NARROW = 32;
// fp32 matrices whose products are made in 64 bits: where with operands of 22 bits and sums of 32 the results are further off than by fp32 products.  (Of 48 matrices of n x m so many by more than half: 4 x 50 26, 16 x 200
// 38, 28 x 2,500 10, 33 x 200 3, 36 x 130 to 700 0, 36 x 1,204 9, 40 x 700 0, 40 x 1,204 4, from 44 on none.)
constexpr uint64_t UPDATE_NARROW_SIDE = 48;
inline bool narrow(uint64_t rows, uint64_t cols)
{
    const uint64_t n = std::min(rows, cols), m = std::max(rows, cols);
    return n <= 36 || (n <= UPDATE_NARROW_SIDE && m > 1024);
}
// Columns of a narrow matrix to a part of its first sums, and to a workgroup of the rest: at least as many as keep its waves busy, and 32 parts and workgroups at most (all of them read all parts).
constexpr uint32_t narrow_part(uint64_t m) { return 256 * (uint32_t)((m + 256 * 32 - 1) / (256 * 32)); }
constexpr uint32_t narrow_parts(uint64_t m) { return (uint32_t)((m + narrow_part(m) - 1) / narrow_part(m)); }
constexpr uint32_t narrow_share(uint64_t m) { return std::max(64u, 16 * (uint32_t)((m + 16 * 32 - 1) / (16 * 32))); }
constexpr uint32_t narrow_shares(uint64_t m) { return (uint32_t)((m + narrow_share(m) - 1) / narrow_share(m)); }
struct UpdateKind {
    bool tiny;                           // up to 64 x TINY_WIDE: a workgroup does it all
    bool split;                          // operands in two parts
    int half_tile, whole_tile;           // of the symmetric products and of the others; 0: by all matrices of a launch
    bool narrow;                         // products in 64 bits (fp32 alone: set by who knows the type)
    bool operator==(const UpdateKind &o) const { return narrow == o.narrow && tiny == o.tiny && split == o.split && half_tile == o.half_tile && whole_tile == o.whole_tile; }
};
// wide_type: two parts whatever the size, which is what a result that is rounded once takes, of any type (rg_update.hip asks for nothing else).
inline UpdateKind update_kind(uint64_t rows, uint64_t cols, bool wide_type, int n_cu)
{
    const uint64_t n = std::min(rows, cols), m = std::max(rows, cols);
    if (n <= 64 && m <= TINY_WIDE) return UpdateKind{true, true, 0, 0, false};
    UpdateKind k{false, wide_type || n <= UPDATE_NARROW, 0, 0, false};
    // Shared tiles where there are so few that they do not fill the chip anyway.
    if (whole_tiles(n, m, 64) <= (uint64_t)n_cu) k.whole_tile = UPDATE_TILE_SHARED;
    if (k.whole_tile || half_tiles(n, 32) <= (uint64_t)n_cu) k.half_tile = UPDATE_TILE_SHARED;
    else if (k.split) k.half_tile = update_tile([&](int tile) { return half_tiles(n, tile); }, n_cu, true);
    return k;
}

}  // namespace rg
