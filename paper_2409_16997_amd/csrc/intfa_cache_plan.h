// How the calls on a quantized cache are carried out: the rules that pick kernels and parts from the sizes of a call, for the host alone (tests ask them which kernel they reach).
#ifndef INTFA_CACHE_PLAN_H
#define INTFA_CACHE_PLAN_H

namespace ifa_cache {

constexpr int TILE_ROWS = 128, TILE_KEYS = 64;                   // of the kernels for many rows
constexpr int MOST_PARTS = 64;

// ---- attention -------------------------------------------------------------------------------------------------
enum AttentionWay {
    WAY_FEW,                   // the 32-row kernel: own keys, with shared keys in front those, too
    WAY_BOTH_FEW,              // one launch, shared keys for the whole batch by 32 rows, own keys by 32 rows
    WAY_BOTH_TILE,             // one launch, shared keys by tiles of 128 rows, own keys by 32 rows
    WAY_TILE,                  // tiles: own keys
    WAY_TILE_FRONT,            // tiles: shared keys, then own ones
    WAY_TILE_APART             // tiles: shared keys for the whole batch, and own keys
};
// In how many parts the shared keys and the own keys of a unit are taken, each part leaving 4 (d + 2) bytes a row.
struct AttentionPlan {
    AttentionWay way;
    int shared, own;                       // parts of the shared keys taken for the whole batch (0: every sequence reads them), and of the own keys
    long rows_shared, rows_own;            // rows of parts: all units x parts x rows
    int ahead;                             // WAY_FEW: tiles that a wavefront copies ahead
    bool once;                             // WAY_FEW: with the non-temporal hint
    bool join() const { return shared > 0 || own > 1; }
    long bytes(int d) const { return (rows_shared + rows_own) * (4L * d + 8); }
};

static inline long row_tiles(bool few, long rows) { return few ? (rows + 31) / 32 : (rows + TILE_ROWS - 1) / TILE_ROWS; }
// Workgroups of a launch of the 32-row kernel: eight shares of the keys at a time, one for each XCD
static inline long few_grid(long units, long splits, long rows) { return (units * splits + 7) / 8 * 8 * row_tiles(true, rows); }
// The kernel for 32 rows, whose wavefronts share the keys out among themselves, or tiles of 128.  Own keys: 32 rows as long as that leaves half of the CUs without one (us, 32 rows / 128, 8 key heads,
// groups of 4, window 4096: 64 queries 20.8 / 22.6, 256 queries 41.6 / 34.7; 2 x 4 heads of d = 64, 300 queries, window 1000: 9.9 / 12.8).  Shared keys: the tiles read them once for
// 128 rows of the batch (64 sequences x 4 rows on 8192 keys 43 / 30 in all).
static inline bool few_rows(bool all, long units, long rows) { return rows <= 32 || (!all && units * ((rows + 31) / 32) <= 128); }
// Parts where there is less than a workgroup for each of `places`, as many as there are, of at least `least` keys each.  Under 512 keys the second launch that joins them costs more than it
// gains (one sequence on 261 keys 6.2 us whole, 7.5 in two; 16 x 8 heads on 4096 of up to 16384 keys 39 in two parts each, 44 in four; one x 8 on 4096 12 in 32, 13 in 16).
static inline int parts_for(long places, long groups, long keys, long least) {
    long parts = keys < 512 ? 1 : places / groups;
    if (parts > keys / least) parts = keys / least;
    return static_cast<int>(parts < 1 ? 1 : parts > MOST_PARTS ? MOST_PARTS : parts);
}

// key_bytes: of a key and its value.  window, sinks <= Nk
static inline AttentionPlan attention_plan(int B, int Hkv, int G, int Nq, int Np, int Nk, int window, int sinks, int key_bytes) {
    const long units = static_cast<long>(B) * Hkv, rows = static_cast<long>(G) * Nq;
    AttentionPlan p = {};
    const long span = static_cast<long>(window) + (Nq < TILE_ROWS ? Nq : TILE_ROWS) + sinks, keys = Nk < span ? Nk : span;
    const bool few = few_rows(false, units, rows);
    p.way = few ? WAY_FEW : WAY_TILE;
    p.own = parts_for(few ? 256 : 512, units * row_tiles(few, rows), keys, few ? 128 : 256);
    // Few keys: every sequence reads the shared ones, too (2 sequences on 300 + 40 keys 6.2 us, with a launch for the parts 7.4; on 600 + 100 12.1 and 9.1).  So it does with many rows of
    // its own, unless tiles of the batch's rows on the shared keys are so many fewer that it pays for the parts: 8 x 8 heads, 4 x 512 queries on 2048 + 512 keys 143 us, with parts 184;
    // 64 x 8 heads, 8 x 10 queries on 4000 + 50 (64 tiles a head for 40: 2400 keys a tile) 106 and 117; 6 x 8 heads, 4 x 40 queries on 32000 + 50 (12 for 8: 16000) 169 and 136.
    if (Np > 0) {
        const long all = rows * B, all_tiles = row_tiles(false, all);
        const bool parts = few ? static_cast<long>(Np) + Nk >= 512 : (B * row_tiles(false, rows) - all_tiles) * Np > 6000 * all_tiles;
        // (own keys in the same launch: a place on every CU is left to them; 64 sequences x 8 heads on 8192 + 512 keys 28.5 us, with 384 places 34, with 512 38)
        if (parts) {
            const bool shared_few = few_rows(true, Hkv, all);
            p.shared = parts_for(few ? 256 : 512, Hkv * row_tiles(shared_few, all), Np, 256);
            p.way = !few ? WAY_TILE_APART : shared_few ? WAY_BOTH_FEW : WAY_BOTH_TILE;
        } else if (!few) {
            p.own = parts_for(512, units * row_tiles(false, rows), keys + Np, 256);
            p.way = WAY_TILE_FRONT;
        }
        p.rows_shared = Hkv * all * p.shared;
    }
    p.rows_own = p.join() ? units * rows * p.own : 0;
    if (p.way == WAY_FEW) {
        // with the non-temporal hint where what is read once does not stay in the caches anyway: 32 x 8 heads on 4096 keys 67 us against 76, 64 x 8 on 512 26 / 28; 4 x 8 on 4096 (50 MB) the same
        const long in_window = window < Nk - sinks ? window : Nk - sinks, read = Nk < in_window + sinks ? Nk : in_window + sinks;
        p.once = row_tiles(true, rows) == 1 && units * read * key_bytes > 64L << 20;
        // One workgroup to a CU copies two tiles ahead; more of them fit with one (64 x 8 heads on 512 keys 26 us, with two 27; 16 x 8 on 4096 in 256 workgroups 41 and 39)
        p.ahead = few_grid(units, p.own, rows) > 256 ? 1 : 2;
    }
    return p;
}

// ---- key weights ---------------------------------------------------------------------------------------------------
// Most rows whose scores are stored, 8 bytes a row and key out and in, rather than K read and multiplied again, d bytes a key.  Stored / again, us, d = 128: 16 sequences x 8 heads x 16384 keys, 8 rows
// 77 / 120, 16 rows 101 / 120; 1 x 8 x 4096, 16 rows 10.3 / 11.0; 32 x 8 x 2000 30.4 / 34.6.  d = 64: 16 x 8 x 16384, 9 rows 63 / 71, 12 rows 73 / 72, 16 rows 86 / 72; 4 x 8 x 8192 17.4 / 18.5, 19.3 / 18.6, 21.3 / 18.7;
// 16 x 8 x 4096 19.7 / 24.1, 21.2 / 23.9, 23.4 / 24.2.
constexpr int STORED_ROWS = 16;
static inline int stored_rows(int d) { return d == 64 ? 12 : STORED_ROWS; }
constexpr int KW_ROWS = 64, KW_KEYS = 256;                       // of a workgroup of the second pass that computes them again

struct WeightsPlan {
    int parts, slices;                     // of the keys in the first pass, of the rows in the second
    bool stored, few, once;                // scores are stored; the first pass by 32 rows (tiles of 128 otherwise), with the non-temporal hint
    long stats, rows, scores, sums;        // bytes
    long stride;                           // of a row of scores
    long bytes() const { return stats + rows + scores + sums; }
};
static inline WeightsPlan weights_plan(int B, int Hkv, int G, int Nq, int Nk, int d) {
    const long units = static_cast<long>(B) * Hkv, rows = static_cast<long>(G) * Nq;
    auto up = [](long n) { return (n + 255) / 256 * 256; };
    WeightsPlan p = {};
    p.stored = rows <= stored_rows(d);
    // The kernel for 32 rows for up to 512 of its tiles of up to 400 K keys in all, then tiles of 128, which read K a quarter as often and take longer to start and to end.  32 rows / 128, us, in all, d = 128 unless
    // stated (key heads x rows x keys): 8 x 400 x 1024 16.0 / 20.3, 32 x 128 x 1024 16.6 / 19.0, 8 x 200 x 4096 19.6 / 21.0, 128 x 64 x 1024 19.4 / 20.3, 128 x 128 x 512 16.8 / 19.4, 12 x 100 x 8192 25.4 / 26.6;
    // 8 x 200 x 8192 26.8 / 25.2, 16 x 256 x 4096 26.6 / 25.3, 64 x 200 x 1024 26.4 / 25.8, 128 x 128 x 2048 34.9 / 30.7, 16 x 100 x 16384 36.5 / 32.2, 256 x 200 x 256 24.1 / 21.1; d = 64, 32 x 512 x 512 14.2 / 17.1,
    // 16 x 512 x 2048 21.0 / 21.9, 8 x 384 x 16384 36.3 / 33.2.  Within .4 % of the faster one over 414 calls of 64 to 16384 keys, 9 % off at worst.
    const long few_tiles = units * ((rows + 31) / 32), tiles = units * ((rows + TILE_ROWS - 1) / TILE_ROWS);
    p.few = rows <= 32 || (few_tiles <= 512 && few_tiles * Nk <= 400 << 10);
    // with the non-temporal hint where K is read once and does not stay in the caches anyway (16 x 8 heads on up to 16384 keys 45.0 us against 47.4)
    p.once = p.few && p.stored && units * Nk * d > 64L << 20;
    // As many parts as there are places for 4 workgroups a CU (16 x 8 heads on up to 16384 keys 41.3 us, for 2 46.2; 32 x 800 rows on 8192 117.9 and 125.2), of at least 512 keys each, or 256 where few
    // rows have to be joined (8 heads, 24 rows on 4096 keys 10.9 and 13.2; 64 rows on 8192 16.7 and 15.2).
    long parts = 1024 / (p.few ? few_tiles : tiles);
    const long least = rows <= 32 ? 256 : 512;
    if (parts > Nk / least) parts = Nk / least;
    p.parts = static_cast<int>(parts < 1 ? 1 : parts > MOST_PARTS ? MOST_PARTS : parts);
    p.stats = p.parts > 1 || p.stored ? up(units * rows * p.parts * 8) : 0;
    p.stride = (Nk + 31L) / 32 * 32;
    if (p.stored) {
        p.scores = up(units * rows * p.stride * 4);
        p.slices = 1;
    } else {
        p.rows = up(units * rows * 8);
        const long groups = units * ((Nk + KW_KEYS - 1) / KW_KEYS), most = (rows + KW_ROWS - 1) / KW_ROWS;
        long slices = (1024 + groups - 1) / groups;              // four workgroups a CU here, too
        if (slices > most) slices = most;
        p.slices = static_cast<int>(slices < 1 ? 1 : slices > 64 ? 64 : slices);
        p.sums = p.slices > 1 ? up(units * Nk * 4L * p.slices) : 0;
    }
    return p;
}

// ---- eviction ------------------------------------------------------------------------------------------------------
constexpr int SEL_THREADS = 1024, SEL_ROUND = 4 * SEL_THREADS;
// Rounds of keys whose weights stay in registers (0: they are read again for each pass)
static inline int evict_rounds(int Nk) { return Nk <= 1 * SEL_ROUND ? 1 : Nk <= 4 * SEL_ROUND ? 4 : Nk <= 8 * SEL_ROUND ? 8 : 0; }

}  // namespace ifa_cache

#endif
