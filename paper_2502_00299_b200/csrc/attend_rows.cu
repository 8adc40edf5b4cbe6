// Attention of many query rows of a KV head over a paged cache: the tokens of a turn (each sequence's own rows, causal or all of them), or one
// token of each sequence of a group that shares a long prefix, whose rows are then read once for all of them.
//
//   out = softmax(q K^T / sqrt(d)) V over the rows that a token sees; with a prefix, over its rows and the sequence's own together
//
// A unit of work is a block of up to 256 query rows - tokens times the heads of a KV head's group, so that grouped heads share what is read - of one set
// (a sequence, a prefix) and KV head, over the set's rows in tiles of 128. A CTA has 12 warps:
//   0-3, 4-7   a query row a thread, 128 each: 64 logits out of tensor memory, their maximum, exponentials and sum, and as bf16 back into tensor memory
//   8          hands out the CTA's pieces of units and brings queries and keys into shared memory, by TMA, as the products read them
//   9          the products (tcgen05, M = 128): S = Q K^T of 64 keys and O += P V. Each half has two such S, so that the next logits are there when the
//              exponentials of the last have been taken, and neither waits for the other (with one S of 128 keys, whose products take 1024 clocks instead of
//              1240, rows and products wait in turn: 4096 tokens 425 us instead of 405, 64 sequences 111 instead of 102)
//   10         brings the values
//   11         looks through values that some of a block's tokens must not see
// A copy takes an elected thread 23 clocks to issue, and a tile 460 besides; two warps, for keys and values, bring a tile of both in 1100 clocks from pages of
// 16 rows, and in 2100 where rows come four at a time. A tile of 256 x 128 logits takes 2048 clocks of exponentials and 2480 of products (their operands
// come out of shared memory at its full rate). What bounds it now, 4096 tokens of 32 heads over 8192 rows, 390 us, 1060 TFLOP/s: 3800 clocks a tile, 54 % of them
// products. 64 keys take their rows 1000 clocks (270 for the maximum, 600 for the exponentials, the rest in barriers), the products of both halves 1900, of which 1400 to
// issue and the rest between them, when the tensor cores mostly run dry.
// One pass over the data: a row's reference moves only when a logit lies more than 2^8 above it, and then its O is scaled in tensor memory. P is rounded
// to bf16 once (2^-8 of a weight, independent from row to row, beside the output's own rounding of 2^-8; a second term for the rest, as attend.cu has, would be half as
// many products again), its sum is taken before that, in 32 bits, as O is.
//
// The tiles of all units stand in one line that is dealt evenly to the CTAs, one an SM, so that few rows over a long cache and many over a short one, of
// any lengths, fill all of them. A unit that several CTAs share leaves (reference, sum, O) records in scratch of the call's own, which a second launch
// joins in the order of the CTAs: same result every time. With a prefix, every row has two units, and all of them are joined there.
#include "decode.cuh"
#include "ptx.cuh"
#include "rows.h"

#include <cuda.h>

namespace chunkkv {

namespace {

__device__ int g_gave_up;                             // a kernel abandoned a bounded wait
__device__ long long g_wait_clocks = kWaitLimitClocks;   // behind which it does, and more for more work (Stop)

constexpr int kTile = 128;                            // rows of a tile of queries, keys or values
constexpr int kBlock = 256;                           // query rows of a unit
constexpr int kRowsThreads = 384;
constexpr int kRowWarps = 8;                          // those with query rows
constexpr int kSub = 64;                              // keys of one S
constexpr int kPieces = 4;                            // pieces handed out ahead
constexpr int kMasks = 8;                             // tiles whose masks are kept
// Tiles that the beginning of a unit counts as. us with 1, 2, 3: 8 x 5 tokens 34.7, 34.7, 35.4; 8 x 448 tokens of 64 dims 47.3, 45.0, 51.0; 64 sequences on
// 32768 rows 90, 95, 101; 23 on three prefixes 41.8, 41.6, 40.8; 4096 tokens 399, 396, 394. A tile of a block with rows for one half counts as much as
// one for both (as half of one: 64 sequences 116): it takes its warps as long.
constexpr int kBegin = 2;
constexpr float kSlack = 8.f;
constexpr float kNoValues = -1.f;                     // the sum of a record of no tiles, which has no O. (One whose logits are all -inf has: its values may be infinite.)
constexpr int kPanelBytes = kTile * 128;              // 64 dims of 128 rows

// ------------------------------------------------------------------------------------------------ units
struct Unit {
    int kind, set, h;        // whose rows
    int t0, tokens, g0, heads;   // query rows: tokens t0 .., heads g0 .. of the group
    int limit, step;         // rows that the first token sees (below 0: none), and how many more each further one does
    int keys;                // rows that the last token sees
    __device__ __forceinline__ int rows() const { return tokens * heads; }
    __device__ __forceinline__ int tiles() const { return (keys + kTile - 1) / kTile; }
    // The unit's part of the line, and how many of its tiles lie before place p of it.
    __device__ __forceinline__ int span() const { return tokens > 0 ? tiles() + kBegin : 0; }
    __device__ __forceinline__ static int tiles_before(int p) { return max(p - kBegin, 0); }
};

// The first block of a set with starts: sets before it take at most this many.
__device__ __forceinline__ int base_of(const AttendRowsArgs& a, const RowSets& s, int i) { return s.starts[i] / a.tokens + i; }
// The set whose blocks hold block x.
__device__ __forceinline__ int set_of(const AttendRowsArgs& a, const RowSets& s, int x) {
    int lo = 0, hi = s.n - 1;
#pragma unroll 1
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (base_of(a, s, mid) <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}
__device__ __forceinline__ Unit unit_of(const AttendRowsArgs& a, int u) {
    Unit r;
    const int first = a.sets[0].slots * a.Hkv;
    r.kind = u >= first;
    const RowSets& s = a.sets[r.kind];
    if (r.kind) u -= first;
    r.h = u / s.slots;
    const int slot = u - r.h * s.slots, x = slot / a.head_blocks;
    r.g0 = (slot - x * a.head_blocks) * a.heads;
    r.heads = min(a.heads, a.G - r.g0);
    int n, begin;                                      // tokens of the set, the block's first
    if (r.kind) {
        r.set = x;
        r.t0 = x;
        n = 1;
        begin = 0;
    } else {
        r.set = set_of(a, s, x);
        // (starts that are not ascending make no address out of range: the tokens lie in [0, T))
        const int t = min(max(s.starts[r.set], 0), a.T);
        n = min(max(s.starts[r.set + 1], t), a.T) - t;
        begin = (x - base_of(a, s, r.set)) * a.tokens;
        r.t0 = t + begin;
    }
    r.tokens = begin >= 0 ? max(min(a.tokens, n - begin), 0) : 0;
    r.step = a.causal && r.kind == 0 ? 1 : 0;
    const int len = min(max(s.lengths[static_cast<size_t>(r.set) * a.Hkv + r.h], 0), s.cap);
    r.limit = r.step ? len - (n - 1 - begin) : len;
    r.keys = max(r.limit + r.step * (r.tokens - 1), 0);
    return r;
}

// The line dealt to n CTAs: the first `more` of them have one more.
struct Share {
    int n, per, more;
    __device__ __forceinline__ Share(int total, int ctas) {
        n = min(total, ctas);
        per = n > 0 ? total / n : 0;
        more = total - per * n;
    }
    __device__ __forceinline__ int begin(int cta) const { return cta * per + min(cta, more); }
    __device__ __forceinline__ int owner(int x) const {
        const int wide = more * (per + 1);
        return x < wide ? x / (per + 1) : more + (x - wide) / per;
    }
};

// ------------------------------------------------------------------------------------------------ shared memory
enum Leave { kOut, kWhole, kPart };
struct Piece {
    int tiles, tile0, subs;  // tiles of this piece (-1: no more pieces), the first, and how many 64 keys they hold
    int kind, set, h, t0, g0, heads, rows;
    int limit, step, keys;
    int stage;               // 0, 1: at most 128 rows, on that half of the CTA; 2: both halves
    int leave, slot;
    int found;               // a value that is not finite stood in a row that not all of the block's tokens see
};
struct Stop {
    long long since[kRowsThreads / 32];               // when a warp that waits began to
    // A warp may have nothing to do while others work on all that the CTA has, so the limit of a wait grows with that: 2^-16 of it (30 us) for a tile, which takes 2 us,
    // and 2^-20 for a unit, 32 of which take a few us to look through.
    long long limit;                                  // (none until the warp that hands out pieces has set it)
    int abort;                                        // a warp has given up
    __device__ __forceinline__ void begin(int tiles, int units) {
        limit = g_wait_clocks + (g_wait_clocks >> 16) * tiles + (g_wait_clocks >> 20) * units;
    }
};
template <int D>
struct RowsSmem {
    static constexpr int kTileBytes = kTile * D * 2;
    static constexpr int kSlots = D == 128 ? 5 : 10;  // tiles of keys or values in flight
    alignas(1024) unsigned char q[D / 64][kBlock][128];   // panels of 64 dims; 128 rows a half of the CTA
    alignas(1024) unsigned char kv[kSlots][kTileBytes];   // panels of 64 dims
    Piece piece[kPieces];
    int4 box[2][kTile / 4];                           // where rows of a tile of keys, or of values, are in the cache
    uint32_t mask[kMasks][4];                         // rows of a tile of keys that are there
    unsigned long long kv_full[kSlots], kv_empty[kSlots];
    // A wait names a phase by its parity, so no barrier may complete two phases while a warp still stands in front of a test for the first of them.
    //   *_empty, p_full, scan, scanned   the next phase needs what the waiting warp does behind its wait, so it cannot come
    //   kv_full, q_full                  the next one needs the buffer given back, which the products' warp does behind its last test
    //   piece_full                       the next one needs piece_empty of every warp that waits
    //   mask_full                        the next one is eight tiles on, and keys are at most five ahead of the rows' weights
    //   s_full                           the next one is the commit of a block that needs these weights of all four warps. In the last but one block of a piece no logits
    //                                    come any more, but the last block's rows may wait for its values to move a reference: it commits here too
    //   o_full                           all values of a piece have been added; the next one needs weights that the warp gives behind this wait. (Not s_full: the next
    //                                    piece's logits, which need nothing of the rows' warps, would complete that once more, in front of a warp that comes late.)
    unsigned long long q_full[2], q_empty[2], s_full[2][2], p_full[2][2], o_full[2], o_empty[2];
    unsigned long long piece_full[kPieces], piece_empty[kPieces], mask_full[kMasks], scan, scanned, drained;
    int warp_sum[kRowsThreads / 32], first_unit, first_at;
    Stop stop;
    uint32_t tmem;
};
static_assert(sizeof(RowsSmem<128>) <= 227 * 1024 && sizeof(RowsSmem<64>) <= 227 * 1024, "shared memory of an SM");

// Whether a warp that has tested n times gives up: another one has, or the limit has passed since its 16th test. For all lanes together.
__device__ __noinline__ bool out_of_time(uint32_t n, Stop* stop) {
    const long long now = clock64();
    long long* since = &stop->since[threadIdx.x >> 5];
    if (n == 16) {
        if ((threadIdx.x & 31) == 0) *since = now;
        __syncwarp();
    } else if (now - *since > stop->limit) {
        *const_cast<volatile int*>(&stop->abort) = 1;
    }
    return __any_sync(0xffffffffu, *const_cast<volatile int*>(&stop->abort));
}
// Bounded wait of a whole warp: all lanes test, 60 clocks a time if the phase is over soon and 7800 if not, until it is; every 16th time they look whether to give up,
// 60 us late at most. Few instructions, as it stands in many places: with ptx.cuh's polling in each of them the kernel was 161 KB of code, which no
// instruction cache holds, with out_of_time inlined 10 KB more than now (4096 tokens over 8192 rows 402 us instead of 388).
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, Stop* stop) {
#pragma unroll 1
    for (uint32_t n = 1; !__all_sync(0xffffffffu, mbar_try_wait(bar, parity)); ++n)
        if ((n & 15u) == 0 && out_of_time(n, stop)) return false;
    return true;
}
// Given up: what is under way lands before the CTA ends, which takes microseconds; until a time that all of a role's copies share.
constexpr long long kLandClocks = 1LL << 26;
__device__ __forceinline__ void wait_landing(uint32_t bar, uint32_t parity, long long until) {
#pragma unroll 1
    while (!__all_sync(0xffffffffu, mbar_try_wait(bar, parity)) && !__any_sync(0xffffffffu, clock64() > until)) {}
}

// What a role needs to walk the pieces.
template <int D>
struct Pieces {
    RowsSmem<D>& sm;
    int at = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ explicit Pieces(RowsSmem<D>& s) : sm(s) {}
    __device__ __forceinline__ void next() {
        if (++at == kPieces) { at = 0; phase ^= 1u; }
    }
    __device__ __forceinline__ bool wait() { return wait_warp(smem_u32(&sm.piece_full[at]), phase, &sm.stop); }
};

// A value that is the same for all lanes, and known to be.
__device__ __forceinline__ int same(int v) { return __shfl_sync(0xffffffffu, v, 0); }

// Descriptors of tiles in shared memory (ptx.cuh) with their upper halves apart, which are all alike: 8-row groups 1024 bytes apart, 128-byte swizzle. The
// lower ones are added to in 32 bits, which halves what the products' warp has to execute.
constexpr uint32_t kDescUpper = (1024 >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t desc_lower(uint32_t at, uint32_t panels) { return (at & 0x3FFFFu) >> 4 | (panels >> 4) << 16; }
// D (+)= A B^T, both in shared memory.
__device__ __forceinline__ void umma_ss(uint32_t d_tmem, uint32_t a_lower, uint32_t b_lower, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d_tmem), "r"(a_lower), "r"(b_lower), "r"(idesc), "r"(accumulate), "r"(kDescUpper)
        : "memory");
}
// P (bf16, in tensor memory) times a tile of values, as they lie: rows of 64 dims, the second operand with its columns (dims) side by side, panels of 64 dims
// kPanelBytes apart.
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lower, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\t"
        "setp.ne.b32 p, %4, 0;\n\tmov.b64 b, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d_tmem), "r"(a_tmem), "r"(b_lower), "r"(idesc), "r"(accumulate), "r"(kDescUpper)
        : "memory");
}
constexpr uint32_t kColumnsSideBySide = 1u << 16;     // in an instruction's descriptor: of the second operand

__device__ __forceinline__ void tmem_st_x32(uint32_t taddr, const float (&v)[32]) {
    const uint32_t* r = reinterpret_cast<const uint32_t*>(v);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]),
        "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
        "r"(r[31]), "r"(taddr)
        : "memory");
}
// Four rows of 64 dims, zeros for rows behind the last, one after the other in shared memory.
__device__ __forceinline__ void gather_rows(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, const int (&row)[4]) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(row[0]), "r"(row[1]), "r"(row[2]), "r"(row[3]), "r"(bar)
        : "memory");
}

// A box of rows of 64 dims.
__device__ __forceinline__ void copy_rows(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int row) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(row), "r"(bar)
                 : "memory");
}

// ------------------------------------------------------------------------------------------------ loading
// q: [T, Hq, d] in boxes of a block's heads and tokens, q_thin: of at most 128 rows. k, v: rows of the cache, [pages * page_size, Hkv d], in boxes of
// a.box rows of 64 dims, or (pages that are no multiple of eight rows) of one row, which are fetched in fours.
struct RowMaps {
    CUtensorMap q, q_thin, k, v;
};
// The first tile that holds rows which the block's first token does not see, or that nobody does.
__device__ __forceinline__ int scan_from(const Piece& x) { return (x.step ? max(x.limit, 0) : x.keys) / kTile; }

// Where the rows of tile `tile` are: lane l has box l of them (a.box rows each), or its four rows; -1: not there.
struct Places {
    int4 at;
    __device__ __forceinline__ void find(const AttendRowsArgs& a, const int32_t* table, int tile, int keys) {
        const int lane = threadIdx.x & 31, rows = a.box > 0 ? a.box : 4, r = tile * kTile + lane * rows;
        at = make_int4(-1, -1, -1, -1);
        if (lane * rows >= kTile || r >= keys) return;
        if (a.box > 0) {
            at.x = paged_row(a.cache, table, r);
        } else {
            at.x = paged_row(a.cache, table, r);
            if (r + 1 < keys) at.y = paged_row(a.cache, table, r + 1);
            if (r + 2 < keys) at.z = paged_row(a.cache, table, r + 2);
            if (r + 3 < keys) at.w = paged_row(a.cache, table, r + 3);
        }
    }
};

// A tile of the head whose dims begin at x. Boxes that are not there are zeros (values) or, skipped, whatever was there (keys: their logits are not looked
// at). The whole warp.
template <int D>
__device__ __forceinline__ void load_tile(const AttendRowsArgs& a, RowsSmem<D>& sm, int slot, const CUtensorMap* map, int x, const int4& at, bool values) {
    const int lane = threadIdx.x & 31, rows = a.box > 0 ? a.box : 4, boxes = kTile / rows;
    const int nowhere = a.cache.num_pages * a.cache.page_size;         // behind the last row: zeros
    const bool any = at.x >= 0 || at.y >= 0 || at.z >= 0 || at.w >= 0;
    const uint32_t take = __ballot_sync(0xffffffffu, lane < boxes && (values || any));
    // (one thread issues, with all that a copy takes known to be the same for the warp: 23 clocks a copy, where lanes that hand over their rows one by one take 180)
    int4* box = sm.box[values];
    box[lane] = make_int4(at.x < 0 ? nowhere : at.x, at.y < 0 ? nowhere : at.y, at.z < 0 ? nowhere : at.z, at.w < 0 ? nowhere : at.w);
    __syncwarp();
    const uint32_t bar = smem_u32(&sm.kv_full[slot]), to = smem_u32(sm.kv[slot]);
    if (elect_one()) {
        mbar_arrive_expect_tx(bar, __popc(take) * rows * (D * 2));
        if (a.box > 0) {
#pragma unroll 4
            for (int i = 0; i < boxes; ++i) {
                if (take >> i & 1u) {
#pragma unroll
                    for (int p = 0; p < D / 64; ++p) copy_rows(to + p * kPanelBytes + i * rows * 128, map, bar, x + 64 * p, box[i].x);
                }
            }
        } else {
#pragma unroll 4
            for (int i = 0; i < boxes; ++i) {
                const int row[4] = {box[i].x, box[i].y, box[i].z, box[i].w};
                if (take >> i & 1u) {
#pragma unroll
                    for (int p = 0; p < D / 64; ++p) gather_rows(to + p * kPanelBytes + i * 512, map, bar, x + 64 * p, row);
                }
            }
        }
    }
    __syncwarp();
}
// n tiles of keys and values were asked for, this warp's are those of `parity`.
template <int D>
__device__ void let_land(RowsSmem<D>& sm, int n, int parity, long long until) {
#pragma unroll 1
    for (int i = max(n - RowsSmem<D>::kSlots, 0); i < n; ++i)
        if ((i & 1) == parity) wait_landing(smem_u32(&sm.kv_full[i % RowsSmem<D>::kSlots]), i / RowsSmem<D>::kSlots & 1, until);
}

// What the loading of keys, or of values, keeps from piece to piece.
template <int D>
struct KeyLoader {
    int n_kv = 0, n_tile = 0;                                          // tiles of keys and values, and of keys, so far
    uint32_t q_phase = 3, q_used = 0;                                  // (the first wait for an empty buffer passes)
    __device__ bool load(const AttendRowsArgs& a, const RowMaps& maps, RowsSmem<D>& sm, const Piece& x) {
        const int lane = threadIdx.x & 31;
        const RowSets& s = a.sets[x.kind];
        const int32_t* table = s.tables + static_cast<size_t>(x.set) * s.max_pages;
        Places next;
        next.find(a, table, x.tile0, x.keys);
        const bool wide = x.stage == 2;
#pragma unroll 1
        for (int half = wide ? 0 : x.stage; half <= (wide ? 1 : x.stage); ++half) {
            if (!wait_warp(smem_u32(&sm.q_empty[half]), q_phase >> half & 1u, &sm.stop)) return false;
            q_phase ^= 1u << half;
            q_used |= 1u << half;
        }
        if (elect_one()) {
            // (both halves of a wide block come as one box a panel, on the first half's barrier; the second's is only arrived at)
            const int half = wide ? 0 : x.stage, rows = wide ? a.tokens * a.heads : a.thin_tokens * a.heads;
            const uint32_t bar = smem_u32(&sm.q_full[half]);
            mbar_arrive_expect_tx(bar, rows * (D * 2));
#pragma unroll
            for (int p = 0; p < D / 64; ++p) tma_load_3d(smem_u32(sm.q[p][half * kTile]), wide ? &maps.q : &maps.q_thin, bar, 64 * p, x.h * a.G + x.g0, x.t0);
            if (wide) mbar_arrive(smem_u32(&sm.q_full[1]));
        }
        __syncwarp();
        const int rows = a.box > 0 ? a.box : 4;
#pragma unroll 1
        for (int t = 0; t < x.tiles; ++t, ++n_tile, n_kv += 2) {
            const Places now = next;
            const int slot = n_kv % RowsSmem<D>::kSlots, base = (x.tile0 + t) * kTile;
            if (!wait_warp(smem_u32(&sm.kv_empty[slot]), (n_kv / RowsSmem<D>::kSlots & 1) ^ 1, &sm.stop)) return false;
            load_tile<D>(a, sm, slot, &maps.k, x.h * D, now.at, false);
            // which rows are there: lane l says it of rows 4 l to 4 l + 3. (The mask's last reader is done: its tile lies further back than there are buffers.)
            uint32_t word;
            if (a.box > 0) {
                const uint32_t got = __ballot_sync(0xffffffffu, now.at.x >= 0);
                word = got >> (4 * lane / rows) & 1u ? 15u : 0u;
            } else {
                word = (now.at.x >= 0 ? 1u : 0u) | (now.at.y >= 0 ? 2u : 0u) | (now.at.z >= 0 ? 4u : 0u) | (now.at.w >= 0 ? 8u : 0u);
            }
            const int left = x.keys - base - 4 * lane;
            word = (left >= 4 ? word : left <= 0 ? 0u : word & ((1u << left) - 1u)) << (4 * (lane & 7));
#pragma unroll
            for (int off = 1; off < 8; off <<= 1) word |= __shfl_xor_sync(0xffffffffu, word, off);
            if ((lane & 7) == 0) sm.mask[n_tile % kMasks][lane >> 3] = word;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.mask_full[n_tile % kMasks]));
            if (t + 1 < x.tiles) next.find(a, table, x.tile0 + t + 1, x.keys);
        }
        return true;
    }
    __device__ void give_up(RowsSmem<D>& sm) {
        const long long until = clock64() + kLandClocks;
        let_land(sm, n_kv, 0, until);
#pragma unroll 1
        for (int half = 0; half < 2; ++half)
            if (q_used >> half & 1u) wait_landing(smem_u32(&sm.q_full[half]), q_phase >> half & 1u, until);
    }
};

template <int D>
__device__ void load_values(const AttendRowsArgs& a, const RowMaps& maps, RowsSmem<D>& sm) {
    const int lane = threadIdx.x & 31;
    Pieces<D> pc(sm);
    int n_kv = 1;
    for (;; pc.next()) {
        if (!pc.wait()) break;
        const int tiles = sm.piece[pc.at].tiles, tile0 = sm.piece[pc.at].tile0, keys = sm.piece[pc.at].keys, x = sm.piece[pc.at].h * D;
        const RowSets& s = a.sets[sm.piece[pc.at].kind];
        const int32_t* table = s.tables + static_cast<size_t>(sm.piece[pc.at].set) * s.max_pages;
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.piece_empty[pc.at]));
        if (tiles < 0) return;
        Places next;
        if (tiles > 0) next.find(a, table, tile0, keys);
        bool fine = true;
#pragma unroll 1
        for (int t = 0; t < tiles; ++t, n_kv += 2) {
            const Places now = next;
            const int slot = n_kv % RowsSmem<D>::kSlots;
            fine = wait_warp(smem_u32(&sm.kv_empty[slot]), (n_kv / RowsSmem<D>::kSlots & 1) ^ 1, &sm.stop);
            if (!fine) break;
            load_tile<D>(a, sm, slot, &maps.v, x, now.at, true);
            if (t + 1 < tiles) next.find(a, table, tile0 + t + 1, keys);
        }
        if (!fine) break;
    }
    let_land(sm, n_kv, 1, clock64() + kLandClocks);
}

// A tile of values of which some of the block's tokens, or all, must not see every row: what is not finite there would reach them as 0 * inf. From the
// first such row on it becomes zero, and each dim's first one is kept: who sees that row gets no number there. A warp.
template <int D, class Each>
__device__ __forceinline__ void each_value(unsigned char* tile, int row0, Each each) {
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int p = 0; p < D / 64; ++p) {
#pragma unroll 2
        for (int row = row0 + (lane >> 3); row < kTile; row += 4)
            each(reinterpret_cast<uint4*>(tile + p * kPanelBytes + row * 128) + (lane & 7), row, 8 * ((lane & 7) ^ (row & 7)) + 64 * p);
    }
}
template <int D>
__device__ __noinline__ void take_out(unsigned char* tile, int row0, int* first_bad, bool first, int row_of) {
    if (first) {
        for (int i = threadIdx.x & 31; i < D; i += 32) first_bad[i] = 0x7fffffff;
        __threadfence_block();
        __syncwarp();
    }
    each_value<D>(tile, row0, [&](uint4* at, int row, int dim) {
        const uint4 v = *at;
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
        bool bad = false;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if ((w[e / 2] >> (16 * (e & 1)) & 0x7f80u) == 0x7f80u) {
                w[e / 2] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
                atomicMin(&first_bad[dim + e], row_of + row);
                bad = true;
            }
        if (bad) *at = make_uint4(w[0], w[1], w[2], w[3]);
    });
    __threadfence();
}
template <int D>
__device__ void scan_values(const AttendRowsArgs& a, RowsSmem<D>& sm) {
    const int lane = threadIdx.x & 31;
    Pieces<D> pc(sm);
    int n_kv = 0;
    uint32_t phase = 0;
    for (;; pc.next()) {
        if (!pc.wait()) return;
        Piece& x = sm.piece[pc.at];
        const int tiles = x.tiles, tile0 = x.tile0, from = scan_from(x), first = x.step ? max(x.limit, 0) : x.keys;
        if (tiles < 0) return;
        bool found = false;
        for (int t = max(from - tile0, 0); t < tiles; ++t) {
            unsigned char* tile = sm.kv[(n_kv + 2 * t + 1) % RowsSmem<D>::kSlots];
            if (!wait_warp(smem_u32(&sm.scan), phase, &sm.stop)) return;
            phase ^= 1u;
            const int row0 = max(first - (tile0 + t) * kTile, 0);
            uint32_t bad = 0;
            each_value<D>(tile, row0, [&](uint4* at, int, int) {
                const uint4 v = *at;
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t y = ~w[e] & 0x7f807f80u;            // a half of zeros: all bits of its exponent are set
                    bad |= (y - 0x00010001u) & ~y & 0x80008000u;
                }
            });
            if (__any_sync(0xffffffffu, bad != 0)) {
                take_out<D>(tile, row0, a.first_bad + (static_cast<size_t>(blockIdx.x) * kPieces + pc.at) * D, !found, (tile0 + t - from) * kTile);
                found = true;
                *reinterpret_cast<volatile int*>(&x.found) = 1;
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.scanned));
        }
        n_kv += 2 * tiles;
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.piece_empty[pc.at]));
    }
}

// ------------------------------------------------------------------------------------------------ the products
// A whole warp, one elected thread of which issues: what the products take is then the same for all lanes, and known to be. Little code, in one line for
// both halves: what other warps of its quarter of the SM have pushed out of the instruction cache is fetched anew, 100 to 400 clocks in which the tensor
// cores run dry. Waits that mostly lie behind it are tested together.
template <int D>
struct Products {
    using Smem = RowsSmem<D>;
    static constexpr uint32_t kS = umma_idesc_bf16(kTile, kSub), kO = umma_idesc_bf16(kTile, D) | kColumnsSideBySide;
    Smem& sm;
    const uint32_t tmem, q_desc, k_desc, v_desc;
    int slot = 0;
    uint32_t kv_phase = 0, q_phase = 0, p_phase = 0, scan_phase = 0, o_phase = 3;      // (a bit a half, or 2 * half + S; nothing has to be read out of O first)
    __device__ __forceinline__ Products(Smem& s, uint32_t t)
        : sm(s), tmem(t), q_desc(desc_lower(smem_u32(s.q[0][0]), 16)), k_desc(desc_lower(smem_u32(s.kv[0]), 16)), v_desc(desc_lower(smem_u32(s.kv[0]), kPanelBytes)) {}
    __device__ __forceinline__ bool wait(unsigned long long& bar, uint32_t phase) const { return wait_warp(smem_u32(&bar), phase, &sm.stop); }
    __device__ __forceinline__ void advance() {
        if (++slot == Smem::kSlots) { slot = 0; kv_phase ^= 1u; }
    }
    // S[sub] of a half, by the first or second 64 keys of the tile in slot s
    __device__ __forceinline__ void logits(int half, int s, int sub) {
        const uint32_t k = k_desc + s * (Smem::kTileBytes >> 4) + sub * (kSub * 128 >> 4), q = q_desc + half * (kPanelBytes >> 4), to = tmem + half * kTile + sub * kSub;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) umma_ss(to, q + (i / 4) * (2 * kPanelBytes >> 4) + (i % 4) * 2, k + (i / 4) * (kPanelBytes >> 4) + (i % 4) * 2, kS, i > 0);
    }
    __device__ __forceinline__ void values(int half, int s, int sub, bool more) {
        const uint32_t v = v_desc + s * (Smem::kTileBytes >> 4) + sub * (kSub * 128 >> 4), p = tmem + half * kTile + sub * kSub, to = tmem + 2 * kTile + half * D;
#pragma unroll
        for (int i = 0; i < kSub / 16; ++i) umma_ts(to, p + i * 8, v + i * (2048 >> 4), kO, more || i > 0);
    }
    // P of a half times values, and the next logits in its place. u: the 64 keys' number, of `subs`.
    template <bool WIDE>
    __device__ __forceinline__ void block(int h0, int u, int subs, int v_slot, int k_slot) {
        const int sub = u & 1;
        const bool more = u + 2 < subs;                                // there is a next S for this one's place
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
            for (int i = 0; i < (WIDE ? 2 : 1); ++i) {
                const int half = WIDE ? i : h0;
                values(half, v_slot, sub, u > 0);
                if (more) logits(half, k_slot, sub);
                // (s_full also in the last but one block, where no S comes any more: it says that these values have been added)
                if (u + 1 < subs) umma_commit(smem_u32(&sm.s_full[half][sub]));
                else umma_commit(smem_u32(&sm.o_full[half]));
                if (u + 3 == subs) umma_commit(smem_u32(&sm.q_empty[half]));
            }
            if (sub == 1 || u + 1 == subs) umma_commit(smem_u32(&sm.kv_empty[v_slot]));
            if (more && (sub == 1 || u + 3 == subs)) umma_commit(smem_u32(&sm.kv_empty[k_slot]));
        }
        __syncwarp();
    }
    // WIDE: both halves; else `only`.
    template <bool WIDE>
    __device__ __forceinline__ bool piece(int subs, int scan, int only) {
        const int h0 = WIDE ? 0 : only;
        if (!wait(sm.q_full[h0], q_phase >> h0 & 1u)) return false;
        q_phase ^= 1u << h0;
        if (WIDE) {
            if (!wait(sm.q_full[1], q_phase >> 1 & 1u)) return false;
            q_phase ^= 2u;
        }
        if (!wait(sm.kv_full[slot], kv_phase)) return false;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll 1
            for (int sub = 0; sub < 2 && sub < subs; ++sub)
#pragma unroll 1
                for (int h = h0; h < (WIDE ? 2 : h0 + 1); ++h) {
                    logits(h, slot, sub);
                    umma_commit(smem_u32(&sm.s_full[h][sub]));
                }
            umma_commit(smem_u32(&sm.kv_empty[slot]));
            if (subs <= 2)
                for (int h = h0; h < (WIDE ? 2 : h0 + 1); ++h) umma_commit(smem_u32(&sm.q_empty[h]));
        }
        __syncwarp();
        advance();
        if (!wait(sm.o_empty[h0], o_phase >> h0 & 1u)) return false;
        o_phase ^= 1u << h0;
        if (WIDE) {
            if (!wait(sm.o_empty[1], o_phase >> 1 & 1u)) return false;
            o_phase ^= 2u;
        }
        int v_slot = 0, k_slot = 0;
        uint32_t v_phase = 0, k_phase = 0;
#pragma unroll 1
        for (int u = 0; u < subs; ++u) {
            if ((u & 1) == 0) {
                v_slot = k_slot = slot;                                // (no next tile: the values' once more, which is as well)
                v_phase = k_phase = kv_phase;
                advance();
                if (u + 2 < subs) {
                    k_slot = slot;
                    k_phase = kv_phase;
                    advance();
                }
                if (__builtin_expect(u >= 2 * scan, 0)) {
                    if (!wait(sm.kv_full[v_slot], v_phase)) return false;
                    if (elect_one()) mbar_arrive(smem_u32(&sm.scan));  // (while the exponentials of this tile are taken)
                    __syncwarp();
                    if (!wait(sm.scanned, scan_phase)) return false;
                    scan_phase ^= 1u;
                }
            }
            const int bit = 2 * h0 + (u & 1);
            // (keys only in the turn that takes them: in the other one their buffer may have been given back already)
            const bool v_in = mbar_try_wait(smem_u32(&sm.kv_full[v_slot]), v_phase), k_in = (u & 1) != 0 || mbar_try_wait(smem_u32(&sm.kv_full[k_slot]), k_phase);
            const bool p_in = mbar_try_wait(smem_u32(&sm.p_full[h0][u & 1]), p_phase >> bit & 1u);
            const bool p1_in = !WIDE || mbar_try_wait(smem_u32(&sm.p_full[1][u & 1]), p_phase >> (2 + (u & 1)) & 1u);
            if (__builtin_expect(!__all_sync(0xffffffffu, v_in && k_in && p_in && p1_in), 0) &&
                !(wait(sm.kv_full[v_slot], v_phase) && ((u & 1) != 0 || wait(sm.kv_full[k_slot], k_phase)) && wait(sm.p_full[h0][u & 1], p_phase >> bit & 1u) &&
                  (!WIDE || wait(sm.p_full[1][u & 1], p_phase >> (2 + (u & 1)) & 1u))))
                return false;
            p_phase ^= (WIDE ? 5u : 1u << (2 * h0)) << (u & 1);
            block<WIDE>(h0, u, subs, v_slot, k_slot);
        }
        return true;
    }
    __device__ __forceinline__ void run() {
        Pieces<D> pc(sm);
        for (;; pc.next()) {
            if (!pc.wait()) return;
            const int tiles = same(sm.piece[pc.at].tiles), subs = same(sm.piece[pc.at].subs), stage = same(sm.piece[pc.at].stage);
            const int scan = same(scan_from(sm.piece[pc.at]) - sm.piece[pc.at].tile0);
            __syncwarp();
            if (elect_one()) mbar_arrive(smem_u32(&sm.piece_empty[pc.at]));
            if (tiles < 0) return;
            if (tiles == 0) continue;
            if (!(stage == 2 ? piece<true>(subs, scan, 0) : piece<false>(subs, scan, stage))) return;
        }
    }
};

// ------------------------------------------------------------------------------------------------ the softmax, a row a thread
__device__ __forceinline__ float row_max(const float (&s)[kSub]) {
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = fmaxf(s[i], s[i + 4]);
#pragma unroll
    for (int i = 8; i < kSub; i += 8)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmax3(x[e], s[i + e], s[i + 4 + e]);
    return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
}

template <int D>
__device__ void softmax_rows(const AttendRowsArgs& a, RowsSmem<D>& sm, uint32_t tmem, int half) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5 & 3;
    const uint32_t mine = static_cast<uint32_t>(w * 32) << 16;         // this warp's lanes of tensor memory
    const uint32_t O = tmem + 2 * kTile + half * D + mine;
    Pieces<D> pc(sm);
    int n_tile = 0;
    uint32_t s_phase = 0, o_phase = 0;                                 // (of s_phase a bit for each S)
    auto wait = [&](int sub) { return wait_warp(smem_u32(&sm.s_full[half][sub]), s_phase >> sub & 1u, &sm.stop); };
    for (;; pc.next()) {
        if (!pc.wait()) return;
        const Piece& x = sm.piece[pc.at];
        const int tiles = x.tiles, subs = x.subs;
        if (tiles < 0) return;
        if (x.stage != 2 && x.stage != half) {
            n_tile += tiles;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.piece_empty[pc.at]));
            continue;
        }
        const int row0 = (x.stage == 2 ? half * kTile : 0) + w * 32, row = row0 + lane;
        const bool any = row0 < x.rows;                                // (of this warp)
        const int tok = row / x.heads, limit = x.limit + x.step * tok;
        const int least = x.limit + x.step * (row0 / x.heads);         // what the warp's first row sees: the least of its rows
        const int first = x.tile0 * kTile;
        // (lanes behind the last row have other tokens' queries, or what was left in shared memory: they have no say in whether references move, which would
        // change how the others' weights are rounded)
        const float slack = row < x.rows ? kSlack : INFINITY;
        float ref = -INFINITY, sum = 0.f;
#pragma unroll 1
        for (int u = 0; u < subs; ++u) {
            const int sub = u & 1, n = (n_tile + (u >> 1)) % kMasks;
            const uint32_t n_phase = (n_tile + (u >> 1)) / kMasks & 1;
            const bool m_in = mbar_try_wait(smem_u32(&sm.mask_full[n]), n_phase), s_in = mbar_try_wait(smem_u32(&sm.s_full[half][sub]), s_phase >> sub & 1u);
            if (__builtin_expect(!__all_sync(0xffffffffu, m_in && s_in), 0) && !(wait_warp(smem_u32(&sm.mask_full[n]), n_phase, &sm.stop) && wait(sub))) return;
            const uint2 m = *reinterpret_cast<const uint2*>(&sm.mask[n][2 * sub]);
            s_phase ^= 1u << sub;
            tc_fence_after();
            if (__builtin_expect(any, 1)) {
                const uint32_t S = tmem + half * kTile + sub * kSub + mine;
                float s[kSub];
                tmem_ld_x32(S, s);
                tmem_ld_x32(S + 32, s + 32);
                const int base = first + u * kSub;
                uint32_t seen[2] = {m.x, m.y};
                const bool part = (m.x & m.y) != 0xffffffffu || least < base + kSub;
                if (__builtin_expect(part, 0)) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int left = limit - base - 32 * i;        // rows of this word that are seen
                        seen[i] &= left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1u;
                    }
                }
                tmem_ld_wait();
                if (__builtin_expect(part, 0)) {
#pragma unroll
                    for (int i = 0; i < kSub; ++i) s[i] = seen[i / 32] >> (i & 31) & 1u ? s[i] : -INFINITY;
                }
                const float z = row_max(s) * a.scale_log2;
                if (__builtin_expect(__any_sync(0xffffffffu, z > ref + slack), 0)) {
                    const float now = fmaxf(ref, z), f = ex2_below(ref, now);
                    ref = now;
                    sum *= f;
                    if (u > 0) {
                        // (the other S is said to be there behind the last products that O took; the next wait for this P)
                        if (!wait(sub ^ 1)) return;
                        tc_fence_after();
#pragma unroll 1
                        for (int i = 0; i < D; i += 32) {
                            float o[32];
                            tmem_ld_x32(O + i, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] *= f;
                            tmem_st_x32(O + i, o);
                        }
                    }
                }
                // weights 2^(s scale - reference), their sum, and as bf16 into the place of the logits
                const float minus = ref == -INFINITY ? 0.f : -ref;
                const unsigned long long scale2 = pack2(a.scale_log2, a.scale_log2), minus2 = pack2(minus, minus);
                unsigned long long acc[2] = {0ull, 0ull};
                float p[kSub / 2];                                     // (pairs of bf16)
#pragma unroll
                for (int e = 0; e < kSub / 2; ++e) {
                    float v0, v1;
                    unpack2(fma2(pack2(s[2 * e], s[2 * e + 1]), scale2, minus2), v0, v1);
                    v0 = ex2_approx(v0);
                    v1 = ex2_approx(v1);
                    acc[e & 1] = add2(acc[e & 1], pack2(v0, v1));
                    p[e] = __uint_as_float(pack_bf16(v0, v1));
                }
                tmem_st_x32(S, p);
                float v0, v1;
                unpack2(add2(acc[0], acc[1]), v0, v1);
                sum += v0 + v1;
                tmem_st_wait();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.p_full[half][sub]));
        }
        n_tile += tiles;
        if (tiles > 0) {                                               // the last products have been added
            if (!wait_warp(smem_u32(&sm.o_full[half]), o_phase, &sm.stop)) return;
            o_phase ^= 1u;
            if (subs > 1) s_phase ^= 1u << (subs & 1);                 // (those before them long since; where no reference moved, nobody has waited for it)
        }
        tc_fence_after();
        if (any) {
            const bool there = row < x.rows;
            const int g = row - tok * x.heads;
            const int token = x.t0 + tok, q = x.h * a.G + x.g0 + g;
            const int slot = x.slot, leave = x.leave;
            const bool found = *reinterpret_cast<const volatile int*>(&x.found) != 0;
            const int* first_bad = a.first_bad + (static_cast<size_t>(blockIdx.x) * kPieces + pc.at) * D;
            const int bad_from = scan_from(x) * kTile;
            // rows of all units of a kind, and this one among them
            const size_t all = static_cast<size_t>(a.T) * a.Hq, whole = static_cast<size_t>(x.h) * a.T * a.G + static_cast<size_t>(token) * a.G + x.g0 + g;
            const float2 ml = make_float2(ref, tiles > 0 ? sum : kNoValues);
            if (there && leave == kPart) a.part_ml[static_cast<size_t>(slot) * a.record_rows + row] = ml;
            if (there && leave == kWhole) a.whole_ml[x.kind * all + whole] = ml;
            const float inv = 1.f / sum;
#pragma unroll 1
            for (int i = 0; i < D; i += 32) {
                float o[32];
                if (tiles > 0) {
                    tmem_ld_x32(O + i, o);
                    tmem_ld_wait();
                }
                if (found) {
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (*const_cast<const volatile int*>(first_bad + i + e) < limit - bad_from) o[e] = __int_as_float(0x7fffffff);
                }
                if (leave == kOut) {
                    if (there) {
                        uint32_t p[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) p[e] = sum == 0.f ? 0u : pack_bf16(o[2 * e] * inv, o[2 * e + 1] * inv);      // (nothing seen: zeros)
                        uint4* to = reinterpret_cast<uint4*>(a.out + (static_cast<size_t>(token) * a.Hq + q) * D + i);
#pragma unroll
                        for (int e = 0; e < 4; ++e) to[e] = make_uint4(p[4 * e], p[4 * e + 1], p[4 * e + 2], p[4 * e + 3]);
                    }
                } else if (there && tiles > 0) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float4 v = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                        if (leave == kPart) a.part_o[(static_cast<size_t>(slot) * (D / 4) + i / 4 + e) * a.record_rows + row] = v;
                        else a.whole_o[(static_cast<size_t>(x.kind) * (D / 4) + i / 4 + e) * all + whole] = v;
                    }
                }
            }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
            if (tiles > 0) mbar_arrive(smem_u32(&sm.o_empty[half]));
            mbar_arrive(smem_u32(&sm.piece_empty[pc.at]));
        }
    }
}

// ------------------------------------------------------------------------------------------------ pieces, and their queries and keys
// The length of the line, and the unit with this CTA's first tile. All threads.
template <int D>
__device__ int deal(const AttendRowsArgs& a, RowsSmem<D>& sm, int cta, int ctas) {
    const int per = (a.units + kRowsThreads - 1) / kRowsThreads;
    const int u0 = min(static_cast<int>(threadIdx.x) * per, a.units), u1 = min(u0 + per, a.units);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int total = 0, at = 0, inc = 0, begin = -1;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {                             // this thread's units added up; then, by one thread if any, looked through for the first
        int place = at;
#pragma unroll 1
        for (int u = u0; u < u1; ++u) {
            const int n = unit_of(a, u).span();
            if (pass == 1 && place <= begin && begin < place + n) {
                sm.first_unit = u;
                sm.first_at = place;
            }
            place += n;
        }
        if (pass == 1) break;
        inc = place;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, inc, off);
            if (lane >= off) inc += v;
        }
        if (lane == 31) sm.warp_sum[warp] = inc;
        __syncthreads();
        at = inc - place;
#pragma unroll 1
        for (int i = 0; i < kRowsThreads / 32; ++i) {
            if (i < warp) at += sm.warp_sum[i];
            total += sm.warp_sum[i];
        }
        inc = at + place;
        begin = Share(total, ctas).begin(cta);
        if (!(at <= begin && begin < inc)) break;
    }
    return total;
}

template <int D>
__device__ void hand_out(const AttendRowsArgs& a, const RowMaps& maps, RowsSmem<D>& sm, int total, int cta, int ctas) {
    const int lane = threadIdx.x & 31;
    KeyLoader<D> keys;
    const Share share(total, ctas);
    if (lane == 0) sm.stop.begin(share.per + 1, a.units);
    const int begin = share.begin(min(cta, share.n)), end = cta < share.n ? share.begin(cta + 1) : begin;
    int at = 0, narrow = 0;
    uint32_t phase = 1;                                                // (the first round's entries are free)
    auto publish = [&](bool fill, const Piece& x) {
        if (!wait_warp(smem_u32(&sm.piece_empty[at]), phase, &sm.stop)) return false;
        if (fill) sm.piece[at] = x;
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.piece_full[at]));
        if (++at == kPieces) { at = 0; phase ^= 1u; }
        return true;
    };
    if (!a.shared && lane == 0) a.begun[2 * cta + 1] = make_int4(0, 0, 0, -1);
    __syncwarp();
    if (begin < end) {
        int u = sm.first_unit, pos = sm.first_at;
#pragma unroll 1
        for (; u < a.units && pos < end; u += 32) {
            Unit x = {};
            int n = 0;
            if (u + lane < a.units) {
                x = unit_of(a, u + lane);
                n = x.span();
            }
            int inc = n;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, inc, off);
                if (lane >= off) inc += v;
            }
            const int start = pos + inc - n;
            const int p0 = max(begin - start, 0), p1 = min(end - start, n);
            uint32_t todo = __ballot_sync(0xffffffffu, n > 0 && p0 < p1);
            Piece y;
            y.tile0 = x.tiles_before(p0);
            y.tiles = x.tiles_before(p1) - y.tile0;
            y.subs = y.tiles > 0 ? (min(x.keys - y.tile0 * kTile, y.tiles * kTile) + kSub - 1) / kSub : 0;
            y.kind = x.kind; y.set = x.set; y.h = x.h; y.t0 = x.t0; y.g0 = x.g0; y.heads = x.heads; y.rows = x.rows();
            y.limit = x.limit; y.step = x.step; y.keys = x.keys;
            y.found = 0;
            const bool begins = p0 == 0, ends = p1 == n;
            y.leave = !(begins && ends) ? kPart : a.shared ? kWhole : kOut;
            y.slot = 2 * cta + (begins ? 1 : 0);
            const bool thin = x.tokens <= a.thin_tokens;
            if (p0 < p1 && begins) {
                const int last = share.owner(start + n - 1);
                if (a.shared) {
                    a.owners[u + lane] = make_int2(cta, last);
                } else if (!ends) {
                    a.begun[2 * cta] = make_int4(x.t0, x.h * a.G + x.g0, x.heads, y.rows);
                    a.begun[2 * cta + 1] = make_int4(0, 0, 0, last);
                }
            }
#pragma unroll 1
            while (todo != 0) {
                const int i = __ffs(todo) - 1;
                todo &= todo - 1;
                const bool one = __shfl_sync(0xffffffffu, thin, i);
                y.stage = one ? narrow : 2;
                if (one) narrow ^= 1;
                const Piece& z = sm.piece[at];
                if (!publish(lane == i, y) || (z.tiles > 0 && !keys.load(a, maps, sm, z))) {
                    keys.give_up(sm);
                    return;
                }
            }
            pos += __shfl_sync(0xffffffffu, inc, 31);
        }
    }
    Piece none = {};
    none.tiles = -1;
    if (!publish(lane == 0, none)) keys.give_up(sm);
}

template <int D>
__global__ void __launch_bounds__(kRowsThreads, 1) attend_rows_kernel(const __grid_constant__ RowMaps maps, const __grid_constant__ AttendRowsArgs a) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    RowsSmem<D>& sm = *reinterpret_cast<RowsSmem<D>*>(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5;
    if (warp == 0) tmem_alloc(smem_u32(&sm.tmem), 512);
    if (tid == 32) {
        for (int i = 0; i < RowsSmem<D>::kSlots; ++i) {
            mbar_init(smem_u32(&sm.kv_full[i]), 1);
            mbar_init(smem_u32(&sm.kv_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sm.q_full[i]), 1);
            mbar_init(smem_u32(&sm.q_empty[i]), 1);
            for (int j = 0; j < 2; ++j) {
                mbar_init(smem_u32(&sm.s_full[i][j]), 1);
                mbar_init(smem_u32(&sm.p_full[i][j]), 4);
            }
            mbar_init(smem_u32(&sm.o_full[i]), 1);
            mbar_init(smem_u32(&sm.o_empty[i]), 4);
        }
        for (int i = 0; i < kPieces; ++i) {
            mbar_init(smem_u32(&sm.piece_full[i]), 1);
            mbar_init(smem_u32(&sm.piece_empty[i]), kRowWarps + 3);    // and those that load values, multiply and look through
        }
        for (int i = 0; i < kMasks; ++i) mbar_init(smem_u32(&sm.mask_full[i]), 1);
        mbar_init(smem_u32(&sm.scan), 1);
        mbar_init(smem_u32(&sm.scanned), 1);
        mbar_init(smem_u32(&sm.drained), 1);
        sm.stop.abort = 0;
        sm.stop.limit = 1LL << 62;
        fence_mbar_init();
    }
    begin_dependent();
    const int total = deal(a, sm, blockIdx.x, gridDim.x);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem;
    // 384 threads of 168 registers, of which 256 take 200 and 128 take 96
    if (warp < kRowWarps) {
        setmaxnreg_inc<200>();
        softmax_rows<D>(a, sm, tmem, warp >> 2);
    } else {
        setmaxnreg_dec<96>();
        if (warp == kRowWarps) {
            hand_out(a, maps, sm, total, blockIdx.x, gridDim.x);
        } else if (warp == kRowWarps + 1) {
            Products<D>(sm, same(tmem)).run();
            if (elect_one()) {
                umma_commit(smem_u32(&sm.drained));                    // (nothing is under way in tensor memory when it is given back)
                int none = 0;
                mbar_wait(smem_u32(&sm.drained), 0, &none);
            }
            __syncwarp();
        } else if (warp == kRowWarps + 2) {
            load_values<D>(a, maps, sm);
        } else {
            scan_values<D>(a, sm);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) {
        tmem_relinquish();
        tmem_dealloc(tmem, 512);
    }
    if (tid == 0 && sm.stop.abort) atomicExch(&g_gave_up, 1);
}

// ------------------------------------------------------------------------------------------------ joining
// A CTA takes as many rows as leave four dims a thread, neighbouring rows in neighbouring lanes, as the records have them. The (reference, sum) of all records of a
// row are read side by side by a warp, which leaves a factor for each; then every thread adds up its dims, with as many loads under way as there are records.
constexpr int kJoinThreads = 256;
template <int D>
struct JoinSmem {
    static constexpr int kRows = kJoinThreads * 4 / D;
    int4 from[2][kRows];                               // first and last CTA (last < first: none), row of their records; 1: one CTA's that has the whole unit
    float factor[2][kRows][kRowsCtas];                 // below 0: a record that has no values
    float sum[kRows];
};

template <int D, bool SHARED>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ AttendRowsArgs a) {
    using Smem = JoinSmem<D>;
    constexpr int kRows = Smem::kRows, kSources = SHARED ? 2 : 1;
    __shared__ Smem sm;
    begin_dependent();
    const int tid = threadIdx.x, lane = tid & 31, rows = a.T * a.G;
    const int chunks = SHARED ? (rows + kRows - 1) / kRows : (a.record_rows + kRows - 1) / kRows;
    const int group = blockIdx.x / chunks, row0 = (blockIdx.x - group * chunks) * kRows;       // a KV head, or the CTA that began a unit
    int4 unit = make_int4(0, 0, 1, rows);              // first token, first head, heads, rows
    int last = 0;
    if constexpr (!SHARED) {
        last = a.begun[2 * group + 1].w;
        unit = a.begun[2 * group];
        if (last < 0 || row0 >= unit.w) return;        // (the whole CTA)
    }
    if (tid < kRows) {
        const int i = row0 + tid;
        int4 x[2] = {make_int4(0, -1, 0, 0), make_int4(0, -1, 0, 0)};
        if (i < unit.w) {
            if constexpr (SHARED) {
                const int b = i / a.G, g = i - b * a.G, hb = g / a.heads;
                auto put = [&](int kind, int u, int row) {
                    const int2 by = a.owners[u];
                    if (by.x >= 0 && by.y >= by.x && by.y < kRowsCtas) x[kind] = make_int4(by.x, by.y, row, by.x == by.y);     // (groups that are not ascending: no address out of range)
                };
                const RowSets &p = a.sets[0], &own = a.sets[1];
                int lo = 0, hi = p.n;                  // how many groups end at or before this sequence
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (p.starts[mid + 1] <= b) lo = mid + 1; else hi = mid;
                }
                if (lo < p.n && p.starts[lo] <= b && p.starts[lo] >= 0) {
                    const int k = b - p.starts[lo], blk = k / a.tokens;
                    put(0, group * p.slots + (base_of(a, p, lo) + blk) * a.head_blocks + hb, (k - blk * a.tokens) * min(a.heads, a.G - hb * a.heads) + g - hb * a.heads);
                }
                put(1, p.slots * a.Hkv + group * own.slots + b * a.head_blocks + hb, g - hb * a.heads);
            } else {
                x[0] = make_int4(group, last, i, 0);
            }
        }
        sm.from[0][tid] = x[0];
        sm.from[1][tid] = x[1];
    }
    __syncthreads();
    const size_t all = static_cast<size_t>(a.T) * a.Hq, head0 = static_cast<size_t>(group) * rows;      // (of the shared form's whole records)
    for (int r = tid >> 5; r < kRows; r += kJoinThreads / 32) {
        constexpr int kOwn = (kRowsCtas + 31) / 32;
        float2 ml[kSources][kOwn];
        float top = -INFINITY;
#pragma unroll
        for (int s = 0; s < kSources; ++s) {
            const int4 x = sm.from[s][r];
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const int c = x.x + lane + 32 * i;
                ml[s][i] = make_float2(-INFINITY, 0.f);
                if (c <= x.y) ml[s][i] = x.w ? a.whole_ml[s * all + head0 + row0 + r] : a.part_ml[static_cast<size_t>(2 * c + (c == x.x ? 1 : 0)) * a.record_rows + x.z];
                top = fmaxf(top, ml[s][i].x);
            }
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        float sum = 0.f;
#pragma unroll
        for (int s = 0; s < kSources; ++s) {
            const int4 x = sm.from[s][r];
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const float2 v = ml[s][i];
                const float f = v.y == kNoValues ? -1.f : ex2_below(v.x, top);
                if (x.x + lane + 32 * i <= x.y) sm.factor[s][r][lane + 32 * i] = f;
                if (f != -1.f) sum += v.y * f;
            }
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        if (lane == 0) sm.sum[r] = sum;
    }
    __syncthreads();
    const int r = tid % kRows, c4 = tid / kRows, i = row0 + r;
    if (i >= unit.w) return;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float f, const float4& y) {
        if (f >= 0.f || f != f) { v.x = fmaf(y.x, f, v.x); v.y = fmaf(y.y, f, v.y); v.z = fmaf(y.z, f, v.z); v.w = fmaf(y.w, f, v.w); }
    };
#pragma unroll
    for (int s = 0; s < kSources; ++s) {
        const int4 x = sm.from[s][r];
        if (SHARED && x.w) {
            add(sm.factor[s][r][0], a.whole_o[(static_cast<size_t>(s) * (D / 4) + c4) * all + head0 + i]);
            continue;
        }
        const float4* o = a.part_o + static_cast<size_t>(c4) * a.record_rows + x.z;
        const size_t slot = static_cast<size_t>(D / 4) * a.record_rows;
#pragma unroll 8
        for (int c = x.x; c <= x.y; ++c) add(sm.factor[s][r][c - x.x], o[(2 * c + (c == x.x ? 1 : 0)) * slot]);
    }
    const float sum = sm.sum[r], inv = 1.f / sum;
    const size_t row = SHARED ? static_cast<size_t>(i / a.G) * a.Hq + static_cast<size_t>(group) * a.G + i % a.G
                              : static_cast<size_t>(unit.x + i / unit.z) * a.Hq + unit.y + i % unit.z;
    *reinterpret_cast<uint2*>(a.out + row * D + 4 * c4) = sum == 0.f ? make_uint2(0u, 0u) : make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
}

size_t up256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }

template <int D>
cudaError_t launch(const AttendRowsArgs& a, const CUtensorMap* maps, int num_sms, cudaStream_t stream) {
    constexpr int smem = sizeof(RowsSmem<D>);
    cudaError_t e = cudaFuncSetAttribute(attend_rows_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    const int ctas = num_sms < kRowsCtas ? num_sms : kRowsCtas;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.stream = stream;
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kRowsThreads);
    cfg.dynamicSmemBytes = smem;
    e = cudaLaunchKernelEx(&cfg, attend_rows_kernel<D>, RowMaps{maps[0], maps[1], maps[2], maps[3]}, a);
    if (e != cudaSuccess) return e;
    cfg.blockDim = dim3(kJoinThreads);
    cfg.dynamicSmemBytes = 0;
    constexpr int rows = JoinSmem<D>::kRows;
    if (a.shared) {
        cfg.gridDim = dim3(static_cast<unsigned>((a.T * a.G + rows - 1) / rows) * a.Hkv);
        return cudaLaunchKernelEx(&cfg, join_kernel<D, true>, a);
    }
    cfg.gridDim = dim3(static_cast<unsigned>(ctas * ((a.record_rows + rows - 1) / rows)));
    return cudaLaunchKernelEx(&cfg, join_kernel<D, false>, a);
}

}  // namespace

AttendRowsPlan attend_rows_plan(int T, int n, int Hq, int Hkv, int d, bool shared) {
    AttendRowsPlan p = {};
    const int G = Hq / Hkv;
    p.head_blocks = (G + kBlock - 1) / kBlock;
    p.heads = (G + p.head_blocks - 1) / p.head_blocks;
    p.tokens = p.head_blocks > 1 ? 1 : kBlock / G;
    p.thin_tokens = kTile / p.heads;
    p.slots0 = n > 0 ? (static_cast<long long>(T) / p.tokens + n) * p.head_blocks : 0;
    p.slots1 = shared ? static_cast<long long>(T) * p.head_blocks : 0;
    p.units = (p.slots0 + p.slots1) * Hkv;
    const long long most = static_cast<long long>(T < p.tokens ? T : p.tokens) * p.heads;
    p.record_rows = static_cast<int>((most + 31) / 32 * 32);
    const size_t rows = static_cast<size_t>(2) * kRowsCtas * p.record_rows, all = shared ? static_cast<size_t>(2) * T * Hq : 0;
    p.off_o = up256(rows * sizeof(float2));
    p.off_begun = up256(p.off_o + rows * d * sizeof(float));
    p.off_bad = up256(p.off_begun + 2 * kRowsCtas * sizeof(int4));
    p.off_owners = up256(p.off_bad + static_cast<size_t>(kRowsCtas) * kPieces * d * sizeof(int));
    p.off_whole_ml = up256(p.off_owners + (shared ? static_cast<size_t>(p.units) * sizeof(int2) : 0));
    p.off_whole_o = up256(p.off_whole_ml + all * sizeof(float2));
    p.bytes = up256(p.off_whole_o + all * d * sizeof(float));
    return p;
}

cudaError_t launch_attend_rows(const AttendRowsArgs& args, const AttendRowsPlan& plan, const CUtensorMap* maps, int d, char* scratch, int num_sms, cudaStream_t stream) {
    AttendRowsArgs a = args;
    a.heads = plan.heads; a.head_blocks = plan.head_blocks; a.tokens = plan.tokens; a.thin_tokens = plan.thin_tokens;
    a.units = static_cast<int>(plan.units);
    a.record_rows = plan.record_rows;
    a.sets[0].slots = static_cast<int>(plan.slots0);
    a.sets[1].slots = static_cast<int>(plan.slots1);
    a.part_ml = reinterpret_cast<float2*>(scratch);
    a.part_o = reinterpret_cast<float4*>(scratch + plan.off_o);
    a.begun = reinterpret_cast<int4*>(scratch + plan.off_begun);
    a.first_bad = reinterpret_cast<int*>(scratch + plan.off_bad);
    a.owners = reinterpret_cast<int2*>(scratch + plan.off_owners);
    a.whole_ml = reinterpret_cast<float2*>(scratch + plan.off_whole_ml);
    a.whole_o = reinterpret_cast<float4*>(scratch + plan.off_whole_o);
    return d == 128 ? launch<128>(a, maps, num_sms, stream) : launch<64>(a, maps, num_sms, stream);
}

cudaError_t attend_rows_status(bool* gave_up) {
    int flag = 0;
    cudaError_t e = cudaMemcpyFromSymbol(&flag, g_gave_up, sizeof(int));
    *gave_up = flag != 0;
    if (e != cudaSuccess || flag == 0) return e;
    flag = 0;
    return cudaMemcpyToSymbol(g_gave_up, &flag, sizeof(int));
}
cudaError_t attend_rows_wait_clocks(long long clocks) {
    if (clocks <= 0) clocks = kWaitLimitClocks;
    return cudaMemcpyToSymbol(g_wait_clocks, &clocks, sizeof(clocks));
}

}  // namespace chunkkv
