// Attention of one new token over a paged cache: out = softmax(q K^T / sqrt(d)) V for every query head, over the rows that its KV head
// has (a length of its own), and, on request, the attention that every row received added to a running sum.
//
// What bounds it is the cache: every row is read once, 4 d bytes for 4 G d operations (G query heads of a KV head), so nothing else must be what
// the memory waits for. A warp works on one KV head, 16 rows a step, with a ring of steps of its own in shared memory that asynchronous
// copies fill (24 KB a warp; with 128 dims three steps, two of them in flight, 128 KB an SM, with 64 six and five, 160 KB) - no warp waits for another. The eight warps of a CTA take neighbouring
// heads of the same rows, which lie side by side in the cache, where there are as many; else several warps a head take rows in turn. The products run
// on the tensor cores with the rows, then the dims, as 16 rows of a product and the heads of a group as its eight columns: S^T = K Q^T and O^T += V^T P^T,
// so that half the products are not empty up to eight heads, a head's statistics and values lie in the same lanes, and V^T comes out of shared memory as it
// is needed. P is split into two bf16 terms, so that its rounding (2^-16) is not seen beside that of the output. A head's reference moves only when a
// logit lies 2^8 above it, which a vote finds without looking for the maximum. 64 sequences of 4160 rows, 8 heads of 128 dims: 166 us, the memory's own
// time. In a long cache an SM takes 46 GB/s of rows, its share of the memory; of pages that repeat, so that they come out of the L2, 90 GB/s (with 64 dims 40
// and 62), and the copies by themselves bring 150 to 180 on every SM at once: with 128 dims neither the L2 nor the steps are what is waited for.
//
// The rows of all units (a sequence's heads that a CTA takes together) are cut into tiles and dealt evenly to the CTAs in one line, so that lengths
// need not be alike; a CTA walks the units in its share and leaves (max, sum, O) records for those that it shares with others, which a second launch
// joins in the order of the CTAs (same result every time). The records live in scratch of the call's own: calls at the same time, and
// captured ones, have nothing in common.
#include "decode.cuh"

#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace chunkkv {

namespace {

constexpr int kAttWarps = 8;
constexpr int kAttThreads = 32 * kAttWarps;
constexpr int kAttStep = 16;                          // rows of a warp's step
constexpr int kRingBytes = 24 * 1024;                 // of a warp
constexpr int kJoinThreads = 128;
constexpr int kSmallRows = 1152;                      // rows of a CTA of the form for short caches, at most
constexpr int kSmallItems = 2048;                     // heads of a call that takes it, at most
constexpr int kJoinHeads = 8;                         // query heads whose weights are added together
static_assert(kAttMaxCtas % 32 == 0, "records are looked at a warp at a time");

__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Four 8 x 8 matrices of 16-bit values out of shared memory, as the first operand of a product or (TURNED) its transpose. Lanes 0 to 15 give the
// addresses of the rows of the first eight columns, the others those of the next eight.
template <bool TURNED>
__device__ __forceinline__ void load_matrices(uint32_t (&a)[4], uint32_t at) {
    if constexpr (TURNED)                             // (rows of the operand are columns there: the second and third change places)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(a[0]), "=r"(a[2]), "=r"(a[1]), "=r"(a[3]) : "r"(at) : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]) : "r"(at) : "memory");
}
// An 8 x 8 matrix of 16-bit values, a pair a lane, transposed.
__device__ __forceinline__ uint32_t turn_matrix(uint32_t v) {
    uint32_t o;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(o) : "r"(v));
    return o;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 16 bytes of global memory into shared memory, or zeros where `there` is false. ONCE: the first to leave the L2.
template <bool ONCE>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool there) {
    if constexpr (ONCE) {
        uint64_t policy;
        asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
        asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0), "l"(policy) : "memory");
    } else {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
    }
}
__device__ __forceinline__ void copies_begin_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// A maximum as the reference of exponents: 0 where nothing was seen.
__device__ __forceinline__ float reference_of(float m) { return m == -INFINITY ? 0.f : m; }
// A row's weight from its logit and its head's (reference, factor): nothing for a row that was not seen, whatever became of the head.
__device__ __forceinline__ float weight_of(float logit, const float2& f) { return logit == -INFINITY ? 0.f : exp2_fast(logit - f.x) * f.y; }

// Rows of a head and of a unit, the `block` heads from h0 on of a sequence.
__device__ __forceinline__ int rows_of(const AttendArgs& a, int bh) { return min(max(a.lengths[bh], 0), a.cache.cap); }
struct Unit {
    int b, h0, heads;     // sequence, its KV heads [h0, h0 + heads)
};
__device__ __forceinline__ Unit unit_of(const AttendArgs& a, int u) {
    const int b = u / a.blocks, h0 = (u - b * a.blocks) * a.block;
    return {b, h0, min(a.block, a.Hkv - h0)};
}
__device__ __forceinline__ int tiles_of(const AttendArgs& a, int u) {
    const Unit un = unit_of(a, u);
    const int32_t* len = a.lengths + un.b * a.Hkv + un.h0;
    int n[kAttWarps], most = 0;
#pragma unroll
    for (int h = 0; h < kAttWarps; ++h) n[h] = len[min(h, un.heads - 1)];       // (side by side: one after the other takes 0.3 us each)
#pragma unroll
    for (int h = 0; h < kAttWarps; ++h) most = max(most, n[h]);
    const int last = min(most, a.cache.cap) + a.tile - 1;
    return a.tile_shift >= 0 ? last >> a.tile_shift : last / a.tile;
}

// The line of tiles: the units in order, each `groups` times its tiles (one for each group of query heads), dealt to n CTAs in shares
// of `per`, the first `more` of them of one more. In front of a unit's tiles stand kBegin that hold no rows, for the time that a CTA takes to
// begin with another unit (table, queries, first rows: 2 to 3 us, as long as 2 to 4 tiles take). us without them, with 2, 3 and 4: 64 sequences of 8
// heads, 300 rows 21.1, 20.5, 20.3, 20.3; 24 of 1200 26.7, 25.5, 25.3, 25.3; of 2 heads, 64 dims, 64 of 2400 21.6, 20.9, 21.1, 21.2.
constexpr int kBegin = 3;
__device__ __forceinline__ int span_of(int tiles) { return tiles > 0 ? tiles + kBegin : 0; }
struct Share {
    int n, per, more;
    __device__ __forceinline__ Share(int total, int n_cta) {    // (no more CTAs than tiles, so that each has one at least)
        n = min(total, n_cta);
        per = n > 0 ? total / n : 0;
        more = total - per * n;
    }
    __device__ __forceinline__ int begin(int cta) const { return cta * per + min(cta, more); }
    __device__ __forceinline__ int owner(int x) const {         // the CTA that tile x falls to
        const int wide = more * (per + 1);
        return x < wide ? x / (per + 1) : more + (x - wide) / per;
    }
};
struct Deal {
    int total;            // the line's length
    int unit;             // the unit that holds the first tile of this CTA
    int first;            // its first tile
};
struct DealSmem {
    int warp[kAttWarps];
    int first, unit;
};

__device__ __forceinline__ Deal deal(const AttendArgs& a, int cta, int n_cta, DealSmem& sm) {
    const int units = a.B * a.blocks, per = (units + kAttThreads - 1) / kAttThreads;
    const int u0 = min(static_cast<int>(threadIdx.x) * per, units), u1 = min(u0 + per, units);
    int mine = 0;
    for (int u = u0; u < u1; ++u) mine += span_of(tiles_of(a, u));
    mine *= a.groups;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, inc, off);
        if (lane >= off) inc += v;
    }
    if (lane == 31) sm.warp[warp] = inc;
    if (threadIdx.x == 0) sm.unit = units;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < kAttWarps; ++w) {
        if (w < warp) inc += sm.warp[w];
        total += sm.warp[w];
    }
    const int tile = Share(total, n_cta).begin(cta);
    int at = inc - mine;
    if (at <= tile && tile < inc) {                             // one thread, if any
        int u = u0;
        for (; u + 1 < u1; ++u) {
            const int t = span_of(tiles_of(a, u)) * a.groups;
            if (tile < at + t) break;
            at += t;
        }
        sm.unit = u;
        sm.first = at;
    }
    __syncthreads();
    return {total, sm.unit, sm.first};
}

// Where records of CTA `cta` are: one for a unit that an earlier CTA has begun, one for a unit that it begins itself; each has a.block KV heads with
// a.group query heads.
__device__ __forceinline__ size_t record(const AttendArgs& a, int cta, bool begins, int h, int q) {
    return (static_cast<size_t>(cta * 2 + (begins ? 1 : 0)) * a.block + h) * a.group + q;
}

// A warp's walk over rows of one KV head, kAttStep at a time and `stride` rows from one step to the next, for up to 8 NH query heads.
// ONCE: keys and values are the first to leave the L2, so that records, logits and sums stay (sums of 16 x 8000 rows 99.6 -> 91.0 us, 8 x 4352 22.1 ->
// 20.9, 9 ragged sequences 43.4 -> 40.4); not for short caches, which stay there themselves (4 x 2000 rows 9.7, 10.4 with it).
template <int D, int NH, bool ONCE>
struct Walk {
    static constexpr int kPieces = D / 8;               // 16-byte pieces of a row
    static constexpr int kRowsOnce = 32 / kPieces;      // rows that one copy instruction of a warp takes
    static constexpr int kCopies = kAttStep / kRowsOnce;
    static constexpr int kHalf = kAttStep * D * 2;      // bytes of a step's keys
    static constexpr int kStages = kRingBytes / (2 * kHalf);
    static constexpr float kSlack = 8.f;                // how far logits may lie above the reference before it moves (in powers of two)

    const PagedCache cache;
    const float scale_log2;
    const uint32_t row_bytes;                           // from a row of the cache to the next
    const uint32_t ring;                                // kRingBytes of shared memory
    const int32_t* table;
    const char *Kh, *Vh;                                // the head's part of the cache's first row, at this lane's piece
    int base, end, stride, heads;                       // rows base, base + 1, ... of a step, up to `end`
    int at[kStages];                                    // rows of the cache of the steps ahead: lane l (and l + 16) row l of a step, -1: none
    uint32_t put[4];                                    // where a lane's piece goes in every fourth copy of a step
    uint32_t get[4];                                    // where a lane's row of 16 x 16 values is, in every fourth
    uint32_t qr[NH][D / 16][2];
    float m[NH][2], l[NH][2], o[NH][D / 16][4];         // of the query heads 8 n + 2 t + e: reference, this lane's part of the sum; O^T

    __device__ __forceinline__ Walk(const AttendArgs& a, const unsigned char* slots)
        : cache(a.cache), scale_log2(a.scale_log2), row_bytes(static_cast<uint32_t>(a.Hkv) * (D * 2)),
          ring(static_cast<uint32_t>(__cvta_generic_to_shared(slots))) {
        // Pieces of row r are exchanged by r mod 8 within 128 bytes, so that neither a copy's quarter nor the eight rows of a matrix meet in a bank.
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (i * kRowsOnce + lane / kPieces) % 8, row = (lane & 7) + (lane & 8);
            put[i] = (lane / kPieces) * (2 * D) + (((lane % kPieces) ^ r) << 4);
            get[i] = row * (2 * D) + (((2 * i + (lane >> 4)) ^ (row & 7)) << 4);
        }
    }

    __device__ __forceinline__ int lookup(int from) const {
        const int r = from + (threadIdx.x & 15);
        return r < end ? paged_row(cache, table, r) : -1;
    }
    __device__ __forceinline__ void copy_step(int rows, uint32_t to) const {
        const int lane = threadIdx.x & 31;
        const bool all = __all_sync(0xffffffffu, rows >= 0);
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int row = __shfl_sync(0xffffffffu, rows, i * kRowsOnce + lane / kPieces);
            const uint32_t dst = to + put[i % 4] + i * kRowsOnce * (2 * D);
            const uint64_t off = static_cast<uint64_t>(static_cast<uint32_t>(all ? row : max(row, 0))) * row_bytes;
            copy_async<ONCE>(dst, Kh + off, all || row >= 0);
            copy_async<ONCE>(dst + kHalf, Vh + off, all || row >= 0);
        }
    }
    // Asks for the first steps. b: sequence, h: KV head, q_row: first of the query heads among all. A group of copies a step, empty ones behind `end`.
    __device__ __forceinline__ void begin(const AttendArgs& a, int b, int h, size_t q_row, int heads_, int base_, int end_, int stride_) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        table = cache.tables + static_cast<size_t>(b) * cache.max_pages;
        const size_t off = static_cast<size_t>(h) * D + 8 * (lane % kPieces);
        Kh = reinterpret_cast<const char*>(a.K + off);
        Vh = reinterpret_cast<const char*>(a.V + off);
        base = base_; end = end_; stride = stride_; heads = heads_;
#pragma unroll
        for (int i = 0; i < kStages; ++i) at[i] = lookup(base + i * stride);
        const __nv_bfloat16* q = a.q + q_row * D + 2 * t;
#pragma unroll
        for (int n = 0; n < NH; ++n)
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    qr[n][i][e] = base < end && 8 * n + g < heads ? *reinterpret_cast<const uint32_t*>(q + static_cast<size_t>(8 * n + g) * D + 16 * i + 8 * e) : 0u;
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) {
            if (base + i * stride < end) copy_step(at[i], ring + i * 2 * kHalf);
            copies_begin_group();
        }
    }
    // keep(n, base, v): the logits v[j][e] of query head 8 n + 2 t + e and row base + 8 j + g (in powers of two; -inf: not seen).
    template <class Keep>
    __device__ __forceinline__ void run(Keep keep) {
        constexpr unsigned kFull = 0xffffffffu;
        const int lane = threadIdx.x & 31, g = lane >> 2;
#pragma unroll
        for (int n = 0; n < NH; ++n) {
            m[n][0] = m[n][1] = -INFINITY;
            l[n][0] = l[n][1] = 0.f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
        }
        int stage = 0;
        for (; base < end; base += stride) {
            copies_wait<kStages - 2>();
            __syncwarp();                                       // (this step has landed, and the one before has been read)
            const int ahead = base + (kStages - 1) * stride;
            if (ahead < end) copy_step(at[kStages - 1], ring + (stage == 0 ? kStages - 1 : stage - 1) * 2 * kHalf);
            copies_begin_group();
            const uint32_t keys = ring + stage * 2 * kHalf, values = keys + kHalf;
            stage = stage == kStages - 1 ? 0 : stage + 1;
            // S^T = K Q^T: rows of the product are the rows g and g + 8 of the step, columns the query heads 2t and 2t + 1
            float s[NH][2][4];
#pragma unroll
            for (int n = 0; n < NH; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[n][0][i] = s[n][1][i] = 0.f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                uint32_t k[4];
                load_matrices<false>(k, keys + get[i % 4] + (i / 4) * 128);
#pragma unroll
                for (int n = 0; n < NH; ++n) mma_bf16(s[n][i & 1], k, qr[n][i][0], qr[n][i][1]);
            }
            uint32_t v[D / 16][4];                              // V^T: rows are dims
#pragma unroll
            for (int i = 0; i < D / 16; ++i) load_matrices<true>(v[i], values + get[i % 4] + (i / 4) * 128);
            const unsigned seen = __ballot_sync(kFull, at[0] >= 0) >> g;       // bits 0 and 8: rows g and g + 8
#pragma unroll
            for (int i = 0; i < kStages - 1; ++i) at[i] = at[i + 1];
            at[kStages - 1] = lookup(ahead + stride);

            float z[NH][2][2];
            bool above = false;
#pragma unroll
            for (int n = 0; n < NH; ++n) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        z[n][j][e] = seen >> (8 * j) & 1u ? (s[n][0][2 * j + e] + s[n][1][2 * j + e]) * scale_log2 : -INFINITY;
                        above |= z[n][j][e] > m[n][e] + kSlack;
                    }
                keep(n, base, z[n]);
            }
            if (__any_sync(kFull, above)) {                     // a new reference: the first step's, and few after it
#pragma unroll
                for (int n = 0; n < NH; ++n) {
                    float factor[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = fmaxf(z[n][0][e], z[n][1][e]);
#pragma unroll
                        for (int off = 4; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, off));
                        const float now = fmaxf(m[n][e], mx);
                        factor[e] = exp2_fast(m[n][e] - reference_of(now));
                        m[n][e] = now;
                        l[n][e] *= factor[e];
                    }
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) { o[n][i][0] *= factor[0]; o[n][i][1] *= factor[1]; o[n][i][2] *= factor[0]; o[n][i][3] *= factor[1]; }
                }
            }
#pragma unroll
            for (int n = 0; n < NH; ++n) {
                const float ref0 = reference_of(m[n][0]), ref1 = reference_of(m[n][1]);
                uint32_t hi[2], lo[2];                          // P, turned from (rows, heads) to the product's second operand
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float p0 = exp2_fast(z[n][j][0] - ref0), p1 = exp2_fast(z[n][j][1] - ref1);
                    l[n][0] += p0;
                    l[n][1] += p1;
                    const uint32_t w = pack_bf16(p0, p1);
                    const float2 r = bf16_pair(w);
                    hi[j] = turn_matrix(w);
                    lo[j] = turn_matrix(pack_bf16(p0 - r.x, p1 - r.y));
                }
                // O^T += V^T P^T: rows of the product are the dims 16 i + g and 16 i + 8 + g, columns the query heads 2t and 2t + 1
#pragma unroll
                for (int i = 0; i < D / 16; ++i) mma_bf16(o[n][i], v[i], hi[0], hi[1]);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) mma_bf16(o[n][i], v[i], lo[0], lo[1]);
            }
        }
        __syncwarp();                                           // (the last step has been read)
    }
    // Another warp's walk over the same head (its values as left by leave) joined to this one.
    template <class From>
    __device__ __forceinline__ void join(const From& other) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int n = 0; n < NH; ++n) {
            const float4 s = other.ml[n][lane];
            const float its_m[2] = {s.x, s.y}, its_l[2] = {s.z, s.w};
            float own[2], its[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float now = fmaxf(m[n][e], its_m[e]), ref = reference_of(now);
                own[e] = exp2_fast(m[n][e] - ref);
                its[e] = exp2_fast(its_m[e] - ref);
                m[n][e] = now;
                l[n][e] = l[n][e] * own[e] + its_l[e] * its[e];
            }
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const float4 x = other.o[n * (D / 16) + i][lane];
                o[n][i][0] = o[n][i][0] * own[0] + x.x * its[0];
                o[n][i][1] = o[n][i][1] * own[1] + x.y * its[1];
                o[n][i][2] = o[n][i][2] * own[0] + x.z * its[0];
                o[n][i][3] = o[n][i][3] * own[1] + x.w * its[1];
            }
        }
    }
    template <class To>
    __device__ __forceinline__ void leave(To& to) const {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int n = 0; n < NH; ++n) {
            to.ml[n][lane] = make_float4(m[n][0], m[n][1], l[n][0], l[n][1]);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) to.o[n * (D / 16) + i][lane] = make_float4(o[n][i][0], o[n][i][1], o[n][i][2], o[n][i][3]);
        }
    }
    // The sums of the query heads from the eight lanes that hold their rows.
    __device__ __forceinline__ void add_up() {
#pragma unroll
        for (int n = 0; n < NH; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], off);
    }
    // Two neighbouring values of query head 8 n + 2 t + e, the dims dim_of(i) and the next (every lane calls this: neighbours exchange one).
    __device__ __forceinline__ int dim_of(int i) const {
        const int g = (threadIdx.x & 31) >> 2;
        return 16 * i + ((g & 1) ? 7 + g : g);
    }
    __device__ __forceinline__ float2 values(int n, int e, int i) const {
        const bool odd = (threadIdx.x & 4) != 0;
        const float x = o[n][i][e], y = o[n][i][e + 2], got = __shfl_xor_sync(0xffffffffu, odd ? x : y, 4);
        return odd ? make_float2(got, y) : make_float2(x, got);
    }
};

// What a warp leaves for the one that joins its head's warps: every lane's (max, sum) and O.
template <int D, int NH>
struct Left {
    float4 o[NH * D / 16][32];
    float4 ml[NH][32];
};
template <int D, int NH>
struct AttSmem {
    // apart from the rings where there is room (a warp's ring can then be filled for the next part while others join), else in the rings' place
    static constexpr bool kApart = kAttWarps * kRingBytes + (kAttWarps - 1) * sizeof(Left<D, NH>) + 1024 <= 227 * 1024;
    alignas(128) unsigned char ring[kAttWarps][kRingBytes];
    alignas(16) unsigned char left_[kApart ? (kAttWarps - 1) * sizeof(Left<D, NH>) : 16];
    DealSmem deal;
    __device__ __forceinline__ Left<D, NH>& left(int warp, int block) {     // of a warp that is not the first of its head
        if constexpr (kApart) return reinterpret_cast<Left<D, NH>*>(left_)[warp - block];
        else return *reinterpret_cast<Left<D, NH>*>(ring[warp]);
    }
};

// D: head dim; NH: query heads of a group in eights.
template <int D, int NH, bool SUMS>
__global__ void __launch_bounds__(kAttThreads, 1) attend_kernel(const AttendArgs a) {
    extern __shared__ __align__(128) char smem_raw[];
    AttSmem<D, NH>& sm = *reinterpret_cast<AttSmem<D, NH>*>(smem_raw);
    begin_dependent();
    const int cta = blockIdx.x, units = a.B * a.blocks;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const Deal dl = deal(a, cta, gridDim.x, sm.deal);
    const Share share(dl.total, gridDim.x);
    if (cta >= share.n || dl.unit >= units) return;
    const int x1 = share.begin(cta + 1);
    // this warp's head in a unit and its rows among those of the head's warps
    const int head = warp % a.block, turn = warp / a.block, turns = a.tile / kAttStep;
    const int G = a.Hq / a.Hkv;
    Walk<D, NH, true> walk(a, sm.ring[warp]);

    // A part of this CTA's share: tiles [tile0, tile1) of a unit, for one group of query heads.
    struct Part {
        Unit un;
        int unit, tiles, first, grp, tile0, tile1;     // (none, where tile1 <= tile0)
        int rows_end;                // of this warp's head, within the part
        __device__ __forceinline__ bool begins() const { return tile0 == 0; }
        __device__ __forceinline__ bool whole() const { return tile0 == 0 && tile1 == tiles; }
    };
    auto part_at = [&](int x, int unit, int first) {            // first: the unit's first tile (of its first group)
        Part p;
        p.unit = unit;
        p.first = first;
        p.un = unit_of(a, unit);
        p.tiles = tiles_of(a, unit);
        p.grp = a.groups == 1 ? 0 : (x - first) / span_of(p.tiles);
        const int begin = first + p.grp * span_of(p.tiles) + kBegin;
        p.tile0 = max(x - begin, 0);
        p.tile1 = min(x1 - begin, p.tiles);
        const bool on = head < p.un.heads && turn < turns;      // (else this warp has no head here)
        p.rows_end = on ? min(rows_of(a, p.un.b * a.Hkv + p.un.h0 + head), p.tile1 * a.tile) : 0;
        return p;
    };
    auto row_of_q = [&](const Part& p) { return static_cast<size_t>(p.un.b) * a.Hq + static_cast<size_t>(p.un.h0 + head) * G + p.grp * 8 * NH; };
    auto begin_part = [&](const Part& p) {
        walk.begin(a, p.un.b, p.un.h0 + head, row_of_q(p), min(8 * NH, G - p.grp * 8 * NH), p.tile0 * a.tile + turn * kAttStep, p.rows_end, a.tile);
    };

    Part p = part_at(share.begin(cta), dl.unit, dl.first);
    if (p.tile1 <= p.tile0) return;
    begin_part(p);
    for (;;) {
        const int heads = walk.heads;                           // query heads of this group
        const size_t q_row = row_of_q(p);
        const int r1 = p.rows_end;
        walk.run([&](int n, int base, const float (&z)[2][2]) {
            if constexpr (SUMS) {
                float* lg = a.logits + (q_row + 8 * n + 2 * t) * a.logit_stride + base + g;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (8 * n + 2 * t + e < heads && base + 8 * j + g < r1) lg[e * a.logit_stride + 8 * j] = z[j][e];
            }
        });

        // the part behind this one, if any: where no other warp's values are joined in the rings' place its first rows are asked for at once
        const int x = p.first + p.grp * span_of(p.tiles) + kBegin + p.tile1;
        Part next = p;
        bool more = x < x1;
        if (more) {
            int unit = p.unit, first = p.first;
            if (p.grp + 1 == a.groups) {                        // on to the next unit that has rows
                first = x;
                do ++unit; while (unit < units && tiles_of(a, unit) == 0);
            }
            more = unit < units;
            if (more) next = part_at(x, unit, first);
            more = more && next.tile0 < next.tile1;
        }
        constexpr bool kApart = AttSmem<D, NH>::kApart;
        if (more && (kApart || turns == 1)) begin_part(next);

        if (turns > 1) {                                        // the warps of a head, joined by its first one in their order
            __syncthreads();                                    // (what was left before has been read)
            if (turn > 0 && turn < turns) walk.leave(sm.left(warp, a.block));
            __syncthreads();
            if (turn == 0)
                for (int w = 1; w < turns; ++w) walk.join(sm.left(warp + w * a.block, a.block));
            if (!kApart) {
                __syncthreads();
                if (more) begin_part(next);
            }
        }
        walk.add_up();
        if (p.begins() && threadIdx.x == 0)
            a.shared_by[static_cast<size_t>(p.unit) * a.groups + p.grp] = make_int2(cta, share.owner(p.first + (p.grp + 1) * span_of(p.tiles) - 1));
        const bool whole = p.whole();
        if (turn == 0 && head < p.un.heads) {
#pragma unroll
            for (int n = 0; n < NH; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int q = 8 * n + 2 * t + e;
                    const bool mine = q < heads;
                    const size_t rec = record(a, cta, p.begins(), head, mine ? q : 0);
                    if (mine && g == 0) {
                        const float2 s = make_float2(walk.m[n][e], walk.l[n][e]);
                        if (!whole) a.part_ml[rec] = s;
                        else if (SUMS) a.whole_ml[q_row + q] = s;           // (a CTA can have many)
                    }
                    const float ll = walk.l[n][e], r = ll == 0.f ? 0.f : 1.f / ll;     // (nothing seen: zeros)
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        const float2 x = walk.values(n, e, i);
                        if (!mine) continue;
                        if (whole) *reinterpret_cast<uint32_t*>(a.out + (q_row + q) * D + walk.dim_of(i)) = pack_bf16(x.x * r, x.y * r);
                        else *reinterpret_cast<float2*>(a.part_o + rec * D + walk.dim_of(i)) = x;
                    }
                }
        }
        if (!more) return;
        p = next;
    }
}

// The join. A query head's records are joined by a team: a warp where few CTAs share a unit, else a CTA, or, of many CTAs, one for every 32 dims.
// The other CTAs add the rows' weights to the sums, kJoinThreads RPT rows of a KV head each.
enum TeamOf { kTeamWarp, kTeamCta, kTeamCtas };
template <int D, TeamOf TEAM>
struct Team {
    static constexpr bool kCta = TEAM != kTeamWarp;
    static constexpr int kThreads = kCta ? kJoinThreads : 32;
    static constexpr int kDims = TEAM == kTeamCtas ? 32 : D;    // of a team
    static constexpr int kParts = kThreads / (kDims / 4);       // groups of threads that take records in turn, 16 bytes of values a thread
    static constexpr int kTeams = kJoinThreads / kThreads;      // in a CTA
    static constexpr int kAhead = TEAM == kTeamCtas ? 10 : (TEAM == kTeamCta ? 8 : 4);     // values asked for before the factors that they wait for
};
template <int D, TeamOf TEAM>
struct JoinSmem {
    alignas(16) float o[kJoinThreads][4];
    float factor[Team<D, TEAM>::kTeams][kAttMaxCtas];
    float top[kJoinThreads / 32], sum[kJoinThreads / 32];
    float2 ml[kJoinHeads];            // (reference, factor) of query heads
};

// RPT: rows of the sums a thread takes; 0: no sums.
template <int D, int NH, int RPT, TeamOf TEAM>
__global__ void __launch_bounds__(kJoinThreads) attend_join_kernel(const AttendArgs a, int join_ctas, int row_blocks) {
    using T = Team<D, TEAM>;
    constexpr unsigned kFull = 0xffffffffu;
    __shared__ JoinSmem<D, TEAM> sm;
    const int G = a.Hq / a.Hkv, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto meet = [] { if constexpr (T::kCta) __syncthreads(); else __syncwarp(); };
    // (the kernel ahead sets this one up after its own wait: lengths, which were there before it, may be read)
    if (static_cast<int>(blockIdx.x) < join_ctas) {
        const int team = threadIdx.x / T::kThreads, id = threadIdx.x % T::kThreads;
        const int item = blockIdx.x * T::kTeams + team, cols = item % (D / T::kDims) * T::kDims, row = item / (D / T::kDims);   // row of q and out
        const bool there = row < a.B * a.Hq;
        const int b = row / a.Hq, hq = row - b * a.Hq, h = hq / G, q = hq - h * G, grp = q / (8 * NH), qg = q - grp * 8 * NH;
        const int blk = h / a.block, unit = b * a.blocks + blk, head = h - blk * a.block;
        const int tiles = there ? tiles_of(a, unit) : 0;
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (!there) return;                                     // (a whole team)
        const int part = id / (T::kDims / 4), c4 = cols + id % (T::kDims / 4) * 4;
        __nv_bfloat16* out = a.out + static_cast<size_t>(row) * D + c4;
        if (tiles == 0) {                                       // no rows: zeros
            if (part == 0) *reinterpret_cast<uint2*>(out) = make_uint2(0u, 0u);
            return;
        }
        const int2 by = a.shared_by[static_cast<size_t>(unit) * a.groups + grp];
        const int n_rec = by.y - by.x + 1;
        if (n_rec == 1) return;                                 // one CTA had the whole unit and wrote it
        auto record_of = [&](int r) { return record(a, by.x + r, r == 0, head, qg); };
        auto values = [&](int r) { return *reinterpret_cast<const float4*>(a.part_o + record_of(r) * D + c4); };
        float4 y[T::kAhead];
#pragma unroll
        for (int i = 0; i < T::kAhead; ++i) {
            const int r = part + i * T::kParts;
            y[i] = r < n_rec ? values(r) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        constexpr int kOwn = (kAttMaxCtas + T::kThreads - 1) / T::kThreads;
        float2 s[kOwn];
        float mm = -INFINITY;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int r = id + i * T::kThreads;
            s[i] = r < n_rec ? a.part_ml[record_of(r)] : make_float2(-INFINITY, 0.f);
            mm = fmaxf(mm, s[i].x);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) mm = fmaxf(mm, __shfl_xor_sync(kFull, mm, off));
        if constexpr (T::kCta) {
            if (lane == 0) sm.top[warp] = mm;
            __syncthreads();
            mm = fmaxf(fmaxf(sm.top[0], sm.top[1]), fmaxf(sm.top[2], sm.top[3]));
        }
        const float ref = reference_of(mm);
        float ll = 0.f;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int r = id + i * T::kThreads;
            const float f = exp2_fast(s[i].x - ref);
            if (r < n_rec) { sm.factor[team][r] = f; ll += s[i].y * f; }
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) ll += __shfl_xor_sync(kFull, ll, off);
        if constexpr (T::kCta) {
            if (lane == 0) sm.sum[warp] = ll;
        }
        meet();
        if constexpr (T::kCta) ll = (sm.sum[0] + sm.sum[1]) + (sm.sum[2] + sm.sum[3]);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        auto add = [&](const float4& z, float f) { v.x = fmaf(z.x, f, v.x); v.y = fmaf(z.y, f, v.y); v.z = fmaf(z.z, f, v.z); v.w = fmaf(z.w, f, v.w); };
#pragma unroll
        for (int i = 0; i < T::kAhead; ++i)
            if (part + i * T::kParts < n_rec) add(y[i], sm.factor[team][part + i * T::kParts]);
#pragma unroll 4
        for (int r = part + T::kAhead * T::kParts; r < n_rec; r += T::kParts) add(values(r), sm.factor[team][r]);
        if constexpr (T::kParts > 1) {                          // the parts, in their order
            *reinterpret_cast<float4*>(sm.o[threadIdx.x]) = v;
            meet();
            if (part == 0) {
                v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int i = 0; i < T::kParts; ++i) add(*reinterpret_cast<const float4*>(sm.o[threadIdx.x + i * (T::kDims / 4)]), 1.f);
            }
        }
        if (part == 0) {
            const float r = ll == 0.f ? 0.f : 1.f / ll;         // (nothing seen: zeros)
            *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(v.x * r, v.y * r), pack_bf16(v.z * r, v.w * r));
        }
        return;
    }
    if constexpr (RPT > 0) {
        constexpr int kJoinRows = RPT * kJoinThreads;
        const int idx = blockIdx.x - join_ctas, bh = idx / row_blocks, b = bh / a.Hkv, h = bh - b * a.Hkv;
        const int blk = h / a.block, unit = b * a.blocks + blk, head = h - blk * a.block;
        const int r0 = (idx - bh * row_blocks) * kJoinRows, r1 = min(rows_of(a, bh), r0 + kJoinRows);
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (r0 >= r1) return;
        const size_t q_row = static_cast<size_t>(b) * a.Hq + static_cast<size_t>(h) * G;
        float* w = a.weights + static_cast<size_t>(bh) * a.cache.cap;
        float acc[RPT], was[RPT];
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int r = r0 + i * kJoinThreads + threadIdx.x;
            acc[i] = 0.f;
            was[i] = r < r1 ? w[r] : 0.f;
        }
        for (int q0 = 0; q0 < G; q0 += kJoinHeads) {
            float lg[kJoinHeads][RPT];                     // (asked for before the statistics that they wait for)
#pragma unroll
            for (int q = 0; q < kJoinHeads; ++q)
#pragma unroll
                for (int i = 0; i < RPT; ++i) {
                    const int r = r0 + i * kJoinThreads + threadIdx.x;
                    lg[q][i] = q0 + q < G && r < r1 ? a.logits[(q_row + q0 + q) * a.logit_stride + r] : -INFINITY;
                }
            __syncthreads();
#pragma unroll
            for (int qw = 0; qw < kJoinHeads; qw += kJoinThreads / 32) {
                const int q = q0 + qw + warp;
                float2 f = make_float2(0.f, 0.f);
                if (q < G) {
                    const int grp = q / (8 * NH), qg = q - grp * 8 * NH;
                    const int2 by = a.shared_by[static_cast<size_t>(unit) * a.groups + grp];
                    constexpr int kOwn = kAttMaxCtas / 32;
                    float2 s[kOwn];
                    float mm = -INFINITY;
#pragma unroll
                    for (int i = 0; i < kOwn; ++i) {
                        const int c = by.x + lane + 32 * i;
                        s[i] = c > by.y ? make_float2(-INFINITY, 0.f) : by.x == by.y ? a.whole_ml[q_row + q] : a.part_ml[record(a, c, c == by.x, head, qg)];
                        mm = fmaxf(mm, s[i].x);
                    }
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) mm = fmaxf(mm, __shfl_xor_sync(kFull, mm, off));
                    const float ref = reference_of(mm);
                    float ll = 0.f;
#pragma unroll
                    for (int i = 0; i < kOwn; ++i) ll += by.x + lane + 32 * i <= by.y ? s[i].y * exp2_fast(s[i].x - ref) : 0.f;
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) ll += __shfl_xor_sync(kFull, ll, off);
                    f = make_float2(ref, ll == 0.f ? 0.f : 1.f / ll);
                }
                if (lane == 0) sm.ml[qw + warp] = f;
            }
            __syncthreads();
#pragma unroll
            for (int q = 0; q < kJoinHeads; ++q) {
                const float2 f = sm.ml[q];
                if (q0 + q < G) {
#pragma unroll
                    for (int i = 0; i < RPT; ++i) acc[i] += weight_of(lg[q][i], f);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int r = r0 + i * kJoinThreads + threadIdx.x;
            if (r < r1) w[r] = was[i] + acc[i];
        }
    }
}

// The form for short caches: a cluster of CTAs works on one (sequence, KV head, group of query heads), each CTA on an even share of its rows, and the
// parts are joined through distributed shared memory: one launch and no scratch. Logits that the sums need stay in shared memory. W: warps of a CTA,
// eight, one CTA an SM, or (more heads than SMs, a CTA each) four, two an SM, so that one's first loads travel while the other works.
template <int D, int NH, int W>
struct SmallSmem {
    union {
        alignas(128) unsigned char ring[W][kRingBytes];
        float4 o[W][NH * D / 16][33];                 // the warps' parts as their lanes hold them (the rings are idle then)
    };
    alignas(16) float2 warp_ml[W][8 * NH];
    alignas(16) float cta_o[8 * NH][D];               // this CTA's part, which the others read
    float2 cta_ml[8 * NH];
    float2 all[8 * NH];                               // (reference, factor) of the query heads
    // float logits[a.group][a.small_rows] behind it
};

template <int D, int NH, bool SUMS, int W>
__global__ void __launch_bounds__(32 * W, 8 / W) attend_small_kernel(const AttendArgs a) {
    constexpr int kSmallWarps = W, kSmallThreads = 32 * W;
    extern __shared__ __align__(128) char smem_raw[];
    SmallSmem<D, NH, W>& sm = *reinterpret_cast<SmallSmem<D, NH, W>*>(smem_raw);
    float* logits = reinterpret_cast<float*>(smem_raw + sizeof(SmallSmem<D, NH, W>));
    begin_dependent();
    cg::cluster_group cluster = cg::this_cluster();
    const int n_cta = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int item = blockIdx.x / n_cta, bh = item / a.groups, grp = item - bh * a.groups, b = bh / a.Hkv, h = bh - b * a.Hkv;
    const int G = a.Hq / a.Hkv, heads = min(8 * NH, G - grp * 8 * NH);
    const size_t q_row = static_cast<size_t>(b) * a.Hq + static_cast<size_t>(h) * G + grp * 8 * NH;
    const int n = rows_of(a, bh), steps = (n + kAttStep - 1) / kAttStep;
    const int r0 = rank * steps / n_cta * kAttStep, r1 = min((rank + 1) * steps / n_cta * kAttStep, n);
    Walk<D, NH, false> walk(a, sm.ring[warp]);
    walk.begin(a, b, h, q_row, heads, r0 + warp * kAttStep, r1, kSmallWarps * kAttStep);
    walk.run([&](int nn, int base, const float (&z)[2][2]) {
        if constexpr (SUMS) {
            float* lg = logits + (8 * nn + 2 * t) * a.small_rows + (base - r0) + g;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (8 * nn + 2 * t + e < heads) lg[e * a.small_rows + 8 * j] = z[j][e];
        }
    });
    constexpr int kOwnRows = SUMS ? (kSmallRows + kSmallThreads - 1) / kSmallThreads : 1;
    float* sums = SUMS ? a.weights + static_cast<size_t>(bh) * a.cache.cap : nullptr;
    float was[kOwnRows];                              // (asked for before the joining)
    if constexpr (SUMS) {
#pragma unroll
        for (int i = 0; i < kOwnRows; ++i) was[i] = r0 + tid + i * kSmallThreads < r1 ? sums[r0 + tid + i * kSmallThreads] : 0.f;
    }
    walk.add_up();
    __syncthreads();                                  // (every ring is idle)
#pragma unroll
    for (int nn = 0; nn < NH; ++nn) {
        if (g == 0) *reinterpret_cast<float4*>(&sm.warp_ml[warp][8 * nn + 2 * t]) = make_float4(walk.m[nn][0], walk.l[nn][0], walk.m[nn][1], walk.l[nn][1]);
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
            sm.o[warp][nn * (D / 16) + i][lane] = make_float4(walk.o[nn][i][0], walk.o[nn][i][1], walk.o[nn][i][2], walk.o[nn][i][3]);
    }
    __syncthreads();
    for (int e = tid; e < heads * (D / 4); e += kSmallThreads) {
        const int q = e / (D / 4), c4 = e % (D / 4) * 4;
        float2 s[kSmallWarps];
        float mm = -INFINITY, ll = 0.f;
#pragma unroll
        for (int w = 0; w < kSmallWarps; ++w) { s[w] = sm.warp_ml[w][q]; mm = fmaxf(mm, s[w].x); }
        const float ref = reference_of(mm);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kSmallWarps; ++w) {
            const float f = exp2_fast(s[w].x - ref);
            const float* o = reinterpret_cast<const float*>(&sm.o[w][q / 8 * (D / 16) + c4 / 16][4 * (c4 % 8) + q % 8 / 2]) + (q & 1) + c4 / 8 % 2 * 2;
            const float4 y = make_float4(o[0], o[16], o[32], o[48]);       // (the next dim is four lanes further)
            ll = fmaf(s[w].y, f, ll);
            v.x = fmaf(y.x, f, v.x); v.y = fmaf(y.y, f, v.y); v.z = fmaf(y.z, f, v.z); v.w = fmaf(y.w, f, v.w);
        }
        *reinterpret_cast<float4*>(&sm.cta_o[q][c4]) = v;
        if (c4 == 0) sm.cta_ml[q] = make_float2(mm, ll);
    }
    cluster.sync();
    // the CTAs' parts: a lane takes one of them, n_cta neighbouring lanes join an item (one thread for all of them took 2.9 us of reads from afar)
    const int c = tid & (n_cta - 1), slot = tid / n_cta, slots = kSmallThreads / n_cta;
    auto top = [&](float x) {
        for (int off = 1; off < n_cta; off <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
        return x;
    };
    auto sum = [&](float x) {
        for (int off = 1; off < n_cta; off <<= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
        return x;
    };
    for (int e0 = 0; e0 < heads * (D / 4); e0 += kSmallThreads) {       // every CTA an even share of the items
        const int e = min(e0 + rank * slots + slot, heads * (D / 4) - 1), q = e / (D / 4), c4 = e % (D / 4) * 4;
        const float2 s = *cluster.map_shared_rank(&sm.cta_ml[q], c);
        const float4 y = *reinterpret_cast<const float4*>(cluster.map_shared_rank(&sm.cta_o[q][c4], c));
        const float f = exp2_fast(s.x - reference_of(top(s.x))), ll = sum(s.y * f);
        const float r = ll == 0.f ? 0.f : 1.f / ll;                     // (nothing seen: zeros)
        const float v0 = sum(y.x * f), v1 = sum(y.y * f), v2 = sum(y.z * f), v3 = sum(y.w * f);
        if (c == 0) *reinterpret_cast<uint2*>(a.out + (q_row + q) * D + c4) = make_uint2(pack_bf16(v0 * r, v1 * r), pack_bf16(v2 * r, v3 * r));
    }
    if constexpr (SUMS) {
        for (int q0 = 0; q0 < heads; q0 += slots) {
            const int q = min(q0 + slot, heads - 1);
            const float2 s = *cluster.map_shared_rank(&sm.cta_ml[q], c);
            const float ref = reference_of(top(s.x)), ll = sum(s.y * exp2_fast(s.x - ref));
            if (c == 0) sm.all[q] = make_float2(ref, ll == 0.f ? 0.f : 1.f / ll);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kOwnRows; ++i) {
            const int r = r0 + tid + i * kSmallThreads;
            if (r >= r1) break;
            float add = 0.f;
#pragma unroll 4
            for (int q = 0; q < heads; ++q) add += weight_of(logits[q * a.small_rows + r - r0], sm.all[q]);
            sums[r] = was[i] + add;
        }
    }
    cluster.sync();                                   // (a CTA's part is there until all have read it)
}

// Shared memory that a CTA of that form may have.
constexpr int small_smem(int warps) { return warps == 8 ? 227 * 1024 : 113 * 1024; }

cudaLaunchAttribute cluster_of(int ctas) {
    cudaLaunchAttribute a;
    a.id = cudaLaunchAttributeClusterDimension;
    a.val.clusterDim.x = ctas;
    a.val.clusterDim.y = 1;
    a.val.clusterDim.z = 1;
    return a;
}

template <int D, int NH, bool SUMS, int W>
cudaError_t launch_small(const AttendArgs& a, const AttendPlan& plan, int device, cudaStream_t stream) {
    const int smem = static_cast<int>(sizeof(SmallSmem<D, NH, W>)) + (SUMS ? plan.group * plan.small_rows * 4 : 0);
    auto kernel = attend_small_kernel<D, NH, SUMS, W>;
    static uint64_t set_on = 0;                                 // devices; the caller holds the library's lock
    if ((set_on >> device & 1u) == 0) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, small_smem(W));
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);     // (of 16)
        if (e != cudaSuccess) return e;
        set_on |= 1ull << device;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.B * a.Hkv * a.groups * plan.cluster));
    cfg.blockDim = dim3(32 * W);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1] = cluster_of(plan.cluster);
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <int D, int NH, int RPT, TeamOf TEAM>
cudaError_t launch_join(const AttendArgs& a, cudaLaunchConfig_t cfg) {
    using T = Team<D, TEAM>;
    const int row_blocks = RPT > 0 ? (a.cache.cap + RPT * kJoinThreads - 1) / (RPT > 0 ? RPT * kJoinThreads : 1) : 0;
    const int join_ctas = (a.B * a.Hq * (D / T::kDims) + T::kTeams - 1) / T::kTeams;
    cfg.gridDim = dim3(static_cast<unsigned>(join_ctas + a.B * a.Hkv * row_blocks));
    cfg.blockDim = dim3(kJoinThreads);
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, attend_join_kernel<D, NH, RPT, TEAM>, a, join_ctas, row_blocks);
}

template <int D, int NH, int RPT>
cudaError_t launch_teams(const AttendArgs& a, const cudaLaunchConfig_t& cfg, int n_cta) {
    // records of a unit, where lengths are alike: up to 4 a warp has in flight at once, up to 32 a CTA
    const int records = n_cta / (a.B * a.blocks * a.groups) + 2;
    if (records <= 4) return launch_join<D, NH, RPT, kTeamWarp>(a, cfg);
    if (records <= 36) return launch_join<D, NH, RPT, kTeamCta>(a, cfg);
    return launch_join<D, NH, RPT, kTeamCtas>(a, cfg);
}

template <int D, int NH, bool SUMS>
cudaError_t launch_attend_t(const AttendArgs& a, int n_cta, int device, cudaStream_t stream) {
    constexpr int smem = sizeof(AttSmem<D, NH>);
    static_assert(smem <= 227 * 1024, "an SM's shared memory");
    auto kernel = attend_kernel<D, NH, SUMS>;
    static uint64_t set_on = 0;                                 // devices; the caller holds the library's lock
    if ((set_on >> device & 1u) == 0) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        set_on |= 1ull << device;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(n_cta);
    cfg.blockDim = dim3(kAttThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
    if (e != cudaSuccess) return e;
    // few rows a CTA where there are few of them (two threads' worth of loads in flight then), else enough for about one wave
    if constexpr (SUMS) {
        const long long rows = static_cast<long long>(a.B) * a.Hkv * a.cache.cap;
        return rows <= 2LL * kJoinThreads * 8 * n_cta ? launch_teams<D, NH, 2>(a, cfg, n_cta) : launch_teams<D, NH, 8>(a, cfg, n_cta);
    } else {
        return launch_teams<D, NH, 0>(a, cfg, n_cta);
    }
}

}  // namespace

template <int W>
static size_t small_bytes(int d, int nh) {
    return d == 128 ? (nh == 1 ? sizeof(SmallSmem<128, 1, W>) : sizeof(SmallSmem<128, 2, W>)) : (nh == 1 ? sizeof(SmallSmem<64, 1, W>) : sizeof(SmallSmem<64, 2, W>));
}

// Scratch: (max, sum) and O of two records a CTA, the CTAs that share a unit; where sums are asked for, (max, sum) of the units that one CTA had and
// the logits of all rows.
AttendPlan attend_plan(int B, int Hq, int Hkv, int d, int cap, bool sums, bool wide) {
    AttendPlan p;
    const int G = Hq / Hkv;
    p.nh = G > 8 ? 2 : 1;
    p.groups = (G + 8 * p.nh - 1) / (8 * p.nh);
    p.group = G < 8 * p.nh ? G : 8 * p.nh;
    p.blocks = (Hkv + kAttWarps - 1) / kAttWarps;               // as many heads a CTA as it has warps, and blocks of heads alike
    p.block = (Hkv + p.blocks - 1) / p.blocks;
    p.tile = kAttWarps / p.block * kAttStep;
    p.tile_shift = -1;
    for (int s = 0; s < 31; ++s)
        if (p.tile == 1 << s) p.tile_shift = s;
    const long long tiles = static_cast<long long>(B) * p.blocks * p.groups * ((cap + p.tile - 1) / p.tile);
    p.max_ctas = static_cast<int>(tiles < kAttMaxCtas ? tiles : kAttMaxCtas);
    // Short caches: as many CTAs a head as are resident beside each other (7 clusters of 16, 15 of 8, 33 of 4, 74 of 2 on 148 SMs), up to 1024 rows each
    // (sequences need not be alike), or, where even shares of all SMs would not be many rows less, kSmallRows. us in one launch and in two, 128 dims: one sequence of 8 heads, 100 / 2000 / 4352 / 6000 / 9000 rows 4.7 and 6.8 / 6.2 and 9.2 / 9.0 and 11.8 / 10.4 and 13.2 / 14.0 and 16.0;
    // 16 of them, 300 / 1000 rows 6.2 and 10.1 / 15.5 and 17.7, of unlike lengths 5.9 and 9.4 / 12.8 and 14.4; 8 of 4 heads, 7 query heads each, 4352 rows 17.3 and 18.7,
    // unlike 15.1 and 15.7, with sums 19.9 and 19.9, unlike 17.3 and 16.3; 4 of them, sums, 4352 rows (1088 a CTA, 64 CTAs) 15.2 and 14.3;
    // one of 2 heads, 64 dims, 4352 / 9000 rows 6.2 and 7.3 / 7.7 and 8.2. With sums, between 1024 and kSmallRows: 18 of 8 heads, 1080 rows 19.6 and 21.8, unlike
    // 15.8 and 16.5; 4 of 8 heads, 4340 rows 19.3 and 20.3, unlike 16.2 and 15.8; 8 of 4 heads, 64 dims, 15.0 and 16.0, unlike alike; 4 query heads each,
    // 19.2 and 18.9, unlike 16.3 and 15.6.
    // Clusters of 16 take 0.5 us longer to launch: 3 sequences of 2 heads, 12 query heads each, 300 / 4000 rows 7.5 / 9.9 us with 16, 6.8 / 15.6 without.
    // More heads than SMs, a CTA of four warps each: 24 sequences of 8 heads, 100 / 300 / 600 / 1000 rows 5.3 and 9.4 / 8.6 and 12.3 / 14.6 and 16.7 / 20.6 and
    // 22.6. More than are resident: a CTA of the long form takes a sequence's heads, up to eight, together, so it depends on them. One launch against two: 64
    // sequences of 8 heads, 160 / 240 rows -13 / -4 %, with sums +4 / +10 %, 111 sequences +4 to +30 %; 256 of 2 heads, 64 dims, 320 / 480 rows -22 / -5 %,
    // 444 sequences, 160 / 320 rows -15 / -2 %.
    const long long items = static_cast<long long>(B) * Hkv * p.groups;
    p.cluster = items <= 7 && cap > 1536 && wide ? 16 : items <= 15 ? 8 : items <= 33 ? 4 : items <= 74 ? 2 : 1;
    p.warps = items <= 148 ? 8 : 4;
    const long long steps = (cap + kAttStep - 1) / kAttStep, rows = (steps + p.cluster - 1) / p.cluster * kAttStep;
    const long long kept = rows + 4;                            // (logits of four neighbouring pairs of heads lie in different banks)
    const size_t fixed = p.warps == 8 ? small_bytes<8>(d, p.nh) : small_bytes<4>(d, p.nh);
    const long long most = items <= 148 && rows - items * cap / 148 > 300 ? 1024
                           : items <= 296                                 ? kSmallRows
                           : items <= 592                                 ? (p.block > 4 ? 160 : 400)
                           : items <= kSmallItems && p.block <= 4         ? 160
                                                                          : 0;
    const bool few = rows <= most;
    p.small_rows = static_cast<int>(few ? kept : 0);
    if (!few || (sums && (p.groups > 1 || fixed + 4ull * p.group * kept > static_cast<size_t>(small_smem(p.warps))))) p.cluster = 0;
    if (p.cluster > 0) {
        p.off_o = p.off_whole = p.off_shared = p.off_logits = 0;
        p.bytes = kAttNoScratch;
        return p;
    }
    const size_t heads = static_cast<size_t>(p.max_ctas) * 2 * p.block * p.group;
    p.logit_stride = (cap + 3) / 4 * 4;
    p.off_o = (heads * sizeof(float2) + 255) / 256 * 256;
    p.off_whole = p.off_o + heads * d * sizeof(float);
    p.off_shared = p.off_whole + (sums ? (static_cast<size_t>(B) * Hq * sizeof(float2) + 255) / 256 * 256 : 0);
    p.off_logits = p.off_shared + (static_cast<size_t>(B) * p.blocks * p.groups * sizeof(int2) + 255) / 256 * 256;
    p.bytes = p.off_logits + (sums ? static_cast<size_t>(B) * Hq * p.logit_stride * sizeof(float) : 0);
    return p;
}

// A cluster of 16 CTAs, an SM's shared memory each, needs 16 SMs of one GPC, which parts of a device may not have. (One instantiation answers for all:
// a CTA an SM is what each of them takes.)
bool attend_wide_clusters() {
    auto kernel = attend_small_kernel<128, 1, false, 8>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(16);
    cfg.blockDim = dim3(256);
    cfg.dynamicSmemBytes = small_smem(8);
    cudaLaunchAttribute attr[1] = {cluster_of(16)};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, small_smem(8));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg);
    if (e != cudaSuccess) cudaGetLastError();                   // (said to nobody: the other forms run)
    return e == cudaSuccess && clusters > 0;
}

cudaError_t launch_attend(const AttendArgs& args, const AttendPlan& plan, int d, char* scratch, int num_sms, int device, cudaStream_t stream) {
    if (args.B <= 0) return cudaSuccess;
    AttendArgs a = args;
    a.groups = plan.groups;
    a.group = plan.group;
    a.blocks = plan.blocks;
    a.block = plan.block;
    a.tile = plan.tile;
    a.tile_shift = plan.tile_shift;
    a.part_ml = reinterpret_cast<float2*>(scratch);
    a.part_o = reinterpret_cast<float*>(scratch + plan.off_o);
    a.whole_ml = reinterpret_cast<float2*>(scratch + plan.off_whole);
    a.shared_by = reinterpret_cast<int2*>(scratch + plan.off_shared);
    a.logits = reinterpret_cast<float*>(scratch + plan.off_logits);
    a.logit_stride = plan.logit_stride;
    const int n = num_sms < plan.max_ctas ? num_sms : plan.max_ctas;
    const bool sums = a.weights != nullptr;
    if (plan.cluster > 0) {
        a.small_rows = plan.small_rows;
#define CKV_SMALL_W(D, NH, W) (sums ? launch_small<D, NH, true, W>(a, plan, device, stream) : launch_small<D, NH, false, W>(a, plan, device, stream))
#define CKV_SMALL(D, NH) (plan.warps == 8 ? CKV_SMALL_W(D, NH, 8) : CKV_SMALL_W(D, NH, 4))
        if (d == 128) return plan.nh == 1 ? CKV_SMALL(128, 1) : CKV_SMALL(128, 2);
        return plan.nh == 1 ? CKV_SMALL(64, 1) : CKV_SMALL(64, 2);
#undef CKV_SMALL
#undef CKV_SMALL_W
    }
#define CKV_ATTEND(D, NH) (sums ? launch_attend_t<D, NH, true>(a, n, device, stream) : launch_attend_t<D, NH, false>(a, n, device, stream))
    if (d == 128) return plan.nh == 1 ? CKV_ATTEND(128, 1) : CKV_ATTEND(128, 2);
    return plan.nh == 1 ? CKV_ATTEND(64, 1) : CKV_ATTEND(64, 2);
#undef CKV_ATTEND
}

}  // namespace chunkkv
