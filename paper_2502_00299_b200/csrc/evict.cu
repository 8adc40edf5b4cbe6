// Eviction from a paged cache by the sums of the attention that its rows received: every head with more than `budget` rows goes back to
// at most that many. Of its first C chunks of c rows the k with the largest sums stay (ties to the lower chunk), and the r rows behind them, the window
// among them, always do. Rows move as little as they can: kept chunks below place k stay where they are, the j-th kept chunk at or above it
// fills the j-th free place below it, and the r rows follow, in their order. (Attention does not depend on the order of rows; with the chunks in
// ascending order nearly every row behind the first evicted chunk would move.)
//
// A cluster of 1, 2, 4 or 8 CTAs works on a head. Each finds the selection itself - a chain of latencies on a few thousand keys: select.cuh's body with keys
// in registers up to 24 a thread, beyond that (or for more kept chunks than it lists) a radix select that reads them again - and takes its
// part of the moves. Places in the way of one another are kept apart by cluster barriers: nobody writes before all have read the sums; the chunks
// move before the rows behind them, whose new places may be those chunks' old ones; those rows move in blocks from the lowest on, each read by
// all before any is written, the first of them (mostly the only one) before the chunks move.
#include "decode.cuh"
#include "select.cuh"

#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace chunkkv {

namespace {

constexpr int kEvThreads = 512;
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvAhead = 4;               // 16-byte pieces that a thread has in flight
constexpr int kEvRows = 1024;             // rows whose places are looked up at once

struct RadixSmem {
    alignas(16) int hist[kSelBins];
    int4 cnt[kEvWarps];                   // a warp's chunks: above the threshold, equal to it; the same below place k
    uint2 range[kEvWarps];
    int warp_tot[kEvWarps];
    int2 found;
};
union EvictSmem {
    SelectSmem sel;
    RadixSmem radix;
};
constexpr int kEvMaxKeys = 24;            // keys of a thread in registers, at most

template <int N>
struct Keys { static constexpr int value = N; };     // of a thread

// Order of sums: not-a-number above everything (as torch sorts it), -0 as +0.
__device__ __forceinline__ uint32_t evict_key(float x) { return x != x ? 0xffffffffu : select_order_key(x); }

template <int VPR>
__global__ void __launch_bounds__(kEvThreads, 2) evict_kernel(const EvictArgs a) {
    constexpr unsigned kFull = 0xffffffffu;
    extern __shared__ __align__(16) char smem_raw[];
    EvictSmem& sm = *reinterpret_cast<EvictSmem*>(smem_raw);
    unsigned short* from = reinterpret_cast<unsigned short*>(smem_raw + sizeof(EvictSmem));    // kept chunks at or above place k
    unsigned short* to = from + a.list_cap;                                                    // free places below it
    int2* rows_at = reinterpret_cast<int2*>(to + a.list_cap);                                  // places in the cache of kEvRows rows and of where they go
    uint32_t* kbuf = reinterpret_cast<uint32_t*>(rows_at);                                     // before that: keys, where there is room for them
    begin_dependent();
    cg::cluster_group cluster = cg::this_cluster();
    const int n_cta = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int bh = blockIdx.x / n_cta, b = bh / a.Hkv, h = bh - b * a.Hkv;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int part = rank * kEvThreads + tid, parts = n_cta * kEvThreads;                      // this thread in the cluster
    const int32_t* table = a.cache.tables + static_cast<size_t>(b) * a.cache.max_pages;
    float* weights = a.weights + static_cast<size_t>(bh) * a.cache.cap;
    int32_t* idx = a.out_idx + static_cast<size_t>(bh) * a.budget;
    const int n = min(max(a.lengths[bh], 0), a.cache.cap), c = a.c;
    if (n <= a.budget) {                                            // (the whole cluster)
        // (a budget may be any number up to 2^31 - 1, so that the last step of the index goes beyond it; all other counts here are below 2^30)
        for (unsigned i = part; i < static_cast<unsigned>(a.budget); i += parts) idx[i] = i < static_cast<unsigned>(n) ? static_cast<int>(i) : -1;
        return;
    }
    const int C = (n - a.w) / c, r = n - C * c, k = (a.budget - r) / c;     // k < C, as n is above the budget

    // ---- which chunks stay: lists of those that move and of the places that are free
    auto key_of = [&](int ch) -> uint32_t {
        if (c == 1) return evict_key(weights[ch]);
        const float* w = weights + static_cast<size_t>(ch) * c;
        double sum = 0.0;                                           // (in order and 64 bits, rounded once: equal sums are equal)
        for (int i0 = 0; i0 < c; i0 += 8) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i0 + i < c ? w[i0 + i] : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += static_cast<double>(v[i]);
        }
        return evict_key(static_cast<float>(sum));
    };
    auto stay_put = [&] {                                           // (rows that move overwrite theirs behind the barrier)
        for (int i = part; i < k * c; i += parts) idx[i] = i;
    };
    const unsigned short* moved = from;
    int stay = 0;
    if (k > 0 && C <= kEvMaxKeys * kEvThreads && C <= a.key_cap && k <= kSelCap) {
        const int per = (C + kEvThreads - 1) / kEvThreads;
        auto select = [&](auto keys_of_thread) {
            constexpr int KPT = decltype(keys_of_thread)::value;
            uint32_t lo = 0xffffffffu, hi = 0u;
            auto take = [&](int ch, uint32_t key) {
                kbuf[ch] = key;
                lo = min(lo, key);
                hi = max(hi, key);
            };
            if (c == 1) {                                           // (all loads before the first use)
                float v[KPT];
#pragma unroll
                for (int u = 0; u < KPT; ++u) v[u] = tid + u * kEvThreads < C ? weights[tid + u * kEvThreads] : 0.f;
                stay_put();
#pragma unroll
                for (int u = 0; u < KPT; ++u)
                    if (tid + u * kEvThreads < C) take(tid + u * kEvThreads, evict_key(v[u]));
            } else {
                for (int ch = tid; ch < C; ch += kEvThreads) take(ch, key_of(ch));
                stay_put();
            }
            lo = __reduce_min_sync(kFull, lo);
            hi = __reduce_max_sync(kFull, hi);
            if (lane == 0) sm.sel.warp_sums[warp] = static_cast<unsigned long long>(hi) << 32 | lo;
            select_clear(sm.sel);
            __syncthreads();
            select_staged<KPT>(kbuf, C, k, sm.sel);
        };
        if (per <= 2) select(Keys<2>{});
        else if (per <= 4) select(Keys<4>{});
        else if (per <= 6) select(Keys<6>{});
        else if (per <= 8) select(Keys<8>{});
        else if (per <= 10) select(Keys<10>{});
        else if (per <= 12) select(Keys<12>{});
        else select(Keys<kEvMaxKeys>{});
        // The kept chunks are in ascending order: `stay` of them lie below k, and the j-th free place below k is j + i, where i of them lie below it.
        const unsigned short* kept = sm.sel.sel;
        auto count = [&](int most, auto before) {                   // of the first `most`, those that come first and of which that holds
            int lo_i = 0, hi_i = most;
            while (lo_i < hi_i) {
                const int mid = (lo_i + hi_i) >> 1;
                if (before(mid)) lo_i = mid + 1;
                else hi_i = mid;
            }
            return lo_i;
        };
        stay = count(k, [&](int i) { return kept[i] < k; });
        for (int j = tid; j < k - stay; j += kEvThreads) to[j] = static_cast<unsigned short>(j + count(stay, [&](int i) { return kept[i] - i <= j; }));
        __syncthreads();
        moved = kept + stay;
    } else if (k > 0) {
        stay_put();
        const bool staged = C <= a.key_cap;
        auto key_at = [&](int ch) { return staged ? kbuf[ch] : key_of(ch); };
        uint32_t lo = 0xffffffffu, hi = 0u;
#pragma unroll 4
        for (int ch = tid; ch < C; ch += kEvThreads) {
            const uint32_t key = key_of(ch);
            if (staged) kbuf[ch] = key;
            lo = min(lo, key);
            hi = max(hi, key);
        }
        lo = __reduce_min_sync(kFull, lo);
        hi = __reduce_max_sync(kFull, hi);
        if (lane == 0) sm.radix.range[warp] = make_uint2(lo, hi);
        for (int i = tid; i < kSelBins; i += kEvThreads) sm.radix.hist[i] = 0;
        __syncthreads();
        const uint2 mm = sm.radix.range[lane & (kEvWarps - 1)];
        uint32_t base = __reduce_min_sync(kFull, mm.x), span = __reduce_max_sync(kFull, mm.y) - base;
        int need = k;                                               // the need-th largest key in [base, base + span]
        for (int round = 0; span != 0u; ++round) {
            const int shift = max(0, 21 - __clz(span));             // (span >> shift) < kSelBins
            if (round > 0) {
                for (int i = tid; i < kSelBins; i += kEvThreads) sm.radix.hist[i] = 0;
                __syncthreads();
            }
            for (int ch = tid; ch < C; ch += kEvThreads) {
                const uint32_t dlt = key_at(ch) - base;             // (a key below base wraps to more than span)
                if (dlt <= span) atomicAdd(&sm.radix.hist[dlt >> shift], 1);
            }
            __syncthreads();
            // thread t has the bins 2047 - 4t .. 2044 - 4t, so a prefix over threads counts from the top
            const int4 b4 = *reinterpret_cast<const int4*>(sm.radix.hist + kSelBins - 4 - 4 * tid);
            const int cnt[4] = {b4.w, b4.z, b4.y, b4.x};
            const int sum = (cnt[0] + cnt[1]) + (cnt[2] + cnt[3]);
            int inc = sum;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int v = __shfl_up_sync(kFull, inc, off);
                if (lane >= off) inc += v;
            }
            if (lane == 31) sm.radix.warp_tot[warp] = inc;
            __syncthreads();
            inc += __reduce_add_sync(kFull, lane < warp ? sm.radix.warp_tot[lane & (kEvWarps - 1)] : 0);
            if (inc - sum < need && need <= inc) {                  // one thread
                int above = inc - sum, q = 0;
#pragma unroll
                for (int i = 0; i < 3; ++i)                         // (unrolled: cnt stays in registers)
                    if (q == i && above + cnt[i] < need) { above += cnt[i]; q = i + 1; }
                sm.radix.found = make_int2(kSelBins - 1 - 4 * tid - q, need - above);
            }
            __syncthreads();
            const int2 f = sm.radix.found;
            need = f.y;
            const uint32_t sub = static_cast<uint32_t>(f.x) << shift;
            base += sub;
            span = min((1u << shift) - 1u, span - sub);
        }
        const uint32_t thresh = base;
        const int need_eq = need;                                   // of those equal to it, the first so many are kept

        // ---- lists of the moves. A warp has a block of consecutive chunks and walks it 32 at a time.
        const int rows = (C + kEvThreads - 1) / kEvThreads, first = warp * rows * 32;
        const unsigned below = (1u << lane) - 1u;
        int4 mine = make_int4(0, 0, 0, 0);
        for (int u = 0; u < rows; ++u) {
            const int ch = first + 32 * u + lane;
            const uint32_t key = ch < C ? key_at(ch) : 0u;
            const unsigned gt = __ballot_sync(kFull, ch < C && key > thresh), eq = __ballot_sync(kFull, ch < C && key == thresh);
            const unsigned low = __ballot_sync(kFull, ch < k);
            mine.x += __popc(gt);
            mine.y += __popc(eq);
            mine.z += __popc(gt & low);
            mine.w += __popc(eq & low);
        }
        if (lane == 0) sm.radix.cnt[warp] = mine;
        __syncthreads();
        int gt_run = 0, eq_run = 0, low_gt = 0, low_eq = 0;
#pragma unroll
        for (int v = 0; v < kEvWarps; ++v) {
            const int4 x = sm.radix.cnt[v];
            if (v < warp) { gt_run += x.x; eq_run += x.y; }
            low_gt += x.z;
            low_eq += x.w;
        }
        stay = low_gt + min(low_eq, need_eq);
        for (int u = 0; u < rows; ++u) {
            const int ch = first + 32 * u + lane;
            const uint32_t key = ch < C ? key_at(ch) : 0u;
            const bool gt = ch < C && key > thresh, eq = ch < C && key == thresh;
            const unsigned gtm = __ballot_sync(kFull, gt), eqm = __ballot_sync(kFull, eq);
            const int eq_before = eq_run + __popc(eqm & below);
            const int before = gt_run + __popc(gtm & below) + min(eq_before, need_eq);     // kept chunks before this one
            const bool kept = gt || (eq && eq_before < need_eq);
            if (ch < k) {
                if (!kept) to[ch - before] = static_cast<unsigned short>(ch);
            } else if (kept) {
                from[before - stay] = static_cast<unsigned short>(ch);
            }
            gt_run += __popc(gtm);
            eq_run += __popc(eqm);
        }
    }
    const int moves = k - stay;                                     // as many move as places below k are free
    cluster.sync();          // the lists are there, and every CTA has read the sums and the length

    // ---- the rows. A thread holds pieces of 16 bytes; a row's keys and values are 2 VPR of them.
    constexpr int kPieces = 2 * VPR;
    uint4 *K = a.K + static_cast<size_t>(h) * VPR, *V = a.V + static_cast<size_t>(h) * VPR;
    const size_t row_vecs = static_cast<size_t>(a.Hkv) * VPR;
    const int chunk_rows = moves * c, dst_r = k * c, src_r = C * c;
    auto piece = [&](int at, int vec) { return (vec < VPR ? K + vec : V + (vec - VPR)) + static_cast<size_t>(at) * row_vecs; };   // of the cache's row `at`

    // the r rows behind the chunks go in blocks of kEvAhead pieces a thread (a piece more a row: its sum)
    constexpr int kItems = kPieces + 1;
    const long long items = static_cast<long long>(r) * kItems, block = static_cast<long long>(kEvAhead) * parts;
    uint4 w[kEvAhead];
    void* w_to[kEvAhead];                                           // NULL: none, or its page is outside the cache
    auto load_block = [&](long long i0) {
#pragma unroll
        for (int u = 0; u < kEvAhead; ++u) {
            const long long i = i0 + static_cast<long long>(u) * parts + part;
            w_to[u] = nullptr;
            if (i >= items) continue;
            const int row = static_cast<int>(i / kItems), vec = static_cast<int>(i % kItems);
            if (vec < kPieces) {
                const int from_at = paged_row(a.cache, table, src_r + row), to_at = paged_row(a.cache, table, dst_r + row);
                w[u] = from_at >= 0 ? load_once(piece(from_at, vec)) : make_uint4(0, 0, 0, 0);
                if (to_at >= 0) w_to[u] = piece(to_at, vec);
            } else {
                w[u].x = __float_as_uint(weights[src_r + row]);
                w_to[u] = weights + dst_r + row;
            }
        }
    };
    auto store_block = [&](long long i0) {
#pragma unroll
        for (int u = 0; u < kEvAhead; ++u) {
            const long long i = i0 + static_cast<long long>(u) * parts + part;
            if (w_to[u] == nullptr) continue;
            if (static_cast<int>(i % kItems) < kPieces) *static_cast<uint4*>(w_to[u]) = w[u];
            else *static_cast<float*>(w_to[u]) = __uint_as_float(w[u].x);
        }
    };
    load_block(0);

    // the chunks: every CTA takes an even share of their rows. Where those are in the cache is looked up once a row, kEvRows rows at a time, and their sums
    // move with that; then groups of threads copy a row each, kEvAhead rows in flight. (Looked up piece by piece, 32 x 8 heads of 4352 rows took 34.2 us instead of 31.0.)
    const int m0 = static_cast<int>(static_cast<long long>(chunk_rows) * rank / n_cta), m1 = static_cast<int>(static_cast<long long>(chunk_rows) * (rank + 1) / n_cta);
    for (int b0 = m0; b0 < m1; b0 += kEvRows) {
        const int nb = min(kEvRows, m1 - b0);
        for (int i = tid; i < nb; i += kEvThreads) {
            const int j = (b0 + i) / c, off = (b0 + i) - j * c, src = moved[j] * c + off, dst = to[j] * c + off;
            rows_at[i] = make_int2(paged_row(a.cache, table, src), paged_row(a.cache, table, dst));
            weights[dst] = weights[src];
            idx[dst] = src;
        }
        __syncthreads();
        const int vec = tid % kPieces;
        for (int i0 = tid / kPieces; i0 < nb; i0 += kEvAhead * (kEvThreads / kPieces)) {
            uint4 v[kEvAhead];
            int to_at[kEvAhead];
#pragma unroll
            for (int u = 0; u < kEvAhead; ++u) {
                const int i = i0 + u * (kEvThreads / kPieces);
                const int2 at = i < nb ? rows_at[i] : make_int2(-1, -1);
                to_at[u] = at.y;
                v[u] = at.x >= 0 && at.y >= 0 ? load_once(piece(at.x, vec)) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int u = 0; u < kEvAhead; ++u)
                if (to_at[u] >= 0) *piece(to_at[u], vec) = v[u];
        }
        __syncthreads();
    }
    cluster.sync();          // the chunks' old places may be written now, and those of the first block
    store_block(0);
    for (long long i0 = block; i0 < items; i0 += block) {
        load_block(i0);
        cluster.sync();
        store_block(i0);
    }
    if (items > block) cluster.sync();       // (no block of sums is read any more: those behind the last row become zero)
    const int len = dst_r + r;
    for (int i = len + part; i < n; i += parts) weights[i] = 0.f;
    for (int i = part; i < a.budget - dst_r; i += parts) idx[dst_r + i] = i < r ? src_r + i : -1;
    if (part == 0) a.lengths[bh] = len;
}

}  // namespace

EvictPlan evict_plan(int cap, int c, int smem_limit) {
    EvictPlan p;
    const long long chunks = cap / c;
    // at most half the chunks move: as many as places below k are free, and k of C chunks are kept
    const long long list = (chunks / 2 + 8) / 8 * 8;        // (kbuf behind the lists is 16-byte aligned)
    p.fits = chunks <= kSelMaxChunks;
    p.list_cap = p.fits ? static_cast<int>(list) : 0;
    const long long fixed = sizeof(EvictSmem) + 4LL * p.list_cap;
    const long long keys = (smem_limit - fixed) / 4;
    p.key_cap = static_cast<int>(chunks + 4 <= keys ? (chunks + 3) / 4 * 4 : 0);
    p.smem_bytes = static_cast<int>(fixed + (p.key_cap > 2 * kEvRows ? 4LL * p.key_cap : 8LL * kEvRows));
    return p;
}

cudaError_t launch_evict(const EvictArgs& args, const EvictPlan& plan, int B, int d, int num_sms, cudaStream_t stream) {
    if (B <= 0) return cudaSuccess;
    EvictArgs a = args;
    a.list_cap = plan.list_cap;
    a.key_cap = plan.key_cap;
    auto kernel = d == 128 ? evict_kernel<16> : evict_kernel<8>;
    if (plan.smem_bytes > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, plan.smem_bytes);
        if (e != cudaSuccess) return e;
    }
    const long long units = static_cast<long long>(B) * a.Hkv;
    int ctas = 1;
    while (ctas < 8 && units * ctas * 2 <= 2LL * num_sms) ctas *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(units * ctas));
    cfg.blockDim = dim3(kEvThreads);
    cfg.dynamicSmemBytes = plan.smem_bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

}  // namespace chunkkv
