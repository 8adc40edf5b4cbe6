// The rotary embedding in the forms that rotate.cu does not have: tables of angles, scaled for long contexts or not; heads that turn as
// neighbouring pairs or as two halves, whole or in their first `rot` dims; and a turn's tokens, many of each sequence, on their way into the
// paged cache.
//
//   tables   cos/sin[p][i] = scale * cos/sin((first + p) w_i)
//   rows     y = x * rsqrt(mean(x^2) + eps) * gain (optional); of dims 0 .. rot - 1 the pairs (j, k) = (i, i + rot / 2) or (2i, 2i + 1) become
//            (y_j cos_i - y_k sin_i, y_k cos_i + y_j sin_i); the others stay y
//
// all in 32 bits, rounded once (bf16 outputs: 2^-8; the arithmetic keeps 1e-6).
#include "decode.cuh"
#include "rows.h"

namespace chunkkv {

namespace {

// ------------------------------------------------------------------------------------------------ tables
// What bounds it is the writing, 8 bytes a pair of angles. An angle is kept as a fraction of a turn in 64 bits that wrap, so that a position is an
// addition, the reduction to a turn costs nothing and is exact, and 2^30 positions are as good as one: the upper 32 bits (2^-32 of a turn, 1.5e-9
// rad) go to an eighth of a turn and into the Taylor series of sine and cosine there (to x^9 and x^8: 3e-8). A thread keeps four pairs of the row and walks
// down the positions; a warp's stores are whole lines. 131072 positions of 64 pairs: 14.4 us (4.7 TB/s written), with eight CTAs an SM whose threads read their
// turns out of the constants 16.4.
constexpr int kTabThreads = 256;

__device__ __forceinline__ void sincos_turn(unsigned long long turn, float scale, float& s, float& c) {
    const int32_t hi = static_cast<int32_t>(turn >> 32);
    const uint32_t quarter = (static_cast<uint32_t>(hi) + 0x20000000u) >> 30;
    const float x = static_cast<float>(static_cast<int32_t>(static_cast<uint32_t>(hi) - (quarter << 30))) * 1.4629180792671596e-9f;    // 2 pi / 2^32
    const float y = x * x;
    const float sn = x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
    const float cs = fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 40320, -1.f / 720), 1.f / 24), -0.5f), 1.f);
    s = (quarter & 1u) ? cs : sn;
    c = (quarter & 1u) ? sn : cs;
    s *= (quarter & 2u) ? -scale : scale;
    c *= ((quarter + 1u) & 2u) ? -scale : scale;
}

__global__ void __launch_bounds__(kTabThreads) tables_kernel(const TableArgs a) {
    begin_dependent();
    const int per_row = a.rot / 8, rows = blockDim.x / per_row;              // (blockDim.x = rows * per_row)
    const int i4 = threadIdx.x % per_row * 4;
    long long p = static_cast<long long>(blockIdx.x) * rows + threadIdx.x / per_row;
    const long long stride = static_cast<long long>(gridDim.x) * rows;
    __shared__ unsigned long long turn[kMaxRot / 2];          // (lanes read different ones, which the constant cache serves one after the other)
    if (threadIdx.x < a.rot / 2) turn[threadIdx.x] = a.turn[threadIdx.x];
    __syncthreads();
    unsigned long long at[4], step[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned long long w = turn[i4 + e];
        at[e] = (a.first + static_cast<unsigned long long>(p)) * w;
        step[e] = static_cast<unsigned long long>(stride) * w;
    }
    for (; p < a.n_pos; p += stride) {
        float4 c, s;
        sincos_turn(at[0], a.scale, s.x, c.x);
        sincos_turn(at[1], a.scale, s.y, c.y);
        sincos_turn(at[2], a.scale, s.z, c.z);
        sincos_turn(at[3], a.scale, s.w, c.w);
        const size_t o = static_cast<size_t>(p) * (a.rot / 2) + i4;
        *reinterpret_cast<float4*>(a.cos_t + o) = c;
        *reinterpret_cast<float4*>(a.sin_t + o) = s;
#pragma unroll
        for (int e = 0; e < 4; ++e) at[e] += step[e];
    }
}

// ------------------------------------------------------------------------------------------------ rows
// A row is read by d / 16 lanes with two pieces of 16 bytes each, whose pairs never leave the lane: dims 8l and rot / 2 + 8l on of a row that
// turns in halves (lanes behind them hold two pieces that stay as they are), pieces l and l + d / 16 of one that turns in pairs. A warp works on one token: its
// angles are read once for all heads. Memory bounds it, so rows of two steps are in flight, with 28 warps an SM, as in rotate.cu.
constexpr int kRowThreads = 128;
constexpr int kRowCtas = 7;          // of an SM
constexpr int kRowAhead = 2;

__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

template <int D, bool PAIRS>
struct Turned {
    static constexpr int kLanes = D / 16, kRows = 32 / kLanes;
    int pa, pb;              // this lane's pieces of a row
    bool ta, tb;             // whether they turn
    float co[8], si[8];      // angles: of halves, pair i of (piece a, piece b); of neighbours, four pairs of piece a, then of piece b

    __device__ __forceinline__ void angles(const RotateRowsArgs& a, int l, int pos) {
        const int half = a.rot / 16;
        if constexpr (PAIRS) {
            pa = l; pb = l + kLanes;
            ta = 8 * pa < a.rot; tb = 8 * pb < a.rot;
        } else {
            ta = tb = l < half;
            pa = ta ? l : 2 * l; pb = ta ? l + half : 2 * l + 1;
        }
        const size_t row = static_cast<size_t>(pos) * (a.rot / 2);
        const int ca = PAIRS ? 4 * pa : 8 * l, cb = PAIRS ? 4 * pb : 8 * l + 4;
        const float4 one = make_float4(1.f, 1.f, 1.f, 1.f), none = make_float4(0.f, 0.f, 0.f, 0.f);
        const float4 c0 = ta ? *reinterpret_cast<const float4*>(a.r.cos_t + row + ca) : one, c1 = tb ? *reinterpret_cast<const float4*>(a.r.cos_t + row + cb) : one;
        const float4 s0 = ta ? *reinterpret_cast<const float4*>(a.r.sin_t + row + ca) : none, s1 = tb ? *reinterpret_cast<const float4*>(a.r.sin_t + row + cb) : none;
        co[0] = c0.x; co[1] = c0.y; co[2] = c0.z; co[3] = c0.w; co[4] = c1.x; co[5] = c1.y; co[6] = c1.z; co[7] = c1.w;
        si[0] = s0.x; si[1] = s0.y; si[2] = s0.z; si[3] = s0.w; si[4] = s1.x; si[5] = s1.y; si[6] = s1.z; si[7] = s1.w;
    }
    // One row: norm and turn of this lane's two pieces. (Values that stay are not multiplied by 1 and 0: they may be infinite.)
    __device__ __forceinline__ void apply(uint4& x, uint4& y, bool norm, float eps, const uint4& gx, const uint4& gy) const {
        float r = 1.f;
        if (norm) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 a = bf16_pair(word(x, i)), b = bf16_pair(word(y, i));
                sum = fmaf(a.x, a.x, fmaf(a.y, a.y, fmaf(b.x, b.x, fmaf(b.y, b.y, sum))));
            }
#pragma unroll
            for (int off = 1; off < kLanes; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            r = rsqrtf(sum * (1.f / D) + eps);
        }
        uint32_t u[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float2 a = bf16_pair(word(x, i)), b = bf16_pair(word(y, i));
            if (norm) {
                const float2 ga = bf16_pair(word(gx, i)), gb = bf16_pair(word(gy, i));
                a.x *= r * ga.x; a.y *= r * ga.y; b.x *= r * gb.x; b.y *= r * gb.y;
            }
            if constexpr (PAIRS) {
                u[i] = ta ? pack_bf16(a.x * co[i] - a.y * si[i], a.y * co[i] + a.x * si[i]) : pack_bf16(a.x, a.y);
                v[i] = tb ? pack_bf16(b.x * co[4 + i] - b.y * si[4 + i], b.y * co[4 + i] + b.x * si[4 + i]) : pack_bf16(b.x, b.y);
            } else {
                const float c0 = co[2 * i], c1 = co[2 * i + 1], s0 = si[2 * i], s1 = si[2 * i + 1];
                u[i] = ta ? pack_bf16(a.x * c0 - b.x * s0, a.y * c1 - b.y * s1) : pack_bf16(a.x, a.y);
                v[i] = ta ? pack_bf16(b.x * c0 + a.x * s0, b.y * c1 + a.y * s1) : pack_bf16(b.x, b.y);
            }
        }
        x = make_uint4(u[0], u[1], u[2], u[3]);
        y = make_uint4(v[0], v[1], v[2], v[3]);
    }
};

// How many of the n ascending values are at most t, by the 32 lanes of a warp together: 32 sequences take one step, a thousand two.
__device__ __forceinline__ int count_up_to(const int32_t* v, int n, int t) {
    const int lane = threadIdx.x & 31;
    int lo = 0;
    for (int len = n; len > 0;) {
        const int step = (len + 31) / 32, i = lo + (lane + 1) * step - 1;
        const int c = __popc(__ballot_sync(0xffffffffu, (lane + 1) * step <= len && v[i] <= t));
        len = min(step - 1, len - c * step);
        lo += c * step;
    }
    return lo;
}

// Work item: `steps` steps of kRows heads of one token, out of ceil(Hq / kRows) steps of queries, then as many as the KV heads take of keys and, with a
// cache, of values.
template <int D, bool PAIRS, bool CACHE>
__global__ void __launch_bounds__(kRowThreads, kRowCtas) rotate_rows_kernel(const RotateRowsArgs args) {
    using Turn = Turned<D, PAIRS>;
    constexpr int kL = Turn::kLanes, kR = Turn::kRows;
    const RotateArgs& a = args.r;
    begin_dependent();
    const int lane = threadIdx.x & 31, l = lane & (kL - 1), slot = lane / kL;
    const int q_steps = (a.Hq + kR - 1) / kR, k_steps = (a.Hkv + kR - 1) / kR;
    const int all = q_steps + (CACHE ? 2 : 1) * k_steps;
    const int per_token = (all + a.steps - 1) / a.steps;
    const long long item = static_cast<long long>(blockIdx.x) * (kRowThreads / 32) + (threadIdx.x >> 5);
    const long long tok = item / per_token;
    if (tok >= a.T) return;                                              // (a whole warp)
    const int t = static_cast<int>(tok);
    const int s0 = static_cast<int>(item % per_token) * a.steps, s1 = min(s0 + a.steps, all);
    const __nv_bfloat16* x = a.qkv + static_cast<size_t>(t) * a.row_elems;
    const int pos = a.positions[t];
    int seq = 0, back = 0;                                               // the token's sequence; its row is lengths - back
    if constexpr (CACHE) {
        seq = count_up_to(args.starts + 1, args.B, t);
        if (seq >= args.B || args.starts[seq] > t) return;               // in no sequence: nothing of it is written
        back = args.starts[seq + 1] - t;
        if (back <= 0) return;                                           // (starts that are not ascending)
    }
    const bool known = static_cast<unsigned>(pos) < static_cast<unsigned>(a.n_pos);
    Turn turn;
    turn.angles(args, l, known ? pos : 0);
    const int oa = 8 * turn.pa, ob = 8 * turn.pb;

    // the heads of steps [b, e) of one part (queries, keys): loads of kRowAhead rows ahead of their use
    auto part = [&](int b, int e, int H, int first, const __nv_bfloat16* gain, auto place) {
        if (b >= e) return;
        const bool norm = gain != nullptr;
        uint4 ga = make_uint4(0, 0, 0, 0), gb = ga;
        if (norm) {
            ga = *reinterpret_cast<const uint4*>(gain + oa);
            gb = *reinterpret_cast<const uint4*>(gain + ob);
        }
        for (int s = b; s < e; s += kRowAhead) {
            uint4 u[kRowAhead], v[kRowAhead];
            __nv_bfloat16* o[kRowAhead];
#pragma unroll
            for (int n = 0; n < kRowAhead; ++n) {
                const int h = (s + n) * kR + slot;
                u[n] = v[n] = make_uint4(0, 0, 0, 0);
                if (s + n < e && h < H && known) {
                    const __nv_bfloat16* p = x + static_cast<size_t>(first + h) * D;
                    u[n] = load_once(p + oa);
                    v[n] = load_once(p + ob);
                }
            }
#pragma unroll
            for (int n = 0; n < kRowAhead; ++n) o[n] = s + n < e && (s + n) * kR + slot < H ? place((s + n) * kR + slot) : nullptr;      // (looked up while the rows travel)
#pragma unroll
            for (int n = 0; n < kRowAhead; ++n) {
                if (s + n >= e) break;                                   // (uniform: the norm's shuffles take the whole warp)
                turn.apply(u[n], v[n], norm, a.eps, ga, gb);
                if (!known) u[n] = v[n] = make_uint4(0, 0, 0, 0);
                if (o[n] != nullptr) {
                    *reinterpret_cast<uint4*>(o[n] + oa) = u[n];
                    *reinterpret_cast<uint4*>(o[n] + ob) = v[n];
                }
            }
        }
    };
    // this token's row in the cache for head h, or NULL
    auto cached = [&](__nv_bfloat16* cache, int h) -> __nv_bfloat16* {
        const int len = a.lengths[static_cast<size_t>(seq) * a.Hkv + h];
        if (len < back || len - back >= a.cache.cap) return nullptr;
        const int at = paged_row(a.cache, a.cache.tables + static_cast<size_t>(seq) * a.cache.max_pages, len - back);
        return at < 0 ? nullptr : cache + (static_cast<size_t>(at) * a.Hkv + h) * D;
    };

    part(s0, min(s1, q_steps), a.Hq, 0, a.gain_q,
         [&](int h) { return a.out_q + static_cast<size_t>(t) * a.q_token + static_cast<size_t>(h) * a.q_head; });
    part(max(s0 - q_steps, 0), min(s1 - q_steps, k_steps), a.Hkv, a.Hq, a.gain_k, [&](int h) {
        if constexpr (CACHE) return cached(a.cache_K, h);
        else return a.out_k + static_cast<size_t>(t) * a.k_token + static_cast<size_t>(h) * a.k_head;
    });
    if constexpr (CACHE) {
        for (int s = max(s0 - q_steps - k_steps, 0); s < s1 - q_steps - k_steps; ++s) {
            const int h = s * kR + slot;
            if (h >= a.Hkv) continue;
            const __nv_bfloat16* p = x + static_cast<size_t>(a.Hq + a.Hkv + h) * D;
            const uint4 u = load_once(p + 8 * l), v = load_once(p + 8 * (l + kL));
            __nv_bfloat16* o = cached(a.cache_V, h);
            if (o != nullptr) {
                *reinterpret_cast<uint4*>(o + 8 * l) = u;
                *reinterpret_cast<uint4*>(o + 8 * (l + kL)) = v;
            }
        }
    }
}

cudaLaunchConfig_t dependent(dim3 grid, dim3 block, cudaStream_t stream, cudaLaunchAttribute* attr) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.stream = stream;
    attr->id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr->val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

template <int D, bool PAIRS>
cudaError_t launch_rows(const cudaLaunchConfig_t& cfg, const RotateRowsArgs& a) {
    return a.r.cache_K != nullptr ? cudaLaunchKernelEx(&cfg, rotate_rows_kernel<D, PAIRS, true>, a) : cudaLaunchKernelEx(&cfg, rotate_rows_kernel<D, PAIRS, false>, a);
}

}  // namespace

cudaError_t launch_tables(const TableArgs& a, int num_sms, cudaStream_t stream) {
    if (a.n_pos <= 0) return cudaSuccess;
    const int per_row = a.rot / 8, rows = kTabThreads / per_row;
    const long long blocks = (static_cast<long long>(a.n_pos) + rows - 1) / rows, most = 4LL * num_sms;      // (a round of them: to begin takes a thread eight products of 64 bits)
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = dependent(dim3(static_cast<unsigned>(blocks < most ? blocks : most)), dim3(rows * per_row), stream, &attr);
    return cudaLaunchKernelEx(&cfg, tables_kernel, a);
}

cudaError_t launch_rotate_rows(const RotateRowsArgs& args, int d, bool interleaved, int num_sms, cudaStream_t stream) {
    if (args.r.T <= 0) return cudaSuccess;
    RotateRowsArgs a = args;
    const int rows = 512 / d;
    const int all = (a.r.Hq + rows - 1) / rows + (a.r.cache_K != nullptr ? 2 : 1) * ((a.r.Hkv + rows - 1) / rows);
    // A token's heads are shared by so many warps that there are four rounds of those that an SM has room for, if there are as many steps: the last round is then
    // mostly full, and the angles are read a few times at most.
    const long long want = 4LL * (kRowThreads / 32) * kRowCtas * num_sms;
    const int share = static_cast<int>(want / a.r.T < 1 ? 1 : (want / a.r.T > all ? all : want / a.r.T));
    a.r.steps = (all + share - 1) / share;
    const long long items = static_cast<long long>(a.r.T) * ((all + a.r.steps - 1) / a.r.steps);
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = dependent(dim3(static_cast<unsigned>((items + kRowThreads / 32 - 1) / (kRowThreads / 32))), dim3(kRowThreads), stream, &attr);
    if (d == 128) return interleaved ? launch_rows<128, true>(cfg, a) : launch_rows<128, false>(cfg, a);
    return interleaved ? launch_rows<64, true>(cfg, a) : launch_rows<64, false>(cfg, a);
}

}  // namespace chunkkv
