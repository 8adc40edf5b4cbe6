// Queries and keys of a fused QKV activation, normalised head by head (root mean square, optional) and turned by the rotary
// embedding of their positions in one pass over the data: for a prompt's tokens into token-major outputs, or for one token a
// sequence with keys and values going straight to their row of a paged cache.
//
//   y = x * rsqrt(mean(x^2) + eps) * gain;   out[i] = y[i] cos - y[i + d/2] sin,   out[i + d/2] = y[i + d/2] cos + y[i] sin
//
// in 32 bits, rounded once to bf16 (the sum of d <= 128 squares of bf16 values and three products keep ~1e-6 of a value, the rounding
// 4e-3). A row is read by d / 16 lanes: lane l holds elements 8l .. 8l + 7 of both halves, so a pair never leaves its lane, loads and
// stores are 16 bytes wide, and a norm takes log2(d / 16) shuffles. A warp works on one token: its angles are read once for all heads.
#include "decode.cuh"

namespace chunkkv {

namespace {

// 28 warps an SM with two rows of every lane in flight: 32768 tokens of 40 heads 110 us; 24 warps 115, 32 warps (spills) 112, 16 warps with four
// rows 121; CTAs of 256 threads, whose last wave is coarser, 114 to 117.
constexpr int kRotThreads = 128;
constexpr int kRotCtas = 7;         // of an SM
constexpr int kRotAhead = 2;        // rows a lane has in flight

template <int D>
struct Rot {
    static constexpr int kLanes = D / 16;           // lanes of a row
    static constexpr int kRows = 32 / kLanes;       // rows of a warp's step
};

__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// One row: both halves of this lane's elements, normalised and turned, a pair of neighbours at a time (few values are live beside the rows in flight).
template <int D>
__device__ __forceinline__ void turn(uint4& lo, uint4& hi, bool norm, float eps, const uint4& gain_lo, const uint4& gain_hi, const float* co,
                                     const float* si) {
    float r = 1.f;
    if (norm) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 a = bf16_pair(word(lo, i)), b = bf16_pair(word(hi, i));
            sum = fmaf(a.x, a.x, fmaf(a.y, a.y, fmaf(b.x, b.x, fmaf(b.y, b.y, sum))));
        }
#pragma unroll
        for (int off = 1; off < Rot<D>::kLanes; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        r = rsqrtf(sum * (1.f / D) + eps);
    }
    uint32_t x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float2 a = bf16_pair(word(lo, i)), b = bf16_pair(word(hi, i));
        if (norm) {
            const float2 ga = bf16_pair(word(gain_lo, i)), gb = bf16_pair(word(gain_hi, i));
            a.x *= r * ga.x; a.y *= r * ga.y; b.x *= r * gb.x; b.y *= r * gb.y;
        }
        const float c0 = co[2 * i], c1 = co[2 * i + 1], s0 = si[2 * i], s1 = si[2 * i + 1];
        x[i] = pack_bf16(a.x * c0 - b.x * s0, a.y * c1 - b.y * s1);
        y[i] = pack_bf16(b.x * c0 + a.x * s0, b.y * c1 + a.y * s1);
    }
    lo = make_uint4(x[0], x[1], x[2], x[3]);
    hi = make_uint4(y[0], y[1], y[2], y[3]);
}

// Work item: `steps` steps of kRows heads of one token, out of ceil(Hq / kRows) steps of queries, then as many as the KV heads take of
// keys and, with a cache, of values.
template <int D, bool CACHE>
__global__ void __launch_bounds__(kRotThreads, kRotCtas) rotate_kernel(const RotateArgs a) {
    constexpr int kL = Rot<D>::kLanes, kR = Rot<D>::kRows;
    begin_dependent();
    const int lane = threadIdx.x & 31, l = lane & (kL - 1), slot = lane / kL;
    const int q_steps = (a.Hq + kR - 1) / kR, k_steps = (a.Hkv + kR - 1) / kR;
    const int all = q_steps + (CACHE ? 2 : 1) * k_steps;
    const int per_token = (all + a.steps - 1) / a.steps;
    const long long item = static_cast<long long>(blockIdx.x) * (kRotThreads / 32) + (threadIdx.x >> 5);
    const long long tok = item / per_token;
    if (tok >= a.T) return;                                              // (a whole warp)
    const int t = static_cast<int>(tok);
    const int s0 = static_cast<int>(item % per_token) * a.steps, s1 = min(s0 + a.steps, all);
    const __nv_bfloat16* x = a.qkv + static_cast<size_t>(t) * a.row_elems + 8 * l;

    float co[8], si[8];
    const int pos = a.positions[t];
    const bool known = static_cast<unsigned>(pos) < static_cast<unsigned>(a.n_pos);
    {
        const size_t at = static_cast<size_t>(known ? pos : 0) * (D / 2) + 8 * l;
        const float4 *c4 = reinterpret_cast<const float4*>(a.cos_t + at), *s4 = reinterpret_cast<const float4*>(a.sin_t + at);
        const float4 c0 = c4[0], c1 = c4[1], n0 = s4[0], n1 = s4[1];
        co[0] = c0.x; co[1] = c0.y; co[2] = c0.z; co[3] = c0.w; co[4] = c1.x; co[5] = c1.y; co[6] = c1.z; co[7] = c1.w;
        si[0] = n0.x; si[1] = n0.y; si[2] = n0.z; si[3] = n0.w; si[4] = n1.x; si[5] = n1.y; si[6] = n1.z; si[7] = n1.w;
    }

    // the heads of steps [b, e) of one part (queries, keys): loads of kRotAhead rows ahead of their use
    auto part = [&](int b, int e, int H, int first, const __nv_bfloat16* gain, auto place) {
        if (b >= e) return;
        const bool norm = gain != nullptr;
        uint4 g_lo = make_uint4(0, 0, 0, 0), g_hi = g_lo;
        if (norm) {
            g_lo = *reinterpret_cast<const uint4*>(gain + 8 * l);
            g_hi = *reinterpret_cast<const uint4*>(gain + D / 2 + 8 * l);
        }
        for (int s = b; s < e; s += kRotAhead) {
            uint4 lo[kRotAhead], hi[kRotAhead];
#pragma unroll
            for (int u = 0; u < kRotAhead; ++u) {
                const int h = (s + u) * kR + slot;
                lo[u] = hi[u] = make_uint4(0, 0, 0, 0);
                if (s + u < e && h < H && known) {
                    const __nv_bfloat16* p = x + static_cast<size_t>(first + h) * D;
                    lo[u] = load_once(p);
                    hi[u] = load_once(p + D / 2);
                }
            }
#pragma unroll
            for (int u = 0; u < kRotAhead; ++u) {
                if (s + u >= e) break;                                   // (uniform: the norm's shuffles take the whole warp)
                const int h = (s + u) * kR + slot;
                turn<D>(lo[u], hi[u], norm, a.eps, g_lo, g_hi, co, si);
                if (!known) lo[u] = hi[u] = make_uint4(0, 0, 0, 0);
                __nv_bfloat16* o = h < H ? place(h) : nullptr;
                if (o != nullptr) {
                    *reinterpret_cast<uint4*>(o) = lo[u];
                    *reinterpret_cast<uint4*>(o + D / 2) = hi[u];
                }
            }
        }
    };
    // this token's place in the cache for head h, or NULL
    auto cached = [&](__nv_bfloat16* cache, int h) -> __nv_bfloat16* {
        const int row = a.lengths[static_cast<size_t>(t) * a.Hkv + h] - 1;
        if (row < 0 || row >= a.cache.cap) return nullptr;
        const int at = paged_row(a.cache, a.cache.tables + static_cast<size_t>(t) * a.cache.max_pages, row);
        return at < 0 ? nullptr : cache + (static_cast<size_t>(at) * a.Hkv + h) * D + 8 * l;
    };

    part(s0, min(s1, q_steps), a.Hq, 0, a.gain_q,
         [&](int h) { return a.out_q + static_cast<size_t>(t) * a.q_token + static_cast<size_t>(h) * a.q_head + 8 * l; });
    part(max(s0 - q_steps, 0), min(s1 - q_steps, k_steps), a.Hkv, a.Hq, a.gain_k, [&](int h) {
        if constexpr (CACHE) return cached(a.cache_K, h);
        else return a.out_k + static_cast<size_t>(t) * a.k_token + static_cast<size_t>(h) * a.k_head + 8 * l;
    });
    if constexpr (CACHE) {
        for (int s = max(s0 - q_steps - k_steps, 0); s < s1 - q_steps - k_steps; ++s) {
            const int h = s * kR + slot;
            __nv_bfloat16* o = h < a.Hkv ? cached(a.cache_V, h) : nullptr;
            if (o != nullptr) {
                const __nv_bfloat16* p = x + static_cast<size_t>(a.Hq + a.Hkv + h) * D;
                const uint4 lo = load_once(p), hi = load_once(p + D / 2);
                *reinterpret_cast<uint4*>(o) = lo;
                *reinterpret_cast<uint4*>(o + D / 2) = hi;
            }
        }
    }
}

}  // namespace

cudaError_t launch_rotate(const RotateArgs& args, int d, int num_sms, cudaStream_t stream) {
    if (args.T <= 0) return cudaSuccess;
    RotateArgs a = args;
    const bool cached = a.cache_K != nullptr;
    const int rows = d == 128 ? Rot<128>::kRows : Rot<64>::kRows;
    const int all = (a.Hq + rows - 1) / rows + (cached ? 2 : 1) * ((a.Hkv + rows - 1) / rows);
    // a warp takes as many of a token's heads as leave 32 warps an SM: the angles are read once for them; few tokens are spread as far as they go
    const long long per = static_cast<long long>(a.T) * all / (32LL * num_sms);
    a.steps = static_cast<int>(per < 1 ? 1 : (per > all ? all : per));
    const long long items = static_cast<long long>(a.T) * ((all + a.steps - 1) / a.steps);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((items + kRotThreads / 32 - 1) / (kRotThreads / 32)));
    cfg.blockDim = dim3(kRotThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (d == 128) return cached ? cudaLaunchKernelEx(&cfg, rotate_kernel<128, true>, a) : cudaLaunchKernelEx(&cfg, rotate_kernel<128, false>, a);
    return cached ? cudaLaunchKernelEx(&cfg, rotate_kernel<64, true>, a) : cudaLaunchKernelEx(&cfg, rotate_kernel<64, false>, a);
}

}  // namespace chunkkv
