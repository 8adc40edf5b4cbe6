// Host-side declarations of the kernels for turns of many tokens and for shared prefixes (rotate_rows.cu, attend_rows.cu).
#pragma once
#include "decode.h"

#include <cuda.h>

namespace chunkkv {

// Tables of the rotary embedding (rotate_rows.cu): row p, pair i turns by (first + p) * turn[i] / 2^64 of a full turn.
constexpr int kMaxRot = 128;
struct TableArgs {
    unsigned long long turn[kMaxRot / 2];
    int n_pos, rot;
    unsigned long long first;                 // modulo 2^64, as the products are
    float scale;
    float *cos_t, *sin_t;                     // [n_pos, rot / 2]
};
cudaError_t launch_tables(const TableArgs& args, int num_sms, cudaStream_t stream);

// Queries and keys of T tokens normalised and rotated, in halves or in neighbouring pairs, the first `rot` dims: RotateArgs with two
// more, and, with a cache, tokens starts[b] to starts[b + 1] - 1 as the last rows of sequence b.
struct RotateRowsArgs {
    RotateArgs r;                             // r.lengths [B, Hkv]
    int rot;
    const int32_t* starts;                    // [B + 1]
    int B;
};
cudaError_t launch_rotate_rows(const RotateRowsArgs& args, int d, bool interleaved, int num_sms, cudaStream_t stream);

// Attention of many rows a KV head over a paged cache (attend_rows.cu): the tokens of a turn, or of the sequences that share a prefix. A set is a table
// with the rows that its tokens see; set i has the tokens starts[i] to starts[i + 1] - 1, or (starts NULL) token i.
constexpr int kRowsCtas = 148;                // CTAs of a launch, at most
struct RowSets {
    const int32_t *tables, *lengths, *starts; // [n, max_pages], [n, Hkv], [n + 1] or NULL
    int n, max_pages, cap;
    int slots;                                // blocks of tokens and heads of a KV head, some of them empty
};
struct AttendRowsArgs {
    __nv_bfloat16* out;
    RowSets sets[2];                          // shared prefixes: the prefixes, then the sequences' own rows; else the sequences, and nothing
    PagedCache cache;                         // page_size, num_pages, magic, shift (tables and cap: of the sets)
    int T, Hq, Hkv, G;
    bool causal, shared;
    float scale_log2;                         // log2(e) / sqrt(d)
    int heads, head_blocks, tokens;           // a block: this many heads of a group (head_blocks such blocks) and tokens
    int thin_tokens;                          // tokens of a block that takes at most 128 rows
    int box;                                  // rows of the cache that are fetched together; 0: single ones, in fours
    int units, record_rows;
    float2* part_ml;                          // [2 CTAs][record_rows] of units that several CTAs share: (reference, sum)
    float4* part_o;                           // [2 CTAs][d / 4][record_rows]
    int4* begun;                              // [CTAs][2]: the unit that a CTA begins and does not end
    int* first_bad;                           // [CTAs][pieces][d]: of a piece's dims, the first row with a value that is not finite
    int2* owners;                             // [units]: first and last CTA (shared)
    float2* whole_ml;                         // [2][Hkv][T G] of units that one CTA has (shared)
    float4* whole_o;                          // [2][d / 4][Hkv][T G]
};
struct AttendRowsPlan {
    long long slots0, slots1, units;
    int heads, head_blocks, tokens, thin_tokens, record_rows;
    size_t off_o, off_begun, off_bad, off_owners, off_whole_ml, off_whole_o, bytes;
};
// T tokens in n sets; shared: T sequences in n groups.
AttendRowsPlan attend_rows_plan(int T, int n, int Hq, int Hkv, int d, bool shared);
// maps: of the queries [T, Hq, d], boxes of 64 dims, plan.heads heads and plan.tokens, or plan.thin_tokens, tokens; of the cache's rows, keys and values
// [num_pages * page_size, Hkv d], boxes of 64 dims and args.box rows, or one.
cudaError_t launch_attend_rows(const AttendRowsArgs& args, const AttendRowsPlan& plan, const CUtensorMap* maps, int d, char* scratch, int num_sms,
                               cudaStream_t stream);
// Whether a kernel of the current device gave up on a bounded wait since the last call.
cudaError_t attend_rows_status(bool* gave_up);
// For tests: the clocks behind which a wait of the current device's kernels is abandoned (0: as ever).
cudaError_t attend_rows_wait_clocks(long long clocks);

}  // namespace chunkkv
