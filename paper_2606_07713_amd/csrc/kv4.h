// Internal launch interface and layout of the four-bit key/value cache
// (kv4.hip, kv4_attn.hip).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace moa {

// The pool, and which token is where (moa_kv4.h).
struct Kv4Cache {
    unsigned char* base;
    const int* seq_lens;
    const int* new_lens;    // or null: n of them
    const int* table;       // [B][max_pages], or null: sequence b has page b
    long long page_bytes;   // of one head
    int B, hk, n, d;
    int page, num_pages, max_pages;
};

// New keys and values into the cache, or the values that it holds out of it.
struct Kv4Rows {
    Kv4Cache c;
    const void* kin; const void* vin;   // write
    void* kout; void* vout;             // read
    long long ks[3], vs[3];             // element strides (batch, head, row)
    bool bf16;
};

// Quads (aligned fours) of tokens that a run of n touches at most: (n + 3) / 4
// where it begins at one, one more elsewhere.
inline int kv4_quads(long long n) { return (int)((n + 6) / 4); }
// Workgroups of a write or read: d/8 of 256 threads for each sequence, head and quad.
inline long long kv4_row_blocks(long long B, long long hk, long long n, long long d) {
    const long long per = 256 / (d / 8);
    return (B * hk * kv4_quads(n) + per - 1) / per;
}

hipError_t launch_kv4_write(const Kv4Rows& p, hipStream_t stream);
hipError_t launch_kv4_read(const Kv4Rows& p, hipStream_t stream);

struct Kv4Attn {
    Kv4Cache c;
    const void* q;
    void* o;
    float* lse;             // nullable
    long long qs[3], os[3];
    int hq;
    float scale;
    bool causal, out_bf16;
    // Key splits (1 = none) and their partial states: [B][hq][n][splits][d]
    // fp32, then [B][hq][n][splits][2] (reference in log2 units, sum).
    int splits;
    float* ws;
};

// Rows (queries times heads of a group) that one workgroup of the attention takes.
int kv4_rows_per_block(int rows);

hipError_t launch_kv4_attn(const Kv4Attn& p, hipStream_t stream);

}  // namespace moa
