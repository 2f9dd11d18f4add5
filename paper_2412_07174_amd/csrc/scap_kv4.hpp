// The 4-bit key/value cache: layout of a block, the quantiser's arithmetic, argument blocks and launchers.
//
// A block holds one kv head's keys and values of one page of P tokens, D channels each, in groups of 32 channels:
//   key codes    [P][D/2] bytes            channel 2i in the low nibble, 2i + 1 in the high one: a token's row is contiguous
//   value codes  [P/4][D/8][4] words       channel 8o + i of a token in nibble i; the words of four tokens side by side
//   key scales   [P][D/32] words           fp16 s, fp16 c
//   value scales [P/4][D/32][2][4] fp16    s of four tokens, then their c
// Each part is laid out as the attention kernel's lanes take it (scap_kv4_attention.hip): the keys' product contracts over channels, so a
// lane holds channels of one token; the values' contracts over tokens, so a lane holds four tokens of one channel octet.
// Codes and key scales are whole words of a token's own.  Its value scales are single halves of words that its neighbours share, written
// with 2-byte stores: tokens of one call, of different workgroups, lie side by side there, so such a word is never read, changed and written back.
//
// A code q stands for s * (q + 64) + c.  The offset makes widening one instruction: a nibble put into bits 4-7 of the fp16
// 64.0 is 64 + q exactly, and one packed fp16 fma gives the value.  c, the value of code -64, is rounded to fp16: it moves
// the grid by at most |c| * 2^-11: 0.035 s where the group is centred (c = -71.5 s), more, as any fp16 offset, where it lies far from 0.
#pragma once

#include "scap_device.hpp"
#include "scap_internal.hpp"

namespace scap {

constexpr int kKv4Group = 32;
constexpr float kKv4Bias = 64.f;
constexpr uint32_t kKv4BadScale = 0x7E007E00u;  // s = c = NaN: an unreadable token

__host__ __device__ constexpr int64_t kv4_block_bytes(int D, int P) { return (int64_t)P * D * 5 / 4; }

// byte offsets of the parts of a block
struct Kv4Layout {
    int D, P;
    __host__ __device__ int64_t vcodes() const { return (int64_t)P * (D / 2); }
    __host__ __device__ int64_t kscales() const { return (int64_t)P * D; }
    __host__ __device__ int64_t vscales() const { return (int64_t)P * D + (int64_t)P * (D / 8); }
    __host__ __device__ int64_t bytes() const { return kv4_block_bytes(D, P); }
};

struct Kv4Pool {
    char* pool;        // [layers][pages][heads][block]
    int32_t* refs;     // [pages]
    int64_t pages;
    int heads, D, P, lgP, layers;
    __host__ __device__ Kv4Layout layout() const { return {D, P}; }
    __host__ __device__ int64_t page_bytes() const { return heads * kv4_block_bytes(D, P); }
    __host__ __device__ int64_t layer_bytes() const { return pages * page_bytes(); }
};

// Sequences of a call: sequence b's new tokens are starts[b] .. starts[b+1] - 1 of the call's, at positions lens[b] - n_b .. lens[b] - 1.
struct Kv4Seqs {
    const int32_t* starts;  // [B + 1]
    const int32_t* table;   // [B][S]
    const int32_t* lens;    // [B]
    int B, S, T;
};

struct Kv4TokensArgs {
    Kv4Pool p;
    Kv4Seqs s;
    int layer, dt;
    const uint16_t* k;  // append: inputs
    const uint16_t* v;
    int64_t k_st, k_sh, v_st, v_sh;  // strides in elements
    uint16_t* k_out;    // read: outputs [T][heads][D]
    uint16_t* v_out;
};

struct Kv4AttnArgs {
    Kv4Pool p;
    Kv4Seqs s;
    int layer, dt;
    const uint16_t* q;
    int64_t q_st, q_sh;
    uint16_t* out;  // [T][H][D]
    float* lse;     // [T][H] or null
    int H, G;       // query heads, query heads per kv head
    float scale;    // softmax scale * log2(e)
    int causal, window;
    double inv_G;   // 1 / G
    int places;     // workgroups of a kv head that the key axis is split for: as many as run at once
    int min_chunk;  // tokens
    int32_t* counters;
    float* partial;
    int64_t slot_floats;  // floats of one workgroup's partial result
    int slot_rows;        // a sequence with more rows is not cut into chunks
    uint32_t partial_bytes;  // what lies at `partial`: accesses beyond are dropped
};

int launch_kv4_append(const Kv4TokensArgs& a, hipStream_t stream);
int launch_kv4_read(const Kv4TokensArgs& a, hipStream_t stream);

struct Kv4AttnPlan {
    int rt, waves;       // row tiles of 16 per wavefront, wavefronts of a workgroup
    bool staged;
    int64_t grid;        // workgroups
    int places;          // workgroups of a kv head that run at once
    int min_chunk;       // tokens
    int64_t slot_floats;
    int slot_rows;
};
Kv4AttnPlan plan_kv4_attention(int D, int kv_heads, int64_t B, int64_t T, int G, int64_t max_new);
// bytes of partial results that a call of up to T tokens may leave
size_t kv4_partial_bytes(int D, int kv_heads, int64_t T, int G, int64_t max_new);
int launch_kv4_attention(const Kv4AttnArgs& a, const Kv4AttnPlan& plan, hipStream_t stream);

int launch_kv4_reserve(const Kv4Pool& p, int32_t* table, int S, int B, const int32_t* old_lens, const int32_t* new_lens,
                       int32_t* info, int32_t* scratch, hipStream_t stream);
int launch_kv4_fork(const Kv4Pool& p, const int32_t* table, const int32_t* lens, int B_in, const int32_t* parents, int B_out,
                    int32_t* table_out, int32_t* lens_out, int S, hipStream_t stream);
int launch_kv4_free(const Kv4Pool& p, int32_t* table, int S, int B, const int32_t* keep_from, const int32_t* keep_to,
                    hipStream_t stream);
int launch_kv4_compact(const Kv4Pool& p, const int32_t* table, int S, int B, int32_t* table_out, int32_t* refs_out,
                       int32_t* info, int32_t* scratch, hipStream_t stream);
int launch_kv4_copy_pages(const Kv4Pool& from, const Kv4Pool& to, const int32_t* src, const int32_t* dst, int64_t n,
                          hipStream_t stream);
constexpr int kKv4MaxReserve = 4096;  // sequences of one reserving call: their needs are held in LDS
// int32 words of scratch the page calls need
inline size_t kv4_page_scratch_words(int64_t pages, int64_t B) { return 64 + 2 * (size_t)B + 3 * (size_t)pages; }

// ---------------------------------------------------------------------------------------------- device side
// first page of (layer, page, head)
__device__ __forceinline__ const char* kv4_block(const Kv4Pool& p, int layer, int64_t page, int head) {
    return p.pool + (layer * p.pages + page) * p.page_bytes() + head * kv4_block_bytes(p.D, p.P);
}

// page of slot `s` of a row, or -1 where the table names none of this pool
__device__ __forceinline__ int kv4_page(const Kv4Pool& p, const int32_t* row, int s) {
    const int e = row[s];
    return (uint32_t)e < (uint64_t)p.pages ? e : -1;
}

// New tokens of sequence b, with starts and lens brought into range whatever the caller's arrays hold.
struct Kv4Span {
    int first, n, len;  // first token of the call, number of new tokens, length with them
};
__device__ __forceinline__ Kv4Span kv4_span(const Kv4Seqs& s, int P, int b) {
    const int a = min(max(s.starts[b], 0), s.T), e = min(max(s.starts[b + 1], a), s.T);
    const int64_t cap = (int64_t)s.S * P;
    const int len = (int)min((int64_t)max(s.lens[b], 0), cap);
    return {a, e - a, len};
}

// Two values rounded to nearest even.
__device__ __forceinline__ uint32_t round16(float x, float y, int dt) {
    typedef __bf16 b2_t __attribute__((ext_vector_type(2)));
    typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
    if (dt == kBF16) return __builtin_bit_cast(uint32_t, b2_t{(__bf16)x, (__bf16)y});
    return __builtin_bit_cast(uint32_t, h2_t{(_Float16)x, (_Float16)y});
}

}  // namespace scap
