// Attention over the 4-bit cache, for any number of new tokens per sequence.
//
//   S[t, r] = k_t . q_r,   P = 2^(a S - m),   O[r, :] = sum_t P[t, r] v_t / sum_t P[t, r]
//
// A kv head's G query heads and a sequence's new tokens are the rows r of one product.  A wavefront takes RT tiles of 16 rows and walks over 32
// tokens at a time; both products are formed transposed, S^T = K Q^T and O^T = V^T P^T, with the 16 x 16 x 32 fp16 matrix
// instruction.  So the probabilities leave the first product in the very lanes that the second takes them from, and a lane takes
// both cache operands as its words lie in a block: that is the order in which each product contracts.  Up to 16 rows, and more while they are
// few, the operands stay in registers and the loop touches no LDS; blocks of 256 rows widen 64 tokens at a time into LDS for
// all eight wavefronts (Stage).
//
// Widening: value = s (q + 64) + c, one bit-field insert and half a packed fp16 fma per value.  Roundings to 16 bits, all of them fp16
// and all relative 2^-11 or less: a widened key or value (the exact one has 18 bits), a query (scaled by a power of two per row
// so that its largest channel lies in [1, 2): bf16 values lose nothing above 2^-24 of that), a probability (kept in
// [2^-14, 2^15]: 2^kShift times the usual one).  Sums, maxima and the running state are fp32.
//
// What bounds it: with one row tile the read of the cache, once there is enough of it (16 sequences of 32768 tokens, 8 heads of 128 channels:
// 114 us, 5.9 TB/s), else a chain of eight dependent trips to memory (905 tokens: 9.5 us).  With many rows the steps of the longest
// block, one behind the other (prompts of 2048 and 1409 tokens: 32 steps of 64 tokens where a place has 25 on average; 79 us, 0.64 PFLOP/s),
// and in a step products and vector instructions that two wavefronts a SIMD, which meet at a barrier, hardly overlap: each is busy about a
// quarter of the time, LDS 15 %.
#include <type_traits>

#include "scap_gemv_parts.hpp"
#include "scap_kv4.hpp"
#include "scap_kv4_split.hpp"

namespace scap {

namespace {

typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef float f4_t __attribute__((ext_vector_type(4)));

constexpr int kOcc1 = 4, kOcc2 = 2;  // wavefronts on a SIMD, with one and with two row tiles each
constexpr int kStagedWaves = 8;      // wavefronts of a workgroup, staged
constexpr int kSplitRows = 64;  // staged: rows of a sequence, up to which a workgroup's wavefronts share 32 of them and split the tokens
constexpr int kUnits = 256;      // compute units
constexpr int kTile = 32;        // tokens a wavefront takes at a time
// Tokens of a workgroup, at least, where the key axis is split: one row tile (905 tokens of 8 heads, us: 128 9.6, 256 10.5, 512 11.5), two.
constexpr int kMinChunk1 = 128, kMinChunk2 = 256;
constexpr float kShift = 10.f;   // probabilities are held times 2^kShift ...
constexpr float kSlack = 5.f;    // ... and the running maximum is moved only when it is passed by more than 2^kSlack
constexpr float kNone = -3.402823466e38f;  // maximum of nothing (finite: 2^(-inf - kNone) is 0 and no NaN)
// From this size of a maximum on, scores are rounded before it is taken off.  One fma, which is cheaper, takes it off the exact product: the maximum's
// own probability is then 2^(its rounding) instead of 1, which below is 1 in fp16 and from 2^23 on would be past its range or 0.
constexpr float kFar = 4096.f;

__device__ __forceinline__ h2_t as_h2(uint32_t u) { return __builtin_bit_cast(h2_t, u); }
__device__ __forceinline__ uint32_t as_u32(h2_t h) { return __builtin_bit_cast(uint32_t, h); }

union Frag {
    h8_t v;
    h2_t h[4];
    uint32_t u[4];
};

// 64 + code, twice, of the nibbles at bits 4-7 of either half
__device__ __forceinline__ h2_t widen(uint32_t x, uint32_t magic) { return as_h2((x & 0x00F000F0u) | magic); }

// What one tile takes from the cache, as it lies there.
template <int D>
struct RawKeys {
    static constexpr int KW = D / 32;  // words of codes per lane and 16 tokens: D / 4 channels, all of one group
    uint32_t k[2][KW];
    uint32_t s[2];
};
struct RawValues {
    uint4 v[2], s[2];  // four tokens of an octet of channels; s of the four, c of the four
};

// A lane's place in the four parts of a block, for 16 tokens from its first one on: keys are taken as (token = lane & 15,
// channels from (lane >> 4) * D / 4), values as (octet = lane & 15, or & 7 of 64 channels; tokens 4 * (lane >> 4) .. + 3).
// What 16 tokens share -- page, head, first token -- goes into a scalar address, so a load costs no vector instruction but itself.
template <int D>
struct Places {
    uint32_t kc, ks, vc, vs;
    __device__ __forceinline__ Places() {
        const uint32_t lane = lane_id(), lo = lane & 15, quarter = lane >> 4, octet = lane & (D / 8 - 1);
        kc = lo * (D / 2) + quarter * (D / 8);
        ks = lo * (D / 8) + (D == 64 ? quarter >> 1 : quarter) * 4;
        vc = (quarter * (D / 8) + octet) * 16;
        vs = (quarter * (D / 32) + (octet >> 2)) * 16;
    }
};
// ONCE: no other workgroup reads these words (a sequence of one block of rows), so they claim no cache lines: 137 -> 127 us on
// 16 x 32768 tokens of 8 heads.
template <typename T, bool ONCE>
__device__ __forceinline__ T load_at(const char* base, uint32_t off) {
    typedef uint32_t vec_t __attribute__((ext_vector_type(sizeof(T) / 4)));
    const vec_t* p = reinterpret_cast<const vec_t*>(base + off);
    return __builtin_bit_cast(T, ONCE ? __builtin_nontemporal_load(p) : *p);
}

template <int D, bool ONCE>
__device__ __forceinline__ void load_keys(RawKeys<D>& r, int half, const char* block, int slot, int P, const Places<D>& at) {
    const Kv4Layout L = {D, P};
    const char* codes = block + slot * (D / 2);
    if constexpr (D == 64) {
        const uint2 t = load_at<uint2, ONCE>(codes, at.kc);
        r.k[half][0] = t.x, r.k[half][1] = t.y;
    } else {
        const uint4 t = load_at<uint4, ONCE>(codes, at.kc);
        r.k[half][0] = t.x, r.k[half][1] = t.y, r.k[half][2] = t.z, r.k[half][3] = t.w;
    }
    r.s[half] = load_at<uint32_t, ONCE>(block + L.kscales() + slot * (D / 8), at.ks);
}

template <int D, bool ONCE>
__device__ __forceinline__ void load_values(RawValues& r, int half, const char* block, int slot, int P, const Places<D>& at) {
    const Kv4Layout L = {D, P};
    r.v[half] = load_at<uint4, ONCE>(block + L.vcodes() + slot * (D / 2), at.vc);
    r.s[half] = load_at<uint4, ONCE>(block + L.vscales() + slot * (D / 8), at.vs);
}

// Rows of the product and what they see.
struct Rows {
    int first, n;         // of the sequence's G * new tokens
    int lo, hi;           // tokens that any of the rows sees
    int lo_all, hi_all;   // tokens that all of them see
};

struct Work {
    int b, head, block, chunk, chunks;
    int slot, counter;    // of the partial result and the arrivals; chunks > 1 only
    bool split;           // the wavefronts share rows and split the tokens (else the other way round)
    Kv4Span span;
};

// row / G: one fp64 product is off by at most one below 2^31
__device__ __forceinline__ int over_group(const Kv4AttnArgs& a, int row) {
    int i = (int)((double)row * a.inv_G);
    i -= i * a.G > row;
    i += (i + 1) * a.G <= row;
    return i;
}

__device__ __forceinline__ Rows rows_of(const Kv4AttnArgs& a, const Kv4Span& sp, int first, int most) {
    Rows r;
    r.first = first;
    r.n = min(most, sp.n * a.G - first);
    if (r.n <= 0) return {first, 0, 0, 0, 0, 0};
    const int p0 = sp.len - sp.n + over_group(a, first), p1 = sp.len - sp.n + over_group(a, first + r.n - 1);  // positions, maybe < 0
    r.hi = a.causal ? max(p1 + 1, 0) : sp.len;
    r.hi_all = a.causal ? max(p0 + 1, 0) : sp.len;
    r.lo = a.window ? max(p0 - a.window + 1, 0) : 0;
    r.lo_all = a.window ? max(p1 - a.window + 1, 0) : 0;
    return r;
}

// inclusive prefix sum across the wavefront in six adds, without LDS
template <typename T>
__device__ __forceinline__ T dpp_scan(T v) {
    const auto add = [&](auto ctrl, auto rows) {
        constexpr int C = decltype(ctrl)::value, R = decltype(rows)::value;
        v += __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), C, R, 0xF, true));
    };
    add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xF>{});  // row_shr 1, 2, 4, 8
    add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xF>{});
    add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xF>{});
    add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xF>{});
    const T last = v;
    v += __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, last), 0x142, 0xA, 0xF, false));  // row_bcast 15
    const T row = v;
    v += __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, row), 0x143, 0xC, 0xF, false));   // row_bcast 31
    return v;
}
__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }
__device__ __forceinline__ float last_lane(float v) { return read_lane_f(v, 63); }

// The workgroup's share.  Every workgroup works out the whole distribution from the lengths alone: the key axis is cut into chunks of
// about 1 / target of all the work, so that one long sequence among short ones is spread over as many workgroups as a batch of
// equal ones, and the host need not know any length.
template <int RT, int WAVES, bool STAGED>
__device__ __forceinline__ bool find_work(const Kv4AttnArgs& a, Work& w) {
    const int lane = lane_id(), heads = a.p.heads;
    constexpr int ROWS = 16 * RT;
    struct Seq {
        Kv4Span sp;
        int blocks, range;
    };
    const auto load = [&](int b) {
        Seq q = {{0, 0, 0}, 0, 0};
        if (b >= a.s.B) return q;
        q.sp = kv4_span(a.s, a.p.P, b);
        const int rows = q.sp.n * a.G;
        q.blocks = !STAGED || rows <= kSplitRows ? (rows + ROWS - 1) / ROWS : (rows + WAVES * ROWS - 1) / (WAVES * ROWS);
        const int p0 = q.sp.len - q.sp.n;
        q.range = max(q.sp.len - (a.window ? max(p0 - a.window + 1, 0) : 0), 0);
        return q;
    };
    const Seq first = load(lane);  // the only ones, as a rule
    const auto each = [&](auto body) {
        for (int base = 0; base < a.s.B; base += kWave)
            if (body(base, base == 0 ? first : load(base + lane))) break;
    };
    const auto cut = [&](const Seq& q, int chunk, float inv) {
        return kv4_cut(q.range, q.sp.n * a.G, chunk, inv, a.places, a.slot_rows);
    };
    float total = 0.f;  // work, in rows' blocks times tokens
    int n = 0;
    each([&](int, const Seq& q) {
        total += last_lane(dpp_scan((float)q.blocks * (float)q.range));
        n += last_lane(dpp_scan(q.blocks));
        return false;
    });
    float inv = 0.f;
    const int chunk = kv4_choose_chunk(total, n, max(a.places, 1), a.min_chunk, inv, [&](int chunk, float inv) {
        int items = 0;
        each([&](int, const Seq& q) {
            items += last_lane(dpp_scan(q.blocks * cut(q, chunk, inv)));
            return false;
        });
        return items;
    });
    int item = blockIdx.x / heads, slots = 0, counters = 0;
    w.head = blockIdx.x - item * heads;
    bool found = false;
    each([&](int base, const Seq& q) {
        const int chunks = cut(q, chunk, inv);
        const int items = q.blocks * chunks;
        const int end = dpp_scan(items);
        const int send = dpp_scan(chunks > 1 ? items : 0), cend = dpp_scan(chunks > 1 ? q.blocks : 0);
        const uint64_t past = __ballot(end > item);
        if (past == 0) {
            item -= last_lane(end);
            slots += last_lane(send);
            counters += last_lane(cend);
            return false;
        }
        const int l = __builtin_ctzll(past);
        const int in = item - __builtin_amdgcn_readlane(end - items, l);
        w.b = base + l;
        w.chunks = __builtin_amdgcn_readlane(chunks, l);
        const int nb = __builtin_amdgcn_readlane(q.blocks, l);
        const int from = nb == 1 ? 0 : in / w.chunks;
        w.block = nb - 1 - from;  // the last rows, which see most, first
        w.chunk = in - from * w.chunks;
        const bool parts = w.chunks > 1;
        w.slot = (slots + __builtin_amdgcn_readlane(send, l) - (parts ? nb * w.chunks - in : 0)) * heads + w.head;
        w.counter = (counters + __builtin_amdgcn_readlane(cend, l) - (parts ? nb - from : 0)) * heads + w.head;
        w.span = {__builtin_amdgcn_readlane(q.sp.first, l), __builtin_amdgcn_readlane(q.sp.n, l), __builtin_amdgcn_readlane(q.sp.len, l)};
        w.split = !STAGED || w.span.n * a.G <= kSplitRows;
        found = true;
        return true;
    });
    return found;
}

// One row tile's queries: lane (row = lane & 15, quarter) holds the channels that it holds of a key, in the order in which widening
// leaves them, times 2^-e with e the exponent of the row's largest.  back: 2^e.  A row with an infinity is NaN throughout: its scores are
// infinite or NaN, their softmax is NaN in either case, and scores of -infinity alone would look like a row that sees nothing.
template <int D>
__device__ __forceinline__ void load_queries(const Kv4AttnArgs& a, const Work& w, int row, bool live, Frag* q, float& back) {
    constexpr int KW = D / 32;
    const int quarter = lane_id() >> 4;
    float x[KW][8];
    uint32_t most = 0;
    const int i = live ? over_group(a, row) : 0, g = live ? row - i * a.G : 0;
    const uint16_t* p = a.q + (int64_t)(w.span.first + i) * a.q_st + (int64_t)(w.head * a.G + g) * a.q_sh + quarter * (D / 4);
#pragma unroll
    for (int o = 0; o < KW; ++o) {
        const uint4 t = live ? load_octet(p + 8 * o) : make_uint4(0, 0, 0, 0);
        const uint32_t h[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t b = (h[j >> 1] >> (16 * (j & 1))) & 0xFFFFu;
            x[o][j] = a.dt == kBF16 ? bf16_bits_to_f32(b) : f16_bits_to_f32(b);
            most = max(most, __float_as_uint(x[o][j]) & 0x7FFFFFFFu);  // bits of |x| order as |x| (NaN on top)
        }
    }
    most = max(most, (uint32_t)__shfl_xor((int)most, 16, kWave));
    most = max(most, (uint32_t)__shfl_xor((int)most, 32, kWave));
    const uint32_t ex = most >> 23;
    const bool scaled = most != 0 && ex < 255;
    const uint32_t e = min(max(ex, 1u), 253u);
    const float f = scaled ? __uint_as_float((254u - e) << 23) : most == 0 ? 1.f : __builtin_nanf("");
    back = scaled ? __uint_as_float(e << 23) : 1.f;
#pragma unroll
    for (int o = 0; o < KW; ++o)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            q[o].h[j][0] = (_Float16)(x[o][j] * f);
            q[o].h[j][1] = (_Float16)(x[o][j + 4] * f);
        }
}

template <int D, int RT>
struct State {
    Frag q[RT][D / 32];
    f4_t o[RT][D / 16];
    f4_t l[RT];     // sum of the probabilities, in every element; kept current in [0] only
    float m[RT];    // running maximum (base 2)
    float past[RT]; // what a score has to pass for it to be moved: kSlack above, any score where it is far
    float w[RT], base[RT];  // a probability is 2^(w score + base)
    float a[RT];    // score -> base-2 logarithm
    int lo[RT], hi[RT];  // what my row of the tile sees
};

// A lane's keys of 16 tokens, widened: what the first product takes.
template <int D>
__device__ __forceinline__ void widen_keys(const uint32_t (&w)[D / 32], uint32_t scale, uint32_t magic, Frag (&k)[D / 32]) {
    const h2_t sc = as_h2(scale);
    const h2_t ss = {sc[0], sc[0]}, cc = {sc[1], sc[1]};
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        k[i].h[0] = __builtin_elementwise_fma(widen(w[i] << 4, magic), ss, cc);
        k[i].h[1] = __builtin_elementwise_fma(widen(w[i], magic), ss, cc);
        k[i].h[2] = __builtin_elementwise_fma(widen(w[i] >> 4, magic), ss, cc);
        k[i].h[3] = __builtin_elementwise_fma(widen(w[i] >> 8, magic), ss, cc);
    }
}

// A lane's values of 32 tokens, widened, two product tiles (2b, 2b + 1) at a time, of those from 2 from on: body(i, operand).
template <int D, typename F>
__device__ __forceinline__ void widen_values(const RawValues& raw, int b0, int b1, int from, uint32_t magic, F body) {
    h2_t sc[2][4];  // s of tokens 0 1, 2 3, then c of the same
#pragma unroll
    for (int half = 0; half < 2; ++half)
        sc[half][0] = as_h2(raw.s[half].x), sc[half][1] = as_h2(raw.s[half].y), sc[half][2] = as_h2(raw.s[half].z), sc[half][3] = as_h2(raw.s[half].w);
    const uint32_t upper = D == 64 ? (uint32_t)(lane_id() & 8) >> 2 : 0u;  // 64 channels: lanes 8-15 take the octet's upper half
#pragma unroll
    for (int b = b0; b < b1; ++b) {
        // byte b of two tokens' words: nibble 2b in bits 0-3, 2b + 1 in bits 4-7 of either half
        const uint32_t sel = 0x0C040C00u + ((uint32_t)(b + from) + upper) * 0x00010001u;
        uint32_t x[2][2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            x[half][0] = __builtin_amdgcn_perm(raw.v[half].y, raw.v[half].x, sel);
            x[half][1] = __builtin_amdgcn_perm(raw.v[half].w, raw.v[half].z, sel);
        }
#pragma unroll
        for (int odd = 0; odd < 2; ++odd) {
            Frag v;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    v.h[2 * half + e] = __builtin_elementwise_fma(widen(odd ? x[half][e] : x[half][e] << 4, magic), sc[half][e], sc[half][2 + e]);
            body(2 * b + odd, v);
        }
    }
}

// A token that no row sees may hold anything, and one that some rows do not see must not reach them as 0 * NaN: its value scales become
// 0.  (The rows that do see an unreadable token are NaN by its key's scales already.)  t: the first of the lane's four tokens.
__device__ __forceinline__ uint4 cover(const uint4& s, int t, int lo, int hi, bool ok) {
    uint32_t x[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t sh = 16 * (e & 1), ms = 0x7C00u << sh;
        const bool drop = t + e < lo || t + e >= hi || !ok || (x[e >> 1] & ms) == ms || (x[2 + (e >> 1)] & ms) == ms;
        if (drop) x[e >> 1] &= ~(0xFFFFu << sh), x[2 + (e >> 1)] &= ~(0xFFFFu << sh);
    }
    return make_uint4(x[0], x[1], x[2], x[3]);
}

// Scores of 16 tokens from t on that a row does not see.
template <int D, int RT>
__device__ __forceinline__ void hide(const State<D, RT>& st, int r, int t, bool ok, f4_t& s) {
    const uint32_t at = (uint32_t)(t + 4 * (lane_id() >> 4) - st.lo[r]), span = ok ? (uint32_t)(st.hi[r] - st.lo[r]) : 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = at + e < span ? s[e] : -__builtin_inff();
    __builtin_amdgcn_sched_barrier(0);  // (one set of masks at a time: scalar registers)
}

// S^T of 16 tokens
template <int D, int RT>
__device__ __forceinline__ void scores(const State<D, RT>& st, const Frag (&k)[D / 32], f4_t (&s)[RT]) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        {
            f4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < D / 32; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[i].v, st.q[r][i].v, acc, 0, 0, 0);
            s[r] = acc;
        }
    }
}

// The state brought up to the maximum of N times 16 tokens' scores.  Those of rows whose maximum is far become what is left above it.
template <int D, int RT, int N>
__device__ __forceinline__ void raise(State<D, RT>& st, int r, f4_t (&s)[N][RT]) {
    float most = s[0][r][0];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) most = fmaxf(most, s[n][r][e]);
    most *= st.a[r];
    if (__ballot(most > st.past[r]) != 0) {
        most = fmaxf(most, __shfl_xor(most, 16, kWave));
        most = fmaxf(most, __shfl_xor(most, 32, kWave));
        const float m = fmaxf(st.m[r], most);
        const float f = __builtin_amdgcn_exp2f(st.m[r] - m);
        st.m[r] = m;
        st.l[r][0] *= f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) st.o[r][i] *= f;
        const bool far = fabsf(m) >= kFar && m != kNone;
        st.past[r] = far ? -__builtin_inff() : m + kSlack;
        st.base[r] = far ? kShift : kShift - m;
        st.w[r] = far ? 1.f : st.a[r];
        if (__ballot(far) != 0) {
#pragma clang fp contract(off)
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][r][e] = far ? s[n][r][e] * st.a[r] - m : s[n][r][e];
        }
    }
}

// Probabilities of one row tile and 32 tokens.
template <int D, int RT>
__device__ __forceinline__ Frag probabilities(const State<D, RT>& st, int r, const f4_t& s0, const f4_t& s1) {
    Frag p;
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const f4_t& s = half ? s1 : s0;
            const float x = __builtin_amdgcn_exp2f(fmaf(s[2 * e], st.w[r], st.base[r]));
            const float y = __builtin_amdgcn_exp2f(fmaf(s[2 * e + 1], st.w[r], st.base[r]));
            p.h[2 * half + e] = h2_t{(_Float16)x, (_Float16)y};
        }
    return p;
}

// Adds the probabilities up: one product with a matrix of ones, which leaves every quarter of the wavefront the sum over all.
template <int D, int RT>
__device__ __forceinline__ void add_ones(State<D, RT>& st, int r, const Frag& p) {
    Frag one;
    one.u[0] = one.u[1] = one.u[2] = one.u[3] = 0x3C003C00u;
    st.l[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(one.v, p.v, st.l[r], 0, 0, 0);
}

// Many rows: WAVES times ROWS of them share what is widened.  64 tokens lie in LDS as the products' operands -- a wavefront
// has widened 16 tokens' keys, or half the product tiles of 32 tokens' values, and leaves them in the very lanes that use them -- and the
// next 64 are widened into a second buffer while these are multiplied; the words behind those are on their way.
constexpr int kWide = 64;
template <int D>
constexpr int kStageHalf = kWide * D * 2;  // bytes of the keys, and of the values

// Pages ahead of the loop: lane l holds where the (k0 + l)-th 16 tokens that the wavefront takes have their page, in units of 16 bytes from
// the layer's first page (kNoPage: nowhere), and the next 64 are on their way.  A scalar load per page instead would be waited for
// in every round, at the barrier's pace.
constexpr uint32_t kNoPage = 0xFFFFFFFFu;
template <typename TOKEN>
struct Ahead {
    const int32_t* row;
    int S, lgP, k0;
    uint32_t pages, unit, now, next;
    uint64_t there;  // lanes of `now` that have a page
    TOKEN token;
    __device__ __forceinline__ Ahead(const int32_t* row, int S, const Kv4Pool& p, TOKEN token)
        : row(row), S(S), lgP(p.lgP), k0(0), pages((uint32_t)p.pages), unit((uint32_t)(p.page_bytes() >> 4)), token(token) {
        now = load(0);
        next = load(kWave);
        there = __ballot(now != kNoPage);
    }
    __device__ __forceinline__ uint32_t load(int k) const {
        const int s = token(k + lane_id()) >> lgP;
        const uint32_t e = s < S ? (uint32_t)row[s] : kNoPage;
        return e < pages ? e * unit : kNoPage;
    }
    // from here on k and those up to the next multiple of 64 are asked for
    __device__ __forceinline__ void reach(int k) {
        if (k - k0 < kWave) return;
        k0 += kWave;
        now = next;
        next = load(k0 + kWave);
        there = __ballot(now != kNoPage);
    }
    __device__ __forceinline__ uint32_t operator[](int k) const { return __builtin_amdgcn_readlane(now, k - k0); }
    // whether N of them from k on have a page, a bit each
    template <int N>
    __device__ __forceinline__ uint32_t have(int k) const { return (uint32_t)(there >> (k - k0)) & ((1u << N) - 1); }
};

template <int D, int WAVES>
struct Stage {
    static_assert(WAVES == 4 || WAVES == 8, "four shares of keys and four of values");
    static constexpr int KW = D / 32, MO = D / 16;
    RawKeys<D> rk;  // [0] only
    RawValues rv;
    uint32_t vok;  // whether the values' two 16s have pages

    static __device__ __forceinline__ bool keys(int wave) { return WAVES == 4 || wave < 4; }
    static __device__ __forceinline__ bool values(int wave) { return WAVES == 4 || wave >= 4; }

    // loads of my share of 64 tokens from tok on
    // (k: the first of their four 16s)
    template <typename AHEAD, typename BLOCK>
    __device__ __forceinline__ void fetch(int wave, int tok, int k, int P, const AHEAD& pages, const BLOCK& block_of, const Places<D>& at) {
        if (keys(wave)) {
            const int t = tok + 16 * wave;
            load_keys<D, false>(rk, 0, block_of(pages[k + wave]), t & (P - 1), P, at);
        }
        if (values(wave)) {
            const int t = tok + 32 * ((wave & 3) >> 1);
            vok = pages.template have<2>(k + (wave & 2));
            load_values<D, false>(rv, 0, block_of(pages[k + (wave & 2)]), t & (P - 1), P, at);
            load_values<D, false>(rv, 1, block_of(pages[k + (wave & 2) + 1]), (t + 16) & (P - 1), P, at);
        }
    }
    __device__ __forceinline__ void widen_into(int wave, char* buf, int tok, bool edge, const Rows& all, uint32_t magic) {
        uint4* out = reinterpret_cast<uint4*>(buf) + lane_id();
        if (keys(wave)) {
            Frag k[KW];
            widen_keys<D>(rk.k[0], rk.s[0], magic, k);
#pragma unroll
            for (int i = 0; i < KW; ++i) out[(wave * KW + i) * kWave] = make_uint4(k[i].u[0], k[i].u[1], k[i].u[2], k[i].u[3]);
        }
        if (values(wave)) {
            const int pair = (wave & 3) >> 1, part = wave & 1, t = tok + 32 * pair + 4 * (lane_id() >> 4);
            if (edge || vok != 3) {
                rv.s[0] = cover(rv.s[0], t, all.lo, all.hi, vok & 1);
                rv.s[1] = cover(rv.s[1], t + 16, all.lo, all.hi, vok & 2);
            }
            uint4* v = out + kStageHalf<D> / 16 + (pair * MO + part * (MO / 2)) * kWave;
            widen_values<D>(rv, 0, MO / 4, part * (MO / 4), magic, [&](int i, const Frag& f) { v[i * kWave] = make_uint4(f.u[0], f.u[1], f.u[2], f.u[3]); });
        }
    }
};

// 64 staged tokens from t on
template <int D, int RT>
__device__ __forceinline__ void multiply_staged(State<D, RT>& st, const char* buf, int t, bool edge, uint32_t ok) {
    constexpr int KW = D / 32, MO = D / 16;
    const uint4* in = reinterpret_cast<const uint4*>(buf) + lane_id();
    f4_t s[4][RT];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        Frag k[KW];
#pragma unroll
        for (int i = 0; i < KW; ++i) {
            const uint4 x = in[(n * KW + i) * kWave];
            k[i].u[0] = x.x, k[i].u[1] = x.y, k[i].u[2] = x.z, k[i].u[3] = x.w;
        }
        scores<D, RT>(st, k, s[n]);
    }
    if (edge) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int r = 0; r < RT; ++r) hide<D, RT>(st, r, t + 16 * n, (ok >> n) & 1, s[n][r]);
    }
    Frag p[RT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r)
        {
            raise<D, RT, 4>(st, r, s);
#pragma unroll
            for (int u = 0; u < 2; ++u) p[r][u] = probabilities<D, RT>(st, r, s[2 * u][r], s[2 * u + 1][r]);
        }
    const uint4* v = in + kStageHalf<D> / 16;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
            add_ones<D, RT>(st, r, p[r][u]);
#pragma unroll
        for (int i = 0; i < MO; ++i) {
            const uint4 x = v[(u * MO + i) * kWave];
            Frag f;
            f.u[0] = x.x, f.u[1] = x.y, f.u[2] = x.z, f.u[3] = x.w;
#pragma unroll
            for (int r = 0; r < RT; ++r)
                st.o[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.v, p[r][u].v, st.o[r][i], 0, 0, 0);
        }
    }
}

// channel of product tile i, element e of a lane's accumulator: the lane's value octet is 4 quarter + e of the 16 in a tile
template <int D>
__device__ __forceinline__ int first_channel(int quarter, int e) {
    const int o = 4 * quarter + e;
    return D == 64 ? 8 * (o & 7) + 4 * (o >> 3) : 8 * o;
}

// N channels of one finished row
template <int N>
__device__ __forceinline__ void store_row(const Kv4AttnArgs& a, const Work& w, int row, int d, const float* x) {
    const int i = over_group(a, row), g = row - i * a.G;
    uint16_t* p = a.out + ((int64_t)(w.span.first + i) * a.H + w.head * a.G + g) * a.p.D + d;
    uint32_t o[N / 2];
#pragma unroll
    for (int j = 0; j < N / 2; ++j) o[j] = round16(x[2 * j], x[2 * j + 1], a.dt);
    if constexpr (N == 8) *reinterpret_cast<uint4*>(p) = make_uint4(o[0], o[1], o[2], o[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(o[0], o[1]);
}
__device__ __forceinline__ void store_lse(const Kv4AttnArgs& a, const Work& w, int row, float m, float l) {
    if (!a.lse) return;
    const int i = over_group(a, row), g = row - i * a.G;
    a.lse[(int64_t)(w.span.first + i) * a.H + w.head * a.G + g] =
        l == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l) - kShift) * 0.69314718055994531f;
}

// A partial result: [row][D] sums, then [row] (maximum, sum of probabilities), through the device's coherence point.
template <int D>
struct Partial {
    __amdgpu_buffer_rsrc_t r;
    uint32_t base, ml;  // bytes
    __device__ __forceinline__ Partial(const Kv4AttnArgs& a, int slot)
        : r(make_raw_buffer(a.partial, a.partial_bytes)),
          base((uint32_t)(slot * a.slot_floats * 4)),
          ml(base + (uint32_t)(a.slot_floats / (D + 2) * D * 4)) {}
    __device__ __forceinline__ void put(int row, int d, float4 v) const { store_coherent16(r, base + (row * D + d) * 4, v); }
    __device__ __forceinline__ void put_ml(int row, float m, float l) const { store_coherent8(r, ml + row * 8, make_float2(m, l)); }
};

}  // namespace

template <int D, int RT, int WAVES, bool STAGED>
__global__ __launch_bounds__(WAVES * kWave, RT == 1 ? kOcc1 : kOcc2) void kv4_attention_kernel(Kv4AttnArgs a) {
    constexpr int ROWS = 16 * RT, THREADS = WAVES * kWave;
    constexpr int LD = D + 4;             // a row of the joining buffer: 4 words more spread 16 rows over all banks
    constexpr int CH = D / 16;            // channels of a lane that lie together
    constexpr int V4 = D / 4;
    constexpr int JOIN = WAVES * 16 * LD / 4, STAGE = STAGED ? 4 * kStageHalf<D> / 16 : 0;
    __shared__ float4 s_buf[JOIN > STAGE ? JOIN : STAGE];  // what is staged, then what is joined
    __shared__ float2 s_ml[WAVES * 16];
    __shared__ int s_last;
    float* s_o = reinterpret_cast<float*>(s_buf);  // [WAVES][16][LD]
    Work w;
    if (!find_work<RT, WAVES, STAGED>(a, w)) return;
    const int wave = uniform(threadIdx.x / kWave), lane = lane_id(), lo16 = lane & 15, quarter = lane >> 4;
    uint32_t magic = 0x54005400u;
    asm volatile("" : "+v"(magic));  // in a vector register: an instruction takes one scalar operand

    const int first = w.split ? w.block * ROWS : (w.block * WAVES + wave) * ROWS;
    const Rows rows = rows_of(a, w.span, first, ROWS);
    const int nrt = (rows.n + 15) >> 4;
    // the workgroup's tokens: an equal part of what its rows see, in whole tiles
    constexpr int TILE = kTile;
    const Rows all = w.split ? rows : rows_of(a, w.span, w.block * WAVES * ROWS, WAVES * ROWS);
    const int granule = w.split ? TILE : kWide;
    const int t_lo = all.lo & ~(granule - 1);
    const int tiles = all.hi > t_lo ? (all.hi - t_lo + granule - 1) / granule : 0;
    const int per = w.chunks == 1 ? tiles : (tiles + w.chunks - 1) / w.chunks;
    const int c0 = min(w.chunk * per, tiles), c1 = min(c0 + per, tiles);
    const int32_t* row_table = a.s.table + (int64_t)w.b * a.s.S;
    const char* head_base = kv4_block(a.p, a.layer, 0, w.head);
    const int Pm = a.p.P - 1;
    const Places<D> at;
    const auto block_of = [&](uint32_t page) { return head_base + ((uint64_t)(page == kNoPage ? 0 : page) << 4); };
    State<D, RT> st;
    const auto begin = [&]() {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = first + 16 * r + lo16;
            const bool live = row < first + rows.n;
            float back = 1.f;
            load_queries<D>(a, w, row, live, st.q[r], back);
            st.a[r] = a.scale * back;
            const Rows mine = rows_of(a, w.span, live ? row : 0, live ? 1 : 0);
            st.lo[r] = mine.lo, st.hi[r] = mine.hi;
            st.m[r] = st.past[r] = kNone;
            st.w[r] = st.a[r], st.base[r] = kShift - kNone;
            st.l[r] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < D / 16; ++i) st.o[r][i] = f4_t{0.f, 0.f, 0.f, 0.f};
        }

    };
    if (!STAGED || w.split) {
        // every WAVES-th tile
        int t = t_lo + TILE * (c0 + wave);
        const int t_end = t_lo + TILE * c1, step = TILE * WAVES;
        const auto fetch_keys = [&](RawKeys<D>& r, int tok, uint32_t pg0, uint32_t pg1) {
            load_keys<D, RT == 1>(r, 0, block_of(pg0), tok & Pm, a.p.P, at);
            load_keys<D, RT == 1>(r, 1, block_of(pg1), (tok + 16) & Pm, a.p.P, at);
        };
        const auto fetch_values = [&](RawValues& r, int tok, uint32_t pg0, uint32_t pg1) {
            load_values<D, RT == 1>(r, 0, block_of(pg0), tok & Pm, a.p.P, at);
            load_values<D, RT == 1>(r, 1, block_of(pg1), (tok + 16) & Pm, a.p.P, at);
        };
        // One tile's words are held at a time: the keys' registers take the next tile's as soon as the scores are formed, the
        // values' when theirs are added.  The first words are asked for before the queries.
        RawKeys<D> rk;
        RawValues rv;
        const int t0 = t;
        Ahead pages(row_table, a.s.S, a.p, [=](int k) { return t0 + (k >> 1) * step + (k & 1) * 16; });
        uint32_t pg0 = pages[0], pg1 = pages[1], have = pages.template have<2>(0);
        if (t < t_end) {
            fetch_keys(rk, t, pg0, pg1);
            fetch_values(rv, t, pg0, pg1);
        }
        __builtin_amdgcn_sched_barrier(0);
        begin();
        for (int k = 0; t < t_end; k += 2) {
            const int tn = t + step;
            const bool more = tn < t_end;
            pages.reach(k + 2);
            const uint32_t n0 = pages[k + 2], n1 = pages[k + 3], next_have = pages.template have<2>(k + 2);
            f4_t s[2][RT];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                Frag k[D / 32];
                widen_keys<D>(rk.k[half], rk.s[half], magic, k);
                scores<D, RT>(st, k, s[half]);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (more) fetch_keys(rk, tn, n0, n1);
            if (!(t >= rows.lo_all && t + TILE <= rows.hi_all && have == 3)) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const bool ok = (have >> half) & 1;
                    const int th = t + 16 * half;
#pragma unroll
                    for (int r = 0; r < RT; ++r) hide<D, RT>(st, r, th, ok, s[half][r]);
                    rv.s[half] = cover(rv.s[half], th + 4 * quarter, rows.lo, rows.hi, ok);
                }
            }
            Frag p[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r)
                {
                    raise<D, RT, 2>(st, r, s);
                    p[r] = probabilities<D, RT>(st, r, s[0][r], s[1][r]);
                }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int r = 0; r < RT; ++r)
                add_ones<D, RT>(st, r, p[r]);
            widen_values<D>(rv, 0, D / 32, 0, magic, [&](int i, const Frag& v) {
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    st.o[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v.v, p[r].v, st.o[r][i], 0, 0, 0);
            });
            __builtin_amdgcn_sched_barrier(0);
            if (more) fetch_values(rv, tn, n0, n1);
            have = next_have;
            t = tn;
        }
    } else {
        char* stage = reinterpret_cast<char*>(s_buf);
        Stage<D, STAGED ? WAVES : kStagedWaves> sg;
        int t = t_lo + kWide * c0;
        const int t_end = t_lo + kWide * c1;
        const auto whole = [&](int tok) { return tok >= all.lo_all && tok + kWide <= all.hi_all; };
        const int t0 = t;
        Ahead pages(row_table, a.s.S, a.p, [=](int k) { return t0 + 16 * k; });
        uint32_t have = pages.template have<4>(0), next_have = pages.template have<4>(4);
        if (t < t_end) sg.fetch(wave, t, 0, a.p.P, pages, block_of, at);
        __builtin_amdgcn_sched_barrier(0);
        begin();
        if (t < t_end) {
            sg.widen_into(wave, stage, t, !whole(t), all, magic);
            if (t + kWide < t_end) sg.fetch(wave, t + kWide, 4, a.p.P, pages, block_of, at);
        }
        for (int k = 0; t < t_end; t += kWide, k += 4) {
            char* buf = stage + (k & 4) / 4 * (2 * kStageHalf<D>);
            char* other = stage + (~k & 4) / 4 * (2 * kStageHalf<D>);
            __syncthreads();  // staged by all, and the other buffer read by all
            pages.reach(k + 8);
            const int tn = t + kWide;
            if (tn < t_end) {
                sg.widen_into(wave, other, tn, !whole(tn), all, magic);
                if (tn + kWide < t_end) sg.fetch(wave, tn + kWide, k + 8, a.p.P, pages, block_of, at);
            }
            if (nrt > 0 && t < rows.hi && t + kWide > rows.lo) {
                multiply_staged<D, RT>(st, buf, t, !(t >= rows.lo_all && t + kWide <= rows.hi_all && have == 15), have);
            }
            have = next_have, next_have = pages.template have<4>(k + 8);
        }
    }

    const bool parts = w.chunks > 1;
    const Partial<D> part(a, parts ? w.slot : 0);
    if (STAGED && !w.split) {
        // rows of my own: finished, or a partial result of the chunk
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = first + 16 * r + lo16;
            if (r >= nrt || row >= first + rows.n) continue;
            const int in = wave * ROWS + 16 * r + lo16;
            const float l = st.l[r][0], f = parts ? 1.f : (l == 0.f ? 0.f : 1.f / l);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x[CH];
#pragma unroll
                for (int i = 0; i < CH; ++i) x[i] = st.o[r][i][e] * f;
                const int d = first_channel<D>(quarter, e);
                if (!parts) store_row<CH>(a, w, row, d, x);
                else
#pragma unroll
                    for (int i = 0; i < CH; i += 4) part.put(in, d + i, make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]));
            }
            if (quarter == 0) {
                if (!parts) store_lse(a, w, row, st.m[r], l);
                else part.put_ml(in, st.m[r], l);
            }
        }
    } else {
        // the same rows in all wavefronts: joined through LDS, 16 rows at a time
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            if (r >= nrt) break;
            if (16 * r + lo16 < rows.n) {
                if (quarter == 0) s_ml[wave * 16 + lo16] = make_float2(st.m[r], st.l[r][0]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float* p = s_o + (wave * 16 + lo16) * LD + first_channel<D>(quarter, e);
#pragma unroll
                    for (int i = 0; i < CH; ++i) p[i] = st.o[r][i][e];
                }
            }
            __syncthreads();
            for (int i = threadIdx.x; i < min(16, rows.n - 16 * r) * V4; i += THREADS) {
                const int in = i / V4, d = (i % V4) * 4, row = 16 * r + in;
                float m = kNone, l = 0.f;
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int v = 0; v < WAVES; ++v) m = fmaxf(m, s_ml[v * 16 + in].x);
#pragma unroll
                for (int v = 0; v < WAVES; ++v) {
                    const float2 ml = s_ml[v * 16 + in];
                    const float f = __builtin_amdgcn_exp2f(ml.x - m);
                    l += ml.y * f;
                    const float4 y = *reinterpret_cast<const float4*>(s_o + (v * 16 + in) * LD + d);
                    x.x += y.x * f, x.y += y.y * f, x.z += y.z * f, x.w += y.w * f;
                }
                if (!parts) {
                    const float g = l == 0.f ? 0.f : 1.f / l;
                    const float o[4] = {x.x * g, x.y * g, x.z * g, x.w * g};
                    store_row<4>(a, w, first + row, d, o);
                    if (d == 0) store_lse(a, w, first + row, m, l);
                } else {
                    part.put(row, d, x);
                    if (d == 0) part.put_ml(row, m, l);
                }
            }
            if (RT > 1) __syncthreads();
        }
    }
    if (!parts) return;

    // The last workgroup of the rows joins the chunks: a thread takes four channels of a row and every GROUPS-th chunk.
    wait_memory_ops();
    __syncthreads();
    if (threadIdx.x == 0)
        s_last = __hip_atomic_fetch_add(a.counters + w.counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == w.chunks - 1;
    __syncthreads();
    if (!s_last) return;
    if (threadIdx.x == 0) store_dev(a.counters + w.counter, 0);  // ready for the next call
    const Partial<D> p0(a, w.slot - w.chunk * a.p.heads);
    const uint32_t stride = (uint32_t)(a.slot_floats * 4 * a.p.heads);
    const int base_row = w.split ? first : w.block * WAVES * ROWS;
    const int items = all.n * V4;
    constexpr int FLY = 8;
    constexpr int PASS = THREADS;          // items of a pass
    for (int i0 = 0; i0 < items; i0 += PASS) {
        const int n = min(items - i0, PASS), groups = min(PASS / n, w.chunks);
        const int g = threadIdx.x / n, i = i0 + threadIdx.x % n;
        const int row = i / V4, d = (i % V4) * 4;
        float m = kNone, l = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (g < groups) {
            for (int c = g; c < w.chunks; c += FLY * groups) {
                float2 ml[FLY];
                float4 y[FLY];
#pragma unroll
                for (int u = 0; u < FLY; ++u) {
                    const int cu = min(c + u * groups, w.chunks - 1);
                    const uint32_t off = (uint32_t)cu * stride;
                    const auto t = __builtin_amdgcn_raw_buffer_load_b64(p0.r, (int)(p0.ml + off + row * 8), 0, kAuxDeviceCoherent);
                    ml[u] = make_float2(__uint_as_float(t[0]), __uint_as_float(t[1]));
                    y[u] = load_coherent16(p0.r, p0.base + off + (row * D + d) * 4);
                }
                float mm = m;
#pragma unroll
                for (int u = 0; u < FLY; ++u) {
                    if (c + u * groups >= w.chunks) ml[u] = make_float2(-__builtin_inff(), 0.f);
                    mm = fmaxf(mm, ml[u].x);
                }
                const float f = __builtin_amdgcn_exp2f(m - mm);
                m = mm;
                l *= f;
                x.x *= f, x.y *= f, x.z *= f, x.w *= f;
#pragma unroll
                for (int u = 0; u < FLY; ++u) {
                    const float h = __builtin_amdgcn_exp2f(ml[u].x - mm);
                    if (c + u * groups < w.chunks) {
                        l += ml[u].y * h;
                        x.x += y[u].x * h, x.y += y[u].y * h, x.z += y[u].z * h, x.w += y[u].w * h;
                    }
                }
            }
            s_buf[threadIdx.x] = x;
            s_buf[THREADS + threadIdx.x] = make_float4(m, l, 0.f, 0.f);
        }
        __syncthreads();
        if (g == 0) {
            for (int v = 1; v < groups; ++v) {
                const float4 y = s_buf[v * n + threadIdx.x], ml = s_buf[THREADS + v * n + threadIdx.x];
                const float mm = fmaxf(m, ml.x), f = __builtin_amdgcn_exp2f(m - mm), h = __builtin_amdgcn_exp2f(ml.x - mm);
                m = mm;
                l = l * f + ml.y * h;
                x.x = x.x * f + y.x * h, x.y = x.y * f + y.y * h, x.z = x.z * f + y.z * h, x.w = x.w * f + y.w * h;
            }
            const float k = l == 0.f ? 0.f : 1.f / l;
            const float o[4] = {x.x * k, x.y * k, x.z * k, x.w * k};
            store_row<4>(a, w, base_row + row, d, o);
            if (d == 0) store_lse(a, w, base_row + row, m, l);
        }
        __syncthreads();
    }
}

namespace {

template <int D, int RT, int WAVES, bool STAGED>
int launch(const Kv4AttnArgs& a, const Kv4AttnPlan& plan, hipStream_t stream) {
    kv4_attention_kernel<D, RT, WAVES, STAGED><<<(uint32_t)plan.grid, WAVES * kWave, 0, stream>>>(a);
    return hipGetLastError() == hipSuccess ? SCAP_OK : SCAP_ERR_HIP;
}

template <int D>
int launch_of(const Kv4AttnArgs& a, const Kv4AttnPlan& plan, hipStream_t stream) {
    if (plan.rt == 1) return plan.waves == 8 ? launch<D, 1, 8, false>(a, plan, stream) : launch<D, 1, 4, false>(a, plan, stream);
    if (plan.staged) return launch<D, 2, kStagedWaves, true>(a, plan, stream);
    return plan.waves == 8 ? launch<D, 2, 8, false>(a, plan, stream) : launch<D, 2, 4, false>(a, plan, stream);
}

}  // namespace

// One row tile: wavefronts of a workgroup.  Eight where few row sets (sequences times kv heads) are cut into many chunks, since half as many
// partial results are joined; four where sets are many, since chunks that fill the chip evenly are easier to find.  us, eight / four:
// 8 sets of 16000 tokens 19.9 / 29.7, 32 of 4096 18.5 / 24.1, 64 of 4096 19.6 / 21.2, 128 of 16000 69.8 / 69.8; 192 of 16000 108 / 101, ragged
// 64.5 / 57.6; 384 ragged to 4096 47.7 / 34.3, 768 of 1000 36.9 / 30.2, 2048 of 1000 79.5 / 70.5.  What that leaves: 256 ragged to 1000
// 16.6 / 18.2, 512 of 1000 24.8 / 27.8, of 4096 64.4 / 67.2.
constexpr int64_t kFewSets1 = 192;
// The same for two row tiles that split tokens, by heads times blocks of 32 rows: 8 heads x 16 sequences x 64 rows of 2000 tokens 28.9 / 34.5, 4 x 4 x
// 384 26.6 / 34.4, 8 x 4 x 256 of 16000 135 / 142; beyond 4 x 16 x 256 of 2000 53.0 / 42.7, 32 x 4 x 128 50.3 / 41.0, 8 x 16 x 256 98.3 / 79.7.
constexpr int64_t kFewSets2 = 400;

// Two row tiles: blocks of 32 rows whose tokens the wavefronts split, or, from so many rows of all heads on, blocks of 256 that share what is
// staged.  The latter do less work, but where they are few they are cut into chunks whose partial results of 256 rows one workgroup
// joins.  us, blocks of 32 / of 256 rows (heads x sequences x rows, tokens): 128 channels, 8 x 1 x 128, 2000 19 / 40; 8 x 4 x 256, 2000
// 29 / 79, 16000 135 / 155; 8 x 16 x 256, 2000 100 / 119; beyond 8 x 16 x 384, 2000 143 / 97; 32 x 16 x 128, 2000 198 / 151; 64 channels, 8 x
// 4 x 128, 2000 19 / 26, 16000 53 / 57; beyond 8 x 16 x 128, 2000 41 / 42, x 256 75 / 62.  What that leaves, long contexts of few rows: 128
// channels 8 x 4 x 384, 16000 237 / 213, 4 x 16 x 192, 16000 242 / 206; 64 channels 8 x 4 x 384, 16000 171 / 128.
static bool staged_pays(int D, int64_t rows_of_all_heads) { return rows_of_all_heads > (D == 64 ? 12287 : 32768); }

// floats of a partial result: sums, maximum and sum of the probabilities of an even number of rows
static int64_t slot_floats(int D, int64_t rows) { return (rows + 1) / 2 * 2 * (D + 2); }

Kv4AttnPlan plan_kv4_attention(int D, int kv_heads, int64_t B, int64_t T, int G, int64_t max_new) {
    Kv4AttnPlan p;
    const int64_t most = (max_new < T ? max_new : T) * G;  // rows of a sequence, if the caller's max_new holds
    p.rt = most <= 16 ? 1 : 2;
    const int64_t rows = 16 * p.rt;
    const bool staged = p.rt == 2 && staged_pays(D, T * G * kv_heads);
    p.staged = staged;
    p.min_chunk = p.rt == 1 ? kMinChunk1 : kMinChunk2;
    // Row blocks of all sequences, at most: one each, and one more per 256 rows (staged; two each up to 64 rows) or per wavefront's rows.
    // What the chunks add to them, and what room they need: scap_kv4_split.hpp.
    const int64_t block_rows = staged ? kStagedWaves * rows : rows;
    const int64_t blocks = (staged ? 2 * B : B) + T * G / block_rows;
    p.waves = staged ? kStagedWaves : (p.rt == 1 ? B * kv_heads < kFewSets1 : blocks * kv_heads <= kFewSets2) ? 8 : 4;
    p.places = kUnits * 4 * (p.rt == 1 ? kOcc1 : kOcc2) / p.waves / kv_heads;
    if (p.places < 1) p.places = 1;
    p.grid = (blocks + p.places + 2) * kv_heads;
    p.slot_rows = (int)(most <= rows ? most : T * G);
    p.slot_floats = slot_floats(D, p.slot_rows < block_rows ? p.slot_rows : block_rows);
    return p;
}

size_t kv4_partial_bytes(int D, int kv_heads, int64_t T, int G, int64_t max_new) {
    // of every plan that a call of up to T tokens may get
    const int64_t most = (max_new < T ? max_new : T) * G;
    size_t need = 0;
    const auto take = [&](int waves_at_once, int least_waves, int64_t rows, int64_t limit) {
        const int64_t places = waves_at_once / least_waves / kv_heads;
        if (places <= 1) return;  // nothing is cut
        const size_t n = 2 * (size_t)(places + 2) * kv_heads * slot_floats(D, rows < limit ? rows : limit) * 4;
        if (n > need) need = n;
    };
    take(kUnits * 4 * kOcc1, 4, 16, most);
    if (most > 16) {
        take(kUnits * 4 * kOcc2, 4, 32, T * G);
        if (staged_pays(D, T * G * kv_heads)) take(kUnits * 4 * kOcc2, kStagedWaves, kStagedWaves * 32, T * G);
    }
    return need;
}

int launch_kv4_attention(const Kv4AttnArgs& a, const Kv4AttnPlan& plan, hipStream_t stream) {
    return a.p.D == 64 ? launch_of<64>(a, plan, stream) : launch_of<128>(a, plan, stream);
}

}  // namespace scap
