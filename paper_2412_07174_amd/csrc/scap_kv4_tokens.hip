// Filling the 4-bit cache (append) and reading it back.  Both move a token of one kv head with D/8 lanes per vector, 16 bytes a lane: a group
// of 32 channels is four neighbouring lanes, whose minimum and maximum take two lane permutations each.  Bound by instructions and latency:
// 12297 tokens of 8 heads of 128 channels 19.6 us in (2.6 + 0.8 TB/s), 15 us out; 16 tokens 3.3 us in, 2.9 out, three trips to memory.
#include "scap_kv4.hpp"

namespace scap {

namespace {

constexpr int kThreads = 256;

struct Place {
    int page;  // -1: nowhere
    int slot;
};

// Where tokens t0 .. t0 + NT - 1 of the call lie: 64 sequences are compared at a time, and the lane that finds a token among its own
// knows the position.  Wavefront-uniform.
template <int NT>
__device__ __forceinline__ void find_places(const Kv4Pool& p, const Kv4Seqs& s, int t0, Place (&at)[NT]) {
    int row[NT], pos[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) row[j] = -1, pos[j] = 0;
    for (int base = 0; base < s.B; base += kWave) {
        const int b = base + lane_id();
        int first = 0, end = 0, len = 0;
        if (b < s.B) first = s.starts[b], end = s.starts[b + 1], len = s.lens[b];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int t = t0 + j;
            const uint64_t mine = __ballot(first <= t && t < end && t < s.T);
            if (mine != 0) {
                const int l = __builtin_ctzll(mine);
                row[j] = base + l;
                pos[j] = __builtin_amdgcn_readlane(len - end, l) + t;
            }
        }
    }
    int entry[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const bool has = row[j] >= 0 && pos[j] >= 0 && (int64_t)pos[j] < (int64_t)s.S * p.P;
        entry[j] = has ? s.table[(int64_t)row[j] * s.S + (pos[j] >> p.lgP)] : -1;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int e = uniform(entry[j]);
        at[j] = {(uint32_t)e < (uint64_t)p.pages ? e : -1, pos[j] & (p.P - 1)};
    }
}

// A unit's place in a page: 32-bit offsets of its lanes' words in the parts of its block, to which a token adds a scalar.
template <int D>
struct UnitPlace {
    uint32_t codes, scales;
    bool is_v;
    __device__ __forceinline__ UnitPlace(const Kv4Pool& p, int unit, bool is_v, int o) : is_v(is_v) {
        const Kv4Layout L = {D, p.P};
        const uint32_t block = (uint32_t)unit * (uint32_t)L.bytes();  // a page has less than 2^32 bytes
        codes = block + (is_v ? (uint32_t)L.vcodes() + 16u * o : 4u * o);
        scales = block + (is_v ? (uint32_t)L.vscales() + 16u * (o >> 2) : (uint32_t)L.kscales() + 4u * (o >> 2));
    }
    __device__ __forceinline__ uint32_t codes_of(int slot) const {
        return codes + (is_v ? (uint32_t)((slot >> 2) * (2 * D) + (slot & 3) * 4) : (uint32_t)(slot * (D / 2)));
    }
    __device__ __forceinline__ uint32_t scales_of(int slot) const {
        return scales + (is_v ? (uint32_t)((slot >> 2) * (D / 2) + (slot & 3) * 2) : (uint32_t)(slot * (D / 8)));
    }
};

// 8 inputs from a 2-byte aligned address that nobody reads again (non-temporal: 37.3 -> 35.5 us for 12297 tokens in and out)
__device__ __forceinline__ uint4 load_octet_once(const uint16_t* p) {
    typedef uint32_t vec_t __attribute__((ext_vector_type(4), aligned(2)));
    const vec_t t = __builtin_nontemporal_load(reinterpret_cast<const vec_t*>(p));
    return make_uint4(t.x, t.y, t.z, t.w);
}

// over the four lanes that hold a group, NaN if any is (the maximum and minimum of IEEE 754-2019)
template <bool MAX>
__device__ __forceinline__ float over_group(float v) {
    const auto with = [&](float o) { return MAX ? __builtin_elementwise_maximum(v, o) : __builtin_elementwise_minimum(v, o); };
    v = with(__int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xB1, 0xF, 0xF, true)));  // quad_perm 1 0 3 2
    v = with(__int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4E, 0xF, 0xF, true)));  // quad_perm 2 3 0 1
    return v;
}

// An fp32 result, rounded to fp16.  It stays one of fp32 first: the compiler would round an fma once, straight to fp16, which is another number where
// the two roundings meet in a tie (15.5 of fp16's smallest, an exact quotient of two bf16 values, say).
__device__ __forceinline__ uint32_t f16_bits(float f) {
    asm("" : "+v"(f));
    const _Float16 h = (_Float16)f;
    return __builtin_bit_cast(uint16_t, h);
}

__device__ __forceinline__ _Float16 f16_of(uint32_t bits) { return __builtin_bit_cast(_Float16, (uint16_t)bits); }

__device__ __forceinline__ void widen_octet(const uint4& raw, int dt, float (&x)[8]) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (dt == kBF16) {
            x[2 * j] = __uint_as_float(w[j] << 16), x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        } else {
            x[2 * j] = f16_bits_to_f32(w[j] & 0xFFFFu), x[2 * j + 1] = f16_bits_to_f32(w[j] >> 16);
        }
    }
}

// One octet of a group of 32 channels that four neighbouring lanes hold: its word of codes, and the group's scales.
// The quotient (x - c) / s is the one that an IEEE division gives: r = RN(1 / s), and one step from the exact residual.  Clamped to
// 64 .. 79, an addend whose last place is 1 rounds it to the nearest even integer and leaves q in the low 16 bits of the sum.
// About 10 instructions a value: 1.5 * 2^23 + 2^16 - 64 below takes the place of rounding, subtracting, converting and masking.
__device__ __forceinline__ uint32_t quantise(const uint4& raw, int dt, uint32_t& scales, bool& bad) {
    float x[8];
    widen_octet(raw, dt, x);
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) lo = __builtin_elementwise_minimum(lo, x[j]), hi = __builtin_elementwise_maximum(hi, x[j]);
    lo = over_group<false>(lo);
    hi = over_group<true>(hi);
    // (hi - lo) / 15, correctly rounded: a product, and one step from its exact residual.  No number where x has an infinity or a NaN
    const float range = hi - lo, r15 = 1.f / 15.f, q15 = range * r15;
    const uint32_t sb = f16_bits(fmaf(fmaf(-q15, 15.f, range), r15, q15));
    const float s = f16_bits_to_f32(sb);
    const uint32_t cb = f16_bits(lo - kKv4Bias * s);
    const float c = f16_bits_to_f32(cb);
    // What the largest code stands for, as attention forms it: no number of fp16 where that is none, nor where s or c is (an infinite s
    // makes c infinite with the other sign).  No code stands for less than c, so an infinity can only be this one.
    const _Float16 top = __builtin_elementwise_fma((_Float16)(kKv4Bias + 15.f), f16_of(sb), f16_of(cb));
    bad = (__builtin_bit_cast(uint16_t, top) & 0x7C00u) == 0x7C00u;
    scales = sb | (cb << 16);
    // 1 / s correctly rounded: one step from the hardware's, whose error it squares to 2^-46, and no quotient of an 11-bit s lies within
    // 2^-36 of the middle between two floats
    const float r0 = __builtin_amdgcn_rcpf(s), r = s == 0.f ? 0.f : fmaf(fmaf(-s, r0, 1.f), r0, r0);
    uint32_t u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float d = x[j] - c;
        float q = d * r;
        q = fmaf(fmaf(-q, s, d), r, q);
        q = __builtin_amdgcn_fmed3f(q, kKv4Bias, kKv4Bias + 15.f);
        u[j] = __float_as_uint(q + (12582912.f + 65536.f - kKv4Bias));
    }
    // (bits above the 16 low ones fall out with the last step)
    uint32_t n[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) n[j] = (u[2 * j + 1] << 4) | u[2 * j];
    return __builtin_amdgcn_perm((n[3] << 8) | n[2], (n[1] << 8) | n[0], 0x05040100u);
}

}  // namespace

// NT tokens from NT * blockIdx.x on; blockIdx.y: slices of their heads.  A unit of 2 * D/8 lanes holds a head's key (lower half) and value.  The
// inputs are asked for before their places are known: a workgroup is two memory trips long, not four.
template <int D, int NT>
__global__ __launch_bounds__(kThreads) void kv4_append_kernel(Kv4TokensArgs a) {
    constexpr int LPV = D / 8;        // lanes per vector
    constexpr int LPU = 2 * LPV;      // lanes per unit
    const int t0 = blockIdx.x * NT;
    const int unit = blockIdx.y * (kThreads / LPU) + threadIdx.x / LPU;
    const int lane = threadIdx.x % LPU;
    const bool is_v = lane >= LPV;
    const int o = lane % LPV;  // octet
    const bool live = unit < a.p.heads;
    const int64_t st = is_v ? a.v_st : a.k_st;
    const uint16_t* in = (is_v ? a.v + unit * a.v_sh : a.k + unit * a.k_sh) + 8 * o;
    uint4 raw[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) raw[j] = live && t0 + j < a.s.T ? load_octet_once(in + (t0 + j) * st) : make_uint4(0, 0, 0, 0);
    Place at[NT];
    find_places<NT>(a.p, a.s, t0, at);
    const UnitPlace<D> mine(a.p, unit, is_v, o);
    const uint64_t mask = (LPU == 64 ? ~0ull : ((1ull << LPU) - 1)) << (lane_id() / LPU * LPU);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        uint32_t scales;
        bool bad;
        uint32_t codes = quantise(raw[j], a.dt, scales, bad);
        // one unreadable group makes the token unreadable for this head
        if ((__ballot(bad) & mask) != 0) codes = 0, scales = kKv4BadScale;
        if (!live || at[j].page < 0) continue;
        char* page = const_cast<char*>(kv4_block(a.p, a.layer, at[j].page, 0));
        *reinterpret_cast<uint32_t*>(page + mine.codes_of(at[j].slot)) = codes;
        if ((o & 3) == 0) {
            char* sc = page + mine.scales_of(at[j].slot);
            if (!is_v) {
                *reinterpret_cast<uint32_t*>(sc) = scales;
            } else {
                *reinterpret_cast<uint16_t*>(sc) = (uint16_t)scales;
                *reinterpret_cast<uint16_t*>(sc + 8) = (uint16_t)(scales >> 16);
            }
        }
    }
}

template <int D, int NT>
__global__ __launch_bounds__(kThreads) void kv4_read_kernel(Kv4TokensArgs a) {
    constexpr int LPV = D / 8, LPU = 2 * LPV;
    const int t0 = blockIdx.x * NT;
    const int unit = blockIdx.y * (kThreads / LPU) + threadIdx.x / LPU;
    Place at[NT];
    find_places<NT>(a.p, a.s, t0, at);
    if (unit >= a.p.heads) return;
    const int lane = threadIdx.x % LPU;
    const bool is_v = lane >= LPV;
    const int o = lane % LPV;
    const UnitPlace<D> mine(a.p, unit, is_v, o);
    uint32_t codes[NT], scales[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const char* page = kv4_block(a.p, a.layer, max(at[j].page, 0), 0);
        const char* sc = page + mine.scales_of(at[j].slot);
        codes[j] = *reinterpret_cast<const uint32_t*>(page + mine.codes_of(at[j].slot));
        // a key's s and c are one word; a value's lie 8 bytes apart
        scales[j] = *reinterpret_cast<const uint16_t*>(sc) | (uint32_t)*reinterpret_cast<const uint16_t*>(sc + (is_v ? 8 : 2)) << 16;
        if (at[j].page < 0) scales[j] = 0;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        if (t0 + j >= a.s.T) break;
        const float s = f16_bits_to_f32(scales[j] & 0xFFFFu), c = f16_bits_to_f32(scales[j] >> 16);
        // bytes 64 + q of the even and of the odd channels; s (q + 64) is exact in fp32: one rounding to the sum, one to the output's type
        const uint32_t even = (codes[j] & 0x0F0F0F0Fu) | 0x40404040u, odd = ((codes[j] >> 4) & 0x0F0F0F0Fu) | 0x40404040u;
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = round16(fmaf(s, (float)((even >> (8 * i)) & 0xFFu), c), fmaf(s, (float)((odd >> (8 * i)) & 0xFFu), c), a.dt);
        uint16_t* out = (is_v ? a.v_out : a.k_out) + ((int64_t)(t0 + j) * a.p.heads + unit) * D + 8 * o;
        *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

namespace {

// Tokens per workgroup: one while that leaves compute units idle, then four.
constexpr int kMany = 4, kManyFrom = 2048;
bool many(const Kv4TokensArgs& a) { return a.s.T >= kManyFrom; }

template <typename F>
int launch_tokens(const Kv4TokensArgs& a, int nt, hipStream_t stream, F kernel) {
    const int per = kThreads / (a.p.D / 4);  // heads a workgroup takes
    kernel<<<dim3((a.s.T + nt - 1) / nt, (a.p.heads + per - 1) / per), kThreads, 0, stream>>>(a);
    return hipGetLastError() == hipSuccess ? SCAP_OK : SCAP_ERR_HIP;
}

}  // namespace

int launch_kv4_append(const Kv4TokensArgs& a, hipStream_t stream) {
    if (many(a)) return launch_tokens(a, kMany, stream, a.p.D == 64 ? kv4_append_kernel<64, kMany> : kv4_append_kernel<128, kMany>);
    return launch_tokens(a, 1, stream, a.p.D == 64 ? kv4_append_kernel<64, 1> : kv4_append_kernel<128, 1>);
}

int launch_kv4_read(const Kv4TokensArgs& a, hipStream_t stream) {
    if (many(a)) return launch_tokens(a, kMany, stream, a.p.D == 64 ? kv4_read_kernel<64, kMany> : kv4_read_kernel<128, kMany>);
    return launch_tokens(a, 1, stream, a.p.D == 64 ? kv4_read_kernel<64, 1> : kv4_read_kernel<128, 1>);
}

}  // namespace scap
