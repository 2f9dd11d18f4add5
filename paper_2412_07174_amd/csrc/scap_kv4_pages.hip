// Pages of the 4-bit cache: allocation with copy on write, forking, freeing, compaction, copies.
//
// What a pool holds is described by refs[page] alone -- the number of table entries that name the page, 0 = free -- and an allocation takes
// the lowest free pages in the order of the call's sequences.  So no list lives between calls, every result is a function of the
// arguments, and a call can be recorded into a graph.  The price is one scan of refs per allocation, by one workgroup: 5 us for 8 rows and 128
// pages, 8 us for 128 rows and 1024 pages, most of it dependent trips to memory.  Copies run at 4-5 TB/s in and out (28 MB of shared last
// pages in 13 us, 44 MB to the front in 18).
#include "scap_kv4.hpp"

namespace scap {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kMaxSeqs = kKv4MaxReserve;
constexpr int kMissing = -2;  // a partly filled last page that the table does not name

// Sum over the workgroup of one number per wavefront, and the sum of those before mine.
__device__ __forceinline__ int wave_offsets(int* s_sum, int mine, int& total) {
    const int wave = uniform(threadIdx.x / kWave);
    __syncthreads();  // s_sum may still be read
    if (lane_id() == 0) s_sum[wave] = mine;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
        const int v = s_sum[w];
        before += w < wave ? v : 0;
        total += v;
    }
    return before;
}

// The pages are split into one contiguous run per wavefront: body(page, exists) for 64 pages at a time, whole wavefront.
template <typename F>
__device__ __forceinline__ void for_my_pages(int pages, F body) {
    const int wave = uniform(threadIdx.x / kWave);
    const int run = (pages + kPlanWaves * kWave - 1) / (kPlanWaves * kWave) * kWave;
    const int lo = wave * run, hi = min(pages, lo + run);
    for (int p = lo; p < hi; p += kWave) body(p + lane_id(), p + lane_id() < hi);
}

// scratch: [0] number of pairs; [64 ..) src, dst pairs; then the compaction's lists
struct Scratch {
    int32_t* count;
    int32_t* pairs;
    int32_t* map;
    int32_t* movers;
    int32_t* holes;
};
__host__ __device__ __forceinline__ Scratch carve(int32_t* s, int64_t pages) {
    // compaction: at most pages / 2 pairs, kept as two lists
    return {s, s + 64, s + 64, s + 64 + pages, s + 64 + 2 * pages};
}

}  // namespace

__global__ __launch_bounds__(kPlanThreads) void kv4_reserve_plan_kernel(Kv4Pool p, int32_t* table, int S, int B,
                                                                    const int32_t* __restrict__ old_lens,
                                                                    const int32_t* __restrict__ new_lens, int32_t* info,
                                                                    int32_t* scratch) {
    __shared__ int s_first[kMaxSeqs + 1];  // pages needed by the sequences before
    __shared__ int s_last[kMaxSeqs];       // the partly filled last page where others hold it too; kMissing; or -1
    __shared__ int s_sum[kPlanWaves];
    __shared__ int s_pairs, s_over;
    const int tid = threadIdx.x, P = p.P;
    const int64_t cap = (int64_t)S * P;
    if (tid == 0) s_pairs = 0, s_over = 0;
    __syncthreads();
    for (int b = tid; b < B; b += kPlanThreads) {
        const int o = max(old_lens[b], 0), n = new_lens[b];
        int32_t* row = table + (int64_t)b * S;
        // Pages past the old length (a block of drafted tokens that was cut, say) leave before any are taken: those up to the first slot that
        // names none, and all in slots that the new length takes.
        const int taken = n > o ? (n - 1) >> p.lgP : -1;
        constexpr int FLY = 4;
        bool more = true;
        for (int s = (int)(((int64_t)o + P - 1) >> p.lgP); s < S && more; s += FLY) {
            int32_t e[FLY];
#pragma unroll
            for (int u = 0; u < FLY; ++u) e[u] = s + u < S ? row[s + u] : -1;
#pragma unroll
            for (int u = 0; u < FLY; ++u) {
                more = more && (e[u] != -1 || s + u <= taken);
                if (!more || e[u] == -1) continue;
                if ((uint32_t)e[u] < (uint64_t)p.pages) atomicSub(&p.refs[e[u]], 1);
                row[s + u] = -1;
            }
        }
        if (n > cap) s_over = 1;
    }
    __syncthreads();
    for (int b = tid; b < B; b += kPlanThreads) {
        const int o = max(old_lens[b], 0), n = new_lens[b];
        int last = -1;
        if (n > o && n <= cap && (o & (P - 1))) {
            last = kv4_page(p, table + (int64_t)b * S, o >> p.lgP);
            if (last < 0) last = kMissing;
            else if (p.refs[last] < 2) last = -1;
        }
        s_last[b] = last;
    }
    __syncthreads();
    int running = 0;
    for (int base = 0; base < B; base += kPlanThreads) {
        const int b = base + tid;
        int need = 0;
        bool first = false;  // the old last page's slot takes one
        if (b < B) {
            const int o = max(old_lens[b], 0), n = new_lens[b];
            if (n > o && n <= cap) need = ((n - 1) >> p.lgP) - ((o - 1) >> p.lgP);  // (-1 >> lgP = -1: none before)
            const int last = s_last[b];
            if (last >= 0) {
                // holders of the same page before this one in the call have left it by then; the last holder keeps it
                int rank = 0;
                for (int i = 0; i < b; ++i) rank += s_last[i] == last;
                first = p.refs[last] - rank > 1;
            } else {
                first = last == kMissing;
            }
            need += first;
        }
        const int inc = wave_inclusive_scan(need);
        int total;
        const int before = wave_offsets(s_sum, __shfl(inc, kWave - 1, kWave), total);
        // the sign bit says so
        if (b < B) s_first[b] = (running + before + inc - need) | (first ? 1 << 31 : 0);
        running += total;
    }
    const int total = running;
    int mine = 0, n_free;
    for_my_pages((int)p.pages, [&](int page, bool exists) { mine += __popcll(__ballot(exists && p.refs[page] == 0)); });
    int k = wave_offsets(s_sum, mine, n_free);
    const bool over = s_over != 0;
    if (over || total > n_free) {
        if (tid == 0) {
            info[0] = over ? -1 : total - n_free;
            info[1] = info[2] = 0;
            info[3] = n_free;
            scratch[0] = 0;
        }
        return;
    }
    const Scratch sc = carve(scratch, p.pages);
    for_my_pages((int)p.pages, [&](int page, bool exists) {
        if (k >= total) return;  // uniform
        const uint64_t set = __ballot(exists && p.refs[page] == 0);
        const int i = k + lanes_below(set);
        k += __popcll(set);
        if (!((set >> lane_id()) & 1) || i >= total) return;
        int lo = 0, hi = B - 1;  // the last sequence whose first page is not past i
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if ((s_first[mid] & 0x7FFFFFFF) <= i) lo = mid;
            else hi = mid - 1;
        }
        const int b = lo, f = s_first[b];
        int j = i - (f & 0x7FFFFFFF);
        const int o = max(old_lens[b], 0);
        int slot;
        if (f < 0 && j == 0) {
            slot = o >> p.lgP;
            const int from = s_last[b];
            if (from >= 0) {
                atomicSub(&p.refs[from], 1);  // others hold it too: never to 0
                const int at = atomicAdd(&s_pairs, 1);
                sc.pairs[2 * at] = from;
                sc.pairs[2 * at + 1] = page;
            }
        } else {
            slot = ((o - 1) >> p.lgP) + 1 + j - (f < 0);
        }
        table[(int64_t)b * S + slot] = page;
        p.refs[page] = 1;
    });
    __syncthreads();
    if (tid == 0) {
        info[0] = 0;
        info[1] = total;
        info[2] = s_pairs;
        info[3] = n_free - total;
        scratch[0] = s_pairs;
    }
}

namespace {

// Copies of pages, all layers: a task is kPiece bytes of one page of one layer.
constexpr int kCopyThreads = 256;
constexpr int kPiece = kCopyThreads * 16 * 4;

__device__ __forceinline__ void copy_piece(const char* src, char* dst, int64_t at, int64_t bytes) {
    const int64_t i0 = at + threadIdx.x * 16;
    uint4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (i0 + u * kCopyThreads * 16 < bytes) v[u] = load_weights16(src + i0 + u * kCopyThreads * 16);
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (i0 + u * kCopyThreads * 16 < bytes) *reinterpret_cast<uint4*>(dst + i0 + u * kCopyThreads * 16) = v[u];
}

// Page src(i) of `from` to page dst(i) of `to` for i < n.
template <typename SRC, typename DST>
__device__ __forceinline__ void copy_pages(const Kv4Pool& from, const Kv4Pool& to, int64_t n, SRC src, DST dst) {
    const int64_t page = from.page_bytes();
    const int pieces = (int)((page + kPiece - 1) / kPiece);
    const int64_t tasks = n * from.layers * pieces;
    for (int64_t t = blockIdx.x; t < tasks; t += gridDim.x) {
        const int piece = (int)(t % pieces);
        const int64_t rest = t / pieces;
        const int layer = (int)(rest % from.layers);
        const int64_t i = rest / from.layers;
        const int64_t s = src(i), d = dst(i);
        if ((uint64_t)s >= (uint64_t)from.pages || (uint64_t)d >= (uint64_t)to.pages) continue;
        copy_piece(from.pool + (layer * from.pages + s) * page, to.pool + (layer * to.pages + d) * page,
                   (int64_t)piece * kPiece, page);
    }
}

}  // namespace

__global__ __launch_bounds__(kCopyThreads) void kv4_copy_on_write_kernel(Kv4Pool p, int32_t* scratch) {
    const Scratch sc = carve(scratch, p.pages);
    copy_pages(p, p, sc.count[0], [&](int64_t i) { return sc.pairs[2 * i]; }, [&](int64_t i) { return sc.pairs[2 * i + 1]; });
}

__global__ __launch_bounds__(kCopyThreads) void kv4_copy_pages_kernel(Kv4Pool from, Kv4Pool to, const int32_t* src,
                                                                  const int32_t* dst, int64_t n) {
    copy_pages(from, to, n, [&](int64_t i) { return src[i]; }, [&](int64_t i) { return dst[i]; });
}

__global__ __launch_bounds__(kPlanThreads) void kv4_compact_plan_kernel(Kv4Pool p, int32_t* refs_out, int32_t* info,
                                                                    int32_t* scratch) {
    __shared__ int s_sum[kPlanWaves];
    const Scratch sc = carve(scratch, p.pages);
    const int pages = (int)p.pages, tid = threadIdx.x;
    int mine = 0, live;
    for_my_pages(pages, [&](int page, bool exists) { mine += __popcll(__ballot(exists && p.refs[page] > 0)); });
    wave_offsets(s_sum, mine, live);
    int holes = 0, movers = 0, moved, unused;
    for_my_pages(pages, [&](int page, bool exists) {
        const bool held = exists && p.refs[page] > 0;
        holes += __popcll(__ballot(exists && !held && page < live));
        movers += __popcll(__ballot(held && page >= live));
    });
    holes = wave_offsets(s_sum, holes, unused);
    movers = wave_offsets(s_sum, movers, moved);
    for_my_pages(pages, [&](int page, bool exists) {
        const int r = exists ? p.refs[page] : 0;
        const uint64_t hole = __ballot(exists && r <= 0 && page < live), mover = __ballot(r > 0 && page >= live);
        if ((hole >> lane_id()) & 1) sc.holes[holes + lanes_below(hole)] = page;
        if ((mover >> lane_id()) & 1) sc.movers[movers + lanes_below(mover)] = page;
        else if (exists) sc.map[page] = page;
        holes += __popcll(hole);
        movers += __popcll(mover);
        if (exists && refs_out != p.refs) refs_out[page] = r;
    });
    __syncthreads();  // one workgroup: its own stores are visible to it behind the barrier
    for (int i = tid; i < moved; i += kPlanThreads) {
        const int from = sc.movers[i], to = sc.holes[i];
        sc.map[from] = to;
        refs_out[to] = p.refs[from];
        refs_out[from] = 0;
    }
    if (tid == 0) {
        info[0] = live;
        info[1] = moved;
        info[2] = info[3] = 0;
        scratch[0] = moved;
    }
}

__global__ __launch_bounds__(kCopyThreads) void kv4_compact_move_kernel(Kv4Pool p, const int32_t* table, int64_t entries,
                                                                    int32_t* table_out, int32_t* scratch) {
    const Scratch sc = carve(scratch, p.pages);
    const int64_t n = sc.count[0];
    for (int64_t i = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; i < entries; i += (int64_t)gridDim.x * kCopyThreads) {
        const int e = table[i];
        table_out[i] = (uint32_t)e < (uint64_t)p.pages ? sc.map[e] : e;
    }
    copy_pages(p, p, n, [&](int64_t i) { return sc.movers[i]; }, [&](int64_t i) { return sc.holes[i]; });
}

__global__ __launch_bounds__(256) void kv4_fork_kernel(Kv4Pool p, const int32_t* table, const int32_t* lens, int B_in,
                                                   const int32_t* parents, int32_t* table_out, int32_t* lens_out, int S) {
    const int per = (S + 255) / 256, row = blockIdx.x / per, s = blockIdx.x % per * 256 + threadIdx.x;
    const int from = parents[row];
    const bool has = (uint32_t)from < (uint32_t)B_in;
    const int len = has ? max(lens[from], 0) : 0;
    if (s == 0) lens_out[row] = len;
    if (s >= S) return;
    const int used = (int)(((int64_t)len + p.P - 1) >> p.lgP);
    int e = -1;
    if (s < used) {
        e = kv4_page(p, table + (int64_t)from * S, s);
        if (e >= 0) atomicAdd(&p.refs[e], 1);
    }
    table_out[(int64_t)row * S + s] = e;
}

__global__ __launch_bounds__(256) void kv4_free_kernel(Kv4Pool p, int32_t* table, int S, const int32_t* keep_from,
                                                   const int32_t* keep_to) {
    const int per = (S + 255) / 256, row = blockIdx.x / per, s = blockIdx.x % per * 256 + threadIdx.x;
    if (s >= S) return;
    // a first token alone keeps all from there on
    const int64_t from = keep_from ? keep_from[row] : 0, to = keep_to ? keep_to[row] : keep_from ? (int64_t)S << p.lgP : 0;
    const int64_t at = (int64_t)s << p.lgP;
    if (from < to && at < to && at + p.P > from) return;  // holds a kept token
    const int64_t i = (int64_t)row * S + s;
    const int e = table[i];
    if (e == -1) return;
    table[i] = -1;
    if ((uint32_t)e < (uint64_t)p.pages) atomicSub(&p.refs[e], 1);
}

namespace {

int done() { return hipGetLastError() == hipSuccess ? SCAP_OK : SCAP_ERR_HIP; }

constexpr int kCopyGroups = 2048;

}  // namespace

int launch_kv4_reserve(const Kv4Pool& p, int32_t* table, int S, int B, const int32_t* old_lens, const int32_t* new_lens,
                       int32_t* info, int32_t* scratch, hipStream_t stream) {
    kv4_reserve_plan_kernel<<<1, kPlanThreads, 0, stream>>>(p, table, S, B, old_lens, new_lens, info, scratch);
    const int64_t most = (int64_t)B * p.layers * ((p.page_bytes() + kPiece - 1) / kPiece);
    kv4_copy_on_write_kernel<<<(int)(most < kCopyGroups ? most : kCopyGroups), kCopyThreads, 0, stream>>>(p, scratch);
    return done();
}

int launch_kv4_fork(const Kv4Pool& p, const int32_t* table, const int32_t* lens, int B_in, const int32_t* parents, int B_out,
                    int32_t* table_out, int32_t* lens_out, int S, hipStream_t stream) {
    kv4_fork_kernel<<<(S + 255) / 256 * B_out, 256, 0, stream>>>(p, table, lens, B_in, parents, table_out, lens_out, S);
    return done();
}

int launch_kv4_free(const Kv4Pool& p, int32_t* table, int S, int B, const int32_t* keep_from, const int32_t* keep_to,
                    hipStream_t stream) {
    kv4_free_kernel<<<(S + 255) / 256 * B, 256, 0, stream>>>(p, table, S, keep_from, keep_to);
    return done();
}

int launch_kv4_compact(const Kv4Pool& p, const int32_t* table, int S, int B, int32_t* table_out, int32_t* refs_out,
                       int32_t* info, int32_t* scratch, hipStream_t stream) {
    kv4_compact_plan_kernel<<<1, kPlanThreads, 0, stream>>>(p, refs_out, info, scratch);
    kv4_compact_move_kernel<<<kCopyGroups, kCopyThreads, 0, stream>>>(p, table, (int64_t)B * S, table_out, scratch);
    return done();
}

int launch_kv4_copy_pages(const Kv4Pool& from, const Kv4Pool& to, const int32_t* src, const int32_t* dst, int64_t n,
                          hipStream_t stream) {
    const int64_t tasks = n * from.layers * ((from.page_bytes() + kPiece - 1) / kPiece);
    kv4_copy_pages_kernel<<<(int)(tasks < kCopyGroups ? tasks : kCopyGroups), kCopyThreads, 0, stream>>>(from, to, src, dst, n);
    return done();
}

}  // namespace scap
