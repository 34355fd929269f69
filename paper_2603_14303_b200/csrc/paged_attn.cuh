// What the decode kernels over a paged cache share: how the rows are divided among blocks, how pages are looked up, and how partial results
// are joined.
#pragma once

#include <cooperative_groups.h>

#include "decode_fold.cuh"
#include "paged.cuh"

namespace sc {
namespace pg {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kTile = 16;                 // rows a warp takes at a time
constexpr int kHeads = 8;                 // most query heads of a unit
constexpr int kMaxBlocks = 448;           // of a launch
constexpr int kCluster = 8;               // most blocks of a party
constexpr int kMergeGroup = 8;            // partial sums read together
constexpr unsigned kShortStretch = 64;    // tiles per block below which stretches are cut at the units' ends
constexpr unsigned kLongUnit = 192;       // mean tiles of a unit from which one block on each SM is better than two
constexpr int kLeast = 2;                 // tiles per warp that a stretch has at least
constexpr int kMaxD = 256;
__host__ __device__ constexpr int part_floats(int d) { return kHeads * d + 2 * kHeads; }   // a partial sum: acc[8][d], m[8], l[8]

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int src_bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, int src_bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }

// ---- how attention's work is shared out ----------------------------------------------------
// The rows of every head, in tiles, form one line: entry after entry of `lens`, its heads (and groups of query heads: "units")
// after one another.  A launch's parties (blocks, or clusters of blocks) take equal stretches of it, so that a batch is
// balanced whatever its lengths are, and nothing about them has to be known on the host.  A party's stretch is cut into
// segments at the units' ends.  A unit inside one stretch is finished there; the parties that share one leave partial sums,
// each in one of two slots of its own (the unit its stretch begins in, and the one it ends in), and the last to arrive joins them.
// Arrival counters, one per party (the first of those that share a unit), lie at the front of the workspace in a place of the same size
// for every shape and kernel, so that no call's partial sums lie where another one's counters are.
constexpr size_t kTicketBytes = 4096;
struct Line {
    const int32_t* lens;
    int entries, per_entry, cap, parties;   // per_entry: units of an entry
    int spare;                              // tiles that every unit takes besides (see divide())

    __device__ __forceinline__ int len(int e) const { return max(min(lens[e], cap), 0); }
    // Of a unit of n rows: whole rounds of a block's warps, so that a unit of one row takes the place that its round does (512 sequences of 10 to
    // 100 rows 63 us, 86 without; 40 of 6 to 60 rows 8.2 and 21).  The tiles behind its rows are nobody's work.
    __host__ __device__ __forceinline__ int tiles_of(int n) const { return n > 0 ? ((n - 1) / (kTile * kWarps) + 1) * kWarps + spare : 0; }
    __device__ __forceinline__ int tiles(int e) const { return tiles_of(len(e)); }
    static __host__ __device__ __forceinline__ int tiles_with_rows(int n) { return n > 0 ? (n - 1) / kTile + 1 : 0; }   // (n may be 2^31 - 1)
    // Positions on the line are 32-bit numbers, which the entry point sees to: several divisions lie on the way to the first load.
};
struct Place {              // a position on the line
    int entry, unit, tile;
    unsigned at;            // of the unit's first tile
};

// The tiles of up to kCutEntries entries, entry lane + 32 i in t[i], which both steps below look at.
constexpr int kCutEntries = 128;
struct Few { unsigned t[kCutEntries / 32]; };
// Length of the line.  All lanes of a warp call it.
__device__ __forceinline__ unsigned total_of(const Line& line, int lane, Few& few) {
    unsigned sum = 0;
    int n[kCutEntries / 32];
#pragma unroll
    for (int i = 0; i < kCutEntries / 32; ++i) n[i] = line.lens[min(lane + 32 * i, line.entries - 1)];   // (unconditional: requested together)
#pragma unroll
    for (int i = 0; i < kCutEntries / 32; ++i) {
        few.t[i] = lane + 32 * i < line.entries ? line.tiles_of(max(min(n[i], line.cap), 0)) : 0;
        sum += few.t[i];
    }
    for (int e0 = kCutEntries + lane; e0 < line.entries + lane; e0 += 8 * 32) {
        int m[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = line.lens[min(e0 + 32 * i, line.entries - 1)];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += e0 + 32 * i < line.entries ? line.tiles_of(max(min(m[i], line.cap), 0)) : 0;
    }
    return __reduce_add_sync(kFull, sum) * line.per_entry;
}

// The place of tile `at` of the line (at < total).  All lanes of a warp call it.
__device__ __forceinline__ Place place_of(const Line& line, unsigned at, int lane) {
    unsigned before = 0;
    for (int e0 = 0;; e0 += 32) {
        const int nt = e0 + lane < line.entries ? line.tiles(e0 + lane) : 0;
        const unsigned mine = (unsigned)nt * line.per_entry, upto = before + warp_scan_add((int)mine, lane);
        const unsigned past = __ballot_sync(kFull, upto > at);
        if (past != 0) {
            const int src = __ffs(past) - 1;
            const unsigned start = __shfl_sync(kFull, upto - mine, src), t = __shfl_sync(kFull, nt, src);
            Place p;
            p.entry = e0 + src;
            p.unit = (at - start) / t;
            p.at = start + p.unit * t;
            p.tile = at - p.at;
            return p;
        }
        before = __shfl_sync(kFull, upto, 31);
    }
}

// A line whose stretches would be short is cut at the units' ends instead, so that a party has one segment and fills its pipeline once:
// every unit in as many equal parts as have `longest` tiles at most, `longest` the least for which there are parties enough (at most an
// eighth over it).  For at most kCutEntries entries and no more units than parties.  All lanes of a warp call it.
struct Part { int entry, unit, tile, take, index, parts; };   // take 0: this party has none
__device__ __forceinline__ Part part_of(const Line& line, const Few& few, unsigned longest, unsigned party, int lane) {
    constexpr int kN = kCutEntries / 32;
    const auto& t = few.t;
    unsigned c[kN], sum;
    for (;; longest += longest / 8 + 1) {
        sum = 0;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            c[i] = 32 * i < line.entries ? (t[i] + longest - 1) / longest : 0;
            sum += c[i];
        }
        sum = __reduce_add_sync(kFull, sum) * line.per_entry;
        if (sum <= (unsigned)line.parties) break;
    }
    Part r = {0, 0, 0, 0, 0, 0};
    if (party >= sum) return r;
    unsigned before = 0;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const unsigned mine = c[i] * line.per_entry, upto = before + warp_scan_add((int)mine, lane);
        const unsigned past = __ballot_sync(kFull, upto > party);
        if (past != 0) {
            const int src = __ffs(past) - 1;
            const unsigned start = __shfl_sync(kFull, upto - mine, src), parts = __shfl_sync(kFull, c[i], src);
            const unsigned nt = __shfl_sync(kFull, t[i], src), each = (nt + parts - 1) / parts;
            r.entry = src + 32 * i;
            r.unit = (party - start) / parts;
            r.index = (party - start) - r.unit * parts;
            r.parts = parts;
            r.tile = r.index * each;
            r.take = min(each, nt - r.tile);   // ((parts - 1) * each < nt)
            return r;
        }
        before = __shfl_sync(kFull, upto, 31);
    }
    return r;
}

// The next unit that has tiles (one follows: the caller has tiles left).
__device__ __forceinline__ void next_unit(const Line& line, Place& p, int tiles_here) {
    p.at += tiles_here;
    p.tile = 0;
    if (++p.unit < line.per_entry) return;
    p.unit = 0;
    do ++p.entry; while (line.tiles(p.entry) == 0);
}

// How a launch is divided: into parties of clusters of `cluster` blocks.  A line of fewer tiles than short_below: each block of a cluster stands
// for itself.  One of long_from or more: the first long_parties only.  blocks_of(cluster): blocks that an SM holds; one_per_sm: whether long lines
// are better off with one block on each SM.
struct Division { int cluster; unsigned short_below, long_from; int long_parties; };
Division divide(Line& line, int sms, int (*blocks_of)(int cluster, int d), int d, bool one_per_sm);
static_assert(kCluster <= dm::kMaxCluster, "");

// A party as one of its blocks sees it.
struct Party {
    int csize, crank, party;     // blocks of the party, this one's rank, the party's number
    bool in_step;                // the cluster's blocks are known to have started
    bool cut;                    // stretches are cut at the units' ends
    unsigned stretch, from, left;
    Part own;

    // Before the kernel waits for the one before it.  Of a cluster: the barriers for what its blocks hand each other.
    __device__ __forceinline__ void set_up(unsigned long long (&bar)[2]) {
        csize = (int)cooperative_groups::this_cluster().num_blocks();
        crank = (int)cooperative_groups::this_cluster().block_rank();
        party = blockIdx.x / csize;
        in_step = csize == 1;
        if (csize == 1) return;
        if (threadIdx.x == 0) {
            umma::mbar_init(smem_u32(&bar[0]), 1);
            umma::mbar_init(smem_u32(&bar[1]), 1);
            umma::mbar_fence_init();
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");   // (waited for before the first hand-over)
    }
    __device__ __forceinline__ void step() {      // every block of the cluster has started
        if (in_step) return;
        __syncwarp();                             // (its callers come from branches and loops of some of a warp's threads)
        asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
        in_step = true;
    }
    // Whether the block has anything to do.
    __device__ __forceinline__ bool plan(Line& line, const Division& how, int lane) {
        Few few;
        const unsigned total = total_of(line, lane, few);
        if (total < how.short_below) {
            step();
            csize = 1; crank = 0; party = blockIdx.x;
            line.parties = gridDim.x;
        }
        if (total >= how.long_from) line.parties = how.long_parties;
        stretch = max((total + line.parties - 1) / line.parties, (unsigned)(csize * kWarps * kLeast));
        cut = stretch < kShortStretch * csize && line.entries <= kCutEntries && line.entries * line.per_entry <= line.parties;
        from = 0;
        if (cut) {
            own = part_of(line, few, stretch, party, lane);
            left = own.take;
        } else {
            if (csize == 1) stretch = (stretch + kWarps - 1) / kWarps * kWarps;   // whole rounds
            from = min((uint64_t)party * stretch, (uint64_t)total);
            left = min(stretch, total - from);
        }
        return left > 0;
    }
    __device__ __forceinline__ Place begin(const Line& line, int lane) const {
        return cut ? Place{own.entry, own.unit, own.tile, 0u} : place_of(line, from, lane);
    }
};

// Which head a unit is: units of an entry are its KV heads (of a table that all share) times groups of query heads.
struct Unit {
    int b, h, g0, nh;            // sequence, KV head, first query head of the group within it, query heads
    template <typename T>
    __device__ __forceinline__ Unit(const Pages<T>& pages, int entry, int unit, int G, int group) {
        b = pages.table_heads > 1 ? entry / pages.table_heads : entry;
        int rest = 0;
        if (G > group) {
            const int groups = (G + group - 1) / group;
            rest = unit % groups;
            unit /= groups;
        }
        h = pages.table_heads > 1 ? entry - b * pages.table_heads : unit;
        g0 = rest * group;
        nh = min(group, G - g0);
    }
};

__device__ __forceinline__ void store_out4(__nv_bfloat16* dst, const float4& o, float l) {   // (no row: zeros; l not a number: not a number)
    const float inv = l != 0.f ? 1.f / l : 0.f;
    store4(dst, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
}
__device__ __forceinline__ void store_out4(float* dst, const float4& o, float l) {
    const bool any = l != 0.f;
    store4(dst, make_float4(any ? o.x / l : 0.f, any ? o.y / l : 0.f, any ? o.z / l : 0.f, any ? o.w / l : 0.f));
}

// Heads without rows.
template <typename T, typename P>
__device__ __forceinline__ void zero_empty(const P& pages, const Line& line, int Hq, int G, int group, int d, T* __restrict__ out) {
    for (int e = blockIdx.x; e < line.entries; e += gridDim.x) {
        if (line.len(e) > 0) continue;
        const int d4 = d / 4;
        for (int i = threadIdx.x; i < line.per_entry * group * d4; i += kThreads) {
            const Unit u(pages, e, i / (group * d4), G, group);
            const int g = i / d4 % group;
            if (g < u.nh) store_out4(out + ((int64_t)u.b * Hq + u.h * G + u.g0 + g) * d + i % d4 * 4, make_float4(0.f, 0.f, 0.f, 0.f), 0.f);
        }
    }
}

// Pages are looked up for kBatch of a warp's tiles at a time (its j-th is tile first + j * kWarps), a batch ahead: one load, whose latency
// is longer than a tile takes.  kWhole (page_size a multiple of 16: a tile lies in one page): lane l has the batch's l-th tile; else the
// row lane & 15 of its (l / 16)-th.  x: the page, -1: no such row;  y: the row's (the tile's first row's) place in it.
template <bool kWhole>
struct Finder {
    static constexpr int kBatch = kWhole ? 32 : 2;
    const int32_t* table;
    int page_size, page_bits, len, first, n;     // page_bits: of a page_size that is a power of two, else -1; n: the warp's tiles
    int2 batch, next;

    __device__ __forceinline__ int2 look_up(int j0, int lane) const {
        const int j = j0 + (kWhole ? lane : lane >> 4);
        int2 at = make_int2(-1, 0);
        if (j >= n) return at;
        const int row = (first + j * kWarps) * kTile + (kWhole ? 0 : lane & 15);
        if (row < len) {
            const int slot = page_bits >= 0 ? row >> page_bits : row / page_size;
            at = make_int2(table[slot], row - slot * page_size);
        }
        return at;
    }
    __device__ __forceinline__ void start(int lane) { batch = look_up(0, lane); next = look_up(kBatch, lane); }
    __device__ __forceinline__ int2 get(int j, int lane) {      // j = 0, 1, ... in turn
        if (j % kBatch == 0 && j > 0) {
            batch = next;
            next = look_up(j + kBatch, lane);
        }
        const int src = kWhole ? j & 31 : (j & 1) * 16 + (lane & 15);
        return make_int2(__shfl_sync(kFull, batch.x, src), __shfl_sync(kFull, batch.y, src));
    }
};

// What the blocks of a cluster hand each other, for two segments by turns.
__host__ __device__ constexpr int recv_o_bytes(int d, int heads) { return (heads * (d / 4) + kCluster) * 16; }   // slices of O, rounded up
__host__ __device__ constexpr int recv_bytes(int d, int heads) { return recv_o_bytes(d, heads) + kCluster * kHeads * 8; }   // and m, l

// A block that gave up on a hand-over takes part in no other: for its later segments it hands nothing on and waits for nothing, and what it has to give
// is not a number.  The cluster's other blocks miss its slices at the next segment and give up there.  So nobody's bytes come to a place or a phase that
// is still in use: who hands something over for the segment after the next has had everybody's slices of the next one, and those a block hands on when it
// is done with the one before.
//
// A segment's sums become results or go to whoever joins them.  sum(e4): four columns of a head (e4 = head * d / 4 + column / 4) over the
// block's warps; ml(head): their m and l.  All threads of the block call it, behind a barrier; they may be anywhere in it when it returns.
struct Joiner {
    unsigned long long* bar;     // [2]
    unsigned char* recv;
    int* last_shared;
    int32_t* tickets;
    float* part;
    int32_t* status;
    int heads;                   // most of a unit
    unsigned turn;               // segments handed over: which barrier and place, and its phase
    bool got;                    // no wait has given up: of this thread's in a segment, of the block's behind next()
    unsigned long long limit_ns = umma::kWaitLimitNs;

    template <typename T, typename Sum, typename Ml>
    __device__ __forceinline__ void join(Party& me, const Place& p, int nt, int take, int nh, int d, T* __restrict__ out, Sum&& sum, Ml&& ml) {
        const bool whole = take == nt;
        const int d4n = d / 4, n4 = nh * d4n, slice = (n4 + me.csize - 1) / me.csize, e_lo = min(me.crank * slice, n4), e_hi = min(e_lo + slice, n4);
        const int stride = part_floats(d);
        float* mine = part + (size_t)(2 * me.party + (!me.cut && p.at > me.from)) * stride;
        const auto give = [&](int e4, const float4& acc, float m, float l) {
            const int hd = e4 / d4n, d4 = e4 % d4n * 4;
            if (whole) {
                store_out4(out + (int64_t)hd * d + d4, acc, l);
            } else {
                *reinterpret_cast<float4*>(mine + hd * d + d4) = acc;
                if (d4 == 0 || e4 == e_lo) { mine[kHeads * d + hd] = m; mine[kHeads * d + kHeads + hd] = l; }   // (the same from every slice of the head)
            }
        };
        if (me.csize == 1) {
            for (int e4 = threadIdx.x; e4 < n4; e4 += kThreads) {
                const float2 v = ml(e4 / d4n);
                give(e4, sum(e4), v.x, v.y);
            }
        } else {
            // Every block hands slice r of its sums to block r, which folds it.  A block's receiving places are used by turns: who hands it
            // something for the segment after the next has its slice of the next one, so it is done with this one.
            const uint32_t b = smem_u32(&bar[turn & 1]);
            unsigned char* to_me = recv + (turn & 1) * recv_bytes(d, heads);
            float4* recv_o = reinterpret_cast<float4*>(to_me);
            float* recv_ml = reinterpret_cast<float*>(to_me + recv_o_bytes(d, heads));
            if (got) {
                if (threadIdx.x == 0) umma::mbar_expect_tx(b, (uint32_t)(me.csize * ((e_hi - e_lo) * 16 + kHeads * 8)));
                me.step();
                for (int e4 = threadIdx.x; e4 < n4; e4 += kThreads) {
                    const int to = e4 / slice;
                    dm::hand_over(dm::mapa(smem_u32(recv_o + me.crank * slice + (e4 - to * slice)), to), dm::mapa(b, to), sum(e4));
                }
                for (int x = threadIdx.x; x < me.csize * kHeads; x += kThreads) {
                    const float2 v = ml(x & 7);
                    dm::hand_over(dm::mapa(smem_u32(recv_ml + me.crank * 2 * kHeads + (x & 7) * 2), x >> 3), dm::mapa(b, x >> 3), v.x, v.y);
                }
                got = dm::slices_arrived(b, limit_ns, turn >> 1 & 1);
                if (!got) set_status(status, SC_ERR_TIMEOUT);
                ++turn;
            }
            for (int e4 = e_lo + threadIdx.x; e4 < e_hi; e4 += kThreads) {
                dm::Folded f = dm::fold_slices(recv_o, recv_ml, me.csize, slice, e4 - e_lo, e4 / d4n, got);
                // Where they have not all arrived, m and l as well: they come from every slice of a head, the last one to be stored stays, and
                // whichever m and l are left together give these columns as NaN and the head's others right or as NaN.
                if (!got) { f.m = INFINITY; f.l = __int_as_float(0x7fffffff); }
                give(e4, f.o, f.m, f.l);
            }
        }
        if (whole) return;
        // Parties that share a unit: the last one to bring a slice joins the slice's parts in order.
        const unsigned first = me.cut ? me.party - me.own.index : p.at / me.stretch;
        const unsigned last = me.cut ? first + me.own.parts - 1 : (p.at + nt - 1) / me.stretch;
        int32_t* ticket = tickets + (first * me.csize + me.crank);   // (a party begins one shared unit at most)
        __syncthreads();   // (what the block's threads have written is released with the first one's arrival)
        if (threadIdx.x == 0) {
            int t;
            asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;\n" : "=r"(t) : "l"(ticket) : "memory");
            *last_shared = t == (int)(last - first);
            if (*last_shared) *ticket = 0;   // ready for the next call
        }
        __syncthreads();
        if (!*last_shared) return;
        for (int e4 = e_lo + threadIdx.x; e4 < e_hi; e4 += kThreads) {
            const int hd = e4 / d4n, d4 = e4 % d4n * 4;
            float m = -INFINITY, l = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            for (unsigned j0 = first; j0 <= last; j0 += kMergeGroup) {
                float mv[kMergeGroup], lv[kMergeGroup];
                float4 ov[kMergeGroup];
#pragma unroll
                for (int j = 0; j < kMergeGroup; ++j) {
                    const bool ok = j0 + j <= last;
                    const unsigned w = ok ? j0 + j : first;
                    const float* sp = part + (size_t)(2 * w + (!me.cut && p.at > w * me.stretch)) * stride;
                    mv[j] = ok ? __ldcg(sp + kHeads * d + hd) : -INFINITY;
                    lv[j] = __ldcg(sp + kHeads * d + kHeads + hd);
                    ov[j] = __ldcg(reinterpret_cast<const float4*>(sp + hd * d + d4));
                }
                float nm = m;
#pragma unroll
                for (int j = 0; j < kMergeGroup; ++j) nm = fmaxf(nm, mv[j]);
                if (nm == -INFINITY) continue;   // nothing but parts without rows so far
                const float c = m == -INFINITY ? 0.f : exp2f(m - nm);
                l *= c; acc.x *= c; acc.y *= c; acc.z *= c; acc.w *= c;
                m = nm;
#pragma unroll
                for (int j = 0; j < kMergeGroup; ++j) {
                    if (mv[j] == -INFINITY) continue;
                    const float w = exp2f(mv[j] - m);
                    l = fmaf(w, lv[j], l);
                    acc.x = fmaf(w, ov[j].x, acc.x); acc.y = fmaf(w, ov[j].y, acc.y);
                    acc.z = fmaf(w, ov[j].z, acc.z); acc.w = fmaf(w, ov[j].w, acc.w);
                }
            }
            store_out4(out + (int64_t)hd * d + d4, acc, l);
        }
    }
    // Between two segments, in place of a barrier of the block's threads.
    __device__ __forceinline__ void next(const Party& me) {
        if (me.csize == 1) __syncthreads(); else got = __syncthreads_and(got);
    }
    // The last step.  Where a hand-over was given up on, the block's shared memory stays until the cluster's other blocks have left (each of
    // their waits ends, and a thread that has left is not waited for) and what they handed over has landed: of the last phase that was
    // waited for here; who handed something over for the one after it has waited for this block's slices meanwhile, to the limit.
    __device__ __forceinline__ void leave(const Party& me) {
        if (me.csize == 1 || __all_sync(kFull, got)) return;
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
        umma::mbar_wait<true>(smem_u32(&bar[(turn - 1) & 1]), (turn - 1) >> 1 & 1, limit_ns);
    }
};

}  // namespace pg
}  // namespace sc
