// Attention of the few new tokens of every sequence (one, or the gamma + 1 rows of a verification pass) over its paged K,V rows:
//   S_j = scale * q . k_j for the keys j at or before the row's position,  o = sum_j softmax(S)_j v_j.
//
// Bound by the cached rows' bytes: they are read once for all queries of a KV head, as they lie (8 bits or 16), and widened in
// registers on their way into mma.sync (M = 16 queries, fp16 or, for bf16 caches, bf16; sums fp32).  Scales of 8-bit rows stay
// outside the products: with k_j = sk_j kc_j and v_j = sv_j vc_j,
//   S_j = (scale sk_j)(q . kc_j),   o = sum_j w_j vc_j / sum_j w_j / sv_j   with w_j = exp(S_j) sv_j = 2^(S_j log2 e + log2 sv_j):
// the running maximum is taken of the latter exponent, so that w_j, which is rounded to fp16 for the second product, is at most
// about 1 whatever the scales are, and one exponential per score serves both sums.
//
// Work: tiles of 64 keys of a segment (sequence, block of queries, KV head).  The lengths are known on the device only, so every
// CTA adds them up and takes an equal, contiguous run of all tiles (the longest sequence does not decide, whatever the capacity of
// the page table); a segment that several CTAs share leaves (maximum, sum, weighted rows) per CTA in the workspace, and a second
// kernel joins them in order.  No atomics: the same bits every time.
//
// A CTA has four groups of warps; a group takes 16 of a tile's 64 keys, a warp of it 16 queries.  One more warp asks for the tiles
// of the whole run, segment after segment, by TMA (halves of 32 keys, which never straddle a page, with the shared-memory
// swizzle), through a ring of stages with a barrier to fill and one to free each; the others never wait for one another within a segment.
#include <algorithm>

#include "paged.cuh"
#include "tc_util.cuh"

namespace spec {
namespace {

using namespace tc;

constexpr int kTileKeys = 64;
constexpr int kGroups = 4;       // warps along a tile's keys, 16 keys each
constexpr int kMostCtas = 592;   // 148 SMs x 4
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.0f;   // the running maximum may lag by this: w <= 2^8 stays in fp16's range

__device__ int g_paged_error;  // set when the bounded wait for a tile or for its place ran out (0 = none)

struct AttnArgs {
    Paged cache;
    const void* pool;
    const float* scales;
    const void* q;
    void* out;
    const int32_t* lengths;
    float* partial;    // [slots][queries of a block][D]
    float2* partial_ml;  // [slots][queries of a block]: maximum, sum
    long long q_stride;
    float scale;
    int batch, rows, n_heads, group, blocks, units;  // blocks: of queries per (sequence, KV head); units = batch * blocks
    int q_bf16, grid;
};

// Copies that count their bytes on a barrier: a box of 32 rows of a plane (K or V of a page and head), and a run of bytes.
__device__ __forceinline__ void load_box(void* to, const CUtensorMap* map, int x, int row, int plane, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(smem_u32(to)), "l"(map), "r"(x), "r"(row), "r"(plane), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void load_bulk(void* to, const void* from, int bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(to)), "l"(from), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

template <bool BF16>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint4& a, uint32_t b0, uint32_t b1) {
    if constexpr (BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
    if constexpr (BF16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&v);
    } else {
        const __half2 v = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
}
// Bytes 2 i and 2 i + 1 (STEP 1) of four codes, or bytes i and i + 2 (STEP 2), as two fp16 values.
template <int KV, int STEP>
__device__ __forceinline__ void widen(uint32_t codes, uint32_t& first, uint32_t& second) {
    if constexpr (KV == SPEC_DTYPE_INT8) {
        // code + 128 as the low bits of 1024.0, minus 1152: exact
        const uint32_t biased = codes ^ 0x80808080u;
        const uint32_t x = __byte_perm(biased, 0x64646464u, STEP == 1 ? 0x4140 : 0x4240), y = __byte_perm(biased, 0x64646464u, STEP == 1 ? 0x4342 : 0x4341);
        const __half2 off = __floats2half2_rn(1152.0f, 1152.0f);
        const __half2 a = __hsub2(*reinterpret_cast<const __half2*>(&x), off), b = __hsub2(*reinterpret_cast<const __half2*>(&y), off);
        first = *reinterpret_cast<const uint32_t*>(&a);
        second = *reinterpret_cast<const uint32_t*>(&b);
    } else {
        if constexpr (STEP == 2) codes = __byte_perm(codes, 0u, 0x3120);
        asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}" : "=r"(first), "=r"(second) : "r"(codes));
    }
}

// The hardware's approximations, subnormal results as zeros: 2^x to two units of the last place, log2 to 2^-22, 1/x to one unit.
__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float log2_of(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float reciprocal_of(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Whether a NaN or an infinity is among 16 bytes of a row.
template <int KV>
__device__ __forceinline__ bool not_numbers(const uint4& v) {
    const uint32_t words[4] = {v.x, v.y, v.z, v.w};
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (KV == SPEC_DTYPE_E4M3) {
#pragma unroll
            for (int j = 0; j < 4; ++j) any |= (words[i] >> (8 * j) & 0x7fu) == 0x7fu;
        } else {
            constexpr uint32_t exponent = KV == SPEC_DTYPE_BF16 ? 0x7f80u : 0x7c00u;
            any |= (words[i] & exponent) == exponent || (words[i] >> 16 & exponent) == exponent;
        }
    }
    return any;
}

// One segment of a CTA's run of tiles.
struct Segment {
    int unit, head, tile0, tile1, tiles, limit;  // limit: keys before it exist for some row of the block
};

// Tiles of a unit (sequence, block of queries): the keys up to the position of the block's last row.
template <int QT>
__device__ __forceinline__ int unit_limit(const AttnArgs& a, int unit) {
    const int b = unit / a.blocks, block = unit - b * a.blocks;
    const long long capacity = static_cast<long long>(a.cache.width) << a.cache.page_shift;
    const int length = a.lengths[b];
    const int last_row = min(a.rows - 1, (block * QT + QT - 1) / a.group);
    const long long limit = static_cast<long long>(length) - a.rows + last_row + 1;
    return static_cast<int>(max(0ll, min(min(limit, static_cast<long long>(length)), capacity)));
}

// The unit in which tile `wanted` of all lies, with the tiles (of one KV head) before it; and the sum over all units.
// `wanted(total)` is called once the sum is known.  All threads of the block; `scratch`: 40 long longs.
template <int QT, typename F>
__device__ __forceinline__ void find_unit(const AttnArgs& a, long long* scratch, F wanted, long long& total, int& unit, long long& before) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    long long base = 0, target = 0;
    unit = -1;
    for (int round = a.units > static_cast<int>(blockDim.x) ? 0 : 1; round < 2; ++round) {  // (more units than threads: add up first, look then)
        if (round == 1 && a.units > static_cast<int>(blockDim.x)) {
            total = base * a.cache.n_kv;
            target = wanted(total);
            base = 0;
        }
        for (int u0 = 0; u0 < a.units; u0 += blockDim.x) {
            const int u = u0 + threadIdx.x;
            const long long mine = u < a.units ? (unit_limit<QT>(a, u) + kTileKeys - 1) / kTileKeys : 0;
            long long upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long up = __shfl_up_sync(kFullMask, upto, o);
                if (lane >= o) upto += up;
            }
            __syncthreads();  // (scratch is free)
            if (lane == 31) scratch[warp] = upto;
            __syncthreads();
            long long all = 0, front = 0;
            for (int w = 0; w < warps; ++w) {
                if (w < warp) front += scratch[w];
                all += scratch[w];
            }
            upto += base + front;
            if (round == 1) {
                if (a.units <= static_cast<int>(blockDim.x)) {
                    total = all * a.cache.n_kv;
                    target = wanted(total);
                }
                if ((upto - mine) * a.cache.n_kv <= target && target < upto * a.cache.n_kv) {
                    scratch[32] = u;
                    scratch[33] = upto - mine;
                }
            }
            base += all;
        }
    }
    if (total == 0 || target >= total) return;
    __syncthreads();
    unit = static_cast<int>(scratch[32]);
    before = scratch[33];
}

__device__ __forceinline__ long long first_tile(long long total, int cta, int ctas) { return total * cta / ctas; }
__device__ __forceinline__ int owner_of(long long total, long long tile, int ctas) { return static_cast<int>(((tile + 1) * ctas - 1) / total); }
__device__ __forceinline__ int ctas_of(long long total, int grid) { return static_cast<int>(min(total, static_cast<long long>(grid))); }

template <int D, int KV, int MT>
struct Shape {
    static constexpr bool kEight = KV == SPEC_DTYPE_E4M3 || KV == SPEC_DTYPE_INT8;
    static constexpr bool kBf16 = KV == SPEC_DTYPE_BF16;
    static constexpr int kRowBytes = D * (kEight ? 1 : 2);
    static constexpr int kBoxBytes = kRowBytes < 128 ? kRowBytes : 128;  // of a row in one copy: what the swizzle spans
    static constexpr int kBoxes = kRowBytes / kBoxBytes;
    static constexpr int kChunks = kRowBytes / 16;
    static constexpr int kQueries = 16 * MT;
    static constexpr int kComputeWarps = kGroups * MT;
    static constexpr int kThreads = 32 * (kComputeWarps + 1);  // and the warp that asks for the tiles
    static constexpr int kOperandBytes = kTileKeys * kRowBytes;  // K or V of a tile
    static constexpr int kStageBytes = 2 * kOperandBytes;
    static constexpr int kScaleBytes = kEight ? 2 * kTileKeys * 4 : 0;
    static constexpr int kQueryBytes = kQueries * D * 2;
    static constexpr int kMerge = 2 * MT * 16 * (D + 2) * 4;  // two groups' states
    static constexpr int kPerSm = MT == 1 ? (kRowBytes <= 128 ? 3 : 2) : 1;
    static constexpr int kFixed = kMerge + kQueryBytes + kQueries * 4 + 40 * 8 + 1024 /* alignment */ + 256 /* barriers, notes */;
    static constexpr int kStagesThatFit = ((227 * 1024 + 1024) / kPerSm - 1024 - kFixed) / (kStageBytes + kScaleBytes);
    static constexpr int kStages = kStagesThatFit < 8 ? kStagesThatFit : 8;
    static constexpr int kSmem = kStages * (kStageBytes + kScaleBytes) + kFixed;
    static_assert(kStages >= 2, "a ring");
    // Place of 16-byte chunk c of row r in a K or V tile, as the copies' swizzle leaves it: rows whose chunks meet in the reads
    // below lie in different banks.
    static __device__ __forceinline__ int place(int r, int c) {
        if constexpr (kBoxBytes == 64) return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
        else return (c >> 3) * (kTileKeys * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
    }
    // Which of eight keys a lane quad n reads, and column n of a score tile stands for: neighbours differ in the bit that moves a
    // row's chunks to the other half of the banks.
    static __device__ __forceinline__ int key_of(int n) { return kBoxBytes == 64 ? n : (n & 1) * 4 + (n >> 1); }
};

// The tiles of a CTA's run, segment by segment.
template <int QT>
struct Run {
    long long left;  // tiles, the present segment's among them
    Segment g;
    __device__ __forceinline__ void open(const AttnArgs& a) {  // what follows from unit
        g.limit = unit_limit<QT>(a, g.unit);
        g.tiles = (g.limit + kTileKeys - 1) / kTileKeys;
    }
    __device__ __forceinline__ void close() { g.tile1 = static_cast<int>(min(static_cast<long long>(g.tiles), g.tile0 + left)); }
    __device__ __forceinline__ bool next(const AttnArgs& a) {
        left -= g.tile1 - g.tile0;
        if (left <= 0) return false;
        g.tile0 = 0;
        if (++g.head == a.cache.n_kv) {
            g.head = 0;
            do {
                ++g.unit;
                open(a);
            } while (g.limit == 0);
        }
        close();
        return true;
    }
};

template <int THREADS>
__device__ __forceinline__ void compute_sync() { asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory"); }

template <int D, int KV, int MT>
__global__ void __launch_bounds__(Shape<D, KV, MT>::kThreads, Shape<D, KV, MT>::kPerSm)
paged_attention_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ AttnArgs a) {
    using S = Shape<D, KV, MT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    float* ring_scales = reinterpret_cast<float*>(ring + S::kStages * S::kStageBytes);  // [stage][K, V][64]
    float* merge = reinterpret_cast<float*>(ring + S::kStages * (S::kStageBytes + S::kScaleBytes));
    uint4* q_frag = reinterpret_cast<uint4*>(merge + S::kMerge / 4);                 // [MT][D / 16][32 lanes]
    float* q_factor = reinterpret_cast<float*>(q_frag + S::kQueryBytes / 16);  // what a row's products are multiplied with
    long long* scratch = reinterpret_cast<long long*>(q_factor + S::kQueries);
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(scratch + 40);
    uint64_t* empty_bar = full_bar + S::kStages;
    int* notes = reinterpret_cast<int*>(empty_bar + S::kStages);  // [stage]: keys of the tile that there are, and which of its halves were fetched

    const int warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(&full_bar[s], 1);
            mbar_init(&empty_bar[s], S::kComputeWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    pdl_trigger();  // (behind the wait: the joining kernel reads the lengths ahead of its own)

    long long total = 0, before = 0;
    int unit = 0, ctas = 0;
    find_unit<S::kQueries>(a, scratch, [&](long long sum) {
        ctas = max(1, ctas_of(sum, a.grid));
        return static_cast<int>(blockIdx.x) < ctas ? first_tile(sum, blockIdx.x, ctas) : sum;
    }, total, unit, before);
    if (unit < 0) return;  // (more CTAs than tiles)
    Run<S::kQueries> run;
    Segment& g = run.g;
    {
        const long long first = first_tile(total, blockIdx.x, ctas), within = first - before * a.cache.n_kv;
        run.left = first_tile(total, blockIdx.x + 1, ctas) - first;
        g.unit = unit;
        run.open(a);
        g.head = static_cast<int>(within / g.tiles);
        g.tile0 = static_cast<int>(within - static_cast<long long>(g.head) * g.tiles);
        run.close();
    }
    __syncthreads();  // (barriers are there for all)
    uint32_t limit = kSpinLimit;  // of every wait; one that has run out leaves one try to the others, and the CTA ends with its error noted

    if (warp == S::kComputeWarps) {
        // ---- the tiles of the whole run, through the ring: halves of 32 keys, which lie in one page each ----
        const bool leader = elect_one();
        int stage = 0, use = 0;
        do {
            const int b = g.unit / a.blocks;
            const int32_t* pages = a.cache.table + static_cast<size_t>(b) * a.cache.width;
            for (int t = g.tile0; t < g.tile1; ++t) {
                int page[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int key = t * kTileKeys + 32 * h;
                    page[h] = key < g.limit ? pages[key >> a.cache.page_shift] : -1;
                    if (page[h] >= a.cache.pages) page[h] = -1;
                }
                if (use > 0 && !mbar_wait_warp(&empty_bar[stage], (use - 1) & 1, limit)) limit = 1;
                if (leader) {
                    const int halves = (page[0] >= 0 ? 1 : 0) + (page[1] >= 0 ? 1 : 0);
                    notes[stage] = min(kTileKeys, g.limit - t * kTileKeys) | (page[0] >= 0 ? 256 : 0) | (page[1] >= 0 ? 512 : 0);
                    mbar_expect_tx(&full_bar[stage], halves * (S::kStageBytes + S::kScaleBytes) / 2);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (page[h] < 0) continue;
                        const int slot = (t * kTileKeys + 32 * h) & ((1 << a.cache.page_shift) - 1);
#pragma unroll
                        for (int which = 0; which < 2; ++which) {
                            const int plane = (page[h] * 2 + which) * a.cache.n_kv + g.head;
                            uint8_t* to = ring + stage * S::kStageBytes + which * S::kOperandBytes + h * 32 * S::kBoxBytes;
#pragma unroll
                            for (int box = 0; box < S::kBoxes; ++box)
                                load_box(to + box * (kTileKeys * 128), &map, box * (S::kEight ? 128 : 64), slot, plane, &full_bar[stage]);
                            if constexpr (S::kEight)
                                load_bulk(ring_scales + (stage * 2 + which) * kTileKeys + 32 * h,
                                          a.scales + (static_cast<long long>(plane) << a.cache.page_shift) + slot, 128, &full_bar[stage]);
                        }
                    }
                }
                __syncwarp();
                if (++stage == S::kStages) { stage = 0; ++use; }
            }
        } while (run.next(a));
        if (limit != kSpinLimit) {  // nothing may still be on its way when the CTA leaves
            for (int s = 0; s < S::kStages; ++s) {
                mbar_wait(&full_bar[s], 0, 1 << 14);
                mbar_wait(&full_bar[s], 1, 1 << 14);
            }
            if (lane == 0) atomicCAS(&g_paged_error, 0, 1);
        }
        return;
    }

    const int mt = warp % MT, group = warp / MT;
    const int r0 = lane >> 2, c = lane & 3;
    constexpr int kCompute = 32 * S::kComputeWarps;
    int stage = 0, use = 0;
    do {
        const int b = g.unit / a.blocks, block = g.unit - b * a.blocks;
        const int length = a.lengths[b];

        // ---- the block's queries, in the order in which the products take them ----
        // Lane c of a quad reads dims E (4 i + c) + 4 s .. + 3 of a key row (E elements to 16 bytes), so step E/4 i + s of the
        // product takes the same dims of the query.  fp16 rows are brought to a largest magnitude in [1, 2) by a power of two.
        constexpr int E = 16 / (S::kRowBytes / D), kPerChunk = E / 4;
        for (int row = warp; row < S::kQueries; row += S::kComputeWarps) {
            const int query = block * S::kQueries + row, i = query / a.group;
            const bool there = i < a.rows;
            float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (there && lane < D / 4) {
                const int head = g.head * a.group + query - i * a.group;
                const size_t at = (static_cast<size_t>(b) * a.rows + i) * a.q_stride + head * D + 4 * lane;
                if (a.q_bf16) load_row(static_cast<const __nv_bfloat16*>(a.q) + at, true, v);
                else load_row(static_cast<const __half*>(a.q) + at, true, v);
            }
            float back = 1.0f;
            if constexpr (!S::kBf16) {
                uint32_t largest = 0u;
#pragma unroll
                for (int j = 0; j < 4; ++j) largest = max(largest, magnitude(v[j]));
                largest = __reduce_max_sync(kFullMask, largest);
                if (largest != 0u && largest < 0x7f800000u) {
                    const int e = max(-120, min(120, static_cast<int>(largest >> 23) - 127));
                    back = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
                    const float by = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] *= by;
                }
            }
            if (lane < D / 4) {
                const int dim = 4 * lane, chunk = dim / E, step = (chunk >> 2) * kPerChunk + (dim % E) / 4;
                uint32_t* to = reinterpret_cast<uint32_t*>(q_frag + ((row >> 4) * (D / 16) + step) * 32 + (row & 7) * 4 + (chunk & 3)) + ((row >> 3) & 1);
                to[0] = pack2<S::kBf16>(v[0], v[1]);
                to[2] = pack2<S::kBf16>(v[2], v[3]);
            }
            if (lane == 0) q_factor[row] = back * a.scale * kLog2e;
        }
        compute_sync<kCompute>();

        // positions of this thread's two queries; one that does not exist sees nothing
        int seen[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = (block * S::kQueries + mt * 16 + r0 + 8 * h) / a.group;
            seen[h] = i < a.rows ? static_cast<int>(max(-1ll, static_cast<long long>(length) - a.rows + i)) : -1;
        }
        const int seen_by_all = static_cast<int>(max(-1ll, static_cast<long long>(length) - a.rows + min(a.rows - 1, block * S::kQueries / a.group)));
        const float factor[2] = {q_factor[mt * 16 + r0], q_factor[mt * 16 + r0 + 8]};

        float o[D / 8][4], top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int n = 0; n < D / 8; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[n][j] = 0.0f;

        for (int t = g.tile0; t < g.tile1; ++t) {
            if (!mbar_wait_warp(&full_bar[stage], use & 1, limit)) limit = 1;
            const uint8_t* keys = ring + stage * S::kStageBytes;
            uint8_t* values = ring + stage * S::kStageBytes + S::kOperandBytes;
            const float* consts = ring_scales + stage * 2 * kTileKeys;
            const int note = notes[stage];
            // keys of this warp's sixteen that there are (they lie in one half of the tile)
            const int there = note & (group >= kGroups / 2 ? 512 : 256) ? max(0, min(16, (note & 255) - 16 * group)) : 0;
            const int first_key = t * kTileKeys + group * 16;

            // A weight of zero does not hide a V row that is no number from the product.  Rows that are not there (left from
            // before, or of other sequences) are cleared; rows that some of the block's queries see and others do not are looked at,
            // and one with such a value is taken out and told to those who see it.
            const bool hidden = KV != SPEC_DTYPE_INT8 && first_key + 15 > seen_by_all && seen_by_all + 1 < g.limit;
            uint32_t bad = 0u;  // a bit per key
            if (KV != SPEC_DTYPE_INT8 && (there < 16 || hidden)) {
                if (hidden) {
                    for (int i = lane; i < 16 * S::kChunks; i += 32) {
                        const int r = i / S::kChunks;
                        if (r < there && not_numbers<KV>(*reinterpret_cast<const uint4*>(values + S::place(group * 16 + r, i % S::kChunks)))) bad |= 1u << r;
                    }
                    bad = __reduce_or_sync(kFullMask, bad);
                    // (the warps with the same keys look before one of them clears)
                    if constexpr (MT > 1) asm volatile("bar.sync %0, %1;" ::"r"(2 + group), "n"(32 * MT) : "memory");
                }
                for (int i = lane; i < 16 * S::kChunks; i += 32) {
                    const int r = i / S::kChunks;
                    if (r >= there || (bad >> r & 1u)) *reinterpret_cast<uint4*>(values + S::place(group * 16 + r, i % S::kChunks)) = make_uint4(0u, 0u, 0u, 0u);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // (before the next copy into this stage)
            }
            float s[2][4];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[n][j] = 0.0f;
            const uint4* queries = q_frag + mt * (D / 16) * 32 + lane;
#pragma unroll
            for (int i = 0; i < S::kChunks / 4; ++i) {
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const uint4 w = *reinterpret_cast<const uint4*>(keys + S::place(group * 16 + n * 8 + S::key_of(r0), 4 * i + c));
                    if constexpr (S::kEight) {
                        const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            uint32_t b0, b1;
                            widen<KV, 1>(words[k], b0, b1);
                            mma16816<S::kBf16>(s[n], queries[(4 * i + k) * 32], b0, b1);
                        }
                    } else {
                        mma16816<S::kBf16>(s[n], queries[(2 * i) * 32], w.x, w.y);
                        mma16816<S::kBf16>(s[n], queries[(2 * i + 1) * 32], w.z, w.w);
                    }
                }
            }
            // ---- exponents, their running maximum, weights ----
            float inv[2][2];
            float now[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    inv[n][x] = 1.0f;
                    if constexpr (S::kEight) {
                        const int key = group * 16 + n * 8 + S::key_of(2 * c + x);
                        const float sk = consts[key], sv = consts[kTileKeys + key], raise = log2_of(sv);
                        inv[n][x] = reciprocal_of(sv);
#pragma unroll
                        for (int h = 0; h < 2; ++h) s[n][2 * h + x] = fmaf(s[n][2 * h + x], sk * factor[h], raise);
                    } else {
#pragma unroll
                        for (int h = 0; h < 2; ++h) s[n][2 * h + x] *= factor[h];
                    }
                }
            if (there < 16 || first_key + 15 > seen_by_all) {  // keys that are not there, or not for every query
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int key = n * 8 + S::key_of(2 * c + x);
                        bool number = !(bad >> key & 1u);
                        if constexpr (S::kEight) number = number && magnitude(consts[kTileKeys + group * 16 + key]) < 0x7f800000u;
                        // (a row of V that is no number makes the exponent none for who sees it, and no one else's sum)
                        if (!number || key >= there) inv[n][x] = 0.0f;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float& e = s[n][2 * h + x];
                            if (!number) e = NAN;
                            if (key >= there || first_key + key > seen[h]) e = -INFINITY;
                        }
                    }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) now[h] = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                now[h] = fmaxf(now[h], __shfl_xor_sync(kFullMask, now[h], 1));
                now[h] = fmaxf(now[h], __shfl_xor_sync(kFullMask, now[h], 2));
            }
            if (__any_sync(kFullMask, now[0] > top[0] + kSlack || now[1] > top[1] + kSlack)) {
                float shrink[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float higher = fmaxf(top[h], now[h]);
                    shrink[h] = top[h] == -INFINITY ? 0.0f : exp2_of(top[h] - higher);
                    top[h] = higher;
                    sum[h] *= shrink[h];
                }
#pragma unroll
                for (int n = 0; n < D / 8; ++n) {
                    o[n][0] *= shrink[0];
                    o[n][1] *= shrink[0];
                    o[n][2] *= shrink[1];
                    o[n][3] *= shrink[1];
                }
            }
            uint4 p;
            {
                const float from[2] = {top[0] == -INFINITY ? 0.0f : top[0], top[1] == -INFINITY ? 0.0f : top[1]};
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[n][j] = exp2_of(s[n][j] - from[j >> 1]);
                        sum[j >> 1] = fmaf(s[n][j], inv[n][j & 1], sum[j >> 1]);
                    }
                p.x = pack2<S::kBf16>(s[0][0], s[0][1]);
                p.y = pack2<S::kBf16>(s[0][2], s[0][3]);
                p.z = pack2<S::kBf16>(s[1][0], s[1][1]);
                p.w = pack2<S::kBf16>(s[1][2], s[1][3]);
            }
            // ---- weights times values: key 2 c, 2 c + 1 (and + 8) of the product are the columns of the scores ----
            const uint32_t v_base = smem_u32(values);
            const int v_row = group * 16 + ((lane >> 3) & 1) * 8 + S::key_of(lane & 7);
#pragma unroll
            for (int i = 0; i < S::kChunks / 2; ++i) {
                uint32_t w[4];
                ldmatrix4_trans(w, v_base + S::place(v_row, 2 * i + (lane >> 4)));
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if constexpr (S::kEight) {
                        uint32_t even0, odd0, even1, odd1;
                        widen<KV, 2>(w[2 * h], even0, odd0);
                        widen<KV, 2>(w[2 * h + 1], even1, odd1);
                        mma16816<S::kBf16>(o[2 * (2 * i + h)], p, even0, even1);
                        mma16816<S::kBf16>(o[2 * (2 * i + h) + 1], p, odd0, odd1);
                    } else {
                        mma16816<S::kBf16>(o[2 * i + h], p, w[2 * h], w[2 * h + 1]);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty_bar[stage]);
            if (++stage == S::kStages) { stage = 0; ++use; }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            sum[h] += __shfl_xor_sync(kFullMask, sum[h], 1);
            sum[h] += __shfl_xor_sync(kFullMask, sum[h], 2);
        }
        // ---- the four groups' states become one: groups 2, 3 into 0, 1, then 1 into 0 ----
#pragma unroll
        for (int step = kGroups / 2; step > 0; step >>= 1) {
            compute_sync<kCompute>();  // (whoever read the place before is done)
            if (group >= step && group < 2 * step) {
                float* to = merge + ((group - step) * MT + mt) * 16 * (D + 2) + lane;
#pragma unroll
                for (int n = 0; n < D / 8; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) to[(n * 4 + j) * 32] = o[n][j];
                if (c == 0) {
                    float* ml = merge + ((group - step) * MT + mt) * 16 * (D + 2) + 16 * D;
                    ml[r0] = top[0];
                    ml[r0 + 8] = top[1];
                    ml[16 + r0] = sum[0];
                    ml[16 + r0 + 8] = sum[1];
                }
            }
            compute_sync<kCompute>();
            if (group < step) {
                const float* from = merge + (group * MT + mt) * 16 * (D + 2);
                float keep[2], take[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float other = from[16 * D + r0 + 8 * h], higher = fmaxf(top[h], other);
                    keep[h] = top[h] == -INFINITY ? 0.0f : exp2_of(top[h] - higher);
                    take[h] = other == -INFINITY ? 0.0f : exp2_of(other - higher);
                    sum[h] = sum[h] * keep[h] + from[16 * D + 16 + r0 + 8 * h] * take[h];
                    top[h] = higher;
                }
#pragma unroll
                for (int n = 0; n < D / 8; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[n][j] = o[n][j] * keep[j >> 1] + from[lane + (n * 4 + j) * 32] * take[j >> 1];
            }
        }
        if (group == 0) {
            const bool whole = g.tile0 == 0 && g.tile1 == g.tiles;
            const long long slot = static_cast<long long>(blockIdx.x) + static_cast<long long>(g.unit) * a.cache.n_kv + g.head;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = mt * 16 + r0 + 8 * h, query = block * S::kQueries + row, i = query / a.group;
                if (i >= a.rows) continue;
                const float by = whole ? (sum[h] == 0.0f ? 0.0f : __fdividef(1.0f, sum[h])) : 1.0f;
                const size_t at = ((static_cast<size_t>(b) * a.rows + i) * a.n_heads + g.head * a.group + query - i * a.group) * D;
                float* part = a.partial + (slot * S::kQueries + row) * D;
                if (!whole && c == 0) a.partial_ml[slot * S::kQueries + row] = make_float2(top[h], sum[h]);
#pragma unroll
                for (int n = 0; n < D / 8; n += 2) {
                    // 8-bit rows: tiles n, n + 1 hold the even and the odd dims of 16; 16-bit rows: 8 dims each
                    if constexpr (S::kEight) {
                        const float v[4] = {o[n][2 * h] * by, o[n + 1][2 * h] * by, o[n][2 * h + 1] * by, o[n + 1][2 * h + 1] * by};
                        const int dim = 8 * n + 4 * c;
                        if (!whole) *reinterpret_cast<float4*>(part + dim) = *reinterpret_cast<const float4*>(v);
                        else if (a.q_bf16) store_row(static_cast<__nv_bfloat16*>(a.out) + at + dim, true, v);
                        else store_row(static_cast<__half*>(a.out) + at + dim, true, v);
                    } else {
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            const int dim = 8 * (n + m) + 2 * c;
                            const float x = o[n + m][2 * h] * by, y = o[n + m][2 * h + 1] * by;
                            if (!whole) *reinterpret_cast<float2*>(part + dim) = make_float2(x, y);
                            else if (a.q_bf16) *reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(a.out) + at + dim) = pack2<true>(x, y);
                            else *reinterpret_cast<uint32_t*>(static_cast<__half*>(a.out) + at + dim) = pack2<false>(x, y);
                        }
                    }
                }
            }
        }
        compute_sync<kCompute>();  // (the queries' place is free for the next segment's)
    } while (run.next(a));
    if (limit != kSpinLimit && lane == 0) atomicCAS(&g_paged_error, 0, 2);
}

// Joins the states of a segment that several CTAs had, in their order; a segment without a key gets its zeros here.  SHARE warps of
// a CTA have one query: they take its pieces in turn, eight at a time with all their loads in flight.  Where segments are few, and
// have many pieces, four warps to a query (17 pieces, one after the other in a warp: 14.6 us for the whole call, so 11.6), else one
// (384 segments of seven queries: 37 us for the whole call, 40 with four).
template <int D, int QT, int SHARE>
__global__ void __launch_bounds__(128)
join_kernel(const __grid_constant__ AttnArgs a) {
    constexpr int kPer = D / 32, kBatch = 8, kWarps = 4;
    __shared__ long long counts[2 * kWarps];
    __shared__ float states[SHARE][D + 2];
    pdl_trigger();
    const int unit = blockIdx.x / a.cache.n_kv, head = blockIdx.x - unit * a.cache.n_kv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = unit / a.blocks, block = unit - b * a.blocks;
    const int row = blockIdx.y * (kWarps / SHARE) + warp / SHARE, query = block * QT + row, i = query / a.group;
    // (the lengths may be read ahead of the wait: the kernel in front lets this one start behind its own wait only)
    const int limit = unit_limit<QT>(a, unit), tiles = (limit + kTileKeys - 1) / kTileKeys;
    long long total = 0, front = 0;
    {  // tiles of all units, and of those before this one
        long long all = 0, mine = 0;
        for (int u = threadIdx.x; u < a.units; u += 32 * kWarps) {
            const int n = (unit_limit<QT>(a, u) + kTileKeys - 1) / kTileKeys;
            all += n;
            if (u < unit) mine += n;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            all += __shfl_xor_sync(kFullMask, all, o);
            mine += __shfl_xor_sync(kFullMask, mine, o);
        }
        if (lane == 0) {
            counts[warp] = all;
            counts[kWarps + warp] = mine;
        }
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) {
            total += counts[w];
            front += counts[kWarps + w];
        }
        total *= a.cache.n_kv;
        front = front * a.cache.n_kv + static_cast<long long>(head) * tiles;
    }
    if (row >= QT || i >= a.rows) return;
    pdl_wait();
    const size_t at = ((static_cast<size_t>(b) * a.rows + i) * a.n_heads + head * a.group + query - i * a.group) * D;
    float v[kPer] = {}, top = -INFINITY, sum = 0.0f;
    if (tiles > 0) {
        const int ctas = ctas_of(total, a.grid), first = owner_of(total, front, ctas), last = owner_of(total, front + tiles - 1, ctas);
        if (first == last) return;  // (written by the CTA that had all of it)
        const long long slot0 = static_cast<long long>(unit) * a.cache.n_kv + head;
        for (int p0 = first + warp % SHARE; p0 <= last; p0 += SHARE * kBatch) {
            float2 ml[kBatch];
            float part[kBatch][kPer];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int p = p0 + k * SHARE;
                ml[k] = make_float2(-INFINITY, 0.0f);
                if (p <= last) {
                    ml[k] = a.partial_ml[(slot0 + p) * QT + row];
                    const float* from = a.partial + ((slot0 + p) * QT + row) * D + kPer * lane;
#pragma unroll
                    for (int j = 0; j < kPer; ++j) part[k][j] = from[j];
                }
            }
            float higher = top;
#pragma unroll
            for (int k = 0; k < kBatch; ++k) higher = fmaxf(higher, ml[k].x);
            const float keep = top == -INFINITY ? 0.0f : exp2_of(top - higher);
            sum *= keep;
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[j] *= keep;
            top = higher;
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (p0 + k * SHARE > last) continue;
                const float w = ml[k].x == -INFINITY ? 0.0f : exp2_of(ml[k].x - top);
                sum = fmaf(w, ml[k].y, sum);
#pragma unroll
                for (int j = 0; j < kPer; ++j) v[j] = fmaf(w, part[k][j], v[j]);
            }
        }
    }
    if constexpr (SHARE > 1) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) states[warp][kPer * lane + j] = v[j];
        if (lane == 0) {
            states[warp][D] = top;
            states[warp][D + 1] = sum;
        }
        __syncthreads();
        if (warp > 0) return;
        top = -INFINITY;
        sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kPer; ++j) v[j] = 0.0f;
#pragma unroll
        for (int k = 0; k < SHARE; ++k) top = fmaxf(top, states[k][D]);
#pragma unroll
        for (int k = 0; k < SHARE; ++k) {
            const float w = states[k][D] == -INFINITY ? 0.0f : exp2_of(states[k][D] - top);
            sum = fmaf(w, states[k][D + 1], sum);
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[j] = fmaf(w, states[k][kPer * lane + j], v[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if (sum != 0.0f) v[j] = __fdividef(v[j], sum);  // (a NaN stays; a row without a key has zeros)
        if (a.q_bf16) static_cast<__nv_bfloat16*>(a.out)[at + kPer * lane + j] = __float2bfloat16_rn(v[j]);
        else static_cast<__half*>(a.out)[at + kPer * lane + j] = __float2half_rn(v[j]);
    }
}

// 16-query tiles of a block: two where the queries of a (sequence, KV head) are more than sixteen.  (Four do not fit: sixteen
// warps and the one that fetches leave 96 registers to a thread, and 64 of them are the weighted sum.)
int query_tiles(int rows, int group) { return static_cast<long long>(rows) * group <= 16 ? 1 : 2; }

size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

// The pool as planes [page, K or V, head] of page_size rows, fetched in boxes of 32 rows (128 bytes of each, or the whole row).
int rows_map(const AttnArgs& a, bool eight, int d, int box_bytes, CUtensorMap* out) {
    const int bytes = eight ? 1 : 2;
    const unsigned long long page = 1ull << a.cache.page_shift, planes = 2ull * a.cache.pages * a.cache.n_kv;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(d), page, planes};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(d) * bytes, page * d * bytes};
    const cuuint32_t box[3] = {static_cast<cuuint32_t>(box_bytes / bytes), 32, 1};
    return encode_map(eight ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, a.pool, dims, strides, box,
                      box_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, out);
}

template <int D, int KV, int MT>
int launch(const AttnArgs& args, cudaStream_t stream) {
    using S = Shape<D, KV, MT>;
    static std::atomic<unsigned long long> configured{0};
    int status = allow_shared_memory(configured, paged_attention_kernel<D, KV, MT>, S::kSmem);
    if (status != SPEC_OK) return status;
    AttnArgs a = args;
    a.grid = 148 * S::kPerSm;
    CUtensorMap map;
    status = rows_map(a, S::kEight, D, S::kBoxBytes, &map);
    if (status != SPEC_OK) return status;
    status = launch_pdl(paged_attention_kernel<D, KV, MT>, dim3(a.grid), dim3(S::kThreads), S::kSmem, stream, map, a);
    if (status != SPEC_OK) return status;
    const int segments = a.units * a.cache.n_kv, queries = static_cast<int>(std::min<long long>(S::kQueries, static_cast<long long>(a.rows) * a.group));
    if (segments * 4 <= a.grid) return launch_pdl(join_kernel<D, S::kQueries, 4>, dim3(segments, queries), dim3(128), 0, stream, a);
    return launch_pdl(join_kernel<D, S::kQueries, 1>, dim3(segments, (queries + 3) / 4), dim3(128), 0, stream, a);
}

template <int D, int KV>
int launch_tiles(const AttnArgs& a, cudaStream_t stream) {
    return query_tiles(a.rows, a.group) == 1 ? launch<D, KV, 1>(a, stream) : launch<D, KV, 2>(a, stream);
}

template <int D>
int launch_kv(const AttnArgs& a, int kv_dtype, cudaStream_t stream) {
    switch (kv_dtype) {
        case SPEC_DTYPE_FP16: return launch_tiles<D, SPEC_DTYPE_FP16>(a, stream);
        case SPEC_DTYPE_BF16: return launch_tiles<D, SPEC_DTYPE_BF16>(a, stream);
        case SPEC_DTYPE_E4M3: return launch_tiles<D, SPEC_DTYPE_E4M3>(a, stream);
        default: return launch_tiles<D, SPEC_DTYPE_INT8>(a, stream);
    }
}

bool fits(int batch, int rows, int n_heads, int n_kv_heads, int d_head) {
    return batch >= 1 && batch <= 65535 && rows >= 1 && rows <= 65536 && n_kv_heads >= 1 && n_kv_heads <= 1024 && n_heads >= n_kv_heads &&
           n_heads % n_kv_heads == 0 && n_heads <= 65536 && (d_head == 64 || d_head == 128);
}
long long units_of(int batch, int rows, int group, int queries) { return static_cast<long long>(batch) * ((static_cast<long long>(rows) * group + queries - 1) / queries); }

}  // namespace

int paged_attention_take_error() {
    int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_paged_error, sizeof(int)) != cudaSuccess) return -1;
    if (v) cudaMemcpyToSymbol(g_paged_error, &zero, sizeof(int));
    return v;
}

}  // namespace spec

extern "C" size_t spec_paged_attention_workspace_bytes(int batch, int rows, int n_heads, int n_kv_heads, int d_head) {
    using namespace spec;
    if (!fits(batch, rows, n_heads, n_kv_heads, d_head)) return 0;
    const int group = n_heads / n_kv_heads, queries = 16 * query_tiles(rows, group);
    const size_t slots = kMostCtas + static_cast<size_t>(units_of(batch, rows, group, queries)) * n_kv_heads;
    return align256(slots * queries * d_head * 4) + align256(slots * queries * 8);
}

extern "C" int spec_paged_attention(const void* q, int dtype, int64_t q_stride, const void* pool, const float* scales, int kv_dtype, int pages,
                                    int page_size, const int32_t* page_table, int max_pages, const int32_t* lengths, int batch, int rows, int n_heads,
                                    int n_kv_heads, int d_head, float scale, void* out, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace spec;
    const char* who = "spec_paged_attention";
    if (dtype != SPEC_DTYPE_BF16 && dtype != SPEC_DTYPE_FP16) return fail(SPEC_ERR_BAD_ARG, "%s: dtype %d (bf16 or fp16)", who, dtype);
    if (rows < 0 || batch < 0) return fail(SPEC_ERR_BAD_ARG, "%s: batch=%d rows=%d", who, batch, rows);
    if (rows == 0 || batch == 0) return SPEC_OK;
    if (!fits(batch, rows, n_heads, n_kv_heads, d_head)) return fail(SPEC_ERR_BAD_ARG, "%s: batch=%d rows=%d n_heads=%d n_kv_heads=%d d_head=%d", who, batch, rows, n_heads, n_kv_heads, d_head);
    AttnArgs a{};
    const int status = check_paged(who, pool, scales, kv_dtype, pages, page_size, n_kv_heads, d_head, page_table, max_pages, batch, &a.cache);
    if (status != SPEC_OK) return status;
    if ((kv_dtype == SPEC_DTYPE_FP16 || kv_dtype == SPEC_DTYPE_BF16) && kv_dtype != dtype) return fail(SPEC_ERR_BAD_ARG, "%s: a 16-bit cache needs queries of its own type", who);
    if (!(scale > -3.0e38f && scale < 3.0e38f)) return fail(SPEC_ERR_BAD_ARG, "%s: scale must be finite", who);
    if (!q || !out || !lengths) return fail(SPEC_ERR_BAD_ARG, "%s: null pointer", who);
    if (!aligned_to(q, 8) || !aligned_to(out, 8) || q_stride % 4 || !aligned_to(lengths, 4)) return fail(SPEC_ERR_BAD_ARG, "%s: q and out have to start on 8 bytes, q's rows too", who);
    if (q_stride < static_cast<int64_t>(n_heads) * d_head) return fail(SPEC_ERR_BAD_ARG, "%s: q's row stride is below the heads' elements", who);
    if (scales && !aligned_to(scales, 16)) return fail(SPEC_ERR_BAD_ARG, "%s: scales have to start on 16 bytes", who);
    if (static_cast<long long>(pages) * 2 * n_kv_heads > 0x7fffffffll) return fail(SPEC_ERR_BAD_ARG, "%s: pages=%d", who, pages);
    a.group = n_heads / n_kv_heads;
    const int queries = 16 * query_tiles(rows, a.group);
    const long long units = units_of(batch, rows, a.group, queries);
    if (units * n_kv_heads > 0x7fffffff - kMostCtas) return fail(SPEC_ERR_BAD_ARG, "%s: too many rows for one call", who);
    if (!workspace || workspace_bytes < spec_paged_attention_workspace_bytes(batch, rows, n_heads, n_kv_heads, d_head) || !aligned_to(workspace, 256))
        return fail(SPEC_ERR_BAD_ARG, "%s: workspace missing, too small or not 256-byte aligned", who);
    const size_t slots = kMostCtas + static_cast<size_t>(units) * n_kv_heads;
    a.pool = pool;
    a.scales = scales;
    a.q = q;
    a.out = out;
    a.lengths = lengths;
    a.partial = static_cast<float*>(workspace);
    a.partial_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + align256(slots * queries * d_head * 4));
    a.q_stride = q_stride;
    a.scale = scale;
    a.batch = batch;
    a.rows = rows;
    a.n_heads = n_heads;
    a.units = static_cast<int>(units);
    a.blocks = a.units / batch;
    a.q_bf16 = dtype == SPEC_DTYPE_BF16;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return d_head == 64 ? launch_kv<64>(a, kv_dtype, st) : launch_kv<128>(a, kv_dtype, st);
}
