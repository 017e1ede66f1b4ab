// Attention of the few new tokens of every sequence (one, or the gamma + 1 rows of a verification pass) over its paged K,V rows:
//   S_j = scale * q . k_j for the keys j at or before the row's position,  o = sum_j softmax(S)_j v_j.
//
// Bound by the cached rows' bytes: they are read once for all queries of a KV head, as they lie (8 bits or 16), and widened in
// registers on their way into mma.sync (M = 16 queries, fp16 or, for bf16 caches, bf16; sums fp32).  Scales of 8-bit rows stay
// outside the products: with k_j = sk_j kc_j and v_j = sv_j vc_j,
//   S_j = (scale sk_j)(q . kc_j),   o = sum_j w_j vc_j / sum_j w_j / sv_j   with w_j = exp(S_j) sv_j = 2^(S_j log2 e + log2 sv_j):
// the running maximum is taken of the latter exponent, so that w_j, which is rounded to fp16 for the second product, is at most
// about 1 whatever the scales are, and one exponential per score serves both sums.  What fp16 takes from a small w_j is small beside what
// the largest one adds; rows of zeros, which add nothing, are kept out of the maximum (kScaleOfZeros).
//
// Work: tiles of 64 keys of a segment (sequence, block of queries, KV head).  The lengths are known on the device only, so every
// CTA adds them up and takes an equal, contiguous run of all slots (the longest sequence does not decide, whatever the capacity of
// the page table): a segment has a slot per tile and kSwitch more in front of them, since the CTAs with many short segments decide
// else.  A segment that several CTAs share leaves (maximum, sum, weighted rows) per CTA in the workspace, and a second
// kernel joins them in order.  No atomics: the same bits every time.
//
// More than 32 queries to a KV head: paged_attention_wide.cuh.  Up to there a CTA has four warps, each with 16 of a tile's 64 keys and all
// queries of the block, 8, 16 or 32.  The keys take the M side of both
// products (scores [key][query], weighted rows [dim][query]): queries come in eights then, and a K or V fragment is widened once
// for all of them.  (Queries on the M side, sixteen at least: twice the multiplications and registers for a lone token of four
// heads.)  One more warp asks for the tiles of the whole run, segment after segment, by TMA (halves of 32 keys, which never straddle a
// page, with the shared-memory swizzle) through a ring of stages with a barrier to fill and one to free each; a warp's queries
// are on their way a segment ahead.  The four never wait for one another within a segment.
#include <algorithm>

#include "paged.cuh"
#include "tc_util.cuh"

namespace spec {
namespace {

using namespace tc;

constexpr int kTileKeys = 64;
constexpr int kWarps = 4;        // that compute, with 16 of a tile's keys each
// CTAs of a launch whose blocks have so many queries, at most.
constexpr int most_ctas(int queries) { return 148 * (queries == 8 ? 5 : queries == 16 ? 3 : 2); }
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kSwitch = 3;       // tiles that taking up another segment costs about as much as
constexpr float kNone = -3.0e38f;  // the running maximum where no key has been seen: finite, so that differences stay numbers
// What a V row of zeros is taken to have for a scale, for the 1 that it is stored with, which says nothing and would let such a row set the
// maximum (beside a sink of zeros that led by ten, rows with scales of 2^-12 had weights among fp16's subnormals: outputs off by 7 %).
// Small, so that a row whose scale is s loses nothing to one that leads by 2^(78 + log2 s), and not smaller, since weights below 2^-126
// of the largest are none: beside rows of a scale s, zeros with 2^(log2 s - 62) of their weight and less leave the sum.
constexpr float kScaleOfZeros = 0x1p-64f;
constexpr float kSlack = 8.0f;   // the running maximum may lag by this: w <= 2^8 stays in fp16's range

__device__ int g_paged_error;  // set when the bounded wait for a tile or for its place ran out (0 = none)

struct AttnArgs {
    Paged cache;
    const void* pool;
    const float* scales;
    const void* q;
    void* out;
    const int32_t* lengths;
    // Of each CTA two places: for the segment that began before its run, and for the one that goes on behind it.
    float* partial;      // [CTA][2][queries of a block][D]
    float2* partial_ml;  // [CTA][2][queries of a block]: maximum, sum
    long long q_stride;
    float scale;
    int rows, n_heads, group, blocks, units;  // blocks: of queries per (sequence, KV head); units = batch * blocks
    int q_bf16, q_wide /* q's rows start on 16 bytes */, grid;
    uint32_t by_group;  // ceil(2^32 / group) for groups of two and more
    // The token of a query of a (sequence, KV head); exact, since query * group stays below 2^31.
    __device__ __forceinline__ int token_of(int query) const { return group == 1 ? query : static_cast<int>(__umulhi(static_cast<uint32_t>(query), by_group)); }
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
__device__ __forceinline__ void copy8(void* to, const void* from, bool there) {  // (zeros where there is nothing)
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(there ? 8 : 0) : "memory");
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
__device__ __forceinline__ uint32_t transposed(uint32_t v) {  // an 8 x 8 tile of 16-bit values across the warp
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
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

// Non-zero where a code among 16 bytes of an 8-bit row is not a zero.
template <int KV>
__device__ __forceinline__ uint32_t some_code(const uint4& v) {
    return (v.x | v.y | v.z | v.w) & (KV == SPEC_DTYPE_E4M3 ? 0x7f7f7f7fu : 0xffffffffu);  // (e4m3 has a negative zero)
}

// Keys of a unit (sequence, block of queries): those up to the position of the block's last row.
template <int QT>
__device__ __forceinline__ int unit_limit(const AttnArgs& a, int unit) {
    const int b = a.blocks == 1 ? unit : unit / a.blocks, block = unit - b * a.blocks;
    const int capacity = a.cache.width << a.cache.page_shift;
    const int length = a.lengths[b];
    const int last_row = min(a.rows - 1, a.token_of(block * QT + QT - 1));
    return min(max(0, max(length, 0) - (a.rows - 1 - last_row)), capacity);
}
// Slots of a (unit, KV head): its tiles, and kSwitch more for taking it up, if there are any.
__device__ __forceinline__ int unit_slots(int limit) { return limit > 0 ? (limit + kTileKeys - 1) / kTileKeys + kSwitch : 0; }

// How all slots are shared out: CTA c has the run [first(c), first(c + 1)).
struct Shares {
    int total, ctas, each, more;  // `more` CTAs have one slot above `each`
    __device__ __forceinline__ Shares(int sum, int grid) : total(sum), ctas(max(1, min(sum, grid))) {
        each = static_cast<int>(static_cast<uint32_t>(sum) / static_cast<uint32_t>(ctas));
        more = sum - each * ctas;
    }
    __device__ __forceinline__ int first(int cta) const { return cta * each + min(cta, more); }
    __device__ __forceinline__ int owner(int slot) const {
        const int large = more * (each + 1);
        return slot < large ? static_cast<int>(static_cast<uint32_t>(slot) / static_cast<uint32_t>(each + 1))
                            : more + static_cast<int>(static_cast<uint32_t>(slot - large) / static_cast<uint32_t>(each));
    }
};

// The sum of all units' slots (times the KV heads), and the unit in which this CTA's run begins (-1: it has none) with the slots of one
// KV head before it.  All threads of the block; `scratch`: 24 ints.
template <int QT>
__device__ __forceinline__ int find_unit(const AttnArgs& a, int* scratch, int& unit, int& before) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    if (a.units <= 32) {  // every warp for itself
        const int mine = lane < a.units ? unit_slots(unit_limit<QT>(a, lane)) : 0;
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(kFullMask, upto, o);
            if (lane >= o) upto += up;
        }
        const int total = __shfl_sync(kFullMask, upto, 31) * a.cache.n_kv;
        const Shares shares(total, a.grid);
        unit = -1;
        if (total == 0 || static_cast<int>(blockIdx.x) >= shares.ctas) return total;
        unit = __ffs(__ballot_sync(kFullMask, shares.first(blockIdx.x) < upto * a.cache.n_kv)) - 1;
        before = __shfl_sync(kFullMask, upto - mine, unit);
        return total;
    }
    const bool fits = a.units <= static_cast<int>(blockDim.x);  // (else: add up first, look then)
    int total = 0, target = 0, base = 0;
    unit = -1;
    for (int round = fits ? 1 : 0; round < 2; ++round) {
        if (round == 1 && !fits) {
            total = base * a.cache.n_kv;
            target = Shares(total, a.grid).first(blockIdx.x);
            base = 0;
        }
        for (int u0 = 0; u0 < a.units; u0 += blockDim.x) {
            const int u = u0 + threadIdx.x;
            const int mine = u < a.units ? unit_slots(unit_limit<QT>(a, u)) : 0;
            int upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int up = __shfl_up_sync(kFullMask, upto, o);
                if (lane >= o) upto += up;
            }
            __syncthreads();  // (scratch is free)
            if (lane == 31) scratch[warp] = upto;
            __syncthreads();
            int all = 0, front = 0;
            for (int w = 0; w < warps; ++w) {
                if (w < warp) front += scratch[w];
                all += scratch[w];
            }
            upto += base + front;
            if (round == 1) {
                if (fits) {
                    total = all * a.cache.n_kv;
                    target = Shares(total, a.grid).first(blockIdx.x);
                }
                if ((upto - mine) * a.cache.n_kv <= target && target < upto * a.cache.n_kv) {
                    scratch[16] = u;
                    scratch[17] = upto - mine;
                }
            }
            base += all;
        }
    }
    if (static_cast<int>(blockIdx.x) >= Shares(total, a.grid).ctas || total == 0) return total;
    __syncthreads();
    unit = scratch[16];
    before = scratch[17];
    return total;
}

template <int D, int KV, int NT>
struct Shape {
    static constexpr bool kEight = KV == SPEC_DTYPE_E4M3 || KV == SPEC_DTYPE_INT8;
    static constexpr bool kBf16 = KV == SPEC_DTYPE_BF16;
    static constexpr int kRowBytes = D * (kEight ? 1 : 2);
    static constexpr int kBoxBytes = kRowBytes < 128 ? kRowBytes : 128;  // of a row in one copy: what the swizzle spans
    static constexpr int kBoxes = kRowBytes / kBoxBytes;
    static constexpr int kChunks = kRowBytes / 16;
    static constexpr int kQueries = 8 * NT;
    // The warp that fetches is one more; 32 queries of 128 dims need more registers than two CTAs of five warps leave to a thread
    // (168), so there it is one of four, whose registers the others take over.
    static constexpr bool kShift = D == 128 && NT == 4;
    static constexpr int kThreads = 32 * (kShift ? 2 * kWarps : kWarps + 1);
    static constexpr int kTaken = 224, kLeft = 32;  // registers then: their sum is twice the 128 of the launch
    static constexpr int kOperandBytes = kTileKeys * kRowBytes;  // K or V of a tile
    static constexpr int kStageBytes = 2 * kOperandBytes;
    static constexpr int kScaleBytes = kEight ? 2 * kTileKeys * 4 : 0;
    static constexpr int kQueryBytes = kQueries * D * 2;
    static constexpr int kJoined = NT < 2 ? NT : 2;             // eights of queries whose states are joined at a time
    static constexpr int kState = kJoined * 8 * (D + 2);        // floats of a warp's state of these
    // Few CTAs with a deep ring each read memory faster than many with a shallow one (16 x 32768 int8 tokens of 128 dims, floor 131
    // us: two CTAs to an SM and five stages 136, three and three 186, four and two 163; 32 x 8192 fp16 tokens of 64 dims, floor 93: two 101, three 118);
    // rows of 64 bytes leave more to compute for each byte (32 x 8192 int8, floor 50: three 90, four 76, five 69).
    static constexpr int kPerSm = NT == 4 || kRowBytes >= 128 ? 2 : NT == 1 ? 5 : 3;
    static_assert(148 * kPerSm <= most_ctas(kQueries), "room for every CTA's pieces");
    static constexpr int kFixed = 2 * kState * 4 + 2 * kQueryBytes + 2 * kQueries * 4 + 24 * 4 + 1024 /* alignment */ + 256 /* barriers, notes */;
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

// A CTA's run of slots, segment by segment.
template <int QT>
struct Run {
    int left;  // slots, from `at` of the present segment on
    int at, unit, head, tile0, tile1, tiles, limit;  // limit: keys before it exist for some row of the block
    __device__ __forceinline__ void open(const AttnArgs& a) {  // what follows from unit
        limit = unit_limit<QT>(a, unit);
        tiles = (limit + kTileKeys - 1) / kTileKeys;
    }
    // The tiles of the present segment; false: the run ends ahead of the first.
    __device__ __forceinline__ bool take() {
        tile0 = max(0, at - kSwitch);
        tile1 = min(tiles, at + left - kSwitch);
        return tile1 > tile0;
    }
    __device__ __forceinline__ bool next(const AttnArgs& a) {
        left -= tiles + kSwitch - at;
        if (left <= kSwitch) return false;
        at = 0;
        if (++head == a.cache.n_kv) {
            head = 0;
            do {
                if (++unit >= a.units) return false;
                open(a);
            } while (limit == 0);
        }
        return take();
    }
};

__device__ __forceinline__ void compute_sync() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory"); }

template <int D, int KV, int NT>
__global__ void __launch_bounds__(Shape<D, KV, NT>::kThreads, Shape<D, KV, NT>::kPerSm)
paged_attention_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ AttnArgs a) {
    using S = Shape<D, KV, NT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    float* ring_scales = reinterpret_cast<float*>(ring + S::kStages * S::kStageBytes);  // [stage][K, V][64]
    float* merge = reinterpret_cast<float*>(ring + S::kStages * (S::kStageBytes + S::kScaleBytes));  // [2] states
    // Queries of this and of the next segment: rows as they came, then [NT][D / 32][32 lanes] in the order in which the products take them.
    uint8_t* queries = reinterpret_cast<uint8_t*>(merge + 2 * S::kState);
    float* query_factor = reinterpret_cast<float*>(queries + 2 * S::kQueryBytes);  // [2][row]: what a row's products are multiplied with
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(query_factor + 2 * S::kQueries);
    uint64_t* empty_bar = full_bar + S::kStages;
    int* notes = reinterpret_cast<int*>(empty_bar + S::kStages);  // [stage]: keys of the tile that there are, and which of its halves were fetched
    int* scratch = notes + S::kStages;                            // [24]

    const int warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(&full_bar[s], 1);
            mbar_init(&empty_bar[s], kWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    pdl_trigger();  // (behind the wait: the joining kernel reads the lengths ahead of its own)

    int unit, before;
    const Shares shares(find_unit<S::kQueries>(a, scratch, unit, before), a.grid);
    if (unit < 0) return;  // (more CTAs than slots)
    Run<S::kQueries> run;
    {
        const int first = shares.first(blockIdx.x), within = first - before * a.cache.n_kv;
        run.left = shares.first(blockIdx.x + 1) - first;
        run.unit = unit;
        run.open(a);
        const int slots = run.tiles + kSwitch;
        run.head = static_cast<int>(static_cast<uint32_t>(within) / static_cast<uint32_t>(slots));
        run.at = within - run.head * slots;
    }
    if (!run.take()) return;
    __syncthreads();  // (barriers are there for all)
    uint32_t limit = kSpinLimit;  // of every wait; one that has run out leaves one try to the others, and the CTA ends with its error noted

    if (warp >= kWarps) {
        if constexpr (S::kShift) {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kLeft));
            if (warp > kWarps) return;
        }
        // ---- the tiles of the whole run, through the ring: halves of 32 keys, which lie in one page each ----
        const bool leader = elect_one();
        int stage = 0, use = 0;
        do {
            const int b = a.blocks == 1 ? run.unit : run.unit / a.blocks;
            const int32_t* pages = a.cache.table + static_cast<size_t>(b) * a.cache.width;
            for (int t = run.tile0; t < run.tile1; ++t) {
                int page[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int key = t * kTileKeys + 32 * h;
                    page[h] = key < run.limit ? pages[key >> a.cache.page_shift] : -1;
                    if (page[h] >= a.cache.pages) page[h] = -1;
                }
                if (use > 0 && !mbar_wait_warp(&empty_bar[stage], (use - 1) & 1, limit)) limit = 1;
                if (leader) {
                    const int halves = (page[0] >= 0 ? 1 : 0) + (page[1] >= 0 ? 1 : 0);
                    notes[stage] = min(kTileKeys, run.limit - t * kTileKeys) | (page[0] >= 0 ? 256 : 0) | (page[1] >= 0 ? 512 : 0);
                    mbar_expect_tx(&full_bar[stage], halves * (S::kStageBytes + S::kScaleBytes) / 2);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (page[h] < 0) continue;
                        const int slot = (t * kTileKeys + 32 * h) & ((1 << a.cache.page_shift) - 1);
#pragma unroll
                        for (int which = 0; which < 2; ++which) {
                            const int plane = (page[h] * 2 + which) * a.cache.n_kv + run.head;
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

    if constexpr (S::kShift) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kTaken));
    const int r0 = lane >> 2, c = lane & 3;
    constexpr int kRows = S::kQueries / kWarps;  // queries that a warp fetches and prepares: warp, warp + 4, ..
    const auto fetch_queries = [&](const Run<S::kQueries>& of, int turn) {
        const int b = a.blocks == 1 ? of.unit : of.unit / a.blocks, block = of.unit - b * a.blocks;
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            const int row = warp + j * kWarps, query = block * S::kQueries + row, token = a.token_of(query);
            const bool there = token < a.rows;
            const size_t at = (static_cast<size_t>(b) * a.rows + token) * a.q_stride + (of.head * a.group + query - token * a.group) * D + 4 * lane;
            if (lane < D / 4) copy8(queries + turn * S::kQueryBytes + row * (2 * D) + 8 * lane, static_cast<const uint16_t*>(a.q) + (there ? at : 0), there);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int stage = 0, use = 0, turn = 0;
    fetch_queries(run, 0);
    while (true) {
        const int b = a.blocks == 1 ? run.unit : run.unit / a.blocks, block = run.unit - b * a.blocks;
        const int length = max(a.lengths[b], 0);
        Run<S::kQueries> ahead = run;
        const bool more = ahead.next(a);

        // ---- the block's queries ----
        // Lane c of a quad reads dims E (4 i + c) + 4 s .. + 3 of a key row (E elements to 16 bytes), so step E/4 i + s of the
        // product takes the same dims of the query.  bf16 rows for fp16 products are brought to a largest magnitude in [1, 2) by a power
        // of two; fp16 rows are taken as they are (their small elements would lose bits so).
        constexpr int E = 16 / (S::kRowBytes / D), kPerChunk = E / 4;
        const uint4* q_frag = reinterpret_cast<const uint4*>(queries + turn * S::kQueryBytes);
        const float* q_factor = query_factor + turn * S::kQueries;
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
        uint32_t packed[kRows][2];
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            const int row = warp + j * kWarps;
            float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (lane < D / 4) {
                const uint8_t* from = queries + turn * S::kQueryBytes + row * (2 * D) + 8 * lane;
                if (a.q_bf16) load_row(reinterpret_cast<const __nv_bfloat16*>(from), true, v);
                else load_row(reinterpret_cast<const __half*>(from), true, v);
            }
            float back = 1.0f;
            if (!S::kBf16 && a.q_bf16) {
                uint32_t largest = 0u;
#pragma unroll
                for (int i = 0; i < 4; ++i) largest = max(largest, magnitude(v[i]));
                largest = __reduce_max_sync(kFullMask, largest);
                if (largest != 0u && largest < 0x7f800000u) {
                    const int e = max(-120, min(120, static_cast<int>(largest >> 23) - 127));
                    back = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
                    const float by = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] *= by;
                }
            }
            packed[j][0] = pack2<S::kBf16>(v[0], v[1]);
            packed[j][1] = pack2<S::kBf16>(v[2], v[3]);
            if (lane == 0) query_factor[turn * S::kQueries + row] = back * a.scale * kLog2e;
        }
        compute_sync();  // (all rows are in registers: their place takes them in the other order)
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            const int row = warp + j * kWarps, dim = 4 * lane, chunk = dim / E, step = (chunk >> 2) * kPerChunk + (dim % E) / 4;
            if (lane < D / 4)
                *reinterpret_cast<uint2*>(queries + turn * S::kQueryBytes + (((row >> 3) * (D / 32) + (step >> 1)) * 32 + (row & 7) * 4 + (chunk & 3)) * 16 + (step & 1) * 8) =
                    make_uint2(packed[j][0], packed[j][1]);
        }
        compute_sync();
        if (more) fetch_queries(ahead, turn ^ 1);  // (the place of the segment before: all warps are behind its products)

        // (this thread's queries: 8 n + 2 c and the next, of each eight n)
        const int seen_by_all = max(-1, length - a.rows + min(a.rows - 1, a.token_of(block * S::kQueries)));

        float o[NT][D / 16][4], top[NT][2], sum[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int m = 0; m < D / 16; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[n][m][j] = 0.0f;
            top[n][0] = top[n][1] = kNone;
            sum[n][0] = sum[n][1] = 0.0f;
        }

        for (int t = run.tile0; t < run.tile1; ++t) {
            if (!mbar_wait_warp(&full_bar[stage], use & 1, limit)) limit = 1;
            const uint8_t* keys = ring + stage * S::kStageBytes;
            uint8_t* values = ring + stage * S::kStageBytes + S::kOperandBytes;
            const float* consts = ring_scales + stage * 2 * kTileKeys + warp * 16;
            const int note = notes[stage];
            // keys of this warp's sixteen that there are (they lie in one half of the tile)
            const int there = note & (warp >= kWarps / 2 ? 512 : 256) ? max(0, min(16, (note & 255) - 16 * warp)) : 0;
            const int first_key = t * kTileKeys + warp * 16;

            // A weight of zero does not hide a V row that is no number from the product.  Rows that are not there (left from
            // before, or of other sequences) are cleared; rows that some of the block's queries see and others do not are looked at,
            // and one with such a value is taken out and told to those who see it.
            const bool hidden = KV != SPEC_DTYPE_INT8 && first_key + 15 > seen_by_all && seen_by_all + 1 < run.limit;
            uint32_t bad = 0u;  // a bit per key
            if (KV != SPEC_DTYPE_INT8 && (there < 16 || hidden)) {
                if (hidden) {
                    for (int i = lane; i < 16 * S::kChunks; i += 32) {
                        const int r = i / S::kChunks;
                        if (r < there && not_numbers<KV>(*reinterpret_cast<const uint4*>(values + S::place(warp * 16 + r, i % S::kChunks)))) bad |= 1u << r;
                    }
                    bad = __reduce_or_sync(kFullMask, bad);
                }
                for (int i = lane; i < 16 * S::kChunks; i += 32) {
                    const int r = i / S::kChunks;
                    if (r >= there || (bad >> r & 1u)) *reinterpret_cast<uint4*>(values + S::place(warp * 16 + r, i % S::kChunks)) = make_uint4(0u, 0u, 0u, 0u);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // (before the next copy into this stage)
                __syncwarp();
            }

            // ---- scores: this thread's keys are key[0], key[1] ----
            const int key[2] = {S::key_of(r0), 8 + S::key_of(r0)};
            // (even and odd steps in sums of their own where queries are few: half as many products wait for one another)
            constexpr bool kApart = NT < 4;
            float s[NT][4], odd[kApart ? NT : 1][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[n][j] = odd[kApart ? n : 0][j] = 0.0f;
#pragma unroll
            for (int i = 0; i < S::kChunks / 4; ++i) {
                uint32_t w[2][4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 v = *reinterpret_cast<const uint4*>(keys + S::place(warp * 16 + key[h], 4 * i + c));
                    w[h][0] = v.x;
                    w[h][1] = v.y;
                    w[h][2] = v.z;
                    w[h][3] = v.w;
                }
#pragma unroll
                for (int k = 0; k < kPerChunk; k += 2) {
                    uint4 rows[2];  // of K, for two steps
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        if constexpr (S::kEight) {
                            widen<KV, 1>(w[0][k + e], rows[e].x, rows[e].z);
                            widen<KV, 1>(w[1][k + e], rows[e].y, rows[e].w);
                        } else {
                            rows[e] = make_uint4(w[0][2 * e], w[1][2 * e], w[0][2 * e + 1], w[1][2 * e + 1]);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const uint4 q = q_frag[(n * (D / 32) + (kPerChunk * i + k) / 2) * 32 + lane];
                        mma16816<S::kBf16>(s[n], rows[0], q.x, q.y);
                        mma16816<S::kBf16>(kApart ? odd[kApart ? n : 0] : s[n], rows[1], q.z, q.w);
                    }
                }
            }
            // ---- exponents, their running maximum, weights ----
            if constexpr (S::kEight) {
                // (written over where it lies, which this warp alone reads, and seldom; 32 sequences of 2048 tokens: up to 4.7 % longer at 64 dims, 2 %
                // shorter to 4 % longer at 128; with a branch among the exponents instead 9 % longer at 64)
                float* scale = ring_scales + (stage * 2 + 1) * kTileKeys + warp * 16 + (lane & 15);
                const bool one = *scale == 1.0f;
                if (__any_sync(kFullMask, one)) {
                    uint32_t some = one ? 0u : 1u;
                    if (one)
#pragma unroll 1
                        for (int x = 0; x < S::kChunks; ++x) some |= some_code<KV>(*reinterpret_cast<const uint4*>(values + S::place(warp * 16 + (lane & 15), x)));
                    __syncwarp();
                    if (some == 0u) *scale = kScaleOfZeros;
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // (before the next copy into this stage)
                    __syncwarp();
                }
            }
            float inv[2] = {1.0f, 1.0f};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float sk = 1.0f, raise = 0.0f;  // (the queries' factors are loaded anew for each tile: they would be two registers each)
                if constexpr (S::kEight) {
                    const float sv = consts[kTileKeys + key[h]];
                    sk = consts[key[h]];
                    raise = log2_of(sv);
                    inv[h] = reciprocal_of(sv);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float2 factor = *reinterpret_cast<const float2*>(q_factor + 8 * n + 2 * c);
                    float x = s[n][2 * h], y = s[n][2 * h + 1];
                    if constexpr (kApart) {
                        x += odd[n][2 * h];
                        y += odd[n][2 * h + 1];
                    }
                    s[n][2 * h] = S::kEight ? fmaf(x, sk * factor.x, raise) : x * factor.x;
                    s[n][2 * h + 1] = S::kEight ? fmaf(y, sk * factor.y, raise) : y * factor.y;
                }
            }
            if (there < 16 || first_key + 15 > seen_by_all) {  // keys that are not there, or not for every query
                bool number[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    number[h] = !(bad >> key[h] & 1u);
                    if constexpr (S::kEight) number[h] = number[h] && magnitude(consts[kTileKeys + key[h]]) < 0x7f800000u;
                    // (a row of V that is no number makes the exponent none for who sees it, and no one else's sum)
                    if (!number[h] || key[h] >= there) inv[h] = 0.0f;
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int i = a.token_of(block * S::kQueries + 8 * n + 2 * c + x);
                        const int seen = i < a.rows ? max(-1, length - a.rows + i) : -1;  // (a query that does not exist sees nothing)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float& e = s[n][2 * h + x];
                            if (!number[h]) e = NAN;
                            if (key[h] >= there || first_key + key[h] > seen) e = -INFINITY;
                        }
                    }
            }
            // The maximum is looked for only where some exponent has left the old one behind by more than the slack.
            bool higher = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int x = 0; x < 2; ++x) higher = higher || fmaxf(s[n][x], s[n][2 + x]) > top[n][x] + kSlack;
            if (__any_sync(kFullMask, higher)) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float shrink[2];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float most = fmaxf(top[n][x], fmaxf(s[n][x], s[n][2 + x]));
#pragma unroll
                        for (int lanes = 4; lanes < 32; lanes <<= 1) most = fmaxf(most, __shfl_xor_sync(kFullMask, most, lanes));
                        shrink[x] = exp2_of(top[n][x] - most);
                        top[n][x] = most;
                        sum[n][x] *= shrink[x];
                    }
#pragma unroll
                    for (int m = 0; m < D / 16; ++m)
#pragma unroll
                        for (int j = 0; j < 4; ++j) o[n][m][j] *= shrink[j & 1];
                }
            }
            uint32_t p[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float w = exp2_of(s[n][2 * h + x] - top[n][x]);
                        sum[n][x] = fmaf(w, inv[h], sum[n][x]);
                        s[n][2 * h + x] = w;
                    }
                    p[n][h] = transposed(pack2<S::kBf16>(s[n][2 * h], s[n][2 * h + 1]));
                }
            }
            // ---- values times weights: rows of V in the order of the keys above ----
            const uint32_t v_base = smem_u32(values);
            const int v_row = warp * 16 + ((lane >> 3) & 1) * 8 + S::key_of(lane & 7);
#pragma unroll
            for (int i = 0; i < S::kChunks / 2; ++i) {
                uint32_t w[4];  // two chunks of eight keys, twice
                ldmatrix4_trans(w, v_base + S::place(v_row, 2 * i + (lane >> 4)));
                if constexpr (S::kEight) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {  // a chunk is sixteen dims: the even ones are rows 0 .. 7 of the product, the odd ones 8 .. 15
                        uint4 v;
                        widen<KV, 2>(w[2 * h], v.x, v.y);
                        widen<KV, 2>(w[2 * h + 1], v.z, v.w);
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma16816<S::kBf16>(o[n][2 * i + h], v, p[n][0], p[n][1]);
                    }
                } else {
                    const uint4 v = make_uint4(w[0], w[2], w[1], w[3]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma16816<S::kBf16>(o[n][i], v, p[n][0], p[n][1]);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty_bar[stage]);
            if (++stage == S::kStages) { stage = 0; ++use; }
        }
        // ---- the four warps' states become one: warps 2, 3 into 0, 1, then 1 into 0 ----
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int lanes = 4; lanes < 32; lanes <<= 1) sum[n][x] += __shfl_xor_sync(kFullMask, sum[n][x], lanes);
#pragma unroll
        for (int n0 = 0; n0 < NT; n0 += S::kJoined) {
            constexpr int kElements = D / 16 * 4 * 32;  // of eight queries
            const auto leave = [&](float* to) {
#pragma unroll
                for (int n = 0; n < S::kJoined; ++n) {
#pragma unroll
                    for (int m = 0; m < D / 16; ++m)
                        reinterpret_cast<float4*>(to + n * kElements)[m * 32 + lane] = make_float4(o[n0 + n][m][0], o[n0 + n][m][1], o[n0 + n][m][2], o[n0 + n][m][3]);
                    if (r0 == 0) {
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            to[S::kJoined * kElements + 16 * n + 2 * c + x] = top[n0 + n][x];
                            to[S::kJoined * kElements + 16 * n + 8 + 2 * c + x] = sum[n0 + n][x];
                        }
                    }
                }
            };
            const auto join = [&](const float* from) {
#pragma unroll
                for (int n = 0; n < S::kJoined; ++n) {
                    float keep[2], take[2];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float &mine = top[n0 + n][x], other = from[S::kJoined * kElements + 16 * n + 2 * c + x];
                        const float most = fmaxf(mine, other);
                        keep[x] = exp2_of(mine - most);
                        take[x] = exp2_of(other - most);
                        sum[n0 + n][x] = sum[n0 + n][x] * keep[x] + from[S::kJoined * kElements + 16 * n + 8 + 2 * c + x] * take[x];
                        mine = most;
                    }
#pragma unroll
                    for (int m = 0; m < D / 16; ++m) {
                        const float4 v = reinterpret_cast<const float4*>(from + n * kElements)[m * 32 + lane];
                        o[n0 + n][m][0] = o[n0 + n][m][0] * keep[0] + v.x * take[0];
                        o[n0 + n][m][1] = o[n0 + n][m][1] * keep[1] + v.y * take[1];
                        o[n0 + n][m][2] = o[n0 + n][m][2] * keep[0] + v.z * take[0];
                        o[n0 + n][m][3] = o[n0 + n][m][3] * keep[1] + v.w * take[1];
                    }
                }
            };
            if (n0 > 0) compute_sync();  // (warp 0 has read the second place)
            if (warp >= 2) leave(merge + (warp - 2) * S::kState);
            compute_sync();
            if (warp < 2) join(merge + warp * S::kState);
            if (warp == 1) leave(merge + S::kState);
            compute_sync();
            if (warp == 0) join(merge + S::kState);
        }
        if (warp == 0) {
            const bool whole = run.tile0 == 0 && run.tile1 == run.tiles;
            const size_t slot = 2 * static_cast<size_t>(blockIdx.x) + (run.tile0 == 0 ? 1 : 0);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int row = 8 * n + 2 * c + x, query = block * S::kQueries + row, i = a.token_of(query);
                    if (i >= a.rows) continue;
                    const float by = whole ? (sum[n][x] == 0.0f ? 0.0f : reciprocal_of(sum[n][x])) : 1.0f;
                    const size_t at = ((static_cast<size_t>(b) * a.rows + i) * a.n_heads + run.head * a.group + query - i * a.group) * D;
                    float* part = a.partial + (slot * S::kQueries + row) * D;
                    if (!whole && r0 == 0) a.partial_ml[slot * S::kQueries + row] = make_float2(top[n][x], sum[n][x]);
#pragma unroll
                    for (int m = 0; m < D / 16; ++m) {
                        const float u = o[n][m][x] * by, v = o[n][m][2 + x] * by;
                        if constexpr (S::kEight) {  // dims 2 r0 and the next
                            const int dim = 16 * m + 2 * r0;
                            if (!whole) *reinterpret_cast<float2*>(part + dim) = make_float2(u, v);
                            else if (a.q_bf16) *reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(a.out) + at + dim) = pack2<true>(u, v);
                            else *reinterpret_cast<uint32_t*>(static_cast<__half*>(a.out) + at + dim) = pack2<false>(u, v);
                        } else {  // dims r0 and r0 + 8
                            const int dim = 16 * m + r0;
                            if (!whole) {
                                part[dim] = u;
                                part[dim + 8] = v;
                            } else if (a.q_bf16) {
                                static_cast<__nv_bfloat16*>(a.out)[at + dim] = __float2bfloat16_rn(u);
                                static_cast<__nv_bfloat16*>(a.out)[at + dim + 8] = __float2bfloat16_rn(v);
                            } else {
                                static_cast<__half*>(a.out)[at + dim] = __float2half_rn(u);
                                static_cast<__half*>(a.out)[at + dim + 8] = __float2half_rn(v);
                            }
                        }
                    }
                }
        }
        if (!more) break;
        run = ahead;
        turn ^= 1;
    }
    if (limit != kSpinLimit && lane == 0) atomicCAS(&g_paged_error, 0, 2);
}

#include "paged_attention_wide.cuh"

// Joins the states of a segment that several CTAs had, in their order; a segment without a key gets its zeros here.  SHARE warps of
// a CTA have one query: they take its pieces in turn, eight at a time with all their loads in flight.  Where segments are few, and
// have many pieces, four warps to a query (17 pieces, one after the other in a warp: 14.6 us for the whole call, so 11.6), else one
// (384 segments of seven queries: 37 us for the whole call, 40 with four).
template <int D, int QT, int SHARE>
__global__ void __launch_bounds__(128)
join_kernel(const __grid_constant__ AttnArgs a) {
    constexpr int kPer = D / 32, kBatch = 8;
    __shared__ int counts[2 * kWarps];
    __shared__ float states[SHARE][D + 2];
    pdl_trigger();
    const int unit = blockIdx.x / a.cache.n_kv, head = blockIdx.x - unit * a.cache.n_kv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = a.blocks == 1 ? unit : unit / a.blocks, block = unit - b * a.blocks;
    const int row = blockIdx.y * (kWarps / SHARE) + warp / SHARE, query = block * QT + row, i = a.token_of(query);
    // (the lengths may be read ahead of the wait: the kernel in front lets this one start behind its own wait only)
    const int limit = unit_limit<QT>(a, unit), tiles = (limit + kTileKeys - 1) / kTileKeys;
    int total = 0, front = 0;
    {  // slots of all units, and those before this segment's first tile
        int all = 0, mine = 0;
        for (int u = threadIdx.x; u < a.units; u += 32 * kWarps) {
            const int n = unit_slots(unit_limit<QT>(a, u));
            all += n;
            if (u < unit) mine += n;
        }
        all = __reduce_add_sync(kFullMask, all);
        mine = __reduce_add_sync(kFullMask, mine);
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
        front = front * a.cache.n_kv + head * (tiles + kSwitch) + kSwitch;
    }
    int first = 0, last = 0;
    if (tiles > 0) {
        const Shares shares(total, a.grid);
        first = shares.owner(front);
        last = shares.owner(front + tiles - 1);
    }
    // (Every CTA waits, also one with nothing to do: the kernel behind waits for this one alone, which must not end ahead of the one in front.)
    pdl_wait();
    if (row >= QT || i >= a.rows) return;
    if (tiles > 0 && first == last) return;  // (written by the CTA that has all of it)
    const size_t at = ((static_cast<size_t>(b) * a.rows + i) * a.n_heads + head * a.group + query - i * a.group) * D;
    float v[kPer] = {}, top = kNone, sum = 0.0f;
    if (tiles > 0) {
        for (int p0 = first + warp % SHARE; p0 <= last; p0 += SHARE * kBatch) {
            float2 ml[kBatch];
            float part[kBatch][kPer];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int p = p0 + k * SHARE;
                ml[k] = make_float2(kNone, 0.0f);
                if (p <= last) {
                    const size_t slot = 2 * static_cast<size_t>(p) + (p == first ? 1 : 0);
                    ml[k] = a.partial_ml[slot * QT + row];
                    const float* from = a.partial + (slot * QT + row) * D + kPer * lane;
#pragma unroll
                    for (int j = 0; j < kPer; ++j) part[k][j] = from[j];
                }
            }
            float higher = top;
#pragma unroll
            for (int k = 0; k < kBatch; ++k) higher = fmaxf(higher, ml[k].x);
            const float keep = exp2_of(top - higher);
            sum *= keep;
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[j] *= keep;
            top = higher;
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (p0 + k * SHARE > last) continue;
                const float w = exp2_of(ml[k].x - top);
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
        top = kNone;
        sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kPer; ++j) v[j] = 0.0f;
#pragma unroll
        for (int k = 0; k < SHARE; ++k) top = fmaxf(top, states[k][D]);
#pragma unroll
        for (int k = 0; k < SHARE; ++k) {
            const float w = exp2_of(states[k][D] - top);
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

// Queries of a block: those of a (sequence, KV head) in eights, two or four of them, and from 33 on the wide kernel's 128.  (32 sequences,
// 8 KV heads of 128 dims: 28 queries over 2048 int8 tokens 61 us so, 75 wide; 72 queries of 12 heads, 48 sequences of 300 int8 tokens, 124
// in blocks of 32, 66 wide; two prompts of 1024 rows, 4096 queries a head, 202 and 105, over bf16 rows 231 and 88.)
int queries_of_block(int rows, int group) {
    const int queries = rows * group;
    return queries <= 8 ? 8 : queries <= 16 ? 16 : queries <= 32 ? 32 : 128;
}

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

// The kernel over the tiles, whose blocks have QT queries, and the one that joins what it leaves.
template <int D, int QT, typename Kernel>
int launch(Kernel kernel, int per_sm, int threads, int registers, int smem, bool eight, int box_bytes, const AttnArgs& args, cudaStream_t stream, std::atomic<unsigned long long>& configured) {
    int status = once_on_this_device(configured, [&]() -> int {
        SPEC_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        cudaFuncAttributes f;  // (a thread that takes registers waits until its block has them: never, were the launch's too few)
        SPEC_CUDA_TRY(cudaFuncGetAttributes(&f, kernel));
        if (f.numRegs < registers) return fail(SPEC_ERR_CUDA, "spec_paged_attention: built with %d registers a thread", f.numRegs);
        return SPEC_OK;
    });
    if (status != SPEC_OK) return status;
    AttnArgs a = args;
    a.grid = 148 * per_sm;
    CUtensorMap map;
    status = rows_map(a, eight, D, box_bytes, &map);
    if (status != SPEC_OK) return status;
    status = launch_pdl(kernel, dim3(a.grid), dim3(threads), smem, stream, map, a);
    if (status != SPEC_OK) return status;
    const int segments = a.units * a.cache.n_kv, queries = static_cast<int>(std::min<long long>(QT, static_cast<long long>(a.rows) * a.group));
    if (segments * 4 <= a.grid) return launch_pdl(join_kernel<D, QT, 4>, dim3(segments, queries), dim3(128), 0, stream, a);
    return launch_pdl(join_kernel<D, QT, 1>, dim3(segments, (queries + 3) / 4), dim3(128), 0, stream, a);
}
template <int D, int KV, int NT>
int launch_narrow(const AttnArgs& a, cudaStream_t stream) {
    using S = Shape<D, KV, NT>;
    static std::atomic<unsigned long long> configured{0};
    return launch<D, S::kQueries>(paged_attention_kernel<D, KV, NT>, S::kPerSm, S::kThreads, S::kShift ? (S::kTaken + S::kLeft) / 2 : 0, S::kSmem, S::kEight, S::kBoxBytes, a, stream, configured);
}
template <int D, int KV>
int launch_wide(const AttnArgs& a, cudaStream_t stream) {
    using S = Wide<D, KV>;
    static std::atomic<unsigned long long> configured{0};
    return launch<D, S::kQueries>(paged_attention_wide_kernel<D, KV>, S::kPerSm, S::kThreads, S::kLaunched, S::kSmem, S::kEight, S::kBoxBytes, a, stream, configured);
}

template <int D, int KV>
int launch_tiles(const AttnArgs& a, cudaStream_t stream) {
    switch (queries_of_block(a.rows, a.group)) {
        case 8: return launch_narrow<D, KV, 1>(a, stream);
        case 16: return launch_narrow<D, KV, 2>(a, stream);
        case 32: return launch_narrow<D, KV, 4>(a, stream);
        default: return launch_wide<D, KV>(a, stream);
    }
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
           n_heads % n_kv_heads == 0 && n_heads / n_kv_heads <= 1024 &&
           static_cast<long long>(rows) * (n_heads / n_kv_heads) <= 1 << 20 && (d_head == 64 || d_head == 128);
}
long long units_of(int batch, int rows, int group, int queries) { return static_cast<long long>(batch) * ((static_cast<long long>(rows) * group + queries - 1) / queries); }

// Places for what two and more CTAs share of a segment: two for each.
size_t slots_for(int queries) { return 2 * static_cast<size_t>(most_ctas(queries)); }

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
    const size_t queries = queries_of_block(rows, n_heads / n_kv_heads), slots = slots_for(static_cast<int>(queries));
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
    const int queries = queries_of_block(rows, a.group);
    const long long units = units_of(batch, rows, a.group, queries);
    // (slots are counted in 32 bits, with room for a CTA's share on top)
    const long long slots_each = (static_cast<long long>(max_pages) * page_size + kTileKeys - 1) / kTileKeys + kSwitch;
    if (units * n_kv_heads > (1ll << 30) / slots_each) return fail(SPEC_ERR_BAD_ARG, "%s: too many rows for one call", who);
    if (!workspace || workspace_bytes < spec_paged_attention_workspace_bytes(batch, rows, n_heads, n_kv_heads, d_head) || !aligned_to(workspace, 256))
        return fail(SPEC_ERR_BAD_ARG, "%s: workspace missing, too small or not 256-byte aligned", who);
    const size_t slots = slots_for(queries);
    a.pool = pool;
    a.scales = scales;
    a.q = q;
    a.out = out;
    a.lengths = lengths;
    a.partial = static_cast<float*>(workspace);
    a.partial_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + align256(slots * queries * d_head * 4));
    a.q_stride = q_stride;
    a.scale = scale;
    a.rows = rows;
    a.n_heads = n_heads;
    a.units = static_cast<int>(units);
    a.blocks = a.units / batch;
    a.q_bf16 = dtype == SPEC_DTYPE_BF16;
    a.q_wide = aligned_to(q, 16) && q_stride % 8 == 0;
    a.by_group = a.group > 1 ? static_cast<uint32_t>((0xffffffffull + a.group) / a.group) : 0u;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return d_head == 64 ? launch_kv<64>(a, kv_dtype, st) : launch_kv<128>(a, kv_dtype, st);
}
