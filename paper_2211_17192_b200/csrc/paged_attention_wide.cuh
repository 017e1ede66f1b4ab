// Attention over paged rows for blocks of up to 128 queries of a KV head (33 and more of them: a verification pass of many heads to a KV
// head, a prompt): part of paged_attention.cu, whose arithmetic, split into runs of tiles and joining kernel it shares.
//
// Here the products are what bounds the mma.sync kernel, so they go to tcgen05.mma, queries on the M side: S = Q K^T from shared
// memory into tensor memory, weights back into the columns that S was in, O += P V with P from there and V as it lies (its keys are the
// K of that product, so it is the operand whose dims are contiguous).  8-bit rows are widened by four warps of their own, from
// the ring that the copies fill into the ring that the products read; 16-bit rows are multiplied where they were copied to.
// A CTA has four warps with a query to a thread (its row of S, no exchange between lanes), the four that widen, one that asks for
// tiles, one that issues the products, and two that only make up the last one's four, since registers are shared out among fours.
// S has two places: K of tile j + 1 is multiplied while the weights of tile j are made; two CTAs share an SM and its 512 columns.
// What bounds it: the chain weights -> second product -> free place -> widened K -> first product of every other tile, and the
// exponentials (1024 of a tile's 3000 cycles); 32 heads over 8 of 128 dims, 512 rows over 8192 tokens: 403 TFLOP/s int8; one prompt of
// 4096 rows 416 us.  (Queries fetched by the widening warps, with shuffles for their maxima: two prompts of 1024 rows 161 us, so 105;
// eight widening warps, K beside V: no faster; the widening loop rolled up instead of its loads in flight together: 77 us for 75.)
#pragma once

template <int D, int KV>
struct Wide {
    static constexpr bool kEight = KV == SPEC_DTYPE_E4M3 || KV == SPEC_DTYPE_INT8, kBf16 = KV == SPEC_DTYPE_BF16;
    static constexpr int kQueries = 128;
    static constexpr int kThreads = 32 * 3 * kWarps, kPerSm = 2;
    // Registers of a thread: 80 at launch, shared out again among the warps of weights, those that widen, and the others; in sum as many.
    static constexpr int kLaunched = 80, kWeights = 144, kWiden = 64, kOthers = 32;
    static_assert(kWeights + kWiden + kOthers == 3 * kLaunched, "a thread that takes registers would wait for ever");
    static constexpr int kRowBytes = D * (kEight ? 1 : 2), kBoxBytes = kRowBytes < 128 ? kRowBytes : 128, kBoxes = kRowBytes / kBoxBytes;
    static constexpr int kRaw = kTileKeys * kRowBytes;    // K or V of a tile as it lies in the cache
    static constexpr int kOperand = kTileKeys * D * 2;    // and in 16 bits: [D / 64][64 keys][128 bytes], swizzled
    static constexpr int kQueryBytes = kQueries * D * 2;  // [D / 64][128 rows][128 bytes], swizzled
    // Operands, K and V of a tile in turn.  8-bit: three, so that K of the next tile takes the place of V of the last one.
    static constexpr int kSlots = kEight ? 3 : D == 128 ? 4 : 8;
    static constexpr int kStages = kEight ? (D == 128 ? 3 : 6) : kSlots;  // of the ring that the copies fill (16-bit: the same one)
    static constexpr int kColumns = 256;                                  // tensor memory: two places for S, then O
    static constexpr int kSmem = kQueryBytes + kSlots * kOperand + (kEight ? kStages * kRaw : 0) + kStages * kTileKeys * 4 + 2 * 3 * kTileKeys * 4 +
                                 (2 * kStages + 2 * kSlots + 7) * 8 + (kStages + 8 + 24 + 1) * 4 + 1024;
    static_assert(kSmem + 1024 <= 228 * 1024 / kPerSm, "two CTAs to an SM");
    static_assert(148 * kPerSm <= most_ctas(kQueries), "room for every CTA's pieces");
    static_assert(2 * kTileKeys + D <= kColumns, "tensor memory");
    // Place of the 16 bytes at dim 8 c of row r in an operand (or, with its rows, among the queries).
    static __device__ __forceinline__ int place16(int rows, int r, int c) { return (c >> 3) * (rows * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4); }
};

// V as operand B: N = dims, contiguous and in boxes of 64, K = keys, a row of 128 bytes each.
__device__ __forceinline__ uint64_t values_desc(uint32_t addr) {
    uint64_t d = smem_desc_sw128(addr) & ~(uint64_t(0x3fff) << 16);
    return d | static_cast<uint64_t>((kTileKeys * 128) >> 4) << 16;  // from box to box of dims
}
__device__ __forceinline__ void mma_queries(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_weights(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void commit_to(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                   "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

template <int D, int KV>
__global__ void __launch_bounds__(Wide<D, KV>::kThreads, Wide<D, KV>::kPerSm)
paged_attention_wide_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ AttnArgs a) {
    using S = Wide<D, KV>;
    constexpr int kQueries = S::kQueries;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* queries = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* operands = queries + S::kQueryBytes;
    uint8_t* raw = S::kEight ? operands + S::kSlots * S::kOperand : operands;
    float* raw_scales = reinterpret_cast<float*>(raw + S::kStages * S::kRaw);  // [stage][64]
    float* info = raw_scales + S::kStages * kTileKeys;  // 8-bit keys, two tiles: [K's scale, log2 of V's, 1 / V's][64]
    uint64_t* raw_full = reinterpret_cast<uint64_t*>(info + 2 * 3 * kTileKeys);
    uint64_t* raw_empty = raw_full + S::kStages;
    uint64_t* op_full = raw_empty + S::kStages;  // an operand as the products take it
    uint64_t* op_empty = op_full + S::kSlots;
    uint64_t* s_full = op_empty + S::kSlots;  // [2]
    uint64_t* p_full = s_full + 2;            // [2] weights written, the tile's info read
    uint64_t* o_done = p_full + 2;            // a tile's second product has ended
    uint64_t* o_empty = o_done + 1;           // a segment's O has been read
    uint64_t* q_full = o_empty + 1;
    int* notes = reinterpret_cast<int*>(q_full + 1);  // [stage]: keys of the tile that there are, and which of its halves were fetched
    uint32_t* edges = reinterpret_cast<uint32_t*>(notes + S::kStages);  // [2] of a tile: its note, a bit per key whose V row has been taken out
    int* scratch = reinterpret_cast<int*>(edges + 8);  // [24]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(scratch + 24);

    const int warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(&raw_full[s], 1);
            mbar_init(&raw_empty[s], kWarps);
        }
        for (int s = 0; s < S::kSlots; ++s) {
            mbar_init(&op_full[s], kWarps);
            mbar_init(&op_empty[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[i], kWarps);
        }
        mbar_init(o_done, 1);
        mbar_init(o_empty, kWarps);
        mbar_init(q_full, kWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    pdl_trigger();  // (behind the wait: the joining kernel reads the lengths ahead of its own)

    int unit, before;
    const Shares shares(find_unit<kQueries>(a, scratch, unit, before), a.grid);
    if (unit < 0) return;  // (more CTAs than slots)
    Run<kQueries> run;
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
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(S::kColumns));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tmem_before_sync();
    __syncthreads();  // (barriers and columns are there for all)
    tmem_after_sync();
    const uint32_t tmem = *tmem_slot, tmem_o = tmem + 2 * kTileKeys;
    uint32_t limit = kSpinLimit;  // of every wait; one that has run out leaves one try to the others, and the CTA ends with its error noted
    const auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (!mbar_wait_warp(bar, parity & 1u, limit)) limit = 1;
    };

    if (warp >= 2 * kWarps) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kOthers));
    if (warp == 8) {
        // ---- K and V of the run's tiles, halves of 32 keys, which lie in one page each ----
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
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    if (use > 0) wait(S::kEight ? &raw_empty[stage] : &op_empty[stage], use - 1);
                    if (leader) {
                        const int halves = (page[0] >= 0 ? 1 : 0) + (page[1] >= 0 ? 1 : 0);
                        notes[stage] = min(kTileKeys, run.limit - t * kTileKeys) | (page[0] >= 0 ? 256 : 0) | (page[1] >= 0 ? 512 : 0);
                        mbar_expect_tx(&raw_full[stage], halves * (S::kRaw / 2 + (S::kEight ? 128 : 0)));
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (page[h] < 0) continue;
                            const int slot = (t * kTileKeys + 32 * h) & ((1 << a.cache.page_shift) - 1);
                            const int plane = (page[h] * 2 + which) * a.cache.n_kv + run.head;
#pragma unroll
                            for (int box = 0; box < S::kBoxes; ++box)
                                load_box(raw + stage * S::kRaw + box * (kTileKeys * 128) + h * 32 * S::kBoxBytes, &map, box * (S::kEight ? 128 : 64), slot, plane, &raw_full[stage]);
                            if constexpr (S::kEight)
                                load_bulk(raw_scales + stage * kTileKeys + 32 * h, a.scales + (static_cast<long long>(plane) << a.cache.page_shift) + slot, 128, &raw_full[stage]);
                        }
                    }
                    __syncwarp();
                    if (++stage == S::kStages) { stage = 0; ++use; }
                }
            }
        } while (run.next(a));
        if (limit != kSpinLimit)  // nothing may still be on its way when the CTA leaves
            for (int s = 0; s < S::kStages; ++s) {
                mbar_wait(&raw_full[s], 0, 1 << 14);
                mbar_wait(&raw_full[s], 1, 1 << 14);
            }
    } else if (warp == 9) {
        // ---- the products ----
        const bool leader = elect_one();
        constexpr uint32_t kType = S::kBf16 ? (1u << 7) | (1u << 10) : 0u;
        constexpr uint32_t kScores = (1u << 4) | kType | (kTileKeys / 8 << 17) | (kQueries / 16 << 24);
        constexpr uint32_t kSums = (1u << 4) | kType | (1u << 16) /* B: dims contiguous */ | (D / 8 << 17) | (kQueries / 16 << 24);
        const uint64_t q_desc = smem_desc_sw128(smem_u32(queries));
        int g = 0, segment = 0;
        do {
            const int n = run.tile1 - run.tile0;
            wait(q_full, segment);
            for (int i = 0; i <= n; ++i) {
                if (i < n) {
                    const int j = g + i, op = 2 * j, slot = op % S::kSlots;
                    wait(&op_full[slot], op / S::kSlots);
                    if (!S::kEight) wait(&raw_full[slot], op / S::kSlots);  // (long over: so that this warp too has seen the copies arrive)
                    // (the weights that lay where this S goes have been used; at a segment's start the second product behind them is under way too)
                    if (i == 0 ? j >= 1 : j >= 2) wait(o_done, i == 0 ? j - 1 : j - 2);
                    tmem_after_sync();
                    if (leader) {
                        const uint64_t k_desc = smem_desc_sw128(smem_u32(operands + slot * S::kOperand));
#pragma unroll
                        for (int k = 0; k < D / 16; ++k)
                            mma_queries(tmem + (j & 1) * kTileKeys, q_desc + (((k >> 2) * (kQueries * 128) + (k & 3) * 32) >> 4),
                                        k_desc + (((k >> 2) * (kTileKeys * 128) + (k & 3) * 32) >> 4), kScores, k > 0 ? 1u : 0u);
                        commit_to(&op_empty[slot]);
                        commit_to(&s_full[j & 1]);
                    }
                    __syncwarp();
                }
                if (i > 0) {
                    const int j = g + i - 1, op = 2 * j + 1, slot = op % S::kSlots;
                    wait(&op_full[slot], op / S::kSlots);
                    if (!S::kEight) wait(&raw_full[slot], op / S::kSlots);  // (long over: so that this warp too has seen the copies arrive)
                    wait(&p_full[j & 1], j >> 1);
                    if (i == 1 && segment > 0) wait(o_empty, segment - 1);
                    tmem_after_sync();
                    if (leader) {
                        const uint64_t v_desc = values_desc(smem_u32(operands + slot * S::kOperand));
#pragma unroll
                        for (int k = 0; k < kTileKeys / 16; ++k)
                            mma_weights(tmem_o, tmem + (j & 1) * kTileKeys + 8 * k, v_desc + ((k * 16 * 128) >> 4), kSums, i > 1 || k > 0 ? 1u : 0u);
                        commit_to(&op_empty[slot]);
                        commit_to(o_done);
                    }
                    __syncwarp();
                }
            }
            g += n;
            ++segment;
        } while (run.next(a));
        if (limit != kSpinLimit) {  // (products may still be under way)
            mbar_wait(o_done, 0, 1 << 14);
            mbar_wait(o_done, 1, 1 << 14);
        }
    } else if (warp >= 2 * kWarps) {
    } else if (warp >= kWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kWiden));
        // ---- operands as the products take them ----
        const int tid = threadIdx.x - 32 * kWarps;
        int stage = 0, use = 0, slot = 0, turn = 0, g = 0;  // use, turn: how often either ring has gone round
        do {
            const int b = a.blocks == 1 ? run.unit : run.unit / a.blocks, block = run.unit - b * a.blocks;
            const int length = max(a.lengths[b], 0);
            const int seen_by_all = max(-1, length - a.rows + min(a.rows - 1, a.token_of(block * kQueries)));
            for (int t = run.tile0; t < run.tile1; ++t, ++g) {
                if (g >= 2) wait(&p_full[g & 1], (g >> 1) - 1);  // (the info and the edge of the tile before the last have been read)
                float* tile_info = info + (g & 1) * 3 * kTileKeys;
                // Rows that some of the block's queries see and others do not: a weight of zero does not hide a V row that is no number
                // from the product, so such a row is taken out and told to those who see it.
                const bool hidden = KV != SPEC_DTYPE_INT8 && t * kTileKeys + kTileKeys - 1 > seen_by_all && seen_by_all + 1 < run.limit;
#pragma unroll 1
                for (int which = 0; which < 2; ++which) {
                    wait(&raw_full[stage], use);
                    const int note = notes[stage], count = note & 255;
                    const auto there = [&](int r) { return r < count && (note & (r < 32 ? 256 : 512)); };
                    const bool edge = count < kTileKeys || (note & 768) != 768;
                    if constexpr (S::kEight) {
                        if (turn > 0) wait(&op_empty[slot], turn - 1);
                    }
                    uint8_t* to = operands + slot * S::kOperand;
                    uint8_t* from = raw + stage * S::kRaw;
                    constexpr int kChunks = S::kRowBytes / 16;  // of a row
                    if (which == 0 && tid < 4) edges[4 * (g & 1) + tid] = tid == 0 ? note : 0;
                    if constexpr (S::kEight) {
                        if (tid < kTileKeys) {
                            float s = raw_scales[stage * kTileKeys + tid];
                            if (which == 0) {
                                tile_info[tid] = there(tid) ? s : 0.0f;
                            } else {
                                if (s == 1.0f) {  // (seldom)
                                    uint32_t some = 0u;
#pragma unroll 1
                                    for (int x = 0; x < S::kRowBytes / 16; ++x) some |= some_code<KV>(*reinterpret_cast<const uint4*>(from + Shape<D, KV, 1>::place(tid, x)));
                                    if (some == 0u) s = kScaleOfZeros;
                                }
                                const bool number = magnitude(s) < 0x7f800000u;
                                tile_info[kTileKeys + tid] = number ? log2_of(s) : NAN;
                                tile_info[2 * kTileKeys + tid] = there(tid) && number ? reciprocal_of(s) : 0.0f;
                            }
                        }
                        if (which == 1 && hidden) asm volatile("bar.sync 2, %0;" ::"n"(32 * kWarps) : "memory");  // (before a bit is set)
                        // (the rows of a chunk's neighbours in i are 128 / kChunks apart: a multiple of eight, so that their places differ by a constant)
                        constexpr int kApart = 128 / kChunks, kSteps = kTileKeys / kApart;
                        const int r0 = tid / kChunks, c = tid % kChunks, first = c >> 2 & 1;  // (first: the lanes of a row in different banks)
                        const uint8_t* at = from + Shape<D, KV, 1>::place(r0, c);
                        uint8_t* to0 = to + S::place16(kTileKeys, r0, 2 * c + first);
                        uint8_t* to1 = to + S::place16(kTileKeys, r0, 2 * c + 1 - first);
                        uint4 codes[kSteps];
#pragma unroll
                        for (int i = 0; i < kSteps; ++i) codes[i] = *reinterpret_cast<const uint4*>(at + i * kApart * S::kRowBytes);
                        if (edge || (KV == SPEC_DTYPE_E4M3 && which == 1 && hidden)) {
#pragma unroll
                            for (int i = 0; i < kSteps; ++i) {
                                const int r = r0 + i * kApart;
                                if (!there(r)) codes[i] = make_uint4(0u, 0u, 0u, 0u);
                                const uint32_t bad = __ballot_sync(kFullMask, KV == SPEC_DTYPE_E4M3 && not_numbers<KV>(codes[i])) >> (lane / kChunks * kChunks) & ((1u << kChunks) - 1);
                                if (which == 1 && hidden && bad) {
                                    codes[i] = make_uint4(0u, 0u, 0u, 0u);
                                    if (c == 0) atomicOr(&edges[4 * (g & 1) + 1 + r / 32], 1u << r % 32);
                                }
                            }
                        }
#pragma unroll
                        for (int i = 0; i < kSteps; ++i) {
                            uint4 half[2];
                            widen<KV, 1>(codes[i].x, half[0].x, half[0].y);
                            widen<KV, 1>(codes[i].y, half[0].z, half[0].w);
                            widen<KV, 1>(codes[i].z, half[1].x, half[1].y);
                            widen<KV, 1>(codes[i].w, half[1].z, half[1].w);
                            *reinterpret_cast<uint4*>(to0 + i * kApart * 128) = first ? half[1] : half[0];
                            *reinterpret_cast<uint4*>(to1 + i * kApart * 128) = first ? half[0] : half[1];
                        }
                    } else {
                        if (edge || (which == 1 && hidden)) {
                            asm volatile("bar.sync 2, %0;" ::"n"(32 * kWarps) : "memory");
#pragma unroll 1
                            for (int i = 0; i < kTileKeys * kChunks / 128; ++i) {
                                const int r = (i * 128 + tid) / kChunks, c = (i * 128 + tid) % kChunks;
                                uint4* at = reinterpret_cast<uint4*>(from + S::place16(kTileKeys, r, c));
                                bool out = !there(r);
                                if (which == 1 && hidden) {
                                    const uint32_t bad = __ballot_sync(kFullMask, !out && not_numbers<KV>(*at)) >> (lane / kChunks * kChunks) & ((1u << kChunks) - 1);
                                    if (bad) {
                                        out = true;
                                        if (c == 0) atomicOr(&edges[4 * (g & 1) + 1 + r / 32], 1u << r % 32);
                                    }
                                }
                                if (out) *at = make_uint4(0u, 0u, 0u, 0u);
                            }
                            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        }
                    }
                    if constexpr (S::kEight) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(&op_full[slot]);
                        if (S::kEight) mbar_arrive(&raw_empty[stage]);
                    }
                    if (++stage == S::kStages) { stage = 0; ++use; }
                    if (++slot == S::kSlots) { slot = 0; ++turn; }
                }
            }
        } while (run.next(a));
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kWeights));
        // ---- weights: a query to a thread ----
        const int row = warp * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
        // A thread's query to its row of the operand; bf16 ones for fp16 products with the largest magnitude brought to [1, 2) by a power of
        // two.  Returns what its scores are multiplied with.
        const auto prepare = [&](const Run<kQueries>& of) -> float {
            const int b = a.blocks == 1 ? of.unit : of.unit / a.blocks, block = of.unit - b * a.blocks, query = block * kQueries + row, token = a.token_of(query);
            float back = 1.0f;
            if (a.token_of(block * kQueries + warp * 32) < a.rows) {
                __align__(16) uint32_t words[D / 2];
                const uint16_t* from = static_cast<const uint16_t*>(a.q) + (static_cast<size_t>(b) * a.rows + token) * a.q_stride + (of.head * a.group + query - token * a.group) * D;
                if (token >= a.rows) {
#pragma unroll
                    for (int i = 0; i < D / 2; ++i) words[i] = 0u;
                } else if (a.q_wide) {
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) reinterpret_cast<uint4*>(words)[i] = reinterpret_cast<const uint4*>(from)[i];
                } else {
#pragma unroll
                    for (int i = 0; i < D / 4; ++i) reinterpret_cast<uint2*>(words)[i] = reinterpret_cast<const uint2*>(from)[i];
                }
                if (!S::kBf16 && a.q_bf16) {
                    uint32_t low = 0u, high = 0u;  // (bits of magnitudes are in their order)
#pragma unroll
                    for (int i = 0; i < D / 2; ++i) {
                        low = max(low, words[i] << 16 & 0x7fff0000u);
                        high = max(high, words[i] & 0x7fff0000u);
                    }
                    const uint32_t largest = max(low, high);
                    float by = 1.0f;
                    if (largest != 0u && largest < 0x7f800000u) {
                        const int e = max(-120, min(120, static_cast<int>(largest >> 23) - 127));
                        back = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
                        by = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
                    }
#pragma unroll
                    for (int i = 0; i < D / 2; ++i) words[i] = pack2<false>(__uint_as_float(words[i] << 16) * by, __uint_as_float(words[i] & 0xffff0000u) * by);
                }
#pragma unroll
                for (int i = 0; i < D / 8; ++i)
                    *reinterpret_cast<uint4*>(queries + S::place16(kQueries, row, i)) = reinterpret_cast<const uint4*>(words)[i];
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full);
            return back * a.scale * kLog2e;
        };
        int g = 0;
        float factor = prepare(run);
        while (true) {
            const int b = a.blocks == 1 ? run.unit : run.unit / a.blocks, block = run.unit - b * a.blocks;
            const int length = max(a.lengths[b], 0), query = block * kQueries + row, token = a.token_of(query);
            const int seen = token < a.rows ? max(-1, length - a.rows + token) : -1;
            const bool live = a.token_of(block * kQueries + warp * 32) < a.rows;  // (some query of this warp exists)
            const int seen_by_all = max(-1, length - a.rows + min(a.rows - 1, a.token_of(block * kQueries + warp * 32)));
            float top = kNone, sum = 0.0f;
            for (int t = run.tile0; t < run.tile1; ++t, ++g) {
                wait(&s_full[g & 1], g >> 1);
                if (live) {
                    const int op = 2 * g + 1;
                    wait(&op_full[op % S::kSlots], op / S::kSlots);  // (the tile's info)
                    tmem_after_sync();
                    const float* tile_info = info + (g & 1) * 3 * kTileKeys;
                    const uint32_t at = tmem + lanes + (g & 1) * kTileKeys;
                    float e[kTileKeys];
                    tmem_ld32(at, e);
                    tmem_ld32(at + 32, e + 32);
                    tmem_ld_wait();
                    const bool masked = edges[4 * (g & 1)] != (768u | kTileKeys) || t * kTileKeys + kTileKeys - 1 > seen_by_all;  // (keys that are not there, or not for every query)
#pragma unroll
                    for (int i = 0; i < kTileKeys; i += 4) {
                        if constexpr (S::kEight) {
                            if (i % 16 == 0) asm volatile("" ::: "memory");  // (all of the info asked for at once would not fit in the registers)
                            const float4 raise = *reinterpret_cast<const float4*>(tile_info + kTileKeys + i), sk = *reinterpret_cast<const float4*>(tile_info + i);
                            e[i] = fmaf(e[i], sk.x * factor, raise.x);
                            e[i + 1] = fmaf(e[i + 1], sk.y * factor, raise.y);
                            e[i + 2] = fmaf(e[i + 2], sk.z * factor, raise.z);
                            e[i + 3] = fmaf(e[i + 3], sk.w * factor, raise.w);
                        } else {
#pragma unroll
                            for (int x = 0; x < 4; ++x) e[i + x] *= factor;
                        }
                    }
                    if (masked) {
                        const uint32_t* edge = edges + 4 * (g & 1);
                        const int last = min(seen - t * kTileKeys, static_cast<int>(edge[0] & 255u) - 1);  // key of the tile
                        const uint32_t seen_of[2] = {edge[0] & 256u && last >= 0 ? 0xffffffffu >> (31 - min(last, 31)) : 0u,
                                                     edge[0] & 512u && last >= 32 ? 0xffffffffu >> (63 - min(last, 63)) : 0u};
                        if (edge[1] | edge[2]) {
#pragma unroll
                            for (int i = 0; i < kTileKeys; ++i)
                                if (edge[1 + i / 32] >> (i % 32) & 1u) e[i] = NAN;
                        }
#pragma unroll
                        for (int i = 0; i < kTileKeys; ++i)
                            if (!(seen_of[i / 32] >> (i % 32) & 1u)) e[i] = -INFINITY;
                    }
                    float most[4] = {kNone, kNone, kNone, kNone};
#pragma unroll
                    for (int i = 0; i < kTileKeys; ++i) most[i & 3] = fmaxf(most[i & 3], e[i]);
                    most[0] = fmaxf(most[0], most[2]);
                    most[1] = fmaxf(most[1], most[3]);
                    most[0] = fmaxf(most[0], most[1]);
                    // The maximum is moved only where an exponent has left the old one behind by more than the slack (a query's own do: what
                    // the others see does not change its result).
                    const bool moves = most[0] > top + kSlack;
                    if (__any_sync(kFullMask, moves)) {
                        const float higher = moves ? most[0] : top, shrink = exp2_of(top - higher);
                        top = higher;
                        sum *= shrink;
                        if (t > run.tile0) {
                            wait(o_done, g - 1);
                            tmem_after_sync();
#pragma unroll
                            for (int m = 0; m < D; m += 16) {
                                uint32_t o[16];
                                tmem_ld16(tmem_o + lanes + m, o);
                                tmem_ld_wait();
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * shrink);
                                tmem_st16(tmem_o + lanes + m, o);
                            }
                        }
                    }
                    float part[2] = {0.0f, 0.0f};
#pragma unroll
                    for (int half = 0; half < kTileKeys; half += 32) {
                        uint32_t p[16];
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            if (i % 16 == 0) asm volatile("" ::: "memory");
                            float w[4];
#pragma unroll
                            for (int x = 0; x < 4; ++x) w[x] = exp2_of(e[half + i + x] - top);
                            if constexpr (S::kEight) {
                                const float4 inv = *reinterpret_cast<const float4*>(tile_info + 2 * kTileKeys + half + i);
                                part[0] = fmaf(w[0], inv.x, part[0]);
                                part[1] = fmaf(w[1], inv.y, part[1]);
                                part[0] = fmaf(w[2], inv.z, part[0]);
                                part[1] = fmaf(w[3], inv.w, part[1]);
                            } else {
                                part[0] += w[0] + w[1];
                                part[1] += w[2] + w[3];
                            }
                            p[i / 2] = pack2<S::kBf16>(w[0], w[1]);
                            p[i / 2 + 1] = pack2<S::kBf16>(w[2], w[3]);
                        }
                        tmem_st16(at + half / 2, p);
                    }
                    sum += part[0] + part[1];
                    tmem_st_wait();
                    tmem_before_sync();
                }
                // A wait tells a phase from its neighbours only.  S of this tile says that the second product before the last has ended, and the
                // waits behind the segment (here for its O, of the issuer for the next S) are for the second product of this tile: the one between
                // them has to have ended first, or they pass a product early where a warp is a tile behind the others.
                if (t + 1 == run.tile1 && t > run.tile0) wait(o_done, g - 1);
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[g & 1]);
            }
            // (all first products of this segment have ended: the next one's queries may take the place of its own)
            Run<kQueries> ahead = run;
            const bool more = ahead.next(a);
            const float factor_ahead = more ? prepare(ahead) : 0.0f;
            wait(o_done, g - 1);
            tmem_after_sync();
            if (live) {
                const bool whole = run.tile0 == 0 && run.tile1 == run.tiles;
                const float by = whole ? (sum == 0.0f ? 0.0f : reciprocal_of(sum)) : 1.0f;
                const size_t at = ((static_cast<size_t>(b) * a.rows + token) * a.n_heads + run.head * a.group + query - token * a.group) * D;
                const size_t slot = 2 * static_cast<size_t>(blockIdx.x) + (run.tile0 == 0 ? 1 : 0);
                if (!whole && token < a.rows) a.partial_ml[slot * kQueries + row] = make_float2(top, sum);
#pragma unroll
                for (int m = 0; m < D; m += 32) {
                    float o[32];
                    tmem_ld32(tmem_o + lanes + m, o);
                    tmem_ld_wait();
                    if (token >= a.rows) {
                    } else if (!whole) {
                        float4* to = reinterpret_cast<float4*>(a.partial + (slot * kQueries + row) * D + m);
#pragma unroll
                        for (int i = 0; i < 8; ++i) to[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    } else {
                        uint2* to = reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at + m);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float x = o[4 * i] * by, y = o[4 * i + 1] * by, z = o[4 * i + 2] * by, w = o[4 * i + 3] * by;
                            to[i] = a.q_bf16 ? make_uint2(pack2<true>(x, y), pack2<true>(z, w)) : make_uint2(pack2<false>(x, y), pack2<false>(z, w));
                        }
                    }
                    __syncwarp();
                }
            }
            tmem_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(o_empty);
            if (!more) break;
            run = ahead;
            factor = factor_ahead;
        }
    }
    if (limit != kSpinLimit && lane == 0) atomicCAS(&g_paged_error, 0, 3);
    __syncwarp();
    tmem_before_sync();
    __syncthreads();
    if (warp == 9) {
        tmem_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kColumns));
    }
}
