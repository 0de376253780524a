// Kernels of the orthogonalised update (Newton-Schulz products).
//
// muon_gemm_kernel  every product of an iteration, on CTA pairs: tcgen05.mma cta_group::2 fed by TMA, two 256-column
//                   accumulators in TMEM, so that the epilogue of a tile runs under the main loop of the next
// muon_moment / muon_load / muon_apply   the streaming passes before and after
//
// A product's tile is 256 x 256 (256 x 128 or 128 x 128 in short lists): each CTA of a pair loads half of the rows of L and
// half of the columns of R, 32 KB per 64-deep k-block, six stages; four MMAs of 256 x 256 x 16 consume them.  Measured on
// four 4096 x 4096 matrices, five steps: 1305 TFLOP/s, the tensor pipe active in 84 % of the cycles, 54 bytes a cycle and SM
// from L2 (of 64), 1.34 GHz under the board's power cap.  Roles of the 12 warps: 0 TMA producer, 1 TMEM owner and MMA
// issuer (leader) or dealer of tiles (peer), 2 and 3 bookkeeping, 4-11 epilogue (a warp reads the 32 TMEM lanes it may read and
// one half of the columns).  The epilogue adds the terms that the iteration needs beside some products, rounds to 16 bits and
// hands 32 x 32 pieces to TMA stores; a symmetric product's tile above the diagonal is stored a second time,
// transposed, so that half of the symmetric products is never computed.
// Bound: the tensor pipe (and with it the board's power).
//
// Every mbarrier wait is bounded, as in the projection kernels: a wait that gives up sets the status word, the roles
// leave the tile loop, what is in flight is drained, TMEM is freed.
#include "muon.h"

#include "../../include/apollo.h"
#include "device_utils.cuh"
#include "host_utils.h"
#include "tc_common.cuh"
#include "tc_ptx.cuh"

namespace apollo {

namespace {

constexpr int MG_THREADS = 384;
constexpr int MG_HALF = 8192;                            // 64 x 64 16-bit floats: one TMA box
constexpr int MG_EPI_WARPS = 8;
constexpr int MG_STAGING = MG_EPI_WARPS * 4096;          // per epilogue warp: a piece of 32 x 32, and the piece transposed
constexpr uint32_t MG_RING = 16;                         // entries of the list in flight
constexpr uint32_t MG_END = 0xFFFFFFFFu;                 // no more entries
template <int TILE> struct GemmCfg {
    static constexpr int BM = MUON_TILES[TILE].m, BN = MUON_TILES[TILE].n;
    static constexpr int L_BYTES = BM / 2 * 128;         // a CTA's half of L, 64 deep
    static constexpr int STAGE = L_BYTES + BN / 2 * 128; // and its half of R
    static constexpr int STAGES = TILE == TILE_WIDE ? 6 : 8;
    static constexpr int SMEM = STAGES * STAGE + MG_STAGING + 768 + 1024;
    static_assert(SMEM <= 227 * 1024 && STAGES <= 8, "shared memory and barriers of a CTA");
};

// Bounded wait until *counter >= need; a set status word ends it at once.
__device__ __forceinline__ bool wait_count(const uint32_t* counter, uint32_t need, volatile int* abort_flag, int32_t* status, int where)
{
    if (need == 0 || ld_acquire_gpu(counter) >= need) return true;
    if (*abort_flag) return false;
    for (uint32_t i = 0; i < TC_WAIT_CAP; ++i) {
        if (i > 64) __nanosleep(64);
        if (ld_acquire_gpu(counter) >= need) return true;
        if ((i & 63u) == 63u && *reinterpret_cast<volatile int32_t*>(status) != STATUS_OK) break;
    }
    *abort_flag = 1;
    atomicCAS(status + 1, 0, where);
    atomicExch(status, STATUS_TIMEOUT);
    return false;
}

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi)
{
    const __half2 p = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ float2 unpack_half2(uint32_t w)
{
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// v += b * (32 values at p): 64 contiguous bytes of one row
__device__ __forceinline__ void add_term(float (&v)[32], float b, const uint4 (&e)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w[4] = { e[i].x, e[i].y, e[i].z, e[i].w };
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = unpack_half2(w[k]);
            v[8 * i + 2 * k] = fmaf(b, f.x, v[8 * i + 2 * k]);
            v[8 * i + 2 * k + 1] = fmaf(b, f.y, v[8 * i + 2 * k + 1]);
        }
    }
}
__device__ __forceinline__ void load_term(uint4 (&e)[4], const __half* p, bool in)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = in ? __ldcg(reinterpret_cast<const uint4*>(p) + i) : make_uint4(0, 0, 0, 0);
}

}  // namespace

// One launch does all products of a group: the host lists the tiles of the first product of every matrix, then those of
// the second, and so on, and the pairs draw them in this order.  A tile waits (bounded) until the products before its
// own are complete for ITS matrix: a counter per matrix, one count per CTA and tile, added after the CTA's stores have
// landed.  Whoever runs draws the next tile, so the earliest unfinished one is always at work and waits for nothing
// that is not: no CTA has to be resident for another to finish.  With several matrices the products before are
// complete by the time a tile comes up, and there is neither a launch nor a drained pipeline between products.
// (Dealing the tiles out by index instead let the pairs drift apart where long and short contractions meet; what
// neighbours share then no longer met in L2: a 7B layer took 11 % more time, at equal cycles.)
//
// Roles that keep latency off the loads and the epilogue:
//   the peer's warp 1  (the leader's issues the MMAs) draws: when its producer begins with a tile, the ticket of the next
//                      one and its entry of the list, which st.async puts into a ring of 16 slots in both CTAs.  (On the
//                      producer's thread the two round trips to L2 held up 1500 cycles of loads in every tile.)
//                      Nobody has to say that a slot is free: the dealer is one tile ahead of the producer, that one at most
//                      STAGES k-blocks (>= one tile each) ahead of the MMAs, those at most two tiles ahead of the
//                      epilogue, so a slot is read long before its turn.
//   warp 2             makes the tensor maps of the tile's product visible to this CTA, waits for the tile's operands and
//                      passes both on (`dep` barriers, same ring)
//   warp 3             counts the tile once the eight epilogue warps say that their stores have landed
//
// Symmetric results are computed in blocks of a tile's rows from the diagonal on; a tile beyond the diagonal block is stored a
// second time, transposed.  (Storing it once, and reading what lies below the diagonal as the transposed tile of what
// lies above, which the tensor cores also take, saves those stores and cost 5 % on 4096 x 4096: operands in that
// order take 10 % more cycles per k-block.)
//
// SPLIT: operands are sums of two 16-bit floats, and the contraction runs over three segments into one accumulator:
// lo hi + hi lo + hi hi (what is dropped, lo lo, is 2^-24 of a term), the small ones first: every addition to a large
// accumulator cuts it toward zero (relative error of X after five steps, 2048 x 2048 normal gradients: 2.0e-5, with
// hi hi first 5.0e-5).  Summing in pieces of 512, rounded to nearest in between, gave 6e-6 at 1.8 times the time, and
// is not done.  TILE: which of MUON_TILES.
template <bool SPLIT, int TILE>
__global__ void __launch_bounds__(MG_THREADS, 1)
muon_gemm_kernel(const GemmOp* __restrict__ ops, const uint64_t* __restrict__ list, uint32_t tiles, uint32_t* __restrict__ ticket,
                 int32_t* __restrict__ status)
{
    using Cfg = GemmCfg<TILE>;
    constexpr int BM = Cfg::BM, BN = Cfg::BN;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (ptx::smem_addr(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - ptx::smem_addr(smem_raw));
    constexpr uint32_t MISC = Cfg::STAGES * Cfg::STAGE + MG_STAGING;
    const uint32_t staging = smem_base + Cfg::STAGES * Cfg::STAGE;
    const uint32_t bars = smem_base + MISC;
    const uint32_t bar_full = bars, bar_done = bars + 64, bar_acc_full = bars + 128, bar_acc_empty = bars + 144, bar_drain = bars + 160, bar_go = bars + 168,
                   bar_landed = bars + 192, bar_entry = bars + 256, bar_dep = bars + 384, slots = bars + 512;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_gen + MISC + 176);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_gen + MISC + 180);

    const uint32_t rank = ptx::cluster_ctarank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < Cfg::STAGES; ++s) {
            ptx::mbar_init(bar_full + 8 * s, 1);         // the leader's arrive.expect_tx for the bytes of both CTAs
            ptx::mbar_init(bar_done + 8 * s, 1);         // the leader's commit
        }
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(bar_acc_full + 8 * b, 1);
            ptx::mbar_init(bar_acc_empty + 8 * b, 2 * (MG_EPI_WARPS + 1));   // both CTAs' epilogue warps and counting warp
        }
        for (int b = 0; b < 4; ++b) ptx::mbar_init(bar_landed + 8 * b, MG_EPI_WARPS);
        for (int b = 0; b < MG_RING; ++b) {
            ptx::mbar_init(bar_entry + 8 * b, 1);        // this CTA's producer, and the entry's 16 bytes
            ptx::mbar_init(bar_dep + 8 * b, 1);          // warp 2
        }
        ptx::mbar_init(bar_drain, 1);
        ptx::mbar_init(bar_go, 1);                       // the peer's producer
        *abort_flag = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 1) {
        ptx::tmem_alloc_pair(ptx::smem_addr(tmem_slot), 512);
        ptx::tmem_relinquish_pair();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::cluster_sync();
    ptx::tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    // all of the above may run while the pass before is still at work
    ptx::grid_launch_dependents();
    ptx::grid_wait_previous();

    uint32_t it = 0, stage = 0, phase = 0;
    auto next_stage = [&]() { ++it; if (++stage == (uint32_t)Cfg::STAGES) { stage = 0; phase ^= 1; } };

    // dealer: fetches entry `n` (ticket t) and hands it to both CTAs
    auto deal = [&](uint32_t n, uint32_t t) {
        const uint32_t b = n % MG_RING;
        uint4 e = make_uint4(MG_END, 0, 0, 0);
        if (t < tiles) {
            const uint64_t p = __ldg(list + t);
            e = make_uint4(tile_field(p, 0, TILE_OP_BITS), tile_field(p, TILE_M_AT, TILE_M_BITS) | tile_field(p, TILE_N_AT, TILE_N_BITS) << 16,
                           tile_field(p, TILE_K_AT, TILE_K_BITS), tile_field(p, TILE_R_AT, 1));
        }
        for (uint32_t c = 0; c < 2; ++c)
            ptx::st_async_v4(ptx::map_to_cta(slots + 16 * b, c), e.x, e.y, e.z, e.w, ptx::map_to_cta(bar_entry + 8 * b, c));
    };
    if (tid == 0) {
        ptx::mbar_arrive_expect_tx(bar_entry, 16);
        if (rank == 1) deal(0, atomicAdd(ticket, 1u));
    }
    int last_op = -1;
    for (uint32_t n = 0;; ++n) {
        // the entry {op, tm | tn << 16, k-blocks, R along n}
        const uint32_t slot = n % MG_RING, ring_phase = (n / MG_RING) & 1;
        if (!__all_sync(0xFFFFFFFFu, wait_phase(bar_entry + 8 * slot, ring_phase, abort_flag, status, 208))) break;
        const uint4 entry = ptx::ld_shared_v4(slots + 16 * slot);
        if (entry.x == MG_END) break;
        const GemmOp* op = ops + entry.x;
        const int tm = (int)(entry.y & 0xFFFFu), tn = (int)(entry.y >> 16), num_kb = (int)entry.z;
        const bool r_mn = entry.w != 0;
        const uint32_t buf = n & 1, use = n >> 1;
        const bool soft = num_kb > 24;                   // long contraction: waits have slack, and sleeping saves power
        const bool new_op = last_op != (int)entry.x;
        last_op = (int)entry.x;

        if (warp == 0) {
            // ---------------- TMA producer (one thread in each CTA) ----------------
            if (lane == 0) {
                ptx::mbar_arrive_expect_tx(bar_entry + 8 * ((n + 1) % MG_RING), 16);
                const void* l_hi = op->l_map[0];
                const void* r_hi = op->r_map[0];
                const void* l_lo = SPLIT ? op->l_map[1] : nullptr;
                const void* r_lo = SPLIT ? op->r_map[1] : nullptr;
                const int seg_k = SPLIT ? num_kb / 3 * 64 : 0;
                const uint64_t pol = ptx::policy_evict_normal();
                const uint32_t full0 = ptx::map_to_cta(bar_full, 0);
                const int m0 = tm * BM + (int)rank * (BM / 2), n0 = tn * BN + (int)rank * (BN / 2);
                const bool ok = wait_phase(bar_dep + 8 * slot, ring_phase, abort_flag, status, 205);
                if (ok && rank == 1) ptx::mbar_arrive(bar_go);
                int k = 0, seg = 0;
                for (int i = 0; ok && i < num_kb; ++i, next_stage()) {
                    const uint32_t s = stage;
                    if (!wait_phase(bar_done + 8 * s, phase ^ 1, abort_flag, status, 201)) break;
                    const uint32_t dst = smem_base + s * Cfg::STAGE, full = full0 + 8 * s;
                    if (rank == 0) ptx::mbar_arrive_expect_tx(bar_full + 8 * s, 2u * Cfg::STAGE);
                    const void* lm = SPLIT && seg == 0 ? l_lo : l_hi;
                    const void* rm = SPLIT && seg == 1 ? r_lo : r_hi;
                    ptx::tma_load_2d_pair(dst, lm, k, m0, full, pol);
                    if (r_mn) {
                        ptx::tma_load_2d_pair(dst + Cfg::L_BYTES, rm, n0, k, full, pol);
                        if (BN == 256) ptx::tma_load_2d_pair(dst + Cfg::L_BYTES + MG_HALF, rm, n0 + 64, k, full, pol);
                    } else {
                        ptx::tma_load_2d_pair(dst + Cfg::L_BYTES, rm, k, n0, full, pol);
                    }
                    k += 64;
                    if (SPLIT && k >= seg_k) { k = 0; ++seg; }
                }
            }
            __syncwarp();
        } else if (warp == 1 && rank == 1) {
            // ---------------- dealer ----------------
            if (lane == 0 && wait_phase(bar_go, n & 1, abort_flag, status, 211)) deal(n + 1, atomicAdd(ticket, 1u));
            __syncwarp();
        } else if (warp == 1) {
            // ---------------- MMA issuer (leader only) ----------------
            if (lane == 0) {
                const uint32_t idesc = ptx::instr_desc_f16_pair(BM, BN, r_mn);
                const uint32_t d_tmem = tmem_base + buf * BN;
                bool ok = wait_phase(bar_acc_empty + 8 * buf, (use & 1) ^ 1, abort_flag, status, 202);
                ptx::tc_fence_after_sync();
                // K-major operand: 64 k = 128 bytes a row, 8-row groups 1024 bytes apart, 16 k = 32 bytes on.
                // n-contiguous R: 64 n = 128 bytes a k-row, 16 k-rows = 2048 bytes on, the next 64 n one box further.
                const uint64_t a_desc0 = ptx::smem_desc_sw128(smem_base, 16, 1024);
                const uint64_t b_desc0 = r_mn ? ptx::smem_desc_sw128(smem_base + Cfg::L_BYTES, MG_HALF, 1024)
                                              : ptx::smem_desc_sw128(smem_base + Cfg::L_BYTES, 16, 1024);
                const uint32_t b_step = r_mn ? 2048u >> 4 : 32u >> 4;
                int i = 0;
                for (; ok && i < num_kb; ++i, next_stage()) {
                    const uint32_t s = stage;
                    if (!wait_phase(bar_full + 8 * s, phase, abort_flag, status, 203)) break;
                    ptx::tc_fence_after_sync();
                    const uint64_t a_desc = a_desc0 + s * (Cfg::STAGE >> 4), b_desc = b_desc0 + s * (Cfg::STAGE >> 4);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        ptx::mma_bf16_pair(d_tmem, a_desc + kk * 2, b_desc + kk * b_step, idesc, (i | kk) != 0 ? 1u : 0u);
                    ptx::mma_commit_pair(bar_done + 8 * s, 3);
                }
                if (ok && i == num_kb) ptx::mma_commit_pair(bar_acc_full + 8 * buf, 3);
            }
            __syncwarp();
        } else if (warp == 2) {
            // ---------------- operands complete? ----------------
            if (lane == 0) {
                bool ok = true;
                if (new_op) {
                    for (int h = 0; h < (SPLIT ? 2 : 1); ++h) {
                        const void* const maps[4] = { op->l_map[h], op->r_map[h], op->out_map[h], op->mir_map[h] };
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (maps[i]) ptx::fence_tensormap_acquire(maps[i]);
                    }
                    ok = wait_count(op->counter, __ldg(&op->need), abort_flag, status, 206);
                    ptx::fence_proxy_async_global();     // other SMs' results, before loads through the async proxy
                }
                if (ok) ptx::mbar_arrive(bar_dep + 8 * slot);
            }
            __syncwarp();
        } else if (warp == 3) {
            // ---------------- count the tile ----------------
            if (lane == 0) {
                uint32_t* counter = op->counter;
                if (soft ? wait_phase_idle(bar_landed + 8 * (n & 3), (n >> 2) & 1, abort_flag, status, 209)
                         : wait_phase(bar_landed + 8 * (n & 3), (n >> 2) & 1, abort_flag, status, 209)) {
                    red_release_gpu_add(counter, 1u);
                    ptx::mbar_arrive_remote(ptx::map_to_cta(bar_acc_empty + 8 * buf, 0));
                }
            }
            __syncwarp();
        } else {
            // ---------------- epilogue ----------------
            const int q = warp & 3, half = (warp - 4) >> 2;
            const int M = __ldg(&op->M), N = __ldg(&op->N), e_pitch = __ldg(&op->e_pitch);
            // Accumulators: 128 rows a CTA lie one per lane; of 64 rows the lower 64 lanes hold the first half of the
            // columns, the upper ones the second.  A warp reads its quarter of the lanes and half of the columns there.
            constexpr int PIECES = BM == 256 ? BN / 64 : BN / 128;
            const int row0 = tm * BM + (int)rank * (BM / 2) + (BM == 256 ? q : q & 1) * 32, row = row0 + lane;
            const int col_first = tn * BN + (BM == 256 ? half : (q & 2) + half) * (32 * PIECES);
            const uint32_t acc = tmem_base + ((uint32_t)(q * 32) << 16) + buf * BN + (uint32_t)(half * 32 * PIECES);
            const float alpha = __ldg(&op->alpha), b1 = __ldg(&op->b1), b2 = __ldg(&op->b2), diag = __ldg(&op->diag);
            const int64_t at0 = (int64_t)row * e_pitch + col_first;
            const __half* e1 = op->e1[0];
            const __half* e2 = SPLIT ? op->e2[0] : nullptr;
            const __half* e1l = SPLIT ? op->e1[1] : nullptr;
            const __half* e2l = SPLIT ? op->e2[1] : nullptr;
            const bool sym = __ldg(&op->sym) != 0, mirror = sym && tn * BN >= (tm + 1) * BM;
            const void* out_map[2] = { op->out_map[0], SPLIT ? op->out_map[1] : nullptr };
            const void* mir_map[2] = { op->mir_map[0], SPLIT ? op->mir_map[1] : nullptr };
            const uint32_t mine = staging + (uint32_t)(warp - 4) * 4096u, mine_t = mine + 2048u;
            const bool ok = __all_sync(0xFFFFFFFFu, wait_phase(bar_dep + 8 * slot, ring_phase, abort_flag, status, 210));
            const bool some = ok && row0 < M && col_first < N, in = some && row < M;
            // the terms beside the product come from L2 (other SMs wrote them in this launch), one piece ahead
            uint4 t1[4], t1l[SPLIT ? 4 : 1];
            if (e1) {
                load_term(t1, e1 + at0, in);
                if constexpr (SPLIT) load_term(t1l, e1l + at0, in);
            }
            const bool acc_ok = ok && __all_sync(0xFFFFFFFFu, soft ? wait_phase_idle(bar_acc_full + 8 * buf, use & 1, abort_flag, status, 204)
                                                                    : wait_phase(bar_acc_full + 8 * buf, use & 1, abort_flag, status, 204));
            ptx::tc_fence_after_sync();
            if (acc_ok && some) {
#pragma unroll 1
                for (int ch = 0; ch < PIECES; ++ch) {
                    const int col = col_first + ch * 32;
                    if (col >= N) break;
                    const int64_t at = at0 + ch * 32;
                    uint4 t2[SPLIT ? 4 : 1], t2l[SPLIT ? 4 : 1];
                    if constexpr (SPLIT) {
                        if (e2) {
                            load_term(t2, e2 + at, in);
                            load_term(t2l, e2l + at, in);
                        }
                    }
                    float v[32];
                    ptx::tmem_ld32(acc + (uint32_t)(ch * 32), v);
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] *= alpha;
                    if (e1) {
                        add_term(v, b1, t1);
                        if constexpr (SPLIT) add_term(v, b1, t1l);
                        if (ch + 1 < PIECES && col + 32 < N) {
                            load_term(t1, e1 + at + 32, in);
                            if constexpr (SPLIT) load_term(t1l, e1l + at + 32, in);
                        }
                    }
                    if constexpr (SPLIT) {
                        if (e2) {
                            add_term(v, b2, t2);
                            add_term(v, b2, t2l);
                        }
                    }
                    if (diag != 0.0f && row >= col && row < col + 32) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] += row == col + i ? diag : 0.0f;
                    }
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = pack_half2(v[2 * i], v[2 * i + 1]);
#pragma unroll
                    for (int h = 0; h < (SPLIT ? 2 : 1); ++h) {
                        // transposed: neighbouring lanes (rows) exchange halves of two columns, the even lane then holds
                        // both rows of the first column, the odd lane of the second; 32 different banks a store
                        uint32_t tr[16];
                        if (mirror) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, w[i], 1);
                                tr[i] = lane & 1 ? __byte_perm(other, w[i], 0x7632) : __byte_perm(w[i], other, 0x5410);
                            }
                        }
                        if (lane == 0) ptx::bulk_wait_read();        // the stores of the last piece have read the staging
                        __syncwarp();
                        // rows of 64 bytes in the 64-byte swizzle of the store's map: the 16-byte unit of a row is
                        // exchanged with bits 1..2 of the row, so that eight lanes hit eight different units
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            ptx::st_shared_v4(mine + (uint32_t)(lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4)), w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
                        if (mirror) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) ptx::st_shared_b32(mine_t + (uint32_t)((2 * i + (lane & 1)) * 64 + (lane >> 1) * 4), tr[i]);
                        }
                        ptx::fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            ptx::tma_store_2d(out_map[h], col, row0, mine);
                            if (mirror) ptx::tma_store_2d(mir_map[h], row0, col, mine_t);
                            ptx::bulk_commit();
                        }
                        if (SPLIT && h == 0) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float2 f = unpack_half2(w[i]);
                                w[i] = pack_half2(v[2 * i] - f.x, v[2 * i + 1] - f.y);
                            }
                        }
                    }
                }
            }
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0 && acc_ok) {
                ptx::mbar_arrive_remote(ptx::map_to_cta(bar_acc_empty + 8 * buf, 0));
                ptx::bulk_wait_all();                    // this warp's part of the tile is in memory (a completed bulk
                ptx::mbar_arrive(bar_landed + 8 * (n & 3));      // store needs no further proxy fence)
            }
            __syncwarp();
        }
        if (__shfl_sync(0xFFFFFFFFu, *abort_flag, 0) != 0) break;
    }

    if (warp >= 4 && lane == 0) ptx::bulk_wait_all();
    // The leader lets the loads of both CTAs and its MMAs finish before either CTA gives up shared memory or TMEM.
    if (tid == 0 && rank == 0) {
        for (uint32_t s = 0; s < (uint32_t)Cfg::STAGES && s < it; ++s) {
            const uint32_t last = s + (it - 1 - s) / Cfg::STAGES * Cfg::STAGES;
            drain_phase(bar_full + 8 * s, (last / Cfg::STAGES) & 1);
        }
    }
    if (rank == 0 && tid == 32) {
        ptx::mma_commit_pair(bar_drain, 1);
        drain_phase(bar_drain, 0);
    }
    // the peer cannot watch the leader's barriers: after a wait gave up it lets its last loads land for 2 ms
    if (rank == 1 && tid == 0 && *abort_flag)
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::cluster_sync();
    if (warp == 1) ptx::tmem_dealloc_pair(tmem_base, 512);
}

// ------------------------------------------------------------------------------------------------------------------
// Streaming passes.  Elements of U: with `STEP` from the momentum (already updated) and the gradient, else U itself.
namespace {

constexpr int MS_THREADS = 256;
constexpr int MS_ROWS = 64, MS_COLS = 64;               // tile of the load and apply kernels
// Where rows are whole vectors on both sides a tile is 32 x this many rows (7B layer: load 320 us with 2, 365 with 4;
// apply 350 with 2, 307 with 4).
constexpr int MS_LOAD_VEC = 2, MS_APPLY_VEC = 4;

__device__ __forceinline__ int find_item(const MuonArgs& a, int tile)
{
    int lo = 0, hi = a.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.tile_begin[mid] <= tile) lo = mid; else hi = mid;
    }
    return lo;
}

template <bool STEP>
__device__ __forceinline__ float update_of(float g, float m, const MuonArgs& a)
{
    if constexpr (!STEP) return g;
    return a.nesterov ? fmaf(a.mu, m, (1.0f - a.mu) * g) : m;
}

// Two neighbours at p + at, `left` of them inside the row; as one access where rows are whole pairs.
__device__ __forceinline__ void pair_at(const float* p, float (&v)[2])
{
    const float2 t = __ldcs(reinterpret_cast<const float2*>(p));
    v[0] = t.x; v[1] = t.y;
}
__device__ __forceinline__ void pair_at(const __nv_bfloat16* p, float (&v)[2])
{
    const uint32_t t = __ldcs(reinterpret_cast<const uint32_t*>(p));
    v[0] = __uint_as_float(t << 16); v[1] = __uint_as_float(t & 0xFFFF0000u);
}
__device__ __forceinline__ float one_at(const float* p) { return __ldcs(p); }
__device__ __forceinline__ float one_at(const __nv_bfloat16* p) { return bf16_bits_to_float((uint32_t)__ldcs(reinterpret_cast<const unsigned short*>(p))); }
template <typename T>
__device__ __forceinline__ void load_pair(const T* p, int64_t at, int left, bool pairs, int64_t numel, float (&v)[2], int32_t* status)
{
    v[0] = v[1] = 0.0f;
    if (left >= 2 && pairs) {
        if (APOLLO_DBG_RANGE(at, at + 1, numel, status)) pair_at(p + at, v);
    } else {
        if (left >= 1 && APOLLO_DBG_RANGE(at, at, numel, status)) v[0] = one_at(p + at);
        if (left >= 2 && APOLLO_DBG_RANGE(at + 1, at + 1, numel, status)) v[1] = one_at(p + at + 1);
    }
}
__device__ __forceinline__ void store2(float* p, const float (&v)[2]) { *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]); }
__device__ __forceinline__ void store2(__nv_bfloat16* p, const float (&v)[2]) { *reinterpret_cast<uint32_t*>(p) = pack_bf16x2(v[0], v[1]); }
__device__ __forceinline__ void store8(float* p, const float (&v)[8])
{
    __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
    __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8])
{
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])));
}

__device__ __forceinline__ void store_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_elem(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

}  // namespace

// A block takes one of the matrix's n_part contiguous pieces (a multiple of 8 elements long): momentum in place,
// squares added in fp32 over eight elements (in fp64 where those leave the range of fp32: entries above 1e19 or below
// 1e-15) and in fp64 from there on, one partial sum per block in a fixed order.
template <typename T, bool STEP>
__global__ void __launch_bounds__(MS_THREADS)
muon_moment_kernel(const __grid_constant__ MuonArgs a, int32_t* __restrict__ status)
{
    __shared__ double scratch[32];
    ptx::grid_launch_dependents();
    const int k = find_item(a, blockIdx.x);
    const MuonItem& it = a.item[k];
    if ((int)blockIdx.x == a.tile_begin[k] && threadIdx.x == 0) {      // counters of the products that follow
        *it.counter = 0;
        *a.ticket = 0;
    }
    const int piece = (int)blockIdx.x - a.tile_begin[k];
    const int64_t numel = (int64_t)it.rows * it.cols;
    const int64_t len = ((numel + it.n_part - 1) / it.n_part + 7) / 8 * 8;
    const int64_t begin = min((int64_t)piece * len, numel), end = min(begin + len, numel);
    const T* __restrict__ G = static_cast<const T*>(it.g);
    float* __restrict__ M = it.m;
    double sum = 0.0;
    auto one = [&](float g, float& m) {
        if constexpr (STEP) m = fmaf(a.mu, m, (1.0f - a.mu) * g);
        return update_of<STEP>(g, m, a);
    };
    for (int64_t e = begin + (int64_t)threadIdx.x * 8; e < end; e += MS_THREADS * 16) {
        // two vectors of eight per round, all loads before the first use
        float g[2][8], m[2][8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t p = e + u * (MS_THREADS * 8);
            const int count = (int)min((int64_t)8, end - p);
            if (count == 8 && APOLLO_DBG_RANGE(p, p + 7, numel, status)) {
                load8_stream(G + p, g[u]);
                if constexpr (STEP) load8_stream(M + p, m[u]);
            } else {
                load8_guarded(G + p, count, g[u]);
                if constexpr (STEP) load8_guarded(M + p, count, m[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t p = e + u * (MS_THREADS * 8);
            const int count = (int)min((int64_t)8, end - p);
            if (count <= 0) break;
            float s = 0.0f;
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                g[u][x] = one(g[u][x], m[u][x]);
                s += g[u][x] * g[u][x];
            }
            if (s >= 1e-30f && s <= 1e38f) {
                sum += (double)s;
            } else {
#pragma unroll
                for (int x = 0; x < 8; ++x) sum += (double)g[u][x] * (double)g[u][x];
            }
            if constexpr (STEP) {
                if (count == 8 && APOLLO_DBG_RANGE(p, p + 7, numel, status)) {
                    reinterpret_cast<float4*>(M + p)[0] = make_float4(m[u][0], m[u][1], m[u][2], m[u][3]);
                    reinterpret_cast<float4*>(M + p)[1] = make_float4(m[u][4], m[u][5], m[u][6], m[u][7]);
                } else {
#pragma unroll
                    for (int x = 0; x < 8; ++x)
                        if (x < count) M[p + x] = m[u][x];
                }
            }
        }
    }
    const double total = block_sum(sum, scratch);
    if (threadIdx.x == 0) it.part[piece] = total;
}

// X = U x_scale / (|U| + eps) as 16-bit floats (high and low part with `SPLIT`), transposed when tall.
template <typename T, bool STEP, bool SPLIT>
__global__ void __launch_bounds__(MS_THREADS)
muon_load_kernel(const __grid_constant__ MuonArgs a, int32_t* __restrict__ status)
{
    __shared__ double scratch[32];
    __shared__ float tile[MS_ROWS][MS_COLS + 1];
    const int k = find_item(a, blockIdx.x);
    const MuonItem& it = a.item[k];
    const int local = (int)blockIdx.x - a.tile_begin[k];
    const int rows = it.rows, cols = it.cols, tiles_c = (cols + MS_COLS - 1) / MS_COLS;
    const bool vectors = muon_stream_vectors(cols, it.tall != 0);
    const int r0 = local / tiles_c * (vectors ? 32 * MS_LOAD_VEC : MS_ROWS), c0 = (local - local / tiles_c * tiles_c) * MS_COLS;
    const T* __restrict__ G = static_cast<const T*>(it.g);
    const float* M = it.m;
    ptx::grid_launch_dependents();
    ptx::grid_wait_previous();
    const int64_t numel = (int64_t)rows * cols, extent = (int64_t)(it.tall ? cols : rows) * it.x_pitch;
    __half* __restrict__ hi = it.x[0];
    __half* __restrict__ lo = it.x[1];
    // the sum of squares comes last: its loads and the reduction hide behind those of the elements
    float pre = 1.0f, f = 0.0f;
    auto factor = [&]() {
        const double norm = sqrt(block_sum((int)threadIdx.x < it.n_part ? it.part[threadIdx.x] : 0.0, scratch));
        const float to = (float)norm + a.eps;
        f = a.x_scale / to;
        if (!(to >= 0x1p-60f && to <= 0x1p74f)) {        // the factor or its product with an element could leave fp32: in two parts
            pre = norm > 1.0 ? 0x1p-64f : 0x1p64f;
            f = (float)(a.x_scale / (norm + (double)a.eps) / pre);
        }
    };
    if (vectors) {
        // rows are whole vectors on both sides
        const int c = c0 + (threadIdx.x & 7) * 8, r1 = r0 + (threadIdx.x >> 3);
        float u[MS_LOAD_VEC][8];
#pragma unroll
        for (int i = 0; i < MS_LOAD_VEC; ++i) {
            const int r = r1 + 32 * i;
            const int64_t at = (int64_t)r * cols + c;
            float m[8];
            if (r < rows && c < cols && APOLLO_DBG_RANGE(at, at + 7, numel, status)) {
                load8_stream(G + at, u[i]);
                if constexpr (STEP) load8_stream(M + at, m);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) u[i][e] = m[e] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) u[i][e] = update_of<STEP>(u[i][e], m[e], a);
        }
        factor();
#pragma unroll
        for (int i = 0; i < MS_LOAD_VEC; ++i) {
            const int r = r1 + 32 * i;
            const int64_t at = (int64_t)r * it.x_pitch + c;
            if (r >= rows || c >= cols || !APOLLO_DBG_RANGE(at, at + 7, extent, status)) continue;
            uint32_t w[4], l[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v0 = u[i][2 * e] * pre * f, v1 = u[i][2 * e + 1] * pre * f;
                w[e] = pack_half2(v0, v1);
                if constexpr (SPLIT) {
                    const float2 h = unpack_half2(w[e]);
                    l[e] = pack_half2(v0 - h.x, v1 - h.y);
                }
            }
            *reinterpret_cast<uint4*>(hi + at) = make_uint4(w[0], w[1], w[2], w[3]);
            if constexpr (SPLIT) *reinterpret_cast<uint4*>(lo + at) = make_uint4(l[0], l[1], l[2], l[3]);
        }
        return;
    }
    // two columns per thread (a pair of elements is read at once where rows are whole pairs), eight rows
    const int c = (threadIdx.x & 31) * 2, rr = threadIdx.x >> 5;
    float u[8][2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + rr + 8 * i;
        const int64_t at = (int64_t)r * cols + c0 + c;
        float m[2];
        load_pair(G, at, r < rows ? cols - c0 - c : 0, cols % 2 == 0, numel, u[i], status);
        if constexpr (STEP) load_pair(M, at, r < rows ? cols - c0 - c : 0, cols % 2 == 0, numel, m, status);
        u[i][0] = update_of<STEP>(u[i][0], m[0], a);
        u[i][1] = update_of<STEP>(u[i][1], m[1], a);
    }
    factor();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        u[i][0] = u[i][0] * pre * f;
        u[i][1] = u[i][1] * pre * f;
    }
    // two neighbours of one row of X (its pitch is a multiple of 64: pairs are always aligned)
    auto put = [&](int64_t at, float v0, float v1) {
        if (!APOLLO_DBG_RANGE(at, at + 1, extent, status)) return;
        const uint32_t w = pack_half2(v0, v1);
        *reinterpret_cast<uint32_t*>(hi + at) = w;
        if constexpr (SPLIT) {
            const float2 h = unpack_half2(w);
            *reinterpret_cast<uint32_t*>(lo + at) = pack_half2(v0 - h.x, v1 - h.y);
        }
    };
    if (!it.tall) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = r0 + rr + 8 * i;
            if (r < rows && c0 + c < cols) put((int64_t)r * it.x_pitch + c0 + c, u[i][0], u[i][1]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) { tile[rr + 8 * i][c] = u[i][0]; tile[rr + 8 * i][c + 1] = u[i][1]; }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int cc = rr + 8 * i;                   // source column = row of X
            if (c0 + cc < cols && r0 + c < rows) put((int64_t)(c0 + cc) * it.x_pitch + r0 + c, tile[c][cc], tile[c + 1][cc]);
        }
    }
}

// W <- W - lr (gain X + wd W), or O = X; X is read back transposed when tall.
template <typename T, bool STEP, bool SPLIT>
__global__ void __launch_bounds__(MS_THREADS)
muon_apply_kernel(const __grid_constant__ MuonArgs a, int32_t* __restrict__ status)
{
    __shared__ float tile[MS_ROWS][MS_COLS + 1];
    ptx::grid_wait_previous();
    if (*reinterpret_cast<volatile int32_t*>(status) != STATUS_OK) return;      // a product gave up: leave the weights
    const int k = find_item(a, blockIdx.x);
    const MuonItem& it = a.item[k];
    const int local = (int)blockIdx.x - a.tile_begin[k];
    const int rows = it.rows, cols = it.cols, tiles_c = (cols + MS_COLS - 1) / MS_COLS;
    const bool vectors = muon_stream_vectors(cols, it.tall != 0);
    const int r0 = local / tiles_c * (vectors ? 32 * MS_APPLY_VEC : MS_ROWS), c0 = (local - local / tiles_c * tiles_c) * MS_COLS;
    T* __restrict__ W = static_cast<T*>(it.w);
    const __half* hi = it.x[0];
    const __half* lo = it.x[1];
    const float f = 1.0f / a.x_scale;                    // a power of two
    const int64_t numel = (int64_t)rows * cols, extent = (int64_t)(it.tall ? cols : rows) * it.x_pitch;
    auto moved = [&](float w, float x) {
        if constexpr (STEP) return fmaf(-a.lr, fmaf(a.wd, w, it.gain * x), w);
        return x;
    };
    if (vectors) {
        const int c = c0 + (threadIdx.x & 7) * 8, r1 = r0 + (threadIdx.x >> 3);
        uint4 x[MS_APPLY_VEC], y[SPLIT ? MS_APPLY_VEC : 1];
        Raw8<T> w[MS_APPLY_VEC];
        bool in[MS_APPLY_VEC];
#pragma unroll
        for (int i = 0; i < MS_APPLY_VEC; ++i) {
            const int r = r1 + 32 * i;
            const int64_t at = (int64_t)r * it.x_pitch + c, aw = (int64_t)r * cols + c;
            in[i] = r < rows && c < cols && APOLLO_DBG_RANGE(at, at + 7, extent, status) && APOLLO_DBG_RANGE(aw, aw + 7, numel, status);
            if (!in[i]) continue;
            x[i] = __ldcs(reinterpret_cast<const uint4*>(hi + at));
            if constexpr (SPLIT) y[i] = __ldcs(reinterpret_cast<const uint4*>(lo + at));
            if constexpr (STEP) w[i] = load_raw8_stream(W + aw);
        }
#pragma unroll
        for (int i = 0; i < MS_APPLY_VEC; ++i) {
            if (!in[i]) continue;
            const uint32_t xw[4] = { x[i].x, x[i].y, x[i].z, x[i].w };
            float v[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 h = unpack_half2(xw[e]);
                v[2 * e] = h.x; v[2 * e + 1] = h.y;
            }
            if constexpr (SPLIT) {
                const uint32_t yw[4] = { y[i].x, y[i].y, y[i].z, y[i].w };
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 h = unpack_half2(yw[e]);
                    v[2 * e] += h.x; v[2 * e + 1] += h.y;
                }
            }
            float old[8];
            if constexpr (STEP) unpack_raw8(w[i], old);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = moved(STEP ? old[e] : 0.0f, v[e] * f);
            store8(W + (int64_t)(r1 + 32 * i) * cols + c, v);
        }
        return;
    }
    const int c = (threadIdx.x & 31) * 2, rr = threadIdx.x >> 5;
    auto get = [&](int64_t at, float (&v)[2]) {          // two neighbours of one row of X; the second may be padding
        if (!APOLLO_DBG_RANGE(at, at + 1, extent, status)) { v[0] = v[1] = 0.0f; return; }
        float2 h = unpack_half2(*reinterpret_cast<const uint32_t*>(hi + at));
        if constexpr (SPLIT) {
            const float2 l = unpack_half2(*reinterpret_cast<const uint32_t*>(lo + at));
            h.x += l.x; h.y += l.y;
        }
        v[0] = h.x * f; v[1] = h.y * f;
    };
    float x[8][2];
    if (!it.tall) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = r0 + rr + 8 * i;
            if (r < rows && c0 + c < cols) get((int64_t)r * it.x_pitch + c0 + c, x[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int cc = rr + 8 * i;
            float v[2] = { 0.0f, 0.0f };
            if (c0 + cc < cols && r0 + c < rows) get((int64_t)(c0 + cc) * it.x_pitch + r0 + c, v);
            tile[c][cc] = v[0]; tile[c + 1][cc] = v[1];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) { x[i][0] = tile[rr + 8 * i][c]; x[i][1] = tile[rr + 8 * i][c + 1]; }
    }
    float w[8][2];
    if constexpr (STEP) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = r0 + rr + 8 * i;
            load_pair(W, (int64_t)r * cols + c0 + c, r < rows ? cols - c0 - c : 0, cols % 2 == 0, numel, w[i], status);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + rr + 8 * i, left = r < rows ? cols - c0 - c : 0;
        const int64_t at = (int64_t)r * cols + c0 + c;
        const float v[2] = { moved(STEP ? w[i][0] : 0.0f, x[i][0]), moved(STEP ? w[i][1] : 0.0f, x[i][1]) };
        if (left >= 2 && cols % 2 == 0) {
            if (APOLLO_DBG_RANGE(at, at + 1, numel, status)) store2(W + at, v);
        } else {
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (e < left && APOLLO_DBG_RANGE(at + e, at + e, numel, status)) store_elem(W + at + e, v[e]);
        }
    }
}

// ------------------------------------------------------------------------------------------------------------------
int muon_stream_tiles(int rows, int cols, bool tall, bool apply)
{
    const int tile_rows = muon_stream_vectors(cols, tall) ? 32 * (apply ? MS_APPLY_VEC : MS_LOAD_VEC) : MS_ROWS;
    return ((rows + tile_rows - 1) / tile_rows) * ((cols + MS_COLS - 1) / MS_COLS);
}

cudaError_t launch_muon_moment(int dtype, bool step, const MuonArgs& a, int tiles, int32_t* d_status, cudaStream_t stream)
{
    if (dtype == APOLLO_DT_BF16) {
        if (step) muon_moment_kernel<__nv_bfloat16, true><<<tiles, MS_THREADS, 0, stream>>>(a, d_status);
        else muon_moment_kernel<__nv_bfloat16, false><<<tiles, MS_THREADS, 0, stream>>>(a, d_status);
    } else {
        if (step) muon_moment_kernel<float, true><<<tiles, MS_THREADS, 0, stream>>>(a, d_status);
        else muon_moment_kernel<float, false><<<tiles, MS_THREADS, 0, stream>>>(a, d_status);
    }
    return cudaGetLastError();
}

// (fp32 weights are always split)
cudaError_t launch_muon_load(int dtype, bool split, bool step, const MuonArgs& a, int tiles, int32_t* d_status, cudaStream_t stream)
{
    const auto kernel = dtype == APOLLO_DT_F32 ? (step ? muon_load_kernel<float, true, true> : muon_load_kernel<float, false, true>)
                        : split                ? (step ? muon_load_kernel<__nv_bfloat16, true, true> : muon_load_kernel<__nv_bfloat16, false, true>)
                                               : (step ? muon_load_kernel<__nv_bfloat16, true, false> : muon_load_kernel<__nv_bfloat16, false, false>);
    return launch_after(kernel, dim3((unsigned)tiles), dim3(MS_THREADS), stream, a, d_status);
}

cudaError_t launch_muon_apply(int dtype, bool split, bool step, const MuonArgs& a, int tiles, int32_t* d_status, cudaStream_t stream)
{
    const auto kernel = dtype == APOLLO_DT_F32 ? (step ? muon_apply_kernel<float, true, true> : muon_apply_kernel<float, false, true>)
                        : split                ? (step ? muon_apply_kernel<__nv_bfloat16, true, true> : muon_apply_kernel<__nv_bfloat16, false, true>)
                                               : (step ? muon_apply_kernel<__nv_bfloat16, true, false> : muon_apply_kernel<__nv_bfloat16, false, false>);
    return launch_after(kernel, dim3((unsigned)tiles), dim3(MS_THREADS), stream, a, d_status);
}

namespace {

template <bool SPLIT, int TILE>
cudaError_t launch_gemm(const GemmOp* d_ops, const uint64_t* d_list, int tiles, uint32_t* d_ticket, MuonLaunch& state, int32_t* d_status, cudaStream_t stream)
{
    const auto kernel = muon_gemm_kernel<SPLIT, TILE>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(state.sm_count / 2 * 2));
    cfg.blockDim = dim3(MG_THREADS);
    cfg.dynamicSmemBytes = GemmCfg<TILE>::SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int& pairs = state.max_pairs[TILE];
    if (pairs == 0) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, GemmCfg<TILE>::SMEM);
        if (e != cudaSuccess) return e;
        int clusters = 0;
        const cudaError_t o = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg);
        if (o != cudaSuccess) return o;
        if (clusters < 1) return cudaErrorLaunchOutOfResources;
        pairs = clusters;
    }
    cfg.numAttrs = 2;
    cfg.gridDim = dim3((unsigned)(2 * (tiles < pairs ? tiles : pairs)));
    return cudaLaunchKernelEx(&cfg, kernel, d_ops, d_list, (uint32_t)tiles, d_ticket, d_status);
}

}  // namespace

cudaError_t launch_muon_gemm(bool split, int tile, const GemmOp* d_ops, const uint64_t* d_list, int tiles, uint32_t* d_ticket, MuonLaunch& state,
                             int32_t* d_status, cudaStream_t stream)
{
    using Launch = cudaError_t (*)(const GemmOp*, const uint64_t*, int, uint32_t*, MuonLaunch&, int32_t*, cudaStream_t);
    static constexpr Launch by_tile[MUON_TILE_KINDS][2] = { { launch_gemm<false, TILE_WIDE>, launch_gemm<true, TILE_WIDE> },
                                                            { launch_gemm<false, TILE_TALL>, launch_gemm<true, TILE_TALL> },
                                                            { launch_gemm<false, TILE_SMALL>, launch_gemm<true, TILE_SMALL> } };
    return by_tile[tile][split](d_ops, d_list, tiles, d_ticket, state, d_status, stream);
}

int muon_encode_maps(const __half* base, int rows, int cols, int pitch, void* maps)
{
    EncodeTiledFn encode = encode_fn();
    if (!encode) return APOLLO_ERR_CUDA;
    const cuuint64_t dims[2] = { (cuuint64_t)cols, (cuuint64_t)rows };
    const cuuint64_t strides[1] = { (cuuint64_t)pitch * 2 };
    const cuuint32_t elem[2] = { 1u, 1u };
    auto make = [&](int kind, cuuint32_t w, cuuint32_t h, CUtensorMapSwizzle sw) {
        const cuuint32_t box[2] = { w, h };
        return encode(static_cast<CUtensorMap*>(maps) + kind, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<__half*>(base), dims, strides, box, elem,
                      CU_TENSOR_MAP_INTERLEAVE_NONE, sw, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    return make(MAP_ROWS, 64, 128, CU_TENSOR_MAP_SWIZZLE_128B) && make(MAP_COLS, 64, 64, CU_TENSOR_MAP_SWIZZLE_128B) &&
           make(MAP_STORE, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B) && make(MAP_MIRROR, 32, 32, CU_TENSOR_MAP_SWIZZLE_NONE)
               ? APOLLO_OK : APOLLO_ERR_CUDA;
}

}  // namespace apollo
