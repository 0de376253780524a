// Structures shared by the host side of the orthogonalised update and its kernels.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace apollo {

// Tiles of a product, rows x columns; the rows are shared by the two CTAs of a pair.
struct MuonTile { int m, n; };
constexpr MuonTile MUON_TILES[] = { { 256, 256 }, { 256, 128 }, { 128, 128 } };
enum { TILE_WIDE, TILE_TALL, TILE_SMALL, MUON_TILE_KINDS };
constexpr int MUON_CHUNK = 48;          // matrices whose pointers travel in one launch of a streaming kernel
constexpr int MUON_PART = 256;          // most partial sums of squares per matrix

// out = alpha L R + b1 E1 + b2 E2 + diag I on stored (scaled) values; L is M x K with k contiguous, R is K x N, with
// k contiguous (r_mn = 0: given as the N x K matrix) or with n contiguous (r_mn = 1).  [0] / [1]: the high and low
// parts of split operands.  sym: M = N and the result is symmetric: it is computed from the diagonal's blocks of
// MuonTile::m rows and columns on, and what lies beyond them also stored transposed.
struct GemmOp {
    const void* l_map[2];               // DEVICE tensor maps
    const void* r_map[2];
    const void* out_map[2];
    const void* mir_map[2];             // sym
    const __half* e1[2];                // same place and pitch as the output; null = none
    const __half* e2[2];                // (split operands only)
    float alpha, b1, b2, diag;
    int32_t M, N, K, e_pitch, sym, r_mn;
    uint32_t* counter;                  // DEVICE: CTAs done with tiles of this matrix, over all its products
    uint32_t need;                      // its value once the products before this one are complete
};
constexpr int MUON_COUNTS_PER_TILE = 2;

// One matrix of a streaming kernel.
struct MuonItem {
    void* w;                            // weights / the orthogonalised result
    const void* g;
    float* m;
    __half* x[2];                       // iterate, m x n (transposed when tall), high and low parts
    double* part;                       // partial sums of squares of U
    uint32_t* counter;                  // GemmOp::counter, zeroed by the first pass
    int32_t rows, cols, x_pitch, n_part;
    int32_t tall;
    float gain;                         // s of the update
};

struct MuonArgs {
    MuonItem item[MUON_CHUNK];
    int32_t tile_begin[MUON_CHUNK + 1];
    int32_t n;
    float mu, eps, x_scale, lr, wd;     // x_scale: the power of two the iterates carry
    int32_t nesterov;
    uint32_t* ticket;                   // DEVICE: next tile of the products, zeroed by the first pass
};

struct MuonLaunch {                     // what the launches of a context need to know about the device
    int sm_count;
    int max_pairs[MUON_TILE_KINDS];     // resident pairs of the kernels by tile; 0 = not asked yet
};

// Sum of squares of U (and M <- mu M + (1 - mu) G with `step`), X = U x_scale / (|U| + eps) in 16 bits, and the end:
// W <- W - lr (gain X + wd W) with `step`, O = X without.
cudaError_t launch_muon_moment(int dtype, bool step, const MuonArgs& a, int tiles, int32_t* d_status, cudaStream_t stream);
cudaError_t launch_muon_load(int dtype, bool split, bool step, const MuonArgs& a, int tiles, int32_t* d_status, cudaStream_t stream);
cudaError_t launch_muon_apply(int dtype, bool split, bool step, const MuonArgs& a, int tiles, int32_t* d_status, cudaStream_t stream);
// Tiles of one matrix in the load and apply kernels, and whether they go by vectors of eight (rows of the matrix and of
// the iterate are whole vectors, and nothing is transposed).
__host__ __device__ inline bool muon_stream_vectors(int cols, bool tall) { return !tall && cols % 8 == 0; }
int muon_stream_tiles(int rows, int cols, bool tall, bool apply);

// A tile of the list in 64 bits (16 bytes a tile were a fortieth of a workspace cut into small groups): the product, its
// place, the k-blocks of its contraction, R along n.
constexpr int TILE_OP_BITS = 21, TILE_M_BITS = 13, TILE_N_BITS = 13, TILE_K_BITS = 16;
constexpr int TILE_M_AT = TILE_OP_BITS, TILE_N_AT = TILE_M_AT + TILE_M_BITS, TILE_K_AT = TILE_N_AT + TILE_N_BITS, TILE_R_AT = TILE_K_AT + TILE_K_BITS;
static_assert(TILE_R_AT == 63, "a tile has 64 bits");
__host__ __device__ inline uint64_t pack_tile(uint32_t op, uint32_t tm, uint32_t tn, uint32_t kb, uint32_t r_mn)
{
    return (uint64_t)op | (uint64_t)tm << TILE_M_AT | (uint64_t)tn << TILE_N_AT | (uint64_t)kb << TILE_K_AT | (uint64_t)r_mn << TILE_R_AT;
}
__host__ __device__ inline uint32_t tile_field(uint64_t tile, int at, int bits) { return (uint32_t)(tile >> at) & ((1u << bits) - 1); }

// All products of a group; d_list: its tiles (DEVICE), d_ticket: DEVICE, zero.
cudaError_t launch_muon_gemm(bool split, int tile, const GemmOp* d_ops, const uint64_t* d_list, int tiles, uint32_t* d_ticket, MuonLaunch& state,
                             int32_t* d_status, cudaStream_t stream);

// Tensor maps of a rows x cols matrix of 16-bit floats (pitch a multiple of 8), 128 bytes each at maps[kind]: boxes of
// 64 x 128 rows (an operand whose rows are contiguous along k) and 64 x 64 (half as many of them, or contiguous along n) to
// load, 32 x 32 to store a piece, and to store it transposed.
enum { MAP_ROWS, MAP_COLS, MAP_STORE, MAP_MIRROR, MUON_MAPS };
int muon_encode_maps(const __half* base, int rows, int cols, int pitch, void* maps);

}  // namespace apollo
