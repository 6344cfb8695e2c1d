// Low-rank adapters beside a frozen layer, forward and backward, for gfx950.
//
// Row m of a batch has the adapter a = index[m] (any value outside 0 .. L-1: none; no index: adapter 0 for every row):
//   H[m] = X[m] A[a]^T                       shrink, contraction over K
//   Y'[m] = Y[m] + s[a] H[m] B[a]^T           expand, contraction over the rank
//   dH[m] = s[a] dY[m] B[a]                   shrink, contraction over N, B turned
//   dX'[m] = dX[m] + dH[m] A[a]               expand, A turned
//   dA[a] = sum_m dH[m]^T X[m],  dB[a] = sum_m s[a] dY[m]^T H[m]      outer, contraction over the rows of the adapter
// The 16-bit tensors enter the matrix cores as they are.  H and dH are fp32 between the kernels; where they are an operand they are
// split into two or three 16-bit terms, so that nothing but the results is rounded to 16 bits.
#include "fp6_common.hpp"

namespace fp6 {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr int kNoAdapter = -1;

// The adapter of a row, or kNoAdapter.
__device__ __forceinline__ int adapter_of(const int32_t* __restrict__ index, int64_t row, int64_t M, int adapters)
{
    if (row >= M) return kNoAdapter;
    if (!index) return 0;
    const int a = index[row];
    return (unsigned)a < (unsigned)adapters ? a : kNoAdapter;
}

template <int FMT>
__device__ __forceinline__ float to_float(uint16_t w)
{
    if (FMT == kE3M2B) return __builtin_bit_cast(float, (uint32_t)w << 16);
    return (float)__builtin_bit_cast(_Float16, w);
}

template <int FMT>
__device__ __forceinline__ uint16_t to_bits(float v)
{
    if (FMT == kE3M2B) return __builtin_bit_cast(uint16_t, (__bf16)v);
    return __builtin_bit_cast(uint16_t, (_Float16)v);
}

// 2^e for e in -126 .. 127
__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// The e that brings values of at most `top` below 2^15 after a multiplication by 2^-e (fp16 terms; 0 where top is 0).  An infinity
// among the values gets the largest e, so that the others stay finite.
__device__ __forceinline__ int exponent_for(float top)
{
    const int e = (int)(__builtin_bit_cast(uint32_t, top) >> 23) - 127;          // top < 2^(e+1)
    return top == 0.0f ? 0 : max(e - 14, -126);
}

// v as the sum of 16-bit numbers, the first term nearest to v and each further one nearest to what is left.  An infinity or NaN is its first term alone.
template <int FMT, int TERMS>
__device__ __forceinline__ void split_terms(float v, uint16_t (&t)[TERMS])
{
    float rest = v;
#pragma unroll
    for (int i = 0; i < TERMS; i++) {
        t[i] = to_bits<FMT>(rest);
        const float f = to_float<FMT>(t[i]);
        rest = fabsf(f) < __builtin_inff() ? rest - f : 0.0f;
    }
}

// ------------------------------------------------------------------ shrink
struct ShrinkLayer {
    const uint16_t* Q;      // [M, C]
    const uint16_t* W;      // [adapters, rank, C], turned: [adapters, C, rank]
    float* P;               // [slices, M, rank]
    int C, rank, slices;
    int first;              // first workgroup of this layer
};

struct ShrinkArgs {
    ShrinkLayer layer[FP6_GROUP_MAX];
    int layers;
    int64_t M;
    const int32_t* index;
    const float* scaling;   // multiplies the result (NULL: nothing does)
    int adapters, slots;
};

// P[slice][m][j] = sum over the slice's c of Q[m][c] W[a][j][c].  A workgroup: 16 * RT rows, one slice of the contraction, whose
// 64-wide units its four wavefronts take in turn; a lane holds 16 consecutive values of a row per unit (whole lines).  The
// distinct adapters of the rows are taken one after another, or one per grid slot: each reads its own A.
template <int FMT, int JT, int RT, bool TURNED>
__global__ __launch_bounds__(256) void lora_shrink_kernel(ShrinkArgs args)
{
    constexpr int kLd = 16 * JT + 8;                       // turned: elements between two rows of the staged unit
    __shared__ __align__(16) unsigned char shared[TURNED && 4 * 64 * kLd * 2 > 4 * RT * JT * 1024 ? 4 * 64 * kLd * 2 : 4 * RT * JT * 1024];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    int which = 0;
    while (which + 1 < args.layers && (int)blockIdx.x >= args.layer[which + 1].first) which++;
    const ShrinkLayer L = args.layer[which];
    const int at = (int)blockIdx.x - L.first, slice = at % L.slices;
    const int64_t m0 = (int64_t)(at / L.slices) * (16 * RT);
    const int rank = L.rank, C = L.C, units = C / 64;
    const int u_begin = slice_begin(units, L.slices, slice) + wave, u_end = slice_begin(units, L.slices, slice + 1);

    // (16 * RT <= 32 rows: lane l looks after row l)
    const int mine = lane < 16 * RT ? adapter_of(args.index, m0 + lane, args.M, args.adapters) : kNoAdapter;
    uint64_t pending = __ballot(mine != kNoAdapter);
    const uint64_t none = ~pending & (((uint64_t)1 << (16 * RT)) - 1);
    float* P = L.P + (size_t)slice * args.M * rank;
    if (blockIdx.y == 0 && none) {                         // rows without an adapter
        for (int e = threadIdx.x; e < 16 * RT * rank; e += 256)
            if ((none >> (e / rank)) & 1 && m0 + e / rank < args.M) P[(size_t)(m0 + e / rank) * rank + e % rank] = 0.0f;
    }
    const uint16_t* q[RT];
#pragma unroll
    for (int t = 0; t < RT; t++) {
        const int64_t row = min(m0 + 16 * t + i, args.M - 1);
        q[t] = L.Q + (size_t)row * C + 16 * g;
    }
    for (int seen = 0; pending; seen++) {
        const int a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(pending));
        const uint64_t rows = __ballot(mine == a);
        pending &= ~rows;
        if (seen % args.slots != (int)blockIdx.y) continue;
        const uint16_t* W = L.W + (size_t)a * rank * C;
        float4v acc[RT][JT];
#pragma unroll
        for (int t = 0; t < RT; t++)
#pragma unroll
            for (int j = 0; j < JT; j++) acc[t][j] = float4v{0, 0, 0, 0};
        for (int u = u_begin; u < u_end; u += 4) {
            u32x4 x[RT][2], w[JT][2];
#pragma unroll
            for (int t = 0; t < RT; t++)
#pragma unroll
                for (int h = 0; h < 2; h++) x[t][h] = *reinterpret_cast<const u32x4*>(q[t] + (size_t)u * 64 + 8 * h);
            if (!TURNED) {
#pragma unroll
                for (int j = 0; j < JT; j++)
#pragma unroll
                    for (int h = 0; h < 2; h++)
                        w[j][h] = *reinterpret_cast<const u32x4*>(W + (size_t)min(16 * j + i, rank - 1) * C + (size_t)u * 64 + 16 * g + 8 * h);
            } else {
                // the unit's 64 rows of W (one piece of memory) through the wavefront's own LDS, read back turned
                unsigned char* own = shared + wave * (64 * kLd * 2);
                const u32x4* piece = reinterpret_cast<const u32x4*>(W + (size_t)u * 64 * rank);
                const int per_row = rank / 8;
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
                for (int p = lane; p < 64 * per_row; p += 64)
                    *reinterpret_cast<u32x4*>(own + ((p / per_row) * kLd + (p % per_row) * 8) * 2) = piece[p];
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int j = 0; j < JT; j++)
#pragma unroll
                    for (int h = 0; h < 2; h++)
#pragma unroll
                        for (int e = 0; e < 2; e++) {
                            typedef short s4 __attribute__((ext_vector_type(4)));
                            const int row = 16 * g + 8 * h + 4 * e + (i >> 2), col = min(16 * j + 4 * (i & 3), rank - 4);
                            const s4 r = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                (__attribute__((address_space(3))) s4*)(own + (row * kLd + col) * 2));
                            const u32x2 d = __builtin_bit_cast(u32x2, r);
                            w[j][h][2 * e] = d[0];
                            w[j][h][2 * e + 1] = d[1];
                        }
            }
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int t = 0; t < RT; t++)
#pragma unroll
                    for (int j = 0; j < JT; j++)
                        acc[t][j] = mfma16x16x32_of<FMT>(__builtin_bit_cast(half8, x[t][h]), __builtin_bit_cast(half8, w[j][h]), acc[t][j]);
        }
        // the four wavefronts' sums meet in LDS, added in their order
        __syncthreads();
        float4v* meet = reinterpret_cast<float4v*>(shared);
#pragma unroll
        for (int t = 0; t < RT; t++)
#pragma unroll
            for (int j = 0; j < JT; j++) meet[(wave * RT * JT + t * JT + j) * 64 + lane] = acc[t][j];
        __syncthreads();
        const float s = args.scaling ? args.scaling[a] : 1.0f;
        for (int tile = wave; tile < RT * JT; tile += 4) {
            float4v v = meet[tile * 64 + lane];
#pragma unroll
            for (int k = 1; k < 4; k++) v += meet[(k * RT * JT + tile) * 64 + lane];
            const int t = tile / JT, j = 16 * (tile % JT) + i;
#pragma unroll
            for (int r = 0; r < 4; r++) {
                const int row = 16 * t + 4 * g + r;
                if (((rows >> row) & 1) && j < rank) P[(size_t)(m0 + row) * rank + j] = v[r] * s;
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ expand
struct ExpandLayer {
    const float* P;         // [slices, M, rank]
    const uint16_t* W;      // [adapters, D, rank], turned: [adapters, rank, D]
    const uint16_t* Y;      // [M, D]
    uint16_t* out;          // [M, D] (may be Y)
    float* hidden;          // [M, rank]: the sum of the slices is kept here (NULL: it is not)
    int D, rank, slices;
    int first;
};

struct ExpandArgs {
    ExpandLayer layer[FP6_GROUP_MAX];
    int layers;
    int64_t M;
    const int32_t* index;
    const float* scaling;
    int adapters, slots, row_tiles;      // row tiles of 16 rows per workgroup
};

// out[m][n] = Y[m][n] + s * sum_j P[m][j] W[n][j].  A wavefront: 64 columns n, 16 rows at a time; the lane of row l % 16 holds 16
// consecutive columns (the rows of the W operand are dealt out so that it does).  P is split into two 16-bit terms; with fp16 each
// row has a power of two that brings it into range.  PACKED (rank <= 16): both terms share one MFMA of contraction 32.
template <int FMT, int JS, bool PACKED, bool TURNED>
__global__ __launch_bounds__(256) void lora_expand_kernel(ExpandArgs args)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    int which = 0;
    while (which + 1 < args.layers && (int)blockIdx.x >= args.layer[which + 1].first) which++;
    const ExpandLayer L = args.layer[which];
    const int blocks = (L.D / 64 + 3) / 4, at = (int)blockIdx.x - L.first;
    const int n0 = ((at % blocks) * 4 + wave) * 64, rank = L.rank, D = L.D;
    if (n0 >= D) return;
    const int64_t tile0 = (int64_t)(at / blocks) * args.row_tiles;

    int held = kNoAdapter;               // the adapter whose operands are in w
    half8 w[4][JS];
    for (int t = 0; t < args.row_tiles; t++) {
        const int64_t m0 = (tile0 + t) * 16, row = m0 + i;
        if (m0 >= args.M) break;
        const int mine = adapter_of(args.index, row, args.M, args.adapters);
        uint64_t pending = __ballot(mine != kNoAdapter) & 0xFFFF;
        const size_t where = (size_t)row * D + n0 + 16 * g;
        if (mine == kNoAdapter && blockIdx.y == 0 && row < args.M) {
            if (L.out != L.Y) {
                const u32x4* from = reinterpret_cast<const u32x4*>(L.Y + where);
                u32x4* to = reinterpret_cast<u32x4*>(L.out + where);
                const u32x4 a = from[0], b = from[1];
                to[0] = a;
                to[1] = b;
            }
            if (L.hidden && n0 == 0)
                for (int j = 4 * g; j < rank; j += 16) *reinterpret_cast<float4v*>(L.hidden + (size_t)row * rank + j) = float4v{0, 0, 0, 0};
        }
        for (int seen = 0; pending; seen++) {
            const int a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(pending));
            pending &= ~(__ballot(mine == a) & 0xFFFF);
            if (seen % args.slots != (int)blockIdx.y) continue;
            // P of this lane's row: eight values per step
            float v[JS][8];
            float top = 0.0f;
#pragma unroll
            for (int s = 0; s < JS; s++) {
                const int k0 = 32 * s + 8 * g, j0 = PACKED && k0 >= rank ? k0 - rank : k0;
#pragma unroll
                for (int e = 0; e < 8; e++) v[s][e] = 0.0f;
                if (mine == a && j0 < rank) {
                    for (int c = 0; c < L.slices; c++) {
                        const float4v* p = reinterpret_cast<const float4v*>(L.P + ((size_t)c * args.M + row) * rank + j0);
                        const float4v lo = p[0], hi = p[1];
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            v[s][e] += lo[e];
                            v[s][4 + e] += hi[e];
                        }
                    }
                    if (L.hidden && n0 == 0 && j0 == k0) {
                        float4v* h = reinterpret_cast<float4v*>(L.hidden + (size_t)row * rank + j0);
                        h[0] = float4v{v[s][0], v[s][1], v[s][2], v[s][3]};
                        h[1] = float4v{v[s][4], v[s][5], v[s][6], v[s][7]};
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; e++) top = fmaxf(top, fabsf(v[s][e]));
            }
            int exponent = 0;
            if (FMT != kE3M2B) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                exponent = exponent_for(top);
                const float down = power_of_two(-exponent);
#pragma unroll
                for (int s = 0; s < JS; s++)
#pragma unroll
                    for (int e = 0; e < 8; e++) v[s][e] *= down;
            }
            if (a != held) {
                held = a;
                const uint16_t* W = L.W + (size_t)a * rank * D;
#pragma unroll
                for (int s = 0; s < JS; s++) {
                    const int k0 = 32 * s + 8 * g, j0 = PACKED && k0 >= rank ? k0 - rank : k0;
#pragma unroll
                    for (int c = 0; c < 4; c++) {
                        const int n = n0 + 16 * (i >> 2) + 4 * c + (i & 3);
                        u32x4 d = u32x4{0, 0, 0, 0};
                        if (j0 < rank) {
                            if (!TURNED) {
                                d = *reinterpret_cast<const u32x4*>(W + (size_t)n * rank + j0);
                            } else {
#pragma unroll
                                for (int e = 0; e < 4; e++)
                                    d[e] = (uint32_t)W[(size_t)(j0 + 2 * e) * D + n] | (uint32_t)W[(size_t)(j0 + 2 * e + 1) * D + n] << 16;
                            }
                        }
                        w[c][s] = __builtin_bit_cast(half8, d);
                    }
                }
            }
            float4v acc[4] = {float4v{0, 0, 0, 0}, float4v{0, 0, 0, 0}, float4v{0, 0, 0, 0}, float4v{0, 0, 0, 0}};
#pragma unroll
            for (int s = 0; s < JS; s++) {
                u32x4 term[2];
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    uint16_t x[2], y[2];
                    split_terms<FMT>(v[s][2 * e], x);
                    split_terms<FMT>(v[s][2 * e + 1], y);
                    term[0][e] = x[0] | (uint32_t)y[0] << 16;
                    term[1][e] = x[1] | (uint32_t)y[1] << 16;
                }
                if (PACKED) {
                    const half8 both = __builtin_bit_cast(half8, 8 * g >= rank ? term[1] : term[0]);
#pragma unroll
                    for (int c = 0; c < 4; c++) acc[c] = mfma16x16x32_of<FMT>(w[c][s], both, acc[c]);
                } else {
#pragma unroll
                    for (int p = 0; p < 2; p++)
#pragma unroll
                        for (int c = 0; c < 4; c++) acc[c] = mfma16x16x32_of<FMT>(w[c][s], __builtin_bit_cast(half8, term[p]), acc[c]);
                }
            }
            if (mine == a) {
                const float up = FMT != kE3M2B ? power_of_two(exponent) : 1.0f, s = args.scaling ? args.scaling[a] : 1.0f;
                u32x4 y[2];
                y[0] = *reinterpret_cast<const u32x4*>(L.Y + where);
                y[1] = *reinterpret_cast<const u32x4*>(L.Y + where + 8);
#pragma unroll
                for (int c = 0; c < 4; c++)
#pragma unroll
                    for (int p = 0; p < 2; p++) {
                        const uint32_t d = y[c >> 1][2 * (c & 1) + p];
                        const float lo = to_float<FMT>((uint16_t)d) + acc[c][2 * p] * up * s;
                        const float hi = to_float<FMT>((uint16_t)(d >> 16)) + acc[c][2 * p + 1] * up * s;
                        y[c >> 1][2 * (c & 1) + p] = to_bits<FMT>(lo) | (uint32_t)to_bits<FMT>(hi) << 16;
                    }
                *reinterpret_cast<u32x4*>(L.out + where) = y[0];
                *reinterpret_cast<u32x4*>(L.out + where + 8) = y[1];
            }
        }
    }
}

// ------------------------------------------------------------------ outer
struct OuterArgs {
    const float* P;          // [slices, M, rank]
    const uint16_t* Q;       // [M, C]
    float* G;                // [splits][adapters][rank][C], BY_COLUMN: [splits][adapters][C][rank]
    int64_t M;
    int C, rank, slices, adapters, splits, accumulate;
    const int32_t* index;
    const float* scaling;
};

constexpr int kChunk = 64;      // rows between two barriers

// G[a][j][c] = sum over the adapter's rows m of P[m][j] Q[m][c].  A workgroup: one adapter, 64 * CT columns, one range of rows, a
// chunk of 64 rows at a time: the rows of Q go to LDS as they are and are read back turned, P is split into 16-bit terms and stored
// turned.  fp16: two terms, and a power of two per chunk and column of P, its products are added up per chunk; bf16: three terms.
// Rows of other adapters count as zeros on both sides (an infinity in one of them does not reach this sum).
template <int FMT, int JT, int CT, bool BY_COLUMN>
__global__ __launch_bounds__(256) void lora_outer_kernel(OuterArgs args)
{
    constexpr int TERMS = FMT == kE3M2B ? 3 : 2;
    constexpr int kCols = 64 * CT, kLdQ = kCols + 16, kLdP = kChunk + 8;       // elements between two rows in LDS
    constexpr int kQv = kChunk * kCols / 8 / 256;                              // 16-byte pieces of Q a thread
    constexpr int kPv = JT;                                                    // float4 of P a thread
    __shared__ __align__(16) uint16_t q_lds[kChunk * kLdQ];
    __shared__ __align__(16) uint16_t p_lds[TERMS][16 * JT][kLdP];
    __shared__ uint32_t top[16 * JT];
    __shared__ __align__(16) float up[16 * JT];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const int a = blockIdx.y, rank = args.rank, C = args.C, per_row = rank / 4;
    const int blocks = (C + kCols - 1) / kCols, split = (int)blockIdx.x / blocks, c0 = ((int)blockIdx.x % blocks) * kCols;
    const int chunks = (int)((args.M + kChunk - 1) / kChunk);
    const int begin = slice_begin(chunks, args.splits, split), end = slice_begin(chunks, args.splits, split + 1);
    const float s = args.scaling ? args.scaling[a] : 1.0f;

    float4v sum[JT][CT];
#pragma unroll
    for (int j = 0; j < JT; j++)
#pragma unroll
        for (int c = 0; c < CT; c++) sum[j][c] = float4v{0, 0, 0, 0};
    for (int chunk = begin; chunk < end; chunk++) {
        const int64_t m0 = (int64_t)chunk * kChunk;
        const uint64_t rows = __ballot(adapter_of(args.index, m0 + lane, args.M, args.adapters) == a);
        if (!rows) continue;                                  // (the same in every wavefront)
        u32x4 q[kQv];
#pragma unroll
        for (int v = 0; v < kQv; v++) {
            const int p = threadIdx.x + 256 * v, row = p / (kCols / 8), col = c0 + (p % (kCols / 8)) * 8;
            q[v] = u32x4{0, 0, 0, 0};
            if (((rows >> row) & 1) && col < C) q[v] = *reinterpret_cast<const u32x4*>(args.Q + (size_t)(m0 + row) * C + col);
        }
        float4v p4[kPv];
#pragma unroll
        for (int v = 0; v < kPv; v++) {
            const int f = threadIdx.x + 256 * v, row = f / per_row, j = (f % per_row) * 4;
            p4[v] = float4v{0, 0, 0, 0};
            if (row < kChunk && ((rows >> row) & 1)) {
                for (int c = 0; c < args.slices; c++)
                    p4[v] += *reinterpret_cast<const float4v*>(args.P + ((size_t)c * args.M + m0 + row) * rank + j);
            }
        }
        __syncthreads();                                      // (the last chunk's operands have been read)
        if (FMT != kE3M2B) {
            if (threadIdx.x < 16 * JT) top[threadIdx.x] = 0;
            __syncthreads();
#pragma unroll
            for (int v = 0; v < kPv; v++) {
                const int f = threadIdx.x + 256 * v, row = f / per_row, j = (f % per_row) * 4;
                if (row < kChunk)
#pragma unroll
                    for (int e = 0; e < 4; e++) atomicMax(&top[j + e], __builtin_bit_cast(uint32_t, fabsf(p4[v][e])));
            }
            __syncthreads();
            if (threadIdx.x < 16 * JT) up[threadIdx.x] = power_of_two(exponent_for(__builtin_bit_cast(float, top[threadIdx.x])));
        }
#pragma unroll
        for (int v = 0; v < kQv; v++) {
            const int p = threadIdx.x + 256 * v, row = p / (kCols / 8), col = (p % (kCols / 8)) * 8;
            *reinterpret_cast<u32x4*>(q_lds + row * kLdQ + col) = q[v];
        }
#pragma unroll
        for (int v = 0; v < kPv; v++) {
            const int f = threadIdx.x + 256 * v, row = f / per_row, j = (f % per_row) * 4;
            if (row < kChunk)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    uint16_t t[TERMS];
                    float x = p4[v][e];
                    if (FMT != kE3M2B) x *= power_of_two(-exponent_for(__builtin_bit_cast(float, top[j + e])));
                    split_terms<FMT>(x, t);
#pragma unroll
                    for (int k = 0; k < TERMS; k++) p_lds[k][j + e][row] = t[k];
                }
        }
        __syncthreads();
        float4v part[JT][CT];
        float4v (&acc)[JT][CT] = FMT == kE3M2B ? sum : part;
        if (FMT != kE3M2B) {
#pragma unroll
            for (int j = 0; j < JT; j++)
#pragma unroll
                for (int c = 0; c < CT; c++) part[j][c] = float4v{0, 0, 0, 0};
        }
#pragma unroll
        for (int step = 0; step < kChunk / 32; step++) {
            half8 p[JT][TERMS];
#pragma unroll
            for (int j = 0; j < JT; j++)
#pragma unroll
                for (int k = 0; k < TERMS; k++) p[j][k] = *reinterpret_cast<const half8*>(&p_lds[k][16 * j + i][32 * step + 8 * g]);
#pragma unroll
            for (int c = 0; c < CT; c++) {
                typedef short s4 __attribute__((ext_vector_type(4)));
                u32x4 d;
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const int row = 32 * step + 8 * g + 4 * e + (i >> 2), col = (wave * CT + c) * 16 + 4 * (i & 3);
                    const s4 r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(q_lds + row * kLdQ + col));
                    const u32x2 b = __builtin_bit_cast(u32x2, r);
                    d[2 * e] = b[0];
                    d[2 * e + 1] = b[1];
                }
#pragma unroll
                for (int j = 0; j < JT; j++)
#pragma unroll
                    for (int k = 0; k < TERMS; k++) acc[j][c] = mfma16x16x32_of<FMT>(p[j][k], __builtin_bit_cast(half8, d), acc[j][c]);
            }
        }
        if (FMT != kE3M2B) {
#pragma unroll
            for (int j = 0; j < JT; j++) {
                const float4v f = *reinterpret_cast<const float4v*>(up + 16 * j + 4 * g);
#pragma unroll
                for (int c = 0; c < CT; c++) sum[j][c] += part[j][c] * f;
            }
        }
    }
    float* G = args.G + ((size_t)split * args.adapters + a) * rank * C;
    const bool add = args.accumulate && args.splits == 1;
#pragma unroll
    for (int j = 0; j < JT; j++)
#pragma unroll
        for (int c = 0; c < CT; c++) {
            const int col = c0 + (wave * CT + c) * 16 + i, j0 = 16 * j + 4 * g;
            if (col >= C || j0 >= rank) continue;
            float4v v = sum[j][c] * s;
            if (BY_COLUMN) {
                float4v* to = reinterpret_cast<float4v*>(G + (size_t)col * rank + j0);
                if (add) v += *to;
                *to = v;
            } else {
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    float* to = G + (size_t)(j0 + r) * C + col;
                    *to = add ? *to + v[r] : v[r];
                }
            }
        }
}

// out[k] (+)= the sum over the splits, in their order; two tensors in one launch
struct JoinArgs {
    const float4v* part[2];
    float4v* out[2];
    int64_t count[2];        // float4 of each
    int splits[2];
    int accumulate;
};

__global__ __launch_bounds__(256) void lora_join_kernel(JoinArgs args)
{
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < args.count[0] + args.count[1]; k += (int64_t)gridDim.x * 256) {
        const int w = k >= args.count[0];
        const int64_t e = w ? k - args.count[0] : k;
        float4v v = args.accumulate ? args.out[w][e] : float4v{0, 0, 0, 0};
        for (int c = 0; c < args.splits[w]; c++) v += args.part[w][(size_t)c * args.count[w] + e];
        args.out[w][e] = v;
    }
}

// ------------------------------------------------------------------ plans and launches
static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Rows a shrink workgroup takes, slots its adapters are dealt to, and slices of the contraction: two workgroups for each compute unit
// where the contraction is long enough to be cut (a slice gives each of the four wavefronts at least one unit of 64).
struct ShrinkPlan {
    int row_tiles, slots, slices;
    int64_t groups;
};

static ShrinkPlan plan_shrink(int64_t M, int C, int adapters, bool indexed)
{
    ShrinkPlan p;
    p.row_tiles = M > 64 ? 2 : 1;
    const int64_t rows = 16 * p.row_tiles;
    p.groups = ceil_div(M, rows);
    p.slots = indexed && M <= 64 ? (int)(adapters < rows ? adapters : rows) : 1;
    const int64_t have = p.groups * p.slots, most = C / 64 >= 8 ? C / 256 : 1;
    int64_t slices = ceil_div(512, have);
    if (slices > most) slices = most;
    if (slices > 32) slices = 32;
    p.slices = (int)(slices < 1 ? 1 : slices);
    return p;
}

// Ranges of rows that separate workgroups of the outer products take: two workgroups for each compute unit, of at least four chunks.
static int plan_splits(int64_t M, int C, int cols, int adapters)
{
    const int64_t chunks = ceil_div(M, kChunk), have = ceil_div(C, cols) * adapters;
    int64_t splits = ceil_div(512, have);
    if (splits > chunks / 4) splits = chunks / 4;
    return (int)(splits < 1 ? 1 : (splits > 64 ? 64 : splits));
}

static int outer_columns(int rank) { return rank > 64 ? 128 : 256; }

template <int FMT, int RT, bool TURNED>
static void launch_shrink_rank(const ShrinkArgs& a, int rank, dim3 grid, hipStream_t stream)
{
    if (rank <= 16) hipLaunchKernelGGL((lora_shrink_kernel<FMT, 1, RT, TURNED>), grid, dim3(256), 0, stream, a);
    else if (rank <= 32) hipLaunchKernelGGL((lora_shrink_kernel<FMT, 2, RT, TURNED>), grid, dim3(256), 0, stream, a);
    else if (rank <= 64) hipLaunchKernelGGL((lora_shrink_kernel<FMT, 4, RT, TURNED>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((lora_shrink_kernel<FMT, 8, RT, TURNED>), grid, dim3(256), 0, stream, a);
}

template <int FMT, bool TURNED>
static hipError_t launch_shrink(ShrinkArgs& a, int row_tiles, int64_t workgroups, hipStream_t stream)
{
    int rank = 0;
    for (int l = 0; l < a.layers; l++) rank = a.layer[l].rank > rank ? a.layer[l].rank : rank;
    const dim3 grid((unsigned)workgroups, (unsigned)a.slots);
    if (row_tiles == 1) launch_shrink_rank<FMT, 1, TURNED>(a, rank, grid, stream);
    else launch_shrink_rank<FMT, 2, TURNED>(a, rank, grid, stream);
    return hipGetLastError();
}

template <int FMT, bool TURNED>
static hipError_t launch_expand(ExpandArgs& a, int64_t workgroups, hipStream_t stream)
{
    int rank = 0;
    bool packed = true;
    for (int l = 0; l < a.layers; l++) {
        rank = a.layer[l].rank > rank ? a.layer[l].rank : rank;
        packed = packed && a.layer[l].rank <= 16;
    }
    const dim3 grid((unsigned)workgroups, (unsigned)a.slots);
    if (packed) hipLaunchKernelGGL((lora_expand_kernel<FMT, 1, true, TURNED>), grid, dim3(256), 0, stream, a);
    else if (rank <= 32) hipLaunchKernelGGL((lora_expand_kernel<FMT, 1, false, TURNED>), grid, dim3(256), 0, stream, a);
    else if (rank <= 64) hipLaunchKernelGGL((lora_expand_kernel<FMT, 2, false, TURNED>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((lora_expand_kernel<FMT, 4, false, TURNED>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <int FMT, bool BY_COLUMN>
static hipError_t launch_outer(const OuterArgs& a, hipStream_t stream)
{
    const dim3 grid((unsigned)(ceil_div(a.C, outer_columns(a.rank)) * a.splits), (unsigned)a.adapters);
    if (a.rank <= 16) hipLaunchKernelGGL((lora_outer_kernel<FMT, 1, 4, BY_COLUMN>), grid, dim3(256), 0, stream, a);
    else if (a.rank <= 32) hipLaunchKernelGGL((lora_outer_kernel<FMT, 2, 4, BY_COLUMN>), grid, dim3(256), 0, stream, a);
    else if (a.rank <= 64) hipLaunchKernelGGL((lora_outer_kernel<FMT, 4, 4, BY_COLUMN>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((lora_outer_kernel<FMT, 8, 2, BY_COLUMN>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

// Row tiles of 16 rows that an expand workgroup takes one after another (its operands of W stay in registers): four from the point
// on where enough workgroups remain.
static int expand_row_tiles(int64_t M, int64_t columns)
{
    const int64_t tiles = ceil_div(M, 16), have = tiles * ceil_div(columns, 256);
    return have >= 4096 ? 4 : (have >= 2048 ? 2 : 1);
}

static size_t round_up(size_t bytes) { return (bytes + 255) / 256 * 256; }

size_t lora_workspace(int64_t M, const fp6_lora_problem* pr, int count, int adapters)
{
    size_t need = kZeroBytes;
    for (int l = 0; l < count; l++)
        need += round_up((size_t)plan_shrink(M, (int)pr[l].K, adapters, adapters > 1).slices * M * pr[l].rank * 4);
    return need;
}

template <int FMT>
static hipError_t launch_lora_t(int64_t M, const fp6_lora_problem* pr, int count, int adapters, const int32_t* index, const float* scaling,
                                unsigned char* workspace, hipStream_t stream)
{
    ShrinkArgs s{};
    ExpandArgs e{};
    s.layers = e.layers = count;
    s.M = e.M = M;
    s.index = e.index = index;
    e.scaling = scaling;
    s.adapters = e.adapters = adapters;
    unsigned char* at = workspace + kZeroBytes;
    int64_t shrinks = 0, expands = 0, columns = 0;
    int row_tiles = 1;
    for (int l = 0; l < count; l++) columns += pr[l].N;
    e.row_tiles = expand_row_tiles(M, columns);
    for (int l = 0; l < count; l++) {
        const ShrinkPlan p = plan_shrink(M, (int)pr[l].K, adapters, adapters > 1);
        s.slots = e.slots = p.slots;
        row_tiles = p.row_tiles;
        s.layer[l] = ShrinkLayer{pr[l].X, pr[l].A, (float*)at, (int)pr[l].K, (int)pr[l].rank, p.slices, (int)shrinks};
        e.layer[l] = ExpandLayer{(const float*)at, pr[l].B, pr[l].Y, pr[l].out, pr[l].hidden, (int)pr[l].N, (int)pr[l].rank, p.slices, (int)expands};
        at += round_up((size_t)p.slices * M * pr[l].rank * 4);
        shrinks += p.groups * p.slices;
        expands += ceil_div(pr[l].N, 256) * ceil_div(ceil_div(M, 16), e.row_tiles);
    }
    const hipError_t err = launch_shrink<FMT, false>(s, row_tiles, shrinks, stream);
    if (err != hipSuccess) return err;
    return launch_expand<FMT, false>(e, expands, stream);
}

hipError_t launch_lora(bool bf16, int64_t M, const fp6_lora_problem* pr, int count, int adapters, const int32_t* index, const float* scaling,
                       void* workspace, hipStream_t stream)
{
    return bf16 ? launch_lora_t<kE3M2B>(M, pr, count, adapters, index, scaling, (unsigned char*)workspace, stream)
                : launch_lora_t<kE3M2>(M, pr, count, adapters, index, scaling, (unsigned char*)workspace, stream);
}

// Workspace of the backward pass behind the zero region: the slices of dH, then the splits of dA and of dB (none where there is one).
struct BackwardPlan {
    ShrinkPlan shrink;
    int splits_a, splits_b;
    size_t dh, da, db;       // bytes
};

static BackwardPlan plan_backward(int64_t M, int64_t N, int64_t K, int rank, int adapters)
{
    BackwardPlan p;
    p.shrink = plan_shrink(M, (int)N, adapters, adapters > 1);
    p.splits_a = plan_splits(M, (int)K, outer_columns(rank), adapters);
    p.splits_b = plan_splits(M, (int)N, outer_columns(rank), adapters);
    p.dh = round_up((size_t)p.shrink.slices * M * rank * 4);
    p.da = p.splits_a > 1 ? round_up((size_t)p.splits_a * adapters * rank * K * 4) : 0;
    p.db = p.splits_b > 1 ? round_up((size_t)p.splits_b * adapters * rank * N * 4) : 0;
    return p;
}

size_t lora_backward_workspace(int64_t M, int64_t N, int64_t K, int rank, int adapters)
{
    const BackwardPlan p = plan_backward(M, N, K, rank, adapters);
    return kZeroBytes + p.dh + p.da + p.db;
}

template <int FMT>
static hipError_t launch_backward_t(const LoraBackward& b, unsigned char* workspace, hipStream_t stream)
{
    const BackwardPlan p = plan_backward(b.M, b.N, b.K, b.rank, b.adapters);
    float* dh = (float*)(workspace + kZeroBytes);
    float* da = (float*)(workspace + kZeroBytes + p.dh);
    float* db = (float*)(workspace + kZeroBytes + p.dh + p.da);
    ShrinkArgs s{};
    s.layers = 1;
    s.M = b.M;
    s.index = b.index;
    s.scaling = b.scaling;
    s.adapters = b.adapters;
    s.slots = p.shrink.slots;
    s.layer[0] = ShrinkLayer{b.dY, b.B, dh, (int)b.N, b.rank, p.shrink.slices, 0};
    hipError_t err = launch_shrink<FMT, true>(s, p.shrink.row_tiles, p.shrink.groups * p.shrink.slices, stream);
    if (err != hipSuccess) return err;
    if (b.out) {
        ExpandArgs e{};
        e.layers = 1;
        e.M = b.M;
        e.index = b.index;
        e.adapters = b.adapters;
        e.slots = p.shrink.slots;
        e.row_tiles = expand_row_tiles(b.M, b.K);
        e.layer[0] = ExpandLayer{dh, b.A, b.dX, b.out, nullptr, (int)b.K, b.rank, p.shrink.slices, 0};
        err = launch_expand<FMT, true>(e, ceil_div(b.K, 256) * ceil_div(ceil_div(b.M, 16), e.row_tiles), stream);
        if (err != hipSuccess) return err;
    }
    const OuterArgs oa{dh, b.X, p.splits_a > 1 ? da : b.dA, b.M, (int)b.K, b.rank, p.shrink.slices, b.adapters, p.splits_a, b.accumulate, b.index, nullptr};
    err = launch_outer<FMT, false>(oa, stream);
    if (err != hipSuccess) return err;
    const OuterArgs ob{b.hidden, b.dY, p.splits_b > 1 ? db : b.dB, b.M, (int)b.N, b.rank, 1, b.adapters, p.splits_b, b.accumulate, b.index, b.scaling};
    err = launch_outer<FMT, true>(ob, stream);
    if (err != hipSuccess || (p.splits_a == 1 && p.splits_b == 1)) return err;
    JoinArgs j{};
    j.accumulate = b.accumulate;
    j.part[0] = (const float4v*)da;
    j.out[0] = (float4v*)b.dA;
    j.count[0] = p.splits_a > 1 ? (int64_t)b.adapters * b.rank * b.K / 4 : 0;
    j.splits[0] = p.splits_a;
    j.part[1] = (const float4v*)db;
    j.out[1] = (float4v*)b.dB;
    j.count[1] = p.splits_b > 1 ? (int64_t)b.adapters * b.rank * b.N / 4 : 0;
    j.splits[1] = p.splits_b;
    const int64_t want = ceil_div(j.count[0] + j.count[1], 256);
    hipLaunchKernelGGL(lora_join_kernel, dim3((unsigned)(want < 4096 ? want : 4096)), dim3(256), 0, stream, j);
    return hipGetLastError();
}

hipError_t launch_lora_backward(bool bf16, const LoraBackward& b, void* workspace, hipStream_t stream)
{
    return bf16 ? launch_backward_t<kE3M2B>(b, (unsigned char*)workspace, stream) : launch_backward_t<kE3M2>(b, (unsigned char*)workspace, stream);
}

}  // namespace fp6
