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

constexpr int kNoAdapter = -1;

// The adapter of a row, or kNoAdapter: what index holds for it (of the last row past the end: the load takes no branch), and whether that is one.
__device__ __forceinline__ int owner_word(const int32_t* __restrict__ index, int64_t row, int64_t M)
{
    return index ? index[min(row, M - 1)] : 0;
}
__device__ __forceinline__ int owner_of(int word, int64_t row, int64_t M, int adapters)
{
    return row < M && (unsigned)word < (unsigned)adapters ? word : kNoAdapter;
}
__device__ __forceinline__ int adapter_of(const int32_t* __restrict__ index, int64_t row, int64_t M, int adapters)
{
    return owner_of(owner_word(index, row, M), row, M, adapters);
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

// A load whose lanes hold a 4 x 16 block of 16-bit numbers row by row, four a lane, and get back its columns.
__device__ __forceinline__ u32x2 read_turned(const uint16_t* p)
{
    typedef short s4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)p));
}

// Accesses of a wavefront to LDS of its own are carried out in order; the compiler has to keep them so.
__device__ __forceinline__ void own_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Loads above stay above: left to itself the compiler moves each one down to its first use, to hold fewer registers, and waits there.
__device__ __forceinline__ void loads_are_issued()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Sixteen rows of 128 bytes as the matrix cores take them: lane l has of row l % 16 the 16-byte pieces l / 16 (a) and 4 + l / 16 (b).  Read or written that
// way an access is half a line of every row; here a and b are exchanged with what goes to and comes from memory in whole lines, eight rows an
// access: a the rows 0 to 7 and b the rows 8 to 15, lane l the row l % 8 and the piece l / 16 + 4 * (l % 16 / 8).  Its own inverse.  All lanes call it.
// (A shrink that read its rows so and gave wrong ones now and then did not do it here: the lanes had asked for another row, by a shift whose amount lay in the
// last register of the kernel.  Every kernel's code is checked for that form.)
__device__ __forceinline__ void deal_lines(u32x4& a, u32x4& b)
{
    constexpr int kByEight = 0x128;      // each lane gets that of the lane eight away among its sixteen
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const int x = (int)a[e], y = (int)b[e];
        a[e] = (uint32_t)__builtin_amdgcn_update_dpp(x, y, kByEight, 0xF, 0xC, false);
        b[e] = (uint32_t)__builtin_amdgcn_update_dpp(y, x, kByEight, 0xF, 0x3, false);
    }
}

// Every load is waited for here: for the end of a branch that loads.  Behind it the compiler would have to wait for all loads, those in flight for
// later among them, whichever way was taken.
__device__ __forceinline__ void loads_are_here() { __builtin_amdgcn_s_waitcnt(0x0F70); }

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

// Wavefronts of a shrink workgroup: four where it takes 64 rows; with few rows as many as share a contraction that is then cut into fewer
// slices (LDS holds their sums, and the staged pieces of a turned W).
template <int JT, int RT>
constexpr int kShrinkWaves = RT > 1 || JT == 8 ? 4 : 8;
template <int JT, int RT, bool TURNED, int WAVES>
constexpr int kShrinkLds = WAVES * (TURNED && 32 * (16 * JT + 8) * 2 > RT * JT * 1024 ? 32 * (16 * JT + 8) * 2 : RT * JT * 1024);

// P[slice][m][j] = sum over the slice's c of Q[m][c] W[a][j][c].  A workgroup: 16 * RT rows, one slice of the contraction, whose
// 64-wide units its wavefronts take in turn; four lanes share a row, and a load of theirs is 64 consecutive bytes of it.  The
// distinct adapters of the rows are taken one after another, or one per grid slot: each reads its own A.
// Bound by its loads: 2048 x 22016 rank 16 26 us for 92 MB (3.5 TB/s; 24 without A; 8 of them before and after the stream), rank 64 37 us: every 64
// rows read A once more out of L2, as many bytes as X.  A plain read of X takes 14.  One row of 4096 4.1 us, a launch.
template <int FMT, int JT, int RT, bool TURNED, int WAVES>
__device__ __forceinline__ void shrink_block(const ShrinkArgs& args, int block, int slot, unsigned char* shared)
{
    constexpr int kLd = 16 * JT + 8;                       // turned: elements between two rows of the staged unit
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    int which = 0;
    while (which + 1 < args.layers && block >= args.layer[which + 1].first) which++;
    const ShrinkLayer L = args.layer[which];
    const int at = block - L.first, slice = at % L.slices;
    const int64_t m0 = (int64_t)(at / L.slices) * (16 * RT);
    const int rank = L.rank, C = L.C, units = C / 64;
    const int u_begin = slice_begin(units, L.slices, slice) + wave, u_end = slice_begin(units, L.slices, slice + 1);

    // (16 * RT <= 64 rows: lane l looks after row l)
    const int mine = lane < 16 * RT ? adapter_of(args.index, m0 + lane, args.M, args.adapters) : kNoAdapter;
    uint64_t pending = __ballot(mine != kNoAdapter);
    const uint64_t none = RT == 4 ? ~pending : ~pending & (((uint64_t)1 << (16 * (RT & 3))) - 1);
    float* P = L.P + (size_t)slice * args.M * rank;
    if (slot == 0 && none) {                               // rows without an adapter
        for (int e = threadIdx.x; e < 16 * RT * rank; e += 64 * WAVES)
            if ((none >> (e / rank)) & 1 && m0 + e / rank < args.M) P[(size_t)(m0 + e / rank) * rank + e % rank] = 0.0f;
    }
    // turned: half a unit's 32 rows of W are one piece of memory, JT times 16 bytes a lane at most; where each goes in LDS
    uint16_t* own = reinterpret_cast<uint16_t*>(shared) + wave * (32 * kLd);
    const int per_row = rank / 8;
    int put[JT];
    if (TURNED) {
#pragma unroll
        for (int k = 0; k < JT; k++) {
            const int p = lane + 64 * k;
            put[k] = (p / per_row) * kLd + (p % per_row) * 8;
        }
    }
    for (int seen = 0; pending; seen++) {
        const int a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(pending));
        const uint64_t rows = __ballot(mine == a);
        pending &= ~rows;
        if (seen % args.slots != slot) continue;
        // (lanes of other rows read one that is this adapter's: what they add up is dropped)
        const int some = __builtin_ctzll(rows);
        const uint16_t* q[RT];
#pragma unroll
        for (int t = 0; t < RT; t++) {
            const int row = (rows >> (16 * t + i)) & 1 ? 16 * t + i : some;
            q[t] = L.Q + (size_t)(m0 + row) * C + 8 * g;
        }
        const uint16_t* W = L.W + (size_t)a * rank * C;
        const uint16_t* wj[JT];
#pragma unroll
        for (int j = 0; j < JT; j++) wj[j] = W + (size_t)min(16 * j + i, rank - 1) * C + 8 * g;
        float4v acc[RT][JT];
#pragma unroll
        for (int t = 0; t < RT; t++)
#pragma unroll
            for (int j = 0; j < JT; j++) acc[t][j] = float4v{0, 0, 0, 0};
        struct Half {
            u32x4 x[RT], w[JT];          // (turned: w is the piece as it lies in memory)
        };
        // half a unit: the k-th of this wavefront's
        auto load = [&](Half& b, int k) {
            const size_t c = (size_t)(u_begin + (k >> 1) * WAVES) * 64 + 32 * (k & 1);
#pragma unroll
            for (int t = 0; t < RT; t++) b.x[t] = *reinterpret_cast<const u32x4*>(q[t] + c);
            if (!TURNED) {
#pragma unroll
                for (int j = 0; j < JT; j++) b.w[j] = *reinterpret_cast<const u32x4*>(wj[j] + c);
            } else {
                const u32x4* piece = reinterpret_cast<const u32x4*>(W + c * rank);
#pragma unroll
                for (int j = 0; j < JT; j++) b.w[j] = piece[min(lane + 64 * j, 32 * per_row - 1)];
            }
        };
        auto compute = [&](const Half& b) {
            if (TURNED) {
                own_lds_order();
#pragma unroll
                for (int k = 0; k < JT; k++)
                    if (lane + 64 * k < 32 * per_row) *reinterpret_cast<u32x4*>(own + put[k]) = b.w[k];
                own_lds_order();
            }
#pragma unroll
            for (int j = 0; j < JT; j++) {
                u32x4 w = b.w[j];
                if (TURNED) {
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        const u32x2 d = read_turned(own + (8 * g + 4 * e + (i >> 2)) * kLd + min(16 * j + 4 * (i & 3), rank - 4));
                        w[2 * e] = d[0];
                        w[2 * e + 1] = d[1];
                    }
                }
#pragma unroll
                for (int t = 0; t < RT; t++)
                    acc[t][j] = mfma16x16x32_of<FMT>(__builtin_bit_cast(half8, b.x[t]), __builtin_bit_cast(half8, w), acc[t][j]);
            }
        };
        if (u_begin < u_end) {
            // one half in flight while another is used (past the end: the last one again, so that the loads need no branch; few rows: none).  One way
            // out of the loop: with more of them the sums are copied from register to register and spilled.
            Half b[2];
            const int n = 2 * ((u_end - 1 - u_begin) / WAVES + 1);
            load(b[0], 0);
            for (int k = 0; k < n; k += 2) {
                load(b[1], k + 1);
                loads_are_issued();
                compute(b[0]);
                if (RT > 1 || k + 2 < n) load(b[0], min(k + 2, n - 1));
                loads_are_issued();
                compute(b[1]);
            }
        }
        // the wavefronts' sums meet in LDS, added in their order
        __syncthreads();
        float4v* meet = reinterpret_cast<float4v*>(shared);
#pragma unroll
        for (int t = 0; t < RT; t++)
#pragma unroll
            for (int j = 0; j < JT; j++) meet[(wave * RT * JT + t * JT + j) * 64 + lane] = acc[t][j];
        __syncthreads();
        const float s = args.scaling ? args.scaling[a] : 1.0f;
        for (int tile = wave; tile < RT * JT; tile += WAVES) {
            float4v v = meet[tile * 64 + lane];
#pragma unroll
            for (int k = 1; k < WAVES; k++) v += meet[(k * RT * JT + tile) * 64 + lane];
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

template <int FMT, int JT, int RT, bool TURNED>
__global__ __launch_bounds__((64 * kShrinkWaves<JT, RT>), (RT > 1 ? 2 : 1)) void lora_shrink_kernel(ShrinkArgs args)
{
    constexpr int WAVES = kShrinkWaves<JT, RT>;
    __shared__ __align__(16) unsigned char shared[kShrinkLds<JT, RT, TURNED, WAVES>];
    shrink_block<FMT, JT, RT, TURNED, WAVES>(args, blockIdx.x, blockIdx.y, shared);
}

// ------------------------------------------------------------------ finish
struct FinishArgs {
    const float* P;          // [slices, M, rank]
    float* sum;              // [M, rank]: the slices added up (NULL: not wanted; may be P: every row is read by the workgroup that writes it)
    uint16_t* terms;         // [M][2][rank]: the sum as two 16-bit terms of a row times 2^exponent
    float* power;            // [M]: 2^exponent
    int64_t M;
    int rank, slices, lanes; // lanes that share a row (a power of two, at least rank / 4)
    const int32_t* index;    // rows without an adapter, which P may hold nothing for, are zeros
    int adapters;
};

// The slices of the contraction added up, and split into the two terms that the expand kernel multiplies with: once a row instead of once a row
// and block of columns.  MANY slices: the four wavefronts of a workgroup take every fourth slice of the same rows, and their sums are added in
// their order (4096 rows, 86 slices of rank 16: 6.2 us, 8.5 with a thread for all slices; 512 rows, 8 slices: 4.6 and 3.3).
template <int FMT, bool MANY>
__global__ __launch_bounds__(256) void lora_finish_kernel(FinishArgs args)
{
    __shared__ float4v meet[MANY ? 3 : 1][64];
    const int lanes = args.lanes, rank = args.rank, lane = threadIdx.x & 63, wave = MANY ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const int64_t row = ((int64_t)blockIdx.x * (MANY ? 64 : 256) + (MANY ? lane : (int)threadIdx.x)) / lanes;
    const int j = 4 * (lane % lanes);
    const bool real = row < args.M && j < rank;
    const int word = owner_word(args.index, row, args.M);
    float4v v = float4v{0, 0, 0, 0};
    const float* p = args.P + (size_t)min(row, args.M - 1) * rank + min(j, rank - 4);
    const size_t step = (size_t)args.M * rank;
#pragma unroll 8
    for (int c = wave; c < args.slices; c += MANY ? 4 : 1) v += *reinterpret_cast<const float4v*>(p + c * step);
    if (MANY) {
        if (wave) meet[wave - 1][lane] = v;
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int w = 0; w < 3; w++) v += meet[w][lane];
    }
    if (!real || owner_of(word, row, args.M, args.adapters) == kNoAdapter) v = float4v{0, 0, 0, 0};
    if (real && args.sum) *reinterpret_cast<float4v*>(args.sum + (size_t)row * rank + j) = v;
    int exponent = 0;
    if (FMT != kE3M2B) {
        float top = fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
        for (int off = 1; off < lanes; off <<= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        exponent = exponent_for(top);
        v *= power_of_two(-exponent);
    }
    if (!real) return;
    uint16_t t[4][2];
#pragma unroll
    for (int e = 0; e < 4; e++) split_terms<FMT>(v[e], t[e]);
    uint16_t* to = args.terms + (size_t)row * 2 * rank + j;
#pragma unroll
    for (int k = 0; k < 2; k++)
        *reinterpret_cast<u32x2*>(to + k * rank) = u32x2{t[0][k] | (uint32_t)t[1][k] << 16, t[2][k] | (uint32_t)t[3][k] << 16};
    if (j == 0) args.power[row] = power_of_two(exponent);
}

// ------------------------------------------------------------------ expand
constexpr int kFewSlices = 8;            // slices at most that the expand kernel adds up itself

struct ExpandLayer {
    const float* P;         // SLICED: [slices, M, rank]; else the power of two of each row
    const uint16_t* terms;  // else: [M][2][rank]
    const uint16_t* W;      // [adapters, D, rank], turned: [adapters, rank, D]
    const uint16_t* Y;      // [M, D]
    uint16_t* out;          // [M, D] (may be Y)
    float* hidden;          // SLICED: [M, rank]: the sum of the slices is kept here (NULL: it is not)
    int D, rank, slices;
    int first;
};

struct ExpandArgs {
    ExpandLayer layer[FP6_GROUP_MAX];
    int layers;
    int64_t M;
    const int32_t* index;
    const float* scaling;
    int adapters, slots, row_tiles;      // row tiles of 16 rows per wavefront
};

constexpr int kExpandLd = 64 + 8;        // turned: elements between two rows of a staged piece of W
template <bool TURNED>
constexpr int kExpandLds = TURNED ? 4 * 32 * kExpandLd * 2 : 16;

// out[m][n] = Y[m][n] + s * sum_j P[m][j] W[n][j].  A wavefront: 64 * CB columns n, 16 rows at a time (the four of a workgroup side by side with
// few rows, else one below the other, so that one of them brings W into the cache for all); the lane of row l % 16 holds two
// pieces of eight consecutive columns of each 64 (the rows of the W operand are dealt out so that it does).  P is two 16-bit terms
// times a power of two per row.  PACKED (rank <= 16): both terms share one MFMA of contraction 32.  W stays in registers from row
// tile to row tile as long as the adapter is the same.  SLICED (few rows): the terms are made here from the slices.
// Bound by Y: 2048 x 8192 rank 16 16.3 us, rank 64 21.6 (as much again of the terms and of W out of L2) for 67 MB; a pass over Y alone takes 10.4, in half
// lines of 16 rows 12.6.  (With half lines, the loads of a tile past the end repeated, and prefetched loads waited for wherever W or the scaling
// might have been loaded: 18.7 and 24.)
template <int FMT, int JS, bool PACKED, bool TURNED, bool SLICED, int CB>
__device__ __forceinline__ void expand_block(const ExpandArgs& args, int block, int slot, unsigned char* shared)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    int which = 0;
    while (which + 1 < args.layers && block >= args.layer[which + 1].first) which++;
    const ExpandLayer L = args.layer[which];
    constexpr int kAcross = (SLICED ? 4 : 1) * 64 * CB;          // columns of a workgroup
    const int rank = L.rank, D = L.D, blocks = (D + kAcross - 1) / kAcross, at = block - L.first;
    const int n0 = (at % blocks) * kAcross + (SLICED ? wave * (64 * CB) : 0);
    const int64_t tile0 = ((int64_t)(at / blocks) * (SLICED ? 1 : 4) + (SLICED ? 0 : wave)) * args.row_tiles;
    const int64_t tiles = min((int64_t)args.row_tiles, (args.M + 15) / 16 - tile0);
    if (n0 >= D || tiles <= 0) return;
    constexpr int TERMS = PACKED ? 1 : 2;

    struct Rows {                        // what a row tile needs: Y, the owner, and P where it is ready
        u32x4 y[CB][2], p[JS][TERMS];
        float power;
        int word, mine;
    };
    auto load_y = [&](Rows& b, int64_t row) {
        const uint16_t* y = L.Y + (size_t)row * D + n0 + 8 * g;
#pragma unroll
        for (int c = 0; c < CB; c++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int off = 64 * c + 32 * h;
                b.y[c][h] = *reinterpret_cast<const u32x4*>(y + (n0 + off < D ? off : 0));
            }
    };
    auto store_y = [&](const Rows& b, int64_t row) {
        uint16_t* to = L.out + (size_t)row * D + n0 + 8 * g;
#pragma unroll
        for (int c = 0; c < CB; c++)
            if (n0 + 64 * c < D) {
                *reinterpret_cast<u32x4*>(to + 64 * c) = b.y[c][0];
                *reinterpret_cast<u32x4*>(to + 64 * c + 32) = b.y[c][1];
            }
    };
    // many rows: Y in whole lines
    const int line_row = i & 7, line_col = n0 + 8 * (g + 4 * (i >> 3));
    auto load_lines = [&](Rows& b, int64_t t) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const uint16_t* y = L.Y + (size_t)(t < tiles ? min((tile0 + t) * 16 + 8 * h + line_row, args.M - 1) : 0) * D + line_col;
#pragma unroll
            for (int c = 0; c < CB; c++) b.y[c][h] = *reinterpret_cast<const u32x4*>(y + (n0 + 64 * c < D ? 64 * c : 0));
        }
    };
    auto store_lines = [&](Rows& b, int64_t t, uint32_t rows) {
#pragma unroll
        for (int c = 0; c < CB; c++) deal_lines(b.y[c][0], b.y[c][1]);
#pragma unroll
        for (int h = 0; h < 2; h++)
            if ((rows >> (8 * h + line_row)) & 1) {
                uint16_t* to = L.out + (size_t)((tile0 + t) * 16 + 8 * h + line_row) * D + line_col;
#pragma unroll
                for (int c = 0; c < CB; c++)
                    if (n0 + 64 * c < D) *reinterpret_cast<u32x4*>(to + 64 * c) = b.y[c][h];
            }
    };
    auto load = [&](Rows& b, int64_t t) {
        const int64_t row = SLICED || t < tiles ? (tile0 + t) * 16 + i : 0;
        b.word = owner_word(args.index, row, args.M);
        const int64_t near = min(row, args.M - 1);
        if (!SLICED) {
            load_lines(b, t);
            const uint16_t* p = L.terms + (size_t)near * 2 * rank;
            b.power = FMT != kE3M2B ? L.P[near] : 1.0f;
#pragma unroll
            for (int s = 0; s < JS; s++)
#pragma unroll
                for (int k = 0; k < TERMS; k++) {
                    // (past the rank: `work` puts zeros in its place)
                    b.p[s][k] = *reinterpret_cast<const u32x4*>(p + k * rank + min(32 * s + 8 * g, (PACKED ? 2 * rank : rank) - 8));
                }
        }
    };

    int held = kNoAdapter;               // the adapter whose operands are in w
    float scale = 1.0f;                  // and its scaling
    u32x4 w[CB][4][JS];
    auto hold = [&](int a) {
        held = a;
        if (!SLICED && args.scaling) scale = args.scaling[a];
        const uint16_t* W = L.W + (size_t)a * rank * D;
#pragma unroll
        for (int s = 0; s < JS; s++) {
            const int k0 = 32 * s + 8 * g, j0 = PACKED && k0 >= rank ? k0 - rank : k0;
#pragma unroll
            for (int c = 0; c < CB; c++) {
                const int nc = n0 + 64 * c < D ? n0 + 64 * c : n0;          // (past the end: columns that are not stored)
                if (!TURNED) {
#pragma unroll
                    for (int t = 0; t < 4; t++) {
                        const int n = nc + 32 * (t >> 1) + 8 * (i >> 2) + 4 * (t & 1) + (i & 3);
                        const u32x4 d = *reinterpret_cast<const u32x4*>(W + (size_t)n * rank + min(j0, rank - 8));
                        w[c][t][s] = j0 < rank ? d : u32x4{0, 0, 0, 0};
                    }
                } else {
                    // 32 rows j of 64 columns through the wavefront's own LDS
                    uint16_t* own = reinterpret_cast<uint16_t*>(shared) + wave * (32 * kExpandLd);
                    u32x4 d[4];
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        const int j = 32 * s + (lane >> 3) + 8 * k;
                        d[k] = *reinterpret_cast<const u32x4*>(W + (size_t)min(j, rank - 1) * D + nc + 8 * (lane & 7));
                    }
                    own_lds_order();
#pragma unroll
                    for (int k = 0; k < 4; k++) *reinterpret_cast<u32x4*>(own + ((lane >> 3) + 8 * k) * kExpandLd + 8 * (lane & 7)) = d[k];
                    own_lds_order();
                    const int row = PACKED ? min(j0, rank - 8) : 8 * g;
#pragma unroll
                    for (int t = 0; t < 4; t++) {
                        u32x4 x;
#pragma unroll
                        for (int e = 0; e < 2; e++) {
                            const u32x2 r = read_turned(own + (row + 4 * e + (i >> 2)) * kExpandLd + 32 * (t >> 1) + 8 * (i & 3) + 4 * (t & 1));
                            x[2 * e] = r[0];
                            x[2 * e + 1] = r[1];
                        }
                        w[c][t][s] = j0 < rank ? x : u32x4{0, 0, 0, 0};
                    }
                }
            }
        }
        if (!SLICED) loads_are_here();
    };

    auto work = [&](Rows& b, int64_t t) {
        // (a tile past this wavefront's: its rows are another's)
        const int64_t row = t < tiles ? (tile0 + t) * 16 + i : args.M;
        b.mine = owner_of(b.word, row, args.M, args.adapters);
        uint64_t pending = __ballot(b.mine != kNoAdapter) & 0xFFFF;
        // (rows to be written: those of an adapter, and where Y lies elsewhere those without one)
        const uint32_t write = SLICED ? 0 : (uint32_t)__ballot(row < args.M && (b.mine != kNoAdapter || L.out != L.Y)) & 0xFFFF;
        if (!SLICED) {
#pragma unroll
            for (int c = 0; c < CB; c++) deal_lines(b.y[c][0], b.y[c][1]);
        }
        if (SLICED && b.mine == kNoAdapter && slot == 0 && row < args.M && L.out != L.Y) {
            // (few rows: Y is read for the adapter at hand, these are copied by themselves)
            const u32x4* from = reinterpret_cast<const u32x4*>(L.Y + (size_t)row * D + n0 + 8 * g);
            u32x4* to = reinterpret_cast<u32x4*>(L.out + (size_t)row * D + n0 + 8 * g);
            const u32x4 y0 = from[0], y1 = from[4];
            to[0] = y0;
            to[4] = y1;
        }
        if (SLICED && L.hidden && n0 == 0 && slot == 0 && b.mine == kNoAdapter && row < args.M)
            for (int j = 4 * g; j < rank; j += 16) *reinterpret_cast<float4v*>(L.hidden + (size_t)row * rank + j) = float4v{0, 0, 0, 0};
        for (int seen = 0; pending; seen++) {
            const int some = __builtin_ctzll(pending), a = __builtin_amdgcn_readlane(b.mine, some);
            pending &= ~(__ballot(b.mine == a) & 0xFFFF);
            if (seen % args.slots != slot) continue;
            if (SLICED) {
                // (lanes of other rows read one that is this adapter's: nothing of theirs is stored)
                const int64_t from = b.mine == a ? row : tile0 * 16 + some;
                load_y(b, from);
                // P of this lane's row, eight values per step: the slices are asked for together, and W behind them
                float v[JS][8];
                float top = 0.0f;
#pragma unroll
                for (int s = 0; s < JS; s++) {
                    const int k0 = 32 * s + 8 * g, j0 = PACKED && k0 >= rank ? k0 - rank : k0;
                    const bool real = b.mine == a && j0 < rank;
                    const float* p = L.P + (size_t)from * rank + min(j0, rank - 8);
                    const size_t step = (size_t)args.M * rank;
                    float4v lo[kFewSlices], hi[kFewSlices];
#pragma unroll
                    for (int c = 0; c < kFewSlices; c++)
                        if (c < L.slices) {
                            lo[c] = *reinterpret_cast<const float4v*>(p + c * step);
                            hi[c] = *reinterpret_cast<const float4v*>(p + c * step + 4);
                        }
                    if (s == 0 && a != held) hold(a);
                    loads_are_issued();
#pragma unroll
                    for (int c = 1; c < kFewSlices; c++)
                        if (c < L.slices) {
                            lo[0] += lo[c];
                            hi[0] += hi[c];
                        }
                    if (real && L.hidden && n0 == 0 && j0 == k0) {
                        float4v* h = reinterpret_cast<float4v*>(L.hidden + (size_t)row * rank + j0);
                        h[0] = lo[0];
                        h[1] = hi[0];
                    }
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        v[s][e] = real ? lo[0][e] : 0.0f;
                        v[s][4 + e] = real ? hi[0][e] : 0.0f;
                        top = fmaxf(top, fmaxf(fabsf(v[s][e]), fabsf(v[s][4 + e])));
                    }
                }
                b.power = 1.0f;
                if (FMT != kE3M2B) {
                    top = fmaxf(top, __shfl_xor(top, 16, 64));
                    top = fmaxf(top, __shfl_xor(top, 32, 64));
                    const int exponent = exponent_for(top);
                    b.power = power_of_two(exponent);
                    const float down = power_of_two(-exponent);
#pragma unroll
                    for (int s = 0; s < JS; s++)
#pragma unroll
                        for (int e = 0; e < 8; e++) v[s][e] *= down;
                }
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
                    if (PACKED) b.p[s][0] = 8 * g >= 2 * rank ? u32x4{0, 0, 0, 0} : (8 * g >= rank ? term[1] : term[0]);
                    else {
                        b.p[s][0] = term[0];
                        b.p[s][TERMS - 1] = term[1];
                    }
                }
            }
            if (SLICED) {
                scale = args.scaling ? args.scaling[a] : 1.0f;
            } else {
                if (a != held) hold(a);
#pragma unroll
                for (int s = 0; s < JS; s++)
#pragma unroll
                    for (int k = 0; k < TERMS; k++)
                        if (32 * s + 8 * g >= (PACKED ? 2 * rank : rank)) b.p[s][k] = u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int c = 0; c < CB; c++) {
                float4v acc[4] = {float4v{0, 0, 0, 0}, float4v{0, 0, 0, 0}, float4v{0, 0, 0, 0}, float4v{0, 0, 0, 0}};
#pragma unroll
                for (int s = 0; s < JS; s++)
#pragma unroll
                    for (int k = 0; k < TERMS; k++)
#pragma unroll
                        for (int t4 = 0; t4 < 4; t4++)
                            acc[t4] = mfma16x16x32_of<FMT>(__builtin_bit_cast(half8, w[c][t4][s]), __builtin_bit_cast(half8, b.p[s][k]), acc[t4]);
                if (b.mine == a) {
#pragma unroll
                    for (int t4 = 0; t4 < 4; t4++)
#pragma unroll
                        for (int p = 0; p < 2; p++) {
                            const uint32_t d = b.y[c][t4 >> 1][2 * (t4 & 1) + p];
                            const float lo = to_float<FMT>((uint16_t)d) + acc[t4][2 * p] * b.power * scale;
                            const float hi = to_float<FMT>((uint16_t)(d >> 16)) + acc[t4][2 * p + 1] * b.power * scale;
                            b.y[c][t4 >> 1][2 * (t4 & 1) + p] = to_bits<FMT>(lo) | (uint32_t)to_bits<FMT>(hi) << 16;
                        }
                }
            }
            if (SLICED && b.mine == a) store_y(b, row);
        }
        if (write) store_lines(b, t, write);
    };

    if (SLICED) {
        Rows b;
        for (int64_t t = 0; t < tiles; t++) {
            load(b, t);
            work(b, t);
        }
    } else {
        // the next row tile is in flight while one is worked on (past the end: all lanes read row 0, which costs little, and nothing is done)
        Rows b[2];
        load(b[0], 0);
        if (args.adapters == 1) hold(0);
        loads_are_issued();
        for (int64_t t = 0; t < tiles; t += 2) {
            load(b[1], t + 1);
            loads_are_issued();
            work(b[0], t);
            load(b[0], t + 2);
            loads_are_issued();
            work(b[1], t + 1);
        }
    }
}

template <int FMT, int JS, bool PACKED, bool TURNED, bool SLICED, int CB>
__global__ __launch_bounds__(256) void lora_expand_kernel(ExpandArgs args)
{
    __shared__ __align__(16) unsigned char shared[kExpandLds<TURNED>];
    expand_block<FMT, JS, PACKED, TURNED, SLICED, CB>(args, blockIdx.x, blockIdx.y, shared);
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
    const uint16_t* W;       // FUSED: [adapters, C, rank]
    float* S;                // FUSED: [blocks of columns][M][rank]
};

constexpr int kChunk = 64;      // rows between two barriers (a lane of a wavefront each)

// (FUSED and rank above 16: W's operands, 64 registers of every lane otherwise, with which a second workgroup would not fit the compute unit)
template <int JT, int CT, bool FUSED>
struct OuterW {
    u32x4 w[JT][2 * CT][64];
};
template <int CT, bool FUSED>
struct OuterW<1, CT, FUSED> {};
template <int JT, int CT>
struct OuterW<JT, CT, false> {};
template <int CT>
struct OuterW<1, CT, false> {};

template <int FMT, int JT, int CT, bool FUSED>
struct OuterLds : OuterW<JT, CT, FUSED> {
    static constexpr int TERMS = FMT == kE3M2B ? 3 : 2, kCols = 64 * CT, kLdQ = kCols + 16, kLdP = kChunk + 8;
    uint16_t q[kChunk * kLdQ];
    uint16_t p[TERMS][16 * JT][kLdP];
    uint32_t top[2][16 * JT];          // largest magnitudes of a chunk's columns of P, for this chunk and the next
    uint64_t rows[kChunk];   // of 64 chunks: which rows are the adapter's
};

// G[a][j][c] = sum over the adapter's rows m of P[m][j] Q[m][c].  A workgroup: one adapter, 64 * CT columns, one range of rows, a
// chunk of 64 rows at a time: the rows of Q go to LDS as they are and are read back turned, P is split into 16-bit terms and stored
// turned, while the next chunk is on its way.  fp16: two terms, and a power of two per chunk and column of P, its products are added
// up per chunk; bf16: three terms.  Rows of other adapters count as zeros on both sides (an infinity in one of them does not reach this
// sum), chunks without a row of this one are passed over.
// Bound by the order of its steps, a chunk's loads, maxima, LDS and products, which two workgroups to a compute unit hide for each other: 4096 x 22016
// rank 16 FUSED 53 us for 180 MB, 3.4 TB/s; rank 128 69 us for 2048 x 8192: P's terms out of LDS, read by every wavefront.
// FUSED: the chunk of Q in LDS is multiplied with W as well, S[block][m][j] = s * sum over the block's columns of Q[m][c] W[a][c][j]: the part of
// a shrink that this block of columns has, so that Q is read once for both.
template <int FMT, int JT, int CT, bool BY_COLUMN, bool FUSED>
__device__ __forceinline__ void outer_block(const OuterArgs& args, int block, int a, OuterLds<FMT, JT, CT, FUSED>& lds)
{
    using Lds = OuterLds<FMT, JT, CT, FUSED>;
    constexpr int TERMS = Lds::TERMS, kCols = Lds::kCols, kLdQ = Lds::kLdQ;
    constexpr int kQv = kChunk * kCols / 8 / 256;                              // 16-byte pieces of Q a thread
    constexpr int kPv = JT;                                                    // float4 of P a thread
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const int rank = args.rank, C = args.C, per_row = rank / 4;
    const int blocks = (C + kCols - 1) / kCols, split = block / blocks, c0 = (block % blocks) * kCols;
    const int chunks = (int)((args.M + kChunk - 1) / kChunk);
    const int begin = slice_begin(chunks, args.splits, split), end = slice_begin(chunks, args.splits, split + 1);
    const float s = args.scaling ? args.scaling[a] : 1.0f;
    const bool even = (per_row & (per_row - 1)) == 0;                          // lanes of the same columns lie a power of two apart

    int prow[kPv], pj[kPv];
#pragma unroll
    for (int v = 0; v < kPv; v++) {
        const int f = threadIdx.x + 256 * v;
        prow[v] = f / per_row;
        pj[v] = (f % per_row) * 4;
    }
    const int qcol = (threadIdx.x % (kCols / 8)) * 8, qrow = threadIdx.x / (kCols / 8);
    constexpr int kQstep = 256 / (kCols / 8);

    float4v sum[JT][CT];
#pragma unroll
    for (int j = 0; j < JT; j++)
#pragma unroll
        for (int c = 0; c < CT; c++) sum[j][c] = float4v{0, 0, 0, 0};

    // FUSED: W of the block's columns as operands, turned in LDS (each wavefront multiplies 16 rows with all columns)
    constexpr int kSteps = FUSED ? kCols / 32 : 1, kLdW = 16 * JT + 8;
    constexpr bool kSharedW = FUSED && JT > 1;
    u32x4 w[FUSED && !kSharedW ? JT : 1][kSharedW ? 1 : kSteps];
    if constexpr (FUSED) {
        static_assert(kCols * kLdW <= kChunk * kLdQ, "W of the columns fits where the chunk of Q lies");
        const int per = rank / 8, pieces = min(kCols, C - c0) * per;
        const u32x4* from = reinterpret_cast<const u32x4*>(args.W + ((size_t)a * C + c0) * rank);
        for (int p = threadIdx.x; p < kCols * per; p += 256)
            *reinterpret_cast<u32x4*>(lds.q + (p / per) * kLdW + (p % per) * 8) = p < pieces ? from[p] : u32x4{0, 0, 0, 0};
        __syncthreads();
        auto operand = [&](int j, int k) {
            u32x4 v;
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const u32x2 d = read_turned(lds.q + (32 * k + 8 * g + 4 * e + (i >> 2)) * kLdW + min(16 * j + 4 * (i & 3), rank - 4));
                v[2 * e] = d[0];
                v[2 * e + 1] = d[1];
            }
            return v;
        };
        if constexpr (kSharedW) {
#pragma unroll
            for (int p = 0; p < JT * kSteps / 4; p++) {
                const int at = wave + 4 * p;
                lds.w[at / kSteps][at % kSteps][lane] = operand(at / kSteps, at % kSteps);
            }
        } else {
#pragma unroll
            for (int j = 0; j < JT; j++)
#pragma unroll
                for (int k = 0; k < kSteps; k++) w[j][k] = operand(j, k);
        }
    }
    // The rows of this adapter, 64 chunks at a time: one load a lane and chunk, all under way together.
    int batch = begin;
    uint64_t todo = 0;               // chunks of the batch that have rows and are still to be done
    auto gather = [&]() {
        __syncthreads();
        int owner[kChunk / 4];
        auto row_of = [&](int v) { return (int64_t)(batch + wave + 4 * v) * kChunk + lane; };
        if (args.index) {
#pragma unroll
            for (int v = 0; v < kChunk / 4; v++) owner[v] = args.index[min(row_of(v), args.M - 1)];
            loads_are_issued();
        } else {
#pragma unroll
            for (int v = 0; v < kChunk / 4; v++) owner[v] = 0;
        }
#pragma unroll
        for (int v = 0; v < kChunk / 4; v++) {
            const uint64_t r = __ballot(owner[v] == a && batch + wave + 4 * v < end && row_of(v) < args.M);
            if (lane == 0) lds.rows[wave + 4 * v] = r;
        }
        __syncthreads();
        todo = __ballot(lds.rows[lane] != 0);
    };
    auto find = [&](uint64_t& rows) {          // the next chunk with rows of this adapter, or end
        while (!todo) {
            batch += kChunk;
            if (batch >= end) return end;
            gather();
        }
        const int k = __builtin_ctzll(todo);
        todo &= todo - 1;
        rows = lds.rows[k];
        rows = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(rows >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)rows);
        return batch + k;
    };
    // Loads take no branch: lanes of rows that are not the adapter's, and of columns past the end, read a row, or column, that is.  They count as
    // zeros where the operands are put into LDS.
    u32x4 q[kQv];
    float4v p4[kPv];
    auto load = [&](int chunk, uint64_t rows) {
        const int64_t m0 = (int64_t)chunk * kChunk;
        const int some = __builtin_ctzll(rows);
        const uint16_t* from = args.Q + (size_t)m0 * C + (c0 + qcol < C ? c0 + qcol : c0);
#pragma unroll
        for (int v = 0; v < kQv; v++) {
            const int row = qrow + kQstep * v;
            q[v] = *reinterpret_cast<const u32x4*>(from + (size_t)((rows >> row) & 1 ? row : some) * C);
        }
        auto p_of = [&](int v) { return args.P + (size_t)(m0 + (prow[v] < kChunk && ((rows >> (prow[v] & 63)) & 1) ? prow[v] : some)) * rank + pj[v]; };
#pragma unroll
        for (int v = 0; v < kPv; v++) p4[v] = *reinterpret_cast<const float4v*>(p_of(v));
        if (args.slices > 1) {
#pragma unroll
            for (int v = 0; v < kPv; v++) {
#pragma unroll 8
                for (int c = 1; c < args.slices; c++) p4[v] += *reinterpret_cast<const float4v*>(p_of(v) + (size_t)c * args.M * rank);
            }
        }
    };
    uint64_t rows = 0;
    if (begin < end) gather();
    int chunk = begin < end ? find(rows) : end;
    if (chunk < end) load(chunk, rows);
    int turn = 0;
    if (FMT != kE3M2B) {
        if (threadIdx.x < 16 * JT) lds.top[0][threadIdx.x] = 0;
        __syncthreads();
    }
    while (chunk < end) {
#pragma unroll
        for (int v = 0; v < kPv; v++)
            if (!(prow[v] < kChunk && ((rows >> (prow[v] & 63)) & 1))) p4[v] = float4v{0, 0, 0, 0};
        if (FMT != kE3M2B) {
#pragma unroll
            for (int v = 0; v < kPv; v++) {
                uint32_t m[4];                                    // (magnitudes order like their bits, NaN above all)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const float x = fabsf(p4[v][e]);
                    m[e] = __builtin_bit_cast(uint32_t, x);
                }
                if (even) {
                    for (int off = per_row; off < 64; off <<= 1) {
#pragma unroll
                        for (int e = 0; e < 4; e++) m[e] = max(m[e], (uint32_t)__shfl_xor((int)m[e], off, 64));
                    }
                }
                if (prow[v] < kChunk && (!even || lane < per_row)) {
#pragma unroll
                    for (int e = 0; e < 4; e++) atomicMax(&lds.top[turn][pj[v] + e], m[e]);
                }
            }
        }
        if (rows != ~0ull || c0 + kCols > C) {
#pragma unroll
            for (int v = 0; v < kQv; v++)
                if (!((rows >> (qrow + kQstep * v)) & 1) || c0 + qcol >= C) q[v] = u32x4{0, 0, 0, 0};
        }
        __syncthreads();                                          // (the largest are known, and the last chunk's operands have been read)
        if (FMT != kE3M2B && threadIdx.x < 16 * JT) lds.top[turn ^ 1][threadIdx.x] = 0;
#pragma unroll
        for (int v = 0; v < kQv; v++) *reinterpret_cast<u32x4*>(lds.q + (qrow + kQstep * v) * kLdQ + qcol) = q[v];
#pragma unroll
        for (int v = 0; v < kPv; v++) {
            if (prow[v] < kChunk) {
                float down[4] = {1.0f, 1.0f, 1.0f, 1.0f};
                if (FMT != kE3M2B) {
                    const u32x4 top = *reinterpret_cast<const u32x4*>(&lds.top[turn][pj[v]]);
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const uint32_t t = top[e];
                        down[e] = power_of_two(-exponent_for(__builtin_bit_cast(float, t)));
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    uint16_t t[TERMS];
                    split_terms<FMT>(p4[v][e] * down[e], t);
#pragma unroll
                    for (int k = 0; k < TERMS; k++) lds.p[k][pj[v] + e][prow[v]] = t[k];
                }
            }
        }
        __syncthreads();
        const uint64_t these = rows;
        const int64_t m0 = (int64_t)chunk * kChunk + 16 * wave + 4 * g;
        chunk = find(rows);
        if (chunk < end) load(chunk, rows);
        loads_are_issued();
        if constexpr (FUSED) {
            float4v d[JT];
#pragma unroll
            for (int j = 0; j < JT; j++) d[j] = float4v{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < kSteps; k++) {
                const half8 x = *reinterpret_cast<const half8*>(lds.q + (16 * wave + i) * kLdQ + 32 * k + 8 * g);
#pragma unroll
                for (int j = 0; j < JT; j++) {
                    u32x4 v;
                    if constexpr (kSharedW) v = lds.w[j][k][lane];
                    else v = w[j][k];
                    d[j] = mfma16x16x32_of<FMT>(x, __builtin_bit_cast(half8, v), d[j]);
                }
            }
            float* S = args.S + ((size_t)(block % blocks) * args.M + m0) * rank;
#pragma unroll
            for (int j = 0; j < JT; j++)
#pragma unroll
                for (int r = 0; r < 4; r++)
                    if (((these >> (16 * wave + 4 * g + r)) & 1) && 16 * j + i < rank) S[(size_t)r * rank + 16 * j + i] = d[j][r] * s;
        }
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
                for (int k = 0; k < TERMS; k++) p[j][k] = *reinterpret_cast<const half8*>(&lds.p[k][16 * j + i][32 * step + 8 * g]);
#pragma unroll
            for (int c = 0; c < CT; c++) {
                u32x4 d;
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const u32x2 b = read_turned(lds.q + (32 * step + 8 * g + 4 * e + (i >> 2)) * kLdQ + (wave * CT + c) * 16 + 4 * (i & 3));
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
                const u32x4 top = *reinterpret_cast<const u32x4*>(&lds.top[turn][16 * j + 4 * g]);
                float4v f;
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const uint32_t t = top[r];
                    f[r] = power_of_two(exponent_for(__builtin_bit_cast(float, t)));
                }
#pragma unroll
                for (int c = 0; c < CT; c++) sum[j][c] += part[j][c] * f;
            }
        }
        turn ^= 1;
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

template <int FMT, int JT, int CT, bool BY_COLUMN, bool FUSED>
__global__ __launch_bounds__(256) void lora_outer_kernel(OuterArgs args)
{
    __shared__ __align__(16) OuterLds<FMT, JT, CT, FUSED> lds;
    outer_block<FMT, JT, CT, BY_COLUMN, FUSED>(args, blockIdx.x, blockIdx.y, lds);
}

// ------------------------------------------------------------------ two independent steps of the backward pass in one launch
// A launch costs 7 to 9 us beside its work here: the first loads of its workgroups, and at its end the write-back of what lies in the caches.  The
// workgroups of two steps that do not read one another's results hide that for each other.
template <int FMT, int JT>
union FirstLds {
    unsigned char shrink[kShrinkLds<JT, 1, true, 4>];
    OuterLds<FMT, JT, 2, false> outer;
};

// few rows: dS, and the gradient of B
template <int FMT, int JT>
__global__ __launch_bounds__(256) void lora_first_kernel(ShrinkArgs shrink, int shrinks, OuterArgs outer)
{
    __shared__ __align__(16) FirstLds<FMT, JT> lds;
    const int blocks = (outer.C + 127) / 128 * outer.splits, id = (int)blockIdx.x;
    if (id < shrinks * shrink.slots) shrink_block<FMT, JT, 1, true, 4>(shrink, id % shrinks, id / shrinks, lds.shrink);
    else outer_block<FMT, JT, 2, true, false>(outer, (id - shrinks * shrink.slots) % blocks, (id - shrinks * shrink.slots) / blocks, lds.outer);
}

template <int FMT, int JT, int CT>
union SecondLds {
    unsigned char expand[kExpandLds<true>];
    OuterLds<FMT, JT, CT, false> outer;
};

// the gradient of A, and dX: 4096 x 8192 rank 16 49 us for 201 MB, 4.1 TB/s
template <int FMT, int JT, int CT, bool SLICED>
__global__ __launch_bounds__(256) void lora_second_kernel(ExpandArgs expand, int expands, OuterArgs outer)
{
    __shared__ __align__(16) SecondLds<FMT, JT, CT> lds;
    // (in turn, a workgroup of the one beside one of the other, they took longer: 56 us became 59, at rank 128 120 became 157)
    const int blocks = (outer.C + 64 * CT - 1) / (64 * CT) * outer.splits, outers = blocks * outer.adapters, id = (int)blockIdx.x;
    if (id < outers) outer_block<FMT, JT, CT, false, false>(outer, id % blocks, id / blocks, lds.outer);
    else expand_block<FMT, JT <= 2 ? 1 : JT / 2, JT == 1, true, SLICED, SLICED || JT == 8 ? 1 : 2>(expand, (id - outers) % expands, (id - outers) / expands, lds.expand);
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
        #pragma unroll 8
        for (int c = 0; c < args.splits[w]; c++) v += args.part[w][(size_t)c * args.count[w] + e];
        args.out[w][e] = v;
    }
}

// ------------------------------------------------------------------ plans and launches
static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Up to this many rows the slices of a shrink are added up by the kernels that read them; above it a launch of its own adds them up, once
// (128 x 4096 x 4096 9.6 us, with that launch 13.7; 333 x 13824 x 5120 with five adapters 27 and 23, gradients of 512 x 8192 x 8192, rank 64,
// 55 and 45).
constexpr int64_t kFewRows = 256;
// Up to this many rows a shrink workgroup takes 16 of them and its adapters are dealt to workgroups of their own, above it 64 and one adapter
// after another (333 x 5120 with five adapters 8.1 us against 17).
constexpr int64_t kNarrowRows = 512;
// Up to this many rows the expand kernel's adapters are dealt to workgroups of their own as well: with more, those that find nothing to do cost
// more than they save (256 x 8192 with eight adapters 15.9 us, here 10.4).
constexpr int64_t kSlotRows = 64;

// Rows a shrink workgroup takes, slots its adapters are dealt to, and slices of the contraction: two workgroups for each compute unit
// (one, with few rows) where the contraction is long enough to be cut (a slice gives each wavefront at least one unit of 64).
struct ShrinkPlan {
    int row_tiles, slots, slices;
    int64_t groups;
};

static ShrinkPlan plan_shrink(int64_t M, int C, int rank, int adapters)
{
    ShrinkPlan p;
    const bool narrow = M <= kNarrowRows;
    p.row_tiles = narrow ? 1 : (rank > 64 ? 2 : 4);
    const int64_t rows = 16 * p.row_tiles;
    p.groups = ceil_div(M, rows);
    p.slots = narrow ? (int)(adapters < rows ? adapters : rows) : 1;
    const int waves = !narrow || rank > 64 ? 4 : 8, limit = M > kFewRows ? 16 : kFewSlices;
    const int64_t have = p.groups * (M <= kSlotRows ? p.slots : 1), most = C / (64 * waves);
    int64_t slices = ceil_div(narrow ? 256 : 512, have);
    if (slices > most) slices = most;
    if (slices > limit) slices = limit;
    p.slices = (int)(slices < 1 ? 1 : slices);
    return p;
}

static int expand_slots(int64_t M, const ShrinkPlan& p) { return M <= kSlotRows ? p.slots : 1; }

// Columns of an outer workgroup, and ranges of rows that separate workgroups take.  Where two workgroups fit a compute unit 512 are a round (516 took
// 70 us where 430 take 54: the last four had a round to themselves); a workgroup needs about 4 us beside its chunks and 3 (128 columns: 2.2) for each, adapters sharing
// the rows in runs (in mixed order each of them reads every chunk that has a row of its own, and the same plan takes longer: gradients of 2048 x 8192 x 8192, rank 16,
// four adapters 64 us in runs, 90 mixed); every range costs a tensor of partial sums, written and read at 4 TB/s, and together they cost a launch.
struct OuterPlan {
    int columns, splits;
};

// Workgroups of an outer product that a compute unit holds at a time, by their registers: two where a wavefront has 256 of a SIMD's 512 at most, as up to
// rank 64, one above (2048 x 8192 x 8192, rank 128: 203 us, counted as two 223).  Ranks above 32 with 256 columns count as two although fp16, and dA beside
// dX in bf16, have one: counted as one they get 128 columns, which read P twice as often (4096 x 22016 x 8192, rank 64: 276 and 207 us became 282 and 245).
static int outer_resident(int rank) { return rank > 64 ? 1 : 2; }

static OuterPlan plan_outer(int64_t M, int C, int rank, int adapters, bool fused)
{
    OuterPlan best{256, 1};
    double least = 1e30;
    const int64_t chunks = ceil_div(M, kChunk);
    for (int columns = 256; columns >= 128; columns -= 128) {
        if (columns == 256 ? rank > 64 || M <= kFewRows : fused) continue;
        const int64_t have = ceil_div(C, columns) * adapters;
        for (int splits = 1; splits <= 64 && splits <= chunks; splits++) {
            const double chunk = columns == 256 ? 3.0 : 2.2, mine = (double)ceil_div(chunks, (int64_t)splits * adapters);
            const double partial = splits > 1 ? 4.0 + 8e-6 * splits * adapters * rank * C / 4 : 0.0;
            const double cost = (double)ceil_div(have * splits, 256 * outer_resident(rank)) * (4.0 + chunk * mine) + partial;
            if (cost < least) {
                least = cost;
                best = OuterPlan{columns, splits};
            }
        }
    }
    return best;
}

// The gradient of B and the shrink of dY in one reading of dY: the shrink's parts, one per 256 columns, cost rank / 64 of what they save.
static bool fuses(int64_t M, int rank) { return M > kFewRows && rank <= 32; }

// (turned: ranks above 32 only, which is where dY is not read for dB and dS together, and up to kFewRows the shrink shares a launch)
template <int FMT, bool TURNED>
static hipError_t launch_shrink(const ShrinkArgs& a, bool narrow, int64_t workgroups, hipStream_t stream)
{
    int rank = 0;
    for (int l = 0; l < a.layers; l++) rank = a.layer[l].rank > rank ? a.layer[l].rank : rank;
    const dim3 grid((unsigned)workgroups, (unsigned)a.slots), block(256);
    if constexpr (!TURNED) {
        if (rank <= 16) {
            if (narrow) hipLaunchKernelGGL((lora_shrink_kernel<FMT, 1, 1, TURNED>), grid, dim3(64 * kShrinkWaves<1, 1>), 0, stream, a);
            else hipLaunchKernelGGL((lora_shrink_kernel<FMT, 1, 4, TURNED>), grid, block, 0, stream, a);
            return hipGetLastError();
        }
        if (rank <= 32) {
            if (narrow) hipLaunchKernelGGL((lora_shrink_kernel<FMT, 2, 1, TURNED>), grid, dim3(64 * kShrinkWaves<2, 1>), 0, stream, a);
            else hipLaunchKernelGGL((lora_shrink_kernel<FMT, 2, 4, TURNED>), grid, block, 0, stream, a);
            return hipGetLastError();
        }
    }
    if (rank <= 64) {
        if (narrow) hipLaunchKernelGGL((lora_shrink_kernel<FMT, 4, 1, TURNED>), grid, dim3(64 * kShrinkWaves<4, 1>), 0, stream, a);
        else hipLaunchKernelGGL((lora_shrink_kernel<FMT, 4, 4, TURNED>), grid, block, 0, stream, a);
    } else {
        if (narrow) hipLaunchKernelGGL((lora_shrink_kernel<FMT, 8, 1, TURNED>), grid, dim3(64 * kShrinkWaves<8, 1>), 0, stream, a);
        else hipLaunchKernelGGL((lora_shrink_kernel<FMT, 8, 2, TURNED>), grid, block, 0, stream, a);
    }
    return hipGetLastError();
}

template <int FMT>
static hipError_t launch_finish(const float* P, float* sum, uint16_t* terms, float* power, int64_t M, int rank, int slices, const int32_t* index,
                                int adapters, hipStream_t stream)
{
    int lanes = 2;
    while (4 * lanes < rank) lanes *= 2;
    const FinishArgs f{P, sum, terms, power, M, rank, slices, lanes, index, adapters};
    if (slices > 32) hipLaunchKernelGGL((lora_finish_kernel<FMT, true>), dim3((unsigned)ceil_div(M * lanes, 64)), dim3(256), 0, stream, f);
    else hipLaunchKernelGGL((lora_finish_kernel<FMT, false>), dim3((unsigned)ceil_div(M * lanes, 256)), dim3(256), 0, stream, f);
    return hipGetLastError();
}

// Columns of an expand workgroup
static int expand_across(bool few, int rank) { return few ? 256 : (rank > 64 ? 64 : 128); }

template <int FMT>
static hipError_t launch_expand(const ExpandArgs& a, bool few, int rank, int64_t workgroups, hipStream_t stream)
{
    const dim3 grid((unsigned)workgroups, (unsigned)a.slots), block(256);
    bool packed = true;
    for (int l = 0; l < a.layers; l++) packed = packed && a.layer[l].rank <= 16;
    if (few) {
        if (packed) hipLaunchKernelGGL((lora_expand_kernel<FMT, 1, true, false, true, 1>), grid, block, 0, stream, a);
        else if (rank <= 32) hipLaunchKernelGGL((lora_expand_kernel<FMT, 1, false, false, true, 1>), grid, block, 0, stream, a);
        else if (rank <= 64) hipLaunchKernelGGL((lora_expand_kernel<FMT, 2, false, false, true, 1>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((lora_expand_kernel<FMT, 4, false, false, true, 1>), grid, block, 0, stream, a);
    } else {
        if (packed) hipLaunchKernelGGL((lora_expand_kernel<FMT, 1, true, false, false, 2>), grid, block, 0, stream, a);
        else if (rank <= 32) hipLaunchKernelGGL((lora_expand_kernel<FMT, 1, false, false, false, 2>), grid, block, 0, stream, a);
        else if (rank <= 64) hipLaunchKernelGGL((lora_expand_kernel<FMT, 2, false, false, false, 2>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((lora_expand_kernel<FMT, 4, false, false, false, 1>), grid, block, 0, stream, a);
    }
    return hipGetLastError();
}

// 64 * CT columns a workgroup: 256 for ranks up to 64 only.  By column (the gradient of B): ranks above 32, the others' shares dY's reading with the shrink or,
// up to kFewRows, its launch.
template <int FMT, int CT, bool BY_COLUMN>
static hipError_t launch_outer_rank(const OuterArgs& a, dim3 grid, hipStream_t stream)
{
    if constexpr (!BY_COLUMN) {
        if (a.rank <= 16) {
            hipLaunchKernelGGL((lora_outer_kernel<FMT, 1, CT, BY_COLUMN, false>), grid, dim3(256), 0, stream, a);
            return hipGetLastError();
        }
        if (a.rank <= 32) {
            hipLaunchKernelGGL((lora_outer_kernel<FMT, 2, CT, BY_COLUMN, false>), grid, dim3(256), 0, stream, a);
            return hipGetLastError();
        }
    }
    if (a.rank <= 64) {
        hipLaunchKernelGGL((lora_outer_kernel<FMT, 4, CT, BY_COLUMN, false>), grid, dim3(256), 0, stream, a);
    } else {
        if constexpr (CT == 2) hipLaunchKernelGGL((lora_outer_kernel<FMT, 8, CT, BY_COLUMN, false>), grid, dim3(256), 0, stream, a);
        else return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

template <int FMT, bool BY_COLUMN>
static hipError_t launch_outer(const OuterArgs& a, int columns, hipStream_t stream)
{
    const dim3 grid((unsigned)(ceil_div(a.C, columns) * a.splits), (unsigned)a.adapters);
    if constexpr (BY_COLUMN) {
        if (a.S) {
            if (a.rank <= 16) hipLaunchKernelGGL((lora_outer_kernel<FMT, 1, 4, true, true>), grid, dim3(256), 0, stream, a);
            else hipLaunchKernelGGL((lora_outer_kernel<FMT, 2, 4, true, true>), grid, dim3(256), 0, stream, a);
            return hipGetLastError();
        }
    }
    return columns == 128 ? launch_outer_rank<FMT, 2, BY_COLUMN>(a, grid, stream) : launch_outer_rank<FMT, 4, BY_COLUMN>(a, grid, stream);
}

template <int FMT>
static hipError_t launch_first(const ShrinkArgs& s, int shrinks, const OuterArgs& o, hipStream_t stream)
{
    const dim3 grid((unsigned)(shrinks * s.slots + ceil_div(o.C, 128) * o.splits * o.adapters)), block(256);
    if (o.rank <= 16) hipLaunchKernelGGL((lora_first_kernel<FMT, 1>), grid, block, 0, stream, s, shrinks, o);
    else if (o.rank <= 32) hipLaunchKernelGGL((lora_first_kernel<FMT, 2>), grid, block, 0, stream, s, shrinks, o);
    else if (o.rank <= 64) hipLaunchKernelGGL((lora_first_kernel<FMT, 4>), grid, block, 0, stream, s, shrinks, o);
    else hipLaunchKernelGGL((lora_first_kernel<FMT, 8>), grid, block, 0, stream, s, shrinks, o);
    return hipGetLastError();
}

template <int FMT, int CT, bool SLICED>
static hipError_t launch_second_rank(const ExpandArgs& e, int expands, const OuterArgs& o, hipStream_t stream)
{
    const dim3 grid((unsigned)(expands * e.slots + ceil_div(o.C, 64 * CT) * o.splits * o.adapters)), block(256);
    if (o.rank <= 16) hipLaunchKernelGGL((lora_second_kernel<FMT, 1, CT, SLICED>), grid, block, 0, stream, e, expands, o);
    else if (o.rank <= 32) hipLaunchKernelGGL((lora_second_kernel<FMT, 2, CT, SLICED>), grid, block, 0, stream, e, expands, o);
    else if (o.rank <= 64) hipLaunchKernelGGL((lora_second_kernel<FMT, 4, CT, SLICED>), grid, block, 0, stream, e, expands, o);
    else if constexpr (CT == 2) hipLaunchKernelGGL((lora_second_kernel<FMT, 8, CT, SLICED>), grid, block, 0, stream, e, expands, o);
    else return hipErrorInvalidValue;          // (the grid counts columns by 256, which ranks above 64 do not take)
    return hipGetLastError();
}

template <int FMT>
static hipError_t launch_second(const ExpandArgs& e, bool few, int64_t expands, const OuterArgs& o, int columns, hipStream_t stream)
{
    if (few) return launch_second_rank<FMT, 2, true>(e, (int)expands, o, stream);
    return columns == 128 ? launch_second_rank<FMT, 2, false>(e, (int)expands, o, stream)
                          : launch_second_rank<FMT, 4, false>(e, (int)expands, o, stream);
}

// Row tiles of 16 rows that a wavefront of the expand kernel takes one after another (its operands of W stay in registers, and the next tile's loads
// are in flight): as many as make the workgroups one round of two to a compute unit.
static int expand_row_tiles(int64_t M, int64_t column_blocks)
{
    if (M <= kFewRows) return 1;
    const int64_t t = ceil_div(ceil_div(M, 64) * column_blocks, 512);
    return (int)(t < 1 ? 1 : (t > 16 ? 16 : t));
}

static int64_t expand_groups(int64_t M, bool few, int row_tiles) { return ceil_div(M, 16 * (few ? 1 : 4) * row_tiles); }

static size_t round_up(size_t bytes) { return (bytes + 255) / 256 * 256; }

// What lies behind the zero region for one shrink: the slices; with more than a few rows the terms and powers of two made of them.
struct ShrinkSpace {
    size_t slices, terms, power, bytes;
};

static ShrinkSpace shrink_space(const ShrinkPlan& p, int64_t M, int64_t rank)
{
    ShrinkSpace s{};
    s.slices = round_up((size_t)p.slices * M * rank * 4);
    if (M > kFewRows) {
        s.terms = round_up((size_t)M * rank * 4);
        s.power = round_up((size_t)M * 4);
    }
    s.bytes = s.slices + s.terms + s.power;
    return s;
}

// The rank that decides which kernels run: the largest of the group.
static int group_rank(const fp6_lora_problem* pr, int count)
{
    int rank = 0;
    for (int l = 0; l < count; l++) rank = (int)pr[l].rank > rank ? (int)pr[l].rank : rank;
    return rank;
}

size_t lora_workspace(int64_t M, const fp6_lora_problem* pr, int count, int adapters)
{
    size_t need = kZeroBytes;
    const int rank = group_rank(pr, count);
    for (int l = 0; l < count; l++) need += shrink_space(plan_shrink(M, (int)pr[l].K, rank, adapters), M, pr[l].rank).bytes;
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
    const bool few = M <= kFewRows;
    const int rank = group_rank(pr, count), across = expand_across(few, rank);
    unsigned char* at = workspace + kZeroBytes;
    int64_t shrinks = 0, expands = 0, columns = 0;
    for (int l = 0; l < count; l++) columns += ceil_div(pr[l].N, across);
    e.row_tiles = expand_row_tiles(M, columns);
    for (int l = 0; l < count; l++) {
        const ShrinkPlan p = plan_shrink(M, (int)pr[l].K, rank, adapters);
        const ShrinkSpace space = shrink_space(p, M, pr[l].rank);
        s.slots = p.slots;
        e.slots = expand_slots(M, p);
        s.layer[l] = ShrinkLayer{pr[l].X, pr[l].A, (float*)at, (int)pr[l].K, (int)pr[l].rank, p.slices, (int)shrinks};
        e.layer[l] = ExpandLayer{few ? (const float*)at : (const float*)(at + space.slices + space.terms), (const uint16_t*)(at + space.slices),
                                 pr[l].B, pr[l].Y, pr[l].out, pr[l].hidden, (int)pr[l].N, (int)pr[l].rank, p.slices, (int)expands};
        at += space.bytes;
        shrinks += p.groups * p.slices;
        expands += ceil_div(pr[l].N, across) * expand_groups(M, few, e.row_tiles);
    }
    hipError_t err = launch_shrink<FMT, false>(s, M <= kNarrowRows, shrinks, stream);
    for (int l = 0; l < count && !few && err == hipSuccess; l++)
        err = launch_finish<FMT>(s.layer[l].P, pr[l].hidden, const_cast<uint16_t*>(e.layer[l].terms), const_cast<float*>(e.layer[l].P), M,
                                 (int)pr[l].rank, s.layer[l].slices, index, adapters, stream);
    if (err != hipSuccess) return err;
    return launch_expand<FMT>(e, few, rank, expands, stream);
}

hipError_t launch_lora(bool bf16, int64_t M, const fp6_lora_problem* pr, int count, int adapters, const int32_t* index, const float* scaling,
                       void* workspace, hipStream_t stream)
{
    return bf16 ? launch_lora_t<kE3M2B>(M, pr, count, adapters, index, scaling, (unsigned char*)workspace, stream)
                : launch_lora_t<kE3M2>(M, pr, count, adapters, index, scaling, (unsigned char*)workspace, stream);
}

// Workspace of the backward pass behind the zero region: the slices of dH and what is made of them, then the splits of dA and of dB (none
// where there is one).
struct BackwardPlan {
    ShrinkPlan shrink;
    ShrinkSpace space;
    OuterPlan a, b;
    bool fused;
    size_t da, db;           // bytes
};

static BackwardPlan plan_backward(int64_t M, int64_t N, int64_t K, int rank, int adapters)
{
    BackwardPlan p;
    p.fused = fuses(M, rank);
    p.a = plan_outer(M, (int)K, rank, adapters, false);
    p.b = plan_outer(M, (int)N, rank, adapters, p.fused);
    p.shrink = plan_shrink(M, (int)N, rank, adapters);
    if (p.fused) p.shrink.slices = (int)ceil_div(N, p.b.columns);
    p.space = shrink_space(p.shrink, M, rank);
    p.da = p.a.splits > 1 ? round_up((size_t)p.a.splits * adapters * rank * K * 4) : 0;
    p.db = p.b.splits > 1 ? round_up((size_t)p.b.splits * adapters * rank * N * 4) : 0;
    return p;
}

size_t lora_backward_workspace(int64_t M, int64_t N, int64_t K, int rank, int adapters)
{
    const BackwardPlan p = plan_backward(M, N, K, rank, adapters);
    return kZeroBytes + p.space.bytes + p.da + p.db;
}

template <int FMT>
static hipError_t launch_backward_t(const LoraBackward& b, unsigned char* workspace, hipStream_t stream)
{
    const BackwardPlan p = plan_backward(b.M, b.N, b.K, b.rank, b.adapters);
    const bool few = b.M <= kFewRows;
    unsigned char* at = workspace + kZeroBytes;
    float* dh = (float*)at;
    uint16_t* terms = (uint16_t*)(at + p.space.slices);
    float* power = (float*)(at + p.space.slices + p.space.terms);
    float* da = (float*)(at + p.space.bytes);
    float* db = (float*)(at + p.space.bytes + p.da);
    hipError_t err = hipSuccess;
    const OuterArgs ob{b.hidden, b.dY, p.b.splits > 1 ? db : b.dB, b.M, (int)b.N, b.rank, 1, b.adapters, p.b.splits, b.accumulate, b.index, b.scaling,
                       p.fused ? b.B : nullptr, p.fused ? dh : nullptr};
    ShrinkArgs s{};
    s.layers = 1;
    s.M = b.M;
    s.index = b.index;
    s.scaling = b.scaling;
    s.adapters = b.adapters;
    s.slots = p.shrink.slots;
    s.layer[0] = ShrinkLayer{b.dY, b.B, dh, (int)b.N, b.rank, p.shrink.slices, 0};
    const int64_t shrinks = p.shrink.groups * p.shrink.slices;
    if (few) {
        err = launch_first<FMT>(s, (int)shrinks, ob, stream);
    } else {
        if (!p.fused) err = launch_shrink<FMT, true>(s, b.M <= kNarrowRows, shrinks, stream);
        // (right behind the shrink, where it is not part of it: what the last-level cache still holds of dY is read from there)
        if (err == hipSuccess) err = launch_outer<FMT, true>(ob, p.b.columns, stream);
        // the sum over the slices goes where the first slice lies
        if (err == hipSuccess) err = launch_finish<FMT>(dh, dh, terms, power, b.M, b.rank, p.shrink.slices, b.index, b.adapters, stream);
    }
    if (err != hipSuccess) return err;
    const OuterArgs oa{dh, b.X, p.a.splits > 1 ? da : b.dA, b.M, (int)b.K, b.rank, few ? p.shrink.slices : 1, b.adapters, p.a.splits, b.accumulate,
                       b.index, nullptr, nullptr, nullptr};
    if (b.out) {
        const int across = expand_across(few, b.rank);
        ExpandArgs e{};
        e.layers = 1;
        e.M = b.M;
        e.index = b.index;
        e.adapters = b.adapters;
        e.slots = expand_slots(b.M, p.shrink);
        e.row_tiles = expand_row_tiles(b.M, ceil_div(b.K, across));
        e.layer[0] = ExpandLayer{few ? dh : power, terms, b.A, b.dX, b.out, nullptr, (int)b.K, b.rank, p.shrink.slices, 0};
        err = launch_second<FMT>(e, few, ceil_div(b.K, across) * expand_groups(b.M, few, e.row_tiles), oa, p.a.columns, stream);
    } else {
        err = launch_outer<FMT, false>(oa, p.a.columns, stream);
    }
    if (err != hipSuccess || (p.a.splits == 1 && p.b.splits == 1)) return err;
    JoinArgs j{};
    j.accumulate = b.accumulate;
    j.part[0] = (const float4v*)da;
    j.out[0] = (float4v*)b.dA;
    j.count[0] = p.a.splits > 1 ? (int64_t)b.adapters * b.rank * b.K / 4 : 0;
    j.splits[0] = p.a.splits;
    j.part[1] = (const float4v*)db;
    j.out[1] = (float4v*)b.dB;
    j.count[1] = p.b.splits > 1 ? (int64_t)b.adapters * b.rank * b.N / 4 : 0;
    j.splits[1] = p.b.splits;
    const int64_t want = ceil_div(j.count[0] + j.count[1], 256);
    hipLaunchKernelGGL(lora_join_kernel, dim3((unsigned)(want < 4096 ? want : 4096)), dim3(256), 0, stream, j);
    return hipGetLastError();
}

hipError_t launch_lora_backward(bool bf16, const LoraBackward& b, void* workspace, hipStream_t stream)
{
    return bf16 ? launch_backward_t<kE3M2B>(b, (unsigned char*)workspace, stream) : launch_backward_t<kE3M2>(b, (unsigned char*)workspace, stream);
}

}  // namespace fp6
