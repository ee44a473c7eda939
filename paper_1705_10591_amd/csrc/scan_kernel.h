// The scan over tokens, what its forms share: h[t] = exp(d[t] A) h[t-1] + d[t] u[t] B[t] for every channel and state.
//
// The recurrence is elementwise, so the work goes to the vector ALU: a product, an exponential, a product and two
// multiply-adds for each (token, channel, state).  What shapes the kernels:
//  * A lane is a channel and a wave has R states of 64 channels: B[t] and C[t] are then the same for a whole wave and come
//    through scalar registers, which costs the vector ALU nothing.  The W waves of a workgroup have the other states of the
//    same channels (four waves of 1, 2 or 4 states, or eight of 4); what all states of a channel share (d, d u, the sum
//    over states) goes through LDS.
//  * Tokens come in tiles of kT = 16.  Thread by thread a tile's 16 x 64 values are loaded and stored in runs of E = 16 / W
//    channels, and d, its softplus and the gate are computed once, not once per wave.
//  * bc_kernel lays B and C out for the scalar loads first: fp32, [N][G][tiles][W][8 pairs of tokens][4 + 4 of B, 4 + 4 of C], R of each 4
//    used, zeros behind the end of a sequence and beyond state S.  With d = 0 there too, tokens that do not count leave the state as it is,
//    and the loops need no masks.
//  * Scalar loads come back in any order, so that a wait for one is a wait for all: a tile is walked in steps of kStep = 4
//    tokens.  A step waits for its operands, asks for those of the next one (64 of B and C in scalar registers, d and d u from
//    LDS), writes the sums of the last one, and calculates.
//    A short call (a few tiles, no chunks) would wait for that kernel longer than it takes itself: its workgroups lay a tile's B
//    and C out in LDS and read them from there, 16 bytes a lane that are the same for all.  LDS has time for that
//    only where the vector ALU has gaps.
//  * A call with too few (sequence, channel block) pairs for the chip cuts its sequences into chunks: a first launch
//    runs each chunk from a state of zero, and each workgroup of the second begins by putting together what the chunks
//    before it leave, since a chunk changes the state it is given by the factor exp(A sum d) alone.
//
// Measured, bf16, 16 states: 16 x 2048 x 4096 in 525 us, 38 clocks for 64 (token, channel, state) of which the five
// instructions above are 25 (20 for the chain of product, exponential, product and multiply-add, 4.7 for another multiply-add;
// by itself exp2 takes 9); 1 x 16384 x 4096 in two passes 184 + 249 us; 4 x 2048 x 4096 gradient 160 + 423 + 16 us.
#pragma once
#include "tokens.h"

namespace dconv {

constexpr int kT = 16;               // tokens of a tile
constexpr int kR = 4;                // states of a wave, at most
constexpr int kStep = 4;             // tokens whose operands are fetched together
constexpr int kMaxStates = 32;       // eight waves

typedef float f8 __attribute__((ext_vector_type(8), aligned(16)));
typedef const __attribute__((address_space(4))) f8* bc_ptr;        // constant memory: scalar loads

// B of kStep tokens, and C where it is needed (WITH_C): pairs of tokens, four states each.
template <bool WITH_C> struct BC {
    f8 vb[kStep / 2], vc[WITH_C ? kStep / 2 : 1];
    // (not one template: a template argument loses the alignment of f8, 16 bytes in the caller's workspace and in LDS)
    __device__ __forceinline__ void load(bc_ptr p)
    {
#pragma unroll
        for (int i = 0; i < kStep / 2; ++i) {
            vb[i] = p[2 * i];
            if (WITH_C) vc[i] = p[2 * i + 1];
        }
    }
    __device__ __forceinline__ void load(const f8* p)
    {
#pragma unroll
        for (int i = 0; i < kStep / 2; ++i) {
            vb[i] = p[2 * i];
            if (WITH_C) vc[i] = p[2 * i + 1];
        }
    }
    __device__ __forceinline__ float b(int k, int r) const { return vb[k / 2][k % 2 * kR + r]; }
    __device__ __forceinline__ float c(int k, int r) const { return vc[k / 2][k % 2 * kR + r]; }
};

struct Rows {                        // a token tensor: base, elements between sequences and tokens
    void* p;
    int64_t n, l;
    template <typename T> __device__ __forceinline__ T* at(int seq, int64_t t, int c) const
    {
        return (T*)p + seq * n + t * l + c;
    }
};

struct ScanParams {
    Rows u, delta, z, out, dout, du, ddelta, dz, B, Cm;
    int64_t b_g, c_g;                // elements between groups of B and C
    const float *A, *D, *delta_bias, *state, *dstate_out;
    float *state_out, *dstate, *starts;
    const int* lengths;
    const float* bc;
    float *ends, *dsum;              // of the chunks: states [N][chunks][blocks][W][64][R], sums of d [N][chunks][blocks][64]
    float *back;                     // ... and of the way back, laid out like ends
    float *cum;                      // sums of d from a chunk's start to each tile's [N][tiles][blocks][64], where starts begin
                                     // every chunk at zero; null where they are the states themselves
    float *part_bc;                  // gradients of B and C: [blocks][N][tiles][2][W][64], see scan_grad.hip
    float *part_A, *part_D, *part_bias;   // [N][chunks][blocks][W][64][R], [N][chunks][blocks][64]
    int N, L, C, S, G, softplus;
    int group, gblocks, blocks;      // channels of a group, its blocks of 64, all blocks
    int tiles, chunk_tiles, chunks;  // of L tokens
    int64_t total;                   // workgroups
};

// What a workgroup works on.
struct ScanPlace {
    int n, chunk, block, g, c0, nc;  // sequence, chunk, channel block; group, first channel, channels of the block
    int len, tile0, tile1, stop;     // the sequence's tokens; the chunk's tiles, those with tokens that count end at stop
};

__device__ __forceinline__ ScanPlace scan_place(const ScanParams& p)
{
    ScanPlace a;
    const unsigned b = blockIdx.x, r = b / (unsigned)p.blocks;
    a.block = b - r * p.blocks;
    a.chunk = r / (unsigned)p.N;
    a.n = r - a.chunk * p.N;
    a.g = a.block / p.gblocks;
    const int k = a.block - a.g * p.gblocks;
    a.c0 = a.g * p.group + k * kWave;
    a.nc = min(kWave, p.group - k * kWave);
    a.len = length_of(p.lengths, a.n, p.L);
    a.tile0 = a.chunk * p.chunk_tiles;
    a.tile1 = min(a.tile0 + p.chunk_tiles, p.tiles);
    a.stop = max(a.tile0, min(a.tile1, (a.len + kT - 1) / kT));
    return a;
}

// ... of a wave and tile; a token takes one f8's worth
__device__ __forceinline__ bc_ptr bc_of(const ScanParams& p, const ScanPlace& a, int tile, int W, int wave)
{
    return (bc_ptr)(p.bc) + ((((int64_t)a.n * p.G + a.g) * p.tiles + tile) * W + wave) * kT;
}

// d of a run of channels, before the tokens that do not count are masked.
template <int E> __device__ __forceinline__ void steps_of(bool soft, const float (&raw)[E], float (&d)[E])
{
#pragma unroll
    for (int i = 0; i < E; ++i) d[i] = raw[i];
    if (!soft) return;
#pragma unroll
    for (int i = 0; i < E; ++i) d[i] = softplus(raw[i]);
}

// A run of E values in LDS, whose rows begin at multiples of 16 bytes.
template <int E> __device__ __forceinline__ Run<float, E> lds_run(const float* p)
{
    return load_run<E>((const float*)__builtin_assume_aligned(p, E >= 4 ? 16 : 4 * E));
}

// Nothing moves past this point: what is written above it is under way before what is written below begins.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// All scalar loads and LDS operations so far are done (s_waitcnt lgkmcnt(0)).  Without it the wait would come at the first use of
// a step's operands, behind the requests for the next step's, and wait for those too.
__device__ __forceinline__ void arrived()
{
    in_order();
    __builtin_amdgcn_s_waitcnt(0xc07f);
    in_order();
}

// All loads from memory so far are done, and stores (s_waitcnt vmcnt(0)).  The next tile's values are waited for where they have been
// under way for most of a tile and before this tile's results are stored: at their first use the wait would be for those stores too.
__device__ __forceinline__ void fetched()
{
    in_order();
    __builtin_amdgcn_s_waitcnt(0x0f70);
    in_order();
}

// A thread's share of the tiles of a token tensor: one token a tile, E channels.  It walks by whole tiles, so that a tile
// costs one 64-bit addition.
template <typename T, int E> struct Share {
    T* p;
    int64_t step;
    __device__ __forceinline__ Share(const Rows& rows, int n, int t, int c) : p(rows.at<T>(n, t, c)), step(rows.l * kT) {}
    // the step in vector registers, where B and C take most of the scalar ones and there are vector ones to spare
    __device__ __forceinline__ void spare() { asm("" : "+v"(step)); }
    __device__ __forceinline__ void forward() { p += step; }
    __device__ __forceinline__ void back() { p -= step; }
    __device__ __forceinline__ auto load(int nv) const { return load_some<E>(p, nv); }
    __device__ __forceinline__ void store(int nv, const float (&v)[E]) const { store_some<E>(p, nv, v); }
};

// Index of this lane's states among those of all channels.
template <int W, int R>
__device__ __forceinline__ int64_t lane_states(const ScanParams& p, const ScanPlace& a, int64_t row, int wave, int lane)
{
    return (((row * p.blocks + a.block) * W + wave) * kWave + lane) * R;
}

// A decay constant whose product with log2 e is finite: exp(0 A) is 1 at tokens that do not count and over chunks that hold none,
// and 0 times an infinity would be NaN.  Steps of more than 5e-37 decay to 0 all the same.  (NaN stays NaN.)
__device__ __forceinline__ float finite_decay(float a) { return a < -2e38f ? -2e38f : a; }

// The states from s0 on of a channel in a user's [C][S], of which those beyond S are 0.
template <int R> __device__ __forceinline__ void load_states(const float* p, int s0, int S, bool ok, float (&v)[R])
{
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = 0.f;
    if (ok) load_some<R>(p + s0, S - s0, v);
}

// ... of the decay constants
template <int R> __device__ __forceinline__ void load_decays(const float* p, int s0, int S, bool ok, float (&v)[R])
{
    load_states(p, s0, S, ok, v);
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = finite_decay(v[r]);
}

// ... in the library's own arrays
template <int R> __device__ __forceinline__ void load_states(const float* p, float (&v)[R])
{
    const Run<float, R> t = load_run<R>((const float*)__builtin_assume_aligned(p, 4 * R));
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = t[r];
}
template <int R> __device__ __forceinline__ void store_states(float* p, const float (&v)[R])
{
    store_some<R>((float*)__builtin_assume_aligned(p, 4 * R), R, v);
}

// host side (scan.hip)
int scan_waves(int S);               // W
int scan_wave_states(int S);         // R
bool scan_sizes_ok(const dconv_scan_args& a);
int scan_check(const dconv_scan_args* a, int form);        // 0 prompt, 1 gradient, 2 step
struct ScanPlan { int waves, states, group, gblocks, blocks, tiles, chunks, chunk_tiles; };
ScanPlan scan_plan(const dconv_scan_args& a, bool grad);
ScanParams scan_params(const dconv_scan_args& a, const ScanPlan& pl);
bool scan_short(const dconv_scan_args& a, const ScanPlan& pl);
int64_t scan_bc_floats(const dconv_scan_args& a, const ScanPlan& pl);
int64_t scan_chunk_floats(const dconv_scan_args& a, const ScanPlan& pl);      // ends and dsum
int64_t scan_starts_floats(const dconv_scan_args& a);
int launch_scan_bc(const dconv_scan_args& a, const ScanPlan& pl, float* bc, hipStream_t st);
int launch_scan_forward(const dconv_scan_args& a, ScanParams p, const ScanPlan& pl, bool out, hipStream_t st);

}  // namespace dconv
