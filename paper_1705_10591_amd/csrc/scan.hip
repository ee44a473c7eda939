// The scan over tokens: prompts (scan_kernel.h says how the work is divided).
#include "scan_kernel.h"

namespace dconv {

namespace {

// B and C of a token and wave, side by side in fp32: thread i has the i-th eight of the layout.
template <typename T>
__global__ void __launch_bounds__(kThreads)
bc_kernel(Rows B, Rows C, int64_t b_g, int64_t c_g, const int* lengths, float* bc, int N, int L, int G, int S, int W,
          int tiles)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t unit = i / kT, tile = unit / W, seq = tile / tiles;
    const int s0 = (int)(unit - tile * W) * kR;
    const int t = (int)(tile - seq * tiles) * kT + (int)(i - unit * kT), n = (int)(seq / G), g = (int)(seq - (int64_t)n * G);
    if (n >= N) return;
    float b[kR] = {}, c[kR] = {};
    if (t < length_of(lengths, n, L)) {
        load_some<kR>(B.at<const T>(n, t, 0) + g * b_g + s0, S - s0, b);
        if (C.p) load_some<kR>(C.at<const T>(n, t, 0) + g * c_g + s0, S - s0, c);
    }
    store_states(bc + i * 8, b);
    store_states(bc + i * 8 + kR, c);
}

// OUT: the outputs of all tokens, with the states wanted on the way; otherwise the states alone, and with `ends` those of each chunk
// begun at zero (the first at the call's state, which is kept for the second launch in the last chunk's place).
// WHOLE: the block has 64 channels, so that no run of them is cut.
template <int W, bool OUT> struct ScanLds {
    float2 step[kT][kWave];                             // d, d u
    float ysum[OUT ? W : 1][kT][kWave];
};

template <typename T, int W, bool OUT, bool WHOLE>
__device__ __forceinline__ void scan_block(const ScanParams& p, const ScanPlace& a, ScanLds<W, OUT>& lds, bool ends)
{
    constexpr int E = kT / W;
    auto& step = lds.step;
    auto& ysum = lds.ysum;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = a.c0 + lane, s0 = wave * kR;
    const bool ok = WHOLE || lane < a.nc;
    // a thread's share of a tile: one token, E channels
    const int tt = tid / (kWave / E), tc = (tid & (kWave / E - 1)) * E, nv = WHOLE ? E : a.nc - tc, ec = a.c0 + tc;

    float A[kR], h[kR] = {}, dtotal = 0.f;
    load_states(p.A + (int64_t)c * p.S, s0, p.S, ok, A);
#pragma unroll
    for (int r = 0; r < kR; ++r) A[r] *= kLog2e;
    const int64_t own = ((int64_t)a.n * p.C + c) * p.S;
    const int64_t row = (int64_t)a.n * p.chunks;
    if (ends) {
        if (a.chunk == 0) {
            if (p.state) load_states(p.state + own, s0, p.S, ok, h);
            store_states(p.ends + lane_states(p, a, row + p.chunks - 1, W, wave, lane), h);
        }
    } else if (p.chunks == 1) {
        if (p.state) load_states(p.state + own, s0, p.S, ok, h);
    } else if (a.chunk == 0) {
        load_states(p.ends + lane_states(p, a, row + p.chunks - 1, W, wave, lane), h);
    } else {
        for (int k = 0; k < a.chunk; ++k) {
            float e[kR];
            load_states(p.ends + lane_states(p, a, row + k, W, wave, lane), e);
            const float d = p.dsum[((row + k) * p.blocks + a.block) * kWave + lane];
#pragma unroll
            for (int r = 0; r < kR; ++r) h[r] = __builtin_fmaf(exp2_(d * A[r]), h[r], e[r]);
        }
    }

    float dbias[E] = {}, skip[E] = {};
    if (nv > 0) {
        if (p.delta_bias) load_some<E>(p.delta_bias + ec, nv, dbias);
        if (OUT && p.D) load_some<E>(p.D + ec, nv, skip);
    }
    const bool gate = OUT && p.z.p;
    int t = a.tile0 * kT + tt;
    Share<const T, E> pu(p.u, a.n, t, ec), pd(p.delta, a.n, t, ec), pz(p.z, a.n, t, ec);
    Share<T, E> po(p.out, a.n, t, ec);
    Run<T, E> u{}, dl{}, z{};
    auto fetch = [&](int at) {
        if (at < a.len && nv > 0) {
            u = pu.load(nv);
            dl = pd.load(nv);
            if (gate) z = pz.load(nv);
        }
        pu.forward(); pd.forward(); pz.forward();
    };
    if (a.tile0 < a.stop) fetch(t);
    BC bc, next;
    if (a.tile0 < a.stop) bc.load(bc_of(p, a, a.tile0, W, wave));
    for (int tile = a.tile0; tile < a.stop; ++tile, t += kT, po.forward()) {
        float raw[E], d_[E], u_[E];
        const Run<T, E> zc = z;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            raw[i] = dl[i] + dbias[i];
            u_[i] = u[i];
        }
        steps_of(p.softplus, raw, d_);
        if ((tile + 1) * kT > a.len) {                    // (a sequence's last tile)
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if (t >= a.len) d_[i] = u_[i] = 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < E; ++i) step[tt][tc + i] = make_float2(d_[i], d_[i] * u_[i]);
        if (tile + 1 < a.stop) fetch(t + kT);
        meet();
        if (p.starts && !ends) store_states(p.starts + lane_states(p, a, (int64_t)a.n * p.tiles + tile, W, wave, lane), h);
        float2 d[kStep], dn[kStep];
#pragma unroll
        for (int k = 0; k < kStep; ++k) d[k] = step[k][lane];
        const bc_ptr here = bc_of(p, a, tile, W, wave), after = bc_of(p, a, min(tile + 1, a.stop - 1), W, wave);
#pragma unroll
        for (int k0 = 0; k0 < kT; k0 += kStep) {
            const bool more = k0 + kStep < kT;
            next.load(more ? here + (k0 + kStep) / 2 : after);
#pragma unroll
            for (int k = 0; k < kStep; ++k)
                if (more) dn[k] = step[k0 + kStep + k][lane];
            in_order();
#pragma unroll
            for (int k = 0; k < kStep; ++k) {
                float y = 0.f;
#pragma unroll
                for (int r = 0; r < kR; ++r) {
                    h[r] = __builtin_fmaf(exp2_(d[k].x * A[r]), h[r], d[k].y * bc.b(k, r));
                    if (OUT) y = r ? __builtin_fmaf(bc.c(k, r), h[r], y) : bc.c(k, r) * h[r];
                }
                if (OUT) ysum[wave][k0 + k][lane] = y;
                else dtotal += d[k].x;
            }
            in_order();
            bc = next;
#pragma unroll
            for (int k = 0; k < kStep; ++k) d[k] = dn[k];
        }
        meet();
        if (OUT && nv > 0 && t < p.L) {
            float y[E];
#pragma unroll
            for (int i = 0; i < E; ++i) {
                y[i] = skip[i] * u_[i];
#pragma unroll
                for (int w = 0; w < W; ++w) y[i] += ysum[w][tt][tc + i];
                if (gate) y[i] *= zc[i] * sigmoid(zc[i]);
            }
            if (t >= a.len) {
#pragma unroll
                for (int i = 0; i < E; ++i) y[i] = 0.f;
            }
            po.store(nv, y);
        }
    }
    if (OUT && nv > 0) {
        const float zero[E] = {};
        for (int tile = a.stop; tile < a.tile1; ++tile, t += kT, po.forward())       // tiles that do not count
            if (t < p.L) po.store(nv, zero);
    }
    if (ends) {
        store_states(p.ends + lane_states(p, a, row + a.chunk, W, wave, lane), h);
        if (wave == 0) p.dsum[((row + a.chunk) * p.blocks + a.block) * kWave + lane] = dtotal;
    } else if (p.state_out && a.chunk == p.chunks - 1 && ok) {
        store_some<kR>(p.state_out + own + s0, p.S - s0, h);
    }
}

template <typename T, int W, bool OUT>
__global__ void __launch_bounds__(kWave * W)
scan_kernel(ScanParams p, bool ends)
{
    __shared__ ScanLds<W, OUT> lds;
    const ScanPlace a = scan_place(p);
    if (a.nc == kWave) scan_block<T, W, OUT, true>(p, a, lds, ends);
    else scan_block<T, W, OUT, false>(p, a, lds, ends);
}

template <typename T, int W>
void launch_kernel(const ScanParams& p, bool out, bool ends, int64_t blocks, hipStream_t st)
{
    if (out)
        hipLaunchKernelGGL((scan_kernel<T, W, true>), dim3((unsigned)blocks), dim3(kWave * W), 0, st, p, false);
    else
        hipLaunchKernelGGL((scan_kernel<T, W, false>), dim3((unsigned)blocks), dim3(kWave * W), 0, st, p, ends);
}

template <typename T>
void launch_waves(const ScanParams& p, int W, bool out, bool ends, int64_t blocks, hipStream_t st)
{
    switch (W) {
    case 1: return launch_kernel<T, 1>(p, out, ends, blocks, st);
    case 2: return launch_kernel<T, 2>(p, out, ends, blocks, st);
    case 4: return launch_kernel<T, 4>(p, out, ends, blocks, st);
    default: return launch_kernel<T, 8>(p, out, ends, blocks, st);
    }
}

void launch_typed(const ScanParams& p, int dtype, int W, bool out, bool ends, int64_t blocks, hipStream_t st)
{
    switch (dtype) {
    case DCONV_DTYPE_F16: return launch_waves<_Float16>(p, W, out, ends, blocks, st);
    case DCONV_DTYPE_BF16: return launch_waves<__bf16>(p, W, out, ends, blocks, st);
    default: return launch_waves<float>(p, W, out, ends, blocks, st);
    }
}

Rows rows_of(const dconv_tokens& t) { return Rows{t.p, t.sn, t.sl}; }

}  // namespace

int scan_waves(int S) { return S <= 4 ? 1 : S <= 8 ? 2 : S <= 16 ? 4 : 8; }

bool scan_sizes_ok(const dconv_scan_args& a)
{
    if (!(a.N > 0 && a.L > 0 && a.L <= kMaxTokens && a.C > 0 && a.S > 0 && a.S <= kMaxStates && a.G > 0 && a.C % a.G == 0))
        return false;
    // (sizes in floating point, so that no product overflows)
    if ((double)a.N * a.L * a.C * kMaxStates >= kMaxElements) return false;
    const ScanPlan pl = scan_plan(a, false);             // (a gradient has no more chunks)
    return (double)a.N * pl.blocks * pl.chunks <= 2147483647.0 &&
           (double)a.N * a.G * pl.tiles * kT * pl.waves <= 2147483647.0 * kThreads;
}

ScanPlan scan_plan(const dconv_scan_args& a, bool grad)
{
    ScanPlan pl;
    pl.waves = scan_waves(a.S);
    pl.group = a.C / a.G;
    pl.gblocks = (pl.group - 1) / kWave + 1;
    pl.blocks = a.G * pl.gblocks;
    pl.tiles = (a.L + kT - 1) / kT;
    // Chunks cost another launch that does most of the work again, so there are none where the channels alone give the
    // chip nearly two waves a SIMD, nor for a few tiles.  Otherwise as many as give it eight (gradients, whose registers let two
    // be there at a time: four) in chunks of four tiles or more, or half of that in chunks of two.  Measured, S = 16,
    // us for 1 chunk and those of the rule (sequences x tokens x channels):
    //   scan      1 x 256 x 2048  41, 26    1 x 4096 x 4096   531, 131    4 x 2048 x 4096  274, 224    8 x 2048 x 4096   352, (407)
    //   gradient  1 x 256 x 2048 134, 75    1 x 4096 x 4096  1463, 449    4 x 2048 x 4096  928, 799    8 x 2048 x 4096  1261, (1402)
    const double alone = (double)a.N * pl.blocks * pl.waves;
    pl.chunks = 1;
    if (alone < 1792 && pl.tiles >= 6) {
        const int most = grad ? (int)(4096 / alone) : (int)(8192 / alone);
        const int longer = most < pl.tiles / 4 ? most : pl.tiles / 4, shorter = most / 2 < pl.tiles / 2 ? most / 2 : pl.tiles / 2;
        pl.chunks = longer > shorter ? longer : shorter;
        if (pl.chunks < 2) pl.chunks = 1;
    }
    pl.chunk_tiles = (pl.tiles + pl.chunks - 1) / pl.chunks;
    pl.chunks = (pl.tiles + pl.chunk_tiles - 1) / pl.chunk_tiles;
    return pl;
}

int64_t scan_bc_floats(const dconv_scan_args& a, const ScanPlan& pl)
{
    return (int64_t)a.N * a.G * pl.tiles * kT * pl.waves * 2 * kR;
}

int64_t scan_chunk_floats(const dconv_scan_args& a, const ScanPlan& pl)
{
    return pl.chunks > 1 ? (int64_t)a.N * pl.chunks * pl.blocks * kWave * (pl.waves * kR + 1) : 0;
}

int64_t scan_starts_floats(const dconv_scan_args& a)
{
    const ScanPlan pl = scan_plan(a, false);
    return (int64_t)a.N * pl.tiles * pl.blocks * pl.waves * kWave * kR;
}

ScanParams scan_params(const dconv_scan_args& a, const ScanPlan& pl)
{
    ScanParams p{};
    p.u = rows_of(a.u); p.delta = rows_of(a.delta); p.z = rows_of(a.z); p.out = rows_of(a.out);
    p.dout = rows_of(a.dout); p.du = rows_of(a.du); p.ddelta = rows_of(a.ddelta); p.dz = rows_of(a.dz);
    p.A = a.A; p.D = a.D; p.delta_bias = a.delta_bias; p.state = a.state; p.dstate_out = a.dstate_out;
    p.state_out = a.state_out; p.dstate = a.dstate; p.starts = (float*)a.starts;
    p.lengths = a.lengths;
    p.N = a.N; p.L = a.L; p.C = a.C; p.S = a.S; p.G = a.G; p.softplus = a.softplus;
    p.group = pl.group; p.gblocks = pl.gblocks; p.blocks = pl.blocks;
    p.tiles = pl.tiles; p.chunk_tiles = pl.chunk_tiles; p.chunks = pl.chunks;
    p.total = (int64_t)a.N * pl.blocks * pl.chunks;
    return p;
}

int launch_scan_bc(const dconv_scan_args& a, const ScanPlan& pl, float* bc, hipStream_t st)
{
    const int64_t n = (int64_t)a.N * a.G * pl.tiles * kT * pl.waves;
    const dim3 grid((unsigned)((n + kThreads - 1) / kThreads));
    begin_launch();
    auto go = [&](auto* kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, rows_of(a.B), rows_of(a.Cm), a.B.sg, a.Cm.sg, a.lengths, bc,
                           a.N, a.L, a.G, a.S, pl.waves, pl.tiles);
    };
    if (a.dtype == DCONV_DTYPE_F16) go(&bc_kernel<_Float16>);
    else if (a.dtype == DCONV_DTYPE_BF16) go(&bc_kernel<__bf16>);
    else go(&bc_kernel<float>);
    return launch_status();
}

int launch_scan_forward(const dconv_scan_args& a, ScanParams p, const ScanPlan& pl, bool out, hipStream_t st)
{
    begin_launch();
    if (pl.chunks > 1)                                        // (the last chunk's end is nobody's start)
        launch_typed(p, a.dtype, pl.waves, false, true, p.total - (int64_t)a.N * pl.blocks, st);
    launch_typed(p, a.dtype, pl.waves, out, false, p.total, st);
    return launch_status();
}

int scan_check(const dconv_scan_args* a, int form)
{
    if (!a) return DCONV_NULL_POINTER;
    const int e = token_bytes(a->dtype);
    if (!e) return DCONV_UNSUPPORTED;
    if (!scan_sizes_ok(*a)) return DCONV_BAD_SHAPE;
    const bool grad = form == 1, step = form == 2;
    if (step && (a->L != 1 || a->M <= 0 || (!a->slots && a->M < a->N))) return DCONV_BAD_SHAPE;
    if (!a->u.p || !a->delta.p || !a->B.p || !a->A) return DCONV_NULL_POINTER;
    if (form == 0) {
        if (a->out.p ? !a->Cm.p : (!a->starts && !a->state_out)) return DCONV_NULL_POINTER;
    } else if (step) {
        if (!a->out.p || !a->Cm.p || !a->state_out) return DCONV_NULL_POINTER;
    } else if (!a->Cm.p || !a->dout.p || !a->du.p || !a->ddelta.p || !a->dB.p || !a->dC.p || !a->dA ||
               (a->z.p && !a->dz.p)) {
        return DCONV_NULL_POINTER;
    }
    for (const dconv_tokens* t : {&a->u, &a->delta, &a->z, &a->out, &a->B, &a->Cm, &a->dout, &a->du, &a->ddelta, &a->dz,
                                  &a->dB, &a->dC})
        if (!aligned_to(t->p, e)) return DCONV_BAD_SHAPE;
    for (const void* q : {(const void*)a->A, (const void*)a->D, (const void*)a->delta_bias, (const void*)a->state,
                          (const void*)a->state_out, (const void*)a->dstate_out, (const void*)a->dstate, (const void*)a->dA,
                          (const void*)a->dD, (const void*)a->ddelta_bias, (const void*)a->starts, (const void*)a->lengths,
                          (const void*)a->slots})
        if (!aligned_to(q, 4)) return DCONV_BAD_SHAPE;
    if (!step) {
        if (!a->workspace) return DCONV_NULL_POINTER;
        if (!aligned_to(a->workspace, 16)) return DCONV_BAD_SHAPE;
        if (a->workspace_bytes < dconv_scan_workspace(a, grad)) return DCONV_SCRATCH_EXCEEDED;
    }
    return DCONV_OK;
}

}  // namespace dconv

using namespace dconv;

extern "C" {

long long dconv_scan_starts(const dconv_scan_args* a)
{
    return a && token_bytes(a->dtype) && scan_sizes_ok(*a) ? 4 * scan_starts_floats(*a) : -1;
}

int dconv_scan(const dconv_scan_args* a, void* stream)
{
    const int rc = scan_check(a, 0);
    if (rc != DCONV_OK) return rc;
    const ScanPlan pl = scan_plan(*a, false);
    ScanParams p = scan_params(*a, pl);
    float* ws = (float*)a->workspace;
    p.bc = ws;
    p.ends = ws + scan_bc_floats(*a, pl);
    p.dsum = p.ends + (int64_t)a->N * pl.chunks * pl.blocks * pl.waves * kWave * kR;
    const int rb = launch_scan_bc(*a, pl, ws, (hipStream_t)stream);
    return rb != DCONV_OK ? rb : launch_scan_forward(*a, p, pl, a->out.p != nullptr, (hipStream_t)stream);
}

}  // extern "C"
