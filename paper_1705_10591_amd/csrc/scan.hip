// The scan over tokens: prompts (scan_kernel.h says how the work is divided).
#include "scan_kernel.h"

namespace dconv {

namespace {

// B and C in fp32 as the scans read them: thread i has token i % 16 of a wave and tile.
template <typename T>
__global__ void __launch_bounds__(kThreads)
bc_kernel(Rows B, Rows C, int64_t b_g, int64_t c_g, const int* lengths, float* bc, int N, int L, int G, int S, int W,
          int R, int tiles)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t unit = i / kT, tile = unit / W, seq = tile / tiles;
    const int s0 = (int)(unit - tile * W) * R, ns = min(R, S - s0);
    const int t = (int)(tile - seq * tiles) * kT + (int)(i - unit * kT), n = (int)(seq / G), g = (int)(seq - (int64_t)n * G);
    if (n >= N) return;
    float b[kR] = {}, c[kR] = {};
    if (t < length_of(lengths, n, L)) {
        load_some<kR>(B.at<const T>(n, t, 0) + g * b_g + s0, ns, b);
        if (C.p) load_some<kR>(C.at<const T>(n, t, 0) + g * c_g + s0, ns, c);
    }
    float* to = bc + (i & ~(int64_t)1) * 8 + (i & 1) * kR;
    store_states(to, b);
    store_states(to + 2 * kR, c);
}

// OUT: the outputs of all tokens, with the states wanted on the way; otherwise the states alone, and with `ends` those of each chunk
// begun at zero (the first at the call's state, which is kept for the second launch in the last chunk's place).
// WHOLE: the block has 64 channels, so that no run of them is cut.
// SHORT: B and C by way of LDS.
template <int W, bool OUT, bool SHORT> struct ScanLds {
    float2 step[kT][kWave];                             // d, d u
    float ysum[OUT ? W : 1][kT][kWave];
    f8 bc[SHORT ? W : 1][kT];                           // as in memory
};

template <typename T, int W, int R, bool OUT, bool SHORT, bool WHOLE>
__device__ __forceinline__ void scan_block(const ScanParams& p, const ScanPlace& a, ScanLds<W, OUT, SHORT>& lds, bool ends)
{
    constexpr int E = kT / W;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = a.c0 + lane, s0 = wave * R;
    const bool ok = WHOLE || lane < a.nc;
    // a thread's share of a tile: one token, E channels
    const int tt = tid / (kWave / E), tc = (tid & (kWave / E - 1)) * E, nv = WHOLE ? E : a.nc - tc, ec = a.c0 + tc;

    float A[R], h[R] = {}, dtotal = 0.f;
    load_decays(p.A + (int64_t)c * p.S, s0, p.S, ok, A);
#pragma unroll
    for (int r = 0; r < R; ++r) A[r] *= kLog2e;
    const int64_t own = ((int64_t)a.n * p.C + c) * p.S;
    const int64_t row = (int64_t)a.n * p.chunks;
    if (ends) {
        if (a.chunk == 0) {
            if (p.state) load_states(p.state + own, s0, p.S, ok, h);
            store_states(p.ends + lane_states<W, R>(p, a, row + p.chunks - 1, wave, lane), h);
        }
    } else if (p.chunks == 1) {
        if (p.state) load_states(p.state + own, s0, p.S, ok, h);
    } else if (a.chunk == 0) {
        load_states(p.ends + lane_states<W, R>(p, a, row + p.chunks - 1, wave, lane), h);
    } else {
        for (int k = 0; k < a.chunk; ++k) {
            float e[R];
            load_states(p.ends + lane_states<W, R>(p, a, row + k, wave, lane), e);
            const float d = p.dsum[((row + k) * p.blocks + a.block) * kWave + lane];
#pragma unroll
            for (int r = 0; r < R; ++r) h[r] = __builtin_fmaf(exp2_(d * A[r]), h[r], e[r]);
        }
    }

    float dbias[E] = {}, skip[E] = {};
    if (nv > 0) {
        if (p.delta_bias) load_some<E>(p.delta_bias + ec, nv, dbias);
        if (OUT && p.D) load_some<E>(p.D + ec, nv, skip);
    }
    const bool gate = OUT && p.z.p;
    int t = a.tile0 * kT + tt;                            // of this thread in the tile at hand
    Share<const T, E> pu(p.u, a.n, t, ec), pd(p.delta, a.n, t, ec), pz(p.z, a.n, t, ec);
    Share<T, E> po(p.out, a.n, t, ec);
    pu.spare(); pd.spare(); pz.spare(); po.spare();
    Run<T, E> u{}, dl{}, z{}, ul{}, zl{};                 // of the tile fetched, the one at hand
    // SHORT: B and C of a token and wave by each of the first 16 W threads
    const int bt = tid / W, bw = tid % W, bs = min(R, p.S - bw * R);
    Run<T, R> rb{}, rc{};
    auto fetch = [&](int at) {
        if constexpr (SHORT) {
            const int tok = at - tt + bt;
            rb = rc = Run<T, R>{};
            if (bt < kT && tok < a.len) {
                rb = load_some<R>(p.B.at<const T>(a.n, tok, bw * R) + a.g * p.b_g, bs);
                if (OUT) rc = load_some<R>(p.Cm.at<const T>(a.n, tok, bw * R) + a.g * p.c_g, bs);
            }
        }
        if (at < a.len && nv > 0) {
            u = pu.load(nv);
            dl = pd.load(nv);
            if (gate) z = pz.load(nv);
        }
        pu.forward(); pd.forward(); pz.forward();
    };
    auto prepare = [&](int tile, int at) {                // the tile fetched, for the loop
        float raw[E], d_[E], u_[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            raw[i] = dl[i] + dbias[i];
            u_[i] = u[i];
        }
        steps_of(p.softplus, raw, d_);
        if ((tile + 1) * kT > a.len) {                    // (a sequence's last tile)
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if (at >= a.len) d_[i] = u_[i] = 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < E; ++i) lds.step[tt][tc + i] = make_float2(d_[i], d_[i] * u_[i]);
        if constexpr (SHORT) {
            if (bt < kT) {
                float* to = (float*)&lds.bc[bw][bt & ~1] + (bt & 1) * kR;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    to[r] = rb[r];
                    if (OUT) to[2 * kR + r] = rc[r];
                }
            }
        }
    };
    auto finish = [&](int tile, int at) {                 // the tile at hand: sums over waves, gate
        if (nv > 0 && at < p.L) {
            float y[E];
#pragma unroll
            for (int i = 0; i < E; ++i) y[i] = skip[i] * ul[i];
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const Run<float, E> part = lds_run<E>(&lds.ysum[w][tt][tc]);
#pragma unroll
                for (int i = 0; i < E; ++i) y[i] += part[i];
            }
            if (gate) {
#pragma unroll
                for (int i = 0; i < E; ++i) y[i] *= zl[i] * sigmoid(zl[i]);
            }
            if ((tile + 1) * kT > a.len) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    if (at >= a.len) y[i] = 0.f;
                }
            }
            po.store(nv, y);
        }
        po.forward();
    };
    BC<OUT> bc, next;
    if (a.tile0 < a.stop) {
        fetch(t);
        if (!SHORT) bc.load(bc_of(p, a, a.tile0, W, wave));
    }
    for (int tile = a.tile0; tile < a.stop; ++tile, t += kT) {
        const auto& step = lds.step;
        auto& ysum = lds.ysum;
        prepare(tile, t);
        ul = u; zl = z;
        if (tile + 1 < a.stop) fetch(t + kT);
        meet();
        if (p.starts && !ends) store_states(p.starts + lane_states<W, R>(p, a, (int64_t)a.n * p.tiles + tile, wave, lane), h);
        float2 d[kStep], dn[kStep];
        float ys[kStep];
#pragma unroll
        for (int k = 0; k < kStep; ++k) d[k] = step[k][lane];
        const bc_ptr here = SHORT ? nullptr : bc_of(p, a, tile, W, wave);
        const bc_ptr after = SHORT ? nullptr : bc_of(p, a, min(tile + 1, a.stop - 1), W, wave);
        if (SHORT) bc.load(&lds.bc[wave][0]);
#pragma unroll
        for (int k0 = 0; k0 < kT; k0 += kStep) {
            const bool more = k0 + kStep < kT;
            arrived();
            if (!SHORT) next.load(more ? here + k0 + kStep : after);
            else if (more) next.load(&lds.bc[wave][k0 + kStep]);
#pragma unroll
            for (int k = 0; k < kStep; ++k) {
                if (more) dn[k] = step[k0 + kStep + k][lane];
                if (OUT && k0) ysum[wave][k0 - kStep + k][lane] = ys[k];
            }
            in_order();
#pragma unroll
            for (int k = 0; k < kStep; ++k) {
                float y = 0.f;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    h[r] = __builtin_fmaf(exp2_(d[k].x * A[r]), h[r], d[k].y * bc.b(k, r));
                    if (OUT) y = r ? __builtin_fmaf(bc.c(k, r), h[r], y) : bc.c(k, r) * h[r];
                }
                if (OUT) ys[k] = y;
                else dtotal += d[k].x;
            }
            in_order();
            bc = next;
#pragma unroll
            for (int k = 0; k < kStep; ++k) d[k] = dn[k];
        }
        if (OUT) {
#pragma unroll
            for (int k = 0; k < kStep; ++k) ysum[wave][kT - kStep + k][lane] = ys[k];
        }
        fetched();
        meet();
        if (OUT) finish(tile, t);
    }
    if (OUT && nv > 0) {
        const float zero[E] = {};
        for (int tile = a.stop; tile < a.tile1; ++tile, t += kT, po.forward())       // tiles that do not count
            if (t < p.L) po.store(nv, zero);
    }
    if (ends) {
        store_states(p.ends + lane_states<W, R>(p, a, row + a.chunk, wave, lane), h);
        if (wave == 0) p.dsum[((row + a.chunk) * p.blocks + a.block) * kWave + lane] = dtotal;
    } else if (p.state_out && a.chunk == p.chunks - 1 && ok) {
        store_some<R>(p.state_out + own + s0, p.S - s0, h);
    }
}

template <typename T, int W, int R, bool OUT, bool SHORT>
__global__ void __launch_bounds__(kWave * W)
scan_kernel(ScanParams p, bool ends)
{
    __shared__ ScanLds<W, OUT, SHORT> lds;
    const ScanPlace a = scan_place(p);
    if (a.nc == kWave) scan_block<T, W, R, OUT, SHORT, true>(p, a, lds, ends);
    else scan_block<T, W, R, OUT, SHORT, false>(p, a, lds, ends);
}

template <typename T, int W, int R>
void launch_kernel(const ScanParams& p, bool out, bool ends, int64_t blocks, hipStream_t st)
{
    const dim3 grid((unsigned)blocks), threads(kWave * W);
    if (!p.bc) hipLaunchKernelGGL((scan_kernel<T, W, R, true, true>), grid, threads, 0, st, p, false);
    else if (out) hipLaunchKernelGGL((scan_kernel<T, W, R, true, false>), grid, threads, 0, st, p, false);
    else hipLaunchKernelGGL((scan_kernel<T, W, R, false, false>), grid, threads, 0, st, p, ends);
}

template <typename T>
void launch_states(const ScanParams& p, bool out, bool ends, int64_t blocks, hipStream_t st)
{
    if (p.S <= 4) launch_kernel<T, 4, 1>(p, out, ends, blocks, st);
    else if (p.S <= 8) launch_kernel<T, 4, 2>(p, out, ends, blocks, st);
    else if (p.S <= 16) launch_kernel<T, 4, 4>(p, out, ends, blocks, st);
    else launch_kernel<T, 8, 4>(p, out, ends, blocks, st);
}

void launch_typed(const ScanParams& p, int dtype, bool out, bool ends, int64_t blocks, hipStream_t st)
{
    switch (dtype) {
    case DCONV_DTYPE_F16: return launch_states<_Float16>(p, out, ends, blocks, st);
    case DCONV_DTYPE_BF16: return launch_states<__bf16>(p, out, ends, blocks, st);
    default: return launch_states<float>(p, out, ends, blocks, st);
    }
}

Rows rows_of(const dconv_tokens& t) { return Rows{t.p, t.sn, t.sl}; }

}  // namespace

int scan_waves(int S) { return S <= 16 ? 4 : 8; }
int scan_wave_states(int S) { return S <= 4 ? 1 : S <= 8 ? 2 : 4; }

bool scan_sizes_ok(const dconv_scan_args& a)
{
    if (!(a.N > 0 && a.L > 0 && a.L <= kMaxTokens && a.C > 0 && a.C <= kMaxChannels && a.S > 0 && a.S <= kMaxStates && a.G > 0 && a.C % a.G == 0))
        return false;
    // (sizes in floating point, so that no product overflows)
    if ((double)a.N * a.L * a.C * kMaxStates >= kMaxElements) return false;
    const ScanPlan pl = scan_plan(a, false);             // (where a gradient has more chunks there are few blocks)
    // (threads of the largest grids: the scans', bc_kernel's, the sums')
    const double bc = (double)a.N * a.G * pl.tiles * pl.waves;
    const double most = (double)kMaxThreads - kThreads;
    return (double)a.N * pl.blocks * pl.chunks * pl.waves * kWave <= most && bc * kT <= most &&
           bc * (kT / 8 * kWave) + pl.blocks * (kMaxStates + 2.0) * kThreads <= most;
}

ScanPlan scan_plan(const dconv_scan_args& a, bool grad)
{
    ScanPlan pl;
    pl.waves = scan_waves(a.S);
    pl.states = scan_wave_states(a.S);
    pl.group = a.C / a.G;
    pl.gblocks = (pl.group - 1) / kWave + 1;
    pl.blocks = a.G * pl.gblocks;
    pl.tiles = (a.L + kT - 1) / kT;
    // Chunks cost another launch that does most of the work again, so there are none where the channels alone give the
    // chip one and a half waves a SIMD (two in gradients, whose registers let no more be there at a time, and with up to four states,
    // where most of the work is the channels'), nor for a few tiles.  Otherwise as many as give it eight (six with up to four
    // states, of which six are there at a time in 16 bits and five in fp32; gradients four, and four chunks at least) in chunks of four
    // tiles or more, or half of that in chunks of two.  Measured in bf16 with 16 states, us for 1 chunk and for the rule's (sequences x
    // tokens x channels; in brackets what the rule leaves in one):
    //   scan      1 x 256 x 2048   32, 20   1 x 4096 x 4096   422, 132   3 x 2048 x 4096  216, 171   8 x 2048 x 4096   306, (387)
    //   4 states  6 x 512 x 4096    61, 50   6 x 2048 x 4096   228, 168, in fp32 267, 258            7 x 1024 x 4096   120, 107
    //   gradient  1 x 256 x 2048  101, 35   1 x 4096 x 4096  1408, 318   4 x 2048 x 4096  753, 604   8 x 2048 x 4096  1132, (1152)
    // Few channels make many chunks, and each workgroup joins all those before its own, one memory round trip at a time:
    //   scan      1 x 16384 x 64   1681, 163 (512 chunks)   1 x 16384 x 256  1684, 108   1 x 131072 x 64   13396, 667 (2048 chunks)
    //   gradient  1 x 16384 x 64   5587, 203                1 x 16384 x 256  5580, 248   1 x 131072 x 64   44754, 799
    // No more chunks than the square root of twice the tiles would take 85, 90, 234 and 166, 172, 458 there, but 67 instead of 47 for
    // the gradient of 1 x 2048 x 128.
    const double alone = (double)a.N * pl.blocks * pl.waves;
    pl.chunks = 1;
    if (alone < (grad || a.S <= 4 ? 2048 : 1536) && pl.tiles >= (grad ? 6 : 10)) {
        int most = (int)((grad ? 4096 : a.S <= 4 ? 6144 : 8192) / alone);
        if (grad && most < 4) most = 4;
        const int longer = most < pl.tiles / 4 ? most : pl.tiles / 4, shorter = most / 2 < pl.tiles / 2 ? most / 2 : pl.tiles / 2;
        pl.chunks = longer > shorter ? longer : shorter;
        if (pl.chunks < 2) pl.chunks = 1;
    }
    pl.chunk_tiles = (pl.tiles + pl.chunks - 1) / pl.chunks;
    pl.chunks = (pl.tiles + pl.chunk_tiles - 1) / pl.chunk_tiles;
    return pl;
}

// Short calls: up to six tiles where the chip has at most two waves a SIMD.  Measured, us a call without and with
// (sequences x tokens x channels, 16 states, bf16): 1 x 16 x 2048 16.5, 12.0; 1 x 64 x 2048 16.7, 12.0; 8 x 64 x 4096 17.6, 15.5;
// 32 x 64 x 4096 40.4, 43.3; 8 x 256 x 4096 43.6, 45.2; 8 x 1024 x 4096 152, 167.
bool scan_short(const dconv_scan_args& a, const ScanPlan& pl)
{
    return a.out.p && pl.chunks == 1 && pl.tiles <= 6 && (double)a.N * pl.blocks * pl.waves <= 2048;
}

int64_t scan_bc_floats(const dconv_scan_args& a, const ScanPlan& pl)
{
    return (int64_t)a.N * a.G * pl.tiles * kT * pl.waves * 2 * kR;
}

int64_t scan_chunk_floats(const dconv_scan_args& a, const ScanPlan& pl)
{
    return pl.chunks > 1 ? (int64_t)a.N * pl.chunks * pl.blocks * kWave * (pl.waves * pl.states + 1) : 0;
}

int64_t scan_starts_floats(const dconv_scan_args& a)
{
    const ScanPlan pl = scan_plan(a, false);
    return (int64_t)a.N * pl.tiles * pl.blocks * pl.waves * kWave * pl.states;
}

ScanParams scan_params(const dconv_scan_args& a, const ScanPlan& pl)
{
    ScanParams p{};
    p.u = rows_of(a.u); p.delta = rows_of(a.delta); p.z = rows_of(a.z); p.out = rows_of(a.out);
    p.dout = rows_of(a.dout); p.du = rows_of(a.du); p.ddelta = rows_of(a.ddelta); p.dz = rows_of(a.dz);
    p.A = a.A; p.D = a.D; p.delta_bias = a.delta_bias; p.state = a.state; p.dstate_out = a.dstate_out;
    p.state_out = a.state_out; p.dstate = a.dstate; p.starts = (float*)a.starts;
    p.B = rows_of(a.B); p.Cm = rows_of(a.Cm); p.b_g = a.B.sg; p.c_g = a.Cm.sg;
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
                           a.N, a.L, a.G, a.S, pl.waves, pl.states, pl.tiles);
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
        launch_typed(p, a.dtype, false, true, p.total - (int64_t)a.N * pl.blocks, st);
    launch_typed(p, a.dtype, out, false, p.total, st);
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
                          (const void*)a->dD, (const void*)a->ddelta_bias, (const void*)a->lengths,
                          (const void*)a->slots})
        if (!aligned_to(q, 4)) return DCONV_BAD_SHAPE;
    if (!step && !aligned_to(a->starts, 16)) return DCONV_BAD_SHAPE;
    const long long need = step ? 0 : dconv_scan_workspace(a, grad);
    if (need) {
        if (!a->workspace) return DCONV_NULL_POINTER;
        if (!aligned_to(a->workspace, 16)) return DCONV_BAD_SHAPE;
        if (a->workspace_bytes < need) return DCONV_SCRATCH_EXCEEDED;
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
    if (scan_short(*a, pl)) return launch_scan_forward(*a, p, pl, true, (hipStream_t)stream);
    p.bc = ws;
    p.ends = ws + scan_bc_floats(*a, pl);
    p.dsum = p.ends + (int64_t)a->N * pl.chunks * pl.blocks * pl.waves * kWave * pl.states;
    const int rb = launch_scan_bc(*a, pl, ws, (hipStream_t)stream);
    return rb != DCONV_OK ? rb : launch_scan_forward(*a, p, pl, a->out.p != nullptr, (hipStream_t)stream);
}

}  // extern "C"
