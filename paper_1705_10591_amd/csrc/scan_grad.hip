// Gradients of the scan over tokens (scan_kernel.h says how the work is divided).
//
// With dy = dout z sigmoid(z), a = exp(d A) and g[t] the gradient of h[t]:
//   g[t]  = C[t] dy[t] + a[t+1] g[t+1]
//   dC[t] = sum_c dy h[t],  dB[t] = sum_c g d u,  q = sum_s g B,  e = g a h[t-1]
//   du = d q + D dy,  d(delta) = (sum_s e A + u q) sigmoid(delta + bias),  dA = sum_t e d,  dz = dout y (z sigmoid(z))'
// States are needed in the order opposite to the one they are made in: they are kept at the start of every tile
// (`starts`), and a tile of 16 tokens makes its own again in registers, 4 decays and 4 states a token and lane, before it
// walks back.  About 20 vector instructions for each (token, channel, state) bound the call, not its memory.
// A call in chunks that is not given starts makes all that they need in one pass (sweep_kernel): the states of each tile
// as if its chunk began at zero, what the chunk leaves, and what it would leave going back, which is a sum over tokens of
// C dy times the decays from the chunk's start, products that the pass can carry along.
//
// dB and dC are sums over channels, that is over lanes: 2 x 4 values a token.  Adding each over 64 lanes would take
// more instructions than all the rest (6 each).  Pairs of values are added over half of the lanes instead, one value left in
// either half (two instructions a pair with the swaps of 32 and 16 lanes), so that the number of values halves with the
// lanes they still have to be added over: 2.2 instructions a value, and at the end lane l of a wave has the sum of
// value l of 64 (B and C of 8 tokens and 4 states, say).  Channel blocks meet in a second kernel, in the same order on every call.
//
// The sums over all tokens (dA, dD and that of the bias) are in 32 bits over what a thread has of a chunk, dA by tiles, and in 64 bits from
// there on.  Off by, of their norms, 4 x 2048 x 4096 and 16 x 2048 x 128: dA 4.5e-7 and 2.6e-7 (all in 32 bits 6.0e-7, 3.7e-7), dD 1.2e-7
// and 6.2e-8 (1.5e-7, 2.1e-7), the bias' 2.6e-7 and 1.9e-7 (2.8e-7, 3.3e-7), at the same speed.
#include "scan_kernel.h"

namespace dconv {

namespace {

__device__ __forceinline__ unsigned bits(float v) { return __builtin_bit_cast(unsigned, v); }
__device__ __forceinline__ float value(unsigned v) { return __builtin_bit_cast(float, v); }

// lanes 0..31: a over lanes l, l + 32; lanes 32..63: b
__device__ __forceinline__ float fold32(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(bits(a), bits(b), false, false);
    return value(r[0]) + value(r[1]);
}

// lanes with bit 4 clear: a over l, l + 16; set: b
__device__ __forceinline__ float fold16(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(bits(a), bits(b), false, false);
    return value(r[0]) + value(r[1]);
}

// lanes with bit BIT clear: a over this lane and its partner by CTRL, whose bit is the other one; set: b.  The mask of those
// lanes is a constant: one that is compared for would take a pair of scalar registers.
template <int CTRL, int BIT> __device__ __forceinline__ float fold(float a, float b)
{
    constexpr uint64_t kUpper = BIT == 8 ? 0xff00ff00ff00ff00ull : BIT == 4 ? 0xf0f0f0f0f0f0f0f0ull : BIT == 2 ? 0xccccccccccccccccull
                                                                                                              : 0xaaaaaaaaaaaaaaaaull;
    const bool upper = __builtin_amdgcn_inverse_ballot_w64(kUpper);
    const float keep = upper ? b : a, give = upper ? a : b;
    return keep + value(__builtin_amdgcn_update_dpp(0, bits(give), CTRL, 0xf, 0xf, true));
}

// Tokens whose sums over lanes make a register: 64 values of 4 states, 64 of 2, 32 of 1 (twice each).
__host__ __device__ constexpr int gathered(int R) { return R == 4 ? 8 : 16; }

constexpr int kAcross8 = 0x128, kAcross4 = 0x141, kAcross2 = 0x4e, kAcross1 = 0xb1;   // lane bits 3, 2, 1, 0

// What each chunk but the first leaves of g at its start, begun at zero (the last: at the gradient of the call's last
// state), and its sum of d.
template <typename T, int W, int R, bool WHOLE>
__device__ __forceinline__ void back_block(const ScanParams& p, const ScanPlace& a, float2 (&step)[kT][kWave])   // d, dy
{
    constexpr int E = kT / W;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = a.c0 + lane, s0 = wave * R;
    const int tt = tid / (kWave / E), tc = (tid & (kWave / E - 1)) * E, nv = WHOLE ? E : a.nc - tc, ec = a.c0 + tc;
    float A[R], carry[R] = {}, dtotal = 0.f, dbias[E] = {};
    const bool ok = WHOLE || lane < a.nc;
    load_decays(p.A + (int64_t)c * p.S, s0, p.S, ok, A);
#pragma unroll
    for (int r = 0; r < R; ++r) A[r] *= kLog2e;
    if (a.chunk == p.chunks - 1 && p.dstate_out)
        load_states(p.dstate_out + ((int64_t)a.n * p.C + c) * p.S, s0, p.S, ok, carry);
    if (nv > 0 && p.delta_bias) load_some<E>(p.delta_bias + ec, nv, dbias);
    const bool gate = p.z.p != nullptr;
    int t = (a.stop - 1) * kT + tt;
    Share<const T, E> pd(p.delta, a.n, t, ec), pg(p.dout, a.n, t, ec), pz(p.z, a.n, t, ec);
    Run<T, E> dl{}, go{}, z{};
    auto fetch = [&](int at) {
        if (at < a.len && nv > 0) {
            dl = pd.load(nv);
            go = pg.load(nv);
            if (gate) z = pz.load(nv);
        }
        pd.back(); pg.back(); pz.back();
    };
    BC<true> bc, next;
    if (a.stop > a.tile0) {
        fetch(t);
        bc.load(bc_of(p, a, a.stop - 1, W, wave) + kT - kStep);
    }
    for (int tile = a.stop - 1; tile >= a.tile0; --tile, t -= kT) {
        float raw[E], d_[E], dy[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            raw[i] = dl[i] + dbias[i];
            dy[i] = go[i];
        }
        steps_of(p.softplus, raw, d_);
        if (gate) {
#pragma unroll
            for (int i = 0; i < E; ++i) dy[i] *= z[i] * sigmoid(z[i]);
        }
        if ((tile + 1) * kT > a.len) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if (t >= a.len) d_[i] = dy[i] = 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < E; ++i) step[tt][tc + i] = make_float2(d_[i], dy[i]);
        if (tile > a.tile0) fetch(t - kT);
        meet();
        float2 d[kStep], dn[kStep];
#pragma unroll
        for (int k = 0; k < kStep; ++k) d[k] = step[kT - kStep + k][lane];
        const bc_ptr here = bc_of(p, a, tile, W, wave), after = bc_of(p, a, max(tile - 1, a.tile0), W, wave);
#pragma unroll
        for (int k0 = kT - kStep; k0 >= 0; k0 -= kStep) {
            arrived();
            next.load(k0 ? here + k0 - kStep : after + kT - kStep);
#pragma unroll
            for (int k = 0; k < kStep; ++k)
                if (k0) dn[k] = step[k0 - kStep + k][lane];
            in_order();
#pragma unroll
            for (int k = kStep - 1; k >= 0; --k) {
#pragma unroll
                for (int r = 0; r < R; ++r) carry[r] = exp2_(d[k].x * A[r]) * __builtin_fmaf(bc.c(k, r), d[k].y, carry[r]);
                dtotal += d[k].x;
            }
            in_order();
            bc = next;
#pragma unroll
            for (int k = 0; k < kStep; ++k) d[k] = dn[k];
        }
        meet();
    }
    const int64_t row = (int64_t)a.n * p.chunks + a.chunk;
    store_states(p.back + lane_states<W, R>(p, a, row, wave, lane), carry);
    if (wave == 0) p.dsum[(row * p.blocks + a.block) * kWave + lane] = dtotal;
}

template <typename T, int W, int R>
__global__ void __launch_bounds__(kWave * W)
scan_back_kernel(ScanParams p)
{
    __shared__ float2 step[kT][kWave];
    ScanPlace a = scan_place(p);
    a.chunk += 1;
    a.tile0 += p.chunk_tiles;
    a.tile1 = min(a.tile0 + p.chunk_tiles, p.tiles);
    a.stop = max(a.tile0, min(a.tile1, (a.len + kT - 1) / kT));
    if (a.nc == kWave) back_block<T, W, R, true>(p, a, step);
    else back_block<T, W, R, false>(p, a, step);
}

// One pass over each chunk from a state of zero (the first: the call's): the state at the start of every tile and what d adds
// up to until there, the state and sum at the end, and the gradient that the chunk leaves at its start (begun at
// zero, in the last chunk at the gradient of the call's last state).
struct SweepLds {
    float2 step[kT][kWave];                             // d, d u
    float gout[kT][kWave];                              // dy
};

template <typename T, int W, int R, bool WHOLE>
__device__ __forceinline__ void sweep_block(const ScanParams& p, const ScanPlace& a, SweepLds& lds)
{
    constexpr int E = kT / W;
    auto& step = lds.step;
    auto& gout = lds.gout;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = a.c0 + lane, s0 = wave * R;
    const int tt = tid / (kWave / E), tc = (tid & (kWave / E - 1)) * E, nv = WHOLE ? E : a.nc - tc, ec = a.c0 + tc;
    const bool ok = WHOLE || lane < a.nc, gate = p.z.p != nullptr;
    float A[R], h[R] = {}, q[R] = {}, decay[R], dtotal = 0.f, dbias[E] = {};
    load_decays(p.A + (int64_t)c * p.S, s0, p.S, ok, A);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        A[r] *= kLog2e;
        decay[r] = 1.f;
    }
    const int64_t own = ((int64_t)a.n * p.C + c) * p.S, row = (int64_t)a.n * p.chunks + a.chunk;
    if (a.chunk == 0 && p.state) load_states(p.state + own, s0, p.S, ok, h);
    if (nv > 0 && p.delta_bias) load_some<E>(p.delta_bias + ec, nv, dbias);
    int t = a.tile0 * kT + tt;
    Share<const T, E> pu(p.u, a.n, t, ec), pd(p.delta, a.n, t, ec), pg(p.dout, a.n, t, ec), pz(p.z, a.n, t, ec);
    Run<T, E> u{}, dl{}, go{}, z{};
    auto fetch = [&](int at) {
        if (at < a.len && nv > 0) {
            u = pu.load(nv);
            dl = pd.load(nv);
            go = pg.load(nv);
            if (gate) z = pz.load(nv);
        }
        pu.forward(); pd.forward(); pg.forward(); pz.forward();
    };
    BC<true> bc, next;
    if (a.tile0 < a.stop) {
        fetch(t);
        bc.load(bc_of(p, a, a.tile0, W, wave));
    }
    for (int tile = a.tile0; tile < a.stop; ++tile, t += kT) {
        float raw[E], d_[E], u_[E], dy_[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            raw[i] = dl[i] + dbias[i];
            u_[i] = u[i];
            dy_[i] = go[i];
        }
        steps_of(p.softplus, raw, d_);
        if (gate) {
#pragma unroll
            for (int i = 0; i < E; ++i) dy_[i] *= z[i] * sigmoid(z[i]);
        }
        if ((tile + 1) * kT > a.len) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if (t >= a.len) d_[i] = u_[i] = dy_[i] = 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
            step[tt][tc + i] = make_float2(d_[i], d_[i] * u_[i]);
            gout[tt][tc + i] = dy_[i];
        }
        if (tile + 1 < a.stop) fetch(t + kT);
        meet();
        store_states(p.starts + lane_states<W, R>(p, a, (int64_t)a.n * p.tiles + tile, wave, lane), h);
        if (wave == 0) p.cum[(((int64_t)a.n * p.tiles + tile) * p.blocks + a.block) * kWave + lane] = dtotal;
        float2 d[kStep], dn[kStep];
        float dy[kStep], dyn[kStep];
#pragma unroll
        for (int k = 0; k < kStep; ++k) {
            d[k] = step[k][lane];
            dy[k] = gout[k][lane];
        }
        const bc_ptr here = bc_of(p, a, tile, W, wave), after = bc_of(p, a, min(tile + 1, a.stop - 1), W, wave);
#pragma unroll
        for (int k0 = 0; k0 < kT; k0 += kStep) {
            const bool more = k0 + kStep < kT;
            arrived();
            next.load(more ? here + k0 + kStep : after);
#pragma unroll
            for (int k = 0; k < kStep; ++k) {
                if (!more) continue;
                dn[k] = step[k0 + kStep + k][lane];
                dyn[k] = gout[k0 + kStep + k][lane];
            }
            in_order();
#pragma unroll
            for (int k = 0; k < kStep; ++k) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float e = exp2_(d[k].x * A[r]);
                    h[r] = __builtin_fmaf(e, h[r], d[k].y * bc.b(k, r));
                    decay[r] *= e;
                    q[r] = __builtin_fmaf(decay[r], bc.c(k, r) * dy[k], q[r]);
                }
                dtotal += d[k].x;
            }
            in_order();
            bc = next;
#pragma unroll
            for (int k = 0; k < kStep; ++k) {
                d[k] = dn[k];
                dy[k] = dyn[k];
            }
        }
        meet();
    }
    if (a.chunk == p.chunks - 1 && p.dstate_out) {
        float last[R];
        load_states(p.dstate_out + own, s0, p.S, ok, last);
#pragma unroll
        for (int r = 0; r < R; ++r) q[r] = __builtin_fmaf(decay[r], last[r], q[r]);
    }
    store_states(p.ends + lane_states<W, R>(p, a, row, wave, lane), h);
    store_states(p.back + lane_states<W, R>(p, a, row, wave, lane), q);
    if (wave == 0) p.dsum[(row * p.blocks + a.block) * kWave + lane] = dtotal;
}

template <typename T, int W, int R>
__global__ void __launch_bounds__(kWave * W)
sweep_kernel(ScanParams p)
{
    __shared__ SweepLds lds;
    const ScanPlace a = scan_place(p);
    if (a.nc == kWave) sweep_block<T, W, R, true>(p, a, lds);
    else sweep_block<T, W, R, false>(p, a, lds);
}

template <int W> struct GradLds {
    float2 step[kT][kWave];                             // d, d u
    float gout[kT][kWave];                              // dy
    float sums[3][W][kT][kWave];                        // over a wave's states: C h, g B, e A
};

template <typename T, int W, int R, bool WHOLE>
__device__ __forceinline__ void grad_block(const ScanParams& p, const ScanPlace& a, GradLds<W>& lds)
{
    constexpr int E = kT / W;
    constexpr int kGather = gathered(R);
    auto& step = lds.step;
    auto& gout = lds.gout;
    auto& sums = lds.sums;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = a.c0 + lane, s0 = wave * R;
    const bool ok = WHOLE || lane < a.nc, gate = p.z.p != nullptr;
    const int tt = tid / (kWave / E), tc = (tid & (kWave / E - 1)) * E, nv = WHOLE ? E : a.nc - tc, ec = a.c0 + tc;

    float A[R], carry[R] = {}, dA[R] = {};
    load_decays(p.A + (int64_t)c * p.S, s0, p.S, ok, A);
    const int64_t own = ((int64_t)a.n * p.C + c) * p.S, row = (int64_t)a.n * p.chunks;
    if (a.chunk == p.chunks - 1) {
        if (p.dstate_out) load_states(p.dstate_out + own, s0, p.S, ok, carry);
    } else {
        for (int k = p.chunks - 1; k > a.chunk; --k) {
            float e[R];
            load_states(p.back + lane_states<W, R>(p, a, row + k, wave, lane), e);
            const float d = p.dsum[((row + k) * p.blocks + a.block) * kWave + lane];
#pragma unroll
            for (int r = 0; r < R; ++r) carry[r] = __builtin_fmaf(exp2_(d * (A[r] * kLog2e)), carry[r], e[r]);
        }
    }
    // the state that the chunk begins at, where its tiles' are as if that were zero
    float begin[R] = {};
    const bool later = p.cum && a.chunk;
    if (later) {
        for (int k = 0; k < a.chunk; ++k) {
            float e[R];
            load_states(p.ends + lane_states<W, R>(p, a, row + k, wave, lane), e);
            const float d = p.dsum[((row + k) * p.blocks + a.block) * kWave + lane];
#pragma unroll
            for (int r = 0; r < R; ++r) begin[r] = __builtin_fmaf(exp2_(d * (A[r] * kLog2e)), begin[r], e[r]);
        }
    }
    float dbias[E] = {}, skip[E] = {}, sumD[E] = {}, sumB[E] = {};
    if (nv > 0) {
        if (p.delta_bias) load_some<E>(p.delta_bias + ec, nv, dbias);
        if (p.D) load_some<E>(p.D + ec, nv, skip);
    }
    int t = (a.tile1 - 1) * kT + tt;
    Share<T, E> qu(p.du, a.n, t, ec), qd(p.ddelta, a.n, t, ec), qz(p.dz, a.n, t, ec);
    for (int tile = a.tile1 - 1; tile >= a.stop; --tile, t -= kT) {          // tiles that do not count
        const float zero[E] = {};
        if (nv > 0 && t < p.L) {
            qu.store(nv, zero);
            qd.store(nv, zero);
            if (gate) qz.store(nv, zero);
        }
        qu.back(); qd.back(); qz.back();
    }
    Share<const T, E> pu(p.u, a.n, t, ec), pd(p.delta, a.n, t, ec), pg(p.dout, a.n, t, ec), pz(p.z, a.n, t, ec);
    // what a tile reads, asked for a tile ahead
    Run<T, E> un{}, dln{}, gon{}, zn{};
    float hn[R] = {}, cumn = 0.f;
    auto fetch = [&](int tile, int at) {
        if (p.starts) load_states(p.starts + lane_states<W, R>(p, a, (int64_t)a.n * p.tiles + tile, wave, lane), hn);
        else if (p.state) load_states(p.state + own, s0, p.S, ok, hn);       // (the only tile)
        if (later) cumn = p.cum[(((int64_t)a.n * p.tiles + tile) * p.blocks + a.block) * kWave + lane];
        if (at < a.len && nv > 0) {
            un = pu.load(nv);
            dln = pd.load(nv);
            gon = pg.load(nv);
            if (gate) zn = pz.load(nv);
        }
        pu.back(); pd.back(); pg.back(); pz.back();
    };
    BC<true> bc, next;
    if (a.stop > a.tile0) {
        fetch(a.stop - 1, t);
        bc.load(bc_of(p, a, a.stop - 1, W, wave));
    }
    for (int tile = a.stop - 1; tile >= a.tile0; --tile, t -= kT) {
        Run<T, E> u = un, dl = dln, go = gon, z = zn;
        float h0[R];
#pragma unroll
        for (int r = 0; r < R; ++r) h0[r] = hn[r];
        if (later) {
#pragma unroll
            for (int r = 0; r < R; ++r) h0[r] = __builtin_fmaf(exp2_(cumn * (A[r] * kLog2e)), begin[r], h0[r]);
        }
        float raw[E], d_[E], dy_[E], u_[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            raw[i] = dl[i] + dbias[i];
            u_[i] = u[i];
            dy_[i] = go[i];
        }
        steps_of(p.softplus, raw, d_);
        if (gate) {
#pragma unroll
            for (int i = 0; i < E; ++i) dy_[i] *= z[i] * sigmoid(z[i]);
        }
        if ((tile + 1) * kT > a.len) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if (t >= a.len) d_[i] = u_[i] = dy_[i] = 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
            step[tt][tc + i] = make_float2(d_[i], d_[i] * u_[i]);
            gout[tt][tc + i] = dy_[i];
        }
        if (tile > a.tile0) fetch(tile - 1, t - kT);
        meet();
        const bc_ptr here = bc_of(p, a, tile, W, wave), after = bc_of(p, a, max(tile - 1, a.tile0), W, wave);
        float dec[kT][R], h[kT][R];
        float2 s[kStep], sn[kStep];
        float ys[kStep], qs[kStep];
#pragma unroll
        for (int k = 0; k < kStep; ++k) s[k] = step[k][lane];
#pragma unroll
        for (int k0 = 0; k0 < kT; k0 += kStep) {
            const bool more = k0 + kStep < kT;
            arrived();
            if (more) next.load(here + k0 + kStep);
#pragma unroll
            for (int k = 0; k < kStep; ++k) {
                if (more) sn[k] = step[k0 + kStep + k][lane];
                if (k0) sums[0][wave][k0 - kStep + k][lane] = ys[k];
            }
            in_order();
#pragma unroll
            for (int k = k0; k < k0 + kStep; ++k) {
                float y = 0.f;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    dec[k][r] = exp2_(s[k - k0].x * (A[r] * kLog2e));
                    h[k][r] = __builtin_fmaf(dec[k][r], k ? h[k - 1][r] : h0[r], s[k - k0].y * bc.b(k - k0, r));
                    y = r ? __builtin_fmaf(bc.c(k - k0, r), h[k][r], y) : bc.c(k - k0, r) * h[k][r];
                }
                ys[k - k0] = y;
            }
            in_order();
            if (more) {
                bc = next;
#pragma unroll
                for (int k = 0; k < kStep; ++k) s[k] = sn[k];
            }
        }
        float packed[kGather], dy[kStep], dyn[kStep], dAt[R] = {};
#pragma unroll
        for (int k = 0; k < kStep; ++k) {
            dy[k] = gout[kT - kStep + k][lane];
            sums[0][wave][kT - kStep + k][lane] = ys[k];
        }
#pragma unroll
        for (int k0 = kT - kStep; k0 >= 0; k0 -= kStep) {
            arrived();
            next.load(k0 ? here + k0 - kStep : after);
#pragma unroll
            for (int k = 0; k < kStep; ++k) {
                if (k0 < kT - kStep) {
                    sums[1][wave][k0 + kStep + k][lane] = qs[k];
                    sums[2][wave][k0 + kStep + k][lane] = ys[k];
                }
                if (!k0) continue;
                sn[k] = step[k0 - kStep + k][lane];
                dyn[k] = gout[k0 - kStep + k][lane];
            }
            in_order();
#pragma unroll
            for (int k = k0 + kStep - 1; k >= k0; --k) {
                const int j = k - k0;
                float q = 0.f, ea = 0.f, pair[R];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float g = __builtin_fmaf(bc.c(j, r), dy[j], carry[r]);
                    carry[r] = g * dec[k][r];
                    const float e = carry[r] * (k ? h[k - 1][r] : h0[r]);
                    q = r ? __builtin_fmaf(g, bc.b(j, r), q) : g * bc.b(j, r);
                    ea = r ? __builtin_fmaf(e, A[r], ea) : e * A[r];
                    dAt[r] = __builtin_fmaf(e, s[j].x, dAt[r]);
                    pair[r] = fold32(g * s[j].y, dy[j] * h[k][r]);
                }
                qs[j] = q;
                ys[j] = ea;
                // lane bit 5: B or C; bits 4 and 3 the state, the rest the token, as far as there are states
                if constexpr (R == 4) packed[k & 7] = fold<kAcross8, 8>(fold16(pair[0], pair[2]), fold16(pair[1], pair[3]));
                else packed[k] = fold16(pair[0], pair[R - 1]);
                if (k % kGather == 0) {
                    float f[4], e[2], g[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if constexpr (R == 4) g[i] = packed[i];
                        else g[i] = fold<kAcross8, 8>(packed[i], packed[i + 8]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) f[i] = fold<kAcross4, 4>(g[i], g[i + 4]);
#pragma unroll
                    for (int i = 0; i < 2; ++i) e[i] = fold<kAcross2, 2>(f[i], f[i + 2]);
                    const int64_t at = (((int64_t)a.block * p.N + a.n) * p.tiles + tile) * (kT / kGather) + k / kGather;
                    p.part_bc[(at * W + wave) * kWave + lane] = fold<kAcross1, 1>(e[0], e[1]);
                }
            }
            in_order();
            bc = next;
#pragma unroll
            for (int k = 0; k < kStep; ++k) {
                s[k] = sn[k];
                dy[k] = dyn[k];
            }
        }
#pragma unroll
        for (int k = 0; k < kStep; ++k) {
            sums[1][wave][k][lane] = qs[k];
            sums[2][wave][k][lane] = ys[k];
        }
#pragma unroll
        for (int r = 0; r < R; ++r) dA[r] += dAt[r];
        meet();
        if (nv > 0 && t < p.L) {
            float du[E], dd[E], dz[E], y[E], q[E] = {}, ea[E] = {}, dy[E];
            const Run<float, E> dyr = lds_run<E>(&gout[tt][tc]);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                y[i] = skip[i] * u[i];
                dy[i] = dyr[i];
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const Run<float, E> r0 = lds_run<E>(&sums[0][w][tt][tc]), r1 = lds_run<E>(&sums[1][w][tt][tc]),
                                    r2 = lds_run<E>(&sums[2][w][tt][tc]);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    y[i] += r0[i];
                    q[i] += r1[i];
                    ea[i] += r2[i];
                }
            }
#pragma unroll
            for (int i = 0; i < E; ++i) {
                du[i] = __builtin_fmaf(step[tt][tc + i].x, q[i], skip[i] * dy[i]);
                dd[i] = __builtin_fmaf(u[i], q[i], ea[i]);
                dz[i] = y[i];
                sumD[i] = __builtin_fmaf(dy[i], t < a.len ? u[i] : 0.f, sumD[i]);
            }
            if (p.softplus) {
#pragma unroll
                for (int i = 0; i < E; ++i) dd[i] *= sigmoid(dl[i] + dbias[i]);
            }
            if (gate) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float sg = sigmoid(z[i]);
                    dz[i] *= go[i] * (sg * (1.f + z[i] * (1.f - sg)));
                }
            }
            if ((tile + 1) * kT > a.len) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    if (t >= a.len) du[i] = dd[i] = dz[i] = 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < E; ++i) sumB[i] += dd[i];
            qu.store(nv, du);
            qd.store(nv, dd);
            if (gate) qz.store(nv, dz);
        }
        qu.back(); qd.back(); qz.back();
    }
    if (a.chunk == 0 && p.dstate && ok) store_some<R>(p.dstate + own + s0, p.S - s0, carry);
    store_states(p.part_A + lane_states<W, R>(p, a, row + a.chunk, wave, lane), dA);
    // dD and the gradient of the bias: over the sixteen tokens of a tile
    __syncthreads();
#pragma unroll
    for (int i = 0; i < E; ++i) step[tt][tc + i] = make_float2(sumD[i], sumB[i]);
    __syncthreads();
    if (wave == 0) {
        double sD = 0., sB = 0.;
#pragma unroll
        for (int k = 0; k < kT; ++k) {
            sD += step[k][lane].x;
            sB += step[k][lane].y;
        }
        const int64_t at = ((row + a.chunk) * p.blocks + a.block) * kWave + lane;
        p.part_D[at] = (float)sD;
        p.part_bias[at] = (float)sB;
    }
}

template <typename T, int W, int R>
__global__ void __launch_bounds__(kWave * W, 2)
scan_grad_kernel(ScanParams p)
{
    __shared__ GradLds<W> lds;
    const ScanPlace a = scan_place(p);
    if (a.nc == kWave) grad_block<T, W, R, true>(p, a, lds);
    else grad_block<T, W, R, false>(p, a, lds);
}

// What many workgroups have a part of, in the same order on every call.  The first p.blocks * (W R + 2) workgroups:
// dA, dD and the gradient of the bias from the parts of all sequences and chunks, four waves a quarter each.
__device__ __forceinline__ void sum_params(const ScanParams& p, int W, int R, float* dA, float* dD, float* dbias, double (&red)[4][kWave])
{
    const int values = W * R + 2, block = blockIdx.x / values, v = blockIdx.x - block * values;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t rows = (int64_t)p.N * p.chunks;
    const float* from = v < W * R ? p.part_A + ((int64_t)block * W * kWave + v / R * kWave + lane) * R + v % R
                                  : (v == W * R ? p.part_D : p.part_bias) + (int64_t)block * kWave + lane;
    const int64_t step = (int64_t)p.blocks * kWave * (v < W * R ? W * R : 1);
    double s = 0.;
#pragma unroll 4
    for (int64_t r = wave; r < rows; r += 4) s += from[r * step];
    red[wave][lane] = s;
    __syncthreads();
    const int g = block / p.gblocks, k = block - g * p.gblocks, c = g * p.group + k * kWave + lane;
    if (wave || k * kWave + lane >= p.group) return;
    s = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
    if (v < W * R) {
        if (v < p.S) dA[(int64_t)c * p.S + v] = (float)s;
    } else if (v == W * R) {
        if (dD) dD[c] = (float)s;
    } else if (dbias) {
        dbias[c] = (float)s;
    }
}

// The others: dB and dC from the parts of a group's channel blocks; lane l of a unit has the value that lane l had above.
template <typename T>
__global__ void __launch_bounds__(kThreads)
scan_sum_kernel(ScanParams p, int W, int R, float* dA, float* dD, float* dbias, Rows dB, Rows dC, int64_t b_g, int64_t c_g)
{
    __shared__ double red[4][kWave];
    const int first = p.blocks * (W * R + 2);
    if ((int)blockIdx.x < first) return sum_params(p, W, R, dA, dD, dbias, red);
    const int64_t i = (int64_t)((int)blockIdx.x - first) * kThreads + threadIdx.x;
    const int lane = (int)(i & 63), tokens = gathered(R);
    const int64_t unit = i >> 6, per = (int64_t)p.tiles * (kT / tokens) * W;    // units [G][N][tiles][kT / tokens][W]
    const int64_t seq = unit / per, in = unit - seq * per;
    const int g = (int)(seq / p.N), n = (int)(seq - (int64_t)g * p.N);
    if (g >= p.G) return;
    const int w = (int)(in % W), t = (int)(in / W) * tokens + (lane & (tokens - 1));
    const int r = R == 4 ? (lane >> 4 & 1) * 2 + (lane >> 3 & 1) : lane >> 4 & 1, s = w * R + r;
    if (r >= R || t >= p.L || s >= p.S) return;
    float v = 0.f;
    if (t < length_of(p.lengths, n, p.L)) {
        const float* from = p.part_bc + (((int64_t)g * p.gblocks * p.N + n) * per + in) * kWave + lane;
        const int64_t step = p.N * per * kWave;
#pragma unroll 8
        for (int k = 0; k < p.gblocks; ++k) v += from[k * step];
    }
    if (lane < 32) dB.at<T>(n, t, 0)[g * b_g + s] = (T)v;
    else dC.at<T>(n, t, 0)[g * c_g + s] = (T)v;
}

template <typename T, int W, int R> void launch_kernels(const ScanParams& p, hipStream_t st)
{
    if (p.cum)
        hipLaunchKernelGGL((sweep_kernel<T, W, R>), dim3((unsigned)p.total), dim3(kWave * W), 0, st, p);
    else if (p.chunks > 1)
        hipLaunchKernelGGL((scan_back_kernel<T, W, R>), dim3((unsigned)(p.total - (int64_t)p.N * p.blocks)), dim3(kWave * W), 0, st, p);
    hipLaunchKernelGGL((scan_grad_kernel<T, W, R>), dim3((unsigned)p.total), dim3(kWave * W), 0, st, p);
}

template <typename T> void launch_typed(const dconv_scan_args& a, const ScanParams& p, int W, int R, hipStream_t st)
{
    if (a.S <= 4) launch_kernels<T, 4, 1>(p, st);
    else if (a.S <= 8) launch_kernels<T, 4, 2>(p, st);
    else if (a.S <= 16) launch_kernels<T, 4, 4>(p, st);
    else launch_kernels<T, 8, 4>(p, st);
    const int64_t n = (int64_t)p.N * p.G * p.tiles * (kT / gathered(R)) * W * kWave;
    hipLaunchKernelGGL((scan_sum_kernel<T>), dim3((unsigned)(p.blocks * (W * R + 2) + (n + kThreads - 1) / kThreads)), dim3(kThreads),
                       0, st, p, W, R, a.dA, a.dD, a.ddelta_bias, Rows{a.dB.p, a.dB.sn, a.dB.sl}, Rows{a.dC.p, a.dC.sn, a.dC.sl},
                       a.dB.sg, a.dC.sg);
}

// The workspace of a gradient call, in floats: where its parts begin, and how many there are.
struct GradSpace { int64_t ends, back, dsum, cum, bc_parts, A_parts, D_parts, bias_parts, starts, all; };

GradSpace space_of(const dconv_scan_args& a, const ScanPlan& pl)
{
    const int64_t rows = (int64_t)a.N * pl.chunks * pl.blocks * kWave, states = rows * pl.waves * pl.states;
    const bool chunks = pl.chunks > 1, sweep = chunks && !a.starts;
    GradSpace s;
    int64_t at = scan_bc_floats(a, pl);
    auto take = [&](int64_t n) { const int64_t here = at; at += (n + 3) / 4 * 4; return here; };
    s.ends = take(sweep ? states : 0);
    s.back = take(chunks ? states : 0);
    s.dsum = take(chunks ? rows : 0);
    s.cum = take(sweep ? (int64_t)a.N * pl.tiles * pl.blocks * kWave : 0);
    s.bc_parts = take((int64_t)pl.blocks * a.N * pl.tiles * (kT / gathered(pl.states)) * pl.waves * kWave);
    s.A_parts = take(states);
    s.D_parts = take(rows);
    s.bias_parts = take(rows);
    s.starts = take(a.starts || pl.tiles == 1 ? 0 : scan_starts_floats(a));
    s.all = at;
    return s;
}

}  // namespace

}  // namespace dconv

using namespace dconv;

extern "C" {

long long dconv_scan_workspace(const dconv_scan_args* a, int grad)
{
    if (!a || !token_bytes(a->dtype) || !scan_sizes_ok(*a)) return -1;
    const ScanPlan pl = scan_plan(*a, grad != 0);
    if (!grad && scan_short(*a, pl)) return 0;
    return 4 * (grad ? space_of(*a, pl).all : scan_bc_floats(*a, pl) + scan_chunk_floats(*a, pl));
}

int dconv_scan_grad(const dconv_scan_args* a, void* stream)
{
    int rc = scan_check(a, 1);
    if (rc != DCONV_OK) return rc;
    const hipStream_t st = (hipStream_t)stream;
    const ScanPlan pl = scan_plan(*a, true);
    const GradSpace s = space_of(*a, pl);
    float* ws = (float*)a->workspace;
    ScanParams p = scan_params(*a, pl);
    p.bc = ws;
    p.back = ws + s.back; p.dsum = ws + s.dsum;
    p.part_bc = ws + s.bc_parts; p.part_A = ws + s.A_parts; p.part_D = ws + s.D_parts; p.part_bias = ws + s.bias_parts;
    rc = launch_scan_bc(*a, pl, ws, st);
    if (rc != DCONV_OK) return rc;
    if (!a->starts && pl.tiles > 1) {                    // (a single tile begins at the call's state)
        p.starts = ws + s.starts;
        if (pl.chunks > 1) {
            p.ends = ws + s.ends;
            p.cum = ws + s.cum;
        } else {
            ScanParams forward = p;
            forward.state_out = nullptr;
            rc = launch_scan_forward(*a, forward, pl, false, st);
            if (rc != DCONV_OK) return rc;
        }
    }
    begin_launch();
    if (a->dtype == DCONV_DTYPE_F16) launch_typed<_Float16>(*a, p, pl.waves, pl.states, st);
    else if (a->dtype == DCONV_DTYPE_BF16) launch_typed<__bf16>(*a, p, pl.waves, pl.states, st);
    else launch_typed<float>(*a, p, pl.waves, pl.states, st);
    return launch_status();
}

}  // extern "C"
