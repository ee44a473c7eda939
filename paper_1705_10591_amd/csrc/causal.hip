// The causal convolution over tokens: one filter of F taps for every channel, s[t] = bias + sum_j filt[j] x[t-(F-1)+j],
// out = s sigmoid(s) or s.
//
// With F multiply-adds an element the call is bound by memory: x is read once and out is written once.  The paper's
// sliding window (Sec. 3: a thread keeps the rows that its next output needs in registers and reads one new row a
// step) does that along the tokens: a thread has a run of V channels (16 bytes) and walks a strip of tokens with the
// last F-1 rows in registers, kAhead rows in flight; lanes next to each other have runs next to each other.  Only the
// F-1 rows before a strip are read twice.  Measured: 8 x 4096 x 4096 bf16 with 4 taps 116 us, 4.64 TB/s of the 4.94 that a
// large copy reaches; the gradient of half as many tokens 98 us; one row of 2048 channels 2.4 us, 200 rows of 5120 5.6.
#include "tokens.h"

namespace dconv {

namespace {

constexpr int kAhead = 8;            // rows of a strip that are read together; strips are multiples of it, so that
                                     // only the first one reaches into the state (F - 1 <= 7 rows)
constexpr int kGradAhead = 4;
constexpr int kGradSum = 32;          // tokens that a thread adds up by themselves where it has the registers

struct CausalParams {
    const void *x, *filt, *bias, *state, *dout, *dstate_out;
    void *out, *state_out, *dx, *dstate;
    float* part;
    const int *lengths, *slots;
    int64_t x_n, x_l, o_n, o_l, g_n, g_l, d_n, d_l;
    int L, C, M, silu;
    int vb, sb, vgroups, sgroups, strip;   // runs and strips of a workgroup, groups of each, tokens of a strip
    int64_t total;
};

// Where a thread works: sequence n, its first channel c and how many of the V exist, its first token.
struct Place { int n, c, nv, t0, run, strip, c0; int64_t row; bool ok, whole; };   // c0: of the workgroup; whole: of the wave

template <int V> __device__ __forceinline__ Place place_of(const CausalParams& p)
{
    const int64_t b = near_block(blockIdx.x, p.total);
    const int vg = (int)(b % p.vgroups);
    Place a;
    a.row = b / p.vgroups;
    const int sg = (int)(a.row % p.sgroups);
    a.n = (int)(a.row / p.sgroups);
    a.strip = threadIdx.x / p.vb;
    a.run = threadIdx.x - a.strip * p.vb;
    a.c0 = vg * p.vb * V;
    a.c = a.c0 + a.run * V;
    a.nv = min(V, p.C - a.c);
    const int64_t t0 = ((int64_t)sg * p.sb + a.strip) * p.strip;
    a.t0 = (int)min(t0, (int64_t)p.L);
    a.ok = a.strip < p.sb && a.nv > 0 && t0 < p.L;
    a.whole = __all(a.nv == V || !a.ok);             // none of the wave's runs is cut
    return a;
}

template <typename T, int F, int V>
__device__ __forceinline__ void load_filter(const T* filt, int c, int nv, float (&w)[F][V])
{
    float flat[F * V];
#pragma unroll
    for (int q = 0; q < F; ++q) {
        const Run<T, V> part = load_some<V>(filt + (int64_t)c * F + q * V, nv * F - q * V);
#pragma unroll
        for (int i = 0; i < V; ++i) flat[q * V + i] = part[i];
    }
#pragma unroll
    for (int j = 0; j < F; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) w[j][i] = flat[i * F + j];
}

template <typename T, int F, int V, bool WHOLE>
__device__ __forceinline__ void causal_strip(const CausalParams& p, Place a)
{
    if (WHOLE) a.nv = V;
    const int len = length_of(p.lengths, a.n, p.L), end = min(a.t0 + p.strip, p.L);
    const T* x = (const T*)p.x + a.n * p.x_n + a.c;
    T* out = (T*)p.out + a.n * p.o_n + a.c;
    const int64_t first = (int64_t)a.n * (F - 1) * p.C + a.c;

    // rows are loaded together and without conditions: one that does not count reads the last one that does, and what is
    // made of it is not written
    Run<T, V> in[kAhead], before[F];
    auto fetch = [&](int t0) {
        if (len == 0) return;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) in[k] = load_some<V>(x + min(t0 + k, len - 1) * p.x_l, a.nv);
    };
#pragma unroll
    for (int r = 0; r < F - 1; ++r) {
        const int t = a.t0 - (F - 1) + r;
        before[r] = Run<T, V>{};
        if (t >= 0) {
            if (len) before[r] = load_some<V>(x + min(t, len - 1) * p.x_l, a.nv);
        } else if (p.state) {
            before[r] = load_some<V>((const T*)p.state + first + (int64_t)(F - 1 + t) * p.C, a.nv);
        }
    }
    fetch(a.t0);
    float w[F][V], bias[V] = {}, rows[kAhead + F - 1][V];
    load_filter<T, F, V>((const T*)p.filt, a.c, a.nv, w);
    if (p.bias) load_some<V>((const T*)p.bias + a.c, a.nv, bias);
    // the last F-1 rows of the sequence, by the thread that has read the state's (which they may overwrite)
    if (a.t0 == 0 && p.state_out) {
        for (int r = 0; r < F - 1; ++r) {
            const int t = len - (F - 1) + r;
            float v[V] = {};
            if (t >= 0) load_some<V>(x + t * p.x_l, a.nv, v);
            else if (p.state) load_some<V>((const T*)p.state + first + (int64_t)(F - 1 + t) * p.C, a.nv, v);
            store_some<V>((T*)p.state_out + first + (int64_t)r * p.C, a.nv, v);
        }
    }
#pragma unroll
    for (int r = 0; r < F - 1; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) rows[r][i] = before[r][i];
    for (int t0 = a.t0; t0 < end; t0 += kAhead) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) rows[F - 1 + k][i] = in[k][i];
        if (t0 + kAhead < end) fetch(t0 + kAhead);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            float y[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float s = bias[i];
#pragma unroll
                for (int j = 0; j < F; ++j) s = __builtin_fmaf(w[j][i], rows[k + j][i], s);
                y[i] = t0 + k < len ? (p.silu ? s * sigmoid(s) : s) : 0.f;
            }
            if (t0 + k < end) store_some<V>(out + (t0 + k) * p.o_l, a.nv, y);
        }
#pragma unroll
        for (int r = 0; r < F - 1; ++r)
#pragma unroll
            for (int i = 0; i < V; ++i) rows[r][i] = rows[kAhead + r][i];
    }
}

// (runs that are cut, at the end of a number of channels that V does not divide, have code of their own: branches for them
// around every load and store are more instructions than the rest)
template <typename T, int F, int V>
__global__ void __launch_bounds__(kThreads)
causal_kernel(CausalParams p)
{
    const Place a = place_of<V>(p);
    if (!a.ok) return;
    if (a.whole) causal_strip<T, F, V, true>(p, a);
    else causal_strip<T, F, V, false>(p, a);
}

// Gradients.  With ds[t] = dout[t] silu'(s[t]) (s computed again): dx[r] = sum_j filt[j] ds[r + F-1-j], so a row of dx is
// done F-1 tokens later and a strip walks F-1 tokens beyond its end; dfilt[j] = sum_t ds[t] x[t-(F-1)+j] and
// dbias = sum_t ds[t] are summed over the strip by each thread, over the strips of a workgroup in LDS, and by
// causal_sum_kernel over workgroups, always in the same order.  Bound by memory like the convolution: x and dout
// in, dx out.
//
// What rounds these sums most is the longest one: a strip in 32 bits is off by some 0.3 sqrt(128) 2^-24, and 4 sums of 32 tokens by half of
// that.  LDS and the second kernel add in 64 bits.  Measured on 8 x 2048 x 4096, dfilt off by 1.3e-7 of its norm instead of 2.3e-7, at the
// same speed.  Calls of more than four taps, or of four channels a thread, lack the registers for a second set of sums (8 taps:
// 117 us and 143 with them); their strips are added up in one.
template <typename T, int F, int V, bool WHOLE>
__device__ __forceinline__ void causal_grad_strip(const CausalParams& p, Place a, float (&acc)[F + 1][V])
{
    if (WHOLE) a.nv = V;
    const int len = length_of(p.lengths, a.n, p.L), end = min(a.t0 + p.strip, p.L);
    const T* x = (const T*)p.x + a.n * p.x_n + a.c;
    const T* dout = (const T*)p.dout + a.n * p.g_n + a.c;
    T* dx = (T*)p.dx + a.n * p.d_n + a.c;
    const int64_t first = (int64_t)a.n * (F - 1) * p.C + a.c;
    const int stop = (int)min((int64_t)end + F - 1, (int64_t)kMaxTokens + 16);
    Run<T, V> xn[kGradAhead], gn[kGradAhead], before[F];
    auto fetch = [&](int t0) {                   // (as in causal_kernel)
        if (len == 0) return;
#pragma unroll
        for (int k = 0; k < kGradAhead; ++k) {
            xn[k] = load_some<V>(x + min(t0 + k, len - 1) * p.x_l, a.nv);
            gn[k] = load_some<V>(dout + min(t0 + k, len - 1) * p.g_l, a.nv);
        }
    };
#pragma unroll
    for (int r = 0; r < F - 1; ++r) {
        const int t = a.t0 - (F - 1) + r;
        before[r] = Run<T, V>{};
        if (t >= 0) {
            if (len) before[r] = load_some<V>(x + min(t, len - 1) * p.x_l, a.nv);
        } else if (p.state) {
            before[r] = load_some<V>((const T*)p.state + first + (int64_t)(F - 1 + t) * p.C, a.nv);
        }
    }
#pragma unroll
    for (int k = 0; k < kGradAhead; ++k) xn[k] = gn[k] = Run<T, V>{};
    fetch(a.t0);
    float w[F][V], bias[V] = {}, rows[F][V], ds[F][V] = {}, sum[F + 1][V] = {};
    constexpr bool kJoin = (F + 1) * V <= 10;
    auto join = [&] {
#pragma unroll
        for (int q = 0; q <= F; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                acc[q][i] += sum[q][i];
                sum[q][i] = 0.f;
            }
    };
    load_filter<T, F, V>((const T*)p.filt, a.c, a.nv, w);
    if (p.bias) load_some<V>((const T*)p.bias + a.c, a.nv, bias);
#pragma unroll
    for (int r = 0; r < F - 1; ++r)              // rows[1 ..]: they move down by one before each token
#pragma unroll
        for (int i = 0; i < V; ++i) rows[r + 1][i] = before[r][i];
    for (int t0 = a.t0; t0 < stop; t0 += kGradAhead) {
        Run<T, V> xc[kGradAhead], gc[kGradAhead];
#pragma unroll
        for (int k = 0; k < kGradAhead; ++k) {
            xc[k] = xn[k];
            gc[k] = gn[k];
        }
        if (t0 + kGradAhead < stop) fetch(t0 + kGradAhead);
#pragma unroll
        for (int k = 0; k < kGradAhead; ++k) {
            const int t = t0 + k;
#pragma unroll
            for (int i = 0; i < V; ++i) {
#pragma unroll
                for (int j = 0; j < F - 1; ++j) { rows[j][i] = rows[j + 1][i]; ds[j][i] = ds[j + 1][i]; }
                rows[F - 1][i] = xc[k][i];
                float s = bias[i], d = gc[k][i];
#pragma unroll
                for (int j = 0; j < F; ++j) s = __builtin_fmaf(w[j][i], rows[j][i], s);
                if (p.silu) {
                    const float sg = sigmoid(s);
                    d *= sg * (1.f + s * (1.f - sg));
                }
                d = t < len ? d : 0.f;
                ds[F - 1][i] = d;
                if (t < min(end, len)) {             // (not 0 times what stands before a sequence without tokens)
#pragma unroll
                    for (int j = 0; j < F; ++j) sum[j][i] = __builtin_fmaf(d, rows[j][i], sum[j][i]);
                    sum[F][i] += d;
                }
            }
            // the row that has all of its terms now; before token 0 it is one of the state
            const int r = t - (F - 1);
            if (r < end && (r >= a.t0 || (a.t0 == 0 && p.dstate))) {
                float v[V] = {};
                if (r >= 0 && t < len) {
#pragma unroll
                    for (int j = 0; j < F; ++j)
#pragma unroll
                        for (int i = 0; i < V; ++i) v[i] = __builtin_fmaf(w[j][i], ds[F - 1 - j][i], v[i]);
                } else {
                    // beside the sequence there are no terms: 0 times a filter that is not finite would be NaN
#pragma unroll
                    for (int j = 0; j < F; ++j)
                        if (t >= j && t - j < len) {
#pragma unroll
                            for (int i = 0; i < V; ++i) v[i] = __builtin_fmaf(w[j][i], ds[F - 1 - j][i], v[i]);
                        }
                }
                const int i = r - len + F - 1;               // of state_out, if it went there
                if (p.dstate_out && i >= 0 && i < F - 1) {
                    float e[V];
                    load_some<V>((const T*)p.dstate_out + first + (int64_t)i * p.C, a.nv, e);
                    for (int k2 = 0; k2 < V; ++k2) v[k2] += e[k2];
                }
                if (r >= 0) store_some<V>(dx + r * p.d_l, a.nv, v);
                else store_some<V>((T*)p.dstate + first + (int64_t)(F - 1 + r) * p.C, a.nv, v);
            }
        }
        if (kJoin && (t0 - a.t0) % kGradSum == kGradSum - kGradAhead) join();
    }
    join();
}

template <typename T, int F, int V>
__global__ void __launch_bounds__(kThreads)
causal_grad_kernel(CausalParams p)
{
    __shared__ float red[kThreads * V * (F + 1)];
    const Place a = place_of<V>(p);
    float acc[F + 1][V] = {};
    if (a.ok && a.whole) causal_grad_strip<T, F, V, true>(p, a, acc);
    else if (a.ok) causal_grad_strip<T, F, V, false>(p, a, acc);
    if (!p.part) return;
    // [strip][filter tap, or bias][channel]
    const int wide = p.vb * V, values = wide * (F + 1);
    if (a.strip < p.sb) {
#pragma unroll
        for (int q = 0; q <= F; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) red[(a.strip * (F + 1) + q) * wide + a.run * V + i] = acc[q][i];
    }
    __syncthreads();
    float* part = p.part + a.row * (F + 1) * p.C + a.c0;
    for (int at = threadIdx.x; at < values; at += kThreads) {
        const int q = at / wide, c = at - q * wide;
        double s = 0.;
        for (int k = 0; k < p.sb; ++k) s += red[k * values + at];
        if (a.c0 + c < p.C) part[(int64_t)q * p.C + c] = (float)s;
    }
}

// dfilt[c][j] and dbias[c] from `rows` parts [F + 1][C]: four waves take a quarter of the rows each.
__global__ void __launch_bounds__(kThreads)
causal_sum_kernel(const float* part, int64_t rows, int C, int F, float* dfilt, float* dbias)
{
    __shared__ double red[kThreads];
    const int64_t col = (int64_t)blockIdx.x * kWave + threadIdx.x % kWave, cols = (int64_t)(F + 1) * C;
    const int w = threadIdx.x / kWave;
    double s = 0.;
    if (col < cols) {
#pragma unroll 8
        for (int64_t r = w; r < rows; r += 4) s += part[r * cols + col];
    }
    red[threadIdx.x] = s;
    __syncthreads();
    if (w || col >= cols) return;
    s = (red[threadIdx.x] + red[threadIdx.x + 64]) + (red[threadIdx.x + 128] + red[threadIdx.x + 192]);
    const int j = (int)(col / C), c = (int)(col % C);
    if (j < F) {
        if (dfilt) dfilt[(int64_t)c * F + j] = (float)s;
    } else if (dbias) {
        dbias[c] = (float)s;
    }
}

// One token of each row: the window of F-1 rows is read, used with the new one and written back moved by one.
template <typename T, int F, int V>
__global__ void __launch_bounds__(kThreads)
causal_step_kernel(CausalParams p)
{
    const int n = blockIdx.x / p.vgroups;
    const int slot = slot_of(p.slots, n, p.M);
    const int c = ((blockIdx.x - n * p.vgroups) * kThreads + threadIdx.x) * V, nv = min(V, p.C - c);
    if (nv <= 0) return;
    T* out = (T*)p.out + n * p.o_n + c;
    float y[V] = {};
    if (slot >= 0) {
        float w[F][V], rows[F][V];
        T* st = (T*)p.state_out + (int64_t)slot * (F - 1) * p.C + c;
#pragma unroll
        for (int r = 0; r < F - 1; ++r) load_some<V>(st + (int64_t)r * p.C, nv, rows[r]);
        load_some<V>((const T*)p.x + n * p.x_n + c, nv, rows[F - 1]);
        load_filter<T, F, V>((const T*)p.filt, c, nv, w);
        if (p.bias) load_some<V>((const T*)p.bias + c, nv, y);
#pragma unroll
        for (int r = 0; r < F - 1; ++r) store_some<V>(st + (int64_t)r * p.C, nv, rows[r + 1]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float s = y[i];
#pragma unroll
            for (int j = 0; j < F; ++j) s = __builtin_fmaf(w[j][i], rows[j][i], s);
            y[i] = p.silu ? s * sigmoid(s) : s;
        }
    }
    store_some<V>(out, nv, y);
}

// ---- host ------------------------------------------------------------------------------------------------------------

constexpr int kMaxTaps = 8;

bool sizes_ok(const dconv_causal_args& a)
{
    return a.N > 0 && a.L > 0 && a.L <= kMaxTokens && a.C > 0 && a.C <= kMaxChannels && a.F > 0 && a.F <= kMaxTaps &&
           (double)a.N * a.L * a.C < kMaxElements;
}

// Elements of a run: 16 bytes.  In gradients two, as windows, sums and two inputs of more leave too few waves to hide a load
// behind, and four of an odd number of channels, whose last run is cut.  Sizes alone choose, as the workspace depends on it; that rows
// begin at odd elements makes no difference.  Measured, us with two and four, 4 taps:
//   bf16  4 x 2048 x 2048 32 and 35 (31 and 34 as slices of rows of 4097), x 2049 52 and 46, x 4097 117 and 89, 3 x 1021 x 770 16 and 21
//   fp32  4 x 2048 x 2048 55 and 61 (58 and 66 as slices of rows of 4097), x 2049 82 and 75, x 4097 188 and 137, 3 x 1021 x 770 17 and 23
int run_of(const dconv_causal_args& a, bool grad) { return !grad ? 16 / token_bytes(a.dtype) : a.C % 2 ? 4 : 2; }

// The length of a strip: long ones read fewer rows twice, short ones fill the chip.  Runs and strips of a workgroup (at most
// 256 threads, `most` runs): a short call's gradient has 32 runs by 8 strips, so that more of its sums are joined in
// LDS; measured, us with 64 and 32: 512 x 4096 bf16 11.8 and 10.5, 256 x 256 fp32 10.2 and 9.5, 8 x 2048 x 4096 bf16 99 and 105.
void lay_out(const dconv_causal_args& a, bool grad, CausalParams* p)
{
    const int V = run_of(a, grad), runs = (a.C - 1) / V + 1;
    p->strip = grad ? 128 : 32;
    while (p->strip > kAhead && (double)a.N * runs * ((a.L + p->strip - 1) / p->strip) < 262144.0) p->strip /= 2;
    const int most = !grad ? kThreads : p->strip >= 64 ? 64 : 32;
    p->vgroups = (runs + most - 1) / most;
    p->vb = (runs + p->vgroups - 1) / p->vgroups;
    p->sb = kThreads / p->vb;
    const int64_t strips = ((int64_t)a.L + p->strip - 1) / p->strip;
    if (strips < p->sb) p->sb = (int)strips;
    p->sgroups = (int)((strips + p->sb - 1) / p->sb);
    p->total = (int64_t)a.N * p->sgroups * p->vgroups;
}

int check(const dconv_causal_args* a, bool step, bool grad)
{
    if (!a) return DCONV_NULL_POINTER;
    const int e = token_bytes(a->dtype);
    if (!e) return DCONV_UNSUPPORTED;
    if (!sizes_ok(*a) || (step && (a->L != 1 || a->M <= 0 || (!a->slots && a->M < a->N)))) return DCONV_BAD_SHAPE;
    if (!a->x.p || !a->filt || (!grad && !a->out.p) || (grad && (!a->dout.p || !a->dx.p))) return DCONV_NULL_POINTER;
    if (step && a->F > 1 && !a->state_out) return DCONV_NULL_POINTER;
    // (rows are read by the strips on both sides of them)
    if (!step && (grad ? a->dx.p == a->x.p || a->dx.p == a->dout.p : a->out.p == a->x.p)) return DCONV_BAD_SHAPE;
    for (const void* q : {(const void*)a->x.p, (const void*)a->out.p, (const void*)a->dout.p, (const void*)a->dx.p, a->filt,
                          a->bias, a->state, (const void*)a->state_out, a->dstate_out, (const void*)a->dstate})
        if (!aligned_to(q, e)) return DCONV_BAD_SHAPE;
    for (const void* q : {(const void*)a->dfilt, (const void*)a->dbias, (const void*)a->lengths, (const void*)a->slots})
        if (!aligned_to(q, 4)) return DCONV_BAD_SHAPE;
    return DCONV_OK;
}

CausalParams params_of(const dconv_causal_args& a)
{
    CausalParams p{};
    p.x = a.x.p; p.filt = a.filt; p.bias = a.bias; p.state = a.state; p.dout = a.dout.p; p.dstate_out = a.dstate_out;
    p.out = a.out.p; p.state_out = a.state_out; p.dx = a.dx.p; p.dstate = a.dstate;
    p.lengths = a.lengths; p.slots = a.slots;
    p.x_n = a.x.sn; p.x_l = a.x.sl; p.o_n = a.out.sn; p.o_l = a.out.sl;
    p.g_n = a.dout.sn; p.g_l = a.dout.sl; p.d_n = a.dx.sn; p.d_l = a.dx.sl;
    p.L = a.L; p.C = a.C; p.M = a.M; p.silu = a.silu;
    return p;
}

enum class Form { kPrompt, kGrad, kStep };

template <typename T, int F> int launch(Form form, int run, const CausalParams& p, hipStream_t st)
{
    constexpr int V = 16 / sizeof(T);
    if (p.total > kMaxThreads / kThreads) return DCONV_BAD_SHAPE;
    const dim3 grid((unsigned)p.total);
    begin_launch();
    switch (form) {
    case Form::kPrompt: hipLaunchKernelGGL((causal_kernel<T, F, V>), grid, dim3(kThreads), 0, st, p); break;
    case Form::kGrad:
        if (run == 4) hipLaunchKernelGGL((causal_grad_kernel<T, F, 4>), grid, dim3(kThreads), 0, st, p);
        else hipLaunchKernelGGL((causal_grad_kernel<T, F, 2>), grid, dim3(kThreads), 0, st, p);
        break;
    case Form::kStep: hipLaunchKernelGGL((causal_step_kernel<T, F, V>), grid, dim3(kThreads), 0, st, p); break;
    }
    return launch_status();
}

template <typename T> int launch_taps(Form form, int F, int run, const CausalParams& p, hipStream_t st)
{
    switch (F) {
    case 1: return launch<T, 1>(form, run, p, st);
    case 2: return launch<T, 2>(form, run, p, st);
    case 3: return launch<T, 3>(form, run, p, st);
    case 4: return launch<T, 4>(form, run, p, st);
    case 5: return launch<T, 5>(form, run, p, st);
    case 6: return launch<T, 6>(form, run, p, st);
    case 7: return launch<T, 7>(form, run, p, st);
    default: return launch<T, 8>(form, run, p, st);
    }
}

int launch_typed(Form form, const dconv_causal_args& a, const CausalParams& p, hipStream_t st)
{
    const int run = run_of(a, form == Form::kGrad);
    switch (a.dtype) {
    case DCONV_DTYPE_F16: return launch_taps<_Float16>(form, a.F, run, p, st);
    case DCONV_DTYPE_BF16: return launch_taps<__bf16>(form, a.F, run, p, st);
    default: return launch_taps<float>(form, a.F, run, p, st);
    }
}

int64_t part_rows(const CausalParams& p) { return p.total / p.vgroups; }

// Of causal_sum_kernel, which has more workgroups than causal_grad_kernel where there are few tokens.
int64_t sum_blocks(const dconv_causal_args& a) { return ((int64_t)(a.F + 1) * a.C + kWave - 1) / kWave; }
bool sums_fit(const dconv_causal_args& a) { return sum_blocks(a) <= kMaxThreads / kThreads; }

}  // namespace

}  // namespace dconv

using namespace dconv;

extern "C" {

int dconv_causal(const dconv_causal_args* a, void* stream)
{
    const int rc = check(a, false, false);
    if (rc != DCONV_OK) return rc;
    CausalParams p = params_of(*a);
    lay_out(*a, false, &p);
    return launch_typed(Form::kPrompt, *a, p, (hipStream_t)stream);
}

long long dconv_causal_workspace(const dconv_causal_args* a)
{
    if (!a || !token_bytes(a->dtype) || !sizes_ok(*a) || !sums_fit(*a)) return -1;
    CausalParams p{};
    lay_out(*a, true, &p);
    return part_rows(p) * (a->F + 1) * a->C * 4;
}

int dconv_causal_grad(const dconv_causal_args* a, void* stream)
{
    int rc = check(a, false, true);
    if (rc != DCONV_OK) return rc;
    CausalParams p = params_of(*a);
    lay_out(*a, true, &p);
    const bool sums = a->dfilt || a->dbias;
    if (sums) {
        if (!sums_fit(*a)) return DCONV_BAD_SHAPE;
        if (!a->workspace) return DCONV_NULL_POINTER;
        if (!aligned_to(a->workspace, 16)) return DCONV_BAD_SHAPE;
        if (a->workspace_bytes < dconv_causal_workspace(a)) return DCONV_SCRATCH_EXCEEDED;
        p.part = (float*)a->workspace;
    }
    rc = launch_typed(Form::kGrad, *a, p, (hipStream_t)stream);
    if (rc != DCONV_OK || !sums) return rc;
    begin_launch();
    hipLaunchKernelGGL(causal_sum_kernel, dim3((unsigned)sum_blocks(*a)), dim3(kThreads), 0, (hipStream_t)stream, p.part,
                       part_rows(p), a->C, a->F, a->dfilt, a->dbias);
    return launch_status();
}

int dconv_causal_step(const dconv_causal_args* a, void* stream)
{
    const int rc = check(a, true, false);
    if (rc != DCONV_OK) return rc;
    CausalParams p = params_of(*a);
    const int per = kThreads * (16 / token_bytes(a->dtype));
    p.vgroups = (a->C - 1) / per + 1;
    p.total = (int64_t)a->N * p.vgroups;
    return launch_typed(Form::kStep, *a, p, (hipStream_t)stream);
}

}  // extern "C"
