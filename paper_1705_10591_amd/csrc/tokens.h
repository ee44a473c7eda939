// What the operators over tokens (causal.hip, scan*.hip) share: element types, runs of channels, activations.
#pragma once
#include "common.h"

namespace dconv {

// N elements that lie next to each other.  The hardware takes loads and stores of up to 16 bytes at any address (an odd
// number of channels moves every other row off its alignment), so that there is one kernel for all alignments.
template <typename T, int N> struct Run {
    typedef T vt __attribute__((ext_vector_type(N)));
    vt v;
    __device__ __forceinline__ float operator[](int i) const { return (float)v[i]; }
};
template <typename T> struct Run<T, 1> {
    T v;
    __device__ __forceinline__ float operator[](int) const { return (float)v; }
};

template <int N, typename T> __device__ __forceinline__ Run<T, N> load_run(const T* p)
{
    Run<T, N> r;
    __builtin_memcpy(&r.v, p, sizeof(T) * N);
    return r;
}

// ... of which only the first n exist; the others read as 0.  Nothing is converted here: what is done with a loaded
// value waits for it, and loads are to be under way together.
template <int N, typename T> __device__ __forceinline__ Run<T, N> load_some(const T* p, int n)
{
    Run<T, N> r;
    if (n >= N) {
        r = load_run<N>(p);
    } else if constexpr (N == 1) {
        r.v = (T)0.f;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) r.v[i] = i < n ? p[i] : (T)0.f;
    }
    return r;
}
template <int N, typename T> __device__ __forceinline__ void load_some(const T* p, int n, float (&v)[N])
{
    const Run<T, N> r = load_some<N>(p, n);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = r[i];
}

// v rounded to nearest even; only the first n exist
template <int N, typename T> __device__ __forceinline__ void store_some(T* p, int n, const float (&v)[N])
{
    if constexpr (N == 1) {
        if (n > 0) p[0] = (T)v[0];
    } else {
        typename Run<T, N>::vt t;
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = (T)v[i];
        if (n >= N) {
            __builtin_memcpy(p, &t, sizeof(T) * N);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < n) p[i] = t[i];
        }
    }
}

// All waves of the workgroup have come here and their LDS writes are seen.  __syncthreads() would also wait for the global
// loads that are under way.
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

constexpr int kMaxTokens = 1 << 30;      // of a sequence: token numbers and what is added to them fit 32 bits
constexpr int kMaxChannels = 1 << 30;    // likewise
constexpr int64_t kMaxThreads = 4294967295LL;   // of a launch: a packet holds 32 bits of them
constexpr double kMaxElements = 1.1e18;  // of a tensor, 2^60: sizes in 64 bits do not overflow
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rcp_(float x) { return __builtin_amdgcn_rcpf(x); }

// 1 / (1 + e^-x): exp2 and the reciprocal are good to 1 ulp each, and where e^-x overflows the quotient is 0 as it should be.
__device__ __forceinline__ float sigmoid(float x) { return rcp_(1.f + exp2_(-kLog2e * x)); }

// log(1 + e^x) = max(x, 0) + log(1 + e), e = e^-|x| at most 1.  w = 1 + e rounds off c = e - (w - 1), up to 2^-24; since
// log(1 + e) = log(w) + c / w to first order and c (1 - 1 / w) is at most 2^-24 e, adding c itself leaves errors of an ulp,
// small steps (e << 1, where log(w) has few digits of e) among them.
__device__ __forceinline__ float softplus(float x)
{
    const float e = exp2_(-kLog2e * __builtin_fabsf(x)), w = 1.f + e;
    return fmaxf(x, 0.f) + __builtin_fmaf(kLn2, __builtin_amdgcn_logf(w), e - (w - 1.f));
}

// Tokens of sequence n that count.
__device__ __forceinline__ int length_of(const int* lengths, int n, int L)
{
    return lengths ? min(max(lengths[n], 0), L) : L;
}

// The row of a cache of M that row n of a step works on, -1 for padding: slots outside the cache, and those that an earlier
// row has named.  All threads of a workgroup call it with the same n.
__device__ __forceinline__ int slot_of(const int* slots, int n, int M)
{
    if (!slots) return n;
    const int s = slots[n];
    int twice = 0;
    for (int i = threadIdx.x; i < n; i += blockDim.x) twice |= slots[i] == s;
    return __syncthreads_or(twice) || s < 0 || s >= M ? -1 : s;
}

// Workgroups go round the eight XCDs in turn, each with an L2 of its own: neighbours that share rows get numbers that
// are eight apart.
__device__ __forceinline__ int64_t near_block(int64_t b, int64_t total)
{
    const int64_t each = total >> 3, rest = total & 7, x = b & 7, i = b >> 3;
    return x * each + (x < rest ? x : rest) + i;
}

inline bool aligned_to(const void* p, int bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
inline int token_bytes(int dtype)
{
    return dtype == DCONV_DTYPE_F32 ? 4 : dtype == DCONV_DTYPE_F16 || dtype == DCONV_DTYPE_BF16 ? 2 : 0;
}

}  // namespace dconv
