// What the forward and the backward pass of layer norm on shares have in common (spin_layernorm, spin_layernorm_grad): HBM streams with a chain of truncations in the middle of
// each row.
//
// A row belongs to one wave (up to 256 words) or one workgroup, a thread the columns t, t + threads, ..  Everything that the row's sums are made of is read
// before them and what comes of it stays in registers, so that a row is read once.  The chain of truncations between, some tens of dependent steps on one word a party, is
// run by one wave, a lane a party, from words that were brought into LDS while the rows were read; the opened sums go over eight lanes by DPP.
#pragma once
#include "linear.hpp"
#include "limb_common.hpp"

namespace spin {
namespace {

// ---- sums over lanes ------------------------------------------------------------------------------------------
template <int CONTROL, class T> __device__ inline T moved(T v)
{
    if constexpr (sizeof(T) == 8) {
        const u32 low = __builtin_amdgcn_mov_dpp((int)(u32)v, CONTROL, 0xf, 0xf, true), high = __builtin_amdgcn_mov_dpp((int)(u32)(v >> 32), CONTROL, 0xf, 0xf, true);
        return (T)low | (T)high << 32;
    } else {
        return (T)__builtin_amdgcn_mov_dpp((int)v, CONTROL, 0xf, 0xf, true);
    }
}
constexpr int kNext = 0xB1, kNextPair = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;    // lane ^ 1, lane ^ 2, 7 - lane of 8, 15 - lane of 16
template <class T> __device__ inline T sum8(T v)
{
    v += moved<kNext>(v);
    v += moved<kNextPair>(v);
    return v + moved<kHalfMirror>(v);
}
template <class T> __device__ inline T lane_of(T v, int lane)
{
    if constexpr (sizeof(T) == 8) return (T)(u32)__builtin_amdgcn_readlane((int)(u32)v, lane) | (T)(u32)__builtin_amdgcn_readlane((int)(u32)(v >> 32), lane) << 32;
    else return (T)__builtin_amdgcn_readlane((int)v, lane);
}
template <class T> __device__ inline T wave_sum(T v)
{
    v = sum8(v);
    v += moved<kMirror>(v);
    return lane_of(v, 0) + lane_of(v, 16) + lane_of(v, 32) + lane_of(v, 48);
}

// ---- the chain of a row ---------------------------------------------------------------------------------------
// Lane i of every eight has party i's share; word k of party i is at words[k * NP + i].
template <int NP, class T> struct Chain {
    const T *words;
    int i = threadIdx.x % 8;
    __device__ T at(int k) const { return words[k * NP + min(i, NP - 1)]; }
    __device__ T sum(T share) const { return sum8(i < NP ? share : 0); }
    __device__ T truncate(T share, int k, int f) const     // with words k, k + 1, k + 2
    {
        Opened<T> c{f};
        c.add(sum(share + at(k)));
        return c.truncated(i, at(k + 1), at(k + 2));
    }
    __device__ T open(T share, int k) const { return sum(share - at(k)); }
    __device__ T public_word(T v) const { return i == 0 ? v : 0; }
    // A share of x . y beside dealt word c; x is opened to e against word a, y to f against word b.
    __device__ T product(int c, T e, int a, T f, int b) const { return at(c) + e * (at(b) + public_word(f)) + at(a) * f; }
};

template <int WAVES> constexpr int kRowsAtOnce = WAVES == 1 ? 4 : 1;           // of a workgroup
template <int WAVES> constexpr int kNormBlock = 64 * WAVES * kRowsAtOnce<WAVES>;
template <int WAVES> __device__ inline void row_barrier()
{
    if constexpr (WAVES > 1) {
        __syncthreads();
    } else {                               // a wave's accesses to LDS stay in order
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
}

// A column, new to the compiler: it would carry an address for every array, party and column along, and keep words from where they are read first to where they are used last.
__device__ inline void make_new(u32 &column)
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" : "+v"(column));
}

template <class F> constexpr void for_dim(int rows, int dim, F &&fn)    // waves a row, words a thread
{
    constexpr std::integral_constant<int, 4> four{};
    switch (norm_waves(rows, dim)) {
    case 1: fn(std::integral_constant<int, 1>(), four); break;
    case 4: fn(four, four); break;
    default:
        if (dim <= 2048) fn(std::integral_constant<int, 16>(), std::integral_constant<int, 2>());
        else if (dim <= 4096) fn(std::integral_constant<int, 16>(), four);
        else fn(std::integral_constant<int, 16>(), std::integral_constant<int, 8>());
    }
}

}  // namespace
}  // namespace spin
