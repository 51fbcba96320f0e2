// Linear attention with a decay for each head (pxr_linear_attention_* in include/pxr.h).  gfx950 only.
//
//   S_t = (t begins an episode ? 0 : g S_{t-1}) + k_t v_t^T,   o_t = scale S_t^T q_t,   g = exp(log_decay_h)
//
// Every pass over a rollout is one form, a scan: out_i = out_scale sum_{j <= i} g^(i-j) key_scale (x_i . y_j) z_j + what the
// state before the scan adds.  The forward pass is the scan of (q, k, v).  With do the gradient of the outputs,
//   dq is the scan of (do, v, k): dq_t = scale S_t do_t, and the states are the forward pass' transposed;
//   dk and dv are scans from the last step to the first, of (v, do, q) and of (k, q, do): their state
//     R_t = scale q_t do_t^T + (t + 1 begins an episode ? 0 : g R_{t+1}) gives dk_t = R_t v_t, dv_t = R_t^T k_t.
//
// A scan takes C = 32 steps at a time.  With positions i, j in such a chunk, S the state before it and n of its steps there:
//   P_ij = g^(i-j) key_scale (x_i . y_j) where j <= i and no episode begins in (j, i], else 0
//   out_i = out_scale (sum_j P_ij z_j + [no episode begins up to i] g^(i+1) S^T x_i)
//   S <- [no episode begins] g^n S + sum_j [no episode begins after j] g^(n-1-j) key_scale y_j z_j^T
// and mirrored from the end for the reverse scans, whose state decays on its way out of a step instead of on its way in.
//
// All four products run on the matrix cores, 32 x 32 tiles of 16 summed values, bfloat16 operands, sums in fp32.  A wavefront has 32 columns of z and of the
// state; its state stays in its accumulators [a][32] for the whole scan.  What makes that cheap is that a product's result lies in a lane as the next product
// wants its operand: a lane has one column and, of every 16 rows, the eight 4h .. 4h+3, 8+4h .. 8+4h+3 (h = lane / 32), and an operand's lane has one row and
// eight values of the axis that is summed over, whose order is free as long as both operands agree on it.  So P^T = y x^T (a column is a step i) is the right
// operand of out^T = z^T P^T, and S the left one of S^T x^T, without a move between lanes.  z and y are also wanted with steps along the summed axis: by the
// transposing LDS read.
//
// Roundings.  What is fp32 (P, S, the weighted z, fp32 tensors) goes in as a sum of three bfloat16 parts.  Beside bfloat16 tensors, whose values are one part, the
// three are 8 bits each, cut off one after the other: their sum is the value, all products are formed, and an output has fp32's rounding of sums and its own of
// 2^-9 (P and S as two rounded parts, which leave out 2^-17, took 366 us for the gradients of 512 x 256 with 8 heads of 64, 393 so, rollouts 1 to 4 % less).  Of fp32
// tensors: rounded parts, six products of the nine, the rest is below 2^-25; six instructions of 32 clocks instead of eight of 64 (128 x 256 with 8 heads of 128: 295 us
// with fp32 operands, 243 so; gradients 760, 593).  The last parts of values under 2^-110 are below the smallest normal number and go: such values keep fewer digits.
//
// Bound by memory where heads and environments fill the device: 512 x 256 with 8 heads of 64 in bfloat16 179 us (3.7 TB/s), its gradients 399 (2.9; each step's
// rows are read by up to three scans, from one die's L2, and the vector units are 78 % busy), 4000 single steps of 8 heads 199 (5.3).  Few long rollouts are cut into
// segments, whose own states are found first and joined: 20000 steps of 8 heads of 64 x 128 75 us, twice the reading.  A chunk alone on a compute unit takes 3 us, 5 in
// fp32: instructions, one after the other.  Heads of more than 128 do not fit the registers, and the loop over chunks keeps about 100 of a lane's values in
// scratch: 128 x 256 with 4 heads of 256 1.01 ms in bfloat16, its gradients 2.9 (floors 0.11 and 0.17).
// (Two figures side by side, here and below, were taken together when that choice was made; what was changed since has moved both.)
//
// Steps that hold an infinity or NaN (or what rounds to an infinity of bfloat16) in y or z are taken one by one: 0 times such a value would reach steps that it
// must not.  Where it does reach, parts of an infinity are no numbers, so that a NaN may come out in its place.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "pxr_internal.h"
#include "steps.h"

namespace pxr {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __bf16* p) { return (float)*p; }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__bf16* p, float v) { *p = (__bf16)v; }  // round to nearest even

// One scan: x, y [.., a], z [.., b] -> out [.., b]; state [a][b] per (environment, head), with strides of its own.
struct Scan {
    pxr_tokens x, y, z, out;
    uint32_t a, b;
    const float* state_in;  // null = zeros
    float* state_out;       // null = not wanted
    uint32_t state_row, state_col;
    const float* before;  // [segments - 1][environments * heads][a * b], strides as above: the states before the segments but the first
    float out_scale, key_scale;
    uint32_t reverse;
};

struct Scans {
    Scan s[3];
};

// How the steps are cut: a workgroup takes one segment of one (environment, head) and 32 columns a wavefront.
struct Cut {
    uint32_t n_heads, rows, n_steps;  // rows = environments * heads
    uint32_t segments, seg_steps, tiles, waves, width;  // width: a's, padded
    const LinearAttentionHead* heads;
    const uint8_t* resets;
    int64_t resets_env, resets_step;
};

template <class T>
__device__ __forceinline__ T* head_of(const pxr_tokens& t, uint32_t e, uint32_t h) {
    return static_cast<T*>(t.data) + ((int64_t)e * t.env + (int64_t)h * t.head);
}

// ---- operands: eight values of the summed axis, positions 4h + {0..3, 8..11} of a run of 16

// Eight values as the sum of n bfloat16 operands, the largest first.
template <int n>
struct Parts {
    bf16x8 part[n];
};

// fp32 values as three parts, for products with values of T: cut off to 8 bits each where those are one part (their sum is the value), rounded to nearest where
// they are three themselves (the products that are left out are small).
template <class T>
__device__ __forceinline__ Parts<3> split(f32x8 rest) {
    constexpr bool kCut = sizeof(T) == 2;
    Parts<3> f;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        u32x4 w;  // (two values an instruction: conversions of eight at once come out one by one)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = rest[2 * i], hi = rest[2 * i + 1];
            if (kCut)
                w[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);  // the upper halves of both
            else
                w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));  // round to nearest even
            if (k < 2) {
                rest[2 * i] = lo - __uint_as_float(kCut ? __float_as_uint(lo) & 0xFFFF0000u : w[i] << 16);
                rest[2 * i + 1] = hi - __uint_as_float(kCut ? __float_as_uint(hi) & 0xFFFF0000u : w[i] & 0xFFFF0000u);
            }
        }
        f.part[k] = __builtin_bit_cast(bf16x8, w);
    }
    return f;
}

// Products of parts whose share of the result is above a third part's rounding, the smallest first (all of them where one operand is one part).
template <int n, int m>
__device__ __forceinline__ f32x16 mma(const Parts<n>& a, const Parts<m>& b, f32x16 c) {
#pragma unroll
    for (int order = (n > m ? n : m) - 1; order >= 0; --order)
#pragma unroll
        for (int i = 0; i < n; ++i)
            if (order - i >= 0 && order - i < m) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.part[i], b.part[order - i], c, 0, 0, 0);
    return c;
}

// Tiles of x and y have every run of 16 columns in the order 0-3, 8-11, 4-7, 12-15, so that a lane's eight values are 16 bytes that lie together.  With four a column
// apart a row, 16 rows of them at one column lie in different banks.
__device__ __forceinline__ constexpr uint32_t place(uint32_t c) { return (c & ~12u) | ((c & 4u) << 1) | ((c & 8u) >> 1); }

// From rows that lie along the summed axis: p = the row's run of 16 in LDS, `plane` values from part to part.
template <int n>
__device__ __forceinline__ Parts<n> along(const __bf16* p, uint32_t plane, uint32_t h) {
    Parts<n> f;
#pragma unroll
    for (int k = 0; k < n; ++k) f.part[k] = *reinterpret_cast<const bf16x8*>(p + k * plane + 8 * h);
    return f;
}

// From 16 rows that lie across it: p = the first row's 32 columns in LDS, `stride` values from row to row; the lane's column is lane % 32.
template <bool kPlaced>
__device__ __forceinline__ bf16x8 across(const __bf16* p, uint32_t stride, uint32_t lane) {
    // The transposing read: lane i of 16 gives the address of four columns of row i / 4 and gets four rows of column i.
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const uint32_t h = lane >> 5, i = lane & 15u;
    const __bf16* q = p + (4 * h + (i >> 2)) * stride + (lane & 16u) + (kPlaced ? place(4 * (i & 3u)) : 4 * (i & 3u));
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)q);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(q + 8 * stride));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
template <bool kPlaced>
__device__ __forceinline__ f32x8 across(const float* p, uint32_t stride, uint32_t lane) {
    static_assert(!kPlaced);
    const float* q = p + (4 * (lane >> 5)) * stride + (lane & 31u);
    f32x8 f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = q[(e & 3) * stride + (e >> 2) * 8 * stride];
    return f;
}
template <int n>
__device__ __forceinline__ Parts<n> across_placed(const __bf16* p, uint32_t plane, uint32_t stride, uint32_t lane) {
    Parts<n> f;
#pragma unroll
    for (int k = 0; k < n; ++k) f.part[k] = across<true>(p + k * plane, stride, lane);
    return f;
}

__device__ __forceinline__ f32x8 values(const bf16x8& f) {
    const u32x4 w = __builtin_bit_cast(u32x4, f);
    f32x8 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
    return v;
}
__device__ __forceinline__ f32x8 values(const f32x8& f) { return f; }
__device__ __forceinline__ Parts<1> parts_of(const bf16x8& f) { return {{f}}; }
__device__ __forceinline__ Parts<3> parts_of(const f32x8& f) { return split<float>(f); }
// Half of a product's result in a lane, which is a run of 16 of its rows.
__device__ __forceinline__ f32x8 half(const f32x16& c, int k) {
    return k ? __builtin_shufflevector(c, c, 8, 9, 10, 11, 12, 13, 14, 15) : __builtin_shufflevector(c, c, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ f32x8 eight(const float* lo, const float* hi) {
    return __builtin_shufflevector(*reinterpret_cast<const f32x4*>(lo), *reinterpret_cast<const f32x4*>(hi), 0, 1, 2, 3, 4, 5, 6, 7);
}

// ---- tiles of steps in LDS: rows of `width` values (a multiple of 32), 16 bytes apart from each other so that 16 rows' words at one column lie in
// different banks

template <class T>
constexpr uint32_t kPad = 16 / sizeof(T);
// Parts of a value of x or y in LDS.
template <class T>
constexpr int kParts = sizeof(T) == 2 ? 1 : 3;

// The largest bit patterns of the values, without their signs.
template <class T>
struct Most;
template <>
struct Most<float> {
    uint32_t m = 0;
    __device__ __forceinline__ void with(uint32_t w) { m = max(m, w & 0x7FFFFFFFu); }
    __device__ __forceinline__ bool infinite() const { return m >= 0x7F7F8000u; }  // (what rounds to an infinity of bfloat16 among them)
};
template <>
struct Most<__bf16> {
    u16x2 m = {0, 0};
    __device__ __forceinline__ void with(uint32_t w) { m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu)); }
    __device__ __forceinline__ bool infinite() const { return max(m[0], m[1]) >= 0x7F80u; }
};

// A number that is the same in all lanes and in every chunk, as one that the compiler does not know to be: it would otherwise build the loop over
// chunks once for each answer that a test of it can have.
__device__ __forceinline__ uint32_t again(uint32_t v) {
    v = __builtin_amdgcn_readfirstlane(v);
    asm volatile("" : "+s"(v));
    return v;
}

// A chunk's steps on their way to a tile: C rows of `kWidth` values, dealt to kThreads lanes in vectors of 16 bytes.  The requests of a chunk go out
// together, a chunk ahead.  Rows may begin at any element (the memory takes 16-byte requests at any address).  What a lane asks for is in steps.h: what it
// asks for in place of rows past the last and vectors past a row's end is not written, or written as zeros.  The columns past d are zero from the start and
// nothing writes them.  Rows shorter than a vector are read value by value, when they are written.
// kOperand: a tile of x or y, its columns placed and fp32 values as three planes of bfloat16 parts.
template <class T, int kWidth, int kThreads, bool kOperand>
struct Steps {
    static constexpr bool kSplit = kOperand && sizeof(T) == 4;
    typedef std::conditional_t<kSplit, __bf16, T> E;  // of the tile
    typedef Dealt<sizeof(T), kWidth, kThreads> D;
    static constexpr uint32_t N = D::N, kPerRow = D::kPerRow, kCount = D::kCount, kRowsEach = D::kRowsEach, kStride = kWidth + kPad<E>, kPlane = C * kStride;
    uint32_t row, col, d;
    int64_t step, offset;  // values from row to row; the lane's first vector from the chunk's first value
    u32x4 v[kCount];

    __device__ __forceinline__ Steps(int64_t step, uint32_t d) : row(D::row(threadIdx.x)), col(D::col(threadIdx.x)), d(d), step(step), offset(D::offset(row, col, d, step)) {}
    // n >= 1 rows
    __device__ __forceinline__ void ask(const T* from, uint32_t n) {
        const uint32_t d = again(this->d);
        if (d < N) return forget();
#pragma unroll
        for (uint32_t i = 0; i < kCount; ++i) __builtin_memcpy(&v[i], D::request(from, i, n, row, col, d, step, offset), 16);
    }
    // What was asked for has been put; nothing is in flight.  (Without this the registers would be kept, and copied, from chunk to chunk.)
    __device__ __forceinline__ void forget() {
#pragma unroll
        for (uint32_t i = 0; i < kCount; ++i) asm volatile("" : "=v"(v[i]));
    }
    static __device__ __forceinline__ void put_one(E* row, uint32_t c, T e) {
        E* at = row + (kOperand ? place(c) : c);
        if constexpr (kSplit) {
            float rest = e;
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                at[k * kPlane] = (__bf16)rest;  // round to nearest even
                rest -= (float)at[k * kPlane];
            }
        } else {
            *at = e;
        }
    }
    // The tile's rows past n are zeros.  kCheck: collects bit patterns.
    template <bool kCheck>
    __device__ __forceinline__ void put(const T* from, E* tile, uint32_t n, Most<T>& most) {
        const uint32_t d = again(this->d);
        if (d < N) {
            for (uint32_t i = threadIdx.x; i < C * d; i += kThreads) {
                const uint32_t r = i / d, c = i - r * d;
                const T e = r < n ? from[(int64_t)r * step + c] : (T)0.0f;
                if (kCheck) most.with(sizeof(T) == 4 ? __builtin_bit_cast(uint32_t, (float)e) : __builtin_bit_cast(uint32_t, (float)e) >> 16);
                put_one(tile + r * kStride, c, e);
            }
            return;
        }
#pragma unroll
        for (uint32_t i = 0; i < kCount; ++i) {
            const uint32_t r = row + i * kRowsEach;
            if (C * kPerRow % kThreads && r >= (uint32_t)C) continue;
            u32x4 w = v[i];
            if (n < (uint32_t)C && r >= n) w = u32x4{0, 0, 0, 0};
            if (kCheck)
#pragma unroll
                for (int k = 0; k < 4; ++k) most.with(w[k]);
            if (col + N <= d) {
                if constexpr (kSplit) {
                    f32x4 rest = __builtin_bit_cast(f32x4, w);
#pragma unroll
                    for (int k = 0; k < 3; ++k) {
                        u32x2 p;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            p[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{rest[2 * i], rest[2 * i + 1]}, bf16x2));
                            rest[2 * i] -= __uint_as_float(p[i] << 16);
                            rest[2 * i + 1] -= __uint_as_float(p[i] & 0xFFFF0000u);
                        }
                        *reinterpret_cast<u32x2*>(tile + k * kPlane + r * kStride + place(col)) = p;
                    }
                } else if constexpr (kOperand) {
                    *reinterpret_cast<u32x2*>(tile + r * kStride + place(col)) = u32x2{w[0], w[1]};
                    *reinterpret_cast<u32x2*>(tile + r * kStride + place(col + 4)) = u32x2{w[2], w[3]};
                } else {
                    *reinterpret_cast<u32x4*>(tile + r * kStride + col) = w;
                }
            } else if (col < d) {
                T e[N];
                __builtin_memcpy(e, &w, 16);
#pragma unroll
                for (uint32_t k = 0; k < N; ++k) put_one(tile + r * kStride, d - N + k, e[k]);
            }
        }
    }
};

typedef uint32_t any_u32x4 __attribute__((ext_vector_type(4), aligned(2)));  // at the address of any value

// Positions of a chunk up to and including i, as bits.
__device__ __forceinline__ uint64_t up_to(uint32_t i) { return (2ull << i) - 1ull; }

constexpr uint32_t kLds = 160 * 1024;  // of a compute unit

// LDS of a workgroup.
constexpr uint32_t scan_lds(uint32_t element, uint32_t width, uint32_t waves, bool out) {
    return C * ((out ? 2 : 1) * (width + 8) * 2 * (element == 2 ? 1 : 3) + waves * 32 * element + 16) + (36 + 64 + waves * C + 2) * 4;
}

// Wavefronts that share a SIMD's registers.
constexpr uint32_t waves_per_simd(uint32_t width, uint32_t element) { return width <= 64u && element == 2u ? 3u : width <= 128u ? 2u : 1u; }

// A (a padded to 32, 64, 128 or 256), kWaves wavefronts; kOut: outputs (else the state after a segment alone, from zeros).
template <class T, int A, int kWaves, bool kOut>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(waves_per_simd(A, sizeof(T))))) void scan_kernel(
    const Scans scans, const Cut cut, uint32_t roles, float* local0, float* local1, uint32_t* whole0, uint32_t* whole1) {
    // (requests a chunk ahead take registers; where they do not fit, a chunk's requests go out together when it begins: 256 x 128 with 8 heads of 64 50 us
    // ahead, 53 not; with 4 of 128 x 64 37 not, 40 ahead)
    constexpr bool kAhead = A <= 64;
    constexpr uint32_t kThreads = kWaves * 64, kWidthZ = kWaves * 32, kStrideA = A + kPad<__bf16>, kStrideZ = kWidthZ + kPad<T>;
    constexpr uint32_t kPlane = C * kStrideA, kTile = kPlane * kParts<T>;  // of x and y
    extern __shared__ __align__(16) unsigned char lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, h32 = lane >> 5, col32 = lane & 31u;
    // Workgroups go to the eight dies in turn: those that read the same steps are eight apart, on one die and behind one L2.  So are eight
    // heads that follow each other, whose steps lie side by side in memory (512 x 256 bfloat16, 8 heads of 64: 202 -> 189 us, gradients 480 -> 436).
    const uint32_t per_die = cut.tiles * roles, group = blockIdx.x / (8u * per_die), in_group = blockIdx.x - group * 8u * per_die;
    const uint32_t item = group * 8u + (in_group & 7u), part = in_group >> 3, tile = part / roles, role = part - tile * roles;
    if (item >= cut.rows * (kOut ? cut.segments : cut.segments - 1u)) return;
    const uint32_t seg = item / cut.rows, dealt = item - seg * cut.rows, block = dealt & ~63u;
    const uint32_t row = block + 64u <= cut.rows ? block + ((dealt & 7u) << 3) + ((dealt >> 3) & 7u) : dealt, env = row / cut.n_heads, head = row - env * cut.n_heads;
    const Scan s = scans.s[role];
    const LinearAttentionHead& hd = cut.heads[head];
    const uint32_t n0 = tile * kWidthZ, col = n0 + wave * 32u + col32;
    __bf16* ys = reinterpret_cast<__bf16*>(lds);
    T* zs = reinterpret_cast<T*>(ys + kTile);
    __bf16* xs = reinterpret_cast<__bf16*>(zs + C * kStrideZ);
    float* pw = reinterpret_cast<float*>(xs + (kOut ? kTile : 0));  // g^0 .. g^C
    float* factor = pw + 36;                                               // of P by j - i + 31
    float* weight = factor + 64 + wave * (uint32_t)C;                      // a wavefront's g^(n-1-j)
    uint32_t* flag = reinterpret_cast<uint32_t*>(factor + 64 + kWaves * C);   // [2]
    for (uint32_t i = threadIdx.x; i <= (uint32_t)C; i += kThreads) pw[i] = hd.power[i];
    if (kOut && threadIdx.x < 63u) {
        const int gap = s.reverse ? (int)threadIdx.x - 31 : 31 - (int)threadIdx.x;
        factor[threadIdx.x] = gap >= 0 ? s.out_scale * s.key_scale * hd.power[max(gap, 0)] : 0.0f;
    }
    if (threadIdx.x < 2u) flag[threadIdx.x] = 0;
    const uint32_t widthB = min(s.b - n0, kWidthZ);
    if (s.a < (uint32_t)A || widthB < kWidthZ)
        for (uint32_t i = threadIdx.x; i < (kTile * (kOut ? 2 : 1) * 2 + C * kStrideZ * sizeof(T)) / 16u; i += kThreads) reinterpret_cast<uint4*>(lds)[i] = make_uint4(0, 0, 0, 0);

    const T *xh = head_of<const T>(s.x, env, head), *yh = head_of<const T>(s.y, env, head), *zh = head_of<const T>(s.z, env, head) + n0;
    T* oh = head_of<T>(s.out, env, head);
    const uint8_t* resets = cut.resets ? cut.resets + (int64_t)env * cut.resets_env : nullptr;
    // the segment's steps in the order in which they are taken; in reverse, position p of the scan is step n_steps - 1 - p
    const uint32_t begin = seg * cut.seg_steps, end = min(begin + cut.seg_steps, cut.n_steps);
    Steps<T, A, kThreads, true> y_steps(s.y.step, s.a), x_steps(s.x.step, s.a);
    Steps<T, kWidthZ, kThreads, false> z_steps(s.z.step, widthB);
    uint32_t reset = 0;
    const uint32_t has_resets = cut.resets != nullptr;
    const auto step_of = [&](uint32_t at, uint32_t n) { return first_step(again(s.reverse) != 0u, cut.n_steps, at, n); };  // a chunk's first step in memory
    const auto ask = [&](uint32_t at, uint32_t n) {
        const int64_t t = step_of(at, n);
        reset = again(has_resets) && lane < n ? resets[(t + lane) * cut.resets_step] : 0u;
        y_steps.ask(yh + t * s.y.step, n);
        z_steps.ask(zh + t * s.z.step, n);
        if (kOut) x_steps.ask(xh + t * s.x.step, n);
    };
    if (kAhead && begin < end) ask(begin, min((uint32_t)C, end - begin));

    // the state: a lane's column, rows (r & 3) + 8 (r >> 2) + 4 h32 of every 32
    f32x16 state[A / 32];
    const size_t cells = (size_t)s.a * s.b;
    const float* from = kOut ? (seg ? s.before + ((size_t)(seg - 1u) * cut.rows + row) * cells : s.state_in ? s.state_in + row * cells : nullptr) : nullptr;
    const uint32_t lane_cell = 4 * h32 * s.state_row + min(col, s.b - 1u) * s.state_col;  // (a state has at most 2^16 cells)
#pragma unroll
    for (int db = 0; db < A / 32; ++db) {
        const float* block = from + (size_t)db * 32 * s.state_row;
        if (!from || db * 32u >= s.a) {
            state[db] = (f32x16)0.0f;
            continue;
        } else if (db * 32u + 32u > s.a) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t d = db * 32 + (r & 3) + 8 * (r >> 2) + 4 * h32;
                const float v = from[min(d, s.a - 1u) * s.state_row + min(col, s.b - 1u) * s.state_col];
                state[db][r] = d < s.a ? v : 0.0f;
            }
        } else if (s.state_row == 1u) {  // (transposed: a lane's rows are adjacent, four at a time)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                float v[4];
                __builtin_memcpy(v, block + 2 * r + lane_cell, 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) state[db][r + e] = v[e];
            }
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) state[db][r] = block[((r & 3) + 8 * (r >> 2)) * s.state_row + lane_cell];
        }
        if (n0 + kWidthZ > s.b)
#pragma unroll
            for (int r = 0; r < 16; ++r) state[db][r] = col < s.b ? state[db][r] : 0.0f;
    }
    __syncthreads();

    // the factors of P: position i is a lane's column, j its rows.  The narrower kernels, three wavefronts of which share a SIMD's registers, read them
    // for every chunk (512 x 256 bfloat16 179 -> 169 us; those of 128, two to a SIMD, would lose as much).
    constexpr bool kFactors = kOut && A > 64 && sizeof(T) == 2;
    const uint32_t f0 = 31u + 4u * h32 - col32;
    float factors[kFactors ? 16 : 1];
    if (kFactors)
#pragma unroll
        for (int r = 0; r < 16; ++r) factors[kFactors ? r : 0] = factor[f0 + ((r & 3) + 8 * (r >> 2))];
    // (read, and there, before the loop: a wait for them inside it would be one for the steps asked for ahead as well)
    const auto there = [](float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); };
    const float decay = there(hd.decay), decay_rest = there(hd.decay_rest), decay_chunk = there(hd.decay_chunk), decay_chunk_rest = there(hd.decay_chunk_rest);
    uint32_t singles = 0, turn = 0;  // steps still to be taken one by one
    bool uncut = true, weights_plain = false;
    float owed = 0.0f;
    for (uint32_t at = begin; at < end;) {
        const bool reverse = again(s.reverse) != 0u;
        const uint32_t n = singles ? 1u : min((uint32_t)C, end - at);
        const int64_t t = step_of(at, n);
        if (!kAhead) ask(at, n);
        Most<T> most, unused;
        y_steps.template put<true>(yh + t * s.y.step, ys, n, most);
        z_steps.template put<true>(zh + t * s.z.step, zs, n, most);
        if (kOut) x_steps.template put<false>(xh + t * s.x.step, xs, n, unused);
        if (most.infinite()) flag[turn & 1u] = 1;
        const uint64_t m = __ballot(reset != 0u);
        __syncthreads();
        const bool broken = __builtin_amdgcn_readfirstlane(flag[turn & 1u]) != 0;
        if (threadIdx.x == 0) flag[(turn + 1u) & 1u] = 0;
        ++turn;
        if (broken && n > 1) {
            singles = n;
            if (kAhead) ask(at, 1u);
            __syncthreads();
            continue;
        }
        const uint32_t after = at + n;
        if (singles) --singles;
        if (kAhead && after < end) {
            ask(after, singles ? 1u : min((uint32_t)C, end - after));
        } else {
            y_steps.forget();
            z_steps.forget();
            x_steps.forget();
        }
        // what position `lane` adds to the state; the same for every whole chunk in which no episode begins
        const bool plain = n == (uint32_t)C && m == 0;
        if (!plain || !weights_plain) {
            const bool stays = reverse ? (m & up_to(lane)) == 0 : (m & ~up_to(lane)) == 0;
            if (lane < (uint32_t)C) weight[lane] = lane < n && stays ? s.key_scale * pw[reverse ? lane + 1u : n - 1u - lane] : 0.0f;
            weights_plain = plain;
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }

        // z is in registers before the outputs take its place in LDS
        const auto z0 = across<false>(zs + wave * 32u, kStrideZ, lane), z1 = across<false>(zs + 16 * kStrideZ + wave * 32u, kStrideZ, lane);
        const bool last = A <= 64 || again(s.a) > (uint32_t)A - 32u;  // rows in the state's last block (heads of 96 without it 105 -> 98 us)
        if constexpr (kOut) {
            // out^T = S^T x^T and P^T = y x^T, columns = steps
            f32x16 acc = (f32x16)0.0f, p = (f32x16)0.0f;
#pragma unroll
            for (int k = 0; k < A / 16; ++k) {
                if (A > 64 && k == A / 16 - 2 && !last) break;
                const Parts<kParts<T>> x = along<kParts<T>>(xs + col32 * kStrideA + k * 16, kPlane, h32);
                acc = mma(split<T>(half(state[k / 2], k % 2)), x, acc);
                p = mma(along<kParts<T>>(ys + col32 * kStrideA + k * 16, kPlane, h32), x, p);
            }
            acc *= s.out_scale * pw[reverse ? (col32 < n ? n - 1u - col32 : 0u) : col32 + 1u];
            if (m) {
                const bool into = reverse ? (m & ~up_to(col32)) == 0 : (m & up_to(col32)) == 0;
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[r] = into ? acc[r] : 0.0f;
            }
            // the positions that reach i, [first, past): j <= i and no episode begins in (j, i]; mirrored in reverse.  (A choice and no product with 0:
            // an overflow in a pair that does not count stays out.)
            const uint64_t upto = m & up_to(col32), later = m & ~up_to(col32);
            const uint32_t first = reverse ? col32 : upto ? 63u - (uint32_t)__builtin_clzll(upto) : 0u;
            const uint32_t past = reverse ? (later ? (uint32_t)__builtin_ctzll(later) : 64u) : col32 + 1u;
            uint32_t lowest = 4u * h32 - first, f = f0;
            asm volatile("" : "+v"(f), "+v"(lowest));  // (or what they give with 16 numbers is kept from chunk to chunk)
#pragma unroll
            for (int r = 0; r < 16; ++r) p[r] = lowest + ((r & 3) + 8 * (r >> 2)) < past - first ? p[r] * (kFactors ? factors[kFactors ? r : 0] : factor[f + ((r & 3) + 8 * (r >> 2))]) : 0.0f;
            // out^T += z^T P^T
            acc = mma(parts_of(z0), split<T>(half(p, 0)), acc);
            acc = mma(parts_of(z1), split<T>(half(p, 1)), acc);
            // The outputs take the place of the wavefront's own columns of z in LDS, so that they leave as 16 bytes a lane, rows of 64 or 128
            // bytes, past the caches: they are not read again (512 x 256 bfloat16 186 -> 171 us; parts of rows past the caches 345).
            T* own = zs + wave * 32u;
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                T* w = own + col32 * kStrideZ + 2 * r + 4 * h32;
                if constexpr (sizeof(T) == 2) {
                    const u32x2 v = {__builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{acc[r], acc[r + 1]}, bf16x2)),
                                     __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{acc[r + 2], acc[r + 3]}, bf16x2))};
                    *reinterpret_cast<u32x2*>(w) = v;
                } else {
                    *reinterpret_cast<f32x4*>(w) = f32x4{acc[r], acc[r + 1], acc[r + 2], acc[r + 3]};
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            constexpr uint32_t N = 16 / sizeof(T), kLanes = 32 / N;  // values of a vector, lanes of a row
            const uint32_t c = lane % kLanes * N, have = min(s.b - min(s.b, n0 + wave * 32u), 32u);
#pragma unroll
            for (uint32_t i = 0; i < kLanes / 2; ++i) {
                const uint32_t r = i * (64u / kLanes) + lane / kLanes;
                const any_u32x4 v = *reinterpret_cast<const u32x4*>(own + r * kStrideZ + c);
                if (r >= n || c >= have) continue;
                T* o = oh + (t + r) * s.out.step + (n0 + wave * 32u + c);
                if (c + N <= have) {
                    __builtin_nontemporal_store(v, reinterpret_cast<any_u32x4*>(o));
                } else {
                    T e[N];
                    __builtin_memcpy(e, &v, 16);
#pragma unroll
                    for (uint32_t k = 0; k < N; ++k)
                        if (c + k < have) o[k] = e[k];
                }
            }
        }

        // S <- g^n S + y^T (weights z)
        if (m == 0) {
            if (n == (uint32_t)C) {
                // What the factor's rounding leaves goes into the next chunk's factor, so that products of many stay within a rounding of g^(32 chunks)
                // (the factor and its rest, a product more for each value of the state: gradients of 512 x 256 bfloat16 402 us, 393 so).
                owed += decay_chunk_rest;
                const float keep = decay_chunk + owed;
                owed -= keep - decay_chunk;
#pragma unroll
                for (int db = 0; db < A / 32; ++db) state[db] *= keep;
            } else {
                const float keep = n == 1u ? decay : pw[n], keep_rest = n == 1u ? decay_rest : 0.0f;
#pragma unroll
                for (int db = 0; db < A / 32; ++db)
#pragma unroll
                    for (int r = 0; r < 16; ++r) state[db][r] = __builtin_fmaf(state[db][r], keep, state[db][r] * keep_rest);
            }
        } else {
            uncut = false;
#pragma unroll
            for (int db = 0; db < A / 32; ++db) state[db] = (f32x16)0.0f;
        }
        // In reverse, a chunk whose first step begins an episode adds nothing to the state, and its steps, all weighted with zero, are left out: there may be
        // one among them that is no number.
        if (!(reverse && (m & 1u))) {
#pragma unroll
            for (int k = 0; k < C / 16; ++k) {
                const Parts<3> zp = split<T>(values(k ? z1 : z0) * eight(weight + k * 16 + 4 * h32, weight + k * 16 + 8 + 4 * h32));
#pragma unroll
                for (int db = 0; db < A / 32; ++db) {
                    if (A > 64 && db == A / 32 - 1 && !last) break;
                    state[db] = mma(across_placed<kParts<T>>(ys + k * 16 * kStrideA + db * 32, kPlane, kStrideA, lane), zp, state[db]);
                }
            }
        }
        __syncthreads();
        at = after;
    }

    float* to = kOut ? (seg + 1u == cut.segments && s.state_out ? s.state_out + row * cells : nullptr)
                     : (role ? local1 : local0) + ((size_t)seg * cut.rows + row) * cells;
    if (to && col < s.b) {
#pragma unroll
        for (int db = 0; db < A / 32; ++db) {
            if (db * 32u >= s.a) break;
            float* block = to + (size_t)db * 32 * s.state_row;
            if (db * 32u + 32u <= s.a) {
#pragma unroll
                for (int r = 0; r < 16; ++r) block[((r & 3) + 8 * (r >> 2)) * s.state_row + lane_cell] = state[db][r];
            } else {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (db * 32 + (r & 3) + 8 * (r >> 2) + 4 * h32 < s.a) block[((r & 3) + 8 * (r >> 2)) * s.state_row + lane_cell] = state[db][r];
            }
        }
    }
    if (!kOut && tile == 0 && threadIdx.x == 0) (role ? whole1 : whole0)[seg * cut.rows + row] = uncut ? 1u : 0u;
}

// The segments' own states, one after the other, to the states before the segments that follow: one lane per cell of a state.  kBatch segments' requests
// are on their way while the kBatch before them are added up, as many as there are, 16 at most (89 segments of 8 heads of 64 x 128: 16 at a time 13 us,
// 8 with none on their way 22; 2 segments of 256 states of 128 x 96, whole pass: 2 or 4 at a time 112 us, 8 120).
template <uint32_t kBatch>
__global__ __launch_bounds__(256) void join_kernel(const Cut cut, uint32_t cells, const float* in0, const float* in1, float* local0, float* local1,
                                                   const uint32_t* __restrict__ whole0, const uint32_t* __restrict__ whole1) {
    const uint32_t i = blockIdx.x * 256u + threadIdx.x, row = blockIdx.y;
    if (i >= cells) return;
    const float* in = blockIdx.z ? in1 : in0;
    float* local = blockIdx.z ? local1 : local0;
    const uint32_t* whole = blockIdx.z ? whole1 : whole0;
    const uint32_t last = cut.segments - 2u;
    float next[kBatch];
    uint32_t through_next[kBatch];
    const auto ask = [&](uint32_t k0) {
#pragma unroll
        for (uint32_t k = 0; k < kBatch; ++k) {
            const size_t at = (size_t)min(k0 + k, last) * cut.rows + row;
            next[k] = local[at * cells + i];
            through_next[k] = whole[at];
        }
    };
    ask(0);
    float v = in ? in[(size_t)row * cells + i] : 0.0f;
    const double g = exp(cut.heads[row % cut.n_heads].log_decay * (double)cut.seg_steps);
    const float keep = (float)g, rest = (float)(g - (double)keep);
    for (uint32_t k0 = 0; k0 <= last; k0 += kBatch) {
        float own[kBatch];
        uint32_t through[kBatch];
#pragma unroll
        for (uint32_t k = 0; k < kBatch; ++k) {
            own[k] = next[k];
            through[k] = through_next[k];
        }
        if (k0 + kBatch <= last) ask(k0 + kBatch);
#pragma unroll
        for (uint32_t k = 0; k < kBatch; ++k) {
            if (k0 + k > last) break;
            v = own[k] + (through[k] ? __builtin_fmaf(v, keep, v * rest) : 0.0f);
            local[((size_t)(k0 + k) * cut.rows + row) * cells + i] = v;
        }
    }
}

struct Step {
    pxr_tokens q, k, v, out;
    uint32_t dk, dv, n_heads, rows, lanes;  // rows = environments * heads; lanes that take a row of the state
    float scale;
    const LinearAttentionHead* heads;
    const uint8_t* resets;
    int64_t resets_env;
    float* state;
};

// One step of every environment.  Bound by reading and writing the states: 65536 of 64 x 64 (16384 environments, four heads) in 405 us, 5.3 TB/s.  A lane
// takes kVec adjacent columns, `lanes` lanes a row and the wavefront's other lanes the rows after it; eight rows a lane are on their way while the eight before
// them are worked on.  kVec is 4; a row that is no multiple of 4 has its last vector moved back to its end, where two lanes read the same
// values in one request, work out the same and write the same (1 for rows of less than 4).  kWaves wavefronts share a state (1 or 4): the keys and
// queries of a head lie in LDS, a copy for each wavefront, so that only the sums of four need a barrier.
template <class T, int kVec, int kWaves>
__global__ __launch_bounds__(256) void step_kernel(const Step a) {
    constexpr uint32_t kHeads = 4 / kWaves, kBatch = 8;
    __shared__ __align__(16) float keys[4][256], queries[4][256];
    __shared__ float sums[4][64 * kVec];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, sub = wave % kWaves, row = blockIdx.x * kHeads + wave / kWaves;
    if (kWaves == 1 && row >= a.rows) return;  // (no barrier follows)
    const uint32_t env = row / a.n_heads, head = row - env * a.n_heads;
    const bool cut = a.resets && a.resets[(int64_t)env * a.resets_env] != 0;
    const LinearAttentionHead& hd = a.heads[head];
    const float decay = hd.decay, decay_rest = hd.decay_rest;
    const T *qh = head_of<const T>(a.q, env, head), *kh = head_of<const T>(a.k, env, head), *vh = head_of<const T>(a.v, env, head);
    const uint32_t at = lane & (a.lanes - 1u), first = lane / a.lanes, each = 64u / a.lanes;  // the lane's vector, its row of those taken together
    const bool on = at * kVec < a.dv;
    const uint32_t col = min(at * kVec, a.dv - kVec);
    float* state = a.state + (size_t)row * a.dk * a.dv + col;
    const uint32_t turns = (a.dk + each * kWaves - 1u) / (each * kWaves);
    const auto row_of = [&](uint32_t turn) { return (turn * kWaves + sub) * each + first; };
    float next[kBatch][kVec];
    const auto ask = [&](uint32_t turn) {
#pragma unroll
        for (uint32_t i = 0; i < kBatch; ++i) {
            const uint32_t d = row_of(turn + i);
#pragma unroll
            for (int e = 0; e < kVec; ++e) next[i][e] = 0.0f;
            if (on && d < a.dk) __builtin_memcpy(next[i], state + d * a.dv, sizeof(next[i]));
        }
    };
    if (!cut) ask(0);
    float v[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = load1(vh + col + e);
    for (uint32_t d = lane; d < a.dk; d += 64u) {
        keys[wave][d] = load1(kh + d);
        queries[wave][d] = load1(qh + d);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    float sum[kVec] = {};
    for (uint32_t turn = 0; turn < turns; turn += kBatch) {
        float s[kBatch][kVec];
#pragma unroll
        for (uint32_t i = 0; i < kBatch; ++i)
#pragma unroll
            for (int e = 0; e < kVec; ++e) s[i][e] = cut ? 0.0f : next[i][e];
        if (!cut && turn + kBatch < turns) ask(turn + kBatch);
#pragma unroll
        for (uint32_t i = 0; i < kBatch; ++i) {
            const uint32_t d = row_of(turn + i);
            if (!on || d >= a.dk) continue;
            const float kd = keys[wave][d], qd = queries[wave][d];
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                s[i][e] = __builtin_fmaf(kd, v[e], __builtin_fmaf(s[i][e], decay, s[i][e] * decay_rest));
                sum[e] = __builtin_fmaf(qd, s[i][e], sum[e]);
            }
            __builtin_memcpy(state + d * a.dv, s[i], sizeof(s[i]));
        }
    }
    for (uint32_t m = a.lanes; m < 64u; m <<= 1)
#pragma unroll
        for (int e = 0; e < kVec; ++e) sum[e] += __shfl_xor(sum[e], m);
    if constexpr (kWaves > 1) {
        if (first == 0)
#pragma unroll
            for (int e = 0; e < kVec; ++e) sums[wave][at * kVec + e] = sum[e];
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int e = 0; e < kVec; ++e)
            sum[e] = (sums[0][at * kVec + e] + sums[1][at * kVec + e]) + (sums[2][at * kVec + e] + sums[3][at * kVec + e]);
    }
    if (first == 0 && on) {
        T* o = head_of<T>(a.out, env, head) + col;
#pragma unroll
        for (int e = 0; e < kVec; ++e) store1(o + e, sum[e] * a.scale);
    }
}

int launched(std::string& err) {
    const hipError_t rc = hipGetLastError();
    if (rc == hipSuccess) return PXR_OK;
    err = std::string("kernel launch failed: ") + hipGetErrorString(rc);
    return PXR_ERR_DEVICE;
}

// Wavefronts of a workgroup: enough for z, four at most, and no fewer than it takes to bring the steps of long heads (256 x 128 with 8 heads in bfloat16:
// 64 x 64 two 50 us, four 73; 64 x 128 four 72, two 79; 32 x 32 one 21.9, two 22.6).
uint32_t waves_of(uint32_t a, uint32_t b) { return a > 128u ? 4u : b <= 32u && a <= 64u ? 1u : b <= 64u ? 2u : 4u; }

uint32_t width_of(uint32_t a) { return a <= 32u ? 32u : a <= 64u ? 64u : a <= 128u ? 128u : 256u; }

// Whether one launch takes the three scans of the backward pass: the steps that they share are then read once.  Keys and values of different widths would all
// take the kernel for the larger of both (256 x 128 with 8 heads of 64 x 128 407 us together, 196 apart; 20000 steps of them 257 / 187; 4 x 1000 with 3
// heads of 96 x 48 in fp32, which do not fill the device, 83 / 92).
bool together(const LinearAttentionConsts& c) { return width_of(c.dk) == width_of(c.dv) && waves_of(c.dk, c.dv) == waves_of(c.dv, c.dk); }

// Segments of a rollout's steps: as many as it takes to fill the device (the places that registers and LDS leave on each compute unit), of two chunks at least, and of one for every 4096 cells of a state: a segment costs its state, written, joined and read.  us with a
// workgroup for each place / with two for each compute unit: 30 x 2000 with 8 heads of 64 131 / 198, 64 x 1000 with 4 of 32 50 / 78, 4 x 1000 with 3 of 96 x 48 in
// fp32 62 / 86; 16 x 512 with 16 of 128 x 96, whose two are all there is room for, 126, with four 153.
uint32_t segments_of(const LinearAttentionConsts& c, uint32_t dtype, uint32_t n_envs, uint32_t n_steps, bool backward, uint32_t* seg_steps) {
    const auto fit = [&](uint32_t a, uint32_t b, uint64_t roles) {
        const uint32_t width = width_of(a), waves = waves_of(a, b), tiles = (b + waves * 32u - 1u) / (waves * 32u);
        const uint32_t element = dtype == PXR_F32 ? 4u : 2u;
        const uint64_t places = (uint64_t)c.n_cus * std::min(4u * waves_per_simd(width, element) / waves, kLds / scan_lds(element, width, waves, true));
        return places / ((uint64_t)n_envs * c.n_heads * roles * tiles);
    };
    uint64_t want = fit(c.dk, c.dv, !backward ? 1u : together(c) ? 3u : 1u);
    if (backward && !together(c)) want = std::min(want, fit(c.dv, c.dk, 2u));
    const uint64_t chunks = ((uint64_t)n_steps + C - 1u) / C;
    const uint64_t least = c.dk * c.dv > 2u * 4096u ? c.dk * c.dv / 4096u : 2u;
    if (want > chunks / least) want = chunks / least;
    if (want < 2u) {
        *seg_steps = n_steps;
        return 1u;
    }
    const uint64_t each = (chunks + want - 1u) / want;
    *seg_steps = (uint32_t)(each * C);
    return (uint32_t)((chunks + each - 1u) / each);
}

// Chunks of long heads take more than the 64 KB of LDS that a launch has by default.
template <class T>
hipError_t allow_lds() {
    const void* fns[] = {reinterpret_cast<const void*>(&scan_kernel<T, 128, 2, true>),  reinterpret_cast<const void*>(&scan_kernel<T, 128, 4, true>),
                         reinterpret_cast<const void*>(&scan_kernel<T, 256, 4, true>),  reinterpret_cast<const void*>(&scan_kernel<T, 256, 4, false>)};
    static_assert(scan_lds(sizeof(T), 64, 4, true) <= 64 * 1024 && scan_lds(sizeof(T), 128, 4, false) <= 64 * 1024 && scan_lds(sizeof(T), 256, 4, true) <= kLds);
    for (const void* f : fns)
        if (const hipError_t rc = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds); rc != hipSuccess) return rc;
    return hipSuccess;
}

template <class T, bool kOut>
void enqueue_as(const Scan* s, uint32_t roles, const Cut& cut, float* const* local, uint32_t* const* whole, hipStream_t st) {
    const uint32_t items = cut.rows * (kOut ? cut.segments : cut.segments - 1u);
    const dim3 grid((items + 7u) / 8u * 8u * cut.tiles * roles);
    const Scans scans{{s[0], s[roles > 1 ? 1 : 0], s[roles > 2 ? 2 : 0]}};
#define PXR_SCAN(A, W)                                                                                                                            \
    case A + W:                                                                                                                                   \
        hipLaunchKernelGGL((scan_kernel<T, A, W, kOut>), grid, dim3(W * 64), scan_lds(sizeof(T), A, W, kOut), st, scans, cut, roles, local[0], local[1], \
                           whole[0], whole[1]);                                                                                                   \
        break;
    switch (cut.width + cut.waves) { PXR_SCAN_SHAPES(PXR_SCAN) }
#undef PXR_SCAN
}

template <bool kOut>
void enqueue(uint32_t dtype, const Scan* s, uint32_t roles, const Cut& cut, float* const* local, uint32_t* const* whole, hipStream_t st) {
    if (dtype == PXR_F32)
        enqueue_as<float, kOut>(s, roles, cut, local, whole, st);
    else
        enqueue_as<__bf16, kOut>(s, roles, cut, local, whole, st);
}

void join(const Cut& cut, uint32_t cells, uint32_t sets, const float* in0, const float* in1, float* const* local, uint32_t* const* whole, hipStream_t st) {
    const dim3 grid((cells + 255u) / 256u, cut.rows, sets);
    const uint32_t states = cut.segments - 1u;
    const auto kernel = states > 8u ? join_kernel<16> : states > 4u ? join_kernel<8> : states > 2u ? join_kernel<4> : join_kernel<2>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, cut, cells, in0, in1, local[0], local[1], whole[0], whole[1]);
}

Cut cut_of(const LinearAttentionConsts& c, const pxr_rollout& r, bool backward, uint32_t a, uint32_t b) {
    Cut cut{};
    cut.n_heads = c.n_heads;
    cut.rows = r.n_envs * c.n_heads;
    cut.n_steps = r.n_steps;
    cut.segments = segments_of(c, r.dtype, r.n_envs, r.n_steps, backward, &cut.seg_steps);
    cut.width = width_of(a);
    cut.waves = waves_of(a, b);
    cut.tiles = (b + cut.waves * 32u - 1u) / (cut.waves * 32u);
    cut.heads = c.heads;
    cut.resets = r.d_resets;
    cut.resets_env = r.resets_env;
    cut.resets_step = r.resets_step;
    return cut;
}

// Bytes of one set of segments' states, and of the words beside them.
size_t state_bytes(const LinearAttentionConsts& c, uint32_t n_envs, uint32_t segments) {
    return (size_t)(segments - 1u) * n_envs * c.n_heads * c.dk * c.dv * 4u;
}
size_t whole_bytes(const LinearAttentionConsts& c, uint32_t n_envs, uint32_t segments) {
    return ((size_t)(segments - 1u) * n_envs * c.n_heads * 4u + 15u) & ~(size_t)15u;
}

}  // namespace

int prepare_linear_attention_kernels(std::string& err) {
    hipError_t rc = allow_lds<float>();
    if (rc == hipSuccess) rc = allow_lds<__bf16>();
    if (rc == hipSuccess) return PXR_OK;
    err = std::string("hipFuncSetAttribute(MaxDynamicSharedMemorySize) failed: ") + hipGetErrorString(rc);
    return PXR_ERR_DEVICE;
}

size_t linear_attention_workspace(const LinearAttentionConsts& c, uint32_t dtype, uint32_t n_envs, uint32_t n_steps, bool backward) {
    uint32_t steps;
    const uint32_t segments = segments_of(c, dtype, n_envs, n_steps, backward, &steps);
    const size_t one = ((state_bytes(c, n_envs, segments) + 15u) & ~(size_t)15u) + whole_bytes(c, n_envs, segments);
    return backward ? 2u * one : one;
}

int launch_linear_attention_forward(const LinearAttentionConsts& c, const pxr_rollout& r, const pxr_tokens& out, float* state_out, void* ws,
                                    void* stream, std::string& err) {
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const Cut cut = cut_of(c, r, false, c.dk, c.dv);
    Scan s{r.q, r.k, r.v, out, c.dk, c.dv, r.d_state, state_out, c.dv, 1u, nullptr, c.scale, 1.0f, 0u};
    float* local[2] = {static_cast<float*>(ws), nullptr};
    uint32_t* whole[2] = {reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + ((state_bytes(c, r.n_envs, cut.segments) + 15u) & ~(size_t)15u)), nullptr};
    if (cut.segments > 1u) {
        enqueue<false>(r.dtype, &s, 1u, cut, local, whole, st);
        join(cut, c.dk * c.dv, 1u, r.d_state, nullptr, local, whole, st);
        s.before = local[0];
    }
    enqueue<true>(r.dtype, &s, 1u, cut, local, whole, st);
    return launched(err);
}

int launch_linear_attention_backward(const LinearAttentionConsts& c, const pxr_rollout& r, const pxr_tokens& dout, const float* dstate_out,
                                     const pxr_tokens& dq, const pxr_tokens& dk, const pxr_tokens& dv, float* dstate, void* ws,
                                     void* stream, std::string& err) {
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const Cut cut_v = cut_of(c, r, true, c.dk, c.dv), cut_k = cut_of(c, r, true, c.dv, c.dk);
    const size_t states = (state_bytes(c, r.n_envs, cut_v.segments) + 15u) & ~(size_t)15u, words = whole_bytes(c, r.n_envs, cut_v.segments);
    char* w = static_cast<char*>(ws);
    float* local[2] = {reinterpret_cast<float*>(w), reinterpret_cast<float*>(w + states + words)};
    uint32_t* whole[2] = {reinterpret_cast<uint32_t*>(w + states), reinterpret_cast<uint32_t*>(w + 2u * states + words)};
    if (cut_v.segments > 1u) {
        // the states [dk][dv] of the forward scan and of the reverse one, which dk and dv share
        const Scan both[2] = {Scan{r.q, r.k, r.v, dout, c.dk, c.dv, nullptr, nullptr, c.dv, 1u, nullptr, 1.0f, 1.0f, 0u},
                              Scan{r.k, r.q, dout, dout, c.dk, c.dv, nullptr, nullptr, c.dv, 1u, nullptr, 1.0f, c.scale, 1u}};
        enqueue<false>(r.dtype, both, 2u, cut_v, local, whole, st);
        join(cut_v, c.dk * c.dv, 2u, r.d_state, dstate_out, local, whole, st);
    }
    const Scan three[3] = {Scan{dout, r.v, r.k, dq, c.dv, c.dk, r.d_state, nullptr, 1u, c.dv, local[0], c.scale, 1.0f, 0u},
                           Scan{r.v, dout, r.q, dk, c.dv, c.dk, dstate_out, nullptr, 1u, c.dv, local[1], 1.0f, c.scale, 1u},
                           Scan{r.k, r.q, dout, dv, c.dk, c.dv, dstate_out, dstate, c.dv, 1u, local[1], 1.0f, c.scale, 1u}};
    if (together(c)) {
        enqueue<true>(r.dtype, three, 3u, cut_k, local, whole, st);
    } else {
        enqueue<true>(r.dtype, three, 2u, cut_k, local, whole, st);
        enqueue<true>(r.dtype, three + 2, 1u, cut_v, local, whole, st);
    }
    return launched(err);
}

int launch_linear_attention_step(const LinearAttentionConsts& c, const pxr_rollout& r, float* state, const pxr_tokens& out, void* stream,
                                 std::string& err) {
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    Step a{r.q, r.k, r.v, out, c.dk, c.dv, c.n_heads, r.n_envs * c.n_heads, 1u, c.scale, c.heads, r.d_resets, r.resets_env, state};
    const uint32_t vec = c.dv < 4u ? 1u : 4u;
    while (a.lanes * vec < c.dv) a.lanes *= 2u;
    // A wavefront for a state of up to 16 KB; four for longer ones (8000 of 128 x 128 203 us, with one 217; 32000 of 32 x 32 42, with four 114), and where there are
    // so few that the device has wavefronts to spare (400 of 64 x 64 5.0, with one 5.9; 800 7.7, with one 6.7).
    const bool four = c.dk * c.dv > 4096u || a.rows < 2u * c.n_cus;
    const dim3 grid(four ? a.rows : (a.rows + 3u) / 4u);
#define PXR_STEP(T, V, W) hipLaunchKernelGGL((step_kernel<T, V, W>), grid, dim3(256), 0, st, a)
#define PXR_STEP_AS(T)          \
    if (vec == 1u && four)      \
        PXR_STEP(T, 1, 4);      \
    else if (vec == 1u)         \
        PXR_STEP(T, 1, 1);      \
    else if (four)              \
        PXR_STEP(T, 4, 4);      \
    else                        \
        PXR_STEP(T, 4, 1)
    if (r.dtype == PXR_F32) {
        PXR_STEP_AS(float);
    } else {
        PXR_STEP_AS(__bf16);
    }
#undef PXR_STEP_AS
#undef PXR_STEP
    return launched(err);
}

}  // namespace pxr
