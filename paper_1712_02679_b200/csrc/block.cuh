// Shared by the operators of a transformer block (dropout, layer norm, biased softmax): element types, the dropout
// generator, how the threads of a row share its columns, and sums over them.
#pragma once

#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "common.cuh"

namespace adacomp_impl {

constexpr int kBlockSms = 148;               // SMs of a B200: grids are sized to it, so results do not depend on a query
constexpr u32 kAllLanes = 0xffffffffu;

// ---------------------------------------------------------------------------------
// element types: eight elements at a time, arithmetic in binary32
// ---------------------------------------------------------------------------------

template <u32 TYPE> struct Vec8 { uint4 q[TYPE == ADACOMP_TYPE_F32 ? 2 : 1]; };

__host__ __device__ constexpr u32 type_size(u32 type) { return type == ADACOMP_TYPE_F32 ? 4u : 2u; }

template <u32 TYPE> __device__ inline Vec8<TYPE> load8(const void *base, u64 e)
{
    Vec8<TYPE> v;
    const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const unsigned char *>(base) + e * type_size(TYPE));
    v.q[0] = p[0];
    if constexpr (TYPE == ADACOMP_TYPE_F32) v.q[1] = p[1];
    return v;
}

template <u32 TYPE> __device__ inline void store8(void *base, u64 e, const Vec8<TYPE> &v)
{
    uint4 *p = reinterpret_cast<uint4 *>(static_cast<unsigned char *>(base) + e * type_size(TYPE));
    p[0] = v.q[0];
    if constexpr (TYPE == ADACOMP_TYPE_F32) p[1] = v.q[1];
}

template <u32 TYPE> __device__ inline void widen8(const Vec8<TYPE> &r, float (&v)[8])
{
    const u32 *w = reinterpret_cast<const u32 *>(r.q);
    if constexpr (TYPE == ADACOMP_TYPE_F32) {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = __uint_as_float(w[i]);
    } else if constexpr (TYPE == ADACOMP_TYPE_BF16) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const __half2 h = *reinterpret_cast<const __half2 *>(&w[i]);
            const float2 f = __half22float2(h);
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
}

template <u32 TYPE> __device__ inline Vec8<TYPE> narrow8(const float (&v)[8])
{
    Vec8<TYPE> r;
    u32 *w = reinterpret_cast<u32 *>(r.q);
    if constexpr (TYPE == ADACOMP_TYPE_F32) {
#pragma unroll
        for (int i = 0; i < 8; i++) w[i] = __float_as_uint(v[i]);
    } else if constexpr (TYPE == ADACOMP_TYPE_BF16) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const u32 *>(&b);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const u32 *>(&h);
        }
    }
    return r;
}

template <u32 TYPE> __device__ inline float load1(const void *base, u64 e)
{
    if constexpr (TYPE == ADACOMP_TYPE_F32) return static_cast<const float *>(base)[e];
    else if constexpr (TYPE == ADACOMP_TYPE_BF16)
        return __uint_as_float((u32) static_cast<const unsigned short *>(base)[e] << 16);
    else return __half2float(static_cast<const __half *>(base)[e]);
}

template <u32 TYPE> __device__ inline void store1(void *base, u64 e, float v)
{
    if constexpr (TYPE == ADACOMP_TYPE_F32) static_cast<float *>(base)[e] = v;
    else if constexpr (TYPE == ADACOMP_TYPE_BF16) static_cast<__nv_bfloat16 *>(base)[e] = __float2bfloat16_rn(v);
    else static_cast<__half *>(base)[e] = __float2half_rn(v);
}

// ---------------------------------------------------------------------------------
// two binary32 operations in one instruction (PTX .f32x2, sm_100): these kernels are bound by how many instructions an SM
// issues, not by how many operations it has units for
// ---------------------------------------------------------------------------------

__device__ inline void fma2(float &d0, float &d1, float a0, float a1, float b0, float b1, float c0, float c1)
{
    asm("{\n\t.reg .b64 a, b, c, d;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d0), "=f"(d1)
        : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}

__device__ inline void mul2(float &d0, float &d1, float a0, float a1, float b0, float b1)
{
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "mul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d0), "=f"(d1)
        : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}

__device__ inline void add2(float &d0, float &d1, float a0, float a1, float b0, float b1)
{
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d0), "=f"(d1)
        : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}

// v = v * x + y, v * x, v + x, element by element or with one number
__device__ inline void fma8(float (&v)[8], float x, float y)
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) fma2(v[e], v[e + 1], v[e], v[e + 1], x, x, y, y);
}
__device__ inline void mul8(float (&v)[8], float x)
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) mul2(v[e], v[e + 1], v[e], v[e + 1], x, x);
}
__device__ inline void mul8(float (&v)[8], const float (&x)[8])
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) mul2(v[e], v[e + 1], v[e], v[e + 1], x[e], x[e + 1]);
}
__device__ inline void add8(float (&v)[8], float x)
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) add2(v[e], v[e + 1], v[e], v[e + 1], x, x);
}
__device__ inline void add8(float (&v)[8], const float (&x)[8])
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) add2(v[e], v[e + 1], v[e], v[e + 1], x[e], x[e + 1]);
}
// acc += v, acc += v * x
__device__ inline void sum8(float2 &acc, const float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) add2(acc.x, acc.y, acc.x, acc.y, v[e], v[e + 1]);
}
__device__ inline void dot8(float2 &acc, const float (&v)[8], const float (&x)[8])
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) fma2(acc.x, acc.y, v[e], v[e + 1], x[e], x[e + 1], acc.x, acc.y);
}

// ---------------------------------------------------------------------------------
// how a row's threads share its columns
//
// A row belongs to `tpr` threads (whole warps); each holds NV blocks of eight neighbouring columns.  A warp's blocks lie
// next to each other: block k of lane l of the row's warp w starts at column 8 * ((w * NV + k) * 32 + l).  So a block is
// one group of the dropout generator, parameters are read by whole vectors, and neighbouring lanes hold neighbouring
// columns.
//
// In memory a row may start anywhere (its length need not be a multiple of 8).  ALIGNED rows start on a 16-byte boundary.
// Others start s elements behind one: a block then lies in two 16-byte chunks (three for binary32), which are loaded whole
// and shifted; on the way out a lane joins its first elements with its neighbour's last ones into one whole chunk, and
// only the ends of a warp's or a row's columns are stored element by element.  Chunks are loaded only if they hold an
// element of the block, so no 16-byte granule without an element of the tensor is touched.
// ---------------------------------------------------------------------------------

template <int NV> __device__ inline u32 block_column(u32 k, u32 t) { return (((t >> 5) * NV + k) * 32u + (t & 31u)) * 8u; }

template <u32 TYPE> __host__ __device__ constexpr u32 chunk_elems() { return 16u / type_size(TYPE); }

// A block as loaded, not yet shifted (what a prefetch holds).
template <u32 TYPE, bool ALIGNED> struct Raw { uint4 q[(TYPE == ADACOMP_TYPE_F32 ? 2 : 1) + (ALIGNED ? 0 : 1)]; };

// The chunks of the block from column c of the row at element row_at, as far as they lie before column `end`:
// f(i, address) for each that holds one of its elements.
template <u32 TYPE, bool ALIGNED, typename F>
__device__ inline void for_chunks(const void *base, u64 row_at, u32 c, u32 end, F f)
{
    constexpr u32 per = chunk_elems<TYPE>();
    const u32 s = ALIGNED ? 0u : (u32)row_at & (per - 1u);
    const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const unsigned char *>(base) + (row_at + c - s) * type_size(TYPE));
    constexpr int n = sizeof(Raw<TYPE, ALIGNED>) / 16;
#pragma unroll
    for (int i = 0; i < n; i++)     // chunk i holds columns c - s + i * per and up (the first one: column c)
        if (c + (i ? i * per - s : 0u) < end && (ALIGNED || i * per - s < 8u || i == 0)) f(i, p + i);
}

// Into registers; what is not loaded keeps what it held.
template <u32 TYPE, bool ALIGNED>
__device__ inline void fetch(Raw<TYPE, ALIGNED> &r, const void *base, u64 row_at, u32 c, u32 end)
{
    for_chunks<TYPE, ALIGNED>(base, row_at, c, end, [&](int i, const uint4 *p) { r.q[i] = *p; });
}

__device__ inline void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// w[0..n) = in[shift .. shift + n) for a shift of 0..3 words (the same for the whole warp)
template <int N, int M> __device__ inline void shift_words(const u32 (&in)[M], u32 shift, u32 (&out)[N])
{
    u32 x[N + 1];
#pragma unroll
    for (int i = 0; i <= N; i++) x[i] = (shift & 2u) ? (i + 2 < M ? in[i + 2] : 0u) : (i < M ? in[i] : 0u);
#pragma unroll
    for (int i = 0; i < N; i++) out[i] = (shift & 1u) ? x[i + 1] : x[i];
}

// The block's elements in binary32 (see mask_from for those behind the last one asked for).
template <u32 TYPE, bool ALIGNED>
__device__ inline void unpack(const Raw<TYPE, ALIGNED> &r, u64 row_at, float (&v)[8])
{
    Vec8<TYPE> whole;
    if constexpr (ALIGNED) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(whole.q) / 16); i++) whole.q[i] = r.q[i];
    } else {
        const u32 s = (u32)row_at & (chunk_elems<TYPE>() - 1u);
        u32 *out = reinterpret_cast<u32 *>(whole.q);
        constexpr int n = sizeof(r.q) / 4;
        u32 in[n];
#pragma unroll
        for (int i = 0; i < n / 4; i++) in[4 * i] = r.q[i].x, in[4 * i + 1] = r.q[i].y, in[4 * i + 2] = r.q[i].z, in[4 * i + 3] = r.q[i].w;
        if constexpr (TYPE == ADACOMP_TYPE_F32) {
            u32 y[8];
            shift_words<8>(in, s, y);
#pragma unroll
            for (int i = 0; i < 8; i++) out[i] = y[i];
        } else {
            u32 y[5];
            shift_words<5>(in, s >> 1, y);
#pragma unroll
            for (int i = 0; i < 4; i++) out[i] = __funnelshift_r(y[i], y[i + 1], (s & 1u) * 16u);
        }
    }
    widen8<TYPE>(whole, v);
}

// v: the block from column c; its elements from column `end` on become `fill`.
__device__ inline void mask_from(float (&v)[8], u32 c, u32 end, float fill)
{
    if (c + 8 > end) {
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (c + e >= end) v[e] = fill;
    }
}

// Stores the block's columns before `cols`.  Unless ALIGNED, all lanes of the warp take part; where a lane's block is not a
// row's first, the lane before it holds the block before it.
template <u32 TYPE, bool ALIGNED>
__device__ inline void store_block(void *base, u64 row_at, u32 c, u32 cols, const float (&v)[8])
{
    constexpr u32 per = chunk_elems<TYPE>();
    if constexpr (ALIGNED) {
        if (c + 8 <= cols) store8<TYPE>(base, row_at + c, narrow8<TYPE>(v));
        if (cols & 7u) {                // (what lies behind the row's last column is not this row's)
            if (c < cols && c + 8 > cols) {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (c + e < cols) store1<TYPE>(base, row_at + c + e, v[e]);
            }
        }
        return;
    }
    const u32 s = (u32)row_at & (per - 1u);
    const u32 lane = threadIdx.x & 31u;
    const Vec8<TYPE> mine8 = narrow8<TYPE>(v);
    const u32 *n = reinterpret_cast<const u32 *>(mine8.q);
    uint4 *p = reinterpret_cast<uint4 *>(static_cast<unsigned char *>(base) + (row_at + c - s) * type_size(TYPE));
    const bool first = (s == 0u || (lane > 0u && c > 0u)) && c + per - s <= cols;    // the chunk that starts with the neighbour's elements
    const bool next = s == 0u || (lane < 31u && c + 8u + per - s <= cols);           // the chunk the next lane completes with mine
    if constexpr (TYPE == ADACOMP_TYPE_F32) {
        u32 in[12], out[8];
#pragma unroll
        for (int i = 0; i < 4; i++) in[i] = __shfl_up_sync(kAllLanes, n[4 + i], 1);
#pragma unroll
        for (int i = 0; i < 8; i++) in[4 + i] = n[i];
        shift_words<8>(in, 4u - s, out);
#pragma unroll
        for (int i = 0; i < 8; i++) out[i] = s ? out[i] : n[i];
        const bool second = c + 8u - s <= cols;
        if (first) p[0] = make_uint4(out[0], out[1], out[2], out[3]);
        if (second) p[1] = make_uint4(out[4], out[5], out[6], out[7]);
        if (!(first && second && next)) {
#pragma unroll
            for (u32 e = 0; e < 8; e++)
                if (c + e < cols && (e < 4u - s ? !first : e < 8u - s ? !second : !next)) store1<TYPE>(base, row_at + c + e, v[e]);
        }
    } else {
        u32 in[8], y[5];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            in[i] = __shfl_up_sync(kAllLanes, n[i], 1);
            in[4 + i] = n[i];
        }
        shift_words<5>(in, (8u - s) >> 1, y);
        u32 out[4];
#pragma unroll
        for (int i = 0; i < 4; i++) out[i] = s ? __funnelshift_r(y[i], y[i + 1], (s & 1u) * 16u) : n[i];
        if (first) p[0] = make_uint4(out[0], out[1], out[2], out[3]);
        if (!(first && next)) {
#pragma unroll
            for (u32 e = 0; e < 8; e++)
                if (c + e < cols && (e < 8u - s ? !first : !next)) store1<TYPE>(base, row_at + c + e, v[e]);
        }
    }
}

// The block whose elements begin `s` elements behind p: lanes read neighbouring blocks of a line in shared memory, from
// any element on, by 8-byte and 4-byte reads (s is the same for the warp); an odd 16-bit offset shifts by half a word.
template <u32 TYPE> __device__ inline void read_at(const uint4 *p, u32 s, Vec8<TYPE> &r)
{
    constexpr bool WORDS = TYPE == ADACOMP_TYPE_F32;
    constexpr int N = WORDS ? 8 : 5;
    const u32 first = WORDS ? s : s >> 1;
    const u32 *w = reinterpret_cast<const u32 *>(p) + first;
    u32 x[N + 1];
    if (first & 1u) {
        x[0] = w[0];
#pragma unroll
        for (int i = 1; i + 1 < N + 1; i += 2) {
            if (WORDS && i == N - 1) {
                x[i] = w[i];
            } else {
                const uint2 q = *reinterpret_cast<const uint2 *>(w + i);
                x[i] = q.x, x[i + 1] = q.y;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i + 1 < N; i += 2) {
            const uint2 q = *reinterpret_cast<const uint2 *>(w + i);
            x[i] = q.x, x[i + 1] = q.y;
        }
        if (!WORDS) x[4] = w[4];
    }
    u32 *out = reinterpret_cast<u32 *>(r.q);
#pragma unroll
    for (int i = 0; i < (WORDS ? 8 : 4); i++) out[i] = WORDS ? x[i] : __funnelshift_r(x[i], x[i + 1], (s & 1u) * 16u);
}

// Rows on their way: each thread copies its chunks of the next rows into shared memory (cp.async), so that no register
// holds what has not arrived and nothing is loaded twice.  ALIGNED rows: a thread reads back what it copied itself, and
// nobody waits for anybody.  Others: a warp's chunks form a line of its own, in which every block lies shifted by the row's
// offset; the warp's lanes wait for one another.  On the way out such a row is joined into whole chunks in the same line.
// `arrays` tensors, STAGES rows of each: with two, the next row is copied while one is worked on; with one, for the widest
// rows, only once its places have been read.
template <u32 TYPE, bool ALIGNED, int NV, int THREADS, int STAGES> struct Ring {
    static constexpr u32 kPer = chunk_elems<TYPE>();
    static constexpr int kChunks = 8 / kPer;                        // of a block
    static constexpr u32 kLine = 32 * NV * kChunks + 2;             // a warp's line: one chunk more on either side
    static constexpr u32 kArray = ALIGNED ? NV * kChunks * THREADS : THREADS / 32 * kLine;      // in 16 bytes
    static constexpr size_t bytes(u32 arrays) { return (size_t)STAGES * arrays * kArray * 16; }
    uint4 *base, *mine;     // mine: this thread's first chunk
    u32 arrays, lane;
    __device__ Ring(void *smem, u32 n)
        : base(static_cast<uint4 *>(smem)),
          mine(base + (ALIGNED ? threadIdx.x : (threadIdx.x >> 5) * kLine + 1 + (threadIdx.x & 31u) * kChunks)), arrays(n),
          lane(threadIdx.x & 31u)
    {
    }
    __device__ uint4 *place(u32 turn, u32 array) const { return mine + ((turn & (STAGES - 1)) * arrays + array) * kArray; }
    __device__ void *end() const { return base + STAGES * arrays * kArray; }
    __device__ static constexpr u32 at(int k, int i) { return ALIGNED ? (k * kChunks + i) * THREADS : k * 32 * kChunks + i; }
    // Blocks k = 0, 1, .. start at columns c + 256 k of the row at element row_at; columns before `last` are wanted.
    __device__ void copy(uint4 *to, const void *from, u64 row_at, u32 c, u32 last) const
    {
        const u32 s = ALIGNED ? 0u : (u32)row_at & (kPer - 1u);
        const unsigned char *p = static_cast<const unsigned char *>(from) + (row_at + c - s) * type_size(TYPE);
        const u32 dst = smem_addr(to);
#pragma unroll
        for (int k = 0; k < NV; k++)
#pragma unroll
            for (int i = 0; i < kChunks; i++) {
                const int first = (int)(c + 256 * k + i * kPer) - (int)s;       // a column of this chunk, or below 0
                copy_if(last > 0u && first < (int)last, dst + at(k, i) * 16, p + (256 * k + i * kPer) * type_size(TYPE));
            }
        if (!ALIGNED && s != 0u)
            copy_if(lane == 31u && c + 256 * (NV - 1) + 8u - s < last, dst + at(NV - 1, kChunks) * 16,
                    p + (256 * (NV - 1) + 8u) * type_size(TYPE));
    }
    __device__ static void copy_if(bool on, u32 dst, const void *p)
    {
        asm volatile("{\n\t.reg .pred on;\n\tsetp.ne.u32 on, %2, 0;\n\t@on cp.async.cg.shared.global [%0], [%1], 16;\n\t}" ::"r"(dst),
                     "l"(p), "r"((u32)on)
                     : "memory");
    }
    // Before copies into places that have been read.
    __device__ static void release()
    {
        if (!ALIGNED) __syncwarp();
    }
    // What was asked for before the last request has arrived (one stage: the last request itself).
    __device__ static void wait()
    {
        if (STAGES == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
        if (!ALIGNED) __syncwarp();
    }
    // Block k in binary32 (see mask_from for its elements that were not asked for).
    __device__ static void read(const uint4 *from, int k, u64 row_at, float (&v)[8])
    {
        Vec8<TYPE> r;
        if constexpr (ALIGNED) {
#pragma unroll
            for (int i = 0; i < kChunks; i++) r.q[i] = from[at(k, i)];
        } else {
            read_at<TYPE>(from + at(k, 0), (u32)row_at & (kPer - 1u), r);
        }
        widen8<TYPE>(r, v);
    }
    // The row's elements from column `last` on, in blocks `first` to `count` - 1, become `bits` (an element, repeated).
    __device__ static void fill(uint4 *row, u64 row_at, u32 c, u32 last, int first, int count, u32 bits)
    {
        const int s = ALIGNED ? 0 : (int)((u32)row_at & (kPer - 1u));
        if (!ALIGNED) __syncwarp();
        // (not ALIGNED: one chunk more, which only the last lane's last block has to itself)
#pragma unroll 1
        for (int k = first; k < count; k++)
#pragma unroll
            for (int i = 0; i < kChunks + (ALIGNED ? 0 : 1); i++) {
                if (i == kChunks && threadIdx.x % 32u != 31u) continue;
                const int keep = (int)last - ((int)(c + 256 * k + i * kPer) - s);       // elements of this chunk that stay
                uint4 *p = row + at(k, i);
                if (keep <= 0) {
                    *p = make_uint4(bits, bits, bits, bits);
                } else if (keep < (int)kPer) {
                    uint4 q = *p;
                    u32 *w = reinterpret_cast<u32 *>(&q);
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        if (TYPE == ADACOMP_TYPE_F32) w[j] = j < keep ? w[j] : bits;
                        else w[j] = 2 * j + 1 < keep ? w[j] : 2 * j < keep ? __byte_perm(w[j], bits, 0x5410) : bits;
                    }
                    *p = q;
                }
            }
        if (!ALIGNED) __syncwarp();
    }
    // Places that no copy reaches, where the kernel counts on zeros behind a row's end.
    __device__ void clear(u32 c, u32 last) const
    {
        if constexpr (ALIGNED) {
            for (u32 j = 0; j < STAGES * arrays; j++)
#pragma unroll
                for (int k = 0; k < NV; k++)
#pragma unroll
                    for (int i = 0; i < kChunks; i++)
                        if (c + 256 * k >= last) mine[j * kArray + at(k, i)] = make_uint4(0u, 0u, 0u, 0u);
        }
    }
    // Stores the row's columns before `cols`; `line`: places of this thread's row that have been read, which a row that is
    // not ALIGNED goes through.
    __device__ void store(void *to, u64 row_at, u32 c, u32 cols, const float (&v)[NV][8], uint4 *line) const
    {
        const u32 s = ALIGNED ? 0u : (u32)row_at & (kPer - 1u);
        if (ALIGNED || s == 0u) {
#pragma unroll
            for (int k = 0; k < NV; k++) store_block<TYPE, true>(to, row_at, c + 256 * k, cols, v[k]);
            return;
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < NV; k++) {
            const Vec8<TYPE> r = narrow8<TYPE>(v[k]);
#pragma unroll
            for (int i = 0; i < kChunks; i++) line[at(k, i)] = r.q[i];
        }
        __syncwarp();
        // The warp's columns are first .. end - 1.  Chunks that lie inside them are stored whole, by the lane whose block
        // begins in them ...
        const u32 first = c - 8u * lane, end = min(cols, first + 256u * NV);
        unsigned char *p = static_cast<unsigned char *>(to) + (row_at + c - s) * type_size(TYPE);
#pragma unroll
        for (int k = 0; k < NV; k++) {
            Vec8<TYPE> r;
            read_at<TYPE>(line + at(k, 0) - 1, kPer - s, r);
#pragma unroll
            for (int i = 0; i < kChunks; i++)
                if ((k > 0 || i > 0 || lane > 0u) && c + 256 * k + (i + 1) * kPer - s <= end)
                    *reinterpret_cast<uint4 *>(p + (256 * k + i * kPer) * type_size(TYPE)) = r.q[i];
        }
        // ... and the few elements before the first and behind the last of them one by one, a lane each.
        if (first < end) {
            const u32 from = min(first + kPer - s, end), behind = from + (end - from) / kPer * kPer;
            const u32 col = lane < 8u ? first + lane : behind + lane - 8u;
            if (lane < 16u && (lane < 8u ? col < from : col < end)) {
                const unsigned char *q = reinterpret_cast<const unsigned char *>(line - lane * kChunks) + (col - first) * type_size(TYPE);
                unsigned char *g = static_cast<unsigned char *>(to) + (row_at + col) * type_size(TYPE);
                if (TYPE == ADACOMP_TYPE_F32) *reinterpret_cast<u32 *>(g) = *reinterpret_cast<const u32 *>(q);
                else *reinterpret_cast<unsigned short *>(g) = *reinterpret_cast<const unsigned short *>(q);
            }
        }
    }
};

// A parameter vector (its type known at run time; it starts on a vector boundary).
__device__ inline void load_param(const void *p, u32 type, u32 c, u32 cols, float fill, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = fill;
    if (!p || c >= cols) return;
    if (c + 8 > cols) {
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (c + e < cols)
                v[e] = type == ADACOMP_TYPE_F32 ? load1<ADACOMP_TYPE_F32>(p, c + e)
                       : type == ADACOMP_TYPE_BF16 ? load1<ADACOMP_TYPE_BF16>(p, c + e) : load1<ADACOMP_TYPE_F16>(p, c + e);
    } else if (type == ADACOMP_TYPE_F32) {
        widen8<ADACOMP_TYPE_F32>(load8<ADACOMP_TYPE_F32>(p, c), v);
    } else if (type == ADACOMP_TYPE_BF16) {
        widen8<ADACOMP_TYPE_BF16>(load8<ADACOMP_TYPE_BF16>(p, c), v);
    } else {
        widen8<ADACOMP_TYPE_F16>(load8<ADACOMP_TYPE_F16>(p, c), v);
    }
}

// ---------------------------------------------------------------------------------
// dropout: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011)
// key = seed, counter = (column / 8, row, step, site); the 128 bits are eight 16-bit numbers, one per column of the
// group (low half of a word first).  Sixteen bits per element rather than 32 halve the generator's work; the kept
// fraction is then a multiple of 2^-16, and the factor is the reciprocal of exactly that fraction.
// ---------------------------------------------------------------------------------

struct DropArgs {
    const u64 *rng;          // device: {seed, step}
    u32 site, threshold;     // an element is dropped when its 16 bits are below the threshold (0 .. 65536)
    float factor;
};

struct Drop {
    u32 k0, k1, step, site;
    u32 last;                // threshold * 2^16 - 1
    float factor;
};

// (for thresholds above 0)
__device__ inline Drop drop_begin(const DropArgs &a)
{
    const u64 seed = a.rng[0], step = a.rng[1];
    return {(u32)seed, (u32)(seed >> 32), (u32)step, a.site, (a.threshold << 16) - 1u, a.factor};
}

// The eight 16-bit numbers of N blocks: group[i] of row[i].  The blocks go through the rounds together: they share the
// additions to the key, and (in one row) what the first two rounds make of the counter's constant parts.
template <int N> __device__ inline void drop_words(const Drop &d, const u32 (&row)[N], const u32 (&group)[N], u32 (&out)[N][4])
{
    u32 k0 = d.k0, k1 = d.k1;
#pragma unroll
    for (int i = 0; i < N; i++) out[i][0] = group[i], out[i][1] = row[i], out[i][2] = d.step, out[i][3] = d.site;
#pragma unroll
    for (int r = 0; r < 10; r++) {
#pragma unroll
        for (int i = 0; i < N; i++) {
            u32(&c)[4] = out[i];
            const u64 a = (u64)c[0] * 0xD2511F53u, b = (u64)c[2] * 0xCD9E8D57u;
            c[0] = (u32)(b >> 32) ^ c[1] ^ k0;
            c[2] = (u32)(a >> 32) ^ c[3] ^ k1;
            c[1] = (u32)b;
            c[3] = (u32)a;
        }
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

__device__ inline void drop_words(const Drop &d, u32 row, u32 group, u32 (&out)[4])
{
    const u32 rows[1] = {row}, groups[1] = {group};
    u32 w[1][4];
    drop_words<1>(d, rows, groups, w);
#pragma unroll
    for (int i = 0; i < 4; i++) out[i] = w[0][i];
}

// Whether element e of a block is dropped: its half of the words is below the threshold.  For the high halves a comparison
// of the whole word with threshold * 2^16 - 1 says the same.
__device__ inline bool dropped(const Drop &d, const u32 (&w)[4], int e)
{
    return ((e & 1) ? w[e >> 1] : w[e >> 1] << 16) <= d.last;
}

// v = dropout(v): selected, not multiplied, so that infinities and NaN in dropped places leave zeros.
__device__ inline void drop_apply(const Drop &d, const u32 (&w)[4], float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        float x, y;
        mul2(x, y, v[e], v[e + 1], d.factor, d.factor);
        v[e] = dropped(d, w, e) ? 0.f : x;
        v[e + 1] = dropped(d, w, e + 1) ? 0.f : y;
    }
}

// ---------------------------------------------------------------------------------
// sums over a row's threads
// ---------------------------------------------------------------------------------

__device__ inline float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kAllLanes, v, d);
    return v;
}

// The warp's largest value; NaN is passed over.
__device__ inline float warp_max(float v)
{
    float m;
    asm volatile("redux.sync.max.f32 %0, %1, %2;" : "=f"(m) : "f"(v), "r"(kAllLanes));
    return m;
}

// N sums over the warp at once (N = 1, 2, 4 or 8).  While there are several values left, a step halves them: a lane keeps
// one half of the values and gives away the other, so that N sums take N + 4 - log2 N exchanges instead of 5 N.  Returns
// the sum of value lane / (32 / N).
template <int N> __device__ inline float warp_sums(const float (&v)[N], u32 lane)
{
    float x[N];
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = v[i];
    int d = 16;
#pragma unroll
    for (int n = N; n > 1; n /= 2, d /= 2) {
        const bool up = lane & d;
#pragma unroll
        for (int i = 0; i < n / 2; i++)
            x[i] = (up ? x[i + n / 2] : x[i]) + __shfl_xor_sync(kAllLanes, up ? x[i] : x[i + n / 2], d);
    }
#pragma unroll
    for (; d > 0; d /= 2) x[0] += __shfl_xor_sync(kAllLanes, x[0], d);
    return x[0];
}

// The sum over each half of the warp.
__device__ inline float half_sum(float v)
{
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) v += __shfl_xor_sync(kAllLanes, v, d);
    return v;
}

__device__ inline float from_lane(float v, int lane) { return __shfl_sync(kAllLanes, v, lane); }

// The threads of one row: `tpr` neighbouring threads of a CTA, at most 16 warps.  Rows of up to one warp need no barrier, others meet at
// named barrier 1 + g (at most 15 rows share a CTA then).
struct RowGroup {
    u32 g, t, tpr, warps, warp, lane, first_warp;
    __device__ explicit RowGroup(u32 threads_per_row)
        : g(threadIdx.x / threads_per_row), t(threadIdx.x - g * threads_per_row), tpr(threads_per_row),
          warps(threads_per_row >> 5), warp(t >> 5), lane(t & 31u), first_warp(g * warps)
    {
    }
    __device__ void sync() const
    {
        if (warps == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(g + 1u), "r"(tpr) : "memory");
    }
};

// Where the warps of a row leave N values for one another: slots of 16, those of missing warps zero.
template <int N> struct RowSlots { float v[N][16]; };

// The sums of N values over the threads of a row, in all of them.  `slots`: this row's; the caller alternates between two
// sets and clears both before the first use.
template <int N> __device__ inline void row_sums(float (&v)[N], const RowGroup &rg, RowSlots<N> &slots)
{
    constexpr u32 span = 32 / N;                // lanes that share a value
    const u32 which = rg.lane / span, j = rg.lane % span;
    float x = warp_sums<N>(v, rg.lane);
    if (rg.warps > 1) {
        if (j == 0) slots.v[which][rg.warp] = x;
        rg.sync();
        if constexpr (span >= 16) {
            x = j < 16 ? slots.v[which][j] : 0.f;
        } else if constexpr (span == 8) {
            const float2 p = reinterpret_cast<const float2 *>(slots.v[which])[j];
            x = p.x + p.y;
        } else {
            const float4 p = reinterpret_cast<const float4 *>(slots.v[which])[j];
            x = (p.x + p.y) + (p.z + p.w);
        }
#pragma unroll
        for (int d = (span > 16 ? 16 : (int)span) / 2; d > 0; d /= 2) x += __shfl_xor_sync(kAllLanes, x, d);
    }
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = from_lane(x, i * (int)span);
}

// The CTAs of a cluster meet; what threads 0 .. 31 wrote to one another's shared memory before is seen by all after.  (Only
// they release: a release waits for all the thread's stores, those of the last row among them.)
__device__ inline void cluster_meet()
{
    if (threadIdx.x < 32u) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    else asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// n / d for n < 2^31 by a multiplication (Granlund and Montgomery, "Division by invariant integers using
// multiplication", 1994)
struct FastDiv {
    u32 d, mul, shift;
};

inline FastDiv make_fastdiv(u32 d)
{
    u32 s = 0;
    while ((1ull << s) < d) s++;
    return {d, (u32)(((1ull << 32) * ((1ull << s) - d)) / d + 1), s};
}

__device__ inline u32 fast_div(u32 n, const FastDiv &f) { return (__umulhi(n, f.mul) + n) >> f.shift; }

}  // namespace adacomp_impl
