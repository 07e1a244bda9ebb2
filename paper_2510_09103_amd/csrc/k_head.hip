// Softmax cross entropy of logits s = x W^T that are never kept, and its gradient.
//
//   forward   lse_i = log sum_v exp s_iv,  loss_i = lse_i - s_i,t_i
//   backward  P = w_i (exp(s - lse) - onehot),  dx = f P W,  dW = f P^T x      (f: reduction, scale, upstream gradient)
//
// Forward: a workgroup makes one tile of logits on the matrix cores and leaves only the maximum and the sum of exponentials of its
// columns for every row; a second launch joins them.  Backward: the vocabulary is taken in pieces; for each, P is made from fresh
// logits and stored in the type of x (a piece is about PIECE_BYTES or 2048 vocabulary rows, not the rows x vocab of all logits), then one launch adds
// its part to dx and writes its rows of dW.  The logits are made twice: to keep them in fp32
// takes rows x vocab x 4 bytes, 1 GB for 8192 rows over 32000, which the operator is there to save.  For time alone it would depend on the columns: a
// logit made again costs 2 cols flop, 0.8 ps of the matrix cores at 512 columns and 3.3 ps at 2048 (1240 TFLOP/s), one kept 8 bytes written and
// read, 1.6 ps of memory.  From about 1000 columns on chunks of rows whose logits stay small could be quicker, against a dW that
// is added up in fp32 over the chunks; that is not built, and not measured.
//
// Rows without a target are left out before anything else: the rows that count are packed side by side (padded to whole steps of the
// contraction; where all count and lie well, x itself is read), so masked rows cost nothing, and whatever stands in them (NaN included) reaches no sum.
#include "ew_math.h"
#include "ops_plan.h"

#include <cmath>

namespace adapm {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef u32x2 u32x2_e2 __attribute__((aligned(2), may_alias));
typedef f32x4 f32x4_e4 __attribute__((aligned(4), may_alias));
typedef __attribute__((address_space(3))) unsigned char lds_u8;

constexpr unsigned OOB = 0x80000000u;                 // an offset past every descriptor's end: reads zeros
constexpr int64_t PIECE_BYTES = (int64_t)256 << 20;   // most of P at a time: the size of the last-level cache
constexpr float LOG2E = 1.44269504088896340736f;

struct HeadHeader {
  int n;                                              // rows that count
  int pad[63];
};

// n: rows that count; without any the gradients are zeros, whatever the upstream gradient (infinite or NaN where a loss scale overflowed)
__device__ __forceinline__ float grad_factor(const HeadDev& h, int n) {
  if (n == 0) return 0.f;
  const float f = h.scale * (h.upstream ? *h.upstream : 1.f);
  return h.mean ? f / (float)n : f;
}

// Few rows that count: P travels as two bf16 numbers, P rounded and what that has left out, 2^-17 of it in all.  A gradient in bf16 has an
// error of its own, 1.66e-3 of it in root mean square.  P rounded once adds another, most of it from one element a row, the target's, and it
// does not average out over the rows: from 33 to 4096 of them the whole is 1.07 times the least without weights (the targets' elements
// near -1 lose little) and 1.42 times with weights on the rows (w (p - 1) loses as much as any number); 1.26 and 1.77 at worst in 40 problems
// of 32 rows.  Two numbers leave 1.00.  Where they end is a matter of time: the second numbers are more rows of P, against a second copy
// of x; dW's contraction takes them in, and dx's sums for them are added to those of the first.  Up to 32 rows reading W covers that (32000 x
// 2048, 32 rows with two numbers 96 us, 33 with one 96).  With weights, where they gain most, they are taken up to 1024 rows (512 rows 347 us
// against 224, 1024 rows 620 against 398); beyond, where the products are all of the time, a batch is not made half as long again for them.
// How many rows count is known on the device alone: there is space for the second numbers of up to that many in any batch.
constexpr int TWIN_ROWS = 32, TWIN_ROWS_WEIGHTED = 1024;
__device__ __forceinline__ int twin(const HeadDev& h, int n) { return n > 0 && n <= h.twin_rows ? 1 : 0; }

// ---- rows that count -------------------------------------------------------------------------------------------------
// The few rows of a forward pass whose x can be read where it is are not packed (h.direct): each has a column of logits to itself, and
// one that does not count is left out behind the products.
constexpr int COUNT_ROWS = 1024;                      // rows of a workgroup of the count, and of an entry of its result
constexpr int PACK_ROWS = 16;                         // rows of a workgroup of the packing
constexpr int PACK_GROUPS = 512;                      // few rows: up to so many workgroups, which share the columns (16 x 2048 9.7 -> 4.5 us)
constexpr int DIRECT_ROWS = 256;                      // most rows that are not packed: a tile's, W is what they cost
constexpr int JOINED_ROWS = 32;                       // most of them that one workgroup joins, which leaves the loss itself

__device__ __forceinline__ bool counts(const HeadDev& h, int64_t row) {
  const int64_t t = h.targets[row];
  return t >= 0 && t < h.vocab;
}

// Many rows that all count, as in pre-training, are not copied either: how many count is known before the packing.  8192 rows over
// 32000 x 2048, loss and gradients, 3487 -> 3445 us.
__device__ __forceinline__ bool whole(const HeadDev& h, int n) { return h.whole && n == h.rows; }
static_assert(TWIN_ROWS <= COUNT_ROWS && TWIN_ROWS_WEIGHTED <= COUNT_ROWS, "rows that are read where they are have no second copy");

__device__ __forceinline__ int live_rows(const HeadDev& h) {
  return h.direct ? (int)h.rows : reinterpret_cast<const HeadHeader*>(h.ws + h.lay.head)->n;
}

__global__ __launch_bounds__(256) void count_kernel(HeadDev h) {
  __shared__ int red[4];
  int c = 0;
  for (int i = threadIdx.x; i < COUNT_ROWS; i += 256) {
    const int64_t row = (int64_t)blockIdx.x * COUNT_ROWS + i;
    c += row < h.rows && counts(h, row) ? 1 : 0;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) c += __shfl_xor(c, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = c;
  __syncthreads();
  if (threadIdx.x == 0) reinterpret_cast<int*>(h.ws + h.lay.counts)[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

typedef u32x4 u32x4_e2 __attribute__((aligned(2), may_alias));

// elements c0 .. of a row of `cols` as 16 bytes, zeros behind its end
template <class T>
__device__ __forceinline__ u32x4 piece_of(const T* row, int c0, int cols) {
  constexpr int V = 16 / sizeof(T);
  if (c0 + V <= cols) return *reinterpret_cast<const u32x4_e2*>(row + c0);
  union {
    T t[V];
    u32x4 v;
  } r;
#pragma unroll
  for (int i = 0; i < V; ++i) r.t[i] = c0 + i < cols ? row[c0 + i] : T(0);
  return r.v;
}

// Places of the rows that count (in their order) and their packed copies.  A workgroup finds how many stand before its own from
// the counts of the thousands before and from the targets of its own thousand.
template <class T>
__global__ __launch_bounds__(256) void pack_kernel(HeadDev h) {
  __shared__ unsigned long long red[4];
  __shared__ int place[PACK_ROWS];
  const int64_t r0 = (int64_t)blockIdx.x * PACK_ROWS;
  const int64_t b0 = r0 / COUNT_ROWS;
  unsigned long long c = 0;          // those before the workgroup's rows; where it is wanted, all in the upper half
  constexpr unsigned long long ONE_OF_ALL = 1ull << 32;
  const int* counted = reinterpret_cast<const int*>(h.ws + h.lay.counts);
  for (int64_t i = threadIdx.x; i < b0; i += 256) c += counted[i];
  for (int64_t row = b0 * COUNT_ROWS + threadIdx.x; row < r0; row += 256) c += counts(h, row) ? 1 : 0;
  if (h.rows > COUNT_ROWS) {
    for (int64_t i = threadIdx.x; i * COUNT_ROWS < h.rows; i += 256) c += counted[i] * ONE_OF_ALL;
  } else if (h.twin_rows) {
    for (int64_t row = threadIdx.x; row < h.rows; row += 256) c += counts(h, row) ? ONE_OF_ALL : 0;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) c += __shfl_xor(c, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = c;
  __syncthreads();
  const unsigned long long sum = red[0] + red[1] + red[2] + red[3];
  const int before = (int)(uint32_t)sum, all = (int)(sum >> 32);
  if (threadIdx.x < 64) {
    const int64_t row = r0 + threadIdx.x;
    const bool in = threadIdx.x < PACK_ROWS && row < h.rows;
    const bool live = in && counts(h, row);
    const unsigned long long m = __ballot(live);
    const int j = before + __popcll(m & ((1ull << threadIdx.x) - 1));
    if (in) place[threadIdx.x] = live ? j : -1;
    if (in && blockIdx.y == 0) {
      reinterpret_cast<int*>(h.ws + h.lay.place)[row] = live ? j : -1;
      if (live) {
        reinterpret_cast<int*>(h.ws + h.lay.list)[j] = (int)row;
        reinterpret_cast<int*>(h.ws + h.lay.target)[j] = (int)h.targets[row];
        reinterpret_cast<float*>(h.ws + h.lay.weight)[j] = h.row_weight ? h.row_weight[row] : 1.f;
        if (!h.row_loss) reinterpret_cast<float*>(h.ws + h.lay.lse)[j] = h.lse[row];       // backward
      } else if (h.row_loss) {
        h.row_loss[row] = 0.f;
        h.lse[row] = 0.f;
      }
    }
    if (threadIdx.x == 0 && blockIdx.y == 0 && r0 + PACK_ROWS >= h.rows) reinterpret_cast<HeadHeader*>(h.ws + h.lay.head)->n = before + __popcll(m);
  }
  __syncthreads();
  if (whole(h, all)) return;
  // pieces of 16 bytes of all the rows at once, whatever alignment x has; zeros behind its columns
  constexpr int V = 16 / sizeof(T);
  const int per = h.pitch / V;
  for (int i = blockIdx.y * 256 + threadIdx.x; i < PACK_ROWS * per; i += 256 * gridDim.y) {
    const int r = i / per, c0 = (i - r * per) * V;
    if (r0 + r >= h.rows || place[r] < 0) continue;
    T* to = reinterpret_cast<T*>(h.ws + h.lay.x) + (int64_t)place[r] * h.pitch + c0;
    const u32x4 v = piece_of(reinterpret_cast<const T*>(h.x.p) + (r0 + r) * h.x.stride, c0, h.cols);
    *reinterpret_cast<u32x4*>(to) = v;
    if (twin(h, all)) *reinterpret_cast<u32x4*>(to + (int64_t)all * h.pitch) = v;
  }
}

// W with rows that are no whole, aligned vectors
template <class T>
__global__ __launch_bounds__(256) void pack_w_kernel(HeadDev h) {
  constexpr int V = 16 / sizeof(T);
  const int per = h.pitch / V;
  const int64_t r0 = (int64_t)blockIdx.x * PACK_ROWS;
  for (int i = threadIdx.x; i < PACK_ROWS * per; i += 256) {
    const int r = i / per, c0 = (i - r * per) * V;
    if (r0 + r >= h.vocab) return;
    *reinterpret_cast<u32x4*>(reinterpret_cast<T*>(h.ws + h.lay.w) + (r0 + r) * h.pitch + c0) =
        piece_of(reinterpret_cast<const T*>(h.w.p) + (r0 + r) * h.w.stride, c0, h.cols);
  }
}

// ---- matrix products -------------------------------------------------------------------------------------------------
// A tile of D[m][n] = sum_k A(m, k) B(n, k).  An operand is stored with k along its rows (KC: element (u, k) at u pitch + k) or
// across them (at k pitch + u).  128-byte slices of the contraction (64 bf16 or 32 fp32 values, two steps of fragments: whole cache lines
// where k goes along the rows) are copied straight into one of two to four LDS buffers; which 16-byte piece of a slice a thread fetches is
// exchanged (by the LDS row's number) so that the reads of a fragment fall on different banks without padding.
// bf16: v_mfma_f32_16x16x32, KC fragments are one 16-byte read, the others two transposing reads of 8 bytes.
// fp32: v_mfma_f32_16x16x4, four of them to a 16-byte read; which k meets which instruction is the same for both operands.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t a = (uint64_t)p;
  return (const char*)((uint64_t)(uint32_t)uniform((int)(uint32_t)(a >> 32)) << 32 | (uint32_t)uniform((int)(uint32_t)a));
}

struct Src {
  const char* p;        // element (0, 0)
  int64_t pitch;        // bytes
  int u, k;             // extent of the free index and of the contraction, in elements
};

// Which row of a wavefront's tiles a fragment's row is.  As they come, fragment i, row r: 16 i + r; an accumulator then holds four
// neighbouring rows, 16 apart from those of the next tile.  PAIRS (the vocabulary rows of the logits): two tiles take 32 rows in turns of
// four, so that the accumulators of the two hold eight neighbouring rows, 16 bytes of bf16.
__device__ __forceinline__ constexpr int pair_row(int i, int r) { return 32 * (i >> 1) + 8 * (r >> 2) + 4 * (i & 1) + (r & 3); }

template <class T, int BU, int NTHR, bool KC, bool PAIRS = false>
struct Operand {
  static constexpr int ES = sizeof(T);
  static constexpr int BK = 128 / ES;                 // elements of the contraction in a slice
  static constexpr int BYTES = BU * 128;
  static constexpr int NL = BYTES / (16 * NTHR);      // 16-byte pieces of a thread
  static constexpr int RPC = BU * ES / 16;            // pieces of a row where k goes across
  static_assert(NL * 16 * NTHR == BYTES, "whole pieces");
  // Where a piece stands.  KC: its place among the eight of its row is exchanged by the row's number (PAIRS: by those of its bits in which the
  // rows of one fragment differ).  The 256 bytes of a cycle are those of lanes 0 - 3, 12 - 15, 20 - 23, 24 - 27, and so on in fours:
  // rows 1 and 2 of four go with the next piece of rows 0 and 3.  Else pieces of 32 bytes (bf16; a
  // read touches rows 0 .. 3 and 8 .. 11 of a step at a time) or 64 bytes (fp32; rows 0, 4, 8 and 12) are exchanged by the row, over the
  // 256 bytes of all banks: where an LDS row is 128 or 64 bytes, its number's lowest bits say which half or quarter it lies in already.
  static_assert(KC || (ES == 2 && BU * ES == 64) || BU * ES == 128 || BU * ES >= 256, "exchanged inside a row");
  static __device__ __forceinline__ int swz(int k) {
    if (ES == 4) return BU * ES == 128 ? (k >> 2) & 1 : (k >> 2) & 3;        // 128 bytes: two of the four rows share banks
    if (BU * ES == 64) return (k >> 3) & 1;
    return BU * ES == 128 ? ((k >> 1) & 1) | ((k >> 2) & 2) : (k & 3) | ((k >> 1) & 4);
  }

  static __device__ __forceinline__ int swz_kc(int row) {
    if (!PAIRS) return row & 7;
    const int a = row >> 3;
    return ((a ^ (a << 1 & 2)) & 3) | (row << 1 & 4);
  }

  int off[NL];          // byte offset of a thread's pieces in the slice that starts at k = 0, OOB outside the free index
  int k_in;             // KC: place of its pieces in the slice (the same for all)
  const char* base;

  __device__ __forceinline__ void init(const Src& s, int u0) {
    const int tid = threadIdx.x;
    k_in = 0;
    if (KC) {
      base = s.p + (int64_t)u0 * s.pitch;
      k_in = ((tid & 7) ^ swz_kc(tid >> 3)) * (16 / ES);
#pragma unroll
      for (int i = 0; i < NL; ++i) off[i] = ((tid + NTHR * i) >> 3) * (int)s.pitch + k_in * ES;
    } else {
      base = s.p;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int c = tid + NTHR * i, row = c / RPC, at = c % RPC;
        const int cu = ES == 2 ? ((at >> 1) ^ swz(row)) << 1 | (at & 1) : ((at >> 2) ^ swz(row)) << 2 | (at & 3);
        const int u = u0 + cu * (16 / ES);
        off[i] = u < s.u ? row * (int)s.pitch + u * ES : (int)OOB;
      }
    }
  }

  // Asynchronous copy of the slice at k0.  A lane outside the operand gets zeros, and so do all of them at and behind `end` (<= s.k): every
  // slice is the same number of copies, which is what the waits count.
  __device__ __forceinline__ void copy(const Src& s, int u0, int k0, int end, lds_u8* lds) const {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int left = end - k0, rows = KC ? (s.u - u0 < BU ? s.u - u0 : BU) : left < 0 ? 0 : left < BK ? left : BK;
    const char* from = KC ? base : base + (int64_t)k0 * s.pitch;      // formed, not read, behind the end
    // uniform values that the compiler may have worked out in vector registers
    const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(uniform(from)), 0, uniform(rows * (int)s.pitch), 0x00020000);
    const bool in = k_in < left;
#pragma unroll
    for (int i = 0; i < NL; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)(lds + (NTHR * i + 64 * wave) * 16), 16,
                                               !KC || in ? off[i] : (int)OOB, KC ? uniform(k0 * ES) : 0, 0, 0);
  }
};

// Fragment of 16 rows u .. u + 15 for step ks of a slice: eight (bf16) or four (fp32) values of the contraction for this lane.  `place` is
// the lane's byte for ks = 0 and u = u0, the first row of the wavefront, the fragment's rows are u0 + 16 i: u0 / 16 is a multiple of the number of fragments, a
// power of two, so that i can be exchanged with the lane's number by the same exclusive or.
template <class T, int BU, bool KC, bool PAIRS = false>
__device__ __forceinline__ int fragment_place(int u0) {
  constexpr int ES = sizeof(T);
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
  if (KC) {
    const int row = PAIRS ? pair_row(0, l16) : l16;
    return (u0 + row) * 128 + ((q ^ Operand<T, BU, 64, KC, PAIRS>::swz_kc(row)) << 4);
  }
  // bf16: lane s of a block of 16 points at row s / 4, columns 4 (s % 4) .. + 3 of a 4 x 16 tile; lane i receives column i of the four rows
  const int k = ES == 2 ? q * 8 + (l16 >> 2) : q * 4;
  const int block = (u0 >> 4) ^ Operand<T, BU, 64, KC>::swz(k);
  return k * (BU * ES) + (ES == 2 ? (block << 5) + ((l16 & 3) << 3) : (block << 6) + (l16 << 2));
}
template <class T, int BU, bool KC, bool PAIRS = false>
__device__ __forceinline__ u32x4 fragment(const lds_u8* lds, int place, int i, int ks) {
  constexpr int ES = sizeof(T);
  if (KC) return *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(lds + (place ^ (ks << 6)) + (PAIRS ? pair_row(i, 0) : 16 * i) * 128);
  lds += ks * (64 / ES) * (BU * ES);
  union {
    s16x4 h[2];
    float f[4];
    u32x4 v;
  } r;
  if (ES == 2) {
    const lds_u8* p = lds + (place ^ (i << 5));
#pragma unroll
    for (int h = 0; h < 2; ++h) r.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + h * 4 * (BU * ES)));
  } else {
    const lds_u8* p = lds + (place ^ (i << 6));
#pragma unroll
    for (int j = 0; j < 4; ++j) r.f[j] = *reinterpret_cast<const __attribute__((address_space(3))) float*>(p + j * (BU * ES));
  }
  return r.v;
}

__device__ __forceinline__ f32x4 mma(const u32x4& a, const u32x4& b, f32x4 c, const uint16_t*) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(const u32x4& a, const u32x4& b, f32x4 c, const float*) {
  const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
  return c;
}

// waves WM x WN, each MT x NT tiles of 16 x 16, and DEPTH buffers for slices
template <class T_, int MT_, int NT_, int WM_, int WN_, int DEPTH_ = 2>
struct Cfg {
  typedef T_ T;
  static constexpr int MT = MT_, NT = NT_, WM = WM_, WN = WN_, DEPTH = DEPTH_;
  static constexpr int BM = 16 * MT * WM, BN = 16 * NT * WN, THREADS = 64 * WM * WN;
  static constexpr int SLICE = (BM + BN) * 128;
};
// the buffers, as arrays of their own: the compiler then knows which copies a read has to wait for
#define HEAD_BUFFERS                                                                                                                   \
  __shared__ __attribute__((aligned(128))) unsigned char buffer0[C::SLICE], buffer1[C::SLICE], buffer2[C::DEPTH > 2 ? C::SLICE : 16],  \
      buffer3[C::DEPTH > 3 ? C::SLICE : 16];                                                                                           \
  const Buffers lds{(lds_u8*)buffer0, (lds_u8*)buffer1, (lds_u8*)buffer2, (lds_u8*)buffer3};
struct Buffers {
  lds_u8 *p0, *p1, *p2, *p3;
};

template <class C>
struct Acc {
  f32x4 v[C::MT][C::NT];
};

// What the wavefronts of a tile do.  A slice is four phases, each half of the wavefront's rows of tiles in one step: read the fragments,
// multiply them.  With eight wavefronts there are two on each SIMD, and those of the second half of the workgroup are kept
// one half of a phase behind the first: while one multiplies, with priority, the other reads, and the matrix cores are not left waiting
// for either.  The barriers between the halves of the phases hold them so.  With four wavefronts the workgroups on a compute unit do
// that for one another by chance.
// In the first two phases the slice DEPTH - 1 further on is copied into the buffer that was used last; before the last multiplication
// every wavefront has seen its own copies of the next slice arrive and its last fragments leave the buffer that the next copies go to.
template <class C, bool AKC, bool BKC>
struct Product {
  typedef typename C::T T;
  typedef Operand<T, C::BM, C::THREADS, AKC, AKC> OA;      // k along the rows: the logits' vocabulary rows
  typedef Operand<T, C::BN, C::THREADS, BKC> OB;
  static constexpr int BK = OA::BK, HALF = C::MT / 2;
  static constexpr int COPIES = OA::NL + OB::NL, LEFT = (C::DEPTH - 2) * COPIES;        // LEFT: copies still on their way at that point
  static constexpr bool PAIRED = C::THREADS == 512;
  static_assert(C::MT % 2 == 0, "two halves");
  const Src A, B;
  const int m0, n0, k1;
  const int pa, pb;       // places of the lane's fragments in a slice
  OA a;
  OB b;

  static __device__ __forceinline__ void barrier() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  static __device__ __forceinline__ void turn() {
    if (PAIRED) barrier();
  }
  __device__ __forceinline__ void read_a(u32x4 (&f)[HALF], const lds_u8* slice, int half, int ks) const {
    int place = pa;
    asm volatile("" : "+v"(place));      // worked out here every time: kept for all fragments the addresses would take too many registers
#pragma unroll
    for (int i = 0; i < HALF; ++i) f[i] = fragment<T, C::BM, AKC, AKC>(slice, place, half * HALF + i, ks);
  }
  __device__ __forceinline__ void read_b(u32x4 (&f)[C::NT], const lds_u8* slice, int ks) const {
    int place = pb;
    asm volatile("" : "+v"(place));
#pragma unroll
    for (int j = 0; j < C::NT; ++j) f[j] = fragment<T, C::BN, BKC>(slice + OA::BYTES, place, j, ks);
  }
  static __device__ __forceinline__ void multiply(const u32x4 (&fa)[HALF], const u32x4 (&fb)[C::NT], Acc<C>& acc, int half) {
    if (PAIRED) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < HALF; ++i)
#pragma unroll
      for (int j = 0; j < C::NT; ++j) acc.v[half * HALF + i][j] = mma(fa[i], fb[j], acc.v[half * HALF + i][j], (const T*)nullptr);
    if (PAIRED) __builtin_amdgcn_s_setprio(0);
  }
  // the slice at k in `now`; the one DEPTH - 1 further on goes to `free`
  __device__ __forceinline__ void slice(int k, const lds_u8* __restrict now, lds_u8* __restrict free, Acc<C>& acc) const {
    u32x4 fa[HALF], fb[C::NT];
    read_b(fb, now, 0);
    read_a(fa, now, 0, 0);
    a.copy(A, m0, k + (C::DEPTH - 1) * BK, k1, free);
    turn();
    multiply(fa, fb, acc, 0);
    turn();
    read_a(fa, now, 1, 0);
    b.copy(B, n0, k + (C::DEPTH - 1) * BK, k1, free + OA::BYTES);
    turn();
    multiply(fa, fb, acc, 1);
    turn();
    read_b(fb, now, 1);
    read_a(fa, now, 0, 1);
    turn();
    multiply(fa, fb, acc, 0);
    turn();
    read_a(fa, now, 1, 1);
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LEFT) : "memory");
    barrier();
    multiply(fa, fb, acc, 1);
    turn();
  }
  __device__ __forceinline__ void run(int k0, const Buffers& lds, Acc<C>& acc) {
    a.init(A, m0);
    b.init(B, n0);
    lds_u8* const p[4] = {lds.p0, lds.p1, lds.p2, lds.p3};
#pragma unroll
    for (int i = 0; i < C::DEPTH - 1; ++i) {
      a.copy(A, m0, k0 + i * BK, k1, p[i]);
      b.copy(B, n0, k0 + i * BK, k1, p[i] + OA::BYTES);
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
    barrier();
    const bool second = PAIRED && uniform((int)threadIdx.x) >= 256;
    if (second) barrier();
    for (int k = k0;;) {
      slice(k, p[0], p[C::DEPTH - 1], acc);
      if ((k += BK) >= k1) break;
      slice(k, p[1], p[0], acc);
      if ((k += BK) >= k1) break;
      if (C::DEPTH > 2) {
        slice(k, p[2], p[1], acc);
        if ((k += BK) >= k1) break;
      }
      if (C::DEPTH > 3) {
        slice(k, p[3], p[2], acc);
        if ((k += BK) >= k1) break;
      }
    }
    if (PAIRED && !second) barrier();
    if (LEFT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // no copy outlives the workgroup's use of the buffers
  }
};

// acc = the tile at (m0, n0), contraction over [k0, k1)
template <class C, bool AKC, bool BKC>
__device__ __forceinline__ void product(const Src& A, const Src& B, int m0, int n0, int k0, int k1, const Buffers& lds, Acc<C>& acc) {
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < C::MT; ++i)
#pragma unroll
    for (int j = 0; j < C::NT; ++j) acc.v[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (k0 >= k1) return;
  Product<C, AKC, BKC> p{A, B, uniform(m0), uniform(n0), uniform(k1 < A.k ? (k1 < B.k ? k1 : B.k) : (A.k < B.k ? A.k : B.k)),
                         fragment_place<typename C::T, C::BM, AKC, AKC>((wave % C::WM) * 16 * C::MT),
                         fragment_place<typename C::T, C::BN, BKC>((wave / C::WM) * 16 * C::NT)};
  p.run(uniform(k0), lds, acc);
}

// Order of the tiles of a launch: workgroup i runs on XCD i mod 8, which gets a run of neighbouring tiles, eight along n for each
// along m, so that the tiles that an XCD works on at a time share operands in its L2.  The grid is for all rows, the tiles in use are
// those of the rows that count.
__device__ __forceinline__ void place_tile(int id, int mt, int nt, int& m, int& n) {
  const int total = mt * nt, x = id & 7, per = total >> 3, rest = total & 7;
  const int l = x * per + (x < rest ? x : rest) + (id >> 3);
  const int group = l / (8 * mt), first = group * 8, width = nt - first < 8 ? nt - first : 8, in = l - first * mt;
  n = first + in % width;
  m = in / width;
}

// element (i, j, e) of a wave's accumulators: m = 16 i + 4 (lane / 16) + e, n = 16 j + lane % 16
#define HEAD_LANE                                                                                      \
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4, wave = threadIdx.x >> 6;          \
  const int um = (wave % C::WM) * 16 * C::MT, un = (wave / C::WM) * 16 * C::NT;

template <class T>
__device__ __forceinline__ Src packed_x(const HeadDev& h, int n) {
  if (h.direct || whole(h, n)) return Src{reinterpret_cast<const char*>(h.x.p), h.x.stride * (int)sizeof(T), n, h.cols};
  return Src{h.ws + h.lay.x, (int64_t)h.pitch * (int)sizeof(T), n, h.pitch};
}
template <class T>
__device__ __forceinline__ Src vocab_rows(const HeadDev& h, int64_t first, int64_t rows) {     // rows of W from `first`, k along them
  if (h.w_packed) return Src{h.ws + h.lay.w + first * h.pitch * (int)sizeof(T), (int64_t)h.pitch * (int)sizeof(T), (int)rows, h.pitch};
  return Src{reinterpret_cast<const char*>(h.w.p) + first * h.w.stride * (int)sizeof(T), h.w.stride * (int)sizeof(T), (int)rows, h.cols};
}

// forward: m = vocabulary, n = rows of x
template <class C>
__global__ __launch_bounds__(C::THREADS, C::THREADS == 512 ? 2 : 1) void logits_kernel(HeadDev h, int mt) {
  typedef typename C::T T;
  HEAD_BUFFERS
  const int n = live_rows(h);
  const int nt = (n + C::BN - 1) / C::BN;
  if ((int)blockIdx.x >= mt * nt) return;
  int tm, tn;
  place_tile(blockIdx.x, mt, nt, tm, tn);
  const int m0 = tm * C::BM, n0 = tn * C::BN;
  Acc<C> acc;
  product<C, true, true>(vocab_rows<T>(h, 0, h.vocab), packed_x<T>(h, n), m0, n0, 0, h.cols, lds, acc);
  HEAD_LANE
  const int* target = reinterpret_cast<const int*>(h.ws + h.lay.target);
  float2* part = reinterpret_cast<float2*>(h.ws + h.lay.part) + (int64_t)(tm * C::WM + wave % C::WM) * h.rows;
  float* hit = reinterpret_cast<float*>(h.ws + h.lay.hit);
  const int v0 = m0 + um + 8 * q;       // element (i, j, e): vocabulary row v0 + pair_row(i, e)
  // columns behind the vocabulary's end, in its last tile
  if (m0 + C::BM > h.vocab) {
#pragma unroll
    for (int i = 0; i < C::MT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (v0 + pair_row(i, e) >= h.vocab) {
#pragma unroll
          for (int j = 0; j < C::NT; ++j) acc.v[i][j][e] = -INFINITY;
        }
  }
#pragma unroll
  for (int j = 0; j < C::NT; ++j) {
    const int row = n0 + un + 16 * j + l16;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < C::MT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) top = fmaxf(top, acc.v[i][j][e]);
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    // exp(s - top) = 2^(s L - c) 2^-rest with L = log2 e as fp32, c = top L rounded, rest = top L - c: one multiply-add an element, and what
    // the rounding of c has left out goes into the sum once.  The elements and the rest have the same L, so the top's element is 1 at any
    // size of the logits, and what L leaves out of log2 e (1.9e-8) meets s - top alone.  A wave without a column of the vocabulary leaves (-inf, 0).
    const float c = top == -INFINITY ? 0.f : top * LOG2E, rest = top == -INFINITY ? 0.f : fmaf(top, LOG2E, -c);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < C::MT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(fmaf(acc.v[i][j][e], LOG2E, -c));
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    sum *= __builtin_amdgcn_exp2f(-rest);
    if (row < n) {
      if (q == 0) part[row] = make_float2(top, sum);
      const int rel = (h.direct ? (counts(h, row) ? (int)h.targets[row] : -1) : target[row]) - v0;
      if (rel >= 0 && rel < 16 * C::MT && (rel & 31) < 8) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < C::MT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) s = rel == pair_row(i, e) ? acc.v[i][j][e] : s;
        hit[row] = s;
      }
    }
  }
}

// Joins the tiles' maxima and sums: RL rows a workgroup, whose 1024 / RL slices share the tiles; each row's loss, and the workgroup's
// sum of them.  RL = 8, 128 slices (one row over 32000 columns: 28.5 us with 16 of them, a chain of 63 loads) up to 2048 rows, which fill
// the chip with such workgroups; beyond, RL = 16, whose loads are whole lines (8192 rows over 32000 columns 11 us with RL = 64, 6.8 with 16).
template <int RL>
__global__ __launch_bounds__(1024) void finish_kernel(HeadDev h, int tiles, int last) {
  constexpr int SL = 1024 / RL;
  __shared__ float rm[SL][RL], rs[SL][RL];
  const int n = live_rows(h);
  const int l = threadIdx.x % RL, w = threadIdx.x / RL, row = blockIdx.x * RL + l;
  const float2* part = reinterpret_cast<const float2*>(h.ws + h.lay.part);
  double* sums = reinterpret_cast<double*>(h.ws + h.lay.sums);
  float m = -INFINITY, s = 0.f;
  if (row < n)
    for (int t0 = w; t0 < tiles; t0 += 4 * SL) {
      float2 p[4];                                     // requested together
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = t0 + i * SL < tiles ? part[(int64_t)(t0 + i * SL) * h.rows + row] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (p[i].y == 0.f) continue;                   // a tile behind the vocabulary's end
        const float top = fmaxf(m, p[i].x);
        s = (s == 0.f ? 0.f : s * __builtin_amdgcn_exp2f((m - top) * LOG2E)) + p[i].y * __builtin_amdgcn_exp2f((p[i].x - top) * LOG2E);
        m = top;
      }
    }
  rm[w][l] = m;
  rs[w][l] = s;
  __syncthreads();
#pragma unroll
  for (int o = SL / 2; o > 0; o >>= 1) {
    if (w < o) {
      const float m2 = rm[w + o][l], s2 = rs[w + o][l], top = fmaxf(m, m2);
      s = (s == 0.f ? 0.f : s * __builtin_amdgcn_exp2f((m - top) * LOG2E)) + (s2 == 0.f ? 0.f : s2 * __builtin_amdgcn_exp2f((m2 - top) * LOG2E));
      rm[w][l] = m = top;
      rs[w][l] = s;
    }
    __syncthreads();
  }
  if (threadIdx.x >= 64) return;
  double part_loss = 0.0;
  int counted = n;
  bool in = w == 0 && row < n;
  if (h.direct) {                                      // counted: of interest where this is the one workgroup
    const bool live = in && counts(h, row);
    if (in && !live) {
      h.lse[row] = 0.f;
      h.row_loss[row] = 0.f;
    }
    counted = __popcll(__ballot(live));
    in = live;
  }
  if (in) {
    // the difference of the logits first, which is exact where they are near: a small loss keeps its digits
    const float log_sum = logf(s), lse = m + log_sum, loss = (m - reinterpret_cast<const float*>(h.ws + h.lay.hit)[row]) + log_sum;
    const int to = h.direct ? row : reinterpret_cast<const int*>(h.ws + h.lay.list)[row];
    h.lse[to] = lse;
    h.row_loss[to] = loss;
    const float weight = !h.direct ? reinterpret_cast<const float*>(h.ws + h.lay.weight)[row] : h.row_weight ? h.row_weight[row] : 1.f;
    part_loss = (double)weight * (double)loss;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) part_loss += __shfl_xor(part_loss, o);
  if (threadIdx.x) return;
  if (last) *h.loss = (float)(part_loss * (double)h.scale / (h.mean ? (double)(counted > 0 ? counted : 1) : 1.0));
  else sums[blockIdx.x] = part_loss;
}

__global__ __launch_bounds__(256) void total_kernel(HeadDev h, int groups) {
  __shared__ double red[256];
  const double* sums = reinterpret_cast<const double*>(h.ws + h.lay.sums);
  double s = 0.0;
  for (int i = threadIdx.x; i < groups; i += 256) s += sums[i];
  static_assert(DIRECT_ROWS <= 256, "a thread each");
  const int n = h.direct ? __syncthreads_count((int64_t)threadIdx.x < h.rows && counts(h, threadIdx.x))
                         : reinterpret_cast<const HeadHeader*>(h.ws + h.lay.head)->n;
  red[threadIdx.x] = s;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) *h.loss = (float)(red[0] * (double)h.scale / (h.mean ? (double)(n > 0 ? n : 1) : 1.0));
}

// a batch without rows: loss 0, dW 0
__global__ __launch_bounds__(64) void no_rows_loss_kernel(HeadDev h) { *h.loss = 0.f; }

template <class T>
__global__ __launch_bounds__(256) void no_rows_dw_kernel(HeadDev h) {
  T* to = reinterpret_cast<T*>(h.dw.p) + (int64_t)blockIdx.x * h.dw.stride;
  for (int c = threadIdx.x; c < h.cols; c += 256) to[c] = T(0);
}

// backward: P of the vocabulary rows [first, first + width), m = vocabulary, n = rows of x; zeros up to the piece's pitch
template <class C>
__global__ __launch_bounds__(C::THREADS, C::THREADS == 512 ? 2 : 1) void piece_kernel(HeadDev h, int64_t first, int width, int64_t pitch, int mt) {
  typedef typename C::T T;
  HEAD_BUFFERS
  const int n = reinterpret_cast<const HeadHeader*>(h.ws + h.lay.head)->n;
  const int nt = (n + C::BN - 1) / C::BN;
  if ((int)blockIdx.x >= mt * nt) return;
  int tm, tn;
  place_tile(blockIdx.x, mt, nt, tm, tn);
  const int m0 = tm * C::BM, n0 = tn * C::BN;
  Acc<C> acc;
  product<C, true, true>(vocab_rows<T>(h, first, width), packed_x<T>(h, n), m0, n0, 0, h.cols, lds, acc);
  HEAD_LANE
  T* P = reinterpret_cast<T*>(h.ws + h.lay.p);
  const bool two = uniform(twin(h, n));
#pragma unroll
  for (int j = 0; j < C::NT; ++j) {
    const int row = n0 + un + 16 * j + l16;
    if (row >= n) continue;
    const int target = reinterpret_cast<const int*>(h.ws + h.lay.target)[row] - (int)first - (m0 + um + 8 * q);
    const float weight = reinterpret_cast<const float*>(h.ws + h.lay.weight)[row];
    const float lse = reinterpret_cast<const float*>(h.ws + h.lay.lse)[row], lse2 = lse * LOG2E;
    f32x4 p[C::MT];
#pragma unroll
    for (int i = 0; i < C::MT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        // fp32: the accurate exponential; bf16 rounds P to 8 bits (the matrix cores' operand), the hardware's is far inside that
        p[i][e] = sizeof(T) == 4 ? expf(acc.v[i][j][e] - lse) : __builtin_amdgcn_exp2f(fmaf(acc.v[i][j][e], LOG2E, -lse2));
    if (target >= 0 && target < 16 * C::MT) {        // few lanes ever
#pragma unroll
      for (int i = 0; i < C::MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) p[i][e] -= target == pair_row(i, e) ? 1.f : 0.f;
    }
    if (h.row_weight) {
#pragma unroll
      for (int i = 0; i < C::MT; ++i) p[i] *= weight;
    }
    if (m0 + C::BM > width) {                        // the piece's last tile: zeros up to its pitch
#pragma unroll
      for (int i = 0; i < C::MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) p[i][e] = m0 + um + 8 * q + pair_row(i, e) < width ? p[i][e] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < C::MT; i += 2) {
      const int v = m0 + um + 8 * q + pair_row(i, 0);         // eight neighbouring columns of P
      T* to = P + (int64_t)row * pitch + v;
      if (v < pitch) {
        if (sizeof(T) == 2) {
          u32x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(p[i + e / 2][2 * (e & 1)], p[i + e / 2][2 * (e & 1) + 1]);
          *reinterpret_cast<u32x4*>(to) = w;
          if (two) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              w[e] = pack_bf16x2(p[i + e / 2][2 * (e & 1)] - bf16lo(w[e]), p[i + e / 2][2 * (e & 1) + 1] - bf16hi(w[e]));
            *reinterpret_cast<u32x4*>(to + (int64_t)n * pitch) = w;
          }
        } else {
          *reinterpret_cast<f32x4*>(to) = p[i];
          *reinterpret_cast<f32x4*>(to + 4) = p[i + 1];
        }
      }
    }
  }
}

struct GradPlan {
  int64_t first;          // the piece: vocabulary rows [first, first + width), P's row pitch in elements
  int width;
  int64_t pitch;
  int mt;                 // tiles along the columns (both products)
  int splits, k_split;    // dx: parts of the contraction and their length
  int nt_w;               // dW: tiles along the vocabulary
  int begin;              // first piece: dx's sums are written, not added to
  int first_dw;           // workgroups [first_dw, first_dw + mt nt_w) make dW
};

// backward of a piece: dW (m = columns, n = vocabulary, k = rows of x) and dx (m = columns, n = rows of x, k = the piece's vocabulary)
template <class C>
__global__ __launch_bounds__(C::THREADS, C::THREADS == 512 ? 2 : 1) void grad_kernel(HeadDev h, GradPlan g) {
  typedef typename C::T T;
  HEAD_BUFFERS
  const int live = reinterpret_cast<const HeadHeader*>(h.ws + h.lay.head)->n, n = live << twin(h, live);      // rows of P and of packed x
  const char* P = h.ws + h.lay.p;
  const int64_t pp = g.pitch * (int64_t)sizeof(T);
  const int n_dw = g.mt * g.nt_w;
  HEAD_LANE
  Acc<C> acc;
  const int dw_id = (int)blockIdx.x - g.first_dw;
  if (dw_id >= 0 && dw_id < n_dw) {
    int tm, tn;
    place_tile(dw_id, g.mt, g.nt_w, tm, tn);
    const int m0 = tm * C::BM, n0 = tn * C::BN;
    const Src x = packed_x<T>(h, live);                // k across the rows
    product<C, false, false>(Src{x.p, x.pitch, x.k, n}, Src{P, pp, (int)g.pitch, n}, m0, n0, 0, n,
                             lds, acc);
    const float f = grad_factor(h, live);
#pragma unroll
    for (int j = 0; j < C::NT; ++j) {
      const int v = n0 + un + 16 * j + l16;
      if (v >= g.width) continue;
      T* to = reinterpret_cast<T*>(h.dw.p) + (g.first + v) * h.dw.stride;
#pragma unroll
      for (int i = 0; i < C::MT; ++i) {
        const int c = m0 + um + 16 * i + 4 * q;
        const f32x4 x = acc.v[i][j] * f;
        if (c + 4 <= h.cols) {
          if (sizeof(T) == 2) {
            u32x2 w;
            w[0] = pack_bf16x2(x[0], x[1]);
            w[1] = pack_bf16x2(x[2], x[3]);
            *reinterpret_cast<u32x2_e2*>(to + c) = w;
          } else {
            *reinterpret_cast<f32x4_e4*>(to + c) = x;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (c + e < h.cols) to[c + e] = sizeof(T) == 2 ? (T)pack_bf16x2(x[e], 0.f) : (T)x[e];
        }
      }
    }
    return;
  }
  const int nt = (n + C::BN - 1) / C::BN, per = g.mt * nt, id = dw_id < 0 ? (int)blockIdx.x : dw_id - n_dw;
  if (id >= per * g.splits) return;
  const int split = id / per;
  int tm, tn;
  place_tile(id - split * per, g.mt, nt, tm, tn);
  const int m0 = tm * C::BM, n0 = tn * C::BN;
  const int k0 = split * g.k_split, k1 = k0 + g.k_split < g.width ? k0 + g.k_split : g.width;
  Src W = vocab_rows<T>(h, g.first, g.width);          // k across the rows
  const int cols = W.k;
  W.u = cols;
  W.k = g.width;
  product<C, false, true>(W, Src{P, pp, n, (int)g.pitch}, m0, n0, k0, k1, lds, acc);
  float* sum = reinterpret_cast<float*>(h.ws + h.lay.acc) + (int64_t)split * h.lay.p_rows * h.pitch;
#pragma unroll
  for (int j = 0; j < C::NT; ++j) {
    const int row = n0 + un + 16 * j + l16;
    if (row >= n) continue;
#pragma unroll
    for (int i = 0; i < C::MT; ++i) {
      const int c = m0 + um + 16 * i + 4 * q;
      if (c < h.pitch) {
        f32x4* to = reinterpret_cast<f32x4*>(sum + (int64_t)row * h.pitch + c);
        *to = g.begin ? acc.v[i][j] : *to + acc.v[i][j];
      }
    }
  }
}

// dx of every row of x: the parts of its sum added in a fixed order, zeros where the row does not count.  SL slices of the threads share the
// parts: of few rows there are many (16 rows over 32000 x 2048: 4.5 us, 15.5 with one thread for four columns of all parts).
template <class T, int SL>
__global__ __launch_bounds__(256) void dx_kernel(HeadDev h, int splits) {
  constexpr int LANES = 256 / SL;
  __shared__ f32x4 red[SL > 1 ? SL : 1][SL > 1 ? LANES : 1];
  const int n = reinterpret_cast<const HeadHeader*>(h.ws + h.lay.head)->n;
  const int64_t row = blockIdx.x;
  const int j = reinterpret_cast<const int*>(h.ws + h.lay.place)[row];
  const float f = j < 0 ? 0.f : grad_factor(h, n);      // zeros times infinity are none
  const int l = threadIdx.x % LANES, w = threadIdx.x / LANES, c = ((int)blockIdx.y * LANES + l) * 4;
  const int64_t part = h.lay.p_rows * (int64_t)h.pitch;
  const float* sum = reinterpret_cast<const float*>(h.ws + h.lay.acc) + (j < 0 ? 0 : (int64_t)j * h.pitch) + c;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  if (j >= 0 && c < h.cols) {
#pragma unroll 4
    for (int s = w; s < splits; s += SL) x += *reinterpret_cast<const f32x4*>(sum + s * part);
    if (twin(h, n)) {
      sum += (int64_t)n * h.pitch;
#pragma unroll 4
      for (int s = w; s < splits; s += SL) x += *reinterpret_cast<const f32x4*>(sum + s * part);
    }
  }
  if (SL > 1) {
    red[w][l] = x;
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int s = 1; s < SL; ++s) x += red[s][l];
  }
  if (c >= h.cols) return;
  T* to = reinterpret_cast<T*>(h.dx.p) + row * h.dx.stride;
  x *= f;
  if (c + 4 <= h.cols) {
    if (sizeof(T) == 2) {
      u32x2 v;
      v[0] = pack_bf16x2(x[0], x[1]);
      v[1] = pack_bf16x2(x[2], x[3]);
      *reinterpret_cast<u32x2_e2*>(to + c) = v;
    } else {
      *reinterpret_cast<f32x4_e4*>(to + c) = x;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < h.cols) to[c + e] = sizeof(T) == 2 ? (T)pack_bf16x2(x[e], 0.f) : (T)x[e];
  }
}

// ---- plans ------------------------------------------------------------------------------------------------------------
// Tiles: vocabulary or columns x rows (dW: columns x vocabulary)
typedef Cfg<uint16_t, 8, 4, 2, 4> Big;        // 256 x 256, eight wavefronts
typedef Cfg<uint16_t, 2, 4, 4, 1> Small;      // 128 x 64, four
typedef Cfg<uint16_t, 2, 2, 4, 1, 4> Thin;    // 128 x 32, four; three slices on their way: W streams by
typedef Cfg<float, 4, 4, 2, 2> Big32;         // 128 x 128, four
typedef Cfg<float, 2, 2, 4, 1> Small32;       // 128 x 32, four

// A kind of tile: a compute unit runs per_cu workgroups of it and is through with a slice in `share` then; few of them take `lag` more
struct Shape {
  int kind, bm, bn, wm, threads, per_cu;
  double share, lag;
};
template <class C>
constexpr Shape shape(int kind, int per_cu, double share, double lag) {
  return Shape{kind, C::BM, C::BN, C::WM, C::THREADS, per_cu, share, lag};
}
constexpr int CUS = 256;
constexpr double TILE = 4.0;                  // a tile's beginning and end, in slices
constexpr Shape SHAPES[5] = {shape<Big>(0, 1, 1.57, 0.0), shape<Small>(1, 3, 0.285, 0.45), shape<Thin>(2, 2, 0.25, 0.2),
                             shape<Big32>(3, 2, 1.95, 0.0), shape<Small32>(4, 4, 0.58, 0.0)};
// Those for a type.  Thin is for the forward pass of rows that are one of its tiles, where reading W is all: one row over 32000 x 2048 27
// us, 29 with Small (W in the last-level cache); the products of the backward pass gain nothing from it.
int first_shape(bool bf16) { return bf16 ? 0 : 3; }
int end_shape(bool bf16, bool thin) { return !bf16 ? 5 : thin ? 3 : 2; }

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

}  // namespace
int head_twin_rows(bool bf16, bool weighted) { return !bf16 ? 0 : weighted ? TWIN_ROWS_WEIGHTED : TWIN_ROWS; }
namespace {

// How the backward pass is cut.
struct Cut {
  const Shape* shape;
  int64_t width;      // vocabulary rows of a piece
  int splits;         // parts of dx's contraction over them
  bool dx_first;      // dx's tiles are given out before dW's
  double us;          // what it should take
};

// Time that `slots` take for n1 tiles of length l1 and then n2 tiles of length l2, each taking the next one when it is done.
double finish_time(int64_t n1, double l1, int64_t n2, double l2, int64_t slots) {
  const int64_t full = n1 / slots, rest = n1 % slots;
  const double early = (double)full * l1, late = rest ? early + l1 : early;      // when the free and the busy slots are through with n1
  double end = late;
  if (n2 > 0) {
    // tiles done by the time t: (slots - rest) floor((t - early) / l2) + rest floor((t - late) / l2)
    const double even = ((double)n2 * l2 + (double)(slots - rest) * early + (double)rest * late) / (double)slots;
    for (double t = even > early + l2 ? even : early + l2;; t += 0.25 * l2) {
      const double done = (double)(slots - rest) * std::floor((t - early) / l2 + 1e-9) + (t > late ? (double)rest * std::floor((t - late) / l2 + 1e-9) : 0.0);
      if (done >= (double)n2) {
        end = end > t ? end : t;
        break;
      }
    }
  }
  return end;
}

// The tiles of a piece's gradients are few and unequal: those of dW have the rows of x for their contraction, those of dx the piece's
// vocabulary, which can be cut, at the price of one more fp32 sum of dx to write and read.  Pieces of equal width, the parts of dx and
// which tiles come first are chosen by the time that follows from the tiles, for all rows and for two thirds of them: how many count is
// known on the device alone.  Backward of 8192 rows over 32000 x 512 in 2, 3, 4, 5 pieces 790, 919, 1001, 1164 us (tiles of dW that leave half of
// the chip idle), with two thirds of the rows 584, 600, 706, 786; over 32000 x 2048 2666, 2889, 2560, 2805 and 1900, 1920, 1903, 2111; over
// 50257 x 1600 in 4, 5, 6, 8 pieces 3841, 3440, 3711, 3984 and 2628, 2594, 2666, 2633.
Cut cut_with(int64_t rows, int64_t vocab, int64_t cols, bool bf16, int twin, const Shape& f) {
  const int64_t es = bf16 ? 2 : 4, bk = 128 / es, slots = CUS * f.per_cu;
  const double us_per_byte = 1.0 / 4e6;
  int64_t fewest = ((rows << twin) * vocab * es + PIECE_BYTES - 1) / PIECE_BYTES;
  const int64_t most = (vocab + 2047) / 2048;                         // pieces of at least 2048
  if (fewest > most) fewest = most;
  const int64_t mt = (cols + f.bm - 1) / f.bm, kd = (cols + bk - 1) / bk;
  Cut best{&f, 0, 1, false, 0.0};
  for (int64_t p = fewest; p <= most && p <= 2 * fewest + 3; p += (fewest + 7) / 8) {
    const int64_t width = up((vocab + p - 1) / p, 256), pieces = (vocab + width - 1) / width;
    const int64_t mp = (width + f.bm - 1) / f.bm, tw = mt * ((width + f.bn - 1) / f.bn), kv = width / bk;
    static const int parts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128};
    for (int sp : parts) {
      if (sp > 1 && sp * 256 > width) break;
      const double lx = (double)((kv + sp - 1) / sp) + TILE;
      for (int dx_first = 0; dx_first < 2; ++dx_first) {
        double t = 0.0;
        for (int64_t n = rows; n >= rows * 2 / 3 && n > 0; n = n == rows && rows > 2 ? rows * 2 / 3 : 0) {
          const int64_t nt = (n + f.bn - 1) / f.bn, n2 = n << twin, tx = mt * ((n2 + f.bn - 1) / f.bn) * sp;
          const double lw = (double)((n2 + bk - 1) / bk) + TILE;
          t += (finish_time(mp * nt, (double)kd + TILE, 0, 1.0, slots) +
                (dx_first ? finish_time(tx, lx, tw, lw, slots) : finish_time(tw, lw, tx, lx, slots))) * f.share * f.per_cu +
               8.0 * (double)n2 * (double)cols * sp * us_per_byte;
        }
        t *= (double)pieces;
        if (best.width == 0 || t < best.us) best = Cut{&f, width, sp, dx_first != 0, t};
      }
    }
  }
  return best;
}

// Which tiles the passes take: those with the shorter time.  bf16 over 50257 x 1600, small and big tiles, us forward / backward: 64 rows 37 /
// 131 and 48 / 166, 128 rows 56 / 170 and 49 / 174, 256 rows 76 / 243 and 49 / 199, 1024 rows 223 / 702 and 169 / 549; over 4099 x 256,
// where big tiles are few, 1024 rows 24 / 38 and 26 / 58.
const Shape& forward_shape(int64_t rows, int64_t vocab, int64_t cols, bool bf16) {
  int best = 0;
  double least = 0.0;
  const int from = first_shape(bf16), end = end_shape(bf16, rows <= Thin::BN);
  for (int i = from; i < end; ++i) {
    const Shape& f = SHAPES[i];
    const int64_t tiles = ((vocab + f.bm - 1) / f.bm) * ((rows + f.bn - 1) / f.bn), bk = bf16 ? 64 : 32;
    const double slices = (double)((cols + bk - 1) / bk) + TILE, us = finish_time(tiles, slices, 0, 1.0, CUS) * f.share + slices * f.lag;
    if (i == from || us < least) {
      best = i;
      least = us;
    }
  }
  return SHAPES[best];
}

// The cut depends on the sizes alone (not on which gradients are wanted: the workspace is asked for without knowing) and takes 12 to 25
// microseconds of the host to find: a thread keeps the last ones, one with P as one number and one with two.  A call of the sizes of the call
// before asks for its workspace in 1.5 us; batches whose row counts alternate pay for it every time, up to 1024 rows for both (8192 rows over
// 32000 x 512 14 us, 1000 rows over 50257 x 1600 37).
Cut cut_of(int64_t rows, int64_t vocab, int64_t cols, bool bf16, int twin) {
  struct Last {
    int64_t rows, vocab, cols;
    bool bf16;
    Cut cut;
  };
  static thread_local Last kept[2] = {{-1, 0, 0, false, Cut{nullptr, 0, 1, false, 0.0}}, {-1, 0, 0, false, Cut{nullptr, 0, 1, false, 0.0}}};
  Last& last = kept[twin];
  if (last.rows != rows || last.vocab != vocab || last.cols != cols || last.bf16 != bf16) {
    const int from = first_shape(bf16), end = end_shape(bf16, false);
    Cut best = cut_with(rows, vocab, cols, bf16, twin, SHAPES[from]);
    for (int i = from + 1; i < end; ++i) {
      const Cut c = cut_with(rows, vocab, cols, bf16, twin, SHAPES[i]);
      if (c.us < best.us) best = c;
    }
    last = Last{rows, vocab, cols, bf16, best};
  }
  return last.cut;
}

template <class C>
void logits(const HeadDev& h, hipStream_t s) {
  const int mt = (int)((h.vocab + C::BM - 1) / C::BM), nt = (int)((h.rows + C::BN - 1) / C::BN);
  hipLaunchKernelGGL((logits_kernel<C>), dim3((unsigned)(mt * nt)), dim3(C::THREADS), 0, s, h, mt);
}

template <class C>
void gradients(const HeadDev& h, int64_t width, int splits, hipStream_t s) {
  for (int64_t first = 0; first < h.vocab; first += width) {
    GradPlan g;
    g.first = first;
    g.width = (int)(h.vocab - first < width ? h.vocab - first : width);
    g.pitch = width;
    const int mp = (int)((up(g.width, 64) + C::BM - 1) / C::BM), np = (int)((h.rows + C::BN - 1) / C::BN);
    const int nx = (int)((h.lay.p_rows + C::BN - 1) / C::BN);
    hipLaunchKernelGGL((piece_kernel<C>), dim3((unsigned)(mp * np)), dim3(C::THREADS), 0, s, h, first, g.width, width, mp);
    g.mt = (h.cols + C::BM - 1) / C::BM;
    g.splits = h.dx.p ? splits : 0;
    g.k_split = (int)up((g.width + splits - 1) / splits, 64);
    g.nt_w = h.dw.p ? (g.width + C::BN - 1) / C::BN : 0;
    g.begin = first == 0;
    g.first_dw = h.lay.dx_first && h.dx.p ? g.mt * nx * g.splits : 0;
    hipLaunchKernelGGL((grad_kernel<C>), dim3((unsigned)(g.mt * (g.nt_w + nx * g.splits))), dim3(C::THREADS), 0, s, h, g);
  }
}

template <class T>
void joined(const HeadDev& h, int splits, hipStream_t s) {
  if (splits < 8) hipLaunchKernelGGL((dx_kernel<T, 1>), dim3((unsigned)h.rows, (unsigned)((h.cols + 1023) / 1024)), dim3(256), 0, s, h, splits);
  else hipLaunchKernelGGL((dx_kernel<T, 8>), dim3((unsigned)h.rows, (unsigned)((h.cols + 127) / 128)), dim3(256), 0, s, h, splits);
}

void pack_x(const HeadDev& h, hipStream_t s) {
  if (h.rows > COUNT_ROWS)
    hipLaunchKernelGGL(count_kernel, dim3((unsigned)((h.rows + COUNT_ROWS - 1) / COUNT_ROWS)), dim3(256), 0, s, h);
  const int64_t sets = (h.rows + PACK_ROWS - 1) / PACK_ROWS, turns = (PACK_ROWS * (int64_t)h.pitch * (h.bf16 ? 2 : 4) / 16 + 255) / 256;
  const dim3 grid((unsigned)sets, (unsigned)(sets * turns <= PACK_GROUPS ? turns : sets < PACK_GROUPS ? PACK_GROUPS / sets : 1));
  if (h.bf16) hipLaunchKernelGGL((pack_kernel<uint16_t>), grid, dim3(256), 0, s, h);
  else hipLaunchKernelGGL((pack_kernel<float>), grid, dim3(256), 0, s, h);
}
void pack(const HeadDev& h, hipStream_t s) {
  if (!h.direct) pack_x(h, s);
  if (h.w_packed) {
    const dim3 wgrid((unsigned)((h.vocab + PACK_ROWS - 1) / PACK_ROWS));
    if (h.bf16) hipLaunchKernelGGL((pack_w_kernel<uint16_t>), wgrid, dim3(256), 0, s, h);
    else hipLaunchKernelGGL((pack_w_kernel<float>), wgrid, dim3(256), 0, s, h);
  }
}
}  // namespace

bool head_direct(int64_t rows) { return rows <= DIRECT_ROWS; }
bool head_whole(int64_t rows) { return rows > COUNT_ROWS; }

HeadLayout head_layout(int64_t rows, int64_t vocab, int64_t cols, bool bf16, bool w_packed, bool backward, bool want_dx, int twin_rows) {
  // up to twin_rows of them twice, or all of them once
  const int64_t es = bf16 ? 2 : 4, pitch = up(cols, bf16 ? 64 : 32), twice = 2 * (rows < twin_rows ? rows : twin_rows), rows2 = rows > twice ? rows : twice;
  HeadLayout l;
  l.p_rows = rows2;
  l.width = 0;
  l.splits = 0;
  l.dx_first = false;
  l.kind = 0;
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t o = at;
    at += up(bytes, 256);
    return o;
  };
  l.head = take(sizeof(HeadHeader));
  l.counts = take(4 * ((rows + COUNT_ROWS - 1) / COUNT_ROWS));
  l.list = take(4 * rows);
  l.place = take(4 * rows);
  l.target = take(4 * rows);
  l.weight = take(4 * rows);
  l.lse = take(4 * rows);
  l.x = take(rows2 * pitch * es);
  l.w = w_packed ? take(vocab * pitch * es) : -1;
  l.part = l.hit = l.sums = l.p = l.acc = -1;
  if (!backward) {
    const Shape& f = forward_shape(rows > 0 ? rows : 1, vocab, cols, bf16);
    l.kind = f.kind;
    l.tiles = (int)((vocab + f.bm - 1) / f.bm) * f.wm;
    l.threads = (vocab + f.bm - 1) / f.bm * ((rows + f.bn - 1) / f.bn) * f.threads;
    l.part = take(8 * rows * l.tiles);
    l.hit = take(4 * rows);
    l.sums = take(8 * ((rows + 7) / 8));
  } else {
    const Cut c = cut_of(rows > 0 ? rows : 1, vocab, cols, bf16, rows > 0 && rows <= twin_rows ? 1 : 0);
    l.kind = c.shape->kind;
    l.width = c.width;
    l.splits = c.splits;
    l.dx_first = c.dx_first;
    const Shape& f = *c.shape;
    const int64_t logits = (c.width + f.bm - 1) / f.bm * ((rows + f.bn - 1) / f.bn);
    const int64_t grads = (cols + f.bm - 1) / f.bm * ((c.width + f.bn - 1) / f.bn + (rows2 + f.bn - 1) / f.bn * c.splits);
    l.threads = (logits > grads ? logits : grads) * f.threads;
    l.p = take(rows2 * c.width * es);
    if (want_dx) l.acc = take(4 * rows2 * pitch * c.splits);
  }
  l.bytes = at;
  return l;
}

void launch_head_loss(const HeadDev& h, hipStream_t s) {
  if (h.rows == 0) {
    hipLaunchKernelGGL(no_rows_loss_kernel, dim3(1), dim3(1), 0, s, h);
    return;
  }
  pack(h, s);
  switch (h.lay.kind) {
    case 0: logits<Big>(h, s); break;
    case 1: logits<Small>(h, s); break;
    case 2: logits<Thin>(h, s); break;
    case 3: logits<Big32>(h, s); break;
    default: logits<Small32>(h, s); break;
  }
  const int tiles = h.lay.tiles, rl = h.rows <= 8 ? 8 : h.direct && h.rows <= JOINED_ROWS ? (h.rows <= 16 ? 16 : JOINED_ROWS) : h.rows <= 2048 ? 8 : 16, groups = (int)((h.rows + rl - 1) / rl);
  const dim3 grid((unsigned)groups), block(1024);
  const int last = groups == 1 ? 1 : 0;
  if (rl == 8) hipLaunchKernelGGL((finish_kernel<8>), grid, block, 0, s, h, tiles, last);
  else if (rl == 16) hipLaunchKernelGGL((finish_kernel<16>), grid, block, 0, s, h, tiles, last);
  else hipLaunchKernelGGL((finish_kernel<JOINED_ROWS>), grid, block, 0, s, h, tiles, last);
  if (!last) hipLaunchKernelGGL(total_kernel, dim3(1), dim3(256), 0, s, h, groups);
}

void launch_head_backward(const HeadDev& h, hipStream_t s) {
  if (h.rows == 0) {
    if (!h.dw.p) return;
    if (h.bf16) hipLaunchKernelGGL((no_rows_dw_kernel<uint16_t>), dim3((unsigned)h.vocab), dim3(256), 0, s, h);
    else hipLaunchKernelGGL((no_rows_dw_kernel<float>), dim3((unsigned)h.vocab), dim3(256), 0, s, h);
    return;
  }
  pack(h, s);
  const int64_t width = h.lay.width;
  const int splits = h.lay.splits;
  switch (h.lay.kind) {
    case 0: gradients<Big>(h, width, splits, s); break;
    case 1: gradients<Small>(h, width, splits, s); break;
    case 3: gradients<Big32>(h, width, splits, s); break;
    default: gradients<Small32>(h, width, splits, s); break;
  }
  if (h.dx.p) {
    if (h.bf16) joined<uint16_t>(h, splits, s);
    else joined<float>(h, splits, s);
  }
}

}  // namespace adapm
