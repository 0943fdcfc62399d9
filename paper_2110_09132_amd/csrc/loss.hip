// Softmax cross entropy over the whole vocabulary of a table, forward and backward.
//
//   z[t][v] = x_t . W_v;  lse_t = log sum_v exp z[t][v]
//   loss_t  = lse_t - (1 - e) z[t][target_t] - e sum_v z[t][v] / V
//   g[t][v] = dloss_t (exp(z[t][v] - lse_t) - (1 - e) [v == target_t] - e / V)
//   dx = g W,  dW = g^T x
//
// The logits are never in memory as a whole.  Forward, a workgroup keeps the
// running maximum and sum of its tokens over a run of the vocabulary and the
// runs are joined at the end; backward, g exists for one piece of the
// vocabulary at a time.  Tokens without a target are taken out first, so they
// cost nothing and what stands in their rows reaches no sum.
//
// All products are C[m][n] = sum_k A[m][k] B[n][k] on the bf16 matrix
// instructions, with operands whose rows are contiguous along k, padded with
// zeros to whole tiles.  An fp32 value is the sum of three bf16 values of 8
// significant bits each, without a remainder (the leading bits are cut off, not
// rounded); of the nine products of two such sums the six largest are added up
// (the others are below 2^-24 of the product of the magnitudes).  Measured for
// the alternative, the fp32 matrix instructions: they run at a sixteenth of the
// bf16 rate, the six products at a sixth.
#include <algorithm>
#include <type_traits>

#include "vec.h"
#include "launch.h"

namespace emb {
namespace {

typedef __bf16 frag __attribute__((ext_vector_type(8)));     // 8 values along k of one row
typedef float acc16 __attribute__((ext_vector_type(16)));    // a lane's part of a 32 x 32 tile

constexpr int kTile = 256;     // rows of A per workgroup, and of B but for narrow tiles
constexpr int kStep = 64;      // values along k per step
constexpr int kThreads = 512;  // 8 / kWN waves along m, kWN along n: 32 kWN x 64 each, 4 of 128 x 64 unless said
constexpr int kWide = 4;       // kWN of tiles of 256 x 256; 2: 256 x 128, 1: 256 x 64
constexpr int kMT = 4, kNT = 2;  // 32 x 32 tiles of a wave along m (kWN of them) and n
constexpr int kGrid = 256;     // one workgroup per CU
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLowest = -3.402823466e38f;

// What the first kernel of a call leaves for the others.
struct Plan {
  int live;    // tokens with a target
  int tiles;   // of kTile live tokens
  int splits;  // forward: runs of the vocabulary;  backward: runs of k in dx
  int table_splits;  // backward: runs of k in dW
};

__host__ __device__ constexpr int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
// Tiles of n entries, n < 2^31 (a table that is read where it stands is one piece).
__device__ __forceinline__ int tiles_of(int n) { return static_cast<int>((static_cast<uint32_t>(n) + kTile - 1) / kTile); }

// The products of the planes, the smallest first.
template <int kPlanes>
__device__ __forceinline__ void plane_pair(int i, int& a, int& b) {
  if constexpr (kPlanes == 1) {
    a = b = 0;
  } else {
    constexpr uint32_t kA = 0x001102, kB = 0x010120;  // nibbles from the lowest: (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
    a = (kA >> (4 * i)) & 15;
    b = (kB >> (4 * i)) & 15;
  }
}
template <int kPlanes>
constexpr int kPairs = kPlanes == 1 ? 1 : 6;

// An operand: plane p's row r starts at p + plane * stride + r * ld (elements).
struct Operand {
  const uint16_t* p;
  int64_t plane;
  int64_t ld;
  int rows;  // rows that may be read
};

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)(p)));
}

__device__ __forceinline__ uint64_t uniform64(const void* p) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = static_cast<uint32_t>(uniform(static_cast<int>(a))), hi = static_cast<uint32_t>(uniform(static_cast<int>(a >> 32)));
  return static_cast<uint64_t>(hi) << 32 | lo;
}
// 16 bytes per lane from memory into LDS at `lds` + 16 lane, past the registers.
// The instruction is written out since the compiler, which does not follow what
// it writes, would wait for all of them before every read of LDS; the waits are
// in Product::meet.  It takes `lds` from m0, one wait state after m0 is written.
__device__ __forceinline__ void copy_to_lds(uint32_t lds, uint32_t offset, uint64_t base) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "{m0}"(lds) : "memory");
}

// LDS of two steps: of each the tile of A, then that of B.  A row of 64 values has
// 8 chunks of 16 bytes; chunk c of row r stands at place c ^ (r >> 1 & 7), so that
// the 16 lanes that one cycle of a read serves (16 rows, one chunk each) are in
// all 64 banks.
constexpr int kTileBytes = kTile * kStep * 2;
struct __attribute__((aligned(1024))) Buffers {
  char b[2][2][kTileBytes];
};

// A tile of the result and its range of k (multiples of kStep).
struct Span {
  int m0, n0, k0, k1;
};

// acc += A's rows m0 .. times B's rows n0 .. over k0 .. k1 of every pair of planes.
//
// start() issues the copies of a tile's first two steps, which may be while the tile before it is still being dealt with;
// run() does the products.  One barrier per step: before it every wave has read the whole of the step and its copies of
// the next one have landed; after it the step's buffer takes the copies of the step after that.  The reads of LDS run 16
// values of k ahead of the products, and behind the first products of the values before, whose wait then costs nothing.
// Measured, 16384 x 1024 times 1024 x 16384: 2.0 us a step with reads before each product, 1.8 us so, where the products
// alone would take 1.3 us and the copies alone 1.4 us (64 KB a step and CU; a ring of four steps of 32 values, copies
// spread between the products, prefetches into the L2 and operands tiled in memory changed nothing or made it worse).
//
// kTurned: A stands the other way round, row k has the values of all m.  Its tile then has kStep rows of kTile values, in
// blocks of 32 (64 bytes), of which row k's block b stands at place b ^ (k & 3 | (k >> 3 & 1) << 2), and is read with the
// instruction that hands 16 lanes the columns of a square of 4 x 16: lane l gives the address of 4 values of row
// (l % 16) / 4 and gets the 4 values of column l % 16.  The 64 lanes of a read are in 8 rows, whose blocks the places
// spread over all banks.
typedef __bf16 quad __attribute__((ext_vector_type(4)));
template <int kPlanes, bool kTurned, int kWN = kWide>
class Product {
  static constexpr int kMT = kWN;
  typedef acc16 Acc[kMT][kNT];

 public:
  __device__ __forceinline__ Product(const Operand& a, const Operand& b, Buffers& buffers) : A(a), B(b), lds(buffers) {
    lane = static_cast<int>(threadIdx.x) % kWave;
    wave = uniform(static_cast<int>(threadIdx.x) / kWave);
    base = uniform(lds_address(&buffers) + wave * 4096);
  }
  __device__ __forceinline__ void start(const Span& s) {
    span = s;
    kn = (s.k1 - s.k0) / kStep;
    steps = kn * kPairs<kPlanes>;
    // this lane's place in each of the wave's four copies of 8 rows (turned: of 2)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = wave * 32 + j * 8 + lane / 8, c = (lane % 8) ^ (row >> 1 & 7);
      if constexpr (kTurned) {
        const int k = wave * 8 + j * 2 + lane / 32, f = (k & 3) | (k >> 3 & 1) << 2;
        offA[j] = static_cast<uint32_t>(k * A.ld * 2 + ((lane % 32 / 4 ^ f) * 4 + lane % 4) * 16);
      } else {
        offA[j] = static_cast<uint32_t>(min(row, A.rows - 1 - s.m0) * A.ld * 2 + c * 16);
      }
      if (j < kWN) {
        const int n = wave * 8 * kWN + j * 8 + lane / 8;
        offB[j] = static_cast<uint32_t>(min(n, B.rows - 1 - s.n0) * B.ld * 2 + ((lane % 8) ^ (n >> 1 & 7)) * 16);
      }
    }
    if (steps > 0) copy(0);
    if (steps > 1) copy(1);
  }
  __device__ __forceinline__ void run(Acc& acc) {
    if (steps <= 0) return;
    meet();
    Frags f0, f1;
    read(0, 0, f0);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): so that the loop's waits need to count its own reads only
    for (int s = 0; s < steps; ++s) {
      multiply<0, 1>(f0, acc);
      read(s, 1, f1);
      multiply<1, kMT>(f0, acc);
      multiply<0, 1>(f1, acc);
      read(s, 2, f0);
      multiply<1, kMT>(f1, acc);
      multiply<0, 1>(f0, acc);
      read(s, 3, f1);
      multiply<1, kMT>(f0, acc);
      meet();
      if (s + 2 < steps) copy(s + 2);
      multiply<0, 1>(f1, acc);
      read(s + 1, 0, f0);  // (behind the last step: read and not used)
      multiply<1, kMT>(f1, acc);
    }
  }

 private:
  struct Frags {
    frag a[kMT], b[kNT];
  };
  __device__ __forceinline__ void copy(int s) {
    int pa, pb;
    const int pair = kPlanes == 1 ? 0 : s / kn;
    plane_pair<kPlanes>(pair, pa, pb);
    const int64_t k = span.k0 + (s - pair * kn) * kStep;
    const uint64_t a = uniform64(A.p + pa * A.plane + (kTurned ? k * A.ld + span.m0 : span.m0 * A.ld + k));
    const uint64_t b = uniform64(B.p + pb * B.plane + span.n0 * B.ld + k);
    const uint32_t to = uniform(base + (s & 1) * 2 * kTileBytes), to_b = uniform(to + kTileBytes - wave * (4 - kWN) * 1024);
#pragma unroll
    for (int j = 0; j < 4; ++j) copy_to_lds(to + j * 1024, offA[j], a);
#pragma unroll
    for (int j = 0; j < kWN; ++j) copy_to_lds(to_b + j * 1024, offB[j], b);
  }
  __device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }
  // Values 16 kk .. of step s.
  __device__ __forceinline__ void read(int s, int kk, Frags& f) {
    const int wm = wave / kWN, wn = wave % kWN, row = lane % 32, half = lane / 32;
    const char* at = lds.b[s & 1][0];
    const int place = ((kk * 2 + half) ^ (row >> 1 & 7)) * 16;
#pragma unroll
    for (int i = 0; i < kNT; ++i)
      f.b[i] = *reinterpret_cast<const frag*>(at + kTileBytes + (wn * 64 + row + 32 * i) * 128 + place);
#pragma unroll
    for (int i = 0; i < kMT; ++i) {
      if constexpr (kTurned) {
        const char* q = at + (16 * kk + 8 * half + lane % 16 / 4) * 512 + lane / 16 % 2 * 32 + lane % 4 * 8 +
                        ((wm * kMT + i) ^ (lane % 16 / 4 | half << 2)) * 64;
        typedef __attribute__((address_space(3))) quad* place_of;
        const quad lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((place_of)q);
        const quad hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((place_of)(q + 4 * 512));
        f.a[i] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      } else {
        f.a[i] = *reinterpret_cast<const frag*>(at + (wm * 32 * kMT + row + 32 * i) * 128 + place);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  template <int kFrom, int kTo>
  __device__ __forceinline__ void multiply(const Frags& f, Acc& acc) {
#pragma unroll
    for (int i = kFrom; i < kTo; ++i)
#pragma unroll
      for (int j = 0; j < kNT; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.a[i], f.b[j], acc[i][j], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }

  const Operand A, B;
  Buffers& lds;
  Span span;
  int lane, wave, kn, steps = 0;
  uint32_t base, offA[4], offB[kWN];
};

// Element e of a lane's part of a 32 x 32 tile: column lane % 32, this row.
__device__ __forceinline__ int tile_row(int e, int half) { return 8 * (e / 4) + 4 * half + e % 4; }

// Calls f(i, e, p) for the rows of a lane's part of a wave's tile in order, p at the row's start: base for row 0, ld
// elements from one to the next.  The address is hidden from the compiler every 4 rows: it would form all 64 at once,
// and spill.
template <int kMT, typename T, typename F>
__device__ __forceinline__ void each_row(T* base, int64_t ld, F&& f) {
  T* p = base;
#pragma unroll
  for (int i = 0; i < kMT; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int e = 0; e < 4; ++e) f(i, 4 * q + e, p + e * ld);
      p += 8 * ld;
      asm volatile("" : "+v"(p));
    }
}

template <int kMT>
__device__ __forceinline__ void clear(acc16 (&acc)[kMT][kNT]) {
#pragma unroll
  for (int i = 0; i < kMT; ++i)
#pragma unroll
    for (int j = 0; j < kNT; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
}

// x = p[0] + p[1] + p[2] exactly (but for what is below the smallest bf16), each the leading 8 bits of what is left.
template <int kPlanes>
__device__ __forceinline__ void split(float x, uint32_t (&p)[kPlanes]) {
  if constexpr (kPlanes == 1) {
    p[0] = bf16_pair(x, x) & 0xFFFFu;
  } else {
#pragma unroll
    for (int i = 0; i < kPlanes; ++i) {
      const uint32_t top = __float_as_uint(x) & 0xFFFF0000u;
      p[i] = top >> 16;
      x -= __uint_as_float(top);
    }
  }
}
// Eight values' planes as 16-byte words.
template <int kPlanes>
__device__ __forceinline__ void split8(const float (&v)[8], uint4 (&out)[kPlanes]) {
  uint32_t p[8][kPlanes];
#pragma unroll
  for (int e = 0; e < 8; ++e) split<kPlanes>(v[e], p[e]);
#pragma unroll
  for (int i = 0; i < kPlanes; ++i)
    out[i] = make_uint4(p[0][i] | p[1][i] << 16, p[2][i] | p[3][i] << 16, p[4][i] | p[5][i] << 16,
                        p[6][i] | p[7][i] << 16);
}

// d = mantissa(d) power(d), a power of two and a number in [1, 2) but for its sign (0, subnormal numbers, infinities and NaN:
// d itself and 1).  A token's factor goes into its g before g is rounded as a mantissa, and into its row of x, exactly, as a
// power.
__device__ __forceinline__ bool plain(float d) {
  const uint32_t e = __float_as_uint(d) >> 23 & 255;
  return e != 0 && e != 255;
}
__device__ __forceinline__ float mantissa(float d) {
  return plain(d) ? __uint_as_float((__float_as_uint(d) & 0x807FFFFFu) | 0x3F800000u) : d;
}
__device__ __forceinline__ float power(float d) {
  return plain(d) ? __uint_as_float(__float_as_uint(d) & 0x7F800000u) : 1.0f;
}

// The workgroups of one XCD (every eighth) take neighbouring units.
__device__ __forceinline__ int first_unit() {
  static_assert(kGrid % 8 == 0, "the same number of workgroups on every XCD");
  return static_cast<int>(blockIdx.x) % 8 * (kGrid / 8) + static_cast<int>(blockIdx.x) / 8;
}

// ---------------------------------------------------------------- the tokens that have a target
// One workgroup: the tokens with a target in order (list[slot] = t, slot_of[t] =
// slot, or -1), and the plan: the numbers of runs that take the fewest rounds of
// kGrid workgroups times steps per run, of the vocabulary (forward: nv > 0, its
// tiles), or of k in the two products (backward: nk steps of the piece's entries,
// nd tiles of columns, table_tiles tiles of dW in a piece).
constexpr int kPickThreads = 1024;
constexpr int kPickItems = 8;
__global__ __launch_bounds__(kPickThreads) void pick_kernel(const int32_t* __restrict__ targets, int64_t T, int64_t V,
                                                            int nv, int nk, int nd, int table_tiles, int most, int32_t* __restrict__ list,
                                                            int32_t* __restrict__ slot_of, Plan* plan,
                                                            int32_t* status) {
  __shared__ uint32_t wsum[kPickThreads / kWave];
  const int tid = static_cast<int>(threadIdx.x);
  uint32_t base = 0;
  bool bad = false;
  for (int64_t t0 = 0; t0 < T; t0 += kPickThreads * kPickItems) {
    const int64_t t = t0 + tid * kPickItems;
    int32_t id[kPickItems];
    uint32_t mine = 0;
#pragma unroll
    for (int e = 0; e < kPickItems; ++e) {
      id[e] = t + e < T ? targets[t + e] : -1;
      bad |= id[e] >= V;
      if (id[e] >= V) id[e] = -1;
      mine += id[e] >= 0;
    }
    const uint32_t upto = wave_inclusive_scan(mine);
    if (lane_id() == kWave - 1) wsum[tid / kWave] = upto;
    __syncthreads();
    uint32_t at = base + upto - mine;
#pragma unroll
    for (int w = 0; w < kPickThreads / kWave; ++w) {
      at += w < tid / kWave ? wsum[w] : 0u;
      base += wsum[w];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kPickItems; ++e) {
      if (t + e < T) slot_of[t + e] = id[e] >= 0 ? static_cast<int32_t>(at) : -1;
      if (id[e] >= 0) list[at++] = static_cast<int32_t>(t + e);
    }
  }
  if (__any(bad) && lane_id() == 0) raise_flag(status, EMB_DEV_ID_OUT_OF_RANGE);
  if (tid >= kWave) return;
  // every lane weighs some numbers of runs; the cheapest wins, of equals the smallest
  const auto choose = [&](int units, int work) {
    const int top = min(work, max(1, most / max(1, units)));
    uint64_t best = (1ull << 48) - 65536 + 1;
    for (int s = 1 + tid; s <= top; s += kWave) {
      const uint64_t rounds = (static_cast<uint64_t>(units) * s + kGrid - 1) / kGrid;
      best = min(best, rounds * ((work + s - 1) / s) << 16 | static_cast<uint64_t>(s));
    }
#pragma unroll
    for (int m = 1; m < kWave; m *= 2) {
      const uint32_t lo = __shfl_xor(static_cast<uint32_t>(best), m), hi = __shfl_xor(static_cast<uint32_t>(best >> 32), m);
      best = min(best, static_cast<uint64_t>(hi) << 32 | lo);
    }
    return static_cast<int>(best & 0xFFFF);
  };
  const int tiles = static_cast<int>((base + kTile - 1) / kTile);
  const int splits = nv > 0 ? choose(tiles, nv) : choose(tiles * nd, nk);
  const int table_splits = nv > 0 ? 1 : choose(table_tiles, static_cast<int>((base + kStep - 1) / kStep));
  if (tid == 0) *plan = Plan{static_cast<int>(base), tiles, splits, table_splits};
}

// ---------------------------------------------------------------- operands laid out for the products
// Rows of src (row r, or row list[r]; rows from `valid` on, and columns from D
// on, are zeros) as planes of bf16, in squares of 64: by rows at rows_out
// [kPlanes][plane][ld] and, turned over, at cols_out [kPlanes][plane][ld], there
// times its factor's power of two (factors may be null: 1).
constexpr int kSquare = 64;
constexpr int kPackThreads = 256;
struct Packed {
  uint16_t* p;  // may be null: not written
  int64_t plane, ld;
};
template <typename T>
struct PackJob {
  const T* src;
  int64_t ld;
  const int32_t* list;
  const Plan* plan;
  int64_t rows, squares;  // squares along the rows
  Packed by_row, by_col;
  const float* factors;
};
// The squares from `begin` on of one job and then another: the rows of x and the first piece of the table go together
// (6001 x 300 and 30011 x 300 bf16: 12.2 us).
template <typename T, int kPlanes>
__global__ __launch_bounds__(kPackThreads) void pack_kernel(const PackJob<T> one, const PackJob<T> two, int64_t begin, int D) {
  __shared__ float sq[kSquare][kSquare + 1];
  const int64_t square = begin + blockIdx.x;
  const bool second = square >= one.squares;
  const T* src = second ? two.src : one.src;
  const int64_t ld = second ? two.ld : one.ld;
  const int32_t* list = second ? two.list : one.list;
  const Plan* plan = second ? two.plan : one.plan;
  const Packed by_row = second ? two.by_row : one.by_row, by_col = second ? two.by_col : one.by_col;
  const float* factors = second ? two.factors : one.factors;
  const int64_t valid = plan != nullptr ? plan->live : second ? two.rows : one.rows;
  const int64_t r0 = (second ? square - one.squares : square) * kSquare;
  const int c0 = static_cast<int>(blockIdx.y) * kSquare;
  if (r0 >= round_up(valid, kTile)) return;
  // 8 lanes to a row, so that a wave writes whole lines; rows a and a + 32
  const int tid = static_cast<int>(threadIdx.x), a = tid / 8, b = tid % 8 * 8;
  float v[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t r = r0 + a + 32 * h;
    load_part(src + (r < valid ? (list != nullptr ? list[r] : r) * ld : 0) + c0 + b, r < valid ? D - (c0 + b) : 0, 0.0f, v[h]);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t r = r0 + a + 32 * h;
    if (by_row.p != nullptr) {
      uint4 w[kPlanes];
      split8<kPlanes>(v[h], w);
#pragma unroll
      for (int i = 0; i < kPlanes; ++i)
        *reinterpret_cast<uint4*>(by_row.p + i * by_row.plane + r * by_row.ld + c0 + b) = w[i];
    }
    if (by_col.p != nullptr) {
      const float factor = factors != nullptr && r < valid ? power(factors[list[r]]) : 1.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sq[a + 32 * h][b + e] = factor * v[h][e];
    }
  }
  if (by_col.p == nullptr) return;
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[h][e] = sq[b + e][a + 32 * h];
    uint4 w[kPlanes];
    split8<kPlanes>(v[h], w);
#pragma unroll
    for (int i = 0; i < kPlanes; ++i)
      *reinterpret_cast<uint4*>(by_col.p + i * by_col.plane + (c0 + a + 32 * h) * by_col.ld + r0 + b) = w[i];
  }
}

// ---------------------------------------------------------------- forward
// A unit is a tile of tokens and a run of `per` tiles of the piece's vocabulary.
// The vocabulary is m and the tokens are n, so a lane has 64 logits of each of
// its two tokens: maximum and sum stay in the lane until the run's end.
// partials [unit][3][kTile]: maximum, sum of exponentials, sum of logits.
template <int kPlanes, bool kSmooth>
__global__ __launch_bounds__(kThreads) void loss_kernel(Operand W, Operand X, const Plan* __restrict__ plan, int K,
                                                        int64_t v_begin, int v_count,
                                                        const int32_t* __restrict__ targets,
                                                        const int32_t* __restrict__ list,
                                                        float* __restrict__ at_target, float* __restrict__ partials) {
  __shared__ Buffers lds;
  __shared__ float join[3][kTile];
  const int tid = static_cast<int>(threadIdx.x), lane = tid % kWave, wave = uniform(tid / kWave);
  const int wm = wave / 4, wn = wave % 4, half = lane / 32;
  const int live = uniform(plan->live), tiles = uniform(plan->tiles), splits = uniform(plan->splits);
  const int nv = tiles_of(v_count), per = (nv + splits - 1) / splits;
  struct Units {
    int tiles, splits, u, run, n0;
    __device__ __forceinline__ bool find() {
      if (u >= tiles * splits) return false;
      // four tiles of tokens side by side on each run
      const int group = u / (4 * splits), in = u - group * 4 * splits, wide = min(4, tiles - group * 4);
      run = in / wide;
      n0 = (group * 4 + in % wide) * kTile;
      return true;
    }
  };
  struct Next {
    Units unit;
    int per, nv, K, tile, end;
    __device__ __forceinline__ bool operator()(Span& s) {
      while (tile >= end) {
        if (!unit.find()) return false;
        tile = unit.run * per;
        end = min(nv, tile + per);
        unit.u += kGrid;
      }
      s = Span{tile++ * kTile, unit.n0, 0, K};
      return true;
    }
  };
  Units unit{tiles, splits, first_unit(), 0, 0};
  Next next{unit, per, nv, K, 0, 0};
  Product<kPlanes, false> product(W, X, lds);
  Span ahead;
  if (next(ahead)) product.start(ahead);
  for (; unit.find(); unit.u += kGrid) {
    const int run = unit.run, n0 = unit.n0;
    float top[kNT], sum[kNT], all[kNT];
    int target[kNT];
#pragma unroll
    for (int j = 0; j < kNT; ++j) {
      top[j] = kLowest;
      sum[j] = all[j] = 0.0f;
      const int t = n0 + wn * 64 + j * 32 + lane % 32;
      target[j] = t < live ? static_cast<int>(targets[list[t]] - v_begin) : -1;
    }
    for (int tile = run * per; tile < min(nv, (run + 1) * per); ++tile) {
      acc16 acc[kMT][kNT];
      clear(acc);
      const int m0 = tile * kTile;
      product.run(acc);
      if (next(ahead)) product.start(ahead);
      const int v0 = m0 + wm * 128 + 4 * half;  // + 32 i + tile_row(e, 0): the entry of acc[i][j][e]
      if (m0 > v_count - kTile) {               // rows past the vocabulary's end
#pragma unroll
        for (int i = 0; i < kMT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const bool in_v = v0 + 32 * i + tile_row(e, 0) < v_count;
#pragma unroll
            for (int j = 0; j < kNT; ++j) acc[i][j][e] = in_v ? acc[i][j][e] : -INFINITY;
          }
      }
#pragma unroll
      for (int j = 0; j < kNT; ++j) {
        float m = top[j];
#pragma unroll
        for (int i = 0; i < kMT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) m = fmaxf(m, acc[i][j][e]);
        float s = sum[j] * __builtin_amdgcn_exp2f((top[j] - m) * kLog2e);
        top[j] = m;
#pragma unroll
        for (int i = 0; i < kMT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) s += __builtin_amdgcn_exp2f((acc[i][j][e] - m) * kLog2e);
        sum[j] = s;
        const int rel = target[j] - v0;
        if (__any(rel >= 0 && rel < 128)) {
#pragma unroll
          for (int i = 0; i < kMT; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (rel == 32 * i + tile_row(e, 0)) at_target[n0 + wn * 64 + j * 32 + lane % 32] = acc[i][j][e];
        }
        if (kSmooth) {
          float q = 0.0f;
#pragma unroll
          for (int i = 0; i < kMT; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) q += v0 + 32 * i + tile_row(e, 0) < v_count ? acc[i][j][e] : 0.0f;
          all[j] += q;
        }
      }
    }
    // the other half of the wave has the other rows of the same tokens, the other wave along m likewise
#pragma unroll
    for (int j = 0; j < kNT; ++j) {
      const float m2 = __shfl_xor(top[j], 32), s2 = __shfl_xor(sum[j], 32), a2 = __shfl_xor(all[j], 32);
      const float m = fmaxf(top[j], m2);
      sum[j] = sum[j] * __builtin_amdgcn_exp2f((top[j] - m) * kLog2e) + s2 * __builtin_amdgcn_exp2f((m2 - m) * kLog2e);
      top[j] = m;
      all[j] += a2;
      if (wm == 1 && half == 0) {
        const int n = wn * 64 + j * 32 + lane % 32;
        join[0][n] = top[j];
        join[1][n] = sum[j];
        join[2][n] = all[j];
      }
    }
    __syncthreads();
    if (wm == 0 && half == 0) {
      float* out = partials + (static_cast<int64_t>(run) * tiles + n0 / kTile) * 3 * kTile;
#pragma unroll
      for (int j = 0; j < kNT; ++j) {
        const int n = wn * 64 + j * 32 + lane % 32;
        const float m2 = join[0][n], m = fmaxf(top[j], m2);
        out[n] = m;
        out[kTile + n] = sum[j] * __builtin_amdgcn_exp2f((top[j] - m) * kLog2e) +
                         join[1][n] * __builtin_amdgcn_exp2f((m2 - m) * kLog2e);
        out[2 * kTile + n] = all[j] + join[2][n];
      }
    }
    __syncthreads();
  }
}

// Joins the runs of every token, one wave per token; a token without a target has loss 0 and lse 0.
__global__ __launch_bounds__(kPackThreads) void loss_join_kernel(const Plan* __restrict__ plan,
                                                                 const int32_t* __restrict__ slot_of, int64_t begin,
                                                                 int64_t T, int64_t V, int pieces, int64_t piece_stride,
                                                                 const float* __restrict__ at_target,
                                                                 const float* __restrict__ partials, float smoothing,
                                                                 float* __restrict__ loss, float* __restrict__ lse) {
  const int64_t t = begin + static_cast<int64_t>(blockIdx.x) * (kPackThreads / kWave) + threadIdx.x / kWave;
  if (t >= T) return;
  const int slot = slot_of[t], lane = lane_id();
  if (slot < 0) {
    if (lane == 0) loss[t] = lse[t] = 0.0f;
    return;
  }
  const int tiles = plan->tiles, splits = plan->splits;
  float m = kLowest, s = 0.0f, a = 0.0f;
  for (int i = lane; i < pieces * splits; i += kWave) {
    const float* in = partials + i / splits * piece_stride +
                      (static_cast<int64_t>(i % splits) * tiles + slot / kTile) * 3 * kTile + slot % kTile;
    const float m2 = in[0], top = fmaxf(m, m2);
    s = s * __builtin_amdgcn_exp2f((m - top) * kLog2e) + in[kTile] * __builtin_amdgcn_exp2f((m2 - top) * kLog2e);
    a += in[2 * kTile];
    m = top;
  }
#pragma unroll
  for (int k = 1; k < kWave; k *= 2) {
    const float m2 = __shfl_xor(m, k), s2 = __shfl_xor(s, k), top = fmaxf(m, m2);
    s = s * __builtin_amdgcn_exp2f((m - top) * kLog2e) + s2 * __builtin_amdgcn_exp2f((m2 - top) * kLog2e);
    a += __shfl_xor(a, k);
    m = top;
  }
  if (lane == 0) {
    const float l = m + logf(s);
    lse[t] = l;
    loss[t] = smoothing == 0.0f ? l - at_target[slot]
                                : l - (1.0f - smoothing) * at_target[slot] - smoothing * (a / static_cast<float>(V));
  }
}

// ---------------------------------------------------------------- forward, few tokens
// The tokens' rows stand in LDS, as planes, zeros where there is no target, and the table goes from memory into registers,
// which is what bounds the kernel.  A workgroup has the rows of 16, 32 or 64 tokens: where these are all tokens the table
// is read once, and else once for each such group.  64 rows fit up to 1056 columns of bf16 (352 of fp32, which has three
// planes), 32 up to 2144 (704), 16 up to 4320 (1440): 262144 entries of 1024 columns take 98 us for 1 token and 100 for 64
// in bf16, 205, 205, 388 and 738 us for 1, 16, 32 and 64 tokens in fp32.  Wider rows go the way of many tokens.
// A wave takes 16 entries at a time (16 x 16 x 32 matrix instructions: lane l has 8 values along k of entry l % 16, so a
// load covers 64 bytes of each entry's row, at any alignment).  A lane has 4 logits of one token of every 16: maximum and
// sum stay in the lane until the end.  Workgroups (i, y) take tokens 16 kTok y ..; partials [y][i][3][64].
constexpr int kFew = 64;
constexpr int kFewThreads = 512;
constexpr int kFewWaves = kFewThreads / kWave;
constexpr int kFewLds = 136 << 10;
typedef float acc4 __attribute__((ext_vector_type(4)));
__host__ __device__ constexpr int few_row(int D) { return (D + 31) / 32 * 32 + 8; }  // 16 bytes on: 16 rows in all banks
__host__ __device__ constexpr int few_tokens(int64_t T) { return T <= 16 ? 16 : T <= 32 ? 32 : 64; }
// Tokens that a workgroup takes (0: none, a row does not fit).
int few_fit(int64_t T, int D, int planes) {
  for (int n = few_tokens(T); n >= 16; n /= 2)
    if (static_cast<int64_t>(n) * few_row(D) * planes * 2 <= kFewLds) return n;
  return 0;
}
// Whether a call goes this way: up to 64 tokens, whose time is that of reading the table, and more of them where there is
// so little to compute that the four or five launches of the other way take longer.  Measured (the other way, this one):
// 512 tokens x 1000 x 64 fp32 31.6 and 11.8 us; bf16 1024 x 4000 x 512 33.7 and 22.7, 4096 x 8000 x 64 33.1 and 32.4, 128 x
// 32000 x 1024 44.9 and 51.9; fp32 1000 x 3000 x 512 95.9 and 45.8.
constexpr double kFewWork = 4e9;
bool few(int64_t T, int64_t V, int D, int planes) {
  if (few_fit(T, D, planes) == 0) return false;
  return T <= kFew || (T <= (1 << 16) && 2.0 * T * V * D <= kFewWork);
}

// Eight values along k of one row as an operand of each plane.
template <int kPlanes>
__device__ __forceinline__ void few_split(const Vec<bf16, 8>& v, frag (&out)[kPlanes]) {
  out[0] = __builtin_bit_cast(frag, v.w);
}
template <int kPlanes>
__device__ __forceinline__ void few_split(const Vec<float, 8>& v, frag (&out)[kPlanes]) {
  uint4 w[kPlanes];
  split8<kPlanes>(v.x, w);
#pragma unroll
  for (int p = 0; p < kPlanes; ++p) out[p] = __builtin_bit_cast(frag, w[p]);
}

// The tokens' rows as planes in LDS [kPlanes][16 kTok][few_row(D)], zeros where there is no target.
template <typename T, int kPlanes, int kTok>
__device__ __forceinline__ void few_stage(const T* __restrict__ x, int64_t ldx, int tokens, int64_t V, int D,
                                          const int32_t* __restrict__ targets, uint16_t* rows, int32_t* status) {
  const int ld = few_row(D), chunks = (D + 31) / 32 * 4, plane = kTok * 16 * ld;
  bool bad = false;
  constexpr int kAhead = 4;  // loads in flight
  for (int i0 = static_cast<int>(threadIdx.x); i0 < kTok * 16 * chunks; i0 += kAhead * kFewThreads) {
    int id[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int t = (i0 + k * kFewThreads) / chunks;
      id[k] = t < tokens ? targets[t] : -1;
    }
    Vec<T, 8> v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = i0 + k * kFewThreads, t = i / chunks, c = (i - t * chunks) * 8;
      bad |= id[k] >= V;
      v[k].load(x + (t < tokens ? t * ldx + c : 0), id[k] >= 0 && id[k] < V ? D - c : 0);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = i0 + k * kFewThreads, t = i / chunks, c = (i - t * chunks) * 8;
      if (t >= kTok * 16) break;
      frag f[kPlanes];
      few_split<kPlanes>(v[k], f);
#pragma unroll
      for (int p = 0; p < kPlanes; ++p) *reinterpret_cast<frag*>(rows + p * plane + t * ld + c) = f[p];
    }
  }
  if (blockIdx.x == 0 && __any(bad) && lane_id() == 0) raise_flag(status, EMB_DEV_ID_OUT_OF_RANGE);
  __syncthreads();
}

// Logits of entries b * 16 .. + 15: acc[n][e] of token 16 n + lane % 16, entry b * 16 + 4 (lane / 16) + e.  A row passes
// through two batches of registers, one being multiplied while the other is read (262144 entries of 1024: 1 token bf16 98
// us, 64 tokens 104, fp32 1 token 192, 64 tokens 790; with batches of twice the size and nothing in flight between them 106,
// 118, 231 and 917; a small table in fp32, 64 tokens x 3000 x 512: 18.0 against 16.4).
template <typename T, int kPlanes, int kTok>
__device__ __forceinline__ void few_logits(const T* __restrict__ table, int64_t ldw, int64_t b, int64_t V, int D,
                                           const uint16_t* rows, acc4 (&acc)[kTok]) {
  const int row = static_cast<int>(lane_id()) % 16, group = static_cast<int>(lane_id()) / 16;
  const int ld = few_row(D), plane = kTok * 16 * ld;
  const uint16_t* mine = rows + row * ld + 8 * group;
  const T* w = table + min(b * 16 + row, V - 1) * ldw + 8 * group;
#pragma unroll
  for (int n = 0; n < kTok; ++n) acc[n] = acc4{0.0f, 0.0f, 0.0f, 0.0f};
  const auto multiply = [&](const Vec<T, 8>& v, int k) {
    frag a[kPlanes];
    few_split<kPlanes>(v, a);
#pragma unroll
    for (int n = 0; n < kTok; ++n)
#pragma unroll
      for (int i = 0; i < kPairs<kPlanes>; ++i) {
        int pa, pb;
        plane_pair<kPlanes>(i, pa, pb);
        const frag f = *reinterpret_cast<const frag*>(mine + pb * plane + n * 16 * ld + k);
        acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[pa], f, acc[n], 0, 0, 0);
      }
  };
  constexpr int kBatch = kPlanes > 1 && kTok > 2 ? 2 : 4;  // loads at a time; more would spill
  int k = 0;
  if (D >= 32 * kBatch) {
    Vec<T, 8> v[2][kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) v[0][i].template load<true>(w + 32 * i, 8);
    for (bool more = true; more;) {
#pragma unroll
      for (int h = 0; h < 2 && more; ++h) {
        const int next = k + 32 * kBatch;
        more = next + 32 * kBatch <= D;
        if (more) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i) v[1 - h][i].template load<true>(w + next + 32 * i, 8);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) multiply(v[h][i], k + 32 * i);
        k = next;
      }
    }
  }
  for (; k < D; k += 32) {
    Vec<T, 8> v;
    v.load(w + k, D - k - 8 * group);
    multiply(v, k);
  }
}

template <typename T, int kPlanes, int kTok, bool kSmooth>
__global__ __launch_bounds__(kFewThreads, 4) void loss_few_kernel(int waves, const T* __restrict__ x, int64_t ldx,
                                                                  const T* __restrict__ table, int64_t ldw, int tokens,
                                                                  int64_t V, int D, const int32_t* __restrict__ targets,
                                                                  float* __restrict__ at_target,
                                                                  float* __restrict__ partials, int32_t* status) {
  extern __shared__ __attribute__((aligned(16))) uint16_t rows[];
  __shared__ float join[3][kFewWaves][kTok * 16];
  const int tid = static_cast<int>(threadIdx.x), lane = tid % kWave, wave = uniform(tid / kWave);
  const int row = lane % 16, group = lane / 16;
  const int t0 = static_cast<int>(blockIdx.y) * kTok * 16;  // this workgroup's tokens
  x += t0 * ldx;
  targets += t0;
  at_target += t0;
  tokens = min(tokens - t0, kTok * 16);
  few_stage<T, kPlanes, kTok>(x, ldx, tokens, V, D, targets, rows, status);
  float top[kTok], sum[kTok], all[kTok];
  int target[kTok];
#pragma unroll
  for (int n = 0; n < kTok; ++n) {
    top[n] = kLowest;
    sum[n] = all[n] = 0.0f;
    target[n] = n * 16 + row < tokens ? targets[n * 16 + row] : -1;
  }
  const int64_t blocks = wave < waves ? (V + 15) / 16 : 0, step = static_cast<int64_t>(gridDim.x) * waves;
  for (int64_t b = static_cast<int64_t>(blockIdx.x) * waves + wave; b < blocks; b += step) {
    acc4 acc[kTok];
    few_logits<T, kPlanes, kTok>(table, ldw, b, V, D, rows, acc);
    const int64_t v0 = b * 16 + 4 * group;
#pragma unroll
    for (int n = 0; n < kTok; ++n) {
      float m = top[n], s;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (v0 + e == target[n]) at_target[n * 16 + row] = acc[n][e];
        if (kSmooth) all[n] += v0 + e < V ? acc[n][e] : 0.0f;
        acc[n][e] = v0 + e < V ? acc[n][e] : -INFINITY;
        m = fmaxf(m, acc[n][e]);
      }
      s = sum[n] * __builtin_amdgcn_exp2f((top[n] - m) * kLog2e);
      top[n] = m;
#pragma unroll
      for (int e = 0; e < 4; ++e) s += __builtin_amdgcn_exp2f((acc[n][e] - m) * kLog2e);
      sum[n] = s;
    }
  }
#pragma unroll
  for (int n = 0; n < kTok; ++n) {
#pragma unroll
    for (int d = 16; d < kWave; d *= 2) {
      const float m2 = __shfl_xor(top[n], d), s2 = __shfl_xor(sum[n], d), m = fmaxf(top[n], m2);
      sum[n] = sum[n] * __builtin_amdgcn_exp2f((top[n] - m) * kLog2e) + s2 * __builtin_amdgcn_exp2f((m2 - m) * kLog2e);
      top[n] = m;
      all[n] += __shfl_xor(all[n], d);
    }
    if (group == 0) {
      join[0][wave][n * 16 + row] = top[n];
      join[1][wave][n * 16 + row] = sum[n];
      join[2][wave][n * 16 + row] = all[n];
    }
  }
  __syncthreads();
  if (tid < kTok * 16) {
    float m = join[0][0][tid], s = join[1][0][tid], a = join[2][0][tid];
#pragma unroll
    for (int i = 1; i < kFewWaves; ++i) {
      const float m2 = join[0][i][tid], both = fmaxf(m, m2);
      s = s * __builtin_amdgcn_exp2f((m - both) * kLog2e) + join[1][i][tid] * __builtin_amdgcn_exp2f((m2 - both) * kLog2e);
      a += join[2][i][tid];
      m = both;
    }
    float* out = partials + (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * 3 * kFew + tid;
    out[0] = m;
    out[kFew] = s;
    out[2 * kFew] = a;
  }
}

// One workgroup of one wave per token.
__global__ __launch_bounds__(kWave) void loss_few_join_kernel(int parts, int group, int64_t V, const int32_t* __restrict__ targets,
                                                              const float* __restrict__ at_target,
                                                              const float* __restrict__ partials, float smoothing,
                                                              float* __restrict__ loss, float* __restrict__ lse) {
  const int t = static_cast<int>(blockIdx.x), lane = lane_id();
  const int id = targets[t];
  float m = kLowest, s = 0.0f, a = 0.0f;
  for (int i = lane; i < parts; i += kWave) {
    const float* in = partials + (static_cast<int64_t>(t / group) * parts + i) * 3 * kFew + t % group;
    const float m2 = in[0], top = fmaxf(m, m2);
    s = s * __builtin_amdgcn_exp2f((m - top) * kLog2e) + in[kFew] * __builtin_amdgcn_exp2f((m2 - top) * kLog2e);
    a += in[2 * kFew];
    m = top;
  }
#pragma unroll
  for (int k = 1; k < kWave; k *= 2) {
    const float m2 = __shfl_xor(m, k), s2 = __shfl_xor(s, k), top = fmaxf(m, m2);
    s = s * __builtin_amdgcn_exp2f((m - top) * kLog2e) + s2 * __builtin_amdgcn_exp2f((m2 - top) * kLog2e);
    a += __shfl_xor(a, k);
    m = top;
  }
  if (lane == 0) {
    const bool live = id >= 0 && id < V;
    const float l = m + logf(s), z = live ? at_target[t] : 0.0f;
    lse[t] = live ? l : 0.0f;
    loss[t] = !live ? 0.0f
              : smoothing == 0.0f ? l - z : l - (1.0f - smoothing) * z - smoothing * (a / static_cast<float>(V));
  }
}

// ---------------------------------------------------------------- backward
// g of one piece of the vocabulary, by token [kPlanes][tokens][ld]: without dloss
// where one holds for all tokens (dx and dW take it at their ends; the target's g
// is then near -1, which bf16 holds better than a multiple of it), else with its
// mantissa (factors; dx takes the power of two at its end, dW with the rows of x:
// either way g is rounded once and nothing else is).  A lane has
// single values of a token's row, 4 entries side by side; a wave turns 32 tokens
// x 64 entries at a time through LDS of its own (chunk c of 16 bytes of token
// t's row at place c ^ (t & 7)) and writes 128 bytes of a row at once.
template <int kPlanes>
__global__ __launch_bounds__(kThreads) void grad_logits_kernel(Operand W, Operand X, const Plan* __restrict__ plan,
                                                               int K, int64_t V, int64_t v_begin, int v_count,
                                                               const int32_t* __restrict__ targets,
                                                               const int32_t* __restrict__ list,
                                                               const float* __restrict__ lse_in,
                                                               const float* __restrict__ factors, float smoothing,
                                                               Packed by_token) {
  __shared__ Buffers lds;
  __shared__ __attribute__((aligned(16))) char turns[kThreads / kWave][32 * 128];
  const int tid = static_cast<int>(threadIdx.x), lane = tid % kWave, wave = uniform(tid / kWave);
  const int wm = wave / 4, wn = wave % 4, half = lane / 32;
  const int live = uniform(plan->live), tiles = uniform(plan->tiles);
  const int nv = tiles_of(v_count);
  const float even = smoothing / static_cast<float>(V);
  char* turn = turns[wave];
  struct Next {
    int tiles, nv, K, u;
    __device__ __forceinline__ bool operator()(Span& s) {
      if (u >= tiles * nv) return false;
      const int group = u / (4 * nv), in = u - group * 4 * nv, wide = min(4, tiles - group * 4);
      s = Span{in / wide * kTile, (group * 4 + in % wide) * kTile, 0, K};
      u += kGrid;
      return true;
    }
  };
  Next next{tiles, nv, K, first_unit()};
  Product<kPlanes, false> product(W, X, lds);
  Span ahead;
  int from[kNT];  // the lane's tokens of the tile to come; -1: none
  const auto look = [&](const Span& s) {
#pragma unroll
    for (int j = 0; j < kNT; ++j) {
      const int t = s.n0 + wn * 64 + j * 32 + lane % 32;
      from[j] = t < live ? list[t] : -1;
    }
  };
  bool more = next(ahead);
  if (more) {
    product.start(ahead);
    look(ahead);
  }
  while (more) {
    const int m0 = ahead.m0, n0 = ahead.n0;
    const int mine = wm * 128 + 4 * half;
    int rel[kNT];  // the target from this lane's first entry on
    float l[kNT], d[kNT];
#pragma unroll
    for (int j = 0; j < kNT; ++j) {
      const bool some = from[j] >= 0;
      rel[j] = some ? static_cast<int>(targets[from[j]] - v_begin) - m0 - mine : -1;
      l[j] = some ? lse_in[from[j]] : 0.0f;
      d[j] = some && factors != nullptr ? mantissa(factors[from[j]]) : 1.0f;
    }
    acc16 acc[kMT][kNT];
    clear(acc);
    product.run(acc);
    more = next(ahead);
    if (more) {
      product.start(ahead);
      look(ahead);
    }
#pragma unroll
    for (int j = 0; j < kNT; ++j) {
      const float below = -even * d[j];
#pragma unroll
      for (int i = 0; i < kMT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float z = acc[i][j][e];
          const float x = (z - l[j]) * kLog2e;  // the difference first: z and l may be far from 0
          acc[i][j][e] = fmaf(__builtin_amdgcn_exp2f(x), d[j], below);
        }
      if (__any(rel[j] >= 0 && rel[j] < 128)) {
        const float less = (1.0f - smoothing) * d[j];
#pragma unroll
        for (int i = 0; i < kMT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            if (e % 4 == 0) asm volatile("" : "+v"(rel[j]));  // not all comparisons at once
            if (rel[j] == 32 * i + tile_row(e, 0)) acc[i][j][e] -= less;
          }
      }
      if (m0 + kTile > v_count || n0 + kTile > live) {  // zeros behind the piece's end and the last token
        int end = n0 + wn * 64 + j * 32 + lane % 32 < live ? v_count - m0 - mine : 0;
#pragma unroll
        for (int i = 0; i < kMT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            if (e % 4 == 0) asm volatile("" : "+v"(end));
            acc[i][j][e] = 32 * i + tile_row(e, 0) < end ? acc[i][j][e] : 0.0f;
          }
      }
    }
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
      uint16_t* out = by_token.p + p * by_token.plane + (n0 + wn * 64 + lane / 8) * by_token.ld + m0 + wm * 128 + lane % 8 * 8;
#pragma unroll
      for (int j = 0; j < kNT; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const int i = 2 * h + c / 4, q = c % 4;
            uint2 w;
            if constexpr (kPlanes == 1) {
              w = make_uint2(bf16_pair(acc[i][j][4 * q], acc[i][j][4 * q + 1]),
                             bf16_pair(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]));
            } else {  // the leading 16 bits of each; what is left is for the next plane
              uint32_t top[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                top[e] = __float_as_uint(acc[i][j][4 * q + e]) & 0xFFFF0000u;
                acc[i][j][4 * q + e] -= __uint_as_float(top[e]);
              }
              w = make_uint2(top[0] >> 16 | top[1], top[2] >> 16 | top[3]);
            }
            *reinterpret_cast<uint2*>(turn + lane % 32 * 128 + (c ^ (lane & 7)) * 16 + 8 * half) = w;
          }
          __builtin_amdgcn_wave_barrier();
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int t = 8 * r + lane / 8;
            const uint4 w = *reinterpret_cast<const uint4*>(turn + t * 128 + (lane % 8 ^ (t & 7)) * 16);
            *reinterpret_cast<uint4*>(out + (32 * j + 8 * r) * by_token.ld + 64 * h) = w;
          }
          __builtin_amdgcn_wave_barrier();
        }
    }
  }
}

// The tiles of a product whose k is split into runs.
template <int kWN>
struct Runs {
  int tm, tn, splits, steps, u, run;
  __device__ __forceinline__ bool operator()(Span& s) {
    if (u >= tm * tn * splits) return false;
    run = u / (tm * tn);
    const int in = u - run * tm * tn, per = (steps + splits - 1) / splits;
    s = Span{in / tn * kTile, in % tn * 64 * kWN, min(run * per, steps) * kStep, min((run + 1) * per, steps) * kStep};
    u += kGrid;
    return true;
  }
};

// dx of one piece, added to (the first piece: stored in) parts: A = g by token, B = W by column, k over the piece's
// entries, in `splits` runs.  A lane's 32 kWN sums of tile u stand in the order in which it has them, 4 at a time, at
// parts + (u 8 kWN + (kWN j + i) 4 + q) 2048 + 4 thread, and are the products' starting values: they are read while
// the tile's first copies are on their way (read and added at the end, row by row: 60 us of 500).  With planes of fp32 they
// are added at the end all the same: the small products would lose their last bits against them.
template <int kPlanes, int kWN>
__global__ __launch_bounds__(kThreads) void grad_rows_kernel(Operand G, Operand Wt, const Plan* __restrict__ plan, int nd,
                                                             int K, bool first, float* __restrict__ parts) {
  __shared__ Buffers lds;
  const int tiles = uniform(plan->tiles), splits = uniform(plan->splits);
  Runs<kWN> next{tiles, nd, splits, K / kStep, first_unit(), 0};
  Product<kPlanes, false, kWN> product(G, Wt, lds);
  Span ahead;
  bool more = next(ahead);
  if (more) product.start(ahead);
  while (more) {
    float* mine = parts + static_cast<int64_t>(next.u - kGrid) * kTile * 64 * kWN + threadIdx.x * 4;
    acc16 acc[kWN][kNT];
    clear(acc);
    if (kPlanes == 1 && !first) {
#pragma unroll
      for (int i = 0; i < kWN; ++i)
#pragma unroll
        for (int j = 0; j < kNT; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 v = *reinterpret_cast<const float4*>(mine + ((kWN * j + i) * 4 + q) * 2048);
            acc[i][j][4 * q] = v.x;
            acc[i][j][4 * q + 1] = v.y;
            acc[i][j][4 * q + 2] = v.z;
            acc[i][j][4 * q + 3] = v.w;
          }
    }
    product.run(acc);
    more = next(ahead);
    if (more) product.start(ahead);
#pragma unroll
    for (int i = 0; i < kWN; ++i)
#pragma unroll
      for (int j = 0; j < kNT; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float4* p = reinterpret_cast<float4*>(mine + ((kWN * j + i) * 4 + q) * 2048);
          float4 v = make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
          if (kPlanes > 1 && !first) {
            const float4 old = *p;
            v = make_float4(old.x + v.x, old.y + v.y, old.z + v.z, old.w + v.w);
          }
          *p = v;
        }
  }
}

// dx: the factor (a token's own: its power of two) times the runs' sum of every live token (the first tokens_blocks
// workgroups from `first` on, 8 kWN to a tile), 0 for the others (the rest, kThreads / 8 tokens each).
template <typename T, int kWN>
__global__ __launch_bounds__(kThreads) void grad_rows_join_kernel(int64_t first, const Plan* __restrict__ plan,
                                                                  const int32_t* __restrict__ list,
                                                                  const int32_t* __restrict__ slot_of, int64_t tokens_blocks,
                                                                  int64_t tokens, int D, int nd,
                                                                  const float* __restrict__ parts,
                                                                  const float* __restrict__ dloss, int dloss_step,
                                                                  T* __restrict__ dx, int64_t lddx) {
  const int tid = static_cast<int>(threadIdx.x);
  const int64_t block = first + blockIdx.x;
  if (block >= tokens_blocks) {
    const int64_t t = (block - tokens_blocks) * (kThreads / 8) + tid / 8;
    if (t >= tokens || slot_of[t] >= 0) return;
    const float zero[8] = {};
    for (int c = tid % 8 * 8; c < D; c += 64) store_part(dx + t * lddx + c, D - c, zero);
    return;
  }
  const int tile = static_cast<int>(block / (8 * kWN)), part = static_cast<int>(block % (8 * kWN));  // (kWN j + i) 4 + q
  const int units = plan->tiles * nd, splits = plan->splits, live = plan->live;
  if (tile >= units) return;
  const int lane = tid % kWave, wave = tid / kWave;
  const int m = tile / nd * kTile + wave / kWN * 32 * kWN + part % (4 * kWN) * 8 + 4 * (lane / 32);
  const int d = tile % nd * 64 * kWN + wave % kWN * 64 + part / (4 * kWN) * 32 + lane % 32;
  const float4* p = reinterpret_cast<const float4*>(parts + static_cast<int64_t>(tile) * kTile * 64 * kWN) + part * 512 + tid;
  const int64_t next = static_cast<int64_t>(units) * (kTile * 16 * kWN);
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
  for (int r = 0; r < splits; ++r, p += next) {
    const float4 v = *p;
    s.x += v.x;
    s.y += v.y;
    s.z += v.z;
    s.w += v.w;
  }
  const float row[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (m + e < live && d < D) {
      const int64_t t = list[m + e];
      narrow((dloss_step != 0 ? power(dloss[t]) : dloss[0]) * row[e], dx + t * lddx + d);
    }
}

// dW of one piece: A = g turned over, B = x by column, k over the live tokens, in `table_splits` runs: one writes dW,
// more write parts [run][entries][ld] fp32.  factor: one for all tokens, or null (the rows of x have theirs).
template <typename T, int kPlanes, int kWN>
__global__ __launch_bounds__(kThreads) void grad_table_kernel(Operand G, Operand Xt, const Plan* __restrict__ plan, int nd,
                                                              int v_count, int D, T* __restrict__ dW, int64_t ld,
                                                              float* __restrict__ parts, int64_t parts_ld,
                                                              const float* __restrict__ factor) {
  __shared__ Buffers lds;
  const int tid = static_cast<int>(threadIdx.x), lane = tid % kWave, wave = uniform(tid / kWave);
  const int wm = wave / kWN, wn = wave % kWN, half = lane / 32;
  const int nv = tiles_of(v_count), splits = uniform(plan->table_splits);
  const float times = factor != nullptr && plan->live > 0 ? *factor : 1.0f;  // no token: zeros, whatever it is
  Runs<kWN> next{nv, nd, splits, (uniform(plan->live) + kStep - 1) / kStep, first_unit(), 0};
  Product<kPlanes, true, kWN> product(G, Xt, lds);
  Span ahead;
  bool more = next(ahead);
  if (more) product.start(ahead);
  while (more) {
    const int run = next.run, m0 = ahead.m0, n0 = ahead.n0;
    acc16 acc[kWN][kNT];
    clear(acc);
    product.run(acc);
    more = next(ahead);
    if (more) product.start(ahead);
    const int v0 = m0 + wm * 32 * kWN + 4 * half, d0 = n0 + wn * 64 + lane % 32;
    if (splits > 1) {
      each_row<kWN>(parts + (static_cast<int64_t>(run) * nv * kTile + v0) * parts_ld + d0, parts_ld, [&](int i, int e, float* p) {
#pragma unroll
        for (int j = 0; j < kNT; ++j) p[32 * j] = acc[i][j][e];
      });
    } else {
      each_row<kWN>(dW + v0 * ld + d0, ld, [&](int i, int e, T* p) {
#pragma unroll
        for (int j = 0; j < kNT; ++j)
          if (v0 + 32 * i + tile_row(e, 0) < v_count && d0 + 32 * j < D) narrow(times * acc[i][j][e], p + 32 * j);
      });
    }
  }
}

// dW of one piece where more than one run has a part of it.
template <typename T>
__global__ __launch_bounds__(kPackThreads) void grad_table_join_kernel(const Plan* __restrict__ plan, int v_count, int D,
                                                                       int nvec, const float* __restrict__ parts, int64_t ld,
                                                                       const float* __restrict__ factor,
                                                                       T* __restrict__ dW, int64_t lddt) {
  const int splits = plan->table_splits;
  if (splits == 1) return;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kPackThreads + threadIdx.x;
  const int64_t v = i / nvec;
  if (v >= v_count) return;
  const int c = static_cast<int>(i - v * nvec) * 8;
  const int64_t next = round_up(v_count, kTile) * ld;
  const float* p = parts + v * ld + c;
  float s[8] = {};
  for (int r = 0; r < splits; ++r, p += next) {
    float x[8];
    load_vec(p, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += x[e];
  }
  const float times = factor != nullptr && plan->live > 0 ? *factor : 1.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] *= times;
  store_part(dW + v * lddt + c, D - c, s);
}

// ---------------------------------------------------------------- backward, few tokens
// g has more planes than the rows here, where the products cost nothing: two of bf16 beside rows of bf16.
template <int kPlanes>
constexpr int kGPlanes = kPlanes == 1 ? 2 : 3;
template <int kPlanes>
constexpr int kGPairs = kPlanes == 1 ? 2 : 6;
template <int kPlanes>
__device__ __forceinline__ void g_pair(int i, int& pg, int& pr) {  // planes of g and of the rows, the smallest product first
  if constexpr (kPlanes == 1) {
    pg = 1 - i;
    pr = 0;
  } else {
    plane_pair<kPlanes>(i, pg, pr);
  }
}

// g of 16 entries at a time as in the forward pass, and at once their 16 rows of dW: A = x by column (turned on the way
// from LDS, as in Product), B = g, which a wave turns through LDS of its own.  The rows of A are chosen so that a lane has
// 8 values of one entry's row side by side.  g goes to memory for dx, [kPlanes][16 kTok][ldg].
// a wave's g of one plane: 16 entries, rows of 16 tok tokens (32 at least) and 16 bytes
__host__ __device__ constexpr int few_g(int tok) { return 16 * ((tok < 2 ? 32 : 16 * tok) + 8); }
size_t few_grad_lds(int n, int D, int planes, int waves) {
  return (static_cast<size_t>(n) * few_row(D) * planes + waves * few_g(n / 16) * (planes == 1 ? 2 : 3)) * 2;
}
constexpr int64_t kFewG = int64_t{1} << 30;  // values of g at most: it is kept as a whole
// The waves of a workgroup that LDS leaves room for beside the tokens' rows: 8 or 4, 0 where the other way is taken
// (measured with 4, the other way and this one: bf16 64 tokens x 262144 x 1024 776 and 454 us, 64 x 100000 x 1024 313 and
// 197, 39 x 16512 x 975 107 and 119).
int few_grad(int64_t T, int64_t V, int D, int planes) {
  if (T > kFew || V > kFewG / few_tokens(T)) return 0;
  for (const int waves : {8, 4})
    if (few_grad_lds(few_tokens(T), D, planes, waves) <= (158 << 10)) return waves;
  return 0;
}
template <typename T, int kPlanes, int kTok>
__global__ __launch_bounds__(kFewThreads) void few_grad_kernel(int waves, const T* __restrict__ x, int64_t ldx,
                                                               const T* __restrict__ table, int64_t ldw, int tokens,
                                                               int64_t V, int D, const int32_t* __restrict__ targets,
                                                               const float* __restrict__ lse_in,
                                                               const float* __restrict__ dloss, int dloss_step,
                                                               float smoothing, uint16_t* __restrict__ g_out, int64_t ldg,
                                                               T* __restrict__ dW, int64_t lddt, int32_t* status) {
  extern __shared__ __attribute__((aligned(16))) uint16_t rows[];
  constexpr int kK = kTok < 2 ? 1 : kTok / 2;  // steps of 32 tokens
  constexpr int kLd = (kTok < 2 ? 32 : 16 * kTok) + 8;
  const int tid = static_cast<int>(threadIdx.x), lane = tid % kWave, wave = uniform(tid / kWave);
  const int row = lane % 16, group = lane / 16;
  const int ld = few_row(D), plane = kTok * 16 * ld;
  constexpr int kG = kGPlanes<kPlanes>;
  uint16_t* turn = rows + kPlanes * plane + wave * kG * few_g(kTok);
  few_stage<T, kPlanes, kTok>(x, ldx, tokens, V, D, targets, rows, status);
  if (kTok < 2 && wave < waves) {  // tokens 16 .. 31 have none
    for (int i = lane; i < kG * 16 * 16; i += kWave) turn[i / 256 * few_g(kTok) + i / 16 % 16 * kLd + 16 + i % 16] = 0;
  }
  const float even = smoothing / static_cast<float>(V);
  int target[kTok];
  float l[kTok], d[kTok];
#pragma unroll
  for (int n = 0; n < kTok; ++n) {
    const int t = n * 16 + row;
    const int id = t < tokens ? targets[t] : -1;
    target[n] = id >= 0 && id < V ? id : -1;
    l[n] = target[n] >= 0 ? lse_in[t] : 0.0f;
    d[n] = target[n] >= 0 ? dloss[t * dloss_step] : 0.0f;
  }
  const int64_t blocks = wave < waves ? (V + 31) / 32 * 2 : 0, step = static_cast<int64_t>(gridDim.x) * waves;
  for (int64_t b = static_cast<int64_t>(blockIdx.x) * waves + wave; b < blocks; b += step) {
    acc4 acc[kTok];
    few_logits<T, kPlanes, kTok>(table, ldw, b, V, D, rows, acc);
    const int64_t v0 = b * 16 + 4 * group;
#pragma unroll
    for (int n = 0; n < kTok; ++n) {
      uint32_t w[4][kG];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float g = __builtin_amdgcn_exp2f((acc[n][e] - l[n]) * kLog2e) - even;
        if (v0 + e == target[n]) g -= 1.0f - smoothing;
        split<kG>(target[n] >= 0 && v0 + e < V ? g * d[n] : 0.0f, w[e]);
#pragma unroll
        for (int p = 0; p < kG; ++p)
          turn[p * few_g(kTok) + (4 * group + e) * kLd + n * 16 + row] = static_cast<uint16_t>(w[e][p]);
      }
      if (g_out != nullptr) {
#pragma unroll
        for (int p = 0; p < kG; ++p)
          *reinterpret_cast<uint2*>(g_out + (static_cast<int64_t>(p) * kTok * 16 + n * 16 + row) * ldg + v0) =
              make_uint2(w[0][p] | w[1][p] << 16, w[2][p] | w[3][p] << 16);
      }
    }
    if (dW == nullptr) continue;
    __builtin_amdgcn_wave_barrier();
    frag fg[kG][kK];
#pragma unroll
    for (int p = 0; p < kG; ++p)
#pragma unroll
      for (int k = 0; k < kK; ++k)
        fg[p][k] = *reinterpret_cast<const frag*>(turn + p * few_g(kTok) + row * kLd + 32 * k + 8 * group);
    __builtin_amdgcn_wave_barrier();
    const int64_t v = b * 16 + row;
    for (int c = 0; c < D; c += 32) {
      acc4 out[2] = {};
#pragma unroll
      for (int k = 0; k < kK; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          typedef __attribute__((address_space(3))) quad* place_of;
          frag fx[kPlanes];
#pragma unroll
          for (int p = 0; p < kPlanes; ++p) {  // tokens past the last stand for earlier ones: their g is 0
            const int t = 32 * k + 8 * group + row / 4;
            const uint16_t* q = rows + p * plane + c + 8 * (row % 4) + 4 * h;
            const quad lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((place_of)(q + (t & (kTok * 16 - 1)) * ld));
            const quad hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((place_of)(q + (t + 4 & (kTok * 16 - 1)) * ld));
            fx[p] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          }
#pragma unroll
          for (int i = 0; i < kGPairs<kPlanes>; ++i) {
            int pg, px;
            g_pair<kPlanes>(i, pg, px);
            out[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[px], fg[pg][k], out[h], 0, 0, 0);
          }
        }
      const int at = c + 8 * group;
      const float o[8] = {out[0][0], out[0][1], out[0][2], out[0][3], out[1][0], out[1][1], out[1][2], out[1][3]};
      if (v < V) store_part<true>(dW + v * lddt + at, D - at, o);
    }
  }
}

// dx of few tokens: A = g, B = the table turned over.  A wave takes kSlice columns of 32 entries at a time, lays them in
// LDS of its own (blocks of 32 bytes, block b of row v at place b ^ (v & 3 | (v >> 3 & 1) << 2)) and reads them turned.
// The workgroup's waves have one slice and join their sums in LDS, so that an eighth as much goes through memory:
// parts [workgroups of one slice][tokens][D] (64 tokens x 262144 x 1024 bf16: 222 to 180 us with the join).
template <typename T, int kPlanes>
constexpr int kSlice = kPlanes == 1 ? 128 : 64;
template <typename T, int kPlanes, int kTok>
__global__ __launch_bounds__(kFewThreads, kPlanes == 1 && kTok == 1 ? 4 : 2) void few_rows_kernel(const uint16_t* __restrict__ g, int64_t ldg,
                                                                                 const T* __restrict__ table, int64_t ldw,
                                                                                 int tokens, int64_t V, int D, int slices,
                                                                                 float* __restrict__ parts) {
  constexpr int kCols = kSlice<T, kPlanes>, kChunks = kCols / 8, kRowsAt = kWave / kChunks, kLoads = 32 / kRowsAt;
  constexpr int kBlocks = kCols / 16;
  __shared__ __attribute__((aligned(16))) uint16_t tiles[kFewWaves][kPlanes][32 * kCols];
  const int tid = static_cast<int>(threadIdx.x), lane = tid % kWave, wave = uniform(tid / kWave);
  const int row = lane % 16, group = lane / 16;
  const int slice = static_cast<int>(blockIdx.x) % slices, part = static_cast<int>(blockIdx.x) / slices;
  const int stride = static_cast<int>(gridDim.x) / slices * kFewWaves;
  uint16_t(&tile)[kPlanes][32 * kCols] = tiles[wave];
  const int c0 = slice * kCols, chunk = lane % kChunks, r0 = lane / kChunks;
  const auto place = [](int v, int block) { return (block ^ ((v & 3) | (v >> 3 & 1) << 2) % kBlocks) * 16; };
  acc4 acc[kTok][kBlocks] = {};
  const int64_t steps = (V + 31) / 32;
  Vec<T, 8> w[kLoads];
  const auto load = [&](int64_t s) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int64_t v = s * 32 + i * kRowsAt + r0;
      w[i].template load<true>(table + min(v, V - 1) * ldw + c0 + 8 * chunk, v < V ? D - c0 - 8 * chunk : 0);
    }
  };
  int64_t s = part * kFewWaves + wave;
  if (s < steps) load(s);
  for (; s < steps; s += stride) {
    frag fg[kGPlanes<kPlanes>][kTok];
#pragma unroll
    for (int p = 0; p < kGPlanes<kPlanes>; ++p)
#pragma unroll
      for (int n = 0; n < kTok; ++n)
        fg[p][n] = *reinterpret_cast<const frag*>(g + (static_cast<int64_t>(p) * kTok * 16 + n * 16 + row) * ldg + s * 32 + 8 * group);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      frag f[kPlanes];
      few_split<kPlanes>(w[i], f);
      const int v = i * kRowsAt + r0;
#pragma unroll
      for (int p = 0; p < kPlanes; ++p)
        *reinterpret_cast<frag*>(&tile[p][v * kCols + place(v, chunk / 2) + chunk % 2 * 8]) = f[p];
    }
    if (s + stride < steps) load(s + stride);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      typedef __attribute__((address_space(3))) quad* place_of;
      frag f[kPlanes];
#pragma unroll
      for (int p = 0; p < kPlanes; ++p) {
        const int v = 8 * group + row / 4;
        const quad lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((place_of)&tile[p][v * kCols + place(v, b) + row % 4 * 4]);
        const quad hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((place_of)&tile[p][(v + 4) * kCols + place(v + 4, b) + row % 4 * 4]);
        f[p] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
#pragma unroll
      for (int n = 0; n < kTok; ++n)
#pragma unroll
        for (int i = 0; i < kGPairs<kPlanes>; ++i) {
          int pg, pw;
          g_pair<kPlanes>(i, pg, pw);
          acc[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fg[pg][n], f[pw], acc[n][b], 0, 0, 0);
        }
    }
    __builtin_amdgcn_wave_barrier();
  }
  constexpr int kAtOnce = kBlocks < 8 / kTok ? kBlocks : 8 / kTok, kValues = kAtOnce * kTok * 256;
  static_assert(kValues * 4 <= static_cast<int>(sizeof(tile)), "a wave's sums fit where its tile was");
  float* sums = reinterpret_cast<float*>(tiles);
#pragma unroll
  for (int q = 0; q < kBlocks / kAtOnce; ++q) {
    __syncthreads();
#pragma unroll
    for (int b = 0; b < kAtOnce; ++b)
#pragma unroll
      for (int n = 0; n < kTok; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sums[wave * kValues + ((b * kTok + n) * 16 + 4 * group + e) * 16 + row] = acc[n][q * kAtOnce + b][e];
    __syncthreads();
    for (int i = tid; i < kValues; i += kFewThreads) {
      float v = sums[i];
#pragma unroll
      for (int k = 1; k < kFewWaves; ++k) v += sums[k * kValues + i];
      const int t = i / 16 % (kTok * 16), c = c0 + (q * kAtOnce + i / (kTok * 256)) * 16 + i % 16;
      if (t < tokens && c < D) parts[(static_cast<int64_t>(part) * tokens + t) * D + c] = v;
    }
  }
}

// dx[t][c] = the parts' sum: 32 columns of one token per workgroup, its lanes' groups every 32nd part.  A token without a
// target has 0: its parts are 0 times the table, which is not 0 where the table is not finite.
template <typename T>
__global__ __launch_bounds__(1024) void few_rows_join_kernel(const float* __restrict__ parts, int nparts, int rows, int D,
                                                             int64_t V, const int32_t* __restrict__ targets,
                                                             T* __restrict__ dx, int64_t lddx) {
  __shared__ float red[32][33];
  const int col = static_cast<int>(threadIdx.x) % 32, k = static_cast<int>(threadIdx.x) / 32;
  const int t = static_cast<int>(blockIdx.y), c = static_cast<int>(blockIdx.x) * 32 + col;
  const int id = targets[t];
  float s = 0.0f;
  if (c < D) {
#pragma unroll 8
    for (int p = k; p < nparts; p += 32) s += parts[(static_cast<int64_t>(p) * rows + t) * D + c];
  }
  red[k][col] = s;
  __syncthreads();
  s = group_sum<32>(red[col][k]);
  const int o = static_cast<int>(blockIdx.x) * 32 + k;
  if (col == 0 && o < D) narrow(id >= 0 && id < V ? s : 0.0f, dx + t * lddx + o);
}

// ---------------------------------------------------------------- sizes
// Rows of the table per piece: forward, what is laid out at a time (128 MB of
// bf16); backward, as many as make the piece of g 2^28 elements (2^27 in fp32,
// which has three planes of it).
constexpr int64_t kForwardPiece = int64_t{1} << 26;
constexpr int64_t kMostUnits = 1024;  // forward: units, unless the tokens alone make more
constexpr int64_t kMostParts = 512;   // backward: tiles of dx in parts, unless one run makes more; of dW likewise

struct Sizes {
  int planes;
  int64_t Tp, Kp, Dp, Vp;  // rounded: tokens to tiles, columns to steps, columns to tiles, entries to tiles
  int wn;                  // tiles of dx and dW have 64 wn columns
  bool direct;             // the table is read where it stands
  int64_t piece;           // entries per piece
  int pieces;
};
// Columns of the tiles of dx and dW, over 64: as few tiles' worth as possible, but a narrow tile's column costs more, since
// its operand A is copied for fewer products (16384 tokens x 32768 entries bf16, with 256, 128 and 64 columns: 64 wide 1013,
// 928 and 901 us; 128 wide 1072, 982 and 1196 us; 300 wide 1656, 2077 and 3124 us).
int tile_width(int D) {
  int best = kWide;
  double least = 1e30;
  for (const int wn : {4, 2, 1}) {
    const double cost = static_cast<double>(round_up(D, 64 * wn)) * (wn == 4 ? 1.0 : wn == 2 ? 1.8 : 3.0);
    if (cost < least) {
      least = cost;
      best = wn;
    }
  }
  return best;
}
Sizes sizes_of(int64_t T, int64_t V, int D, bool bf16_in, bool direct, bool backward) {
  Sizes s;
  s.planes = bf16_in ? 1 : 3;
  s.Tp = round_up(T > 0 ? T : 1, kTile);
  s.Kp = round_up(D, kStep);
  s.wn = tile_width(D);
  s.Dp = round_up(D, 64 * s.wn);
  s.Vp = round_up(V, kTile);
  s.direct = direct;
  int64_t piece = backward ? (int64_t{1} << (bf16_in ? 28 : 27)) / s.Tp
                           : direct ? s.Vp : kForwardPiece / (s.Kp * s.planes);
  piece = piece / kTile * kTile;
  if (piece < kTile) piece = kTile;
  s.piece = piece < s.Vp ? piece : s.Vp;
  s.pieces = static_cast<int>((s.Vp + s.piece - 1) / s.piece);
  return s;
}

struct Common {
  Plan* plan;
  int32_t *list, *slot_of;
  uint16_t *x, *w;
};
void carve_common(Carver& c, const Sizes& s, int64_t T, Common& o) {
  o.plan = c.take<Plan>(1);
  o.list = c.take<int32_t>(T);
  o.slot_of = c.take<int32_t>(T);
  o.x = c.take<uint16_t>(s.planes * s.Tp * s.Kp);
  o.w = s.direct ? nullptr : c.take<uint16_t>(s.planes * s.piece * s.Kp);
}
struct Forward : Common {
  float *at_target, *partials;
  int64_t piece_stride;
};
size_t carve(char* base, const Sizes& s, int64_t T, Forward& o) {
  Carver c{base};
  carve_common(c, s, T, o);
  o.at_target = c.take<float>(s.Tp);
  const int64_t units = s.Tp / kTile > kMostUnits ? s.Tp / kTile : kMostUnits;
  o.piece_stride = units * 3 * kTile;
  o.partials = c.take<float>(s.pieces * o.piece_stride);
  return c.size();
}
struct Backward : Common {
  uint16_t *xt, *wt, *g;
  float *parts, *table_parts;
  int64_t g_ld;  // a line more than the piece, so that a tile's rows do not start in the same channel
};
size_t carve(char* base, const Sizes& s, int64_t T, Backward& o) {
  Carver c{base};
  carve_common(c, s, T, o);
  o.xt = c.take<uint16_t>(s.planes * s.Dp * s.Tp);
  o.wt = c.take<uint16_t>(s.planes * s.Dp * s.piece);
  o.g_ld = s.piece + kStep;
  o.g = c.take<uint16_t>(s.planes * s.Tp * o.g_ld);
  const int64_t nd = s.Dp / (64 * s.wn), one = s.Tp / kTile * nd, table = s.piece / kTile * nd;
  o.parts = c.take<float>((one > kMostParts ? one : kMostParts) * kTile * 64 * s.wn);
  o.table_parts = table > kMostParts / 2 ? nullptr : c.take<float>(kMostParts * kTile * 64 * s.wn);
  return c.size();
}

template <typename T, int kPlanes>
void pack(const PackJob<T>& one, const PackJob<T>& two, const Sizes& s, int D, hipStream_t stream) {
  const int64_t squares = one.squares + two.squares, most = 1 << 16;
  for (int64_t b = 0; b < squares; b += most)
    pack_kernel<T, kPlanes><<<dim3(grid_for(squares - b, most), static_cast<unsigned>(s.Kp / kSquare)), kPackThreads, 0,
                              stream>>>(one, two, b, D);
}

template <typename F>
void with_tokens(int n, F&& f) {
  if (n == 16)
    f(std::integral_constant<int, 1>{});
  else if (n == 32)
    f(std::integral_constant<int, 2>{});
  else
    f(std::integral_constant<int, 4>{});
}

struct FewWork {
  float *at_target, *partials;
  int group, groups, across;  // tokens of a workgroup, workgroups side by side over the tokens and over the vocabulary
  int waves;                  // of a workgroup that take entries
};
constexpr int kFewBlocks = 512;
// Waves of a workgroup that take entries, 16 at a time, where there are `blocks` such: where they would not fill `most`
// workgroups, fewer of each, since a wave's chain of loads and products is then what takes the time (all 8, and fewer: 1
// token x 8576 x 960 fp32 28.1 and 18.4 us, its gradient for 7446 x 832 46.9 and 33.2, 364 tokens x 512 x 864 bf16 19.2 and
// 16.1).
int few_waves(int64_t blocks, int64_t most, int limit) {
  const int64_t n = (blocks + most - 1) / most;
  return static_cast<int>(n < limit ? n : limit);
}
size_t carve(char* base, int64_t T, int64_t V, int D, int planes, FewWork& o) {
  o.group = few_fit(T, D, planes);
  o.groups = static_cast<int>((T + o.group - 1) / o.group);
  // two workgroups to a CU where LDS holds them; 128 entries each at least
  const int64_t lds = static_cast<int64_t>(o.group) * few_row(D) * planes * 2;
  const int64_t most = (lds > (72 << 10) ? kGrid : kFewBlocks) / (o.groups < 8 ? 1 : o.groups / 4);
  const int64_t blocks = (V + 15) / 16;
  o.waves = few_waves(blocks, std::max<int64_t>(1, (lds > (72 << 10) ? kGrid : kFewBlocks) / std::max(1, o.groups)), kFewWaves);
  // several groups of tokens: four at least, since each workgroup lays out its tokens (512 x 1000 x 64 fp32 with 1, 4 and
  // 8: 12.0, 10.6 and 10.7 us; 300 x 1000 x 512 fp32 17.1, 17.1 and 20.3)
  if (o.groups > 1) o.waves = std::max(o.waves, 4);
  o.across = static_cast<int>(grid_for((blocks + o.waves - 1) / o.waves, most > 0 ? most : 1));
  Carver c{base};
  o.at_target = c.take<float>(static_cast<size_t>(o.groups) * kFew);
  o.partials = c.take<float>(static_cast<size_t>(o.groups) * o.across * 3 * kFew);
  return c.size();
}

template <typename T, int kPlanes>
void loss_few_call(const LossArgs& a, hipStream_t stream) {
  FewWork w;
  carve(static_cast<char*>(a.workspace), a.T, a.V, a.D, kPlanes, w);
  const size_t lds = static_cast<size_t>(w.group) * few_row(a.D) * kPlanes * 2;
  const auto launch = [&](auto tok, auto smooth) {
    loss_few_kernel<T, kPlanes, tok.value, smooth.value><<<dim3(w.across, w.groups), kFewThreads, lds, stream>>>(
        w.waves, static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.table), a.ldw, static_cast<int>(a.T), a.V, a.D, a.targets,
        w.at_target, w.partials, a.status);
  };
  with_tokens(w.group, [&](auto tok) {
    if (a.smoothing > 0.0f)
      launch(tok, std::true_type{});
    else
      launch(tok, std::false_type{});
  });
  loss_few_join_kernel<<<static_cast<unsigned>(a.T), kWave, 0, stream>>>(w.across, w.group, a.V, a.targets, w.at_target,
                                                                         w.partials, a.smoothing, a.loss, a.lse);
}

template <typename T, int kPlanes>
void loss_call(const LossArgs& a, bool direct, hipStream_t stream) {
  const Sizes s = sizes_of(a.T, a.V, a.D, kPlanes == 1, direct, false);
  Forward w;
  carve(static_cast<char*>(a.workspace), s, a.T, w);
  const T* table = static_cast<const T*>(a.table);
  pick_kernel<<<1, kPickThreads, 0, stream>>>(a.targets, a.T, a.V, static_cast<int>(s.piece / kTile), 0, 1, 1,
                                              static_cast<int>(kMostUnits), w.list, w.slot_of, w.plan, a.status);
  const PackJob<T> rows{static_cast<const T*>(a.x), a.ldx, w.list, w.plan, a.T, s.Tp / kSquare,
                        Packed{w.x, s.Tp * s.Kp, s.Kp}, Packed{}, nullptr};
  if (direct) pack<T, kPlanes>(rows, PackJob<T>{}, s, a.D, stream);
  const Operand X{w.x, s.Tp * s.Kp, s.Kp, static_cast<int>(s.Tp)};
  for (int p = 0; p < s.pieces; ++p) {
    const int64_t v0 = p * s.piece;
    const int count = static_cast<int>(a.V - v0 < s.piece ? a.V - v0 : s.piece);
    Operand W{w.w, s.piece * s.Kp, s.Kp, static_cast<int>(s.piece)};
    if (direct)
      W = Operand{reinterpret_cast<const uint16_t*>(table), 0, a.ldw, static_cast<int>(a.V)};
    else
      pack<T, kPlanes>(p == 0 ? rows : PackJob<T>{},
                       PackJob<T>{table + v0 * a.ldw, a.ldw, nullptr, nullptr, count, round_up(count, kTile) / kSquare,
                                  Packed{w.w, s.piece * s.Kp, s.Kp}, Packed{}, nullptr},
                       s, a.D, stream);
    const auto kernel = a.smoothing > 0.0f ? loss_kernel<kPlanes, true> : loss_kernel<kPlanes, false>;
    kernel<<<kGrid, kThreads, 0, stream>>>(W, X, w.plan, static_cast<int>(s.Kp), v0, count, a.targets, w.list, w.at_target,
                                           w.partials + p * w.piece_stride);
  }
  const int per = kPackThreads / kWave;
  for (int64_t b = 0; b < a.T; b += per * kMaxBlocks)
    loss_join_kernel<<<grid_for((a.T - b + per - 1) / per, kMaxBlocks), kPackThreads, 0, stream>>>(
        w.plan, w.slot_of, b, a.T, a.V, s.pieces, w.piece_stride, w.at_target, w.partials, a.smoothing, a.loss, a.lse);
}

template <typename F>
void with_width(int wn, F&& f) {
  if (wn == 4)
    f(std::integral_constant<int, 4>{});
  else if (wn == 2)
    f(std::integral_constant<int, 2>{});
  else
    f(std::integral_constant<int, 1>{});
}

struct FewGradWork {
  uint16_t* g;
  float* parts;
  int64_t ldg;
  int nparts, slices;
};
size_t carve(char* base, int64_t T, int64_t V, int D, int planes, FewGradWork& o) {
  const int n = few_tokens(T);
  o.ldg = round_up(V, 32);
  o.slices = (D + (planes == 1 ? 128 : 64) - 1) / (planes == 1 ? 128 : 64);
  // a wave to 64 entries, up to one workgroup on each CU, or two where registers and LDS hold them
  const int64_t want = (V + 64 * kFewWaves - 1) / (64 * kFewWaves), most = (planes == 1 && n == 16 ? kFewBlocks : kGrid) / o.slices;
  o.nparts = static_cast<int>(std::max<int64_t>(1, std::min(want, most)));
  Carver c{base};
  o.g = c.take<uint16_t>((planes == 1 ? 2 : 3) * n * o.ldg);
  o.parts = c.take<float>(static_cast<size_t>(o.nparts) * T * D);
  return c.size();
}

template <typename T, int kPlanes>
void loss_grad_few_call(const LossGradArgs& a, hipStream_t stream) {
  FewGradWork w;
  carve(static_cast<char*>(a.workspace), a.T, a.V, a.D, kPlanes, w);
  const int n = few_tokens(a.T);
  const int64_t blocks = (a.V + 31) / 32 * 2;
  const int room = few_grad(a.T, a.V, a.D, kPlanes);
  const int64_t most = few_grad_lds(n, a.D, kPlanes, room) > (78 << 10) ? kGrid : kFewBlocks;
  const int takers = few_waves(blocks, most, room);
  const size_t lds = few_grad_lds(n, a.D, kPlanes, takers);
  const int grid = static_cast<int>(grid_for((blocks + takers - 1) / takers, most));
  const T* table = static_cast<const T*>(a.table);
  with_tokens(n, [&](auto tok) {
    few_grad_kernel<T, kPlanes, tok.value><<<grid, kFewThreads, lds, stream>>>(
        takers, static_cast<const T*>(a.x), a.ldx, table, a.ldw, static_cast<int>(a.T), a.V, a.D, a.targets, a.lse, a.dloss,
        a.dloss_step, a.smoothing, a.dx != nullptr ? w.g : nullptr, w.ldg, static_cast<T*>(a.dtable), a.lddt, a.status);
    if (a.dx == nullptr) return;
    few_rows_kernel<T, kPlanes, tok.value><<<w.nparts * w.slices, kFewThreads, 0, stream>>>(
        w.g, w.ldg, table, a.ldw, static_cast<int>(a.T), a.V, a.D, w.slices, w.parts);
  });
  if (a.dx != nullptr)
    few_rows_join_kernel<T><<<dim3((a.D + 31) / 32, static_cast<unsigned>(a.T)), 1024, 0, stream>>>(
        w.parts, w.nparts, static_cast<int>(a.T), a.D, a.V, a.targets, static_cast<T*>(a.dx), a.lddx);
}

template <typename T, int kPlanes>
void loss_grad_call(const LossGradArgs& a, bool direct, hipStream_t stream) {
  const Sizes s = sizes_of(a.T, a.V, a.D, kPlanes == 1, direct, true);
  Backward w;
  carve(static_cast<char*>(a.workspace), s, a.T, w);
  const T* table = static_cast<const T*>(a.table);
  const float* factors = a.dloss_step != 0 ? a.dloss : nullptr;                   // each token's own
  const float* factor = a.dloss_step == 0 && a.T > 0 ? a.dloss : nullptr;         // one for all
  const int nd = static_cast<int>(s.Dp / (64 * s.wn)), Kp = static_cast<int>(s.Kp);
  pick_kernel<<<1, kPickThreads, 0, stream>>>(a.targets, a.T, a.V, 0, static_cast<int>(s.piece / kStep), nd,
                                              static_cast<int>(s.piece / kTile) * nd,
                                              static_cast<int>(kMostParts), w.list, w.slot_of, w.plan, a.status);
  const PackJob<T> tokens{static_cast<const T*>(a.x), a.ldx, w.list, w.plan, a.T, s.Tp / kSquare,
                          Packed{w.x, s.Tp * s.Kp, s.Kp}, Packed{a.dtable != nullptr ? w.xt : nullptr, s.Dp * s.Tp, s.Tp},
                          factors};
  const bool lay_out = !direct || a.dx != nullptr;
  if (!lay_out) pack<T, kPlanes>(tokens, PackJob<T>{}, s, a.D, stream);
  const Operand X{w.x, s.Tp * s.Kp, s.Kp, static_cast<int>(s.Tp)};
  const Operand Xt{w.xt, s.Dp * s.Tp, s.Tp, Kp};
  for (int p = 0; p < s.pieces; ++p) {
    const int64_t v0 = p * s.piece;
    const int count = static_cast<int>(a.V - v0 < s.piece ? a.V - v0 : s.piece), rows = static_cast<int>(round_up(count, kTile));
    Operand W{w.w, s.piece * s.Kp, s.Kp, static_cast<int>(s.piece)};
    if (direct) W = Operand{reinterpret_cast<const uint16_t*>(table) + v0 * a.ldw, 0, a.ldw, count};
    if (lay_out)
      pack<T, kPlanes>(p == 0 ? tokens : PackJob<T>{},
                       PackJob<T>{table + v0 * a.ldw, a.ldw, nullptr, nullptr, count, rows / kSquare,
                                  Packed{direct ? nullptr : w.w, s.piece * s.Kp, s.Kp},
                                  Packed{a.dx != nullptr ? w.wt : nullptr, s.Dp * s.piece, s.piece}, nullptr},
                       s, a.D, stream);
    grad_logits_kernel<kPlanes><<<kGrid, kThreads, 0, stream>>>(
        W, X, w.plan, Kp, a.V, v0, count, a.targets, w.list, a.lse, factors, a.smoothing,
        Packed{w.g, s.Tp * w.g_ld, w.g_ld});
    const Operand G{w.g, s.Tp * w.g_ld, w.g_ld, static_cast<int>(s.Tp)};
    if (a.dtable != nullptr) {
      T* out = static_cast<T*>(a.dtable) + v0 * a.lddt;
      with_width(s.wn, [&](auto wn) {
        grad_table_kernel<T, kPlanes, wn.value><<<kGrid, kThreads, 0, stream>>>(G, Xt, w.plan, nd, count, a.D, out, a.lddt,
                                                                                w.table_parts, s.Dp, factor);
      });
      if (w.table_parts != nullptr) {
        const int nvec = (a.D + 7) / 8;
        grad_table_join_kernel<T><<<static_cast<unsigned>((static_cast<int64_t>(count) * nvec + kPackThreads - 1) / kPackThreads),
                                    kPackThreads, 0, stream>>>(w.plan, count, a.D, nvec, w.table_parts, s.Dp, factor, out,
                                                  a.lddt);
      }
    }
    if (a.dx != nullptr)
      with_width(s.wn, [&](auto wn) {
        grad_rows_kernel<kPlanes, wn.value><<<kGrid, kThreads, 0, stream>>>(
            G, Operand{w.wt, s.Dp * s.piece, s.piece, Kp}, w.plan, nd, rows, p == 0, w.parts);
      });
  }
  if (a.dx != nullptr && a.T > 0) {
    const int64_t tokens_blocks = s.Tp / kTile * nd * 8 * s.wn, others = (a.T + kThreads / 8 - 1) / (kThreads / 8);
    with_width(s.wn, [&](auto wn) {
      for (int64_t b = 0; b < tokens_blocks + others; b += kMaxBlocks)
        grad_rows_join_kernel<T, wn.value><<<grid_for(tokens_blocks + others - b, kMaxBlocks), kThreads, 0, stream>>>(
            b, w.plan, w.list, w.slot_of, tokens_blocks, a.T, a.D, nd, w.parts, a.dloss, a.dloss_step,
            static_cast<T*>(a.dx), a.lddx);
    });
  }
}

// Whether the products may read the table where it stands: rows of whole steps on 16-byte boundaries.
bool read_direct(const void* table, int64_t ld, int D, bool is_bf16) {
  return is_bf16 && D % kStep == 0 && ld % 8 == 0 && ld < (1 << 22) && reinterpret_cast<uintptr_t>(table) % 16 == 0;
}

}  // namespace

size_t loss_workspace_bytes(int64_t T, int64_t V, int D, bool is_bf16) {
  if (few(T, V, D, is_bf16 ? 1 : 3)) {
    FewWork w;
    return carve(nullptr, T, V, D, is_bf16 ? 1 : 3, w);
  }
  Forward w;
  return carve(nullptr, sizes_of(T, V, D, is_bf16, false, false), T, w);
}

hipError_t launch_loss(const LossArgs& a, hipStream_t stream) {
  if (a.T == 0) return hipSuccess;
  if (few(a.T, a.V, a.D, a.is_bf16 ? 1 : 3)) {
    a.is_bf16 ? loss_few_call<bf16, 1>(a, stream) : loss_few_call<float, 3>(a, stream);
    return hipGetLastError();
  }
  const bool direct = read_direct(a.table, a.ldw, a.D, a.is_bf16);
  a.is_bf16 ? loss_call<bf16, 1>(a, direct, stream) : loss_call<float, 3>(a, direct, stream);
  return hipGetLastError();
}

size_t loss_grad_workspace_bytes(int64_t T, int64_t V, int D, bool is_bf16) {
  if (T > 0 && few_grad(T, V, D, is_bf16 ? 1 : 3) > 0) {
    FewGradWork w;
    return carve(nullptr, T, V, D, is_bf16 ? 1 : 3, w);
  }
  Backward w;
  return carve(nullptr, sizes_of(T, V, D, is_bf16, false, true), T, w);
}

hipError_t launch_loss_grad(const LossGradArgs& a, hipStream_t stream) {
  if (a.T > 0 && few_grad(a.T, a.V, a.D, a.is_bf16 ? 1 : 3) > 0) {
    a.is_bf16 ? loss_grad_few_call<bf16, 1>(a, stream) : loss_grad_few_call<float, 3>(a, stream);
    return hipGetLastError();
  }
  const bool direct = read_direct(a.table, a.ldw, a.D, a.is_bf16);
  a.is_bf16 ? loss_grad_call<bf16, 1>(a, direct, stream) : loss_grad_call<float, 3>(a, direct, stream);
  return hipGetLastError();
}

}  // namespace emb
