// The read-out of a 4-bit rollout policy: logits from hidden states and output embedding that are both MXFP4 rows,
//   out[t, v] = sum over blocks b of 2^(e_t,b + e_v,b) sum_i h[t, b, i] w[v, b, i].
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 rows of the embedding with 16 tokens over four blocks of 32 elements and
// applies both scales: a lane holds one block (16 bytes) of row lane % 16 and the byte of its scale.  Which four blocks go
// together is free as long as both operands agree.  The embedding is the first operand: a lane of the result then has four
// consecutive logits of one token.
#include "ais_internal.h"
#include "device_utils.h"

#include <algorithm>
#include <type_traits>

namespace ais {
namespace {

using namespace dev;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef const __attribute__((address_space(1))) void* glb_ptr;

constexpr int kFp4 = 4;                // the instruction's code of the E2M1 format
constexpr int kGroup = 16;             // blocks whose scales are one 16-byte vector

// c += w h over four blocks, the scales in the words' low bytes.
__device__ __forceinline__ void multiply(f32x4& c, i32x4 w, uint32_t w_scale, i32x4 h, uint32_t h_scale) {
  const i32x8 x = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, y = {h[0], h[1], h[2], h[3], 0, 0, 0, 0};
  c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, kFp4, kFp4, 0, (int)w_scale, 0, (int)h_scale);
}

constexpr int kRowBytes = 128;         // of a slice of eight blocks
// Chunk c (of 16 bytes) of a slice's row lies in LDS at position c ^ swizzle(row): the 16 rows that a fragment read touches lie in
// different 16-byte bank groups.  The rows of a fragment are consecutive ones of the hidden states; in the tile kernel those of
// the embedding are four fours, eight apart (see tile_entry).
__device__ __forceinline__ int swizzle_h(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int swizzle_w(int row) { return (row >> 1 & 1) | (row >> 2 & 6); }

// ---- few rows ---------------------------------------------------------------------------------------------------------
// A decode step reads the whole embedding for a few tokens: 17 bytes a block from HBM, and next to nothing else.  One workgroup
// on every compute unit walks through its share of the vocabulary, 16 entries at a time, with all of LDS as a ring of what is on
// its way.  Its four wavefronts have a quarter of the contraction each, whose hidden states stay in registers.  A wavefront
// copies and awaits its own share of the embedding, whole lines of 128 bytes, and nobody else's; the four sums of a tile meet
// in LDS, and the wavefronts take turns in writing them out.  Bound by reading: 16 rows x 151,936 x 4,096 58 us, 331 MB at 5.7
// TB/s (a sum over 4 GiB reads 6.1).
constexpr int kStreamThreads = 256;
constexpr int kStreamWaves = kStreamThreads / 64;

// NT: tiles of 16 tokens, which hold all rows; GPW: groups of 16 blocks of each wavefront.
template <int NT, int GPW>
struct StreamLds {
  static constexpr int kCodes = GPW * 16 * 2 * kRowBytes;                       // of 16 rows: [group][half][row][128]
  static constexpr int kSlot = kCodes + GPW * 16 * kGroup;                      // and their scales: [group][row][16]
  static constexpr int kCopies = 5 * GPW;                                       // instructions that fill a slot
  static constexpr int kSums = 2 * kStreamWaves * NT * 1024;
  // as many slots as LDS holds; vmcnt counts to 63
  static constexpr int kRoom = (160 * 1024 - kSums) / (kStreamWaves * kSlot), kCount = 63 / kCopies + 1;
  static constexpr int kDepth = kRoom < 8 ? (kRoom < kCount ? kRoom : kCount) : (kCount < 8 ? kCount : 8);
  static_assert(kDepth >= 2, "the next tile is on its way while one is multiplied");
  static constexpr int kRing = kStreamWaves * kDepth * kSlot;
  static constexpr int kBytes = kRing + kSums;
};

template <typename O, int NT, int GPW>
__global__ __launch_bounds__(kStreamThreads) __attribute__((amdgpu_waves_per_eu(1, 1))) void mxfp4_stream_kernel(
    Mxfp4Rows hidden, int n_rows, Mxfp4Rows weight, int vocab, int blocks, O* __restrict__ out, long long out_stride) {
  typedef StreamLds<NT, GPW> L;
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4;
  const int n_tiles = (vocab + 15) / 16;
  const int tile0 = (int)((long long)n_tiles * blockIdx.x / gridDim.x), tile1 = (int)((long long)n_tiles * (blockIdx.x + 1) / gridDim.x);
  if (tile0 >= tile1) return;
  const int block0 = wave * GPW * kGroup;                      // of the wavefront's quarter
  unsigned char* ring = lds + wave * L::kDepth * L::kSlot;
  f32x4* part = reinterpret_cast<f32x4*>(lds + L::kRing);      // [2][wave][NT][lane]

  // ---- the hidden states: in step s of a group lane l has block 4 s + l / 16, whose scale is byte l / 16 of word s.  Blocks beyond
  // a row's end are the last one again, on both sides: codes are finite numbers, and two scales of 2^-127 leave nothing of them.
  i32x4 h[GPW][NT][4];
  uint32_t hs[GPW][NT][4];
#pragma unroll
  for (int g = 0; g < GPW; ++g)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const long long row = min(j * 16 + (lane & 15), n_rows - 1);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int b = block0 + g * kGroup + 4 * s + quarter;
        h[g][j][s] = *reinterpret_cast<const i32x4*>(hidden.codes + row * hidden.codes_stride + 16LL * min(b, blocks - 1));
        hs[g][j][s] = b < blocks ? hidden.scales[row * hidden.scales_stride + b] : 0u;
      }
    }
  uint32_t keep[GPW][4];                                       // of a word of the embedding's scales
#pragma unroll
  for (int g = 0; g < GPW; ++g)
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int left = blocks - (block0 + g * kGroup + 4 * s);
      keep[g][s] = left >= 4 ? ~0u : left > 0 ? (1u << 8 * left) - 1 : 0u;
    }

  // ---- copies: eight rows of a slice to an instruction, a lane the chunk that lies at its place
  const int crow = lane >> 3;
  auto copy = [&](int tile, int slot) {
    unsigned char* to = ring + slot * L::kSlot;
    const int v0 = tile * 16;
#pragma unroll
    for (int g = 0; g < GPW; ++g) {
      unsigned char* codes = to + g * 16 * 2 * kRowBytes;
      if (block0 + g * kGroup < blocks) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int row = 8 * (k & 1) + crow, b = block0 + g * kGroup + 8 * (k >> 1) + ((lane & 7) ^ swizzle_h(row));
          const unsigned char* src =
              weight.codes + (long long)min(v0 + row, vocab - 1) * weight.codes_stride + 16LL * min(b, blocks - 1);
          __builtin_amdgcn_global_load_lds((glb_ptr)src, (lds_ptr)(codes + k * 8 * kRowBytes), 16, 0, 2 /* non-temporal */);
        }
      } else {                                                 // nothing there: as many instructions, of a line that is at hand
#pragma unroll
        for (int k = 0; k < 4; ++k)
          __builtin_amdgcn_global_load_lds((glb_ptr)hidden.codes, (lds_ptr)(codes + k * 8 * kRowBytes), 16, 0, 0);
      }
    }
#pragma unroll
    for (int g = 0; g < GPW; ++g) {
      const int b = block0 + g * kGroup + 4 * (lane & 3);
      const unsigned char* src = weight.scales + (long long)min(v0 + (lane >> 2), vocab - 1) * weight.scales_stride +
                                 min(b, (blocks - 1) & ~3);
      __builtin_amdgcn_global_load_lds((glb_ptr)src, (lds_ptr)(to + L::kCodes + g * 16 * kGroup), 4, 0, 0);
    }
  };
#pragma unroll
  for (int d = 0; d < L::kDepth; ++d) copy(min(tile0 + d, tile1 - 1), d);
  const int a = lane & 15;
  int slot = 0, turn = 0;
  for (int tile = tile0; tile < tile1; ++tile) {
    // the copies into this slot are the oldest ones; stores on their way only make the wait longer
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((L::kDepth - 1) * L::kCopies) : "memory");
    const unsigned char* from = ring + slot * L::kSlot;
    f32x4 c[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) c[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    i32x4 w[GPW][4];
    uint32_t ws[GPW][4];
#pragma unroll
    for (int g = 0; g < GPW; ++g) {
      const u32x4 words = *reinterpret_cast<const u32x4*>(from + L::kCodes + (g * 16 + a) * kGroup);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        w[g][s] = *reinterpret_cast<const i32x4*>(from + ((g * 2 + (s >> 1)) * 16 + a) * kRowBytes +
                                                  ((((s & 1) * 4 + quarter) ^ swizzle_h(a)) << 4));
        ws[g][s] = (words[s] & keep[g][s]) >> (8 * quarter);
      }
    }
#pragma unroll
    for (int g = 0; g < GPW; ++g)
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int j = 0; j < NT; ++j) multiply(c[j], w[g][s], ws[g][s], h[g][j][s], hs[g][j][s]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the slot has been read
    copy(min(tile + L::kDepth, tile1 - 1), slot);              // beyond the last tile: once more, for nobody
    f32x4* mine = part + (turn & 1) * kStreamWaves * NT * 64;
#pragma unroll
    for (int j = 0; j < NT; ++j) mine[(wave * NT + j) * 64 + lane] = c[j];
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    // The buffer is written again two tiles on, behind the next barrier, which the wavefront that reads it now reaches afterwards.
    if ((turn & (kStreamWaves - 1)) == wave) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        f32x4 z = mine[j * 64 + lane];
#pragma unroll
        for (int p = 1; p < kStreamWaves; ++p) z += mine[(p * NT + j) * 64 + lane];
        const int t = j * 16 + a, v = tile * 16 + 4 * quarter;
        if (t >= n_rows) continue;
        O* o = out + (long long)t * out_stride + v;
        if (v + 4 <= vocab) {
          const float x[8] = {z[0], z[1], z[2], z[3]};
          const u32x4 q = Vec<O>::pack(x);
          if constexpr (sizeof(O) == 4)
            *reinterpret_cast<typename Unaligned<O>::four*>(o) = q;
          else
            *reinterpret_cast<typename Unaligned<O>::two*>(o) = {q[0], q[1]};
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (v + e < vocab) Vec<O>::store1(o + e, z[e]);
        }
      }
    }
    slot = slot + 1 == L::kDepth ? 0 : slot + 1;
    ++turn;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // copies for nobody land before the LDS is given back
}

// ---- many rows ----------------------------------------------------------------------------------------------------------
// Tiles of 256 entries of the vocabulary x 64 NJ tokens, eight wavefronts, two along the vocabulary x four along the tokens,
// 128 x 16 NJ logits each.  A step covers eight blocks: 128 bytes, a whole line, of every row, copied straight from global
// memory into one of two LDS buffers; the copies of the next step are on their way while a step is multiplied.  Scales come
// for two steps at a time.  A workgroup walks through its tiles without a pause: the first step of the next tile is copied during
// the last of this one.
// 2,048 rows x 151,936 x 4,096 745 us, 3.4 PFLOP/s.  There copies and LDS reads without the products take 520 us, products and LDS
// reads without the copies 502 (the instructions by themselves 253), and the stores, which all workgroups make at about the same
// time, 115.
//
// The products are written as instructions: the compiler's own form of one may be moved past barriers and waits, and the
// fragments and accumulators of a whole step with it.  It does not know what such a statement is, so what it would wait for is
// waited for here: wait() stands between an ordinary instruction that writes an operand and the products, and settle()
// between the products and the first look at their sums.  Fragments come from LDS reads, whose arrival it does wait for.
// c += w h over four blocks, the scales in byte S of the words.
template <int S>
__device__ __forceinline__ void product(f32x4& c, i32x4 w, uint32_t w_scale, i32x4 h, uint32_t h_scale) {
  if constexpr (S == 0)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                 : "+a"(c) : "v"(w), "v"(h), "v"(w_scale), "v"(h_scale));
  if constexpr (S == 1)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                 : "+a"(c) : "v"(w), "v"(h), "v"(w_scale), "v"(h_scale));
  if constexpr (S == 2)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[1,1,0] cbsz:4 blgp:4"
                 : "+a"(c) : "v"(w), "v"(h), "v"(w_scale), "v"(h_scale));
  if constexpr (S == 3)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[1,1,0] cbsz:4 blgp:4"
                 : "+a"(c) : "v"(w), "v"(h), "v"(w_scale), "v"(h_scale));
}
__device__ __forceinline__ void wait() { asm volatile("s_nop 7"); }
__device__ __forceinline__ void settle() { asm volatile("s_nop 15\n\ts_nop 3"); }

constexpr int kTileThreads = 512;
constexpr int kTileV = 256;
constexpr int kNI = 8;                                        // MFMA tiles of a wavefront along the vocabulary
constexpr int kAhead = 2;
constexpr int kStepBlocks = 8;

// First of the four entries, inside the wavefront's 128, that MFMA tile i leaves in a lane of this quarter: two tiles are 32
// entries, eight consecutive ones to a lane.
__device__ __forceinline__ int tile_entry(int i, int quarter) { return 32 * (i >> 1) + 8 * quarter + 4 * (i & 1); }

struct TilePlan {
  int n_vtiles, n_ttiles, group, per_xcd, n_items;            // tiles of tokens that walk the vocabulary together; items of an XCD
};

template <int NJ>
struct TileLds {
  static constexpr int kTileT = 64 * NJ;
  static constexpr int kW = 0, kH = 2 * kTileV * kRowBytes;                     // two slices of each
  static constexpr int kScales = kH + 2 * kTileT * kRowBytes;                   // two groups of 16 bytes for each row
  static constexpr int kScaleCopies = (kTileV + kTileT + 127) / 128;            // instructions of each wavefront, 128 rows in all
  static constexpr int kScaleBytes = 128 * kScaleCopies * kGroup;
  static constexpr int kBytes = kScales + 2 * kScaleBytes;
};

// What the last group of a row's blocks holds: all 16, nine or more, or no more than eight, which are a step by themselves.
enum Tail { kWhole, kLong, kShort };

template <typename O, int NJ, Tail TAIL>
__global__ __launch_bounds__(kTileThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void mxfp4_tile_kernel(
    Mxfp4Rows hidden, int n_rows, Mxfp4Rows weight, int vocab, int blocks, TilePlan plan, O* __restrict__ out,
    long long out_stride) {
  typedef TileLds<NJ> L;
  constexpr bool RAGGED = TAIL != kWhole;
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4;
  const int wv = wave & 1, wt = wave >> 1;
  // workgroups are dealt to the XCDs in turns; each XCD has a range of items of its own, which its workgroups take in turns
  const int xcd = blockIdx.x & 7, local = blockIdx.x >> 3, locals = gridDim.x >> 3;
  const int item0 = xcd * plan.per_xcd + local, item_end = min((xcd + 1) * plan.per_xcd, plan.n_items);
  if (item0 >= item_end) return;
  auto place = [&](int item, int& v0, int& t0) {
    const int per_group = plan.group * plan.n_vtiles;
    const int g = item / per_group, j = item - g * per_group;
    const int size = min(plan.group, plan.n_ttiles - g * plan.group);
    const int v = j / size;
    v0 = v * kTileV;
    t0 = (g * plan.group + (j - v * size)) * L::kTileT;
  };

  // ---- copies: a wavefront moves rows 8 wave .. 8 wave + 7 (+ 64 q) of a slice, a lane the chunk that lies at lane % 8.
  // Scales: 16 rows of four words to an instruction, the rows of both operands numbered in one go.  Offsets are from the tile's
  // first row, 32 bits.  Blocks beyond a row's end are its last one again: a code is always a finite number, and two scales of
  // 2^-127 leave nothing of it.
  constexpr int kScaleCopies = L::kScaleCopies;
  const unsigned char *w_base, *h_base, *ws_base, *hs_base;
  uint32_t w_off[4], h_off[NJ], s_off[kScaleCopies];
  auto point = [&](int item) {
    int v0, t0;
    place(item, v0, t0);
    const int lane = fresh_thread() & 63, crow = 8 * wave + (lane >> 3);
    w_base = weight.codes + (long long)v0 * weight.codes_stride;
    h_base = hidden.codes + (long long)t0 * hidden.codes_stride;
    ws_base = weight.scales + (long long)v0 * weight.scales_stride;
    hs_base = hidden.scales + (long long)t0 * hidden.scales_stride;
#pragma unroll
    for (int q = 0; q < 4; ++q) w_off[q] = (uint32_t)min(crow + 64 * q, vocab - 1 - v0) * (uint32_t)weight.codes_stride;
#pragma unroll
    for (int q = 0; q < NJ; ++q) h_off[q] = (uint32_t)min(crow + 64 * q, n_rows - 1 - t0) * (uint32_t)hidden.codes_stride;
#pragma unroll
    for (int q = 0; q < kScaleCopies; ++q) {
      const int row = 16 * wave + 128 * q, r = row + (lane >> 2);              // row: the wavefront's first
      s_off[q] = row < kTileV ? (uint32_t)min(r, vocab - 1 - v0) * (uint32_t)weight.scales_stride
                              : (uint32_t)min(r - kTileV, n_rows - 1 - t0) * (uint32_t)hidden.scales_stride;
    }
  };
  const int n_groups = (blocks + kGroup - 1) / kGroup;         // pairs of steps of a tile
  // the cursor of the copies
  int c_item = item0, c_group = 0;
  point(item0);
  auto copy_codes = [&](int half, int to) {                     // of step 2 c_group + half, into buffer `to`
    const int block = c_group * kGroup + half * kStepBlocks;
    const int lane = fresh_thread() & 63, crow = 8 * wave + (lane >> 3);
    const int w_chunk = (lane & 7) ^ swizzle_w(crow), h_chunk = (lane & 7) ^ swizzle_h(crow);
    const uint32_t wb = 16u * (uint32_t)(RAGGED ? min(block + w_chunk, blocks - 1) : block + w_chunk);
    const uint32_t hb = 16u * (uint32_t)(RAGGED ? min(block + h_chunk, blocks - 1) : block + h_chunk);
#pragma unroll
    for (int q = 0; q < 4; ++q)
      __builtin_amdgcn_global_load_lds((glb_ptr)(w_base + (w_off[q] + wb)),
                                       (lds_ptr)(lds + L::kW + to * kTileV * kRowBytes + (8 * wave + 64 * q) * kRowBytes), 16, 0, 0);
#pragma unroll
    for (int q = 0; q < NJ; ++q)
      __builtin_amdgcn_global_load_lds((glb_ptr)(h_base + (h_off[q] + hb)),
                                       (lds_ptr)(lds + L::kH + to * L::kTileT * kRowBytes + (8 * wave + 64 * q) * kRowBytes), 16, 0,
                                       0);
  };
  auto copy_scales = [&](int buffer) {
    const int word = c_group * kGroup + 4 * (fresh_thread() & 3);
    const uint32_t sb = (uint32_t)(RAGGED ? min(word, (blocks - 1) & ~3) : word);
#pragma unroll
    for (int q = 0; q < kScaleCopies; ++q) {
      const unsigned char* base = 16 * wave + 128 * q < kTileV ? ws_base : hs_base;
      __builtin_amdgcn_global_load_lds((glb_ptr)(base + (s_off[q] + sb)),
                                       (lds_ptr)(lds + L::kScales + buffer * L::kScaleBytes + (16 * wave + 128 * q) * kGroup), 4, 0, 0);
    }
  };
  // ---- fragments: in half step h lane takes chunk 2 quarter + h of its row, whose scale is byte 2 (quarter % 2) + h of word
  // quarter / 2 of the step's eight bytes
  const int a = lane & 15;
  const int arow = wv * 128 + 8 * (a >> 2) + (a & 3);          // tile i: + tile_entry(i, 0)
  const int brow = wt * 16 * NJ + a;
  // swizzles do not depend on the MFMA tile: a fragment lies at a constant distance from the first one
  const int w_at[2] = {arow * kRowBytes + ((2 * quarter ^ swizzle_w(arow)) << 4),
                       arow * kRowBytes + (((2 * quarter + 1) ^ swizzle_w(arow)) << 4)};
  const int h_at[2] = {brow * kRowBytes + ((2 * quarter ^ swizzle_h(brow)) << 4),
                       brow * kRowBytes + (((2 * quarter + 1) ^ swizzle_h(brow)) << 4)};

  f32x4 acc[kNI][NJ];
  copy_scales(0);
  copy_codes(0, 0);
  int scale_buffer = 0, buffer = 0;
  for (int item = item0; item < item_end; item += locals) {
#pragma unroll
    for (int i = 0; i < kNI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        asm volatile("" : "+a"(acc[i][j]));
      }
    wait();
    // A group of blocks: two steps, or one.  No branch inside: the compiler would move products across it, and accumulators with them.
    auto two_steps = [&](int g, auto last) __attribute__((always_inline)) {
      constexpr bool kLast = decltype(last)::value;
      constexpr int kHalves = kLast && TAIL == kShort ? 1 : 2;
      uint32_t ws[kNI], hs[NJ];
#pragma unroll
      for (int half = 0; half < kHalves; ++half) {
        // this step's copies, the only ones in flight, have landed everywhere, and nobody reads the step before any more
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (half + 1 < kHalves) {
          copy_codes(1, buffer ^ 1);
        } else {
          if constexpr (kLast) {                // on to the next tile; after the last one once more to its beginning
            c_group = 0;
            c_item = c_item + locals < item_end ? c_item + locals : c_item;
            point(c_item);
          } else {
            ++c_group;
          }
          copy_scales(scale_buffer ^ 1);
          copy_codes(0, buffer ^ 1);
        }
        if (half == 0) {
          const unsigned char* sl = lds + L::kScales + scale_buffer * L::kScaleBytes;
          const int lane = fresh_thread() & 63, quarter = lane >> 4, a = lane & 15;
          const int ws_at = (wv * 128 + 8 * (a >> 2) + (a & 3)) * kGroup + 4 * (quarter >> 1);
          const int hs_at = (kTileV + wt * 16 * NJ + a) * kGroup + 4 * (quarter >> 1);
          const uint32_t pick = (quarter & 1) ? 0x07060302u : 0x05040100u;
          // scales beyond the row's end count as zero
          uint32_t keep = ~0u;
          if (RAGGED) {
            const int left = blocks - g * kGroup - 2 * quarter;
            keep = (left > 0 ? 0xffu : 0u) | (left > 1 ? 0xff00u : 0u) | (left > 8 ? 0xff0000u : 0u) | (left > 9 ? 0xff000000u : 0u);
          }
#pragma unroll
          for (int i = 0; i < kNI; ++i) {
            const uint32_t* r = reinterpret_cast<const uint32_t*>(sl + ws_at + tile_entry(i, 0) * kGroup);
            ws[i] = __builtin_amdgcn_perm(r[2], r[0], pick) & keep;
          }
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            const uint32_t* r = reinterpret_cast<const uint32_t*>(sl + hs_at + 16 * j * kGroup);
            hs[j] = __builtin_amdgcn_perm(r[2], r[0], pick) & keep;
          }
#pragma unroll
          for (int i = 0; i < kNI; ++i) asm volatile("" : "+v"(ws[i]));
#pragma unroll
          for (int j = 0; j < NJ; ++j) asm volatile("" : "+v"(hs[j]));
          wait();
        }
        const unsigned char* wl = lds + L::kW + buffer * kTileV * kRowBytes;
        const unsigned char* hl = lds + L::kH + buffer * L::kTileT * kRowBytes;
        buffer ^= 1;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          // the embedding's fragments are read two MFMA tiles ahead
          i32x4 w[kAhead + 1], b[NJ];
          auto read_w = [&](int i) {
            w[i % (kAhead + 1)] = *reinterpret_cast<const i32x4*>(wl + w_at[h] + tile_entry(i, 0) * kRowBytes);
          };
#pragma unroll
          for (int j = 0; j < NJ; ++j) b[j] = *reinterpret_cast<const i32x4*>(hl + h_at[h] + 16 * j * kRowBytes);
#pragma unroll
          for (int i = 0; i < kAhead; ++i) read_w(i);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int i = 0; i < kNI; ++i) {
            if (i + kAhead < kNI) read_w(i + kAhead);
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
              const i32x4 x = w[i % (kAhead + 1)];
              if (half == 0 && h == 0) product<0>(acc[i][j], x, ws[i], b[j], hs[j]);
              if (half == 0 && h == 1) product<1>(acc[i][j], x, ws[i], b[j], hs[j]);
              if (half == 1 && h == 0) product<2>(acc[i][j], x, ws[i], b[j], hs[j]);
              if (half == 1 && h == 1) product<3>(acc[i][j], x, ws[i], b[j], hs[j]);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      scale_buffer ^= 1;
    };
    for (int g = 0; g + 1 < n_groups; ++g) two_steps(g, std::false_type{});
    two_steps(n_groups - 1, std::true_type{});
    // ---- the finished tile: eight consecutive logits of a token from every two MFMA tiles.  Rows of logits begin anywhere: element by
    // element 333 f32 rows x 50,257 x 1,100 took 94 us, in vectors at any multiple of an element 49.
    settle();
#pragma unroll
    for (int i = 0; i < kNI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) asm volatile("" : "+a"(acc[i][j]));
    int v0, t0;
    place(item, v0, t0);
    const int lane = fresh_thread() & 63, quarter = lane >> 4, brow = wt * 16 * NJ + (lane & 15);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int t = t0 + brow + 16 * j;
      if (t >= n_rows) continue;
      O* row = out + (long long)t * out_stride;
#pragma unroll
      for (int i = 0; i < kNI; i += 2) {
        const int v = v0 + wv * 128 + tile_entry(i, quarter);
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = acc[i + (e >> 2)][j][e & 3];
        if (v + 8 <= vocab) {
          constexpr int N = Vec<O>::N;
#pragma unroll
          for (int e = 0; e < 8; e += N) *reinterpret_cast<typename Unaligned<O>::four*>(row + v + e) = Vec<O>::pack(z + e);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (v + e < vocab) Vec<O>::store1(row + v + e, z[e]);
        }
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // copies for nobody land before the LDS is given back
}

template <typename O, int NJ, Tail TAIL>
int launch_tiles(ais_ctx* ctx, const Mxfp4Rows& hidden, int n_rows, const Mxfp4Rows& weight, int vocab, int blocks, O* out,
                 long long out_stride) {
  typedef TileLds<NJ> L;
  auto kernel = mxfp4_tile_kernel<O, NJ, TAIL>;
  static std::once_flag once[kMaxDevices];
  static bool ok[kMaxDevices];
  if (!allow_dynamic_lds(ctx, reinterpret_cast<const void*>(kernel), L::kBytes, once, ok))
    return hip_fail(ctx, hipErrorInvalidValue);
  TilePlan plan;
  plan.n_vtiles = (vocab + kTileV - 1) / kTileV;
  plan.n_ttiles = (n_rows + L::kTileT - 1) / L::kTileT;
  plan.group = plan.n_ttiles < 8 ? plan.n_ttiles : 8;
  const long long items = (long long)plan.n_vtiles * plan.n_ttiles;
  if (items > 0x7fffffffLL - 8) return AIS_ERR_SIZE;
  plan.n_items = (int)items;
  plan.per_xcd = (plan.n_items + 7) / 8;
  const int locals = plan.per_xcd < (ctx->n_cus + 7) / 8 ? plan.per_xcd : (ctx->n_cus + 7) / 8;
  kernel<<<dim3((unsigned)(8 * locals)), dim3(kTileThreads), L::kBytes, ctx->stream>>>(hidden, n_rows, weight, vocab, blocks, plan,
                                                                                      out, out_stride);
  return hip_fail(ctx, hipGetLastError());
}

template <typename O, int NT, int GPW>
int launch_stream(ais_ctx* ctx, const Mxfp4Rows& hidden, int n_rows, const Mxfp4Rows& weight, int vocab, int blocks, O* out,
                  long long out_stride) {
  auto kernel = mxfp4_stream_kernel<O, NT, GPW>;
  constexpr int kBytes = StreamLds<NT, GPW>::kBytes;
  static std::once_flag once[kMaxDevices];
  static bool ok[kMaxDevices];
  if (!allow_dynamic_lds(ctx, reinterpret_cast<const void*>(kernel), kBytes, once, ok)) return hip_fail(ctx, hipErrorInvalidValue);
  const int tiles = (vocab + 15) / 16;
  kernel<<<dim3((unsigned)std::min(tiles, ctx->n_cus)), dim3(kStreamThreads), kBytes, ctx->stream>>>(hidden, n_rows, weight, vocab, blocks, out, out_stride);
  return hip_fail(ctx, hipGetLastError());
}

template <typename O>
int launch_typed(ais_ctx* ctx, const Mxfp4Rows& hidden, int n_rows, const Mxfp4Rows& weight, int vocab, int blocks, O* out,
                 long long out_stride) {
  const int groups = (blocks + kGroup - 1) / kGroup;
  // Few rows of long contractions: the stream.  A tile of it costs the same however short its quarters are, and 64 rows want
  // twice the registers of 32.  us, stream and tiles, with the quantisation of the hidden states, the embedding not in any cache:
  // 16 rows x 151,936 x 512 24 and 16, x 1,024 26 and 26, x 4,096 61 and 79, 16 x 50,257 x 1,100 15 and 16; 4 x 32,000 x 2,048 14 and 16,
  // x 4,096 (one row) 19 and 26; 32 x 151,936 x 1,024 32 and 27, x 2,048 39 and 45, x 4,096 67 and 85, x 8,192 120 and 176; 64 x
  // 50,304 x 2,048 25 and 20, x 151,936 x 2,048 49 and 48, x 4,096 77 and 91, x 64,000 x 4,096 40 and 36.
  auto stream = [&](auto nt, auto gpw) {
    return launch_stream<O, decltype(nt)::value, decltype(gpw)::value>(ctx, hidden, n_rows, weight, vocab, blocks, out, out_stride);
  };
  typedef std::integral_constant<int, 1> One;
  typedef std::integral_constant<int, 2> Two;
  typedef std::integral_constant<int, 3> Three;
  typedef std::integral_constant<int, 4> Four;
  if (n_rows <= 32 && groups >= 4 && groups <= 16) {
    auto rows = [&](auto nt) {
      return groups <= 4 ? stream(nt, One{}) : groups <= 8 ? stream(nt, Two{}) : groups <= 12 ? stream(nt, Three{}) : stream(nt, Four{});
    };
    return n_rows <= 16 ? rows(One{}) : rows(Two{});
  }
  if (n_rows <= 64 && groups > 4 && groups <= 8) return stream(Four{}, Two{});
  const int tail = blocks % kGroup;
  auto tiles = [&](auto nj) {
    constexpr int NJ = decltype(nj)::value;
    auto run = [&](auto kind) {
      return launch_tiles<O, NJ, decltype(kind)::value>(ctx, hidden, n_rows, weight, vocab, blocks, out, out_stride);
    };
    if (tail == 0) return run(std::integral_constant<Tail, kWhole>{});
    return tail > kStepBlocks ? run(std::integral_constant<Tail, kLong>{}) : run(std::integral_constant<Tail, kShort>{});
  };
  // Tiles of 64, 128 or 256 tokens take about 4 : 5 : 8 of time each (x 4,096: 20, 25 and 42 us), and every compute unit one at a
  // time: what comes out least, the larger ones where that is equal.  us with tiles of 64, 128 and 256: 70 rows x 50,257 x 1,024
  // 21, 16 and 18; 130 x 151,936 x 4,096 153, 130 and 118; 333 x 151,936 x 2,048 147, 106 and 107; 520 x 50,257 x 4,096 156, 112 and
  // 124; 1,000 x 2,000 x 2,048 15, 18 and 23; 2,048 x 32,000 x 4,096 331, 214 and 162.
  auto time = [&](int nj, long long each) {
    const long long items = (long long)((vocab + kTileV - 1) / kTileV) * ((n_rows + 64 * nj - 1) / (64 * nj));
    return ((items + ctx->n_cus - 1) / ctx->n_cus) * each;
  };
  const long long one = time(1, 4), two = time(2, 5), four = time(4, 8);
  if (four <= two && four <= one) return tiles(Four{});
  return two <= one ? tiles(Two{}) : tiles(One{});
}

}  // namespace

int launch_mxfp4_logits(ais_ctx* ctx, const Mxfp4Rows& hidden, int n_rows, const Mxfp4Rows& weight, int vocab, int blocks,
                        void* out, ais_dtype out_dtype, long long out_stride) {
  if (n_rows == 0) return AIS_OK;
  ScopedTimer timer(ctx, AIS_K_MXFP4_LOGITS);
  if (out_dtype == AIS_BF16)
    return launch_typed(ctx, hidden, n_rows, weight, vocab, blocks, static_cast<bf16_t*>(out), out_stride);
  return launch_typed(ctx, hidden, n_rows, weight, vocab, blocks, static_cast<float*>(out), out_stride);
}

}  // namespace ais
