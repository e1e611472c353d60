// Attention of many query rows over the paged 4-bit cache (offq_paged_attention where a sequence brings more
// than 16 rows n * Hq / H per key head: chunks of a prompt, whole prompts, long drafts) on the tensor cores.
//
// A row is one query of one head; the rows of a sequence and key head are taken 256 at a time (two tiles of
// 128) against blocks of 128 cached tokens, as in the prompt kernel: scores, weights and outputs stay in
// tensor memory. What differs:
//   * The codes become operands here. Four warps read codes and (scale, offset) pairs of the next block into
//     registers, widen them to exact 16-bit floats (keys as 16 + u, values as q) and store them as swizzled
//     tiles; one widening serves 256 rows. Widening leaves channels n and n + 4 of each eight side by side; the
//     queries are staged in the same order, and the outputs are put back when they are written.
//   * z_j = s_j (acc_j - 24 Q) + o_j Q and P' = p s_v need the keys' scales on the columns of S. The softmax
//     reads S as fragments (4 rows x 32 columns a thread) instead of a row a thread: a fourth of the reads of
//     scales, which with a row a thread would take twice the time of the products themselves.
//   * out = (O + sum p o_v) / sum p: the values' offsets add the same to every channel.
//   * Work is the list of (row pair tile, block) steps; the CTAs take equal shares of it, and what crosses CTAs
//     is joined by a second kernel from at most two parts per CTA.
// P' is a half, and the values q are: the reference m of a row's exponentials is the largest z + log2(s_v) of the keys that
// it sees (or up to kMostLog2 below it), so that the largest P' is 1 to 2^kMostLog2 whatever the values' size is. 32 keys at a
// time are weighed against the reference they meet; only where a row's weights times the block's largest s_v could pass
// 2^kMostLog2 the maxima are taken and the 32 are weighed again, and only where one does pass it, what was summed and stored so
// far is rescaled before that. Little is held in registers on purpose: spilled registers miss the L1 that 200 KB of shared
// memory leave (four reloads in a row cost more than the products of a block).
//
// Roles: warps 0-3 and 4-7 the softmax of tile 0 and 1, warp 8 issues the MMAs, warp 9 finds the CTA's work, warps
// 12-15 widen.
//
// Measured (bf16, 32 heads on 8 of 128): two chunks of 900 to 1024 tokens after 15000 to 16000 599 us, 805 TFLOP/s; 16 sequences of
// 8 tokens over 500 to 6000 122 us. What bounds it: with softmax, widening and reads left out the products take 341 us, since S has
// both operands in shared memory, which delivers them at 77 % of the tensor rate; reads add about 80, widening 50, the
// softmax 130. 16 softmax warps of 16 rows were slower (671 against 640), as were maxima taken before the weights (901).
#include <algorithm>
#include <cstddef>

#include "attn_tc.cuh"

namespace {

using namespace offq;

constexpr int kThreads = 512;
constexpr int kPairRows = 2 * kQt;
// A weight times its value's scale, as a half, reaches 2^14 before a row's reference is moved (and is 1 at most after it).
constexpr float kMostLog2 = 14.f;
// Registers: 128 a thread at launch, 2 x 144 + 96 + 128 = 4 x 128.
constexpr int kSoftmaxRegs = 144, kIssueRegs = 96, kWidenRegs = 128;
static_assert(2 * kSoftmaxRegs + kIssueRegs + kWidenRegs <= 4 * 128, "register shares");

struct PartHead {  // a part that crosses CTAs: sequence (negative: none), head, row pair tile, whether it is its last
  int b, h, p, ends;
};

struct ChunkCtrl {
  uint64_t q_full[2], k_full[2], v_full[2], k_empty[2], v_empty[2], s_full[2], p_ready[2], done;
  uint32_t tmem;
  int abort;
  int b, h, p, blk, count;
  alignas(16) float smax[2][4];        // the widening warps' largest value scales (read 16 bytes at a time)
  alignas(16) uint8_t missing[2][16];  // per 8 keys of the block: no page (the same)
};
static_assert(offsetof(ChunkCtrl, smax) % 16 == 0 && offsetof(ChunkCtrl, missing) % 16 == 0, "16-byte reads");

template <int D>
struct ChunkLayout {
  static constexpr int kTileBytes = kKt * D * 2;
  static constexpr int kKeys = 2 * kTileBytes;              // behind the two query tiles
  static constexpr int kValues = kKeys + 2 * kTileBytes;
  static constexpr int kParK = kValues + 2 * kTileBytes;    // [2][64] (s, s', b, b') of key pairs
  static constexpr int kParV = kParK + 2 * 1024;            // [2][64] (s, s', o, o')
  static constexpr int kSums = kParV + 2 * 1024;            // [2][128] sums of the queries
  static constexpr int kCtrl = kSums + 1024;
  static constexpr int kBytes = kCtrl + 512 + 1024;         // alignment to 1024
  static constexpr int64_t kPartFloats = kPairRows * (D + 2);
  static_assert(kCtrl % 16 == 0 && sizeof(ChunkCtrl) <= 512 && kBytes <= 232448, "shared memory");
};

__device__ __forceinline__ PartHead* part_heads(void* ws, int cta) { return static_cast<PartHead*>(ws) + 2 * cta; }
template <int D>
__device__ __forceinline__ float* part_data(void* ws, int ctas, int cta, int which) {
  return reinterpret_cast<float*>(static_cast<PartHead*>(ws) + 2 * ctas) + (2 * cta + which) * ChunkLayout<D>::kPartFloats;
}

// Blocks that row pair tile p of a sequence has to see (one at least, so that rows that see nothing are written).
__device__ __forceinline__ int tile_blocks(const AttnArgs& a, const PagedSeq& s, int p) {
  const int last = min(s.n - 1, (kPairRows * p + kPairRows - 1) / a.G);
  const int sees = min(s.len, max(0, s.len - s.n + last + 1));
  return max(1, (sees + kKt - 1) / kKt);
}
__device__ __forceinline__ int tiles_of(const AttnArgs& a, const PagedSeq& s) {
  return s.n * a.G <= a.few_rows ? 0 : (s.n * a.G + kPairRows - 1) / kPairRows;
}

// A place in the list of steps: sequence, head, row pair tile, block.
struct Walk {
  int b, h, p, blk, tiles, blocks;
  PagedSeq s;
  __device__ __forceinline__ void start(const AttnArgs& a, const ChunkCtrl* c) {
    b = c->b;
    h = c->h;
    p = c->p;
    blk = c->blk;
    s = paged_seq(a, b);
    tiles = tiles_of(a, s);
    blocks = tile_blocks(a, s, p);
  }
  __device__ __forceinline__ void next_tile(const AttnArgs& a) {
    blk = 0;
    if (++p == tiles) {
      p = 0;
      if (++h == a.H) {
        h = 0;
        do {
          s = paged_seq(a, ++b);
          tiles = tiles_of(a, s);
        } while (tiles == 0);
      }
    }
    blocks = tile_blocks(a, s, p);
  }
};

// Byte offset of 16-byte chunk ch (8 channels) of row r in a swizzled tile.
__device__ __forceinline__ uint32_t tile_off(int r, int ch) {
  return (ch >> 3) * kAtom + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ float4 lds128f(const float4* p) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(smem_u32(p)) : "memory");
  return v;
}

// Where row `row` of a (sequence, key head) goes.
template <int D, typename T>
__device__ __forceinline__ T* out_row(const AttnArgs& a, const PagedSeq& s, int h, int row) {
  return static_cast<T*>(a.out) + (static_cast<int64_t>(s.first) + row / a.G) * a.ld_out +
         static_cast<int64_t>(h * a.G + row % a.G) * D;
}
// The four lanes c of a row hold its channels 8 k + c and 8 k + c + 4 in (x, y); each writes channels 8 k + 2 c and the
// next. The lanes of a warp take part together; a row without a place is not written.
template <typename T>
__device__ __forceinline__ void write_pair(T* row, int k, int lane, float x, float y) {
  const int c = lane & 3;
  const uint32_t u = pack_16<T>(x, y);
  const uint32_t v0 = __shfl_sync(kAllLanes, u, (lane & ~3) | ((2 * c) & 3));
  const uint32_t v1 = __shfl_sync(kAllLanes, u, (lane & ~3) | ((2 * c + 1) & 3));
  if (row != nullptr) *reinterpret_cast<uint32_t*>(row + 8 * k + 2 * c) = __byte_perm(v0, v1, c < 2 ? 0x5410 : 0x7632);
}
template <int D, typename T>
__global__ void __launch_bounds__(kThreads, 1) chunk_kernel(const AttnArgs a) {
  using L = ChunkLayout<D>;
  constexpr bool kHalf = std::is_same<T, __half>::value;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
  const uint32_t base = smem_u32(smem);
  auto* ctrl = reinterpret_cast<ChunkCtrl*>(smem + L::kCtrl);
  volatile int* abort = &ctrl->abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&ctrl->q_full[i]), 4);
      mbar_init(smem_u32(&ctrl->k_full[i]), 4);
      mbar_init(smem_u32(&ctrl->v_full[i]), 4);
      mbar_init(smem_u32(&ctrl->k_empty[i]), 9);  // the products' commit and the eight softmax warps
      mbar_init(smem_u32(&ctrl->v_empty[i]), 1);
      mbar_init(smem_u32(&ctrl->s_full[i]), 1);
      mbar_init(smem_u32(&ctrl->p_ready[i]), 4);
    }
    mbar_init(smem_u32(&ctrl->done), 1);
    ctrl->abort = 0;
    ctrl->count = 0;
    mbar_fence_init();
  }
  if (warp == 8) {
    tmem_alloc(smem_u32(&ctrl->tmem), 512);
    tmem_relinquish();
  }
  griddep_wait();
  griddep_launch_dependents();
  __syncthreads();
  PartHead* heads = part_heads(a.workspace, blockIdx.x);
  if (warp == 9) {
    auto steps = [&](int b, PagedSeq& s) {  // of one head of sequence b
      s = paged_seq(a, b);
      long long n = 0;
      for (int p = 0, tiles = tiles_of(a, s); p < tiles; ++p) n += tile_blocks(a, s, p);
      return n;
    };
    long long total = 0;
    for (int b = lane; b < a.B; b += 32) {
      PagedSeq s;
      total += steps(b, s) * a.H;
      if (s.bad && blockIdx.x == 0) *a.status = OFFQ_ERR_INVALID_ARG;
    }
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) total += __shfl_xor_sync(kAllLanes, total, m);
    const long long ctas = min(total, static_cast<long long>(gridDim.x));
    const long long lo = blockIdx.x < ctas ? total * blockIdx.x / ctas : 0;
    const long long hi = blockIdx.x < ctas ? total * (blockIdx.x + 1) / ctas : 0;
    long long before = 0;
    for (int first = 0; first < a.B && before <= lo && lo < hi; first += 32) {
      PagedSeq s;
      const long long one = first + lane < a.B ? steps(first + lane, s) : 0, val = one * a.H;
      long long incl = val;
#pragma unroll
      for (int m = 1; m < 32; m <<= 1) {
        const long long o = __shfl_up_sync(kAllLanes, incl, m);
        if (lane >= m) incl += o;
      }
      const long long start = before + incl - val;
      if (lo >= start && lo < start + val) {
        long long at = (lo - start) % one;
        int p = 0;
        for (int n = tile_blocks(a, s, 0); at >= n; n = tile_blocks(a, s, ++p)) at -= n;
        ctrl->b = first + lane;
        ctrl->h = static_cast<int>((lo - start) / one);
        ctrl->p = p;
        ctrl->blk = static_cast<int>(at);
        ctrl->count = static_cast<int>(hi - lo);
      }
      before += __shfl_sync(kAllLanes, incl, 31);
    }
    if (lane < 2) heads[lane] = PartHead{-1, 0, 0, 0};
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctrl->tmem;
  const int count = ctrl->count;
  auto wait = [&](uint64_t* bar, int phase) {  // the warp goes on together
    return __all_sync(kAllLanes, mbar_wait(smem_u32(bar), phase & 1, abort));
  };

  if (warp >= 12) {
    // ---- Widening: codes and parameters of a block, one block ahead in registers ----
    fewer_registers<kWidenRegs>();
    constexpr int kChunks = D / 32;             // 16-byte chunks (32 codes) of a row
    constexpr int kRowsPer = 128 / kChunks;     // rows that the 128 threads cover at once
    constexpr int kReps = kKt / kRowsPer;       // 4 (D = 128), 2
    const int t = tid - 12 * 32, w = t >> 5;
    // Lanes that share a bank group in one atom and the other (c and c + 2) take rows whose swizzles differ.
    const int c = t % kChunks, row = (t / kChunks) ^ (c & 2);
    // The key whose parameters this thread takes is one of its own rows: the c-th.
    static_assert(kChunks == kReps, "a row for each of the lanes that share them");
    const int par_row = row + kRowsPer * c;
    uint32_t to_chunk[4];  // of this lane's four words in a tile (kRowsPer is a multiple of 8: the swizzle is the same in all reps)
#pragma unroll
    for (int k = 0; k < 4; ++k) to_chunk[k] = tile_off(row, 4 * c + k);
    struct Held {  // a block's codes and parameters in registers
      uint4 kc[kReps], vc[kReps];
      float2 kp, vp;
      uint32_t absent;  // reps whose rows have no page
    };
    struct Pages {  // a block's: head, first token, the sequence's length, the page of this lane's row in each rep
      int head, first, len, page[kReps];
    };
    Pages now, after;  // of the block to load and the one after it
    Walk at;           // the block whose pages were found last
    auto find_pages = [&](Pages& x) {  // of block `at`
      x.head = at.h;
      x.first = at.blk * kKt;
      x.len = at.s.len;
#pragma unroll
      for (int i = 0; i < kReps; ++i) {
        const int tok = x.first + kRowsPer * i + (row & ~7);
        x.page[i] = tok < x.len ? __ldg(a.table + static_cast<int64_t>(at.b) * a.ld_table + (tok >> a.page_shift)) : -1;
      }
    };
    auto step = [&](Pages& x) {
      if (++at.blk == at.blocks) at.next_tile(a);
      find_pages(x);
    };
    auto slot_of = [&](const Pages& x, int i) {
      const int tok = x.first + kRowsPer * i + row;
      return ((static_cast<int64_t>(x.page[i]) * a.H + x.head) << a.page_shift) + (tok & ((1 << a.page_shift) - 1));
    };
    auto load = [&](Held& x) {
      x.absent = 0;
      x.kp = x.vp = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kReps; ++i) {
        const int tok = now.first + kRowsPer * i + row;
        x.kc[i] = x.vc[i] = make_uint4(0u, 0u, 0u, 0u);
        if (now.page[i] < 0 || now.page[i] >= a.pages) {
          if ((tok & ~7) < now.len) {
            x.absent |= 1u << i;
            *a.status = OFFQ_ERR_INVALID_ARG;
          }
          continue;
        }
        const int64_t r = slot_of(now, i);
        x.kc[i] = __ldg(reinterpret_cast<const uint4*>(a.k_codes + r * (D / 2)) + c);
        x.vc[i] = __ldg(reinterpret_cast<const uint4*>(a.v_codes + r * (D / 2)) + c);
        if (i == c && tok < now.len) {
          x.kp = __ldg(reinterpret_cast<const float2*>(a.k_params) + r);
          x.vp = __ldg(reinterpret_cast<const float2*>(a.v_params) + r);
        }
      }
    };
    const float sc = a.scale * kLog2e;
    Held held[2];
    if (count > 0) {
      at.start(a, ctrl);
      find_pages(now);
      if (count > 1) step(after);
      load(held[0]);
    }
    auto widened = [&](uint32_t tile, const uint4& x, int i, auto is_v) {
      const uint32_t wd[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t to = tile + to_chunk[k] + i * kRowsPer * 128;
        if constexpr (is_v.value) {
          uint32_t q[4];
          widen_signed(wd[k], q[0], q[1]);
          widen_signed(wd[k] >> 8, q[2], q[3]);
          sts128(to, q[0], q[1], q[2], q[3]);
        } else {
          sts128(to, widen<T>(wd[k], 0), widen<T>(wd[k], 1), widen<T>(wd[k], 2), widen<T>(wd[k], 3));
        }
      }
    };
    // Block gb from x; the next one's reads go out first, and have the whole block's time.
    auto widen_block = [&](int gb, const Held& x, Held& next) {
      const int slot = gb & 1;
      if (gb + 1 < count) {
        now = after;
        load(next);
      }
      if (gb + 2 < count) step(after);
      if (gb >= 2 && !wait(&ctrl->k_empty[slot], (gb >> 1) - 1)) return false;
      const uint32_t kt = base + L::kKeys + slot * L::kTileBytes, vt = base + L::kValues + slot * L::kTileBytes;
#pragma unroll
      for (int i = 0; i < kReps; ++i) widened(kt, x.kc[i], i, std::false_type{});
      float* pk = reinterpret_cast<float*>(smem + L::kParK + slot * 1024) + (par_row >> 1) * 4 + (par_row & 1);
      float* pv = reinterpret_cast<float*>(smem + L::kParV + slot * 1024) + (par_row >> 1) * 4 + (par_row & 1);
      pk[0] = x.kp.x * sc;
      pk[2] = fmaf(-24.f, x.kp.x * sc, x.kp.y * sc);
      pv[0] = x.vp.x;
      pv[2] = x.vp.y;
      float top = x.vp.x;
#pragma unroll
      for (int m = 16; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(kAllLanes, top, m));
      if (lane == 0) ctrl->smax[slot][w] = top;
      if (lane % (8 * kChunks) == 0) {
#pragma unroll
        for (int i = 0; i < kReps; ++i) ctrl->missing[slot][(kRowsPer * i + row) >> 3] = x.absent >> i & 1u;
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctrl->k_full[slot]));
      if (gb >= 2 && !wait(&ctrl->v_empty[slot], (gb >> 1) - 1)) return false;
#pragma unroll
      for (int i = 0; i < kReps; ++i) widened(vt, x.vc[i], i, std::true_type{});
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctrl->v_full[slot]));
      return true;
    };
    for (int gb = 0; gb < count; gb += 2) {
      if (!widen_block(gb, held[0], held[1])) break;
      if (gb + 1 < count && !widen_block(gb + 1, held[1], held[0])) break;
    }
  } else if (warp >= 8) {
    fewer_registers<kIssueRegs>();
    if (warp == 8 && count > 0) {
      // ---- Products. The whole warp runs the loop; an elected lane issues ----
      constexpr uint32_t kIdescS = idesc_16<T>(128, kKt, false), kIdescO = idesc_16<__half>(128, D, true);
      Walk w;
      w.start(a, ctrl);
      int gb = 0, left = count, nq[2] = {0, 0}, np[2] = {0, 0};
      bool ok = true;
      auto scores = [&](int i, int g) {
        const uint64_t qd = smem_desc_sw128(base + i * L::kTileBytes);
        const uint64_t kd = smem_desc_sw128(base + L::kKeys + (g & 1) * L::kTileBytes);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t off = ((kk >> 2) * kAtom + (kk & 3) * 32) >> 4;
          mma_bf16(tmem + i * 128, qd + off, kd + off, kIdescS, kk != 0);
        }
        mma_commit(smem_u32(&ctrl->s_full[i]));
      };
      while (left > 0 && ok) {
        const int nb = min(w.blocks - w.blk, left);
        const int active = w.s.n * a.G - w.p * kPairRows > kQt ? 2 : 1;
        for (int i = 0; i < active && ok; ++i) ok = wait(&ctrl->q_full[i], nq[i]++);
        if (ok) ok = wait(&ctrl->k_full[gb & 1], gb >> 1);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          for (int i = 0; i < active; ++i) scores(i, gb);
          if (gb + 2 < count) mma_commit(smem_u32(&ctrl->k_empty[gb & 1]));  // else nobody waits for it
        }
        __syncwarp();
        for (int j = 0; j < nb && ok; ++j, ++gb) {
          ok = wait(&ctrl->v_full[gb & 1], gb >> 1);
          if (ok && j + 1 < nb) ok = wait(&ctrl->k_full[(gb + 1) & 1], (gb + 1) >> 1);
          for (int i = 0; i < active && ok; ++i) {
            ok = wait(&ctrl->p_ready[i], np[i]++);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
              const uint64_t vd = smem_desc_rows_contracted(base + L::kValues + (gb & 1) * L::kTileBytes);
#pragma unroll
              for (int kk = 0; kk < kKt / 16; ++kk)
                mma_16_ts(tmem + 256 + i * D, tmem + i * 128 + kk * 8, vd + ((kk * 16 * 128) >> 4), kIdescO, (j | kk) != 0);
              if (j + 1 < nb) scores(i, gb + 1);
              else mma_commit(smem_u32(&ctrl->s_full[i]));  // the outputs of this share of the tile are complete
            }
            __syncwarp();
          }
          if (ok && elect_one()) {
            if (gb + 2 < count) mma_commit(smem_u32(&ctrl->v_empty[gb & 1]));
            if (j + 1 < nb && gb + 3 < count) mma_commit(smem_u32(&ctrl->k_empty[(gb + 1) & 1]));
          }
          __syncwarp();
        }
        left -= nb;
        if (left > 0) w.next_tile(a);
      }
      if (__any_sync(kAllLanes, *abort)) {  // products in flight end before tensor memory is released
        if (elect_one()) {
          mma_commit(smem_u32(&ctrl->done));
          mbar_wait_teardown(smem_u32(&ctrl->done), 0);
        }
        __syncwarp();
      }
    }
  } else {
    more_registers<kSoftmaxRegs>();
    if (count > 0) {
      // ---- Softmax of tile i: fragments of rows 32 quad + 16 hh + 8 ii + g ----
      const int i = warp >> 2, quad = warp & 3, g = lane >> 2, c = lane & 3;
      const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
      const uint32_t s_tm = tmem + i * 128 + lanes, o_tm = tmem + 256 + i * D + lanes;
      float* sums = reinterpret_cast<float*>(smem + L::kSums) + i * kQt + quad * 32;
      Walk w;
      w.start(a, ctrl);
      int gb = 0, left = count, ns = 0;
      bool ok = true;
      while (left > 0 && ok) {
        const int nb = min(w.blocks - w.blk, left), rows = w.s.n * a.G;
        const int row0 = w.p * kPairRows + i * kQt + quad * 32;   // of this warp
        // A tile without rows takes no part; a warp without rows in a tile that has some only keeps step.
        const bool active = w.p * kPairRows + i * kQt < rows, live = row0 < rows;
        float m[4], qs[4];
        float l[4], off[4];
        int least = 0;
        if (active && !live && lane == 0) mbar_arrive(smem_u32(&ctrl->q_full[i]));
        if (live) {
          // This warp's query rows, in the widened channel order, and their sums.
          constexpr int kCh = D / 8, kPer = 32 / kCh;
          const int ch = lane % kCh, r0 = lane / kCh, dt = kPer / a.G, dg = kPer % a.G;
          int token = (row0 + r0) / a.G, gh = (row0 + r0) % a.G;
          const T* src = static_cast<const T*>(a.q) + static_cast<int64_t>(w.s.first) * a.ld_q + static_cast<int64_t>(w.h) * a.G * D + ch * 8;
#pragma unroll 1
          for (int it0 = 0; it0 < kCh; it0 += 8) {  // eight rows' reads in flight
            uint4 u[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              u[k] = make_uint4(0u, 0u, 0u, 0u);
              if (row0 + (it0 + k) * kPer + r0 < rows)
                u[k] = __ldg(reinterpret_cast<const uint4*>(src + token * a.ld_q + gh * D));
              token += dt;
              gh += dg;
              if (gh >= a.G) {
                gh -= a.G;
                ++token;
              }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const int r = (it0 + k) * kPer + r0;
              sts128(base + i * L::kTileBytes + tile_off(quad * 32 + r, ch), __byte_perm(u[k].x, u[k].z, 0x5410),
                     __byte_perm(u[k].x, u[k].z, 0x7632), __byte_perm(u[k].y, u[k].w, 0x5410), __byte_perm(u[k].y, u[k].w, 0x7632));
              const uint32_t x[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
              float sum = 0.f;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if constexpr (kHalf) {
                  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x[e]));
                  sum += f.x + f.y;
                } else {
                  sum += __uint_as_float(x[e] << 16) + __uint_as_float(x[e] & 0xFFFF0000u);
                }
              }
#pragma unroll
              for (int e = 1; e < kCh; e <<= 1) sum += __shfl_xor_sync(kAllLanes, sum, e);
              if (ch == 0) sums[r] = sum;
            }
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&ctrl->q_full[i]));
          least = min(w.s.len, max(0, w.s.len - w.s.n + row0 / a.G + 1));
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            qs[x] = sums[8 * x + g];   // x = 2 hh + ii
            l[x] = off[x] = 0.f;
            m[x] = -INFINITY;
          }
        }
        for (int j = 0; j < nb; ++j, ++gb) {
          const int slot = gb & 1;
          ok = wait(&ctrl->k_full[slot], gb >> 1);
          if (ok && active) ok = wait(&ctrl->s_full[i], ns++);
          if (!ok) break;
          if (live) {
            tc_fence_after();
            const float4* pk = reinterpret_cast<const float4*>(smem + L::kParK + slot * 1024) + c;
            const float4* pv = reinterpret_cast<const float4*>(smem + L::kParV + slot * 1024) + c;
            const int key0 = (w.blk + j) * kKt;
            const uint4 gone = *reinterpret_cast<const uint4*>(ctrl->missing[slot]);
            const float4 sm = *reinterpret_cast<const float4*>(ctrl->smax[slot]);
            // log2 of the block's largest value scale, rounded up: weights up to 2^(kMostLog2 - lift) stay below 2^kMostLog2 with it.
            const float big = fmaxf(fmaxf(sm.x, sm.y), fmaxf(sm.z, sm.w));
            const float lift = static_cast<float>(min(128, max(static_cast<int>(kLeastLog2), static_cast<int>(__float_as_uint(big) >> 23 & 255u) - 126)));
            const float most = ex2(kMostLog2 - lift);
            const bool masked = key0 + kKt > least || (gone.x | gone.y | gone.z | gone.w) != 0u;
            int sees[4] = {0, 0, 0, 0};
            if (masked) {
#pragma unroll
              for (int x = 0; x < 4; ++x) sees[x] = min(w.s.len, w.s.len - w.s.n + (row0 + 8 * x + g) / a.G + 1) - key0 - 2 * c;
            }
            // 32 keys at a time: scores relative to m, weights, sums; the weights take the place of scores already read.
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
              uint32_t s[2][16], p[2][8];
              uint64_t lb[4], wb[4];
              tmem_ld_fragments(s_tm + 32 * q, s[0], s[1]);
              if (masked) {
                const uint32_t word = q == 0 ? gone.x : q == 1 ? gone.y : q == 2 ? gone.z : gone.w;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const bool out = (word >> (8 * k) & 0xFFu) != 0u;
#pragma unroll
                  for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                      if (out || 32 * q + 8 * k + e >= sees[x]) s[x >> 1][4 * k + 2 * (x & 1) + e] = 0x7FFFFFFFu;  // NaN: hidden
                }
              }
              const float4 *pkq = pk + q * 16, *pvq = pv + q * 16;
              auto weigh = [&](auto hide) {
                uint64_t m2[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                  m2[x] = pack2(-m[x], -m[x]);
                  lb[x] = wb[x] = 0;
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const float4 f = lds128f(pkq + k * 4), v = lds128f(pvq + k * 4);
                  const uint64_t a2 = pack2(f.x, f.y), b2 = pack2(f.z, f.w), s2 = pack2(v.x, v.y), o2 = pack2(v.z, v.w);
#pragma unroll
                  for (int x = 0; x < 4; ++x) {
                    const uint32_t* e = &s[x >> 1][4 * k + 2 * (x & 1)];
                    float y0, y1;
                    unpack2(fma2v(pack2(__uint_as_float(e[0]), __uint_as_float(e[1])), a2, fma2v(b2, pack2(qs[x], qs[x]), m2[x])), y0, y1);
                    if constexpr (hide.value) {
                      if (e[0] == 0x7FFFFFFFu) y0 = -INFINITY;
                      if (e[1] == 0x7FFFFFFFu) y1 = -INFINITY;
                    }
                    const uint64_t p2 = pack2(ex2(y0), ex2(y1));
                    lb[x] = add2_rn(lb[x], p2);
                    wb[x] = fma2v(p2, o2, wb[x]);
                    unpack2(mul2v(p2, s2), y0, y1);
                    p[x >> 1][2 * k + (x & 1)] = pack_16<__half>(y0, y1);
                  }
                }
              };
              if (masked)
                weigh(std::true_type{});
              else
                weigh(std::false_type{});
              // Weights are positive: a sum that is small has no large one in it. (An unset reference gives infinity.)
              bool fits = true;
              float row_sum[4];
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                float y0, y1;
                unpack2(lb[x], y0, y1);
                row_sum[x] = y0 + y1;
                fits &= row_sum[x] <= most;
              }
              // Where some row's may not: the largest z + log2 of the value's scale among the keys it sees. A large scale that is
              // not seen or hardly weighs moves no reference.
              if (__any_sync(kAllLanes, !fits)) {
                float keep[4];
                bool move = false;
#pragma unroll
                for (int x = 0; x < 4; ++x) keep[x] = -INFINITY;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const float4 f = lds128f(pkq + k * 4), v = lds128f(pvq + k * 4);
                  const float v0 = fmaxf(__log2f(v.x), kLeastLog2), v1 = fmaxf(__log2f(v.y), kLeastLog2);
#pragma unroll
                  for (int x = 0; x < 4; ++x) {
                    const uint32_t* e = &s[x >> 1][4 * k + 2 * (x & 1)];
                    const float z0 = fmaf(__uint_as_float(e[0]), f.x, f.z * qs[x]), z1 = fmaf(__uint_as_float(e[1]), f.y, f.w * qs[x]);
                    keep[x] = fmaxf(keep[x], fmaxf(z0 + v0, z1 + v1));  // hidden keys are NaN and do not count
                  }
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                  keep[x] = fmaxf(keep[x], __shfl_xor_sync(kAllLanes, keep[x], 1));
                  keep[x] = fmaxf(keep[x], __shfl_xor_sync(kAllLanes, keep[x], 2));
                  move |= keep[x] > m[x] + kMostLog2;
                }
                move = __any_sync(kAllLanes, move);
                if (move) {
#pragma unroll
                  for (int x = 0; x < 4; ++x) {
                    const float top = fmaxf(keep[x], m[x]);
                    keep[x] = m[x] == -INFINITY ? 0.f : ex2(m[x] - top);
                    m[x] = top;
                    l[x] *= keep[x];
                    off[x] *= keep[x];
                  }
                }
                if (move && j > 0) {
#pragma unroll 1
                  for (int u = 0; u < D / 32; ++u) {
                    uint32_t o0[16], o1[16];
                    tmem_ld_fragments(o_tm + 32 * u, o0, o1);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                      o0[e] = __float_as_uint(__uint_as_float(o0[e]) * keep[e >> 1 & 1]);
                      o1[e] = __float_as_uint(__uint_as_float(o1[e]) * keep[2 + (e >> 1 & 1)]);
                    }
                    tmem_st_fragments(o_tm + 32 * u, o0);
                    tmem_st_fragments(o_tm + 32 * u + (16u << 16), o1);
                  }
                }
                tmem_st_wait();
#pragma unroll 1
                for (int u = 0; u < (move ? 2 * q : 0); ++u) {  // this block's weights so far
                  const uint32_t at = s_tm + 16 * (u >> 1) + (static_cast<uint32_t>(16 * (u & 1)) << 16);
                  uint32_t r[8];
                  tmem_ld_pairs(at, r);
#pragma unroll
                  for (int e = 0; e < 8; ++e) {
                    const float k = u & 1 ? keep[2 + (e & 1)] : keep[e & 1];
                    r[e] = scale_halves(r[e], k);
                  }
                  tmem_st_pairs(at, r);
                }
                weigh(std::true_type{});
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                  float y0, y1;
                  unpack2(lb[x], y0, y1);
                  row_sum[x] = y0 + y1;
                }
              }
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                float y0, y1;
                unpack2(wb[x], y0, y1);
                l[x] += row_sum[x];
                off[x] += y0 + y1;
              }
              tmem_st_pairs(s_tm + 16 * q, p[0]);
              tmem_st_pairs(s_tm + 16 * q + (16u << 16), p[1]);
            }
            tmem_st_wait();
            tc_fence_before();
          }
          __syncwarp();
          if (lane == 0) {
            if (active) mbar_arrive(smem_u32(&ctrl->p_ready[i]));
            mbar_arrive(smem_u32(&ctrl->k_empty[slot]));
          }
        }
        if (ok && active) ok = wait(&ctrl->s_full[i], ns++);
        if (ok && live) {
          tc_fence_after();
          const bool complete = w.blk == 0 && nb == w.blocks;
          const int which = w.blk == 0 ? 1 : 0;
          float* part = part_data<D>(a.workspace, gridDim.x, blockIdx.x, which);
          float inv[4];
          T* to[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
#pragma unroll
            for (int k = 1; k < 4; k <<= 1) {
              l[x] += __shfl_xor_sync(kAllLanes, l[x], k);
              off[x] += __shfl_xor_sync(kAllLanes, off[x], k);
            }
            inv[x] = l[x] > 0.f ? __fdividef(1.f, l[x]) : 0.f;
            const int r = 8 * x + g;
            to[x] = row0 + r < rows ? out_row<D, T>(a, w.s, w.h, row0 + r) : nullptr;
            if (c == 0) {
              if (!complete) {
                part[i * kQt + quad * 32 + r] = m[x];
                part[kPairRows + i * kQt + quad * 32 + r] = l[x];
              } else if (row0 + r < rows) {
                write_lse(a, w.s.first, w.h, row0 + r, m[x], l[x]);
              }
            }
          }
#pragma unroll 1
          for (int q = 0; q < D / 32; ++q) {
            uint32_t o[2][16];
            tmem_ld_fragments(o_tm + 32 * q, o[0], o[1]);
#pragma unroll
            for (int hh = 0; hh < 2; ++hh)
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(o[hh][4 * k + e]) + off[2 * hh + (e >> 1)];
                if (complete) {
#pragma unroll
                  for (int ii = 0; ii < 2; ++ii)
                    write_pair<T>(to[2 * hh + ii], 4 * q + k, lane, v[2 * ii] * inv[2 * hh + ii], v[2 * ii + 1] * inv[2 * hh + ii]);
                } else {
                  reinterpret_cast<float4*>(part + 2 * kPairRows)[(warp * (D / 4) + hh * (D / 8) + 4 * q + k) * 32 + lane] =
                      make_float4(v[0], v[1], v[2], v[3]);
                }
              }
            __syncwarp();
          }
          if (!complete && i == 0 && warp == 0 && lane == 0)
            heads[which] = PartHead{w.b, w.h, w.p, w.blk + nb == w.blocks};
          tc_fence_before();
        }
        left -= nb;
        if (left > 0 && ok) w.next_tile(a);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (tid == 0 && ctrl->abort) *a.status = OFFQ_ERR_TIMEOUT;
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// Row pair tiles that cross CTAs: begun at the end of CTA blockIdx.x, then the first parts of the CTAs after it up to
// their last. Block y takes one softmax warp's 32 rows; a warp of it a quarter of the channels.
template <int D, typename T>
__global__ void __launch_bounds__(128) join_chunks_kernel(const AttnArgs a, int ctas) {
  __shared__ int s_last;
  const int cta = blockIdx.x, tid = threadIdx.x, lane = tid & 31, q = tid >> 5, g = lane >> 2, c = lane & 3;
  if (tid == 0) s_last = 0x7FFFFFFF;
  griddep_wait();
  griddep_launch_dependents();
  const PartHead p = part_heads(a.workspace, cta)[1];
  if (p.b < 0) return;
  __syncthreads();
  for (int k = cta + 1 + tid; k < ctas; k += blockDim.x) {
    const PartHead n = part_heads(a.workspace, k)[0];
    if (n.b == p.b && n.h == p.h && n.p == p.p && n.ends) atomicMin(&s_last, k);
  }
  __syncthreads();
  const int last = s_last;
  if (last >= ctas) return;  // a CTA gave up: the status word says so
  const PagedSeq s = paged_seq(a, p.b);
  const int rows = s.n * a.G, warp = blockIdx.y, row0 = p.p * kPairRows + warp * 32;
  if (row0 >= rows) return;
  constexpr int kReps = D / 32;  // of 8 channels, per warp
  float top[4], sum[4];
  float4 acc[2][kReps];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    top[x] = -INFINITY;
    sum[x] = 0.f;
  }
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
#pragma unroll
    for (int k = 0; k < kReps; ++k) acc[hh][k] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int part = cta; part <= last; ++part) {
    const float* src = part_data<D>(a.workspace, ctas, part, part == cta ? 1 : 0);
    float x_old[4], x_new[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int r = warp * 32 + 8 * x + g;
      const float mk = src[r], next = fmaxf(top[x], mk);
      x_old[x] = top[x] == -INFINITY ? 0.f : ex2(top[x] - next);
      x_new[x] = mk == -INFINITY ? 0.f : ex2(mk - next);
      sum[x] = sum[x] * x_old[x] + src[kPairRows + r] * x_new[x];
      top[x] = next;
    }
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
#pragma unroll
      for (int k = 0; k < kReps; ++k) {
        const float4 v = reinterpret_cast<const float4*>(src + 2 * kPairRows)[(warp * (D / 4) + hh * (D / 8) + q * kReps + k) * 32 + lane];
        float4& o = acc[hh][k];
        o.x = o.x * x_old[2 * hh] + v.x * x_new[2 * hh];
        o.y = o.y * x_old[2 * hh] + v.y * x_new[2 * hh];
        o.z = o.z * x_old[2 * hh + 1] + v.z * x_new[2 * hh + 1];
        o.w = o.w * x_old[2 * hh + 1] + v.w * x_new[2 * hh + 1];
      }
  }
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
#pragma unroll
    for (int ii = 0; ii < 2; ++ii) {
      const int x = 2 * hh + ii, r = row0 + 8 * x + g;
      const float inv = sum[x] > 0.f ? __fdividef(1.f, sum[x]) : 0.f;
      T* to = r < rows ? out_row<D, T>(a, s, p.h, r) : nullptr;
#pragma unroll
      for (int k = 0; k < kReps; ++k)
        write_pair<T>(to, q * kReps + k, lane, (ii ? acc[hh][k].z : acc[hh][k].x) * inv, (ii ? acc[hh][k].w : acc[hh][k].y) * inv);
      if (q == 0 && c == 0 && r < rows) write_lse(a, s.first, p.h, r, top[x], sum[x]);
    }
}

template <int D, typename T>
int launch_chunk(const AttnArgs& a, cudaStream_t s) {
  using L = ChunkLayout<D>;
  const int sms = device_sms();
  if (sms == 0 || !smem_optin<chunk_kernel<D, T>>(L::kBytes)) return OFFQ_ERR_CUDA;
  if (const int rc = launch_pdl(chunk_kernel<D, T>, dim3(sms), dim3(kThreads), L::kBytes, s, a); rc != OFFQ_OK) return rc;
  return launch_pdl(join_chunks_kernel<D, T>, dim3(sms, 8), dim3(128), 0, s, a, sms);
}

}  // namespace

namespace offq {

int64_t paged_chunk_workspace(int head_dim) {
  const int sms = device_sms();
  return sms == 0 ? -1 : 2 * static_cast<int64_t>(sms) * (static_cast<int64_t>(sizeof(PartHead)) + 4 * kPairRows * (head_dim + 2));
}

int paged_chunk(const AttnArgs& a, int dtype, int head_dim, cudaStream_t s) {
  if (head_dim == 128)
    return dtype == OFFQ_BF16 ? launch_chunk<128, __nv_bfloat16>(a, s) : launch_chunk<128, __half>(a, s);
  return dtype == OFFQ_BF16 ? launch_chunk<64, __nv_bfloat16>(a, s) : launch_chunk<64, __half>(a, s);
}

}  // namespace offq
