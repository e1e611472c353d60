// Attention inside packed prompts (offq_prompt_attention) on the tensor cores.
//
// A work item is two tiles of 128 query rows: the same 128 tokens of two heads that share their keys, or
// 256 tokens of one head where the heads per key head are odd. The grid has a CTA for each item, those furthest into
// their sequences first; a CTA that runs (one per SM) takes over the items of CTAs that have not started yet (cluster
// launch control), so an item's copies and first products run while the last one's outputs are written and shares even
// out by themselves. Per block of 128 keys a tile runs
//   S = Q K^T (operands in shared memory), weights P = 2^(scale log2(e) S - m) by one thread per row,
//   O += P V (P in tensor memory, V as it lies: its rows are contracted).
// S and O stay in tensor memory (2 x 128 + 2 x D columns); P takes the place of its S. While one tile's
// rows are in the softmax the other's products run, so the tensor cores wait only where the softmax is
// the longer of the two.
//
// Roles: warps 0-3 and 4-7 the softmax of tile 0 and 1, warp 8 issues the MMAs, warp 9 the TMA copies, warp 10
// finds the items.
// A row's reference maximum is moved only when a score passes it by 2^8 (kLazy), so O is rescaled rarely and
// by the softmax threads themselves: when S is complete, so is every product issued before it, O's among them. The
// weights of the first 64 keys go to the products while those of the other 64 are made.
//
// Rows past a sequence's end are the next sequence's. As queries they are not written, as keys their
// scores are replaced, and as values they are zeroed in shared memory (0 times infinity is not 0).
//
// Measured (causal): one prompt of 8192, 32 heads on 8 of 128, bf16: 388 us, 1416 TFLOP/s, tensor pipe 58 % on a prompt of 4096;
// S with both operands in shared memory runs at 77 % of the tensor rate at best. 24 prompts of 5 to 2000, 16 heads on 4 of
// 64, f16: 125 us, 680 TFLOP/s: 1.33 us a block of 128 keys and about 2 us an item, latency and not any one pipe (exponentials
// 28 %). Without taking over items 151 us; with two threads a row 148.
#include <algorithm>

#include "attn_tc.cuh"

namespace {

using namespace offq;

constexpr int kThreads = 384;  // two softmax warpgroups, one of single warps
// Registers: 168 a thread at launch, 3 x 168 >= 2 x 208 + 88.
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;
static_assert(2 * kSoftmaxRegs + kOtherRegs <= 3 * 168, "register shares");
// A row's reference is left where it is until a score passes it by this much (in powers of two): weights then reach
// 2^8 at most, far from any overflow, and a rescaling of the sums is rare.
constexpr float kLazy = 8.0f;

template <int D>
struct PromptLayout {
  static constexpr int kTileBytes = kKt * D * 2;
  static constexpr int kSlots = D == 128 ? 5 : 8;           // keys and values in turn
  static constexpr int kRing = 2 * kTileBytes;              // behind the two query tiles
  static constexpr int kCtrl = kRing + kSlots * kTileBytes;
  static constexpr int kBytes = kCtrl + 512 + 1024;         // barriers; alignment to 1024
  static_assert(kBytes <= 232448, "shared memory");
};

struct Item {  // first row and rows of a sequence (no rows: no more items), first token of the tiles, head or head pair
  int first, n, token, unit;
};

struct PromptCtrl {
  uint64_t q_full[2], q_empty[2], tail, done;
  uint64_t full[8], empty[8];
  uint64_t s_full[2], p_ready[2][2];  // weights of 64 keys at a time
  // An item's outputs. Not a further phase of s_full: the next item's scores follow them without an answer from the
  // softmax, and a warp that came after both would wait for a third.
  uint64_t o_full[2];
  uint64_t item_full, item_empty, taken;
  alignas(16) uint32_t answer[4];
  alignas(16) Item item;
  uint32_t tmem;
  int abort;
};
static_assert(sizeof(PromptCtrl) <= 512, "control block");

// Queries of sequence b (its first row in `first`); none where its entries are out of range.
__device__ __forceinline__ int prompt_seq(const AttnArgs& a, int b, int& first, bool& bad) {
  const int c0 = __ldg(a.cu + b), c1 = __ldg(a.cu + b + 1);
  first = c0;
  bad = c0 < 0 || c1 < c0 || c1 > a.Tq;
  return bad ? 0 : c1 - c0;
}

// Asks for the index of a CTA of the grid that has not started (and now never will); 16 bytes arrive on `bar`.
__device__ __forceinline__ void take_over(uint32_t answer, uint32_t bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer),
               "r"(bar)
               : "memory");
}
// The index, or -1 where all have started.
__device__ __forceinline__ int taken_over(uint32_t answer) {
  int x;
  asm volatile(
      "{\n"
      ".reg .b128 a;\n"
      ".reg .pred p;\n"
      "ld.shared.b128 a, [%1];\n"
      "mov.b32 %0, -1;\n"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, a;\n"
      "}\n"
      : "=r"(x)
      : "r"(answer)
      : "memory");
  return x;
}

template <int D, typename T>
__global__ void __launch_bounds__(kThreads, 1)
prompt_kernel(const AttnArgs a, const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
              const __grid_constant__ CUtensorMap vmap) {
  using L = PromptLayout<D>;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
  auto* ctrl = reinterpret_cast<PromptCtrl*>(smem + L::kCtrl);
  volatile int* abort = &ctrl->abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const bool two_heads = (a.G & 1) == 0;
  const int units = two_heads ? a.Hq / 2 : a.Hq;       // per query tile
  const int step = two_heads ? kQt : 2 * kQt;          // tokens per query tile
  if (tid == 0) {
    mbar_init(smem_u32(&ctrl->tail), 1);
    mbar_init(smem_u32(&ctrl->done), 1);
    for (int i = 0; i < 8; ++i) {
      mbar_init(smem_u32(&ctrl->full[i]), 1);
      mbar_init(smem_u32(&ctrl->empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&ctrl->q_full[i]), 1);
      mbar_init(smem_u32(&ctrl->q_empty[i]), 1);
      mbar_init(smem_u32(&ctrl->s_full[i]), 1);
      mbar_init(smem_u32(&ctrl->o_full[i]), 1);
      mbar_init(smem_u32(&ctrl->p_ready[i][0]), 4);
      mbar_init(smem_u32(&ctrl->p_ready[i][1]), 4);
    }
    mbar_init(smem_u32(&ctrl->item_full), 1);
    mbar_init(smem_u32(&ctrl->item_empty), 10);  // the warps that read it
    mbar_init(smem_u32(&ctrl->taken), 1);
    ctrl->abort = 0;
    mbar_fence_init();
  }
  if (warp == 8) {
    tmem_alloc(smem_u32(&ctrl->tmem), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_wait();
  griddep_launch_dependents();
  const uint32_t tmem = ctrl->tmem;
  const uint32_t q_s = smem_u32(smem), ring = q_s + L::kRing;
  auto wait = [&](uint64_t* bar, int phase) {  // the warp goes on together
    return __all_sync(kAllLanes, mbar_wait(smem_u32(bar), phase & 1, abort));
  };
  // Item number k of this CTA, for the warps that work on it; false at the end.
  int head[2], row0[2], blocks[2], most = 0;
  Item item = {};
  auto next_item = [&](int k) {
    if (!wait(&ctrl->item_full, k)) return false;
    item = ctrl->item;
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&ctrl->item_empty));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      head[i] = two_heads ? 2 * item.unit + i : item.unit;
      row0[i] = item.token + (two_heads ? 0 : i * kQt);
      const int sees = a.causal ? min(row0[i] + kQt, item.n) : item.n;
      blocks[i] = row0[i] < item.n ? (sees + kKt - 1) / kKt : 0;
    }
    most = max(blocks[0], blocks[1]);
    return item.n > 0;
  };

  if (warp >= 8) {
    fewer_registers<kOtherRegs>();
    if (warp == 10) {
      // ---- Items: level t of the list holds the t-th tile of every sequence that has one, the highest level first ----
      auto tiles_at = [&](int b, int& first, int& n, bool& bad) {
        n = b < a.B ? prompt_seq(a, b, first, bad) : 0;
        return (n + step - 1) / step;
      };
      int longest = 0;
      for (int b = lane; b < a.B; b += 32) {
        int first, n;
        bool bad = false;
        longest = max(longest, tiles_at(b, first, n, bad));
        if (bad && blockIdx.x == 0) *a.status = OFFQ_ERR_INVALID_ARG;
      }
#pragma unroll
      for (int m = 16; m > 0; m >>= 1) longest = max(longest, __shfl_xor_sync(kAllLanes, longest, m));
      auto above = [&](int t) {  // tiles at level t and higher
        int count = 0;
        for (int b = lane; b < a.B; b += 32) {
          int first, n;
          bool bad = false;
          count += max(0, tiles_at(b, first, n, bad) - t);
        }
#pragma unroll
        for (int m = 16; m > 0; m >>= 1) count += __shfl_xor_sync(kAllLanes, count, m);
        return count;
      };
      const int total = above(0);
      int level = 0, higher = 0, at_level = 0;  // tiles above it and at it
      int taken = 0;  // answers so far; negative after a wait that ran out
      auto take = [&]() {
        const uint32_t bar = smem_u32(&ctrl->taken);
        if (lane == 0) {
          fence_proxy_async_smem();
          mbar_arrive_expect_tx(bar, 16);
          take_over(smem_u32(ctrl->answer), bar);
        }
        __syncwarp();
        if (!wait(&ctrl->taken, taken)) {
          if (lane == 0) mbar_wait_teardown(bar, taken & 1);  // the answer lands before the CTA ends
          __syncwarp();
          taken = -1;
          return -1;
        }
        ++taken;
        int at = 0;  // read by the lane that asks and fences: the next answer is written over this one
        if (lane == 0) at = taken_over(smem_u32(ctrl->answer));
        return __shfl_sync(kAllLanes, at, 0);
      };
      bool more = true;
      for (int k = 0; more; ++k) {
        int at = blockIdx.x;
        if (k > 0) {
          // All warps have begun the last item: take over another CTA's.
          if (!wait(&ctrl->item_empty, k - 1)) break;
          at = take();
        }
        // The grid is sized by what the lengths could be at most: CTAs past the last item are taken, not started.
        while (at >= 0 && at / units >= total) at = take();
        if (taken < 0) break;
        Item found = {0, 0, 0, 0};
        more = at >= 0;
        if (more) {
          const int rank = static_cast<int>(at / units);
          if (rank < higher || rank >= higher + at_level) {  // another level, with above(lo) > rank >= above(hi)
            int lo = 0, hi = longest;
            while (hi - lo > 1) {
              const int mid = (lo + hi) / 2;
              if (above(mid) > rank) lo = mid;
              else hi = mid;
            }
            level = lo;
            higher = above(hi);
            at_level = above(lo) - higher;
          }
          int left = rank - higher;  // of the sequences with a tile at this level, the left-th
          for (int base = 0; base < a.B && left >= 0; base += 32) {
            int first, n;
            bool bad = false;
            const bool has = tiles_at(base + lane, first, n, bad) > level;
            const uint32_t mask = __ballot_sync(kAllLanes, has);
            const int mine = __popc(mask & ((1u << lane) - 1u));
            const uint32_t hit = __ballot_sync(kAllLanes, has && mine == left);
            if (hit != 0) {
              const int from = __ffs(hit) - 1;
              found.first = __shfl_sync(kAllLanes, first, from);
              found.n = __shfl_sync(kAllLanes, n, from);
            }
            left -= __popc(mask);
          }
          found.token = level * step;
          found.unit = static_cast<int>(at % units);
        }
        if (lane == 0) {
          ctrl->item = found;
          mbar_arrive(smem_u32(&ctrl->item_full));
        }
        __syncwarp();
      }
    } else if (warp == 9) {
      // ---- Copies: both query tiles, then K0 V0 K1 V1 ... ----
      int it = 0, tails = 0, nq[2] = {0, 0};
      uint32_t last_tail = 0;  // ring slots whose last copy went to the tail barrier
      bool ok = true;
      for (int k = 0; ok && next_item(k); ++k) {
        const int kv_head = head[0] / a.G, left = item.n - (most - 1) * kKt;  // keys of the last block
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (blocks[i] == 0 || !ok) continue;
          if (nq[i] > 0) ok = wait(&ctrl->q_empty[i], nq[i] - 1);
          if (ok && lane == 0) {
            const uint32_t bar = smem_u32(&ctrl->q_full[i]);
            mbar_arrive_expect_tx(bar, L::kTileBytes);
            for (int c = 0; c < D / 64; ++c)
              tma_load_2d(q_s + i * L::kTileBytes + c * kAtom, &qmap, bar, head[i] * D + 64 * c, item.first + row0[i]);
          }
          if (ok) ++nq[i];
        }
        for (int u = 0; u < 2 * most && ok; ++u) {
          const int slot = it % L::kSlots;
          const bool is_v = u & 1, tail = is_v && u / 2 == most - 1 && left < kKt;
          if (it >= L::kSlots) ok = wait(&ctrl->empty[slot], it / L::kSlots - 1);
          if (!ok) break;
          const uint32_t dst = ring + slot * L::kTileBytes, bar = smem_u32(tail ? &ctrl->tail : &ctrl->full[slot]);
          if (lane == 0) {
            mbar_arrive_expect_tx(bar, L::kTileBytes);
            for (int c = 0; c < D / 64; ++c)
              tma_load_2d(dst + c * kAtom, is_v ? &vmap : &kmap, bar, kv_head * D + 64 * c, item.first + u / 2 * kKt);
          }
          __syncwarp();
          last_tail = tail ? last_tail | 1u << slot : last_tail & ~(1u << slot);
          ++it;
          if (tail) {
            ok = wait(&ctrl->tail, tails++);
            if (!ok) break;
            for (int z = lane; z < (kKt - left) * (D / 8); z += 32) {
              const int r = left + z / (D / 8), ch = z % (D / 8);
              sts_zero16(dst + (ch >> 3) * kAtom + r * 128 + (ch & 7) * 16);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctrl->full[slot]));
          }
        }
      }
      if (*abort && lane == 0) {  // copies in flight land before the CTA ends
        for (int i = 0; i < 2; ++i)
          if (nq[i] > 0) mbar_wait_teardown(smem_u32(&ctrl->q_full[i]), (nq[i] - 1) & 1);
        if (tails > 0) mbar_wait_teardown(smem_u32(&ctrl->tail), (tails - 1) & 1);
        for (int z = max(0, it - L::kSlots); z < it; ++z)
          if (!(last_tail >> (z % L::kSlots) & 1u)) mbar_wait_teardown(smem_u32(&ctrl->full[z % L::kSlots]), (z / L::kSlots) & 1);
      }
      __syncwarp();
    } else if (warp == 8) {
      // ---- Products. The whole warp runs the loop; an elected lane issues ----
      constexpr uint32_t kIdescS = idesc_16<T>(128, kKt, false), kIdescO = idesc_16<T>(128, D, true);
      auto scores = [&](int i, int use) {  // S_i = Q_i K^T
        const uint64_t qd = smem_desc_sw128(q_s + i * L::kTileBytes);
        const uint64_t kd = smem_desc_sw128(ring + use % L::kSlots * L::kTileBytes);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t off = ((kk >> 2) * kAtom + (kk & 3) * 32) >> 4;
          mma_bf16(tmem + i * 128, qd + off, kd + off, kIdescS, kk != 0);
        }
        mma_commit(smem_u32(&ctrl->s_full[i]));
      };
      auto outputs = [&](int i, int use, int part, bool first) {  // O_i += P_i V, 64 keys of it
        const uint64_t vd = smem_desc_rows_contracted(ring + use % L::kSlots * L::kTileBytes);
#pragma unroll
        for (int kk = 4 * part; kk < 4 * part + 4; ++kk)
          mma_16_ts(tmem + 256 + i * D, tmem + i * 128 + kk * 8, vd + ((kk * 16 * 128) >> 4), kIdescO, !first || kk != 0);
      };
      int it = 0, nq[2] = {0, 0}, np[2] = {0, 0};  // ring uses, query tiles, weights so far
      bool ok = true;
      for (int k = 0; ok && next_item(k); ++k) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (blocks[i] > 0 && ok) ok = wait(&ctrl->q_full[i], nq[i]++);
        if (ok) ok = wait(&ctrl->full[it % L::kSlots], it / L::kSlots);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (blocks[i] > 0) {
              scores(i, it);
              if (blocks[i] == 1) mma_commit(smem_u32(&ctrl->q_empty[i]));
            }
          mma_commit(smem_u32(&ctrl->empty[it % L::kSlots]));
        }
        __syncwarp();
        ++it;
        for (int j = 0; j < most && ok; ++j) {
          const int vs = it, ks = it + 1;
          ok = wait(&ctrl->full[vs % L::kSlots], vs / L::kSlots);
          if (ok && j + 1 < most) ok = wait(&ctrl->full[ks % L::kSlots], ks / L::kSlots);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (j >= blocks[i] || !ok) continue;
            ok = wait(&ctrl->p_ready[i][0], np[i]);
            if (!ok) continue;
            tc_fence_after();
            if (elect_one()) outputs(i, vs, 0, j == 0);
            __syncwarp();
            ok = wait(&ctrl->p_ready[i][1], np[i]++);
            if (!ok) continue;
            tc_fence_after();
            if (elect_one()) {
              outputs(i, vs, 1, j == 0);
              if (j + 1 < blocks[i]) {
                scores(i, ks);
                if (j + 2 == blocks[i]) mma_commit(smem_u32(&ctrl->q_empty[i]));
              } else {
                mma_commit(smem_u32(&ctrl->o_full[i]));
              }
            }
            __syncwarp();
          }
          if (!ok) break;
          if (elect_one()) {
            mma_commit(smem_u32(&ctrl->empty[vs % L::kSlots]));
            if (j + 1 < most) mma_commit(smem_u32(&ctrl->empty[ks % L::kSlots]));
          }
          __syncwarp();
          it += j + 1 < most ? 2 : 1;
        }
      }
      // All products and all arrivals of their commits are through before the CTA ends and its tensor memory is released.
      if (elect_one()) {
        mma_commit(smem_u32(&ctrl->done));
        mbar_wait_teardown(smem_u32(&ctrl->done), 0);
      }
      __syncwarp();
    }
  } else {
    more_registers<kSoftmaxRegs>();
    const int i = warp >> 2;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_tm = tmem + i * 128 + lanes, o_tm = tmem + 256 + i * D + lanes;
    const float sc = a.scale * kLog2e;
    int ns = 0, no = 0;
    bool ok = true;
    for (int k = 0; ok && next_item(k); ++k) {
      const int my_blocks = i ? blocks[1] : blocks[0], my_row0 = i ? row0[1] : row0[0], my_head = i ? head[1] : head[0];
      if (my_blocks == 0) continue;
      const int n = item.n, row = my_row0 + (warp & 3) * 32 + lane;   // in the sequence
      float m = -INFINITY, sum = 0.f;
      for (int j = 0; j < my_blocks; ++j) {
        ok = wait(&ctrl->s_full[i], ns++);
        if (!ok) break;
        tc_fence_after();
        uint32_t s[kKt];
        tmem_ld_128cols(s_tm, s);
        if ((j + 1) * kKt > (a.causal ? min(my_row0 + 1, n) : n)) {
          const int valid = (a.causal ? min(row + 1, n) : n) - j * kKt;
#pragma unroll
          for (int e = 0; e < kKt; ++e)
            if (e >= valid) s[e] = 0xFF800000u;  // -inf
        }
        float tops[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int e = 0; e < kKt; e += 2)
          tops[(e >> 1) & 1] = max3(tops[(e >> 1) & 1], __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
        const float top = fmaxf(tops[0], tops[1]) * sc;
        const bool move = top > m + kLazy;
        if (__any_sync(kAllLanes, move)) {
          const float next = move ? top : m;
          const float keep = m == -INFINITY ? 0.f : ex2(m - next);
          m = next;
          sum *= keep;
          if (j > 0) {
#pragma unroll 1
            for (int u = 0; u < D / 16; ++u) {
              uint32_t o[16];
              tmem_ld_16cols(o_tm + 16 * u, o);
              tmem_ld_wait_for(o);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
              tmem_st_16cols(o_tm + 16 * u, o);
            }
          }
        }
        const float mm = m == -INFINITY ? 0.f : m;
        const uint64_t sc2 = pack2(sc, sc), m2 = pack2(-mm, -mm);
        uint64_t part[4] = {0, 0, 0, 0};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t p[16];
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            float x, y;
            unpack2(fma2v(pack2(__uint_as_float(s[32 * q + e]), __uint_as_float(s[32 * q + e + 1])), sc2, m2), x, y);
            x = ex2(x);
            y = ex2(y);
            part[(e >> 1) & 3] = add2_rn(part[(e >> 1) & 3], pack2(x, y));
            p[e / 2] = pack_16<T>(x, y);
          }
          tmem_st_16cols(s_tm + 16 * q, p);
          if (q & 1) {  // the products with these 64 keys may begin
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctrl->p_ready[i][q >> 1]));
          }
        }
        float x, y;
        unpack2(add2_rn(add2_rn(part[0], part[1]), add2_rn(part[2], part[3])), x, y);
        sum += x + y;
      }
      if (ok) ok = wait(&ctrl->o_full[i], no++);
      if (ok) {
        tc_fence_after();
        const float inv = sum > 0.f ? __fdividef(1.f, sum) : 0.f;
        const int64_t t = static_cast<int64_t>(item.first) + row;
#pragma unroll
        for (int q = 0; q < D / 32; ++q) {
          uint32_t o[32];
          tmem_ld_32cols(o_tm + 32 * q, o);
          tmem_ld_wait_for(o);
          if (row < n) {
            uint4* dst = reinterpret_cast<uint4*>(static_cast<T*>(a.out) + t * a.ld_out +
                                                  static_cast<int64_t>(my_head) * D + 32 * q);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t w[4];
#pragma unroll
              for (int k = 0; k < 4; ++k)
                w[k] = pack_16<T>(__uint_as_float(o[8 * e + 2 * k]) * inv, __uint_as_float(o[8 * e + 2 * k + 1]) * inv);
              dst[e] = make_uint4(w[0], w[1], w[2], w[3]);
            }
          }
          __syncwarp();
        }
        if (row < n && a.lse != nullptr) a.lse[t * a.Hq + my_head] = sum > 0.f ? (m + __log2f(sum)) * kLn2 : -INFINITY;
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

int heads_map(CUtensorMap* map, const void* x, int dtype, int64_t rows, int64_t width, int64_t ld) {
  const auto enc = tensor_map_encoder();
  if (enc == nullptr) return OFFQ_ERR_CUDA;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(width), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * 2};
  const cuuint32_t box[2] = {64, 128};
  const cuuint32_t elem_strides[2] = {1, 1};
  const CUresult r = enc(map, dtype == OFFQ_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
                         const_cast<void*>(x), dims, strides, box, elem_strides, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? OFFQ_OK : OFFQ_ERR_CUDA;
}

template <int D, typename T>
int launch_prompt(const AttnArgs& a, int dtype, cudaStream_t s) {
  using L = PromptLayout<D>;
  if (!smem_optin<prompt_kernel<D, T>>(L::kBytes)) return OFFQ_ERR_CUDA;
  CUtensorMap q, k, v;
  if (heads_map(&q, a.q, dtype, a.Tq, static_cast<int64_t>(a.Hq) * D, a.ld_q) != OFFQ_OK ||
      heads_map(&k, a.k, dtype, a.Tq, static_cast<int64_t>(a.H) * D, a.ld_k) != OFFQ_OK ||
      heads_map(&v, a.v, dtype, a.Tq, static_cast<int64_t>(a.H) * D, a.ld_v) != OFFQ_OK)
    return OFFQ_ERR_CUDA;
  const bool two_heads = (a.G & 1) == 0;
  const int64_t step = two_heads ? kQt : 2 * kQt;
  const int64_t tiles = a.Tq / step + std::min<int64_t>(a.B, a.Tq);  // at most: a whole one per step, a ragged one per sequence
  const int64_t grid = tiles * (two_heads ? a.Hq / 2 : a.Hq);
  if (grid > 0x7FFFFFFF) return OFFQ_ERR_UNSUPPORTED;
  return launch_pdl(prompt_kernel<D, T>, dim3(static_cast<unsigned>(grid)), dim3(kThreads), L::kBytes, s, a, q, k, v);
}

}  // namespace

namespace offq {

int prompt_tc(const AttnArgs& a, int dtype, int head_dim, cudaStream_t s) {
  if (head_dim == 128)
    return dtype == OFFQ_BF16 ? launch_prompt<128, __nv_bfloat16>(a, dtype, s) : launch_prompt<128, __half>(a, dtype, s);
  return dtype == OFFQ_BF16 ? launch_prompt<64, __nv_bfloat16>(a, dtype, s) : launch_prompt<64, __half>(a, dtype, s);
}

}  // namespace offq
