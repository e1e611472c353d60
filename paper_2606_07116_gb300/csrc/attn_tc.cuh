// Pieces that the tensor-core attention kernels share: tiles of 128 query rows by 128 keys, scores and
// outputs in tensor memory, one softmax thread per row.
#pragma once

#include <type_traits>

#include "attn.cuh"

namespace offq {

constexpr int kQt = 128;   // query rows of a tile
constexpr int kKt = 128;   // keys of a block
constexpr int kAtom = 128 * 128;  // bytes of 128 rows of one 128-byte swizzle atom (64 channels of 16 bits)

// kind::f16 with fp32 sums: bf16 (1) or f16 (0) operands at bits 7-9 and 10-12, bit 16 set where B's rows are
// contracted (its other dimension is contiguous), N >> 3 at 17, M >> 4 at 24.
template <typename T>
__host__ __device__ constexpr uint32_t idesc_16(int M, int N, bool b_mn_major) {
  const uint32_t f = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
  return (1u << 4) | (f << 7) | (f << 10) | (b_mn_major ? 1u << 16 : 0u) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(M >> 4) << 24);
}

// Descriptor of a [128 keys][D channels] value tile as a B operand contracted over the keys: 128-byte swizzle,
// 64 contiguous channels per row, 8-key groups 1024 bytes apart (bits 32-45), the two halves of 128 channels one
// atom apart (bits 16-29).
__device__ __forceinline__ uint64_t smem_desc_rows_contracted(uint32_t saddr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(kAtom >> 4) << 16;
  d |= static_cast<uint64_t>(1024u >> 4) << 32;
  d |= static_cast<uint64_t>(1u) << 46;
  d |= static_cast<uint64_t>(2u) << 61;
  return d;
}

// D[tmem] (+)= A[tmem] * B[smem], 16-bit operands.
__device__ __forceinline__ void mma_16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                          uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// The lanes for which `yes` holds arrive, and the warp stays together: the instruction is predicated, not branched around.
__device__ __forceinline__ void mbar_arrive_if(uint32_t bar, bool yes) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.u32 p, %1, 0;\n"
      "@p mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];\n"
      "}\n" ::"r"(bar),
      "r"(static_cast<uint32_t>(yes))
      : "memory");
}

// Each thread of the warp reads 128 consecutive 32-bit columns of its TMEM lane; they are there when it returns.
__device__ __forceinline__ void tmem_ld_128cols(uint32_t taddr, uint32_t (&r)[128]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%128];\n"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,"
      "%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%129];\n"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%64,%65,%66,%67,%68,%69,%70,%71,%72,%73,%74,%75,%76,%77,%78,%79,"
      "%80,%81,%82,%83,%84,%85,%86,%87,%88,%89,%90,%91,%92,%93,%94,%95}, [%130];\n"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%96,%97,%98,%99,%100,%101,%102,%103,%104,%105,%106,%107,%108,%109,%110,%111,"
      "%112,%113,%114,%115,%116,%117,%118,%119,%120,%121,%122,%123,%124,%125,%126,%127}, [%131];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=&r"(r[0]), "=&r"(r[1]), "=&r"(r[2]), "=&r"(r[3]), "=&r"(r[4]), "=&r"(r[5]), "=&r"(r[6]), "=&r"(r[7]),
        "=&r"(r[8]), "=&r"(r[9]), "=&r"(r[10]), "=&r"(r[11]), "=&r"(r[12]), "=&r"(r[13]), "=&r"(r[14]), "=&r"(r[15]),
        "=&r"(r[16]), "=&r"(r[17]), "=&r"(r[18]), "=&r"(r[19]), "=&r"(r[20]), "=&r"(r[21]), "=&r"(r[22]), "=&r"(r[23]),
        "=&r"(r[24]), "=&r"(r[25]), "=&r"(r[26]), "=&r"(r[27]), "=&r"(r[28]), "=&r"(r[29]), "=&r"(r[30]), "=&r"(r[31]),
        "=&r"(r[32]), "=&r"(r[33]), "=&r"(r[34]), "=&r"(r[35]), "=&r"(r[36]), "=&r"(r[37]), "=&r"(r[38]), "=&r"(r[39]),
        "=&r"(r[40]), "=&r"(r[41]), "=&r"(r[42]), "=&r"(r[43]), "=&r"(r[44]), "=&r"(r[45]), "=&r"(r[46]), "=&r"(r[47]),
        "=&r"(r[48]), "=&r"(r[49]), "=&r"(r[50]), "=&r"(r[51]), "=&r"(r[52]), "=&r"(r[53]), "=&r"(r[54]), "=&r"(r[55]),
        "=&r"(r[56]), "=&r"(r[57]), "=&r"(r[58]), "=&r"(r[59]), "=&r"(r[60]), "=&r"(r[61]), "=&r"(r[62]), "=&r"(r[63]),
        "=&r"(r[64]), "=&r"(r[65]), "=&r"(r[66]), "=&r"(r[67]), "=&r"(r[68]), "=&r"(r[69]), "=&r"(r[70]), "=&r"(r[71]),
        "=&r"(r[72]), "=&r"(r[73]), "=&r"(r[74]), "=&r"(r[75]), "=&r"(r[76]), "=&r"(r[77]), "=&r"(r[78]), "=&r"(r[79]),
        "=&r"(r[80]), "=&r"(r[81]), "=&r"(r[82]), "=&r"(r[83]), "=&r"(r[84]), "=&r"(r[85]), "=&r"(r[86]), "=&r"(r[87]),
        "=&r"(r[88]), "=&r"(r[89]), "=&r"(r[90]), "=&r"(r[91]), "=&r"(r[92]), "=&r"(r[93]), "=&r"(r[94]), "=&r"(r[95]),
        "=&r"(r[96]), "=&r"(r[97]), "=&r"(r[98]), "=&r"(r[99]), "=&r"(r[100]), "=&r"(r[101]), "=&r"(r[102]), "=&r"(r[103]),
        "=&r"(r[104]), "=&r"(r[105]), "=&r"(r[106]), "=&r"(r[107]), "=&r"(r[108]), "=&r"(r[109]), "=&r"(r[110]), "=&r"(r[111]),
        "=&r"(r[112]), "=&r"(r[113]), "=&r"(r[114]), "=&r"(r[115]), "=&r"(r[116]), "=&r"(r[117]), "=&r"(r[118]), "=&r"(r[119]),
        "=&r"(r[120]), "=&r"(r[121]), "=&r"(r[122]), "=&r"(r[123]), "=&r"(r[124]), "=&r"(r[125]), "=&r"(r[126]), "=&r"(r[127])
      : "r"(taddr), "r"(taddr + 32), "r"(taddr + 64), "r"(taddr + 96)
      : "memory");
}

// The largest of three.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// 32 rows x 32 columns as fragments: with g = lane / 4 and c = lane % 4, r{h}[4 k + 2 i + e] is row 16 h + 8 i + g,
// column 8 k + 2 c + e (k < 4). A thread then meets a quarter of the columns instead of all.
__device__ __forceinline__ void tmem_ld_fragments(uint32_t taddr, uint32_t (&r0)[16], uint32_t (&r1)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%32];\n"
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%33];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=&r"(r0[0]), "=&r"(r0[1]), "=&r"(r0[2]), "=&r"(r0[3]), "=&r"(r0[4]), "=&r"(r0[5]), "=&r"(r0[6]), "=&r"(r0[7]),
        "=&r"(r0[8]), "=&r"(r0[9]), "=&r"(r0[10]), "=&r"(r0[11]), "=&r"(r0[12]), "=&r"(r0[13]), "=&r"(r0[14]), "=&r"(r0[15]),
        "=&r"(r1[0]), "=&r"(r1[1]), "=&r"(r1[2]), "=&r"(r1[3]), "=&r"(r1[4]), "=&r"(r1[5]), "=&r"(r1[6]), "=&r"(r1[7]),
        "=&r"(r1[8]), "=&r"(r1[9]), "=&r"(r1[10]), "=&r"(r1[11]), "=&r"(r1[12]), "=&r"(r1[13]), "=&r"(r1[14]), "=&r"(r1[15])
      : "r"(taddr), "r"(taddr + (16u << 16))
      : "memory");
}
__device__ __forceinline__ void tmem_st_fragments(uint32_t taddr, const uint32_t (&r)[16]) {  // one half's 16 rows
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// Pairs of columns packed into 32-bit columns: row 8 i + g of the 16, 32-bit column 4 k + c: r[2 k + i], k < 4.
__device__ __forceinline__ void tmem_st_pairs(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
      : "memory");
}
__device__ __forceinline__ void tmem_ld_pairs(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x128b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
      : "r"(taddr)
      : "memory");
}

// Registers per thread of this warpgroup from here on (multiples of 8; the shares of all warpgroups add up to no
// more than the launch's).
template <int N>
__device__ __forceinline__ void more_registers() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void fewer_registers() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

template <typename T>
__device__ __forceinline__ uint32_t pack_16(float a, float b) {
  if constexpr (std::is_same<T, __nv_bfloat16>::value) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
}

// A pair of halves times k.
__device__ __forceinline__ uint32_t scale_halves(uint32_t w, float k) {
  const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w));
  return pack_16<__half>(v.x * k, v.y * k);
}

__device__ __forceinline__ uint64_t add2_rn(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

__device__ __forceinline__ void sts_zero16(uint32_t addr) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(addr), "r"(0u) : "memory");
}

}  // namespace offq
