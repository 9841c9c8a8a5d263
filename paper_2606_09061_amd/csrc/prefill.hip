// Prefill-chunk attention on bf16 MFMA (v_mfma_f32_32x32x16_bf16).
//
// Prefill is compute bound (Sec. 1 and 2.1 of the paper): a chunk of c
// queries over s prior keys costs ~c*s + c^2/2 query-key pairs per head (the
// prefill_interaction feature of Table 2 tracks exactly that product).
//
// Work item: a tile of up to 32*RG*NW query rows of one chunk, where a row is
// a (token, q head) pair of the G q heads that share one kv head, so K and V
// are gathered once for all G heads (GQA sharing); plus a key range.  Each
// wave owns RG groups of 32 rows that share every K and V operand read.  The
// build uses RG = 1 (RG = 2 needs more registers than a wave can hold without
// spilling the scores), NW = 4 or 8, and two workgroups per CU, so two waves
// share each SIMD.  Per 64-key step and row group a wave computes
//     S^T (64 keys x 32 queries) = K . Q^T      MFMA, fp32 accumulators
//     online softmax down each query column     fp32, base 2
//     O^T (D x 32 queries)     += V^T . P^T     MFMA, P rounded to bf16
// Computing the transposed products keeps one query per lane column, so the
// softmax is lane-local except for one exchange between the two lane halves.
// The rows of the K operand are loaded in a permuted key order (sigma) that
// makes the score registers of a lane exactly the B operand of the P.V step,
// so probabilities never leave registers.  Q^T stays in registers.
//
// Software pipeline inside each wave.  Iteration j has two phases:
//   phase K: S_{j+1} = K_{j+1} . Q^T   interleaved with   P_j = exp2(T_j)
//   phase V: O += V_j . P_j^T          interleaved with   the row sums of P_j,
//            the running max of S_{j+1} and T_{j+1} = S_{j+1} * scale - max
// so the MFMA pipe always has independent VALU work beside it.  The running
// max moves lazily (only when a score exceeds it by 2^8), and the rescale of
// O it then needs is a uniform branch after phase V.
//
// Gather.  K and V tiles are copied from the paged pools straight into LDS
// with global_load_lds_dwordx4 (16 bytes per lane, no VGPR staging), each
// wave a few 1 KiB pieces of one or two blocks per step, with wave-uniform
// block-table entries.  Per-lane source addresses are permuted so the LDS
// tiles land XOR-swizzled (conflict-free MFMA operand reads).  K and V each
// have two LDS buffers, separate arrays so that every access names its buffer
// at compile time.  The copy of a tile is issued 1.5 iterations before it is
// read; every phase starts with a wait on the copies it needs (the only
// waits on them: see copy16_to_lds) and one barrier.
//
// Output.  A lane's accumulators hold half the features of one row, in runs of four;
// stored directly, every store instruction would touch 32 rows.  Instead each
// wave writes its normalised rows into a private slice of the (then idle) K/V
// buffers and stores them back as whole rows, consecutive lanes taking
// consecutive 16-byte pieces of a row.
#include "decode_body.hpp"
#include "device.hpp"
#include "kernels.hpp"
#include "prefill_tile.hpp"

namespace cpattn {

namespace prefill_impl {

// row groups (32 query rows each) per wave
#ifndef CP_PREFILL_RG
#define CP_PREFILL_RG 1
#endif
constexpr int kPrefillRG = CP_PREFILL_RG;

}  // namespace prefill_impl

using namespace prefill_impl;

template <int D, int B, int G, int NW, int RG>
__global__ __launch_bounds__(NW * 64, RG == 1 ? 2 : 1) void prefill_kernel(
    const PrefillRec* __restrict__ recs, const uint16_t* __restrict__ q,
    const uint16_t* __restrict__ k_cache, const uint16_t* __restrict__ v_cache,
    const int32_t* __restrict__ bt, uint16_t* __restrict__ out, float* __restrict__ part_o,
    float* __restrict__ part_lse, int hq, int hkv, int mbr, float scale_log2,
    const DecodeItem* __restrict__ dec, int n_units) {
  using C = PrefillGeom<D, B, NW>;
  using L = PrefillLayout<D, B>;
  constexpr int NKS = C::NKS, NDT = C::NDT, NQK = C::NQK, NPV = C::NPV, PW = C::PW;
  constexpr int KCH = C::KCH, NBW = C::NBW, kRing = C::kRing;
  constexpr int NP = 16 * RG;  // weight pairs per lane and step
  using T_ = std::true_type;
  using F_ = std::false_type;
  __shared__ __attribute__((aligned(1024))) uint8_t kb0[C::TILE_BYTES];
  __shared__ __attribute__((aligned(1024))) uint8_t kb1[C::TILE_BYTES];
  __shared__ __attribute__((aligned(1024))) uint8_t vb0[C::TILE_BYTES];
  __shared__ __attribute__((aligned(1024))) uint8_t vb1[C::TILE_BYTES];

  // this workgroup's record (the grid is the record list, in the planner's
  // XCD-interleaved order); records with no tokens are idle padding
  const PrefillRec it = recs[blockIdx.x];
  if (it.n_tok == kDecodeBlock) {
    // NW / 4 decode units, one per group of four waves, each on LDS buffers
    // of its own (a decode block copies no tiles); the decode rows' K/V
    // stream from HBM while the tiles' workgroups keep the matrix cores busy
    using DL = decode_impl::DecodeLds<D, G>;
    static_assert(DL::O_BYTES <= C::TILE_BYTES && DL::SMALL_BYTES <= C::TILE_BYTES, "decode LDS");
    static_assert(NW == 4 || NW == 8, "decode groups");
    const int grp = uniform((int)threadIdx.x >> 8);
    const int u = grp == 0 ? it.tok0 : it.pos0;
    const bool active = u >= 0 && u < n_units;
    DecodeItem di{0, 0, 0, 0, -1, 0, 0, 0};
    if (active) di = dec[u / hkv];
    decode_unit<D, B, G>(di, active ? u % hkv : 0, active, (int)threadIdx.x & 255, q, k_cache,
                         v_cache, bt, out, part_o, part_lse, hq, hkv, mbr, scale_log2,
                         decode_impl::DecodeLdsPtrs{reinterpret_cast<float*>(grp == 0 ? kb0 : kb1),
                                                    grp == 0 ? vb0 : vb1});
    return;
  }
  if (it.n_tok <= 0) return;
  using Vis = CausalVis;
  [[maybe_unused]] const Vis vis{};
#include "prefill_tile.inc"
}

template <int D, int B, int G, int NW>
static hipError_t launch_prefill_t(const PrefillRec* recs, int n, int n_units, const AttnArgs& a,
                                   hipStream_t s) {
  hipLaunchKernelGGL((prefill_kernel<D, B, G, NW, kPrefillRG>), dim3(n), dim3(NW * 64), 0, s, recs,
                     a.q, a.k_cache, a.v_cache, a.bt, a.out, a.part_o, a.part_lse, a.hq, a.hkv,
                     a.mbr, a.scale_log2, a.decode, n_units);
  return hipGetLastError();
}

template <int D, int B, int NW>
static hipError_t launch_prefill_g(int G, const PrefillRec* recs, int n, int n_units,
                                   const AttnArgs& a, hipStream_t s) {
  switch (G) {
    case 1: return launch_prefill_t<D, B, 1, NW>(recs, n, n_units, a, s);
    case 2: return launch_prefill_t<D, B, 2, NW>(recs, n, n_units, a, s);
    case 4: return launch_prefill_t<D, B, 4, NW>(recs, n, n_units, a, s);
    case 8: return launch_prefill_t<D, B, 8, NW>(recs, n, n_units, a, s);
  }
  return hipErrorInvalidValue;
}

template <int NW>
static hipError_t launch_prefill_w(int D, int G, const PrefillRec* recs, int n, int n_units,
                                   const AttnArgs& a, hipStream_t s) {
  if (D == 128 && a.block_size == 16) return launch_prefill_g<128, 16, NW>(G, recs, n, n_units, a, s);
  if (D == 128 && a.block_size == 32) return launch_prefill_g<128, 32, NW>(G, recs, n, n_units, a, s);
  if (D == 64 && a.block_size == 16) return launch_prefill_g<64, 16, NW>(G, recs, n, n_units, a, s);
  if (D == 64 && a.block_size == 32) return launch_prefill_g<64, 32, NW>(G, recs, n, n_units, a, s);
  return hipErrorInvalidValue;
}

// 256-row and 128-row tiles: 32 * kPrefillRG rows per wave; one workgroup per
// record.  The launch the plan names also runs the decode units.
hipError_t launch_prefill(int D, int G, const AttnArgs& a, hipStream_t s) {
  constexpr int kWide = kPrefillRowsWide / (32 * kPrefillRG), kNarrow = kPrefillRows / (32 * kPrefillRG);
  const int units = a.n_decode * a.hkv;
  hipError_t e = hipSuccess;
  if (a.n_prefill_wide_items > 0)
    e = launch_prefill_w<kWide>(D, G, a.prefill_wide, a.n_prefill_wide_items,
                                a.decode_in_prefill == 2 ? units : 0, a, s);
  if (e == hipSuccess && a.n_prefill_items > 0)
    e = launch_prefill_w<kNarrow>(D, G, a.prefill, a.n_prefill_items,
                                  a.decode_in_prefill == 1 ? units : 0, a, s);
  return e;
}

}  // namespace cpattn
