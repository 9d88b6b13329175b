// Prompts, and chunks of new tokens, over caches in pages (adsa_prefill_paged).  The kernels are those of dense caches but for where rows are read (Tile, Flow and
// prompt_mass in prompt_device.h, PAGED); every workgroup first looks at the table's entries of all slots of its sequence.
#include "prompt_device.h"

namespace adsa {
namespace {

template <int EB, int D, int WK, bool MOD>
__global__ __launch_bounds__(WK * kWave, (kWavesPerSimd<EB, D>)) void k_paged_prompt(PagedPromptArgs A) { prompt_tile<EB, D, WK, MOD, true>(A); }
template <int D, int W, int MODS, bool SPLIT>
__global__ __launch_bounds__(W * kWave, (kFlowWaves<D, MODS, SPLIT>)) void k_paged_prompt_many(PagedPromptArgs A) { prompt_flow<D, W, MODS, SPLIT, true>(A); }
template <int EB, int D, bool MOD>
__global__ __launch_bounds__(256, EB == 2 ? 2 : 1) void k_paged_prompt_mass(PagedPromptArgs A, int key_tiles) { prompt_mass<EB, D, MOD, true>(A, key_tiles); }

struct PagedKernels {
  static constexpr bool kPaged = true;
  template <int EB, int D, int WK, bool MOD> static auto tile() { return k_paged_prompt<EB, D, WK, MOD>; }
  template <int D, int W, int MODS, bool SPLIT> static auto flow() { return k_paged_prompt_many<D, W, MODS, SPLIT>; }
  template <int EB, int D, bool MOD> static auto mass() { return k_paged_prompt_mass<EB, D, MOD>; }
};

}  // namespace

hipError_t paged_prompt_prepare_kernels() {
  hipError_t e = hipSuccess;
  for (int dtype : {ADSA_F32, ADSA_BF16})
    for (int d : {64, 128})
      for (bool mod : {false, true}) {
        adsa_params p = {};
        p.dtype = dtype;
        p.head_dim = d;
        (void)by_type(p, mod, [&](auto eb, auto hd, auto m) {
          allow_prompt_lds<PagedKernels, decltype(eb)::value, decltype(hd)::value, decltype(m)::value>([&](auto kernel, int bytes) {
            if (e == hipSuccess) e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
          });
          return e;
        });
      }
  return e;
}

hipError_t launch_prefill_paged(const adsa_params& p, const PageArgs& pages, const adsa_tokens& t, const adsa_mods& mods, const PromptPlan& plan, adsa_seq* seqs,
                                const void* q, void* out, float* lse, char* ws, const PromptWorkspace& w, bool accumulate, bool advance, bool split,
                                hipStream_t st) {
  PagedPromptArgs A = {};
  fill_prompt_args(A, p, t, mods, plan, seqs, q, out, lse, ws, w, accumulate, advance);
  A.pages = pages;
  A.slot_stride_b = pages.slot_stride_b;
  A.head_stride_b = pages.head_stride_b;
  return by_type(p, modded(A.mods), [&](auto eb, auto d, auto m) {
    return prompt_launches<PagedKernels, decltype(eb)::value, decltype(d)::value, decltype(m)::value>(A, plan, split, st);
  });
}

}  // namespace adsa
