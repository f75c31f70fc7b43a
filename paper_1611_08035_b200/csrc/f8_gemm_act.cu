// The products with an epilogue (b2_gemm_f8_act): the small kernels of f8_small.cuh with the results of f8_act.cuh.
#include "f8_small.cuh"

namespace b2 {

template int f8_choose<float, true>(const F8ArgsOf<F8ActOut>&, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);
template int f8_choose<float, false>(const F8ArgsOf<F8ActOut>&, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);
template int f8_choose<__nv_bfloat16, true>(const F8ArgsOf<F8ActOut>&, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);
template int f8_choose<__nv_bfloat16, false>(const F8ArgsOf<F8ActOut>&, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);

}  // namespace b2
