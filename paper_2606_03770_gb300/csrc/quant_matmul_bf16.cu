// quant_matmul_bf16.cu -- e2_quant_matmul for a few tokens, x in bf16.
#include "quant_matmul.cuh"

int e2ops::launch_few_bf16(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s)
{
    return launch_type<__nv_bfloat16>(q, f, dev, s);
}
