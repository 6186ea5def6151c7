// quant_matmul_f16.cu -- e2_quant_matmul for a few tokens, x in f16.
#include "quant_matmul.cuh"

int e2ops::launch_few_f16(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s)
{
    return launch_type<__half>(q, f, dev, s);
}
