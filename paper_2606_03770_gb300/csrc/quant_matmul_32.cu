// quant_matmul_32.cu -- e2_quant_matmul for a few tokens, groups of 32 columns.
#include "quant_matmul.cuh"

int e2ops::launch_few_32(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s)
{
    return launch_few_group<32>(q, f, dev, s);
}
