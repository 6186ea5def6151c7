// quant_matmul_64.cu -- e2_quant_matmul for a few tokens, groups of 64 columns.
#include "quant_matmul.cuh"

int e2ops::launch_few_64(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s)
{
    return launch_few_group<64>(q, f, dev, s);
}
