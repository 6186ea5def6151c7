// quant_matmul_128.cu -- e2_quant_matmul for a few tokens, groups of 128 columns.
#include "quant_matmul.cuh"

int e2ops::launch_few_128(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s)
{
    return launch_few_group<128>(q, f, dev, s);
}
