#include <type_traits>
#include "kernels_linear_dma.h"
using namespace afno;
void go(GemmArgs<bf16> g){ hipLaunchKernelGGL((gemm_dma_any<false,true,256,256,128,64,1>),dim3(8),dim3(256),0,0,g); }
