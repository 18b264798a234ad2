// Host-side helpers of the C boundary shared by its translation units (defined in qf_api.cu).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>

#include "../../include/qf.h"
#include "qf_common.cuh"

namespace qf_host {

int validate(const qf_params *p);                        // QF_OK or the error code of these parameters
qf::DevParams dev_params(const qf_params *p);
int check_device(int *sm_count);                         // the current device is a compute-capability 10.x part
int cuda_fail(cudaError_t e, const char *what);          // records the text, returns QF_ERR_CUDA
char *cuda_msg(size_t *len);                             // the buffer qf_strerror(QF_ERR_CUDA) reads
void set_launches(int n);                                // what qf_last_launch_count reports

}  // namespace qf_host
