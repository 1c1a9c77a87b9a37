/* What the Python entry points of the context-free operators know of a tensor, and how it is had from torch (ops_tensor.cpp). */
#pragma once
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "../../include/ditango.h"

enum { MAX_DIM = 8 };
enum { T_BF16 = DT_VALUE_BF16, T_FP16 = DT_VALUE_FP16, T_FP32 = DT_VALUE_FP32, T_FP64, T_I32, T_U8, T_BOOL, T_E4M3, T_COUNT, T_OTHER = -1 };

typedef struct {
    int64_t shape[MAX_DIM], stride[MAX_DIM];
    void *ptr;
    int nd, dtype;
    long device;   /* -1: the host's memory */
} Tensor;

#ifdef __cplusplus
extern "C" {
#endif
extern const char *const tensor_torch_version;   /* the whole one, of the headers */
/* 1; 0: not of torch's own class (its Python attributes count); -1 with an error set */
int tensor_look(PyObject *o, Tensor *x);
/* 0, or -1 with an error set */
int torch_current_device(long *device);
int torch_current_stream(long device, void **stream);
#ifdef __cplusplus
}
#endif
