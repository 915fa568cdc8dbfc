/* kvs_tensor.h -- what the binding's extension reads of a tensor, and the form of its reader in C++. */
#ifndef KVS_TENSOR_H
#define KVS_TENSOR_H

#include <Python.h>

#include <stdint.h>

typedef struct {
    uint64_t at;
    int64_t  shape[4], stride[4];
} kvs_tensor;

/* A tensor of `dims` (at most 4) dimensions and of that dtype: 1; a tensor of other ones: 0; an object that the
 * reader does not know, whose attributes then tell: 2.  Raises nothing. */
typedef int (*kvs_read_tensor_fn)(PyObject* o, PyObject* dtype, int dims, kvs_tensor* out);

#endif
