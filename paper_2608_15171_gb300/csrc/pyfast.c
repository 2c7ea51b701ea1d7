/*
 * _ppasfast: a CPython extension with the calls a serving loop makes on every
 * layer or every step, ppas_kv_append, ppas_rope_append, ppas_attention_step,
 * ppas_shared_attention_step and ppas_sample_tokens, forwarding to the C ABI of
 * libppas.so (include/ppas.h) with argument marshalling only.
 *
 * ctypes spends ~12 us of host time converting the 19 arguments of one
 * attention call; a decode-only step of a few rows takes less than that on
 * the GPU per layer, so with ctypes such steps are bound by the host.  Here
 * the arguments are parsed by PyArg_ParseTuple (pointers as Python ints,
 * the per-row length arrays through the buffer protocol: contiguous int32).
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "ppas.h"

static int int32_buffer(const Py_buffer *b, const char *what) {
    if (b->len % 4 != 0 || b->itemsize != 4 || !PyBuffer_IsContiguous(b, 'C')) {
        PyErr_Format(PyExc_TypeError, "%s must be a contiguous int32 buffer", what);
        return 0;
    }
    return 1;
}

/* attention_step(q, k_cache, v_cache, num_blocks, d_block_tables,
 *                max_blocks_per_seq, q_lens, ctx_lens, n_q_heads, n_kv_heads,
 *                head_dim, scale, out, out_is_fp32, workspace,
 *                workspace_bytes, d_err_flag, stream) -> ppas_status */
static PyObject *py_attention_step(PyObject *self, PyObject *args) {
    unsigned long long q, k, v, tables, out, ws, ws_bytes, err, stream;
    int num_blocks, width, hq, hk, d, out_fp32;
    float scale;
    Py_buffer ql, cl;
    (void)self;
    if (!PyArg_ParseTuple(args, "KKKiKiy*y*iiifKiKKKK", &q, &k, &v, &num_blocks, &tables, &width, &ql, &cl, &hq,
                          &hk, &d, &scale, &out, &out_fp32, &ws, &ws_bytes, &err, &stream))
        return NULL;
    PyObject *res = NULL;
    if (int32_buffer(&ql, "q_lens") && int32_buffer(&cl, "ctx_lens")) {
        if (ql.len != cl.len) {
            PyErr_SetString(PyExc_ValueError, "q_lens and ctx_lens differ in length");
        } else {
            const ppas_status st = ppas_attention_step(
                (const void *)(uintptr_t)q, (const void *)(uintptr_t)k, (const void *)(uintptr_t)v, num_blocks,
                (const int32_t *)(uintptr_t)tables, width, (const int32_t *)ql.buf, (const int32_t *)cl.buf,
                (int32_t)(ql.len / 4), hq, hk, d, scale, (void *)(uintptr_t)out, out_fp32, (void *)(uintptr_t)ws,
                (size_t)ws_bytes, (int32_t *)(uintptr_t)err, (void *)(uintptr_t)stream);
            res = PyLong_FromLong((long)st);
        }
    }
    PyBuffer_Release(&ql);
    PyBuffer_Release(&cl);
    return res;
}

/* kv_append(k_new, v_new, d_slot_mapping, n_tokens, k_cache, v_cache,
 *           num_blocks, n_kv_heads, head_dim, d_err_flag, stream) -> ppas_status */
static PyObject *py_kv_append(PyObject *self, PyObject *args) {
    unsigned long long kn, vn, slots, kc, vc, err, stream;
    int n_tokens, num_blocks, hk, d;
    (void)self;
    if (!PyArg_ParseTuple(args, "KKKiKKiiiKK", &kn, &vn, &slots, &n_tokens, &kc, &vc, &num_blocks, &hk, &d, &err,
                          &stream))
        return NULL;
    const ppas_status st = ppas_kv_append((const void *)(uintptr_t)kn, (const void *)(uintptr_t)vn,
                                          (const int32_t *)(uintptr_t)slots, n_tokens, (void *)(uintptr_t)kc,
                                          (void *)(uintptr_t)vc, num_blocks, hk, d, (int32_t *)(uintptr_t)err,
                                          (void *)(uintptr_t)stream);
    return PyLong_FromLong((long)st);
}

/* rope_append(q, k, v, q_stride, k_stride, v_stride, d_positions,
 *             d_slot_mapping, n_tokens, d_inv_freq, rotary_dim, interleaved,
 *             factor, q_out, k_cache, v_cache, num_blocks, n_q_heads,
 *             n_kv_heads, head_dim, d_err_flag, stream) -> ppas_status */
static PyObject *py_rope_append(PyObject *self, PyObject *args) {
    unsigned long long q, k, v, pos, slots, freq, qo, kc, vc, err, stream;
    long long qs, ks, vs;
    int n_tokens, rotary, inter, num_blocks, hq, hk, d;
    float factor;
    (void)self;
    if (!PyArg_ParseTuple(args, "KKKLLLKKiKiifKKKiiiiKK", &q, &k, &v, &qs, &ks, &vs, &pos, &slots, &n_tokens, &freq,
                          &rotary, &inter, &factor, &qo, &kc, &vc, &num_blocks, &hq, &hk, &d, &err, &stream))
        return NULL;
    const ppas_status st = ppas_rope_append(
        (const void *)(uintptr_t)q, (const void *)(uintptr_t)k, (const void *)(uintptr_t)v, qs, ks, vs,
        (const int32_t *)(uintptr_t)pos, (const int32_t *)(uintptr_t)slots, n_tokens, (const float *)(uintptr_t)freq,
        rotary, inter, factor, (void *)(uintptr_t)qo, (void *)(uintptr_t)kc, (void *)(uintptr_t)vc, num_blocks, hq, hk,
        d, (int32_t *)(uintptr_t)err, (void *)(uintptr_t)stream);
    return PyLong_FromLong((long)st);
}

/* sample_tokens(logits, logits_are_bf16, row_stride, n_rows, vocab,
 *               d_temperature, d_top_k, d_top_p, d_min_p, d_uniform, d_tokens,
 *               d_logprobs, d_err_flag, stream) -> ppas_status */
static PyObject *py_sample_tokens(PyObject *self, PyObject *args) {
    unsigned long long x, t, k, p, m, u, tok, lp, err, stream;
    long long stride;
    int bf16, n_rows, vocab;
    (void)self;
    if (!PyArg_ParseTuple(args, "KiLiiKKKKKKKKK", &x, &bf16, &stride, &n_rows, &vocab, &t, &k, &p, &m, &u, &tok, &lp,
                          &err, &stream))
        return NULL;
    const ppas_status st = ppas_sample_tokens(
        (const void *)(uintptr_t)x, bf16, stride, n_rows, vocab, (const float *)(uintptr_t)t,
        (const int32_t *)(uintptr_t)k, (const float *)(uintptr_t)p, (const float *)(uintptr_t)m,
        (const float *)(uintptr_t)u, (int32_t *)(uintptr_t)tok, (float *)(uintptr_t)lp, (int32_t *)(uintptr_t)err,
        (void *)(uintptr_t)stream);
    return PyLong_FromLong((long)st);
}

/* shared_attention_step(q, k_cache, v_cache, num_blocks, d_block_tables,
 *                       max_blocks_per_seq, group_rows, prefix_lens, ctx_lens,
 *                       n_q_heads, n_kv_heads, head_dim, scale, out, workspace,
 *                       workspace_bytes, d_err_flag, stream) -> ppas_status
 */
static PyObject *py_shared_attention_step(PyObject *self, PyObject *args) {
    unsigned long long q, k, v, tables, out, ws, ws_bytes, err, stream;
    int num_blocks, width, hq, hk, d;
    float scale;
    Py_buffer gr, pl, cl;
    (void)self;
    if (!PyArg_ParseTuple(args, "KKKiKiy*y*y*iiifKKKKK", &q, &k, &v, &num_blocks, &tables, &width, &gr, &pl, &cl, &hq,
                          &hk, &d, &scale, &out, &ws, &ws_bytes, &err, &stream))
        return NULL;
    PyObject *res = NULL;
    if (int32_buffer(&gr, "group_rows") && int32_buffer(&pl, "prefix_lens") && int32_buffer(&cl, "ctx_lens")) {
        /* the C call takes the lengths' number from group_rows */
        long long rows = 0;
        for (Py_ssize_t i = 0; i < gr.len / 4; ++i) rows += ((const int32_t *)gr.buf)[i];
        if (gr.len != pl.len || rows != cl.len / 4) {
            res = PyLong_FromLong(PPAS_ERR_INVALID_ARG);
        } else {
            const ppas_status st = ppas_shared_attention_step(
                (const void *)(uintptr_t)q, (const void *)(uintptr_t)k, (const void *)(uintptr_t)v, num_blocks,
                (const int32_t *)(uintptr_t)tables, width, (int32_t)(gr.len / 4), (const int32_t *)gr.buf,
                (const int32_t *)pl.buf, (const int32_t *)cl.buf, hq, hk, d, scale, (void *)(uintptr_t)out,
                (void *)(uintptr_t)ws, (size_t)ws_bytes, (int32_t *)(uintptr_t)err, (void *)(uintptr_t)stream);
            res = PyLong_FromLong((long)st);
        }
    }
    PyBuffer_Release(&gr);
    PyBuffer_Release(&pl);
    PyBuffer_Release(&cl);
    return res;
}

static PyMethodDef methods[] = {
    {"shared_attention_step", py_shared_attention_step, METH_VARARGS,
     "ppas_shared_attention_step (see include/ppas.h)"},
    {"sample_tokens", py_sample_tokens, METH_VARARGS, "ppas_sample_tokens (see include/ppas.h)"},
    {"rope_append", py_rope_append, METH_VARARGS, "ppas_rope_append (see include/ppas.h)"},
    {"attention_step", py_attention_step, METH_VARARGS, "ppas_attention_step (see include/ppas.h)"},
    {"kv_append", py_kv_append, METH_VARARGS, "ppas_kv_append (see include/ppas.h)"},
    {NULL, NULL, 0, NULL},
};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ppasfast", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__ppasfast(void) { return PyModule_Create(&module); }
