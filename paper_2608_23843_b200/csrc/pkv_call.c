/* The calls that a decode step makes for every layer, for the Python binding: whole numbers in, a status out.  (Through ctypes twenty
 * arguments take 3 us, as long as the launch itself.)  Pointers arrive as numbers, None is NULL. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "pkv.h"

/* One number for each letter of `kinds`: p a pointer (None is NULL), i of 32 bits, l of 64 */
static int numbers(PyObject *const *args, Py_ssize_t n_args, long long *v, const char *kinds, int n) {
    if (n_args != n) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, not %zd", n, n_args);
        return 0;
    }
    for (int i = 0; i < n; ++i) {
        v[i] = 0;
        if (args[i] == Py_None && kinds[i] == 'p') continue;
        v[i] = PyLong_AsLongLong(args[i]);
        if (v[i] == -1 && PyErr_Occurred()) return 0;
        if (kinds[i] == 'i' && (v[i] > INT32_MAX || v[i] < INT32_MIN)) {
            PyErr_Format(PyExc_OverflowError, "argument %d does not fit 32 bits", i);
            return 0;
        }
    }
    return 1;
}

#define AT(type, i) ((type *)(intptr_t)v[i])
#define I32(i) ((int32_t)v[i])
#define CACHE AT(pkv_q4_cache, 0)
#define FUNCTION(name, kinds, call)                                                            \
    static PyObject *name(PyObject *self, PyObject *const *args, Py_ssize_t n_args) {          \
        long long v[sizeof kinds - 1];                                                         \
        pkv_status st;                                                                         \
        (void)self;                                                                            \
        if (!numbers(args, n_args, v, kinds, (int)sizeof kinds - 1)) return NULL;              \
        Py_BEGIN_ALLOW_THREADS st = call;                                                      \
        Py_END_ALLOW_THREADS return PyLong_FromLong(st);                                       \
    }

/* handle, n_seqs, page_table, max_pages, lengths, n_rows, offsets, k, row, head, v, row, head, stream */
FUNCTION(append_kv, "pipiplppllpllp",
         pkv_q4_append_kv(CACHE, I32(1), AT(const int32_t, 2), I32(3), AT(const int32_t, 4), v[5], AT(const int32_t, 6), AT(const void, 7), v[8], v[9],
                          AT(const void, 10), v[11], v[12], AT(void, 13)))
FUNCTION(read_kv, "pipiplppllpllp",
         pkv_q4_read_kv(CACHE, I32(1), AT(const int32_t, 2), I32(3), AT(const int32_t, 4), v[5], AT(const int32_t, 6), AT(void, 7), v[8], v[9],
                        AT(void, 10), v[11], v[12], AT(void, 13)))
/* handle, n_seqs, page_table, max_pages, lengths, n_rows, offsets, max_q_len, max_len, q, row, head, out, row, head, state, workspace, bytes, stream */
FUNCTION(attention, "pipiplpiipllpllpplp",
         pkv_q4_attention(CACHE, I32(1), AT(const int32_t, 2), I32(3), AT(const int32_t, 4), v[5], AT(const int32_t, 6), I32(7), I32(8),
                          AT(const void, 9), v[10], v[11], AT(void, 12), v[13], v[14], AT(float, 15), AT(void, 16), v[17], AT(void, 18)))
/* ... as above, then window, sinks, tree, tree_words */
static pkv_status select_call(const long long *v) {
    const pkv_q4_select sel = {I32(19), I32(20), AT(const uint64_t, 21), I32(22)};
    return pkv_q4_attention_select(CACHE, I32(1), AT(const int32_t, 2), I32(3), AT(const int32_t, 4), v[5], AT(const int32_t, 6), I32(7), I32(8), &sel,
                                   AT(const void, 9), v[10], v[11], AT(void, 12), v[13], v[14], AT(float, 15), AT(void, 16), v[17], AT(void, 18));
}
FUNCTION(attention_select, "pipiplpiipllpllpplpiipi", select_call(v))
/* handle, n_seqs, lengths, n_rows, offsets, max_q_len, parents, window, sinks, tree, tree_words, depths, stream */
FUNCTION(tree_masks, "piplpipiipipp",
         pkv_q4_tree_masks(CACHE, I32(1), AT(const int32_t, 2), v[3], AT(const int32_t, 4), I32(5), AT(const int32_t, 6), I32(7), I32(8),
                           AT(uint64_t, 9), I32(10), AT(int32_t, 11), AT(void, 12)))
/* handle, n_seqs, page_table, max_pages, lengths, n_rows, offsets, paths, max_path, counts, lengths_out, stream */
FUNCTION(keep_rows, "pipiplppippp",
         pkv_q4_keep_rows(CACHE, I32(1), AT(const int32_t, 2), I32(3), AT(const int32_t, 4), v[5], AT(const int32_t, 6), AT(const int32_t, 7), I32(8),
                          AT(const int32_t, 9), AT(int32_t, 10), AT(void, 11)))
/* handle, n_seqs, page_table, max_pages, lengths, rows, spans, ring, counters, window, sinks, lengths_out, spans_out, counters_out, offsets, n_rows,
 * positions, slots, workspace, bytes, stream */
FUNCTION(plan, "pipipppppiipppplppplp",
         pkv_q4_plan(CACHE, I32(1), AT(int32_t, 2), I32(3), AT(const int32_t, 4), AT(const int32_t, 5), AT(const int32_t, 6), AT(int32_t, 7),
                     AT(const int64_t, 8), I32(9), I32(10), AT(int32_t, 11), AT(int32_t, 12), AT(int64_t, 13), AT(int32_t, 14), v[15], AT(int32_t, 16),
                     AT(int64_t, 17), AT(void, 18), v[19], AT(void, 20)))

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef entries[] = {ENTRY(append_kv), ENTRY(read_kv), ENTRY(attention), ENTRY(attention_select), ENTRY(tree_masks), ENTRY(keep_rows), ENTRY(plan), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pkvcall", "Calls of libpkv.so with whole numbers for arguments.", -1, entries, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__pkvcall(void) { return PyModule_Create(&module); }
