// The calls that a decoding loop makes, codegemm_gemm, codegemm_gemm_grouped and those of the cache and of attention, as functions of a Python
// extension module.  Through ctypes such a call spends 2.8 us in the interpreter and in argument conversion before it reaches the library, of the
// 8 us that an eager call of a small layer takes in all (its kernels take 3); here 0.6.  Only the plain form of a call is handled: positional
// arguments, Desc and Plan themselves, tensors (anything with data_ptr()), integer addresses or None.  Every other form, and every
// argument that the plain form refuses, goes to the ctypes functions, which then do and raise what they always did.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <climits>
#include <cstddef>
#include <cstdint>
#include <cstring>
#include <initializer_list>

#include "codegemm.h"

namespace {

typedef int (*gemm_t)(const codegemm_desc*, const codegemm_plan*, const void*, const uint8_t*, const void*, const void*, void*, void*, size_t, void*);
typedef int (*grouped_t)(const codegemm_desc*, const codegemm_plan*, const void*, const codegemm_group_member*, int32_t, void*, size_t, void*);

// Set by prepare() when the binding is imported and by use() when it has loaded a library; with the GIL held, as they are read.
PyTypeObject* desc_type = nullptr;
PyTypeObject* plan_type = nullptr;
PyObject *slow_gemm = nullptr, *slow_grouped = nullptr, *check = nullptr, *data_ptr = nullptr;
gemm_t gemm_at = nullptr;
grouped_t grouped_at = nullptr;
constexpr Py_ssize_t kMaxMembers = 4;

// The bytes of a ctypes structure, held while the view lives.
struct View {
    Py_buffer b;
    bool held = false;
    bool of(PyObject* o, size_t bytes)
    {
        held = PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) == 0;
        return held && (size_t)b.len == bytes;
    }
    ~View() { if (held) PyBuffer_Release(&b); }
};

enum Form { kPlain, kOther, kRaised };

// Address of a tensor, an integer or None.  What a data_ptr() raises is the caller's to see, but for AttributeError, which sends the
// ctypes forms on to int(o).
Form address(PyObject* o, void** at)
{
    if (o == Py_None) { *at = nullptr; return kPlain; }
    if (PyLong_CheckExact(o)) *at = PyLong_AsVoidPtr(o);
    else {
        PyObject* n = PyObject_CallMethodNoArgs(o, data_ptr);
        if (!n) return PyErr_ExceptionMatches(PyExc_AttributeError) ? kOther : kRaised;
        if (!PyLong_CheckExact(n)) { Py_DECREF(n); return kOther; }
        *at = PyLong_AsVoidPtr(n);
        Py_DECREF(n);
    }
    return *at != nullptr || !PyErr_Occurred() ? kPlain : kOther;
}

bool size(PyObject* o, size_t* n)
{
    if (!PyLong_CheckExact(o)) return false;
    *n = PyLong_AsSize_t(o);
    return !(*n == (size_t)-1 && PyErr_Occurred());
}

bool structures(PyObject* d, PyObject* p, View* desc, View* plan)
{
    return Py_TYPE(d) == desc_type && desc->of(d, sizeof(codegemm_desc)) &&
           (p == Py_None || (Py_TYPE(p) == plan_type && plan->of(p, sizeof(codegemm_plan))));
}

PyObject* slowly(PyObject* how, PyObject* const* args, Py_ssize_t nargs, PyObject* names)
{
    if (!how) { PyErr_SetString(PyExc_RuntimeError, "prepare() has not been called"); return nullptr; }
    PyErr_Clear();                                     // whatever stood in the way of the plain form: it will be met again
    return PyObject_Vectorcall(how, args, (size_t)nargs, names);
}

PyObject* result(int status, const char* where)
{
    if (status != 0) return PyObject_CallFunction(check, "is", status, where);
    Py_RETURN_NONE;
}

// (desc, plan, x, packed_codes, codebooks, scales, y, workspace, workspace_bytes, stream=0)
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names)
{
    View desc, plan;
    void *at[6], *stream = nullptr;
    size_t bytes;
    Form form = gemm_at && !names && (n == 9 || n == 10) && structures(a[0], a[1], &desc, &plan) ? kPlain : kOther;
    for (int k = 0; form == kPlain && k < 6; ++k) form = address(a[2 + k], &at[k]);
    if (form == kRaised) return nullptr;
    if (form == kOther || !size(a[8], &bytes) || (n == 10 && !(PyLong_CheckExact(a[9]) && address(a[9], &stream) == kPlain))) return slowly(slow_gemm, a, n, names);
    const gemm_t call = gemm_at;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call(static_cast<const codegemm_desc*>(desc.b.buf), plan.held ? static_cast<const codegemm_plan*>(plan.b.buf) : nullptr, at[0],
                  static_cast<const uint8_t*>(at[1]), at[2], at[3], at[4], at[5], bytes, stream);
    Py_END_ALLOW_THREADS
    return result(status, "codegemm_gemm");
}

// (desc, plan, x, members, workspace, workspace_bytes, stream=0); members: (out_features, packed_codes, codebooks, scales, y) each
PyObject* gemm_grouped(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names)
{
    View desc, plan;
    void *x, *workspace, *stream = nullptr;
    size_t bytes;
    codegemm_group_member group[kMaxMembers] = {};
    int32_t count = 0;
    Form form = grouped_at && !names && (n == 6 || n == 7) && structures(a[0], a[1], &desc, &plan) &&
                (PyList_CheckExact(a[3]) || PyTuple_CheckExact(a[3])) && PySequence_Fast_GET_SIZE(a[3]) <= kMaxMembers ? kPlain : kOther;
    // (a data_ptr() may run any Python, so the list is asked for its length again, and members are held while they are read)
    for (; form == kPlain && count < PySequence_Fast_GET_SIZE(a[3]) && count < kMaxMembers; ++count) {
        PyObject* m = PySequence_Fast_GET_ITEM(a[3], count);
        Py_INCREF(m);
        form = kOther;
        if (PyTuple_CheckExact(m) && PyTuple_GET_SIZE(m) == 5 && PyLong_CheckExact(PyTuple_GET_ITEM(m, 0))) {
            const long rows = PyLong_AsLong(PyTuple_GET_ITEM(m, 0));
            void* at[4];
            if (rows >= INT32_MIN && rows <= INT32_MAX && !(rows == -1 && PyErr_Occurred())) form = kPlain;
            for (int k = 0; form == kPlain && k < 4; ++k) form = address(PyTuple_GET_ITEM(m, 1 + k), &at[k]);
            if (form == kPlain) {
                group[count].out_features = (int32_t)rows;
                group[count].packed_codes = static_cast<const uint8_t*>(at[0]);
                group[count].codebooks = at[1];
                group[count].scales = at[2];
                group[count].y = at[3];
            }
        }
        Py_DECREF(m);
    }
    if (form == kPlain) form = address(a[2], &x);
    if (form == kPlain) form = address(a[4], &workspace);
    if (form == kRaised) return nullptr;
    if (form == kOther || !size(a[5], &bytes) || (n == 7 && !(PyLong_CheckExact(a[6]) && address(a[6], &stream) == kPlain)))
        return slowly(slow_grouped, a, n, names);
    const grouped_t call = grouped_at;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call(static_cast<const codegemm_desc*>(desc.b.buf), plan.held ? static_cast<const codegemm_plan*>(plan.b.buf) : nullptr, x, group, count,
                  workspace, bytes, stream);
    Py_END_ALLOW_THREADS
    return result(status, "codegemm_gemm_grouped");
}

// The calls around the cache.  What each takes in front of its stream: C a cache, A an append's description, T attention's, p an address, i 32 bits,
// z a size.
enum { kAppend, kGather, kDecode, kPrompt, kCalls };
const char* const kTakes[kCalls] = {"CAppppppppp", "Cipppp", "CTpppz", "Tpppppppz"};
const char* const kNames[kCalls] = {"codegemm_kv_append", "codegemm_kv_gather", "codegemm_attn_decode", "codegemm_attn_prompt"};
PyTypeObject *cache_type = nullptr, *append_type = nullptr, *attn_type = nullptr;
PyObject* slow_call[kCalls] = {};
void* call_at[kCalls] = {};

PyObject* attention_call(int which, PyObject* const* a, Py_ssize_t n, PyObject* names)
{
    const char* takes = kTakes[which];
    const Py_ssize_t count = (Py_ssize_t)strlen(takes);
    View view[2];
    void *at[10] = {}, *stream = nullptr;
    size_t bytes = 0;
    long rows = 0;
    Form form = call_at[which] && !names && (n == count || n == count + 1) ? kPlain : kOther;
    int views = 0, addresses = 0;
    for (Py_ssize_t k = 0; form == kPlain && k < count; ++k) {
        PyTypeObject* type = takes[k] == 'C' ? cache_type : takes[k] == 'A' ? append_type : attn_type;
        const size_t size_of = takes[k] == 'C' ? sizeof(codegemm_kv_cache) : takes[k] == 'A' ? sizeof(codegemm_append_desc) : sizeof(codegemm_attn_desc);
        if (takes[k] == 'p') form = address(a[k], &at[addresses++]);
        else if (takes[k] == 'z') form = size(a[k], &bytes) ? kPlain : kOther;
        else if (takes[k] == 'i') {
            rows = PyLong_CheckExact(a[k]) ? PyLong_AsLong(a[k]) : LONG_MIN;
            form = rows >= INT32_MIN && rows <= INT32_MAX && !(rows == -1 && PyErr_Occurred()) ? kPlain : kOther;
        } else if (Py_TYPE(a[k]) != type || !view[views++].of(a[k], size_of)) form = kOther;
    }
    if (form == kRaised) return nullptr;
    if (form == kOther || (n == count + 1 && !(PyLong_CheckExact(a[count]) && address(a[count], &stream) == kPlain))) return slowly(slow_call[which], a, n, names);
    void* const call = call_at[which];
    const void* const first = view[0].b.buf;
    const void* const second = views > 1 ? view[1].b.buf : nullptr;
    int status;
    Py_BEGIN_ALLOW_THREADS
    switch (which) {
    case kAppend:
        status = reinterpret_cast<decltype(&codegemm_kv_append)>(call)(
            static_cast<const codegemm_kv_cache*>(first), static_cast<const codegemm_append_desc*>(second), static_cast<const int32_t*>(at[0]), at[1], at[2], at[3],
            at[4], at[5], static_cast<const float*>(at[6]), at[7], at[8], stream);
        break;
    case kGather:
        status = reinterpret_cast<decltype(&codegemm_kv_gather)>(call)(static_cast<const codegemm_kv_cache*>(first), (int32_t)rows, static_cast<const int32_t*>(at[0]),
                                                                       static_cast<const int32_t*>(at[1]), at[2], at[3], stream);
        break;
    case kDecode:
        status = reinterpret_cast<decltype(&codegemm_attn_decode)>(call)(static_cast<const codegemm_kv_cache*>(first), static_cast<const codegemm_attn_desc*>(second),
                                                                         at[0], at[1], at[2], bytes, stream);
        break;
    default:
        status = reinterpret_cast<decltype(&codegemm_attn_prompt)>(call)(static_cast<const codegemm_attn_desc*>(first), at[0], at[1], at[2],
                                                                         static_cast<const int32_t*>(at[3]), static_cast<const int32_t*>(at[4]), at[5], at[6], bytes, stream);
    }
    Py_END_ALLOW_THREADS
    return result(status, kNames[which]);
}
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names) { return attention_call(kAppend, a, n, names); }
PyObject* kv_gather(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names) { return attention_call(kGather, a, n, names); }
PyObject* attn_decode(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names) { return attention_call(kDecode, a, n, names); }
PyObject* attn_prompt(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names) { return attention_call(kPrompt, a, n, names); }

// (KvCache, AppendDesc, AttnDesc, the ctypes forms of the four calls)
PyObject* prepare_attention(PyObject*, PyObject* args)
{
    PyObject *c, *d, *t, *slow[kCalls];
    if (!PyArg_ParseTuple(args, "O!O!O!OOOO", &PyType_Type, &c, &PyType_Type, &d, &PyType_Type, &t, &slow[0], &slow[1], &slow[2], &slow[3])) return nullptr;
    for (PyObject* o : {c, d, t}) Py_INCREF(o);                         // for the life of the process
    cache_type = reinterpret_cast<PyTypeObject*>(c);
    append_type = reinterpret_cast<PyTypeObject*>(d);
    attn_type = reinterpret_cast<PyTypeObject*>(t);
    for (int k = 0; k < kCalls; ++k) {
        Py_INCREF(slow[k]);
        slow_call[k] = slow[k];
    }
    Py_RETURN_NONE;
}

// (addresses of codegemm_kv_append, codegemm_kv_gather, codegemm_attn_decode, codegemm_attn_prompt)
PyObject* use_attention(PyObject*, PyObject* args)
{
    unsigned long long at[kCalls];
    if (!PyArg_ParseTuple(args, "KKKK", &at[0], &at[1], &at[2], &at[3])) return nullptr;
    for (int k = 0; k < kCalls; ++k) call_at[k] = reinterpret_cast<void*>(static_cast<uintptr_t>(at[k]));
    Py_RETURN_NONE;
}

// (Desc, Plan, the ctypes forms of the two calls, what raises for a status)
PyObject* prepare(PyObject*, PyObject* args)
{
    PyObject *d, *p, *one, *group, *raise;
    if (!PyArg_ParseTuple(args, "O!O!OOO", &PyType_Type, &d, &PyType_Type, &p, &one, &group, &raise)) return nullptr;
    for (PyObject* o : {d, p, one, group, raise}) Py_INCREF(o);        // for the life of the process
    desc_type = reinterpret_cast<PyTypeObject*>(d);
    plan_type = reinterpret_cast<PyTypeObject*>(p);
    slow_gemm = one;
    slow_grouped = group;
    check = raise;
    Py_RETURN_NONE;
}

// (address of codegemm_gemm, address of codegemm_gemm_grouped)
PyObject* use(PyObject*, PyObject* args)
{
    unsigned long long one, group;
    if (!PyArg_ParseTuple(args, "KK", &one, &group)) return nullptr;
    gemm_at = reinterpret_cast<gemm_t>(static_cast<uintptr_t>(one));
    grouped_at = reinterpret_cast<grouped_t>(static_cast<uintptr_t>(group));
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"codegemm_gemm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(gemm)), METH_FASTCALL | METH_KEYWORDS,
     "codegemm_gemm(desc, plan, x, packed_codes, codebooks, scales, y, workspace, workspace_bytes, stream=0)\n--\n\n"},
    {"codegemm_gemm_grouped", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(gemm_grouped)), METH_FASTCALL | METH_KEYWORDS,
     "codegemm_gemm_grouped(desc, plan, x, members, workspace, workspace_bytes, stream=0)\n--\n\n"
     "members: sequence of (out_features, packed_codes, codebooks, scales, y), tensors or raw device addresses."},
    {"codegemm_kv_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(kv_append)), METH_FASTCALL | METH_KEYWORDS,
     "codegemm_kv_append(cache, desc, cu_seqlens, q, k, v, q_norm, k_norm, rope, q_out, k_out, stream=0)\n--\n\n"},
    {"codegemm_kv_gather", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(kv_gather)), METH_FASTCALL | METH_KEYWORDS,
     "codegemm_kv_gather(cache, rows, cu_rows, first, k_out, v_out, stream=0)\n--\n\n"},
    {"codegemm_attn_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(attn_decode)), METH_FASTCALL | METH_KEYWORDS,
     "codegemm_attn_decode(cache, desc, q, out, workspace, workspace_bytes, stream=0)\n--\n\n"},
    {"codegemm_attn_prompt", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(attn_prompt)), METH_FASTCALL | METH_KEYWORDS,
     "codegemm_attn_prompt(desc, q, k, v, cu_q, cu_kv, out, workspace, workspace_bytes, stream=0)\n--\n\n"},
    {"prepare_attention", prepare_attention, METH_VARARGS, nullptr},
    {"use_attention", use_attention, METH_VARARGS, nullptr},
    {"prepare", prepare, METH_VARARGS, nullptr},
    {"use", use, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void)
{
    data_ptr = PyUnicode_InternFromString("data_ptr");
    return data_ptr ? PyModule_Create(&module) : nullptr;
}
