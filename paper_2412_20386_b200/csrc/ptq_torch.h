// What the sources of the extension module _ptq_torch share.
#pragma once

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#define PTQ_METHOD(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}

int ptq_add_block_methods(PyObject *module);      // the operators of include/ptq_block.h; 0 on success
int ptq_add_heads_methods(PyObject *module);      // those of include/ptq_heads.h
int ptq_add_fp8_methods(PyObject *module);        // those of include/ptq_fp8.h
