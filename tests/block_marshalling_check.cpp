// marshalling_check.cpp's module, with the CPU as the current device of the operators around attention too.
#define VA_CURRENT_DEVICE() (-1)
#include "marshalling_check.cpp"

#undef PyInit_marshalling_check
PyMODINIT_FUNC PyInit_block_marshalling_check() { return PyInit_marshalling_check(); }
