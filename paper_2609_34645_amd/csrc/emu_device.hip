// The library's device code as one translation unit, so that libemu.so holds one code object.
#include "emu_exec.hip"
#include "emu_logits.hip"
