// The tile that a thread's packed attention launches are made to take, for measurement sweeps and
// tests: a seam between the library and its Python binding, no part of the C ABI. The
// binding reads HSA_PACKED_TILE=<rows>x<waves> while it holds the interpreter, as an assignment to
// os.environ does: read in the launch, with the interpreter free, it would race with that.
#pragma once

// rows 0: the launch's own choice
extern "C" __attribute__((visibility("default"))) void _hsa_packed_tile(int rows, int waves);
