// Which work a workgroup of the 8-bit and listed attention takes, for test_host_units_work.py; built by the host compiler.
#include "attn_units.h"

extern "C" void units_work_of(uint32_t x, uint32_t y, uint32_t z, uint32_t nx, uint32_t ny, uint32_t nz, int Hkv, int32_t* out) {
  const tempo::UnitsWork w = tempo::units_work(x, y, z, nx, ny, nz, Hkv);
  out[0] = w.hkv;
  out[1] = w.tile;
  out[2] = w.b;
  out[3] = w.split;
}
