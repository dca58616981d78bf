"""MI355X-native hot path of ConQuR's online rotation calibration.

`inputs`  — seeded synthetic activation streams (no method arithmetic).
`binding` — thin ctypes layer over the C-ABI library libconqur.so (HIP kernels).
`attention` — the layer around the calibrated heads: positions and norms of queries and keys, a paged cache of 16-, 8- or
              4-bit keys and values, attention of drafted tokens over it (same library, same manner).
"""
