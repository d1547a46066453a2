#!/bin/bash
# Builds tests/sanitize/layers_validation.cpp against the library's sources with AddressSanitizer and
# UndefinedBehaviorSanitizer on the host code of the entry points on layers' weights (the device code is built plainly;
# the validation-only context it exercises launches no kernels).
#   tests/sanitize/build_layers.sh <output binary>
set -euo pipefail
HERE="$(cd "$(dirname "$0")" && pwd)"
ROOT="$(cd "$HERE/../.." && pwd)"
SRC="$ROOT/paper_2606_09377_amd/csrc"
OUT="$1"
HIPCC="${HIPCC:-/opt/rocm/bin/hipcc}"
SAN=(-Xarch_host -fsanitize=address -Xarch_host -fsanitize=undefined -Xarch_host -fno-sanitize-recover=all
     -Xarch_host -fno-omit-frame-pointer)
TMP="$(mktemp -d)"
trap 'rm -rf "$TMP"' EXIT
OBJS=()
for f in layers orthogonalize; do
  "$HIPCC" -O1 -g -std=c++17 -fPIC --offload-arch=gfx950 "${SAN[@]}" -I "$ROOT/include" -x hip -c "$SRC/$f.hip" -o "$TMP/$f.o" &
  OBJS+=("$TMP/$f.o")
done
for f in gemm elementwise conv alpha noalloc; do
  "$HIPCC" -O1 -std=c++17 -fPIC --offload-arch=gfx950 -I "$ROOT/include" -x hip -c "$SRC/$f.hip" -o "$TMP/$f.o" &
  OBJS+=("$TMP/$f.o")
done
for f in api graph; do
  "$HIPCC" -O1 -g -std=c++17 -fPIC "${SAN[@]}" -I "$ROOT/include" -c "$SRC/$f.cpp" -o "$TMP/$f.o" &
  OBJS+=("$TMP/$f.o")
done
"$HIPCC" -O1 -g -std=c++17 "${SAN[@]}" -I "$ROOT/include" -c "$HERE/layers_validation.cpp" -o "$TMP/driver.o" &
wait
"$HIPCC" "${SAN[@]}" --offload-arch=gfx950 "${OBJS[@]}" "$TMP/driver.o" -o "$OUT"
