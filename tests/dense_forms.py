"""Sizes (b, w, d) by which the dense products' kernels are taken in forms that no other test reaches, for each operand type: rows at multiples of 16 bytes, of 4, and others."""

# (storage, b, d, widths): both activations
GATED = [("bf16", 1, 16390, (200,)), ("bf16", 17, 8200, (200, 201, 202)), ("bf16", 33, 3001, (200, 201, 202)), ("bf16", 65, 16390, (200, 202)), ("bf16", 200, 16390, (202,)),
         ("f32", 1, 16390, (100,)), ("f32", 17, 8200, (100,)), ("f32", 33, 6001, (100, 101)), ("f32", 65, 32701, (100, 101)), ("f32", 200, 32701, (100, 101))]
# (b, d, widths): both storage types and activations
GATED_I8 = [(17, 8200, (401, 404)), (33, 3001, (400, 401)), (65, 16390, (401,)), (200, 16390, (800, 804))]
PROJECT_I8 = [(33, 3001, (401,)), (65, 16390, (400, 401)), (500, 32701, (400, 404))]
# (storage, b, w, d, act)
BACKWARD = [("bf16", 65, 300, 32701, 1)]
