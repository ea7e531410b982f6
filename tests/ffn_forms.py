"""Sizes of a feed-forward block whose products take, between them, every form that there is: tiles of 128 or 256, two places in LDS or four ("deep"),
each tile by one workgroup ("whole"), by several that share k ("shared"), or the last round's shared ("both"), for each of x w_in^T with the gate in its
epilogue, hidden w_out^T, grad w_out with the gate's gradient in it, d_pre w_in, d_pre^T x and grad^T hidden.  Tokens, width, hidden: the six forms."""

PRODUCTS = ("gated", "out", "gated gradient", "x", "w_in", "w_out")
FORMS = {
    (40, 520, 64): ("128 deep whole", "128 whole", "128 deep whole", "128 whole", "128 whole", "128 whole"),
    (1040, 64, 776): ("128 whole", "128 deep whole", "128 whole", "128 shared", "128 deep whole", "128 shared"),
    (40, 1288, 4104): ("128 shared", "128 shared", "128 shared", "128 deep shared", "256 whole", "128 whole"),
    (3000, 5128, 64): ("128 deep shared", "256 whole", "128 deep shared", "256 whole", "128 deep shared", "128 deep shared"),
    (3000, 64, 4104): ("256 whole", "128 shared", "256 whole", "128 deep shared", "128 deep shared", "128 shared"),
    (4100, 1032, 2056): ("256 both", "128 whole", "256 whole", "256 shared", "256 shared", "128 shared"),
    (2056, 4104, 2056): ("128 both", "256 whole", "256 shared", "128 both", "256 both", "256 whole"),
    (4100, 4104, 520): ("256 shared", "128 whole", "128 shared", "256 both", "256 shared", "128 shared"),
    (2056, 1288, 3080): ("256 whole", "128 deep whole", "128 whole", "128 deep whole", "128 both", "128 whole"),
    (4100, 1032, 4104): ("256 both", "256 shared", "128 both", "256 shared", "128 both", "256 shared"),
    (4100, 1544, 4104): ("256 both", "128 whole", "256 both", "256 shared", "256 whole", "128 whole"),
}
