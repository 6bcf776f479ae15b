// The order in which a converter warp of the product kernel waits for a stage, apart from the kernel so that a model of its
// barriers can be driven by it on the CPU.
//
// Two groups of warps convert the stages in turn; where the number of stages is odd, a group meets a stage's barriers only
// every second use, and a parity alone does not tell the use before last from the next one.  That the stage is free --
// the products of its last use are done -- says that its codes' last phase is over as well, so it comes first: the codes'
// barrier can then only be at the phase that is waited for.  (In the other order a copy that lands later than the one
// issued after it lets a group pass on the codes of two uses before.)  The barrier of the free stage itself is never two
// uses behind: the group's own last stage was free, and products are done in order.
#pragma once

namespace mip {

enum StageWait { kStageFree, kStageCodes };
constexpr StageWait kConverterFirst = kStageFree, kConverterSecond = kStageCodes;

}  // namespace mip
